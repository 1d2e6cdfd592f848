"""Refusals of the operators in few bits (4-bit weights, 8-bit cache): every check runs on the host before anything is launched, so none
of this needs a GPU.  The addresses are never followed."""
import ctypes as C
import inspect

import pytest
import torch

from paper_2511_14450_b200 import hyperion as hyp

P = 0x10000                                                 # a well-aligned address


def shape(hq=8, hkv=2, d=128):
    return C.byref(hyp.hyp_attn_shape(hq, hkv, d))


def quantize_args(**kw):
    return list((dict(x=P, type=0, N=5, K=64, stride=64, codes=P, scales=P, stream=None) | kw).values())


def dequantize_args(**kw):
    return list((dict(codes=P, scales=P, N=5, K=64, type=0, out=P, stride=64, stream=None) | kw).values())


def pack_args(**kw):
    return list((dict(codes=P, scales=P, N=5, K=64, swiglu=0, packed=P, nbytes=1 << 30, stream=None) | kw).values())


def gemm_args(**kw):
    return list((dict(a=P, type=1, a_stride=64, packed=P, M=3, N=5, K=64, terms=3, epi=3, out=P, ldo=8, scratch=P, nbytes=1 << 30,
                      stream=None) | kw).values())


def write_args(**kw):
    return list((dict(shape=shape(), fmt=0, n=3, M=7, qkv=P, type=0, stride=1536, rope=P, positions=100, pool=P, table=P, pages=4, cu=P, ctx=P,
                      q_out=P, stream=None) | kw).values())


def read_args(**kw):
    return list((dict(shape=shape(), fmt=1, n=3, pool=P, table=P, pages=4, first=P, lens=P, dst=2 * P, dtable=P, dpages=4, stream=None) | kw).values())


def attend_args(**kw):
    return list((dict(shape=shape(), fmt=0, n=3, q=P, q_stride=1024, pool=P, table=P, pages=4, ctx=P, scratch=P, nbytes=1 << 30, out=P,
                      stream=None) | kw).values())


OPS = {"hyp_op_mx4_quantize": quantize_args, "hyp_op_mx4_dequantize": dequantize_args, "hyp_op_mx4_pack": pack_args,
       "hyp_op_gemm_mx4": gemm_args, "hyp_op_kv8_write": write_args, "hyp_op_kv8_read": read_args, "hyp_op_attn_decode_kv8": attend_args}
MAY_BE_NULL = {"rope", "q_out", "first", "stream"}
E, CAP = hyp.HYP_EINVAL, hyp.HYP_ECAPACITY


def call(name, **kw):
    return getattr(hyp.lib(), name)(*OPS[name](**kw))


@pytest.mark.parametrize("name", OPS)
def test_null_and_misaligned_pointers(name):
    source = inspect.getsource(OPS[name])
    keys = [k for k in ("x", "codes", "scales", "out", "packed", "a", "scratch", "qkv", "pool", "table", "cu", "ctx", "lens", "dst", "dtable", "q")
            if f" {k}=" in source or f"({k}=" in source]
    assert len(keys) >= 3
    for k in keys:
        assert call(name, **{k: None}) == E, k
    for k, by in (("x", 8), ("a", 8), ("packed", 64), ("scratch", 8), ("qkv", 8), ("pool", 8), ("dst", 8), ("q", 8), ("q_out", 8), ("rope", 8)):
        if f" {k}=" in source or f"({k}=" in source:
            assert call(name, **{k: P + by}) == E, k


@pytest.mark.parametrize("name", ["hyp_op_kv8_write", "hyp_op_kv8_read", "hyp_op_attn_decode_kv8"])
def test_cache_shapes_formats_and_counts(name):
    for bad in [(8, 3, 128), (8, 2, 96), (0, 0, 128), (2, 4, 128), (48, 3, 128), (6, 2, 64), (40000, 40000, 64)]:
        assert call(name, shape=shape(*bad)) == E, bad
    assert call(name, shape=None) == E
    for k, v in (("fmt", 2), ("fmt", -1), ("n", 0), ("n", -1), ("n", 65536), ("pages", 0), ("pages", (1 << 26) + 1)):
        assert call(name, **{k: v}) == E, (k, v)


def test_cache_sizes_of_one_operator():
    for kw in (dict(M=0), dict(M=(1 << 26) + 1), dict(type=3), dict(type=-1), dict(stride=1535), dict(stride=1528), dict(stride=1540),
               dict(positions=0), dict(positions=-1)):
        assert call("hyp_op_kv8_write", **kw) == E, kw
    for kw in (dict(dpages=0), dict(dpages=(1 << 26) + 1)):
        assert call("hyp_op_kv8_read", **kw) == E, kw
    for kw in (dict(q_stride=1023), dict(q_stride=1016), dict(q_stride=1028), dict(out=P + 8)):
        assert call("hyp_op_attn_decode_kv8", **kw) == E, kw
    need = hyp.hyp_op_attn_kv8_scratch_bytes((8, 2, 128), 3, 400)
    assert need > 0
    assert call("hyp_op_attn_decode_kv8", pages=400, nbytes=need - 1) == CAP
    assert hyp.hyp_op_attn_kv8_scratch_bytes((8, 2, 128), 70000, 4) == 0
    assert hyp.hyp_op_attn_kv8_scratch_bytes((8, 2, 96), 3, 4) == 0


@pytest.mark.parametrize("name", ["hyp_op_mx4_quantize", "hyp_op_mx4_dequantize", "hyp_op_mx4_pack", "hyp_op_gemm_mx4"])
def test_matrix_sizes(name):
    for kw in (dict(N=0), dict(N=-3), dict(K=0), dict(K=4), dict(K=60), dict(K=(1 << 25) + 8), dict(K=-8)):
        assert call(name, **kw) == E, kw


@pytest.mark.parametrize("name", ["hyp_op_mx4_quantize", "hyp_op_mx4_dequantize", "hyp_op_mx4_pack", "hyp_op_gemm_mx4"])
def test_rows_that_whole_ctas_cannot_count(name):
    assert call(name, N=2 ** 31 - 7, K=8, ldo=2 ** 31 - 1) == E if name == "hyp_op_gemm_mx4" else call(name, N=2 ** 31 - 7, K=8) == E


def test_binding_refuses_sizes_beyond_31_bits():
    class Wide:                                             # what the binding asks of a tensor, without its memory
        dtype, shape, device = torch.float16, (2 ** 32 + 5, 8), "cuda:0"
        get_device, stride, data_ptr = (lambda self: 0), (lambda self: (8, 1)), (lambda self: P)
    refused(hyp._matrix, "here", "x", Wide())
    Wide.shape = (2, 2 ** 31)
    Wide.stride = lambda self: (2 ** 31, 1)
    refused(hyp._matrix, "here", "x", Wide())


def test_matrix_types_and_strides():
    for name in ("hyp_op_mx4_quantize", "hyp_op_mx4_dequantize"):
        for kw in (dict(type=3), dict(type=-1), dict(stride=63), dict(stride=66), dict(type=1, stride=68), dict(type=2, stride=60)):
            assert call(name, **kw) == E, (name, kw)
    for kw in (dict(type=0), dict(type=3), dict(a_stride=56), dict(a_stride=68), dict(M=0), dict(M=(1 << 26) + 1), dict(terms=0), dict(terms=4),
               dict(epi=-1), dict(epi=4), dict(ldo=4), dict(out=P + 2)):
        assert call("hyp_op_gemm_mx4", **kw) == E, kw
    assert call("hyp_op_gemm_mx4", epi=0, out=P + 1) == E
    need = hyp.hyp_op_gemm_mx4_scratch_bytes(3, 64, 3)
    assert need > 0 and call("hyp_op_gemm_mx4", nbytes=need - 1) == CAP
    need = hyp.hyp_op_mx4_packed_bytes(5, 64, False)
    assert need == 128 * 64 + 512 and call("hyp_op_mx4_pack", nbytes=need - 1) == CAP
    assert hyp.hyp_op_mx4_packed_bytes(129, 136, True) == 2 * 2 * 2 * need
    assert call("hyp_op_gemm_mx4", N=1 << 30, K=1 << 20, ldo=1 << 30) != hyp.HYP_OK
    for n, k in ((0, 64), (5, 60), (1 << 30, 1 << 20), (2 ** 31 - 1, 64), (2 ** 31 - 1, 1 << 26), (128, 2 ** 31 - 8)):
        assert hyp.hyp_op_mx4_packed_bytes(n, k, False) == 0
    for m, k, t in ((0, 64, 1), (3, 60, 1), (3, 64, 0), (3, 64, 4), ((1 << 26) + 1, 64, 1)):
        assert hyp.hyp_op_gemm_mx4_scratch_bytes(m, k, t) == 0


def test_scratch_grows_with_rows_and_terms():
    """A buffer made for the largest batch serves the smaller ones."""
    for k in (64, 5120):
        for terms in (1, 2, 3):
            sizes = [hyp.hyp_op_gemm_mx4_scratch_bytes(m, k, terms) for m in range(1, 700)]
            assert sizes == sorted(sizes)
            assert sizes[-1] >= 699 * terms * k


def refused(fn, *args, **kw):
    with pytest.raises(hyp.HyperionError) as e:
        fn(*args, **kw)
    assert e.value.code == hyp.HYP_EINVAL


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x, u8 = torch.zeros(4, 64), torch.zeros(4, 32, dtype=torch.uint8)
    refused(hyp.hyp_op_mx4_quantize, x, u8, torch.zeros(4, 2, dtype=torch.uint8))
    refused(hyp.hyp_op_mx4_quantize, x.double(), u8, u8)
    refused(hyp.hyp_op_mx4_quantize, torch.zeros(()), u8, u8)
    refused(hyp.hyp_op_mx4_dequantize, u8, u8, x)
    refused(hyp.hyp_op_mx4_pack, u8, u8)
    refused(hyp.hyp_op_gemm_mx4, x.half(), u8, 4, 1, hyp.HYP_EPI_STORE_F32, x, u8)
    i32, pool = torch.zeros(2, dtype=torch.int32), torch.zeros(3, 2, 2, 1088, dtype=torch.uint8)
    refused(hyp.hyp_op_kv8_write, (4, 2, 64), 0, torch.zeros(2, 512), pool, i32.view(2, 1), i32, i32)
    refused(hyp.hyp_op_kv8_read, (4, 2, 64), 0, pool, i32.view(2, 1), None, i32, pool, i32.view(2, 1))
    refused(hyp.hyp_op_attn_decode_kv8, (4, 2, 64), 0, torch.zeros(2, 256).half(), pool, i32.view(2, 1), i32, u8, torch.zeros(2, 256).half())
