"""Refusals of the operators over the paged cache: every check runs on the host before anything is launched, so none of
this needs a GPU.  The addresses are never followed."""
import ctypes as C
import inspect
import math

import pytest
import torch

from paper_2511_14450_b200 import hyperion as hyp

P = 0x10000                                                 # a well-aligned address


def shape(hq=8, hkv=2, d=128):
    return C.byref(hyp.hyp_attn_shape(hq, hkv, d))


BAD_SHAPES = [(8, 3, 128), (8, 2, 96), (0, 0, 128), (2, 4, 128), (48, 3, 128), (6, 2, 64)]


def mod_args(**kw):
    a = dict(shape=shape(), mod=C.byref(hyp.hyp_attn_mod(0.0, 0, None, None)), n=3, q=P, q_stride=1024, pool=P, table=P, pages=4, ctx=P,
             scratch=P, nbytes=1 << 30, out=P, stream=None)
    a.update(kw)
    return list(a.values())


def prefill_args(**kw):
    a = dict(shape=shape(), mod=C.byref(hyp.hyp_attn_mod(0.0, 0, None, None)), n=3, M=9, q=P, q_stride=1024, pool=P, table=P, pages=4, cu=P,
             ctx=P, out=P, stream=None)
    a.update(kw)
    return list(a.values())


def scored_args(**kw):
    a = dict(shape=shape(), n=3, q=P, q_stride=1024, pool=P, table=P, pages=4, ctx=P, decay=1.0, w_in=None, w_out=P, ws=64, scratch=P,
             nbytes=1 << 30, out=P, stream=None)
    a.update(kw)
    return list(a.values())


def evict_args(**kw):
    a = dict(shape=shape(), n=3, pool=P, table=P, pages=4, cached=P, w_in=P, ws=64, keep=32, sink=4, recent=8, dst=2 * P, dtable=2 * P,
             dpages=2, kept=P, new=2 * P, w_out=2 * P, wos=32, stream=None)
    a.update(kw)
    return list(a.values())


def shared_args(**kw):
    a = dict(shape=shape(), n=3, q=P, q_stride=1024, pool=P, groups=1, cu=P, ptable=P, ppages=4, plens=P, table=P, pages=4, ctx=P, scratch=P,
             nbytes=1 << 30, out=P, stream=None)
    a.update(kw)
    return list(a.values())


OPS = {"hyp_op_attn_decode_mod": mod_args, "hyp_op_attn_prefill_mod": prefill_args, "hyp_op_attn_decode_scored": scored_args,
       "hyp_op_kv_evict": evict_args, "hyp_op_attn_decode_shared": shared_args}


@pytest.mark.parametrize("name", OPS)
@pytest.mark.parametrize("bad", BAD_SHAPES)
def test_head_layouts_outside_the_documented_ones(name, bad):
    assert getattr(hyp.lib(), name)(*OPS[name](shape=shape(*bad))) == hyp.HYP_EINVAL
    assert getattr(hyp.lib(), name)(*OPS[name](shape=None)) == hyp.HYP_EINVAL


@pytest.mark.parametrize("name", OPS)
def test_null_pointers_and_counts(name):
    make = OPS[name]
    words = set(inspect.getsource(make).replace("(", " ").replace("=", " = ").split())
    keys = [k for k in ("q", "pool", "table", "ctx", "cu", "scratch", "out", "w_out", "cached", "kept", "new", "dst", "dtable", "ptable",
                        "plens", "mod") if k in words]
    assert len(keys) >= 6
    for k in keys:
        assert getattr(hyp.lib(), name)(*make(**{k: None})) == hyp.HYP_EINVAL, k
    for k, v in (("n", 0), ("n", -1), ("n", 70000 if name != "hyp_op_attn_prefill_mod" else 0), ("pages", 0), ("pages", (1 << 26) + 1)):
        assert getattr(hyp.lib(), name)(*make(**{k: v})) == hyp.HYP_EINVAL, (k, v)


@pytest.mark.parametrize("name", [n for n in OPS if n != "hyp_op_kv_evict"])
def test_query_layout(name):
    for kw in (dict(q_stride=1023), dict(q_stride=1016), dict(q_stride=1028), dict(q=P + 8), dict(out=P + 8), dict(pool=P + 8)):
        assert getattr(hyp.lib(), name)(*OPS[name](**kw)) == hyp.HYP_EINVAL, kw


def test_modifications():
    for cap, window in ((-1.0, 0), (math.nan, 0), (math.inf, 0), (0.0, -1), (2.0 ** -11, 0), (2.0 ** 20 * 1.01, 0)):
        m = C.byref(hyp.hyp_attn_mod(cap, window, None, None))
        assert hyp.lib().hyp_op_attn_decode_mod(*mod_args(mod=m)) == hyp.HYP_EINVAL
        assert hyp.lib().hyp_op_attn_prefill_mod(*prefill_args(mod=m)) == hyp.HYP_EINVAL


def test_sizes_of_the_scored_and_evicting_calls():
    L = hyp.lib()
    for kw in (dict(decay=math.nan), dict(decay=math.inf), dict(ws=63), dict(scratch=P + 4)):
        assert L.hyp_op_attn_decode_scored(*scored_args(**kw)) == hyp.HYP_EINVAL, kw
    for kw in (dict(keep=0), dict(sink=-1), dict(recent=-1), dict(sink=30, recent=3), dict(sink=33), dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1),
               dict(dpages=1), dict(wos=31), dict(ws=63), dict(new=P), dict(dst=P, dtable=P), dict(w_out=P)):
        assert L.hyp_op_kv_evict(*evict_args(**kw)) == hyp.HYP_EINVAL, kw
    for kw in (dict(groups=0), dict(groups=70000), dict(ppages=0)):
        assert L.hyp_op_attn_decode_shared(*shared_args(**kw)) == hyp.HYP_EINVAL, kw


def test_small_scratch():
    L = hyp.lib()
    sh = (8, 2, 128)
    need = hyp.hyp_op_attn_mod_scratch_bytes(sh, 3, 4)
    assert need > 0 and L.hyp_op_attn_decode_mod(*mod_args(nbytes=need - 1)) == hyp.HYP_ECAPACITY
    need = hyp.hyp_op_attn_scored_scratch_bytes(sh, 3, 4)
    assert need > 0 and L.hyp_op_attn_decode_scored(*scored_args(nbytes=need - 1)) == hyp.HYP_ECAPACITY
    need = hyp.hyp_op_attn_shared_scratch_bytes(sh, 3, 1, 4, 4)
    assert need > 0 and L.hyp_op_attn_decode_shared(*shared_args(nbytes=need - 1)) == hyp.HYP_ECAPACITY
    assert hyp.hyp_op_attn_mod_scratch_bytes((8, 3, 128), 3, 4) == 0
    assert hyp.hyp_op_attn_scored_scratch_bytes(sh, 0, 4) == 0
    assert hyp.hyp_op_attn_shared_scratch_bytes(sh, 3, 1, 0, 4) == 0


def test_the_binding_refuses_what_does_not_fit():
    f16, i32 = torch.float16, torch.int32
    q, out, pool = torch.zeros(2, 256, dtype=f16), torch.zeros(2, 256, dtype=f16), torch.zeros(3, 2, 2, 16, 64, dtype=f16)
    table, ctx = torch.zeros(2, 1, dtype=i32), torch.zeros(2, dtype=i32)
    scratch, w = torch.zeros(64), torch.zeros(2, 2, 16)
    with pytest.raises(hyp.HyperionError) as e:                                  # tensors of the host
        hyp.hyp_op_attn_decode_mod((4, 2, 64), hyp.AttnMod(), q, pool, table, ctx, scratch, out)
    assert e.value.code == hyp.HYP_EINVAL
    with pytest.raises(hyp.HyperionError):
        hyp.hyp_op_attn_decode_scored((4, 2, 64), q, pool, table, ctx, 1.0, None, w, scratch, out)
    with pytest.raises(hyp.HyperionError):
        hyp.hyp_op_attn_decode_shared((4, 2, 64), q, pool, table[0], table, ctx, table, ctx, scratch, out)
    with pytest.raises(hyp.HyperionError):
        hyp.hyp_op_attn_prefill_mod((4, 2, 64), hyp.AttnMod(), q, pool, table, ctx, ctx, out)
    with pytest.raises(hyp.HyperionError):
        hyp.hyp_op_kv_evict((4, 2, 64), pool, table, ctx, w, 8, 1, 1, pool, table, table, ctx, w)


@pytest.mark.parametrize("heads", [(1, 1, 64), (1, 1, 128), (3, 3, 64), (25, 25, 64), (5, 5, 128), (40, 10, 128), (8, 1, 64)])
def test_the_scores_in_the_scratch_start_on_a_16_byte_boundary(heads):
    """Scores [n_seqs * n_q_heads][16 * pages] lie at the end of the scratch and are read four at a time, so their start, the whole
    less their size, has to be a multiple of 16 bytes (partial rows are head_dim + 2 floats, and may be odd in number)."""
    odd = 0
    for n in (1, 2, 3, 5, 7, 64):
        for pages in (1, 4, 16, 17, 19, 20, 28, 33, 64, 100, 513, 2048):
            total = hyp.hyp_op_attn_scored_scratch_bytes(heads, n, pages)
            scores = 4 * n * heads[0] * 16 * pages
            assert total > scores and (total - scores) % 16 == 0, (n, pages, total - scores)
            parts = hyp.hyp_op_attn_mod_scratch_bytes(heads, n, pages)          # the same partial rows
            assert parts <= total - scores < parts + 16, (n, pages)
            odd += parts % 16 != 0
    assert odd > 0 or heads[0] % 2 == 0, "the sizes were to hold odd numbers of rows"


def test_a_tensor_without_dimensions_is_refused_like_any_other_that_does_not_fit():
    scalar = torch.tensor(3, dtype=torch.int32)
    with pytest.raises(hyp.HyperionError) as e:
        hyp._rows("hyp_op_attn_prefill_mod", "ctx_lens", scalar, torch.int32, scalar.get_device(), ())
    assert e.value.code == hyp.HYP_EINVAL and "ctx_lens" in str(e.value)
    assert hyp._rows("hyp_op_attn_prefill_mod", "ctx_lens", scalar[None], torch.int32, scalar.get_device(), ())[1] == 1


def test_a_modification_follows_its_tensors():
    """Slopes or prefixes that are taken out of a modification after it was made are not used any more (their memory may be gone)."""
    hyp._shape((4, 2, 64))
    slopes, prefix = torch.ones(4), torch.zeros(2, dtype=torch.int32)
    mod = hyp.AttnMod(slopes=slopes, prefix_lens=prefix)
    mod.check("hyp_op_attn_decode_mod", (4, 2, 64), 2, -1)
    assert mod.struct.slopes == slopes.data_ptr() and mod.struct.prefix_lens == prefix.data_ptr()
    mod.slopes = mod.prefix_lens = None
    mod.check("hyp_op_attn_decode_mod", (4, 2, 64), 2, -1)
    assert mod.struct.slopes is None and mod.struct.prefix_lens is None
    mod.slopes = torch.ones(5)
    with pytest.raises(hyp.HyperionError):
        mod.check("hyp_op_attn_decode_mod", (4, 2, 64), 2, -1)


def test_the_size_calls_refuse_the_counts_that_the_calls_refuse():
    sh = (8, 2, 128)
    for n in (65536, 2 ** 31 - 1, 0, -1):
        assert hyp.hyp_op_attn_mod_scratch_bytes(sh, n, 4) == 0
        assert hyp.hyp_op_attn_scored_scratch_bytes(sh, n, 4) == 0
        assert hyp.hyp_op_attn_shared_scratch_bytes(sh, n, 1, 4, 4) == 0
        assert hyp.hyp_op_attn_shared_scratch_bytes(sh, 3, n, 4, 4) == 0
    assert hyp.hyp_op_attn_shared_scratch_bytes(sh, 65535, 65535, 4, 4) > 0
