"""Operators in few bits at the edges of what they are documented for, against definitions in 64 bits.  Tolerances: those derived in
test_gpu_low_bit.py, or given beside the test."""
import math

import pytest
import torch

from paper_2511_14450_b200 import hyperion as hyp
from tests import test_gpu_low_bit as low

pytestmark = pytest.mark.gpu

FORMATS = low.FORMATS
i32, normal, ok = low.i32, low.normal, low.ok


def cache8(x, fmt, extra=0):
    """Pool, table and the held values (fp64) of one sequence of rows x [tokens, 2, n_kv_heads, D]; a page that nobody owns lies in front,
    slots behind the end hold NaN."""
    l, _, hkv, d = x.shape
    pages = (l + 15) // 16
    codes, scales = low.quantized8(x.double(), fmt)
    held = low.numbers(codes, fmt) * scales.double()[..., None]
    c = torch.full((pages * 16, 2, hkv, d), 0xFF, dtype=torch.uint8, device="cuda")
    s = torch.full((pages * 16, 2, hkv), math.nan, device="cuda")
    c[:l], s[:l] = codes, scales
    c, s = c.view(pages, 16, 2, hkv, d).permute(0, 2, 3, 1, 4), s.view(pages, 16, 2, hkv).permute(0, 2, 3, 1)
    pool = torch.full((pages + 1, 2, hkv, 16 * d + 64), 0xFF, dtype=torch.uint8, device="cuda")
    pool[1:] = low.half_page(c.contiguous(), s.contiguous(), d)
    table = torch.cat([torch.arange(1, pages + 1, device="cuda"), torch.zeros(extra, device="cuda")]).to(torch.int32).view(1, -1)
    return pool, table, held


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", [1e28, 1e31, 2.0 ** 100, 1e35])
@pytest.mark.parametrize("heads,l,extra", [((4, 2, 64), 1, 0), ((8, 1, 128), 17, 0), ((8, 2, 128), 700, 0), ((4, 1, 64), 5000, 0), ((2, 2, 64), 40, 300),
                                           ((2, 2, 64), 9000, 0)])
def test_attention_over_very_negative_scores(fmt, size, heads, l, extra):
    """Keys whose scores lie far below what fp16 keys could give, all of them alike: the result is the values' mean, whatever the scales of the
    values (up to 2^6 apart both ways).  One launch, a cluster's join and a join of its own."""
    hq, hkv, d = heads
    x = normal(l, 2, hkv, d, seed=l)
    x[:, 0] = -(normal(1, hkv, d, seed=1).abs() + 0.5) * size
    x[:, 1] *= torch.exp2(torch.randint(-6, 7, (l, hkv, 1), generator=low.gen(2), device="cuda").float())
    pool, table, held = cache8(x, fmt, extra)
    q = (normal(1, hq * d, seed=3).abs() + 0.1).half() / 64
    out = low.attend(heads, fmt, q, pool, table, i32([l - 1]))[0].double().view(hq, d)
    v = held[:, 1].repeat_interleave(hq // hkv, 1)
    want, mean = v.mean(0), v.abs().mean(0)
    # equal weights: half a step of each and of the result; weights below fp16's normal range as in test_gpu_low_bit.attention
    bound = 2.0 ** -11 * (want.abs() + mean) * 1.01 + 2.0 ** -18 * mean + 2.0 ** -25 * 4 * v.abs().amax((0, 2)).view(hq, 1) + 2.0 ** -25
    assert (out.abs().amax() > 0) and ((out - want).abs() <= bound).all(), float(((out - want).abs() / bound).max())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("l,at", [(3, 1), (300, 299), (4000, 1777)])
def test_attention_largest_of_very_negative_scores(fmt, l, at):
    """Scores of -1e33 but for one of about -1e29: that key has all of the weight, also where its value is small beside the others'."""
    heads = (8, 2, 128)
    hq, hkv, d = heads
    x = normal(l, 2, hkv, d, seed=l)
    x[:, 0] = -(normal(1, hkv, d, seed=1).abs() + 0.5) * 1e33
    x[at, 0] *= 1e-4
    x[at, 1] *= 2.0 ** -9
    pool, table, held = cache8(x, fmt)
    q = (normal(1, hq * d, seed=3).abs() + 0.1).half()
    out = low.attend(heads, fmt, q, pool, table, i32([l - 1]))[0].double().view(hq, d)
    want = held[at, 1].repeat_interleave(hq // hkv, 0)
    assert ((out - want).abs() <= 2.0 ** -10 * 1.01 * want.abs() + 2.0 ** -25).all()


@pytest.mark.parametrize("fmt,key", [(hyp.HYP_KV8_INT8, -144.0), (hyp.HYP_KV8_E4M3, -144.0), (hyp.HYP_KV8_INT8, -136.0)])
def test_attention_many_small_weights_beside_a_large_one(fmt, key):
    """40000 keys a warp with weights of e^-18 (or e^-17) beside one of 1: just below (or above) 2^-25 of the largest.  Their values sit in a
    dimension of their own, so that what they lose is seen.  No term of the bound grows with the length."""
    heads, n, pages = (8, 8, 64), 300, 10000
    x = torch.zeros(32, 2, 8, 64, device="cuda")
    x[:, 0, :, 0], x[:, 1, :, 1] = key, 1.0
    x[0, 0], x[0, 1] = 0.0, 0.0
    x[0, 1, :, 0] = 1.0
    pool, two, held = cache8(x, fmt)                                     # a page with the large key in front, one without
    table = two[:, 1:].expand(n, pages).contiguous()
    table[:, 0:8:2] = two[0, 0]                                          # one of each warp's
    q = torch.zeros(n, 8, 64, device="cuda", dtype=torch.float16)
    q[:, :, 0] = 1.0
    out = low.attend(heads, fmt, q.view(n, -1), pool, table, i32([16 * pages - 1] * n)).double().view(n, 8, 64)
    small = math.exp(float(held[1, 0, 0, 0]) / 8) * (16 * pages - 4)
    want = torch.zeros(64, dtype=torch.float64, device="cuda")
    want[0], want[1] = 4 / (4 + small), small / (4 + small)
    assert float(want[1]) > 2.0 ** -11
    assert ((out - want).abs() <= 2.0 ** -10 * 1.01 * want + 2.0 ** -15).all(), float((out - want).abs().max())


def in_a_new_thread(call):
    """Runs `call` as a new thread's first work with CUDA; its exception, if it raised one."""
    import threading
    raised = []

    def body():
        try:
            call()
        except Exception as e:  # noqa: BLE001 - handed to the test
            raised.append(e)
    torch.cuda.synchronize()
    t = threading.Thread(target=body)
    t.start()
    t.join()
    return raised[0] if raised else None


@pytest.mark.parametrize("m", [1, 8, 300])
def test_product_as_first_work_of_a_thread(m):
    n, k = 700, 5120
    codes, scales = low.weights(n, k, seed=1)
    packed = hyp.hyp_op_mx4_pack(codes, scales)
    a, out = normal(m, k, seed=2).half(), torch.zeros(m, n, device="cuda")
    scratch = torch.empty(hyp.hyp_op_gemm_mx4_scratch_bytes(m, k, 3), dtype=torch.uint8, device="cuda")
    assert in_a_new_thread(lambda: hyp.hyp_op_gemm_mx4(a, packed, n, 3, hyp.HYP_EPI_STORE_F32, out, scratch)) is None
    ok()
    held, w = low.in_terms(a, 3), low.values(codes, scales, k)
    assert ((out.double() - held @ w.T).abs() <= low.product_bound(held, w, k)).all()


@pytest.mark.parametrize("f16", [False, True])
def test_16_bit_product_as_first_work_of_a_thread(f16):
    """The operators in 16 bits describe their operands in the same way."""
    m, n, k = 300, 256, 512
    w = normal(n, k, seed=1, std=0.05).bfloat16()
    a = normal(m, k, seed=2).to(torch.float16 if f16 else torch.bfloat16)
    packed = hyp.hyp_op_pack_weight(w, n, False, f16=f16)
    out = torch.zeros(m, n, device="cuda")
    fn = hyp.hyp_op_gemm_f16 if f16 else hyp.hyp_op_gemm
    stream = torch.cuda.current_stream()
    assert in_a_new_thread(lambda: fn(a, packed, n, hyp.HYP_EPI_STORE_F32, out, stream)) is None
    ok()
    want = a.double() @ w.double().T
    assert ((out.double() - want).abs() <= k * 2.0 ** -23 * (a.double().abs() @ w.double().abs().T)).all()


# Eight threads whose first products, on streams and buffers of their own, start together in a fresh process.
FIRST_CALLS = """
import threading
import torch
from paper_2511_14450_b200 import hyperion as hyp
from tests import test_gpu_low_bit as low
n, k, m = 700, 5120, 8
pool = torch.zeros(1, 2, 1, 1088, device="cuda", dtype=torch.uint8)
low.attend((2, 1, 64), 0, torch.zeros(1, 128, device="cuda").half(), pool, low.i32([[0]]), low.i32([0]))
packed = hyp.hyp_op_mx4_pack(*low.weights(n, k, 1))
a = low.normal(m, k, seed=2).half()
outs = [torch.zeros(m, n, device="cuda") for _ in range(8)]
scratch = [torch.empty(hyp.hyp_op_gemm_mx4_scratch_bytes(m, k, 3), dtype=torch.uint8, device="cuda") for _ in range(8)]
streams = [torch.cuda.Stream() for _ in range(8)]
torch.cuda.synchronize()
gate = threading.Barrier(8)
def call(i):
    gate.wait()
    hyp.hyp_op_gemm_mx4(a, packed, n, 3, hyp.HYP_EPI_STORE_F32, outs[i], scratch[i], streams[i])
threads = [threading.Thread(target=call, args=(i,)) for i in range(8)]
for t in threads: t.start()
for t in threads: t.join()
low.ok()
assert outs[0].abs().max() > 0
print("alike", sum(torch.equal(outs[0], o) for o in outs))
"""


def test_product_first_calls_of_many_threads():
    """All threads cut K alike: their sums are the same to the bit."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == ["alike", "8"]


def behind_queued_work(pack, raw):
    """`pack` on a stream of its own, while the current stream still has to write a freed block of the size that the copy needs."""
    want = pack(None).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)                                       # about 0.1 s
    block = torch.empty_like(want)
    block.fill_(0xAA)
    del block
    got = pack(side.cuda_stream if raw else side)
    torch.cuda.synchronize()
    return got, want


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("swiglu", [False, True])
def test_pack_of_4_bit_weights_on_another_stream(swiglu, raw):
    codes, scales = low.weights(1400, 4096, seed=1)
    got, want = behind_queued_work(lambda s: hyp.hyp_op_mx4_pack(codes, scales, swiglu, stream=s), raw)
    assert torch.equal(got, want)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("f16", [False, True])
def test_pack_of_16_bit_weights_on_another_stream(f16, raw):
    w = normal(1400, 1024, seed=1).bfloat16()
    got, want = behind_queued_work(lambda s: hyp.hyp_op_pack_weight(w, 1400, False, stream=s, f16=f16), raw)
    assert torch.equal(got, want)


def test_pack_on_the_default_stream_by_its_address():
    codes, scales = low.weights(200, 512, seed=1)
    assert torch.equal(hyp.hyp_op_mx4_pack(codes, scales, stream=0), hyp.hyp_op_mx4_pack(codes, scales))


def fp32_nearest(x):
    """The fp32 number nearest to a fraction, ties to even."""
    from fractions import Fraction
    import numpy as np
    f = np.float32(float(x))
    near = [np.nextafter(f, np.float32(-np.inf)), f, np.nextafter(f, np.float32(np.inf))]
    return float(min(near, key=lambda v: (abs(Fraction(float(v)) - x), int(v.view(np.uint32)) & 1)))


def test_write_scales_of_rotated_rows_next_to_a_border():
    """Largest magnitudes of 127 M +- 2^-22 and 127 M, M an odd number of 25 bits: a 127th of them lies half a step of fp64, or nothing, away
    from the middle between two fp32 numbers."""
    from fractions import Fraction
    heads, n, d = (1, 1, 64), 300, 64
    ks = [3355445 + 2 * 43 * i for i in range(n)]
    tab = torch.zeros(n, d // 2, 2, device="cuda")
    tab[:, 0, 0], tab[:, 0, 1] = torch.tensor(ks, device="cuda").float(), -2.0 ** -22
    qkv = torch.zeros(3 * n, 3 * d, device="cuda")
    qkv[:, d] = 635.0                                                    # 635 k - b sin
    for i, b in enumerate((1.0, 0.0, -1.0)):
        qkv[i * n:(i + 1) * n, d + d // 2] = b
    pages = (n + 15) // 16
    table = torch.arange(3 * pages, dtype=torch.int32, device="cuda").view(3, pages)
    pool = torch.zeros(3 * pages, 2, 1, 16 * d + 64, dtype=torch.uint8, device="cuda")
    hyp.hyp_op_kv8_write(heads, hyp.HYP_KV8_INT8, qkv, pool, table, i32([0, n, 2 * n, 3 * n]), i32([0, 0, 0]), tab)
    ok()
    got = pool[:, 0, 0, 16 * d:].contiguous().view(torch.float32).view(3, -1)[:, :n].cpu()
    want = torch.tensor([[fp32_nearest((Fraction(635 * k) + b * Fraction(1, 1 << 22)) / 127) for k in ks] for b in (1, 0, -1)])
    assert torch.equal(got, want), int((got != want).sum())
    codes = pool[:, 0, 0, :16 * d].reshape(3, -1, d)[:, :n]
    assert (codes[:, :, 0] == 255).all() and (codes[:, :, 1:32] == 128).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("l,at", [(40, 39), (5000, 3)])
@pytest.mark.parametrize("part", [0, 1])
def test_attention_nan_row_of_no_weight(fmt, l, at, part):
    """A key or value row with a NaN scale makes its sequence's results NaN, a value row whose weight is nothing beside the others' as well."""
    heads = (4, 2, 64)
    x = normal(l, 2, 2, 64, seed=l)
    x[:, 0] = 0.0
    x[at, 0] = -3000.0                                                   # e^-24000 of the others' weight
    pool, table, held = cache8(x, fmt)
    q = torch.ones(1, 256, device="cuda", dtype=torch.float16)
    out = low.attend(heads, fmt, q, pool, table, i32([l - 1]))[0].double().view(4, 64)
    keep = torch.arange(l, device="cuda") != at
    want = held[keep, 1].mean(0).repeat_interleave(2, 0)
    assert ((out - want).abs() <= 2.0 ** -10 * held[:, 1].abs().amax()).all()
    pool[int(table[0, at // 16]), part, 1, 16 * 64 + 4 * (at % 16):16 * 64 + 4 * (at % 16) + 4] = 0xFF
    again = low.attend(heads, fmt, q, pool, table, i32([l - 1]))[0].double().view(4, 64)
    assert torch.isnan(again[2:]).all() and torch.equal(again[:2], out[:2])


@pytest.mark.parametrize("heads,lens,extra", [((40, 10, 128), [1024] * 8, 0), ((8, 2, 128), [2500, 3, 700], 0), ((8, 8, 128), [300] * 40, 200)])
def test_attention_is_the_same_on_every_run(heads, lens, extra):
    hq, hkv, d = heads
    c = low.Cache8(lens, hkv, d, hyp.HYP_KV8_INT8, 71, extra)
    q, ctx = normal(len(lens), hq * d, seed=72).half(), i32([l - 1 for l in lens])
    first = low.attend(heads, hyp.HYP_KV8_INT8, q, c.pool, c.table, ctx)
    for _ in range(5):
        assert torch.equal(low.attend(heads, hyp.HYP_KV8_INT8, q, c.pool, c.table, ctx), first)
