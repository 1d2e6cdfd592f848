"""Operators in few bits against their definitions in 64 bits: microscaled 4-bit matrices and their product, the 8-bit paged cache and
the attention over it.

Tolerances.  Codes, scales and what is read back are exact.  Product: a sum of K fp32 products in any order, every step rounded or
cut off, is off by at most K 2^-23 sum |a w|; a 16-bit result adds half a step (2^-11 or 2^-8 of it); SiLU(g) u has a slope of at
most 1.1 |u| in g and |SiLU(g)| in u, and its own functions are off by 2^-20 of the value.  Attention: as for the fp16 cache: half a
step of the result, half a step (2^-11) of every weight times its value, or 2^-25 of the largest weight times scale a key where a weight is below
fp16's normal range, and 2 e sum p |v| for an error e of the scores (2^-20 of the largest sum |q k| / sqrt(D), and 2^-20 * 8 for the
functions)."""
import math

import numpy as np
import pytest
import torch

from paper_2511_14450_b200 import hyperion as hyp

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 64), (40, 10, 128), (8, 8, 128), (8, 1, 64), (8, 1, 128), (3, 3, 64)]
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
FORMATS = [hyp.HYP_KV8_INT8, hyp.HYP_KV8_E4M3]
FP4 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
E4M3 = torch.tensor([i * 2.0 ** -9 for i in range(8)] + [(8 + i) * 2.0 ** (e - 3) for e in range(-6, 9) for i in range(8) if (e, i) != (8, 7)],
                    dtype=torch.float64)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(*shape, seed=0, std=1.0):
    return torch.randn(*shape, generator=gen(seed), device="cuda") * std


def nearest(y, grid):
    """Places in the ascending grid of the members nearest to |y| (fp64), ties to even places."""
    grid = grid.to(y.device)
    a = y.abs().clamp(max=float(grid[-1]))
    hi = torch.searchsorted(grid, a.contiguous()).clamp(1, len(grid) - 1)
    down, up = a - grid[hi - 1], grid[hi] - a
    return torch.where((down < up) | ((down == up) & ((hi - 1) % 2 == 0)), hi - 1, hi)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def ok():
    torch.cuda.synchronize()
    assert hyp.hyp_device_wait_status(True) == 0


# ---------------------------------------------------------------------------------------------
# microscaled 4-bit matrices
# ---------------------------------------------------------------------------------------------
def quantized(x):
    """(codes, scales) of x as the header defines them, from fp64."""
    n, k = x.shape
    blocks = (k + 31) // 32
    d = torch.zeros(n, blocks * 32, dtype=torch.float64, device=x.device)
    d[:, :k] = x.double()
    d = d.view(n, blocks, 32)
    bad = ~torch.isfinite(d).all(2)
    amax = torch.where(bad, torch.zeros(()).double().to(x.device), d.abs().amax(2))
    e = torch.where(amax > 0, torch.floor(torch.log2(torch.where(amax > 0, amax, torch.ones_like(amax)))) - 2, torch.tensor(-127.0).double().to(x.device))
    e = e.clamp(min=-127)
    place = nearest(torch.where(bad[:, :, None], torch.zeros_like(d), d) * torch.exp2(-e)[:, :, None], FP4)
    code = (place + 8 * (torch.signbit(d) & ~bad[:, :, None])).to(torch.uint8).view(n, -1)[:, :k]
    return code[:, 0::2] | (code[:, 1::2] << 4), torch.where(bad, 255, e + 127).to(torch.uint8)


def values(codes, scales, k):
    """fp64 [n, k]; NaN under a scale of 255."""
    nib = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1).long()
    f = torch.exp2(scales.double() - 127)
    f = torch.where(scales == 255, torch.full_like(f, math.nan), f).repeat_interleave(32, 1)[:, :k]
    return FP4.cuda()[nib & 7] * (1 - 2 * (nib >> 3)).double() * f


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k", [(1, 8), (3, 24), (130, 40), (7, 688), (65, 256), (300, 1032)])
def test_quantize_and_back(dtype, n, k):
    x = normal(n, k + 24, seed=n, std=0.02).to(dtype)[:, 8:8 + k].clone()
    x[0, :4] = torch.tensor([0.0, -0.0, 7.0, -5.0])                      # saturation and a tie at the top
    if n > 2:
        x[1] = 0.0
        x[2, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0]) / 4  # every tie of the grid
    if k > 40 and n > 6:
        x[3, 40], x[4, 33], x[5, :32] = math.inf, math.nan, torch.finfo(dtype).tiny / 4
        x[6, :32] = torch.finfo(dtype).max
    wide = torch.full((n, k + 24), 3.0, dtype=dtype, device="cuda")
    wide[:, 8:8 + k] = x
    codes = torch.full((n, k // 2), 0xAB, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, (k + 31) // 32), 0xAB, dtype=torch.uint8, device="cuda")
    hyp.hyp_op_mx4_quantize(wide[:, 8:8 + k], codes, scales)
    ok()
    want_codes, want_scales = quantized(x)
    assert torch.equal(scales, want_scales)
    # the sign of a zero is free
    sign = lambda c: c & ~torch.where((c & 7) == 0, 8, 0).to(torch.uint8) & ~torch.where((c & 0x70) == 0, 0x80, 0).to(torch.uint8)
    assert torch.equal(sign(codes), sign(want_codes))
    back = torch.full((n, k + 16), 5.0, dtype=dtype, device="cuda")
    hyp.hyp_op_mx4_dequantize(codes, scales, back[:, :k])
    ok()
    want = values(codes, scales, k)
    if dtype == torch.float16:
        want = want.clamp(-65504.0, 65504.0)
    got = back[:, :k]
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want.to(dtype)))
    assert (back[:, k:] == 5.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_dequantize_every_code_and_scale(dtype):
    codes = torch.arange(256, device="cuda").to(torch.uint8).view(1, 256).expand(256, -1)[:, :16 * 16].contiguous()  # 512 nibbles a row
    scales = torch.arange(256, device="cuda").to(torch.uint8).view(256, 1).expand(-1, 16).contiguous()
    out = torch.zeros(256, 512, dtype=dtype, device="cuda")
    hyp.hyp_op_mx4_dequantize(codes, scales, out)
    ok()
    want = values(codes, scales, 512)
    if dtype == torch.float16:
        want = want.clamp(-65504.0, 65504.0)
    want = want.to(dtype)
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out, posinf=1e38, neginf=-1e38), torch.nan_to_num(want, posinf=1e38, neginf=-1e38))


def weights(n, k, seed, spread=4):
    g = gen(seed)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(118, 118 + spread, (n, (k + 31) // 32), generator=g, device="cuda", dtype=torch.uint8)
    return codes, scales


def in_terms(a, terms):
    """The activations as the header's sum of terms (fp64)."""
    m, k = a.shape
    x = torch.zeros(m, (k + 31) // 32 * 32, dtype=torch.float64, device="cuda")
    x[:, :k] = a.double()
    x = x.view(m, -1, 32)
    held = torch.zeros_like(x)
    for _ in range(terms):
        rest = x - held
        amax = rest.abs().amax(2, keepdim=True)
        p = torch.exp2(torch.ceil(torch.log2(amax.clamp(min=2.0 ** -140) / 448)).clamp(min=-127))
        held = held + torch.copysign(E4M3.cuda()[nearest(rest / p, E4M3)], rest) * p
    return held.view(m, -1)[:, :k]


def product_bound(a, w, k):
    return k * 2.0 ** -23 * (a.abs() @ w.abs().T)


def product(a, codes, scales, n, terms, epi, out, swiglu=False, stream=None):
    packed = hyp.hyp_op_mx4_pack(codes, scales, swiglu, stream=stream)
    scratch = torch.full((hyp.hyp_op_gemm_mx4_scratch_bytes(a.shape[0], a.shape[1], terms) + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    hyp.hyp_op_gemm_mx4(a, packed, n, terms, epi, out, scratch, stream=stream)
    return packed, scratch


SHAPES = [(1, 128, 128), (1, 1, 8), (5, 130, 40), (8, 700, 688), (9, 256, 1032), (16, 129, 512), (17, 1000, 256), (33, 300, 2048), (80, 128, 384),
          (81, 256, 264), (128, 640, 512), (129, 200, 640), (257, 384, 520), (300, 130, 1024), (700, 257, 264)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype,terms", [(torch.float16, 3), (torch.bfloat16, 2), (torch.float16, 1), (torch.bfloat16, 3), (torch.float16, 2)])
def test_product(m, n, k, dtype, terms):
    a = normal(m, k + 8, seed=m + k).to(dtype)[:, :k]                     # rows of a wider buffer
    codes, scales = weights(n, k, seed=n)
    out = torch.full((m + 1, n + 5), 9.0, device="cuda")
    product(a, codes, scales, n, terms, hyp.HYP_EPI_STORE_F32, out[:m])
    ok()
    w, held = values(codes, scales, k), in_terms(a, terms)
    err = (out[:m, :n].double() - held @ w.T).abs()
    bound = product_bound(held, w, k)
    assert (err <= bound).all(), float((err / bound).max())
    assert (out[m:] == 9.0).all() and (out[:, n:] == 9.0).all()
    if terms == 3 or dtype == torch.bfloat16 and terms == 2:             # the activations themselves, but for the documented rest
        rest = 2.0 ** (-25 if terms == 3 else -17) * float(a.abs().max()) * w.abs().sum(1)
        err = (out[:m, :n].double() - a.double() @ w.T).abs()
        assert (err <= bound + rest).all(), float((err / bound).max())


@pytest.mark.parametrize("n,k", [(1000, 2000), (130, 5120), (700, 4104), (96, 40)])
@pytest.mark.parametrize("m,dtype,terms", [(1, torch.float16, 3), (1, torch.bfloat16, 2), (2, torch.float16, 2), (3, torch.bfloat16, 1),
                                           (5, torch.float16, 3), (7, torch.bfloat16, 2)])
def test_product_of_few_tokens(n, k, m, dtype, terms):
    """Fewer tokens than a tile has places for, behind a product that left NaN wherever it kept its operands."""
    codes, scales = weights(n, k, seed=n)
    product(torch.full((8, k), math.nan, dtype=dtype, device="cuda"), codes, scales, n, 3, hyp.HYP_EPI_STORE_F32, torch.empty(8, n, device="cuda"))
    a = normal(m, k, seed=m + k).to(dtype)
    out = torch.full((m + 1, n), 9.0, device="cuda")
    product(a, codes, scales, n, terms, hyp.HYP_EPI_STORE_F32, out[:m])
    ok()
    w, held = values(codes, scales, k), in_terms(a, terms)
    assert ((out[:m].double() - held @ w.T).abs() <= product_bound(held, w, k)).all()
    assert (out[m:] == 9.0).all()


@pytest.mark.parametrize("m,n,k", [(1, 100, 64), (8, 688, 256), (33, 200, 688), (129, 136, 520), (500, 130, 256)])
@pytest.mark.parametrize("dtype,terms", [(torch.float16, 3), (torch.bfloat16, 1)])
def test_product_epilogues(m, n, k, dtype, terms):
    step = torch.finfo(dtype).eps / 2
    a = normal(m, k, seed=m + k).to(dtype)
    codes, scales = weights(2 * n, k, seed=n)
    w, held = values(codes, scales, k), in_terms(a, terms)
    y, bound = held @ w.T, product_bound(held, w, k)
    # 16-bit results
    out = torch.full((m, n + 3), 9.0, dtype=dtype, device="cuda")
    product(a, codes[:n], scales[:n], n, terms, hyp.HYP_EPI_STORE_BF16, out)
    ok()
    err = (out[:, :n].double() - y[:, :n]).abs()
    assert (err <= bound[:, :n] + step * (y[:, :n].abs() + bound[:, :n])).all()
    assert (out[:, n:] == 9.0).all()
    # added to what is there
    base = normal(m, n, seed=3)
    res = base.clone()
    product(a, codes[:n], scales[:n], n, terms, hyp.HYP_EPI_RESID_F32, res)
    ok()
    want = base.double() + y[:, :n]
    assert ((res.double() - want).abs() <= bound[:, :n] + 2.0 ** -24 * want.abs() * 1.01).all()
    # gate and up
    out = torch.full((m, n), 9.0, dtype=dtype, device="cuda")
    product(a, codes, scales, n, terms, hyp.HYP_EPI_SWIGLU_BF16, out, swiglu=True)
    ok()
    g, u = y[:, :n], y[:, n:]
    silu = g / (1 + torch.exp(-g))
    want = silu * u
    slack = 1.1 * bound[:, :n] * (u.abs() + bound[:, n:]) + silu.abs() * bound[:, n:] + 2.0 ** -20 * want.abs()
    err = (out.double() - want).abs()
    assert (err <= slack + step * (want.abs() + slack)).all(), float((err / (slack + step * want.abs())).max())


def test_product_extremes_stay_in_their_rows():
    m, n, k = 11, 260, 320
    a = normal(m, k, seed=1).half()
    a[2, 77], a[4, 300], a[5], a[6] = math.inf, math.nan, 0.0, 65504.0
    a[7] = 2.0 ** -24                                                     # the smallest fp16 value
    a[8, ::2] *= 2.0 ** -12
    codes, scales = weights(n, k, seed=2)
    scales[3, 1], scales[200, 9] = 255, 255
    scales[5], scales[6] = 0, 200
    codes[5], codes[7] = 0x77, 0x88                                       # 6 * 2^-127; zeros with a sign
    out = torch.zeros(m, n, device="cuda")
    product(a, codes, scales, n, 3, hyp.HYP_EPI_STORE_F32, out)
    ok()
    nan = torch.isnan(out)
    assert nan[2].all() and nan[4].all() and nan[:, 3].all() and nan[:, 200].all()
    rows, cols = [i for i in range(m) if i not in (2, 4)], [j for j in range(n) if j not in (3, 200)]
    got = out[rows][:, cols].double()
    w, held = values(codes, scales, k)[cols], in_terms(a[rows], 3)
    assert torch.isfinite(got).all()
    # products below fp32's normal range may be lost: K 2^-126
    assert ((got - held @ w.T).abs() <= product_bound(held, w, k) + k * 2.0 ** -126).all()
    assert (got[rows.index(5)] == 0).all()
    sat = torch.zeros(m, n, dtype=torch.float16, device="cuda")
    scales[:] = 130
    product(a, codes, scales, n, 3, hyp.HYP_EPI_STORE_BF16, sat)
    ok()
    big = held @ values(codes, scales, k).T
    past = big.abs() > 70000
    assert past.any() and (sat[rows].double()[past].abs() == 65504).all()


@pytest.mark.parametrize("m", [1, 8, 40])
def test_product_same_on_every_run_and_in_graphs(m):
    n, k = 700, 1024
    a = [normal(m, k, seed=i).half() for i in range(2)]
    codes, scales = weights(n, k, seed=5)
    outs = [torch.zeros(m, n, device="cuda") for _ in range(2)]
    packed, _ = product(a[0], codes, scales, n, 3, hyp.HYP_EPI_STORE_F32, outs[0])
    first = outs[0].clone()
    scratch = [torch.empty(hyp.hyp_op_gemm_mx4_scratch_bytes(m, k, 3), dtype=torch.uint8, device="cuda") for _ in range(2)]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            hyp.hyp_op_gemm_mx4(a[i], packed, n, 3, hyp.HYP_EPI_STORE_F32, outs[i], scratch[i])
        graphs.append(g)
    want = []
    for i in range(2):
        w, held = values(codes, scales, k), in_terms(a[i], 3)
        want.append((held @ w.T, product_bound(held, w, k)))
    side = torch.cuda.Stream()
    for turn in range(3):
        for o in outs:
            o.fill_(-1.0)
        side.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        ok()
        assert torch.equal(outs[0], first)
        assert ((outs[1].double() - want[1][0]).abs() <= want[1][1]).all()
    a[0].copy_(a[1])                                                     # new inputs, the same graph
    graphs[0].replay()
    ok()
    assert torch.equal(outs[0], outs[1])


# ---------------------------------------------------------------------------------------------
# the 8-bit cache
# ---------------------------------------------------------------------------------------------
def half_page(codes, scales, d):
    """uint8 [..., 16 d + 64] of codes [..., 16, d] and scales [..., 16] in the header's order."""
    c = codes
    if d == 128:
        slot, chunk = torch.arange(16, device="cuda")[:, None], torch.arange(8, device="cuda")[None, :]
        c = codes.reshape(*codes.shape[:-1], 8, 16)[..., slot, chunk ^ (4 * (slot & 1)), :].reshape(codes.shape)
    return torch.cat([c.flatten(-2), scales.contiguous().view(torch.uint8).view(*scales.shape[:-1], 64)], -1)


def quantized8(x, fmt):
    """(codes uint8, scales fp32) of fp64 rows x, from the header."""
    bad = ~torch.isfinite(x).all(-1)
    amax = torch.where(bad, torch.zeros(()).double().to(x.device), x.abs().amax(-1))
    zero = amax < 2.0 ** -118
    safe = torch.where(zero, torch.ones_like(amax), amax)
    y = torch.where((bad | zero)[..., None], torch.zeros_like(x), x)
    if fmt == hyp.HYP_KV8_INT8:
        s = (safe / 127).float()
        code = (torch.round(y / s.double()[..., None]) + 128).to(torch.uint8)
    else:
        s = torch.exp2(torch.ceil(torch.log2(safe / 448))).float()
        place = nearest(y / s.double()[..., None], E4M3)
        code = (place + 128 * (torch.signbit(y) & (place > 0))).to(torch.uint8)
    s = torch.where(zero, torch.zeros_like(s), s)
    return code, torch.where(bad, torch.full_like(s, math.nan), s)


def numbers(codes, fmt):
    return codes.double() - 128 if fmt == hyp.HYP_KV8_INT8 else codes.view(torch.float8_e4m3fn).double()


def rope_table(n, d, theta=10000.0):
    a = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * theta ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    return torch.stack([a.cos(), a.sin()], 2).float().contiguous()


def rotated(x, table, pos):
    """x [rows, heads, d] fp64 by the table's (fp32) angles."""
    d = x.shape[2]
    cs = table[pos].double()[:, None]
    a, b = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1)


def same_codes(got, want, fmt):
    if fmt == hyp.HYP_KV8_E4M3:                                          # the sign of a zero is free
        got, want = torch.where(got == 0x80, 0, got), torch.where(want == 0x80, 0, want)
    return torch.equal(got, want)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,rope,with_q", [(torch.float32, True, True), (torch.float32, False, False), (torch.float16, True, False),
                                               (torch.bfloat16, True, True), (torch.bfloat16, False, True)])
def test_write_and_read(heads, fmt, dtype, rope, with_q):
    hq, hkv, d = heads
    # new rows and cached tokens of each sequence: an empty one, one that starts inside a page, padding (-1), one that runs past its table
    rows, ctx, width = [5, 0, 37, 1, 20, 1], [0, 9, 13, 47, 60, -1], 5
    n, m = len(rows), sum(rows)
    qkv = normal(m + 3, (hq + 2 * hkv) * d + 16, seed=hq * d).to(dtype)
    qkv[1, hq * d:(hq + 1) * d] = 0.0                                    # a key of zeros
    qkv[2, (hq + hkv) * d + 3] = math.inf                                # a value with an infinity
    qkv[3, hq * d + 1] = math.nan
    qkv[4, (hq + hkv) * d:(hq + hkv + 1) * d] *= 1e-3
    qkv[6, hq * d:(hq + 1) * d] = torch.arange(d, device="cuda").to(dtype)
    rng = np.random.default_rng(7)
    table = torch.from_numpy(rng.permutation(n * width + 2)[:n * width].reshape(n, width).astype(np.int32)).cuda()
    pool = torch.full((n * width + 2, 2, hkv, 16 * d + 64), 0xAB, dtype=torch.uint8, device="cuda")
    before = pool.clone()
    tab = rope_table(90, d) if rope else None
    cu = i32(np.concatenate([[0], np.cumsum(rows)]).tolist())
    q_out = torch.full((m + 3, hq * d), 9.0, dtype=torch.float16, device="cuda") if with_q else None
    hyp.hyp_op_kv8_write(heads, fmt, qkv, pool, table, cu, i32(ctx), tab, q_out)
    ok()
    x = qkv[:m].double()[:, :(hq + 2 * hkv) * d].view(m, hq + 2 * hkv, d)
    seq = torch.repeat_interleave(torch.arange(n), torch.tensor(rows)).cuda()
    pos = i32(ctx).long()[seq] + torch.arange(m, device="cuda") - cu.long()[seq]
    turned = rotated(x[:, :hq + hkv], tab, pos.clamp(min=0)) if rope else x[:, :hq + hkv]
    if with_q:
        want = turned[:, :hq].reshape(m, hq * d)
        assert ((q_out[:m].double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -22 * 8 + 2.0 ** -25).all()
        assert (q_out[m:] == 9.0).all()
    codes, scales = quantized8(torch.stack([turned[:, hq:], x[:, hq + hkv:]], 1), fmt)     # [m, 2, hkv, d], [m, 2, hkv]
    # every slot of the pool: what belongs to a row, and everything else as it was
    want_codes = before[..., :16 * d].clone()
    want_scales = before[..., 16 * d:].clone()
    half = half_page(torch.zeros(1, 16, d, dtype=torch.uint8, device="cuda"), torch.zeros(1, 16, device="cuda"), d)
    assert half.shape[-1] == 16 * d + 64
    order = torch.arange(d, device="cuda")
    for r in range(m):
        p = int(pos[r])
        if p < 0 or p >= 16 * width:
            continue
        page, slot = int(table[int(seq[r]), p // 16]), p % 16
        place = order ^ (64 * (slot & 1)) if d == 128 else order
        want_codes.view(*want_codes.shape[:3], 16, d)[page, :, :, slot, place] = codes[r]
        want_scales.view(*want_scales.shape[:3], 16, 4)[page, :, :, slot] = scales[r].contiguous().view(torch.uint8).view(2, hkv, 4)
    got_scales, w_scales = pool[..., 16 * d:].contiguous().view(torch.float32), want_scales.contiguous().view(torch.float32)
    assert torch.equal(torch.isnan(got_scales), torch.isnan(w_scales))
    assert torch.equal(torch.nan_to_num(got_scales), torch.nan_to_num(w_scales))
    assert same_codes(pool[..., :16 * d], want_codes, fmt)

    # back to fp16 pages, from the first new token on
    dst = torch.full((n * width, 2, hkv, 16, d), 5.0, dtype=torch.float16, device="cuda")
    dtable = torch.from_numpy(rng.permutation(n * width).reshape(n, width).astype(np.int32)).cuda()
    lens = i32([c + r for c, r in zip(ctx, rows)])
    hyp.hyp_op_kv8_read(heads, fmt, pool, table, i32(ctx), lens, dst, dtable)
    ok()
    want = torch.full_like(dst, 5.0)
    val = (numbers(codes, fmt) * scales.double()[..., None]).clamp(-65504.0, 65504.0).half()
    for r in range(m):
        p = int(pos[r])
        if p < 0 or p >= 16 * width:
            continue
        slot = p % 16
        place = order ^ (8 * (slot & 7))
        want[int(dtable[int(seq[r]), p // 16]), :, :, slot, place] = val[r]
    # a sequence that ends at -1 + 1 = 0 tokens reads nothing
    assert torch.equal(torch.isnan(dst), torch.isnan(want)) and torch.equal(torch.nan_to_num(dst), torch.nan_to_num(want))


def test_write_many_sequences_finds_every_row():
    heads, fmt = (4, 2, 64), hyp.HYP_KV8_INT8
    hq, hkv, d = heads
    for n in (1, 31, 32, 33, 1000, 1025, 4000):
        rows = np.random.default_rng(n).integers(0, 3, n)
        rows[-1] += 1
        m = int(rows.sum())
        qkv = normal(m, (hq + 2 * hkv) * d, seed=n).half()
        table = torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1).contiguous()
        pool = torch.zeros(n, 2, hkv, 16 * d + 64, dtype=torch.uint8, device="cuda")
        cu = i32(np.concatenate([[0], np.cumsum(rows)]).tolist())
        hyp.hyp_op_kv8_write(heads, fmt, qkv, pool, table, cu, torch.zeros(n, dtype=torch.int32, device="cuda"))
        ok()
        seq = torch.repeat_interleave(torch.arange(n), torch.from_numpy(rows)).cuda()
        slot = torch.arange(m, device="cuda") - cu.long()[seq]
        codes, scales = quantized8(qkv.double().view(m, hq + 2 * hkv, d)[:, hq:].view(m, 2, hkv, d), fmt)
        got = pool[..., :16 * d].view(n, 2, hkv, 16, d)[seq, :, :, slot]
        assert torch.equal(got, codes)
        assert torch.equal(pool[..., 16 * d:].contiguous().view(torch.float32)[seq, :, :, slot], scales)


class Cache8:
    """A pool of 0xFF (NaN scales, NaN E4M3 codes) with the rows of n sequences in shuffled pages; page 0 belongs to nobody."""

    def __init__(self, lens, hkv, d, fmt, seed, extra=2, spread=0.0):
        width = max((l + 15) // 16 for l in lens) + extra
        need = sum((l + 15) // 16 for l in lens)
        perm = torch.from_numpy(np.random.default_rng(seed).permutation(need) + 1)
        self.pool = torch.full((need + 1, 2, hkv, 16 * d + 64), 0xFF, dtype=torch.uint8, device="cuda")
        self.table = torch.zeros(len(lens), width, dtype=torch.int32)
        self.k, self.v = [], []
        at = 0
        for i, l in enumerate(lens):
            x = normal(l, 2, hkv, d, seed=seed + i)
            if spread:
                x = x * torch.exp2(normal(l, 2, hkv, 1, seed=seed + 50 + i) * spread * torch.tensor([0.2, 1.0], device="cuda").view(1, 2, 1, 1))
                x[l // 2] *= torch.tensor([1.0, 0.0], device="cuda").view(2, 1, 1)            # values of zeros
            codes, scales = quantized8(x.double(), fmt)
            val = numbers(codes, fmt) * scales.double()[..., None]
            self.k.append(val[:, 0]); self.v.append(val[:, 1])
            for p in range((l + 15) // 16):
                page = int(perm[at]); at += 1
                self.table[i, p] = page
                c = torch.full((2, hkv, 16, d), 0xFF, dtype=torch.uint8, device="cuda")
                s = torch.full((2, hkv, 16), math.nan, device="cuda")
                r = min(16, l - 16 * p)
                c[:, :, :r] = codes[16 * p:16 * p + r].permute(1, 2, 0, 3)
                s[:, :, :r] = scales[16 * p:16 * p + r].permute(1, 2, 0)
                self.pool[page] = half_page(c, s, d)
        self.table = self.table.cuda()


def attention(q, k, v):
    """q [hq, d], k / v [t, hkv, d] (fp64): (out, bound)."""
    hq, d = q.shape
    rep = hq // k.shape[1]
    k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
    s = torch.einsum("hd,thd->ht", q, k) / math.sqrt(d)
    serr = 2.0 ** -20 * (torch.einsum("hd,thd->ht", q.abs(), k.abs()).amax() / math.sqrt(d) + 8.0)
    p = torch.softmax(s, -1)
    out = torch.einsum("ht,thd->hd", p, v)
    size = torch.einsum("ht,thd->hd", p, v.abs())
    # the largest weight times scale, with codes of up to 448 relative to it: 4 rows of |v| cover 127 and 448 / 1.75
    top = (p[:, :, None] * v.abs().transpose(0, 1)).amax((1, 2)).view(hq, 1) * 4
    return out, 2.0 ** -11 * (out.abs() + size) * 1.01 + 2 * serr * size + k.shape[0] * 2.0 ** -25 * top + 2.0 ** -25


def attend(heads, fmt, q, pool, table, ctx):
    out = torch.full((q.shape[0], heads[0] * heads[2]), 7.0, dtype=torch.float16, device="cuda")
    scratch = torch.full((max(16, hyp.hyp_op_attn_kv8_scratch_bytes(heads, q.shape[0], table.shape[1])),), 0xFF, dtype=torch.uint8, device="cuda")
    hyp.hyp_op_attn_decode_kv8(heads, fmt, q, pool, table, ctx, scratch, out)
    ok()
    return out


def check_attention(heads, fmt, lens, seed, extra=2, spread=0.0, std=1.5):
    hq, hkv, d = heads
    c = Cache8(lens, hkv, d, fmt, seed, extra, spread)
    q = (normal(len(lens), (hq + 2) * d, seed=seed + 9) * std).half()[:, :hq * d]
    out = attend(heads, fmt, q, c.pool, c.table, i32([l - 1 for l in lens]))
    for i, l in enumerate(lens):
        if l == 0:
            assert (out[i] == 0).all()
            continue
        want, bound = attention(q[i].double().view(hq, d), c.k[i], c.v[i])
        err = (out[i].double().view(hq, d) - want).abs()
        assert torch.isfinite(out[i]).all(), (i, l)
        assert (err <= bound).all(), (i, l, float((err / bound).max()))


@pytest.mark.parametrize("heads", HEADS + [(4, 1, 128), (2, 1, 64), (4, 2, 128)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_attention(heads, fmt):
    check_attention(heads, fmt, [1, 15, 16, 17, 0, 64, 65, 100, 333], 3)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,lens,extra", [((8, 2, 128), [2500], 0), ((8, 1, 64), [5000, 31], 3), ((40, 10, 128), [1100, 900, 1, 0, 700], 2),
                                              ((4, 2, 64), [9000], 700), ((8, 8, 128), [300] * 40, 1), ((8, 2, 128), [20] * 130, 100)])
def test_attention_splits(heads, fmt, lens, extra):
    check_attention(heads, fmt, lens, 11, extra)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("spread,std", [(6.0, 1.5), (0.0, 12.0), (4.0, 6.0)])
def test_attention_uneven_scales_and_sharp_scores(fmt, spread, std):
    check_attention((8, 2, 128), fmt, [1, 40, 700, 3000], 21, 2, spread, std)


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_first_values_are_zeros(fmt):
    """The first page's values have scales of 0, the later ones large values: the weights' reference has to move."""
    heads, l = (4, 1, 64), 200
    c = Cache8([l], 1, 64, fmt, 31)
    x = normal(l, 2, 1, 64, seed=32)
    x[:16, 1] = 0.0
    x[16:, 1] *= 3000.0
    codes, scales = quantized8(x.double(), fmt)
    for p in range((l + 15) // 16):
        r = min(16, l - 16 * p)
        c_, s_ = torch.full((2, 1, 16, 64), 0xFF, dtype=torch.uint8, device="cuda"), torch.full((2, 1, 16), math.nan, device="cuda")
        c_[:, :, :r], s_[:, :, :r] = codes[16 * p:16 * p + r].permute(1, 2, 0, 3), scales[16 * p:16 * p + r].permute(1, 2, 0)
        c.pool[int(c.table[0, p])] = half_page(c_, s_, 64)
    val = numbers(codes, fmt) * scales.double()[..., None]
    q = normal(1, 256, seed=33).half()
    out = attend(heads, fmt, q, c.pool, c.table, i32([l - 1]))
    want, bound = attention(q[0].double().view(4, 64), val[:, 0], val[:, 1])
    assert ((out[0].double().view(4, 64) - want).abs() <= bound).all()


def test_attention_lengths_past_the_table_and_nan_rows():
    heads, fmt = (8, 2, 128), hyp.HYP_KV8_INT8
    c = Cache8([64, 64, 64], 2, 128, fmt, 41, extra=0)
    q = normal(3, 1024, seed=42).half()
    full = attend(heads, fmt, q, c.pool, c.table, i32([63, 63, 63]))
    past = attend(heads, fmt, q, c.pool, c.table, i32([2 ** 31 - 1, 64, 63]))
    assert torch.equal(full, past)
    assert (attend(heads, fmt, q, c.pool, c.table, i32([-1, -(2 ** 31), 63]))[:2] == 0).all()
    page = int(c.table[1, 2])
    c.pool[page, 0, 1, 16 * 128:16 * 128 + 4] = 0xFF                     # a NaN scale of one key of KV head 1
    out = attend(heads, fmt, q, c.pool, c.table, i32([63, 63, 63])).view(3, 8, 128)
    assert torch.isnan(out[1, 4:]).all()
    keep = full.view(3, 8, 128)
    assert torch.equal(out[0], keep[0]) and torch.equal(out[2], keep[2]) and torch.equal(out[1, :4], keep[1, :4])


@pytest.mark.parametrize("fmt", FORMATS)
def test_cache_beyond_32_bit_offsets(fmt):
    """Pages whose byte offsets pass 2^32."""
    heads, d, hkv = (8, 8, 128), 128, 8
    n_pages = (1 << 32) // (2 * hkv * 2112) + 40
    pool = torch.empty(n_pages, 2, hkv, 2112, dtype=torch.uint8, device="cuda")
    table = i32([[n_pages - 1, 3, n_pages - 17], [n_pages - 30, n_pages - 5, 1]])
    qkv = normal(70, 24 * d, seed=5).half()
    q = torch.empty(70, 8 * d, dtype=torch.float16, device="cuda")
    hyp.hyp_op_kv8_write(heads, fmt, qkv, pool, table, i32([0, 35, 70]), i32([0, 0]), None, q)
    dst = torch.zeros(6, 2, hkv, 16, d, dtype=torch.float16, device="cuda")
    dtable = i32([[0, 1, 2], [3, 4, 5]])
    hyp.hyp_op_kv8_read(heads, fmt, pool, table, None, i32([35, 35]), dst, dtable)
    out = attend(heads, fmt, q[34::35].contiguous(), pool, table, i32([34, 34]))
    codes, scales = quantized8(qkv.double().view(70, 24, d)[:, 8:].view(70, 2, hkv, d), fmt)
    val = numbers(codes, fmt) * scales.double()[..., None]
    for i in range(2):
        want, bound = attention(q[35 * i + 34].double().view(8, d), val[35 * i:35 * i + 35, 0], val[35 * i:35 * i + 35, 1])
        assert ((out[i].double().view(8, d) - want).abs() <= bound).all()
        t = torch.arange(35, device="cuda")
        place = torch.arange(d, device="cuda")[None, :] ^ (8 * (t[:, None] & 7))
        got = dst[dtable[i].long()[t // 16], :, :, t % 16].gather(3, place[:, None, None].expand(-1, 2, hkv, -1))
        assert torch.equal(got, val[35 * i:35 * i + 35].half())


# ---------------------------------------------------------------------------------------------
# together: the attention half of a decode step, and a prompt
# ---------------------------------------------------------------------------------------------
def test_attention_half_of_a_decode_step_in_few_bits():
    """norm -> q/k/v product -> rotate, quantise, append -> attention -> O product added to the stream; captured once, replayed for
    three steps on growing lengths and on a stream of its own.  Each stage is checked on the stage before it as it came out."""
    hid, heads, fmt, n = 256, (4, 2, 64), hyp.HYP_KV8_INT8, 5
    hq, hkv, d = heads
    wide = (hq + 2 * hkv) * d
    wq, wo = quantized(normal(wide, hid, seed=1, std=0.05)), quantized(normal(hid, hq * d, seed=2, std=0.05))
    pq, po = hyp.hyp_op_mx4_pack(*wq), hyp.hyp_op_mx4_pack(*wo)
    gains = torch.ones(hid, dtype=torch.bfloat16, device="cuda")
    start = [0, 15, 16, 40, -1]
    table = torch.randperm(n * 4, generator=gen(3), device="cuda").to(torch.int32).view(n, 4).contiguous()
    pool = torch.full((n * 4, 2, hkv, 16 * d + 64), 0xFF, dtype=torch.uint8, device="cuda")
    tab = rope_table(64, d)
    # what is cached already
    old = [normal(max(s, 0), wide, seed=10 + i).half() for i, s in enumerate(start)]
    cu_old = i32(np.concatenate([[0], np.cumsum([len(o) for o in old])]).tolist())
    hyp.hyp_op_kv8_write(heads, fmt, torch.cat(old), pool, table, cu_old, torch.zeros(n, dtype=torch.int32, device="cuda"), tab)
    x = normal(n, hid, seed=4)
    h = torch.empty(n, hid, dtype=torch.bfloat16, device="cuda")
    qkv = torch.empty(n, wide, device="cuda")
    q = torch.empty(n, hq * d, dtype=torch.float16, device="cuda")
    o = torch.empty(n, hq * d, dtype=torch.float16, device="cuda")
    ctx, cu = i32(start), i32(range(n + 1))
    s1 = torch.empty(hyp.hyp_op_gemm_mx4_scratch_bytes(n, hid, 2), dtype=torch.uint8, device="cuda")
    s2 = torch.empty(hyp.hyp_op_gemm_mx4_scratch_bytes(n, hq * d, 3), dtype=torch.uint8, device="cuda")
    s3 = torch.empty(max(16, hyp.hyp_op_attn_kv8_scratch_bytes(heads, n, 4)), dtype=torch.uint8, device="cuda")

    def step(stream):
        hyp.hyp_op_rmsnorm(x, gains, h, 1e-5, stream)
        hyp.hyp_op_gemm_mx4(h, pq, wide, 2, hyp.HYP_EPI_STORE_F32, qkv, s1, stream)
        hyp.hyp_op_kv8_write(heads, fmt, qkv, pool, table, cu, ctx, tab, q, stream)
        hyp.hyp_op_attn_decode_kv8(heads, fmt, q, pool, table, ctx, s3, o, stream)
        hyp.hyp_op_gemm_mx4(o, po, hid, 3, hyp.HYP_EPI_RESID_F32, x, s2, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep = x.clone(), pool.clone()
    with torch.cuda.stream(side):
        step(side)                                                       # first calls outside the capture
        ok()
        x.copy_(keep[0]); pool.copy_(keep[1])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(side)
    hist = []
    for i, s in enumerate(start):
        y = old[i].double().view(-1, hq + 2 * hkv, d)
        k = rotated(y[:, hq:hq + hkv], tab, torch.arange(len(y), device="cuda"))
        hist.append((k, y[:, hq + hkv:]))
    wqv, wov = values(*wq, hid), values(*wo, hq * d)
    for turn in range(3):
        before = x.clone()
        with torch.cuda.stream(side):
            g.replay()
        ok()
        want = before.double() / torch.sqrt((before.double() ** 2).mean(1, keepdim=True) + 1e-5)
        assert ((h.double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 1e-6).all()
        a = h.double()
        assert ((qkv.double() - a @ wqv.T).abs() <= product_bound(a, wqv, hid) + 2.0 ** -17 * a.abs().max() * wqv.abs().sum(1)).all()
        y = qkv.double().view(n, hq + 2 * hkv, d)
        at = ctx.long().clamp(min=0)
        for i, s in enumerate(start):
            if s < 0:
                assert (o[i] == 0).all()
                continue
            kr = rotated(y[i:i + 1, hq:hq + hkv], tab, at[i:i + 1])
            hist[i] = (torch.cat([hist[i][0], kr]), torch.cat([hist[i][1], y[i:i + 1, hq + hkv:]]))
            k, v = [numbers(c, fmt) * sc.double()[..., None] for c, sc in (quantized8(t, fmt) for t in hist[i])]
            want, bound = attention(q[i].double().view(hq, d), k, v)
            assert ((o[i].double().view(hq, d) - want).abs() <= bound).all(), (turn, i)
        want = before.double() + o.double() @ wov.T
        assert ((x.double() - want).abs() <= product_bound(o.double(), wov, hq * d) + 2.0 ** -23 * want.abs() + 1e-6).all()
        ctx += (ctx >= 0).int()


def test_prompt_through_the_8_bit_cache():
    """A prompt's rows are written, read back into fp16 pages and attended there; the next token attends over the 8-bit pages.  Both
    agree with the read-back values."""
    heads, fmt, rows = (8, 2, 128), hyp.HYP_KV8_E4M3, 70
    hq, hkv, d = heads
    qkv = normal(rows, (hq + 2 * hkv) * d, seed=6)
    tab = rope_table(80, d)
    table = i32([[4, 1, 3, 0, 2]])
    pool = torch.full((5, 2, hkv, 16 * d + 64), 0xFF, dtype=torch.uint8, device="cuda")
    q = torch.empty(rows, hq * d, dtype=torch.float16, device="cuda")
    hyp.hyp_op_kv8_write(heads, fmt, qkv, pool, table, i32([0, rows]), i32([0]), tab, q)
    pages = torch.zeros(5, 2, hkv, 16, d, dtype=torch.float16, device="cuda")
    hyp.hyp_op_kv8_read(heads, fmt, pool, table, None, i32([rows]), pages, table)
    out = torch.empty(rows, hq * d, dtype=torch.float16, device="cuda")
    hyp.hyp_op_attn_prefill(heads, q, pages, table, i32([0, rows]), i32([0]), out)
    last = attend(heads, fmt, q[-1:].contiguous(), pool, table, i32([rows - 1]))
    y = qkv.double().view(rows, hq + 2 * hkv, d)
    k, v = [numbers(c, fmt) * s.double()[..., None] for c, s in
            (quantized8(t, fmt) for t in (rotated(y[:, hq:hq + hkv], tab, torch.arange(rows, device="cuda")), y[:, hq + hkv:]))]
    for r in (0, 15, 16, 40, rows - 1):
        want, bound = attention(q[r].double().view(hq, d), k[:r + 1], v[:r + 1])
        # read back once more rounded: e4m3 values under a power of two are exact in fp16 unless subnormal
        assert ((out[r].double().view(hq, d) - want).abs() <= bound + 2.0 ** -9).all()
    assert ((last[0].double().view(hq, d) - want).abs() <= bound).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,lens,extra", [((8, 2, 128), [3000, 0, 0, 1, 2999, 33, 32, 31, 0], 1200), ((2, 1, 64), [9001], 4000),
                                              ((8, 1, 64), [5] * 60 + [6000] + [0] * 3, 2000), ((40, 10, 128), [4100, 17, 2050, 4096], 900),
                                              ((3, 3, 64), [1, 1, 1], 6000), ((8, 8, 128), [16, 48, 47, 700], 3000)])
def test_attention_even_runs(heads, fmt, lens, extra):
    """Tables wide enough for runs across sequences: empty ones, one that holds everything, runs that end inside pages' pairs."""
    check_attention(heads, fmt, lens, 51, extra)


def test_attention_many_sequences():
    """More sequences than share one list of runs."""
    heads, fmt, n = (2, 1, 64), hyp.HYP_KV8_INT8, 600
    c = Cache8([5, 70, 1000], 1, 64, fmt, 61, 0)
    table = c.table.repeat(n // 3, 1)
    q = normal(n, 128, seed=62).half()
    out = attend(heads, fmt, q, c.pool, table, i32([4, 69, 999] * (n // 3)))
    wide = torch.cat([table, table.new_zeros(n, 9000)], 1)                    # the same lengths in a table that is planned for more
    again = attend(heads, fmt, q, c.pool, wide, i32([4, 69, 999] * (n // 3)))
    for r in (out, again):
        for i in list(range(0, 9)) + [n - 1, n - 2, n - 3, 300, 301, 302]:
            want, bound = attention(q[i].double().view(2, 64), c.k[i % 3], c.v[i % 3])
            assert ((r[i].double().view(2, 64) - want).abs() <= bound).all(), i
