"""The 4-bit product through every kernel and cut that sizes select: both counts of row tiles, terms by a launch of their own (one chunk a thread, two) and
by the CTAs, shares of K behind every epilogue, rings that go round, one and two CTAs to an SM, more than one wave.

Two products a case.  Dense weights, within the bounds of test_gpu_low_bit.py.  Weights with one value a row: sums of one product are exact,
so that results are the activation's terms times the value, to the bit (SwiGLU: to its functions' 2^-20), wherever in K the value sits."""
import pytest
import torch

from paper_2511_14450_b200 import hyperion as hyp
from tests import test_gpu_low_bit as low

H, B = torch.float16, torch.bfloat16
S16, ADD, GLU, F32 = hyp.HYP_EPI_STORE_BF16, hyp.HYP_EPI_RESID_F32, hyp.HYP_EPI_SWIGLU_BF16, hyp.HYP_EPI_STORE_F32
CASES = [(1, 512, 256, H, 3, F32), (3, 70, 64, H, 1, S16), (1, 66, 72, B, 1, ADD), (8, 5120, 5120, H, 3, ADD), (8, 7680, 5120, H, 3, F32), (8, 2048, 4096, H, 3, GLU), (8, 2048, 4096, B, 2, S16), (1, 7680, 5120, H, 3, S16),
         (1, 7680, 5120, B, 2, ADD), (1, 7680, 5120, H, 3, F32), (8, 300, 4104, B, 2, GLU), (8, 300, 4104, H, 3, S16), (8, 300, 4104, H, 3, ADD),
         (64, 5120, 5120, H, 3, ADD), (64, 7680, 5120, B, 2, S16), (512, 5120, 512, H, 3, F32), (2048, 7680, 256, B, 1, F32),
         (520, 200, 5128, H, 1, F32), (520, 200, 5128, H, 2, F32), (520, 200, 5128, H, 3, F32), (520, 200, 5128, B, 1, F32),
         (520, 200, 5128, B, 2, F32), (520, 200, 5128, B, 3, F32), (700, 7700, 2056, H, 3, S16), (700, 7700, 2056, B, 2, ADD),
         (700, 7700, 2056, B, 1, F32), (600, 7700, 2056, H, 3, GLU), (700, 1065, 5048, H, 3, S16), (700, 980, 5776, H, 3, ADD),
         (520, 1194, 5520, B, 3, F32), (8, 9646, 1416, B, 2, ADD), (2, 7065, 1968, H, 2, S16), (2, 4843, 2968, H, 1, F32), (2, 9675, 1352, B, 2, GLU),
         (2, 13037, 2312, H, 1, ADD), (1, 7443, 2592, H, 1, GLU), (300, 712, 3920, H, 3, S16), (520, 1040, 2456, H, 1, ADD),
         (300, 1355, 2464, B, 1, GLU), (300, 976, 2928, H, 3, F32), (2, 20000, 512, B, 1, ADD), (17, 11092, 64, H, 3, S16), (64, 6738, 64, H, 2, F32),
         (130, 5191, 64, B, 3, GLU), (520, 808, 1688, H, 3, GLU), (520, 846, 2648, H, 3, F32), (8, 20049, 2720, H, 3, GLU), (700, 4320, 64, H, 3, ADD),
         (520, 2831, 664, H, 3, ADD), (130, 19737, 144, B, 2, S16), (520, 2696, 848, H, 3, F32),
         (70001, 130, 264, H, 3, F32), (1, 130, 200008, H, 3, F32), (9, 140, 100000, B, 2, GLU)]


def paths(case):
    """What a case goes through, by its plan on the current device (148 SMs where there is none)."""
    m, n, k, dtype, terms, epi = case
    p, kb = hyp.hyp_op_gemm_mx4_plan(m, n, k, terms, epi), (k + 127) // 128
    found = {("kernel", epi, p["row_tiles"], p["own_terms"]), ("tokens", p["token_tiles"] > 1, p["row_tiles"], p["shares"] > 1)}
    if not p["own_terms"]:
        found.add(("terms", dtype, terms, p["chunks"]))
    if p["shares"] > 1:
        found |= {("split", epi, p["row_tiles"]), ("split", "own", p["own_terms"]), ("shares", p["shares"])}
    if -(-kb // p["shares"]) > 2 * p["stages"]:
        found.add(("ring", p["row_tiles"], p["shares"] > 1))
    if p["per_sm"] > 1 and p["ctas"] > 148:
        found.add(("two an SM", epi))
        found.add(("two an SM", p["shares"] > 1))
    if p["ctas"] > 148 * p["per_sm"]:
        found.add(("waves", p["row_tiles"]))
    if p["row_tiles"] == 2 and epi != GLU and (n + 127) // 128 % 2:
        found.add(("odd row tiles",))
    return found


WANTED = ({("kernel", e, a, o) for e in (S16, ADD, GLU, F32) for a in (1, 2) for o in (0, 1) if (e, a) != (GLU, 1)}
          | {("split", e, a) for e in (S16, ADD, GLU, F32) for a in (1, 2) if (e, a) != (GLU, 1)} | {("split", "own", 0), ("split", "own", 1)}
          | {("terms", t, c, u) for t in (H, B) for c in (1, 2, 3) for u in (1, 2)} | {("ring", a, s) for a in (1, 2) for s in (False, True)}
          | {("two an SM", e) for e in (S16, ADD, GLU, F32)} | {("two an SM", True)} | {("waves", 1), ("waves", 2), ("odd row tiles",)}
          | {("tokens", t, a, s) for t in (False, True) for a in (1, 2) for s in (False, True)})


@pytest.mark.gpu
def test_the_cases_reach_every_path():
    missing = WANTED - set().union(*(paths(c) for c in CASES))
    assert not missing, missing


def in_terms(a, terms):
    """The activations as the header's sum of terms (fp64).  448 = 0.875 * 2^9, so the power of two comes from the largest magnitude's own
    parts (a logarithm would have to be exact where it is a whole number)."""
    m, k = a.shape
    x = torch.zeros(m, (k + 31) // 32 * 32, dtype=torch.float64, device="cuda")
    x[:, :k] = a.double()
    x = x.view(m, -1, 32)
    held = torch.zeros_like(x)
    for _ in range(terms):
        rest = x - held
        part, e = torch.frexp(rest.abs().amax(2, keepdim=True))
        p = torch.exp2(torch.where(part > 0, torch.where(part <= 0.875, e - 9, e - 8), -127).clamp(min=-127).double())
        held = held + torch.copysign(low.E4M3.cuda()[low.nearest(rest / p, low.E4M3)], rest) * p
    return held.view(m, -1)[:, :k]


def one_value_a_row(rows, k, seed):
    """Codes with one value other than 0 a row, at places that walk through K, and the scales."""
    g = low.gen(seed)
    at = (torch.arange(rows, device="cuda") * 7919 + 13) % k
    code = torch.randint(1, 8, (rows,), generator=g, device="cuda") + 8 * torch.randint(0, 2, (rows,), generator=g, device="cuda")
    nib = torch.zeros(rows, k, dtype=torch.uint8, device="cuda")
    nib[torch.arange(rows, device="cuda"), at] = code.to(torch.uint8)
    scales = torch.randint(118, 122, (rows, (k + 31) // 32), generator=g, device="cuda", dtype=torch.uint8)
    return nib[:, 0::2] | (nib[:, 1::2] << 4), scales


def run(case, a, codes, scales, base, pad):
    m, n, k, dtype, terms, epi = case
    wide = torch.full((m + 1, n + pad), 9.0, dtype=dtype if epi in (S16, GLU) else torch.float32, device="cuda")
    if epi == ADD:
        wide[:m, :n] = base
    low.product(a, codes, scales, n, terms, epi, wide[:m], epi == GLU)
    low.ok()
    assert (wide[m:] == 9.0).all() and (wide[:, n:] == 9.0).all()
    return wide[:m, :n]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}-{'fp16' if c[3] is H else 'bf16'}-{c[4]}-{c[5]}")
def test_product_paths(case):
    m, n, k, dtype, terms, epi = case
    step, rows = torch.finfo(dtype).eps / 2, 2 * n if epi == GLU else n
    a, base = low.normal(m, k, seed=m + k).to(dtype), low.normal(m, n, seed=3) if epi == ADD else None
    held = in_terms(a, terms)

    codes, scales = low.weights(rows, k, seed=n)
    out = run(case, a, codes, scales, base, -n % 4).double()             # rows of results that start on 16 bytes
    w = low.values(codes, scales, k)
    y, bound = held @ w.T, low.product_bound(held, w, k)
    if epi == GLU:
        g, u = y[:, :n], y[:, n:]
        silu = g / (1 + torch.exp(-g))
        want = silu * u
        bound = 1.1 * bound[:, :n] * (u.abs() + bound[:, n:]) + silu.abs() * bound[:, n:] + 2.0 ** -20 * want.abs()
    else:
        want = y if base is None else base.double() + y
        bound = bound + (2.0 ** -24 * (want.abs() + bound) if epi == ADD else 0.0)
    if epi in (S16, GLU):
        bound = bound + step * (want.abs() + bound) + torch.finfo(dtype).smallest_normal * step
    assert ((out - want).abs() <= bound).all(), float(((out - want).abs() / bound).max())
    del w, y, want, bound, out

    codes, scales = one_value_a_row(rows, k, n + 1)
    out = run(case, a, codes, scales, base, 3)
    y = held @ low.values(codes, scales, k).T                            # exact: the other products are zeros
    assert torch.equal(y.float().double(), y)
    if epi == GLU:
        g, u = y[:, :n], y[:, n:]
        want = g / (1 + torch.exp(-g)) * u
        bound = (step + 2.0 ** -20) * 1.01 * want.abs() + torch.finfo(dtype).smallest_normal * step
        assert ((out.double() - want).abs() <= bound).all()
    elif epi == S16:
        assert torch.equal(out, y.to(dtype))
    else:
        assert torch.equal(out, (y if base is None else base.double() + y).float())
