"""Operators over the paged cache against their definitions in 64 bits: modified scores (prefill and decode), summed
attention weights, eviction, shared prefixes.  Cache slots and pages that no token owns hold NaN, table entries behind a
sequence's end name such a page, queries sit in a wider buffer.

Tolerances.  fp16 outputs: one rounding of the result (2^-11 |out|) and one of every softmax weight (2^-11 sum p |v|, or
2^-25 max |v| a key where a weight, relative to the running maximum, is below 2^-14), plus the scores' fp32 error: a dot
product of D products in fp32 is off by at most D 2^-24 sum |q k|, taken as 2^-20 sum |q k| / sqrt(D) with the function
errors of exp and tanh inside it; an error e of a score changes every weight by the factor 1 + e, the result by 2 e sum p |v|."""
import math

import numpy as np
import pytest
import torch

from paper_2511_14450_b200 import hyperion as hyp

pytestmark = pytest.mark.gpu

HEADS = [(4, 2, 64), (40, 10, 128), (8, 8, 128), (8, 1, 64), (8, 1, 128), (3, 3, 64)]
LENS = [1, 15, 16, 17, 64, 65, 100, 333]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Cache:
    """A pool of NaN with the rows of n sequences in shuffled pages; page 0 belongs to nobody."""

    def __init__(self, lens, hkv, d, seed, extra=2, spare=0):
        g = gen(seed)
        self.lens, self.hkv, self.d = lens, hkv, d
        width = max((l + 15) // 16 for l in lens) + extra
        need = sum((l + 15) // 16 for l in lens) + spare
        perm = torch.from_numpy(np.random.default_rng(seed).permutation(need) + 1)
        self.pool = torch.full((need + 1, 2, hkv, 16, d), float("nan"), dtype=torch.float16, device="cuda")
        self.table = torch.zeros(len(lens), width, dtype=torch.int32)
        self.k, self.v = [], []
        at = 0
        for i, l in enumerate(lens):
            k = torch.randn(l, hkv, d, generator=g, device="cuda").half()
            v = torch.randn(l, hkv, d, generator=g, device="cuda").half()
            self.k.append(k); self.v.append(v)
            for p in range((l + 15) // 16):
                page = int(perm[at]); at += 1
                self.table[i, p] = page
                for kind, x in ((0, k), (1, v)):
                    put(self.pool, page, kind, x[16 * p:16 * p + 16])
        self.spare = perm[at:].to(torch.int32)
        self.table = self.table.cuda()


def put(pool, page, kind, rows):
    """Token rows [slots, hkv, d] into a page, chunk c of slot s at chunk position c ^ (s & 7)."""
    s, hkv, d = rows.shape
    slot = torch.arange(s, device="cuda")
    pos = torch.arange(d // 8, device="cuda")[None, :] ^ (slot[:, None] & 7)
    x = rows.view(s, hkv, d // 8, 8)
    pool.view(*pool.shape[:4], d // 8, 8)[page, kind, :, slot[:, None], pos] = x.permute(1, 0, 2, 3)


def get(pool, table_row, kind, n):
    """Rows 0 .. n-1 behind a table row: [n, hkv, d]."""
    d = pool.shape[4]
    t = torch.arange(n, device="cuda")
    slot = t % 16
    pos = torch.arange(d // 8, device="cuda")[None, :] ^ (slot[:, None] & 7)
    page = table_row[t // 16].long()
    return pool.view(*pool.shape[:4], d // 8, 8)[page[:, None], kind, :, slot[:, None], pos].permute(0, 2, 1, 3).reshape(n, pool.shape[2], d)


def queries(rows, hq, d, seed, std=1.5):
    """Rows of a buffer that also holds other heads."""
    return (torch.randn(rows, (hq + 2) * d, generator=gen(seed), device="cuda") * std).half()[:, :hq * d]


def reference(q, k, v, mask, cap=0.0, bias=None):
    """q [R, hq, d], k / v [T, hkv, d], mask [R, T], bias [hq, R, T]; returns (out [R, hq, d], weights [hq, R, T], bound)."""
    hq, hkv, d = q.shape[1], k.shape[1], k.shape[2]
    q, k, v = q.double(), k.double().repeat_interleave(hq // hkv, 1), v.double().repeat_interleave(hq // hkv, 1)
    s = torch.einsum("rhd,thd->hrt", q, k) / math.sqrt(d)
    serr = 2.0 ** -20 * (torch.einsum("rhd,thd->hrt", q.abs(), k.abs()).amax() / math.sqrt(d) + 8.0)
    if cap:
        s = cap * torch.tanh(s / cap)
        serr = serr + 2.0 ** -20 * cap
    if bias is not None:
        s = s + bias
        serr = serr + 2.0 ** -21 * bias.abs().amax()
    s = s.masked_fill(~mask[None], -math.inf)
    p = torch.softmax(s, -1)
    p = torch.where(mask.any(-1)[None, :, None], p, torch.zeros_like(p))
    out = torch.einsum("hrt,thd->rhd", p, v)
    size = torch.einsum("hrt,thd->rhd", p, v.abs())
    vmax = v.abs().amax() if v.numel() else 0.0
    bound = 2.0 ** -11 * (out.abs() + size) * 1.01 + 2 * serr * size + k.shape[0] * 2.0 ** -25 * vmax + 2.0 ** -25
    return out, p, bound, serr


def close(got, want, bound, what):
    err = (got.double() - want).abs()
    assert torch.isfinite(got.float()).all(), what
    assert (err <= bound).all(), (what, float((err / bound).max()))


def bytes_of(n):
    return torch.full((max(16, n),), 0xFF, dtype=torch.uint8, device="cuda")     # NaN patterns


def run_decode_mod(c, heads, q, ctx, mod):
    out = torch.full((q.shape[0], heads[0] * heads[2]), 7.0, dtype=torch.float16, device="cuda")
    scratch = bytes_of(hyp.hyp_op_attn_mod_scratch_bytes(heads, q.shape[0], c.table.shape[1]))
    hyp.hyp_op_attn_decode_mod(heads, mod, q, c.pool, c.table, ctx, scratch, out)
    torch.cuda.synchronize()
    return out


MODS = [dict(), dict(cap=30.0), dict(slopes=True), dict(window=1), dict(window=20), dict(window=64, prefix=5), dict(prefix=40),
        dict(cap=5.0, slopes=True, window=50, prefix=33)]


def mask_and_bias(pos, total, m, prefix, slopes):
    key = torch.arange(total, device="cuda")[None, :]
    mask = key <= pos[:, None]
    if m.get("window"):
        mask &= key > pos[:, None] - m["window"]
    mask |= key < prefix
    bias = None if slopes is None else -slopes.double()[:, None, None] * (pos[:, None] - key).abs().double()[None]
    return mask, bias


def make_mod(m, hq, n):
    slopes = (torch.arange(1, hq + 1, device="cuda") / hq).float() if m.get("slopes") else None
    pre = torch.tensor([max(0, m["prefix"] - i) for i in range(n)], dtype=torch.int32, device="cuda") if m.get("prefix") else None
    return hyp.AttnMod(softcap=m.get("cap", 0.0), window=m.get("window", 0), slopes=slopes, prefix_lens=pre), slopes, pre


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("m", MODS)
def test_decode_mod(heads, m):
    hq, hkv, d = heads
    c = Cache(LENS, hkv, d, seed=hq + d)
    lens = LENS + [0]                                       # a padding row: nothing to see
    c.table = torch.cat([c.table, torch.zeros_like(c.table[:1])])
    q = queries(len(lens), hq, d, seed=5)
    ctx = torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda")
    mod, slopes, pre = make_mod(m, hq, len(lens))
    out = run_decode_mod(c, heads, q, ctx, mod)
    for i, l in enumerate(LENS):
        mask, bias = mask_and_bias(torch.tensor([l - 1], device="cuda"), l, m, int(pre[i]) if pre is not None else 0, slopes)
        want, _, bound, _ = reference(q[i:i + 1].view(1, hq, d), c.k[i], c.v[i], mask, m.get("cap", 0.0), bias)
        close(out[i].view(1, hq, d), want, bound, (i, l))
    assert (out[-1] == 0).all()


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("m", [dict(cap=30.0), dict(slopes=True, window=700, prefix=33), dict(window=16)])
@pytest.mark.parametrize("lens", [[900, 257, 1000], [7000, 3, 0, 2049], [300 + 7 * i for i in range(60)]])
def test_decode_mod_longer_contexts(heads, m, lens):
    """Splits that join in a cluster, and splits that a second launch joins."""
    hq, hkv, d = heads
    c = Cache([max(l, 1) for l in lens], hkv, d, seed=17)
    q = queries(len(lens), hq, d, seed=18)
    ctx = torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda")
    mod, slopes, pre = make_mod(m, hq, len(lens))
    out = run_decode_mod(c, heads, q, ctx, mod)
    for i, l in enumerate(lens):
        if l == 0:
            assert (out[i] == 0).all()
            continue
        mask, bias = mask_and_bias(torch.tensor([l - 1], device="cuda"), l, m, int(pre[i]) if pre is not None else 0, slopes)
        want, _, bound, _ = reference(q[i:i + 1].reshape(1, hq, d), c.k[i], c.v[i], mask, m.get("cap", 0.0), bias)
        close(out[i].view(1, hq, d), want, bound, (i, l))
    assert hyp.hyp_device_wait_status() == 0


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("m", MODS)
@pytest.mark.parametrize("lens,new", [([37, 5, 64], [37, 2, 20]), ([300, 129, 1, 64], [300, 65, 1, 0]), ([70, 257, 128], [1, 130, 128])])
def test_prefill_mod(heads, m, lens, new):
    hq, hkv, d = heads
    c = Cache(lens, hkv, d, seed=hq + len(lens))
    rows = sum(new)
    q = queries(rows + 3, hq, d, seed=6)                    # three rows behind the last sequence
    cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    ctx = torch.tensor([l - r for l, r in zip(lens, new)], dtype=torch.int32, device="cuda")
    mod, slopes, pre = make_mod(m, hq, len(lens))
    out = torch.full((rows + 3, hq * d), 7.0, dtype=torch.float16, device="cuda")
    hyp.hyp_op_attn_prefill_mod(heads, mod, q, c.pool, c.table, cu, ctx, out)
    torch.cuda.synchronize()
    at = 0
    for i, (l, r) in enumerate(zip(lens, new)):
        if r == 0:
            continue
        pos = torch.arange(l - r, l, device="cuda")
        mask, bias = mask_and_bias(pos, l, m, int(pre[i]) if pre is not None else 0, slopes)
        want, _, bound, _ = reference(q[at:at + r].reshape(r, hq, d), c.k[i], c.v[i], mask, m.get("cap", 0.0), bias)
        close(out[at:at + r].view(r, hq, d), want, bound, (i, l, r))
        at += r
    assert (out[rows:] == 7.0).all()
    assert hyp.hyp_device_wait_status() == 0


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (40, 10, 128)])
@pytest.mark.parametrize("m", [dict(window=16), dict(window=16, prefix=3), dict(window=70, cap=9.0, slopes=True), dict()])
@pytest.mark.parametrize("ctx", [100, 40, 3000])
def test_prefill_mod_where_the_table_is_too_short(heads, m, ctx):
    """Rows whose positions lie behind the last key that the table can name: those that see some of it get what they see, those
    that see nothing zeros."""
    hq, hkv, d = heads
    have, rows = 64, 200
    c = Cache([have], hkv, d, seed=51, extra=0)
    q = queries(rows, hq, d, seed=52)
    mod, slopes, pre = make_mod(m, hq, 1)
    out = torch.full((rows, hq * d), 7.0, dtype=torch.float16, device="cuda")
    hyp.hyp_op_attn_prefill_mod(heads, mod, q, c.pool, c.table, torch.tensor([0, rows], dtype=torch.int32, device="cuda"),
                                torch.tensor([ctx], dtype=torch.int32, device="cuda"), out)
    torch.cuda.synchronize()
    mask, bias = mask_and_bias(torch.arange(ctx, ctx + rows, device="cuda"), have, m, int(pre[0]) if pre is not None else 0, slopes)
    want, _, bound, _ = reference(q.reshape(rows, hq, d), c.k[0], c.v[0], mask, m.get("cap", 0.0), bias)
    close(out.view(rows, hq, d), want, bound, ctx)
    assert (out[~mask.any(1)] == 0).all()
    assert hyp.hyp_device_wait_status() == 0


@pytest.mark.parametrize("heads", [(8, 2, 128), (3, 3, 64)])
@pytest.mark.parametrize("far", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30, 4000])
def test_lengths_far_beyond_the_table(heads, far):
    """A length that the table cannot hold counts as the table's own, up to the largest 32-bit one."""
    hq, hkv, d = heads
    have = 80
    c = Cache([have, have], hkv, d, seed=53, extra=0)
    q = queries(2, hq, d, seed=54)
    far_ctx, ctx = (torch.full((2,), x, dtype=torch.int32, device="cuda") for x in (far, have - 1))
    one = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    mod = hyp.AttnMod(softcap=20.0, window=33, prefix_lens=far_ctx)
    assert torch.equal(run_decode_mod(c, heads, q, far_ctx, hyp.AttnMod()), run_decode_mod(c, heads, q, ctx, hyp.AttnMod()))
    assert torch.equal(run_decode_mod(c, heads, q, far_ctx, mod), run_decode_mod(c, heads, q, ctx, mod))
    w1, w2 = torch.zeros(2, hkv, have, device="cuda"), torch.zeros(2, hkv, have, device="cuda")
    assert torch.equal(run_scored(c, heads, q, far_ctx, 1.0, None, w1), run_scored(c, heads, q, ctx, 1.0, None, w2)) and torch.equal(w1, w2)
    pt = c.table[:1].contiguous()
    assert torch.equal(run_shared(heads, q, c, one, pt, far_ctx[:1], c.table, far_ctx), run_shared(heads, q, c, one, pt, ctx[:1] + 1, c.table, ctx))
    kept, new_lens = torch.empty(2, hkv, 20, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    w1.copy_(torch.rand(w1.shape, generator=gen(55), device="cuda"))
    dst, dtab = torch.zeros(4, 2, hkv, 16, d, dtype=torch.float16, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    hyp.hyp_op_kv_evict(heads, c.pool, c.table, far_ctx, w1, 20, 2, 3, dst, dtab, kept, new_lens, w2)
    assert new_lens.tolist() == [20, 20]
    for b in range(2):
        for h in range(hkv):
            assert kept[b, h].tolist() == evict_reference(w1[b, h].tolist(), have, 20, 2, 3)
    # a prompt's rows behind everything: all keys, or none with a window
    rows = queries(40, hq, d, seed=56)
    cu = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    want, _, bound, _ = reference(rows.reshape(40, hq, d), c.k[0], c.v[0], torch.ones(40, have, dtype=torch.bool, device="cuda"))
    for window in (0, 50):
        out = torch.full((40, hq * d), 7.0, dtype=torch.float16, device="cuda")
        hyp.hyp_op_attn_prefill_mod(heads, hyp.AttnMod(window=window), rows, c.pool, pt, cu, far_ctx[:1], out)
        torch.cuda.synchronize()
        if window:
            assert (out == 0).all()
        else:
            close(out.view(40, hq, d), want, bound, far)
    assert hyp.hyp_device_wait_status() == 0


def test_prefill_mod_without_modification_agrees_with_plain_prefill():
    heads, lens, new = (40, 10, 128), [700, 128, 257], [700, 128, 130]
    c = Cache(lens, 10, 128, seed=3)
    q = torch.randn(sum(new), 40 * 128, generator=gen(1), device="cuda").half()
    cu = torch.tensor([0, 700, 828, 958], dtype=torch.int32, device="cuda")
    ctx = torch.tensor([0, 0, 127], dtype=torch.int32, device="cuda")
    pool = torch.nan_to_num(c.pool)                         # the plain operator wants finite pages
    a, b = torch.empty_like(q), torch.empty_like(q)
    hyp.hyp_op_attn_prefill_mod(heads, hyp.AttnMod(), q, pool, c.table, cu, ctx, a)
    hyp.hyp_op_attn_prefill(heads, q, pool, c.table, cu, ctx, b)
    torch.cuda.synchronize()
    assert (a.float() - b.float()).abs().max() < 2e-2       # the plain operator's own tolerance


def run_scored(c, heads, q, ctx, decay, w_in, w_out):
    out = torch.full((q.shape[0], heads[0] * heads[2]), 7.0, dtype=torch.float16, device="cuda")
    scratch = bytes_of(hyp.hyp_op_attn_scored_scratch_bytes(heads, q.shape[0], c.table.shape[1]))
    hyp.hyp_op_attn_decode_scored(heads, q, c.pool, c.table, ctx, decay, w_in, w_out, scratch, out)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("form", ["apart", "same", "fresh"])
def test_decode_scored(heads, form):
    hq, hkv, d = heads
    lens = LENS + [1500, 0]
    c = Cache(lens[:-1], hkv, d, seed=hq + 2 * d)
    c.table = torch.cat([c.table, torch.zeros_like(c.table[:1])])
    n, width = len(lens), 16 * c.table.shape[1] + 5
    q = queries(n, hq, d, seed=7)
    ctx = torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda")
    w = torch.rand(n, hkv, width, generator=gen(8), device="cuda")
    for i, l in enumerate(lens):
        w[i, :, max(0, l - 1):] = float("nan")             # the new token's slot and what lies behind is not read
    w_in = None if form == "fresh" else w
    w_out = w.clone() if form == "same" else torch.full_like(w, 9.0)
    if form == "same":
        w_in = w_out
    out = run_scored(c, heads, q, ctx, 0.5, w_in, w_out)
    for i, l in enumerate(lens):
        if l == 0:
            assert (out[i] == 0).all()
        else:
            want, p, bound, serr = reference(q[i:i + 1].reshape(1, hq, d), c.k[i], c.v[i], torch.ones(1, l, dtype=torch.bool, device="cuda"))
            close(out[i].view(1, hq, d), want, bound, (i, l))
            got = p[:, 0].view(hkv, hq // hkv, l).sum(1)
            if w_in is not None:
                got[:, :l - 1] += 0.5 * w[i, :, :l - 1].double()
            err = (w_out[i, :, :l].double() - got).abs()
            assert (err <= (2 * serr + 2.0 ** -20) * got).all(), (i, l)
        behind = w_out[i, :, l:]
        assert torch.isnan(behind).all() if form == "same" else (behind == 9.0).all()


@pytest.mark.parametrize("heads", [(3, 3, 64), (1, 1, 128), (1, 1, 64), (5, 5, 128), (25, 25, 64)])
@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("pages", [19, 20, 28, 33])
def test_decode_scored_of_odd_batches_and_heads(heads, n, pages):
    """Odd sequences, heads and splits: the partial rows in front of the scores do not fill whole 16-byte pieces."""
    hq, hkv, d = heads
    lens = [16 * pages - 7, 1, 100][:n]
    c = Cache(lens, hkv, d, seed=pages, extra=0)
    assert c.table.shape[1] == pages
    q = queries(n, hq, d, seed=33)
    ctx = torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda")
    w = torch.rand(n, hkv, 16 * pages, generator=gen(34), device="cuda")
    before = w.double()
    out = run_scored(c, heads, q, ctx, 0.75, w, w)
    for i, l in enumerate(lens):
        want, p, bound, serr = reference(q[i:i + 1].reshape(1, hq, d), c.k[i], c.v[i], torch.ones(1, l, dtype=torch.bool, device="cuda"))
        close(out[i].view(1, hq, d), want, bound, (i, l))
        got = p[:, 0].view(hkv, hq // hkv, l).sum(1)
        got[:, :l - 1] += 0.75 * before[i, :, :l - 1]
        assert ((w[i, :, :l].double() - got).abs() <= (2 * serr + 2.0 ** -20) * got).all(), (i, l)
        assert torch.equal(w[i, :, l:].double(), before[i, :, l:])
    assert hyp.hyp_device_wait_status() == 0


def evict_reference(w, t, keep, sink, recent):
    """Kept slots of one head, in order."""
    if t <= keep:
        return list(range(t))
    key = [-math.inf if math.isnan(x) else x for x in w[:t]]
    fixed = [j for j in range(t) if j < sink or j >= t - recent]
    rest = [j for j in range(t) if not (j < sink or j >= t - recent)]
    rest.sort(key=lambda j: (-key[j], j))
    return sorted(fixed + rest[:keep - sink - recent])


EVICT = [  # lens, keep, sink, recent
    ([100, 7, 40, 41, 333], 40, 4, 10), ([100, 64, 17], 16, 0, 0), ([100, 64, 17], 16, 16, 0), ([100, 64, 17], 16, 0, 16),
    ([100, 64, 17], 16, 6, 10), ([33, 1, 0], 1, 0, 0), ([1025, 2049, 5000], 1000, 1, 7), ([70, 3000], 2999, 2, 2990), ([500, 90], 600, 4, 10),
]


@pytest.mark.parametrize("heads", [(4, 2, 64), (40, 10, 128)])
@pytest.mark.parametrize("lens,keep,sink,recent", EVICT)
@pytest.mark.parametrize("place", ["own pool", "same pool", "in place"])
def test_kv_evict(heads, lens, keep, sink, recent, place):
    hq, hkv, d = heads
    n, kw = len(lens), (keep + 15) // 16
    c = Cache(lens, hkv, d, seed=keep + d, spare=n * kw, extra=1 if place != "in place" else max(1, kw))
    width = 16 * c.table.shape[1]
    w = torch.rand(n, hkv, width, generator=gen(9), device="cuda")
    w = torch.where(w < 0.3, torch.zeros_like(w), w)                  # many ties at zero, of both signs
    w[:, :, 1::5] *= -1.0
    w[:, :, 3::7] = float("nan")
    w[:, :, 5::11] = float("inf")
    w[:, :, 6::13] = float("-inf")
    w[:, :, 8::9] = 0.75                                              # ties in the middle
    cached = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kept = torch.full((n, hkv, keep), 99, dtype=torch.int32, device="cuda")
    new_lens = torch.full((n,), 99, dtype=torch.int32, device="cuda")
    before = w.cpu()
    pool0 = c.pool.clone()
    if place == "in place":
        dst, dtab, wout = c.pool, c.table, w
    else:
        wout = torch.full((n, hkv, keep + 3), 5.0, device="cuda")
        if place == "same pool":
            dst, dtab = c.pool, c.spare.view(n, kw).contiguous().cuda()
        else:
            dst = torch.full((n * kw, 2, hkv, 16, d), 3.0, dtype=torch.float16, device="cuda")
            dtab = torch.from_numpy(np.random.default_rng(1).permutation(n * kw).astype(np.int32)).view(n, kw).cuda()
    hyp.hyp_op_kv_evict(heads, c.pool, c.table, cached, w, keep, sink, recent, dst, dtab, kept, new_lens, wout)
    torch.cuda.synchronize()
    assert new_lens.tolist() == [min(l, keep) for l in lens]
    for b, t in enumerate(lens):
        m = min(t, keep)
        for h in range(hkv):
            want = evict_reference(before[b, h].tolist(), t, keep, sink, recent)
            assert kept[b, h].tolist() == want + [-1] * (keep - m), (b, h)
            assert torch.equal(torch.nan_to_num(wout[b, h, :m].cpu(), nan=123.0), torch.nan_to_num(before[b, h, want], nan=123.0)), (b, h)
            idx = torch.tensor(want, device="cuda", dtype=torch.long)
            for kind, x in ((0, c.k[b]), (1, c.v[b])):
                assert torch.equal(get(dst, dtab[b], kind, m)[:, h], x[idx, h]), (b, h, kind)
        if place == "in place":                                       # behind the new length: as it was
            assert torch.equal(torch.nan_to_num(wout[b, :, m:].cpu(), nan=123.0), torch.nan_to_num(before[b, :, m:], nan=123.0))
        else:
            assert (wout[b, :, m:] == 5.0).all()
    if place == "own pool":
        assert torch.equal(torch.nan_to_num(c.pool, nan=123.0), torch.nan_to_num(pool0, nan=123.0))
        used = torch.zeros(n * kw * 16, dtype=torch.bool, device="cuda")
        for b, t in enumerate(lens):
            s = torch.arange(min(t, keep), device="cuda")
            used[dtab[b][s // 16].long() * 16 + s % 16] = True
        assert (dst.permute(0, 3, 1, 2, 4).reshape(n * kw * 16, -1)[~used] == 3.0).all()


@pytest.mark.parametrize("place", ["own pool", "in place"])
def test_kv_evict_beyond_the_register_range(place):
    """More candidates than the selection keeps in registers (32768)."""
    heads, t, keep, sink, recent = (1, 1, 64), 40001, 20011, 5, 1000
    c = Cache([t, 100], 1, 64, seed=4)
    w = (torch.rand(2, 1, 16 * c.table.shape[1], generator=gen(10), device="cuda") * 4096).floor() / 64     # ties
    before = w.cpu()
    kept = torch.empty(2, 1, keep, dtype=torch.int32, device="cuda")
    new_lens = torch.empty(2, dtype=torch.int32, device="cuda")
    kw = (keep + 15) // 16
    if place == "in place":
        dst, dtab, wout = c.pool, c.table, w
    else:
        dst = torch.zeros(2 * kw, 2, 1, 16, 64, dtype=torch.float16, device="cuda")
        dtab, wout = torch.arange(2 * kw, dtype=torch.int32, device="cuda").view(2, kw), torch.zeros(2, 1, keep, device="cuda")
    hyp.hyp_op_kv_evict(heads, c.pool, c.table, torch.tensor([t, 100], dtype=torch.int32, device="cuda"), w, keep, sink, recent, dst, dtab,
                        kept, new_lens, wout)
    torch.cuda.synchronize()
    want = evict_reference(before[0, 0].tolist(), t, keep, sink, recent)
    assert kept[0, 0].tolist() == want and new_lens.tolist() == [keep, 100]
    assert torch.equal(wout[0, 0, :keep].cpu(), before[0, 0, want])
    idx = torch.tensor(want, device="cuda")
    for kind, x in ((0, c.k[0]), (1, c.v[0])):
        assert torch.equal(get(dst, dtab[0], kind, keep), x[idx])


@pytest.mark.parametrize("keep", [40, 700])
@pytest.mark.parametrize("between", [False, True])
def test_a_decode_step_behind_an_eviction_at_every_overlap_level(keep, between):
    """The step takes its lengths from the eviction before it and appends to the rows that this one moved, also where kernels may be
    launched early and a projection stands in between."""
    heads, n, longest = (8, 2, 128), 24, 1600
    hq, hkv, d = heads
    lens = [longest - 13 * i for i in range(n)]
    c = Cache(lens, hkv, d, seed=41)
    w0 = torch.rand(n, hkv, 16 * c.table.shape[1], generator=gen(42), device="cuda")
    cached = torch.tensor(lens, dtype=torch.int32, device="cuda")
    qkv = torch.randn(n, (hq + 2 * hkv) * d, generator=gen(43), device="cuda")
    angle = torch.arange(longest + 1, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(d // 2, device="cuda") * 2 / d)
    rope = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
    a, wt = torch.randn(4, 512, generator=gen(44), device="cuda").half(), torch.randn(1024, 512, generator=gen(45), device="cuda").bfloat16()
    packed, prod = hyp.hyp_op_pack_weight(wt, 1024, False, f16=True), torch.empty(4, 1024, device="cuda")
    pool0 = c.pool.clone()
    results = []
    for level in (0, 2, 3, 3, 3):
        c.pool.copy_(pool0)
        w, kept = w0.clone(), torch.empty(n, hkv, keep, dtype=torch.int32, device="cuda")
        new_lens = torch.full((n,), 5, dtype=torch.int32, device="cuda")
        out = torch.empty(n, hq * d, dtype=torch.float16, device="cuda")
        torch.cuda.synchronize()
        hyp.hyp_tune(hyp.HYP_TUNE_PDL, level)
        try:
            hyp.hyp_op_kv_evict(heads, c.pool, c.table, cached, w, keep, 4, 16, c.pool, c.table, kept, new_lens, w)
            if between:
                hyp.hyp_op_gemm_f16(a, packed, 1024, hyp.HYP_EPI_STORE_F32, prod)
            hyp.hyp_op_attn_decode_step(heads, qkv, c.pool, c.table, new_lens, rope, 0, out)
        finally:
            hyp.hyp_tune(hyp.HYP_TUNE_PDL, 2)
        torch.cuda.synchronize()
        assert torch.isfinite(out.float()).all()
        results.append((out, torch.nan_to_num(c.pool, nan=123.0), new_lens))
    for r in results[1:]:
        assert all(torch.equal(x, y) for x, y in zip(results[0], r))
    assert results[0][2].tolist() == [keep] * n


def run_shared(heads, q, c, cu, ptable, plens, own_table, ctx):
    out = torch.full((q.shape[0], heads[0] * heads[2]), 7.0, dtype=torch.float16, device="cuda")
    scratch = bytes_of(hyp.hyp_op_attn_shared_scratch_bytes(heads, q.shape[0], plens.shape[0], ptable.shape[1], own_table.shape[1]))
    hyp.hyp_op_attn_decode_shared(heads, q, c.pool, cu, ptable, plens, own_table, ctx, scratch, out)
    torch.cuda.synchronize()
    return out


SHARED = [  # prefix lengths, group sizes, own lengths (cycled)
    ([100], [3], [1, 17, 24]), ([64], [1], [5]), ([1000], [40], [1, 16, 33, 100, 0]), ([0, 129, 1, 500], [2, 0, 5, 18], [7, 0, 1, 48]),
    ([2000, 63], [130, 3], [1, 20]), ([0], [4], [0, 3, 0, 1]),
]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("prefix,sizes,own_lens", SHARED)
def test_decode_shared(heads, prefix, sizes, own_lens):
    hq, hkv, d = heads
    n = sum(sizes)
    own = [own_lens[i % len(own_lens)] for i in range(n)]
    c = Cache(prefix + own, hkv, d, seed=n + d)
    ng = len(prefix)
    pt, ot = c.table[:ng].contiguous(), c.table[ng:, :max(1, (max(own) + 15) // 16 + 1)].contiguous()
    q = queries(n, hq, d, seed=11)
    cu = torch.tensor([sum(sizes[:i]) for i in range(ng + 1)], dtype=torch.int32, device="cuda")
    ctx = torch.tensor([o - 1 for o in own], dtype=torch.int32, device="cuda")
    out = run_shared(heads, q, c, cu, pt, torch.tensor(prefix, dtype=torch.int32, device="cuda"), ot, ctx)
    group = [g for g, s in enumerate(sizes) for _ in range(s)]
    for i in range(n):
        k = torch.cat([c.k[group[i]], c.k[ng + i]])
        v = torch.cat([c.v[group[i]], c.v[ng + i]])
        if k.shape[0] == 0:
            assert (out[i] == 0).all()
            continue
        want, _, bound, _ = reference(q[i:i + 1].reshape(1, hq, d), k, v, torch.ones(1, k.shape[0], dtype=torch.bool, device="cuda"))
        close(out[i].view(1, hq, d), want, bound, (i, own[i]))
    assert hyp.hyp_device_wait_status() == 0


def test_large_scores_and_long_tails():
    """Scores far apart (weights that underflow), and a maximum that grows along the keys, through every operator."""
    heads = (8, 2, 128)
    c = Cache([700], 2, 128, seed=2)
    q = queries(1, 8, 128, seed=3, std=12.0)
    scale = torch.linspace(0.02, 1.0, 700, device="cuda").half()[:, None, None]
    c.k[0] = (c.k[0] * scale).contiguous()
    for p in range(44):
        put(c.pool, int(c.table[0, p]), 0, c.k[0][16 * p:16 * p + 16])
    ctx = torch.tensor([699], dtype=torch.int32, device="cuda")
    mask = torch.ones(1, 700, dtype=torch.bool, device="cuda")
    want, p, bound, serr = reference(q.reshape(1, 8, 128), c.k[0], c.v[0], mask)
    close(run_decode_mod(c, heads, q, ctx, hyp.AttnMod()).view(1, 8, 128), want, bound, "decode")
    w = torch.zeros(1, 2, 16 * c.table.shape[1], device="cuda")
    close(run_scored(c, heads, q, ctx, 1.0, None, w).view(1, 8, 128), want, bound, "scored")
    got = p[:, 0].view(2, 4, 700).sum(1)
    assert ((w[0, :, :700].double() - got).abs() <= (2 * serr + 2.0 ** -20) * got + 2.0 ** -126).all()
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    out = torch.empty(1, 8 * 128, dtype=torch.float16, device="cuda")
    hyp.hyp_op_attn_prefill_mod(heads, hyp.AttnMod(), q, c.pool, c.table, one, ctx, out)
    close(out.view(1, 8, 128), want, bound, "prefill")
    none = torch.tensor([-1], dtype=torch.int32, device="cuda")
    out = run_shared(heads, q, c, one, c.table, torch.tensor([700], dtype=torch.int32, device="cuda"), c.table, none)
    close(out.view(1, 8, 128), want, bound, "shared")


def calls(seed, n=3, longest=200):
    """(name, input, call, outputs) of every operator on a batch, for the tests of streams, graphs and repeats: short contexts
    (one launch each), longer ones (splits that join in a cluster), many or long ones (a second launch joins; shared
    prefixes on row tiles)."""
    heads = (8, 2, 128)
    lens = [longest] + [1 + (37 * (i + 1)) % longest for i in range(n - 1)]
    c = Cache(lens, 2, 128, seed=seed)
    q = queries(n, 8, 128, seed=seed + 1)
    ctx = torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda")
    width = 16 * c.table.shape[1]
    w = torch.rand(n, 2, width, generator=gen(seed + 2), device="cuda")
    wo = torch.zeros_like(w)
    outs = [torch.zeros(n, 8 * 128, dtype=torch.float16, device="cuda") for _ in range(4)]
    mod = hyp.AttnMod(softcap=20.0, window=70)
    pages = c.table.shape[1]
    s1 = bytes_of(hyp.hyp_op_attn_mod_scratch_bytes(heads, n, pages))
    s2 = bytes_of(hyp.hyp_op_attn_scored_scratch_bytes(heads, n, pages))
    s3 = bytes_of(hyp.hyp_op_attn_shared_scratch_bytes(heads, n, 1, pages, pages))
    cu1 = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    cun = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    pl, pt = torch.tensor([longest], dtype=torch.int32, device="cuda"), c.table[:1].contiguous()
    kept = torch.zeros(n, 2, 32, dtype=torch.int32, device="cuda")
    nl = torch.zeros(n, dtype=torch.int32, device="cuda")
    cached = torch.tensor(lens, dtype=torch.int32, device="cuda")
    dst = torch.zeros(2 * n, 2, 2, 16, 128, dtype=torch.float16, device="cuda")
    dt = torch.arange(2 * n, dtype=torch.int32, device="cuda").view(n, 2)
    we = torch.zeros(n, 2, 32, device="cuda")
    return [
        ("decode_mod", q, lambda st=None: hyp.hyp_op_attn_decode_mod(heads, mod, q, c.pool, c.table, ctx, s1, outs[0], st), [outs[0]]),
        ("prefill_mod", q, lambda st=None: hyp.hyp_op_attn_prefill_mod(heads, mod, q, c.pool, c.table, cun, ctx, outs[1], st), [outs[1]]),
        ("scored", q, lambda st=None: hyp.hyp_op_attn_decode_scored(heads, q, c.pool, c.table, ctx, 1.0, w, wo, s2, outs[2], st), [outs[2], wo]),
        ("shared", q, lambda st=None: hyp.hyp_op_attn_decode_shared(heads, q, c.pool, cu1, pt, pl, c.table, ctx, s3, outs[3], st), [outs[3]]),
        ("evict", w, lambda st=None: hyp.hyp_op_kv_evict(heads, c.pool, c.table, cached, w, 32, 2, 5, dst, dt, kept, nl, we, st), [kept, nl, we, dst]),
    ]


BATCHES = [(3, 200), (5, 900), (40, 1500), (2, 9000)]


@pytest.mark.parametrize("n,longest", BATCHES)
def test_graph_replay_takes_new_inputs_and_results_repeat_bit_for_bit(n, longest):
    for i, (name, inp, call, outs) in enumerate(calls(31, n, longest)):
        call()
        torch.cuda.synchronize()
        first = [o.clone() for o in outs]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
            call()
        for o in outs:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs)), name
        fresh = torch.rand(inp.shape, generator=gen(100 + i), device="cuda").to(inp.dtype)
        inp.copy_(fresh)
        g.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in outs]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs)), name
        assert not all(torch.equal(a, b) for a, b in zip(first, outs)), name


@pytest.mark.parametrize("n,longest", BATCHES)
def test_calls_follow_their_stream(n, longest):
    """The inputs are written late on a side stream; the call on that stream has to see them."""
    for i, (name, inp, call, outs) in enumerate(calls(47, n, longest)):
        fresh = torch.rand(inp.shape, generator=gen(200 + i), device="cuda").to(inp.dtype)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        big = torch.randn(4096, 4096, device="cuda")
        with torch.cuda.stream(st):
            for _ in range(4):
                big = big @ big * 1e-3
            inp.copy_(fresh)
            call(st)
        st.synchronize()
        late = [o.clone() for o in outs]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(late, outs)), name


def test_generation_with_a_bounded_cache():
    """The operators as a server would chain them: two sequences grow token by token, every step sums the weights; when the
    cache reaches its limit it is cut in place and generation goes on from the shorter cache.  Every step is held against
    the same run in 64 bits on the rows that are really in the cache."""
    heads, limit, keep, sink, recent = (4, 2, 64), 48, 20, 2, 6
    hq, hkv, d = heads
    lens = [30, 41]
    c = Cache(lens, hkv, d, seed=12, spare=8, extra=0)
    table = torch.zeros(2, 4, dtype=torch.int32)
    table[:, :3] = c.table.cpu()[:, :3]
    spare = c.spare.tolist()
    for b, l in enumerate(lens):
        for p in range((l + 15) // 16, 4):
            table[b, p] = spare.pop()
    table = table.cuda()
    ks, vs = [list(x.unbind(0)) for x in c.k], [list(x.unbind(0)) for x in c.v]
    kept_k = [[[ks[b][j][h] for j in range(lens[b])] for h in range(hkv)] for b in range(2)]
    kept_v = [[[vs[b][j][h] for j in range(lens[b])] for h in range(hkv)] for b in range(2)]
    w = torch.zeros(2, hkv, 64, device="cuda")
    wref = [[[0.0] * lens[b] for _ in range(hkv)] for b in range(2)]
    n = list(lens)
    g = gen(77)
    cuts = 0
    for step in range(25):
        newk, newv = torch.randn(2, 2, hkv, d, generator=g, device="cuda").half().unbind(0)
        q = (torch.randn(2, hq * d, generator=g, device="cuda") * 1.5).half()
        for b in range(2):
            slot = n[b] % 16
            page = int(table[b, n[b] // 16])
            for kind, x in ((0, newk[b]), (1, newv[b])):
                pos = torch.arange(d // 8, device="cuda") ^ (slot & 7)
                c.pool.view(*c.pool.shape[:4], d // 8, 8)[page, kind, :, slot, pos] = x.view(hkv, d // 8, 8)
            for h in range(hkv):
                kept_k[b][h].append(newk[b][h]); kept_v[b][h].append(newv[b][h])
                wref[b][h].append(0.0)
        ctx = torch.tensor(n, dtype=torch.int32, device="cuda")
        cc = type("C", (), {"pool": c.pool, "table": table})
        out = run_scored(cc, heads, q, ctx, 1.0, w, w)
        n = [x + 1 for x in n]
        for b in range(2):
            for h in range(hkv):
                k, v = torch.stack(kept_k[b][h])[:, None], torch.stack(kept_v[b][h])[:, None]
                qq = q[b].view(hkv, hq // hkv, d)[h][None]
                want, p, bound, serr = reference(qq, k, v, torch.ones(1, n[b], dtype=torch.bool, device="cuda"))
                close(out[b].view(hkv, hq // hkv, d)[h][None], want, bound, (step, b, h))
                wref[b][h] = [x + y for x, y in zip(wref[b][h], p[:, 0].sum(0).tolist())]
                err = (w[b, h, :n[b]].double().cpu() - torch.tensor(wref[b][h], dtype=torch.float64)).abs().max()
                assert err < 1e-4, (step, b, h)
        if max(n) >= limit:
            cuts += 1
            kept = torch.empty(2, hkv, keep, dtype=torch.int32, device="cuda")
            new_lens = torch.empty(2, dtype=torch.int32, device="cuda")
            hyp.hyp_op_kv_evict(heads, c.pool, table, torch.tensor(n, dtype=torch.int32, device="cuda"), w, keep, sink, recent, c.pool,
                                table, kept, new_lens, w)
            torch.cuda.synchronize()
            for b in range(2):
                for h in range(hkv):
                    idx = [j for j in kept[b, h].tolist() if j >= 0]
                    kept_k[b][h] = [kept_k[b][h][j] for j in idx]
                    kept_v[b][h] = [kept_v[b][h][j] for j in idx]
                    wref[b][h] = [wref[b][h][j] for j in idx]
                    assert idx[:sink] == list(range(sink)) and idx[-recent:] == list(range(n[b] - recent, n[b]))
            n = new_lens.tolist()
    assert cuts >= 1


def test_scored_then_shared_and_modified_calls_agree_where_they_mean_the_same():
    """With nothing shared, nothing capped and fresh sums, the three decode calls are plain decode attention."""
    heads, lens = (40, 10, 128), [1024, 500, 3]
    c = Cache(lens, 10, 128, seed=13)
    q = queries(3, 40, 128, seed=14)
    ctx = torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda")
    a = run_decode_mod(c, heads, q, ctx, hyp.AttnMod())
    b = run_scored(c, heads, q, ctx, 1.0, None, torch.zeros(3, 10, 16 * c.table.shape[1], device="cuda"))
    cu = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    s = run_shared(heads, q, c, cu, c.table[:1].contiguous(), torch.zeros(1, dtype=torch.int32, device="cuda"), c.table, ctx)
    for i, l in enumerate(lens):
        want, _, bound, _ = reference(q[i:i + 1].reshape(1, 40, 128), c.k[i], c.v[i], torch.ones(1, l, dtype=torch.bool, device="cuda"))
        for o in (a, b, s):
            close(o[i].view(1, 40, 128), want, bound, (i, l))


def test_a_long_cache_far_into_a_large_pool():
    """Page ids whose rows lie more than 2^32 elements behind the pool's start."""
    heads = (8, 8, 128)
    page = 2 * 8 * 16 * 128
    n_pages = 2 ** 32 // page + 40
    c = Cache([300], 8, 128, seed=15)
    pool = torch.empty(n_pages, 2, 8, 16, 128, dtype=torch.float16, device="cuda")
    far = n_pages - 30
    table = c.table.clone()
    for p in range(19):
        pool[far + p] = c.pool[int(c.table[0, p])]
        table[0, p] = far + p
    c.pool, c.table = pool, table
    q = queries(1, 8, 128, seed=16)
    ctx = torch.tensor([299], dtype=torch.int32, device="cuda")
    want, _, bound, _ = reference(q.reshape(1, 8, 128), c.k[0], c.v[0], torch.ones(1, 300, dtype=torch.bool, device="cuda"))
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    w = torch.zeros(1, 8, 16 * table.shape[1], device="cuda")
    close(run_decode_mod(c, heads, q, ctx, hyp.AttnMod()).view(1, 8, 128), want, bound, "decode")
    close(run_scored(c, heads, q, ctx, 1.0, None, w).view(1, 8, 128), want, bound, "scored")
    out = torch.empty(1, 1024, dtype=torch.float16, device="cuda")
    hyp.hyp_op_attn_prefill_mod(heads, hyp.AttnMod(), q, pool, table, one, ctx, out)
    close(out.view(1, 8, 128), want, bound, "prefill")
    none = torch.tensor([-1], dtype=torch.int32, device="cuda")
    close(run_shared(heads, q, c, one, table, torch.tensor([300], dtype=torch.int32, device="cuda"), table, none).view(1, 8, 128), want,
          bound, "shared")
    kept = torch.empty(1, 8, 32, dtype=torch.int32, device="cuda")
    nl = torch.empty(1, dtype=torch.int32, device="cuda")
    hyp.hyp_op_kv_evict(heads, pool, table, torch.tensor([300], dtype=torch.int32, device="cuda"), w, 32, 4, 8, pool, table, kept, nl, w)
    torch.cuda.synchronize()
    for h in range(8):
        assert torch.equal(get(pool, table[0], 0, 32)[:, h], c.k[0][kept[0, h].long(), h])


def test_steep_and_negative_distance_slopes_on_long_prompts():
    """Slopes that move the reference maximum from tile to tile in either direction, with and without a cap."""
    heads, l = (4, 2, 128), 1500
    c = Cache([l], 2, 128, seed=21)
    q = queries(300, 4, 128, seed=22)
    cu = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    ctx = torch.tensor([l - 300], dtype=torch.int32, device="cuda")
    pos = torch.arange(l - 300, l, device="cuda")
    for cap in (0.0, 4.0):
        slopes = torch.tensor([3.0, 0.01, -0.02, 0.0], device="cuda")
        mask, bias = mask_and_bias(pos, l, dict(prefix=200), 200, slopes)
        mod = hyp.AttnMod(softcap=cap, slopes=slopes, prefix_lens=torch.tensor([200], dtype=torch.int32, device="cuda"))
        out = torch.empty(300, 512, dtype=torch.float16, device="cuda")
        hyp.hyp_op_attn_prefill_mod(heads, mod, q, c.pool, c.table, cu, ctx, out)
        torch.cuda.synchronize()
        want, _, bound, _ = reference(q.reshape(300, 4, 128), c.k[0], c.v[0], mask, cap, bias)
        close(out.view(300, 4, 128), want, bound, cap)


def test_scores_beyond_the_caps_polynomial():
    """Scores from far below to far above the cap in one row."""
    heads, l = (4, 2, 128), 400
    c = Cache([l], 2, 128, seed=23)
    q = queries(l, 4, 128, seed=24, std=15.0)
    out = torch.empty(l, 512, dtype=torch.float16, device="cuda")
    cu = torch.tensor([0, l], dtype=torch.int32, device="cuda")
    hyp.hyp_op_attn_prefill_mod(heads, hyp.AttnMod(softcap=10.0), q, c.pool, c.table, cu, torch.zeros(1, dtype=torch.int32, device="cuda"), out)
    torch.cuda.synchronize()
    mask = torch.tril(torch.ones(l, l, dtype=torch.bool, device="cuda"))
    want, _, bound, _ = reference(q.reshape(l, 4, 128), c.k[0], c.v[0], mask, 10.0)
    close(out.view(l, 4, 128), want, bound, "cap")


@pytest.mark.parametrize("n,ng", [(70, 40), (256, 3), (9, 9)])
def test_many_groups_and_large_groups(n, ng):
    """More groups than a warp has lanes (a fixed number of shares each), more row tiles than fit at once."""
    heads = (40, 10, 128)
    rng = np.random.default_rng(n)
    prefix = [int(x) for x in rng.integers(0, 700, ng)]
    cuts = np.sort(rng.integers(0, n + 1, ng - 1)).tolist()
    cu = [0] + cuts + [n]
    own = [int(x) for x in rng.integers(0, 40, n)]
    c = Cache(prefix + own, 10, 128, seed=n)
    pt, ot = c.table[:ng].contiguous(), c.table[ng:, :4].contiguous()
    q = queries(n, 40, 128, seed=25)
    out = run_shared(heads, q, c, torch.tensor(cu, dtype=torch.int32, device="cuda"), pt, torch.tensor(prefix, dtype=torch.int32, device="cuda"), ot,
                     torch.tensor([o - 1 for o in own], dtype=torch.int32, device="cuda"))
    for i in range(n):
        g = sum(1 for x in cu[1:] if x <= i)
        k, v = torch.cat([c.k[g], c.k[ng + i]]), torch.cat([c.v[g], c.v[ng + i]])
        if k.shape[0] == 0:
            assert (out[i] == 0).all()
            continue
        want, _, bound, _ = reference(q[i:i + 1].reshape(1, 40, 128), k, v, torch.ones(1, k.shape[0], dtype=torch.bool, device="cuda"))
        close(out[i].view(1, 40, 128), want, bound, (i, g))
    assert hyp.hyp_device_wait_status() == 0


@pytest.mark.parametrize("cap", [2.0 ** -10, 0.3, 300.0, 2.0 ** 20])
def test_caps_from_the_smallest_to_the_largest(cap):
    """A cap far above the scores leaves them as they are (to fp32 rounding, not to the cap's), a tiny one flattens them."""
    heads, l = (4, 2, 128), 130
    c = Cache([l], 2, 128, seed=26)
    q = queries(l, 4, 128, seed=27)
    mask = torch.tril(torch.ones(l, l, dtype=torch.bool, device="cuda"))
    qq = q.reshape(l, 4, 128)
    want, _, bound, _ = reference(qq, c.k[0], c.v[0], mask, cap)
    if cap > 300.0:
        # the cap's own rounding (2^-20 of it) would hide everything: the bound of the scores as they are, and 2.4e-6 of the
        # largest score |q| |k| / sqrt(D) for the polynomial
        top = qq.double().norm(dim=-1).amax() * c.k[0].double().norm(dim=-1).amax() / math.sqrt(128)
        _, _, bound, _ = reference(qq, c.k[0], c.v[0], mask)
        bound = bound + 2 * 2.4e-6 * top * c.v[0].double().abs().amax()
    mod = hyp.AttnMod(softcap=cap)
    out = torch.empty(l, 512, dtype=torch.float16, device="cuda")
    cu = torch.tensor([0, l], dtype=torch.int32, device="cuda")
    hyp.hyp_op_attn_prefill_mod(list(heads), mod, q, c.pool, c.table, cu, torch.zeros(1, dtype=torch.int32, device="cuda"), out)
    torch.cuda.synchronize()
    close(out.view(l, 4, 128), want, bound, "prefill")
    one = run_decode_mod(c, heads, q[-1:], torch.tensor([l - 1], dtype=torch.int32, device="cuda"), mod)
    close(one.view(1, 4, 128), want[-1:], bound[-1:], "decode")


def test_two_streams_with_a_scratch_each():
    """Calls that may overlap on the GPU, on one cache, each with its own scratch and outputs."""
    a, b = calls(61, 40, 1500), calls(61, 40, 1500)
    alone = []
    for name, inp, call, outs in a:
        call()
        torch.cuda.synchronize()
        alone.append([o.clone() for o in outs])
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for rep in range(5):
        for (_, _, c1, _), (_, _, c2, _) in zip(a, reversed(b)):
            c1(s1)
            c2(s2)
    torch.cuda.synchronize()
    for i in range(len(a)):
        assert all(torch.equal(x, y) for x, y in zip(alone[i], a[i][3])), a[i][0]
        assert all(torch.equal(x, y) for x, y in zip(alone[i], b[i][3])), b[i][0]


@pytest.mark.parametrize("heads", [(8, 2, 128), (40, 10, 128)])
@pytest.mark.parametrize("lens", [[1, 300, 17, 0, 80], [5000, 40, 333], [64] * 50])
def test_tables_much_wider_than_the_sequences(heads, lens):
    """Rows of a table made for long contexts (splits are planned by its width), sequences of any length in it."""
    hq, hkv, d = heads
    c = Cache([max(l, 1) for l in lens], hkv, d, seed=31, extra=700)
    n = len(lens)
    q = queries(n, hq, d, seed=32)
    ctx = torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda")
    w = torch.zeros(n, hkv, 16 * c.table.shape[1], device="cuda")
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    a = run_decode_mod(c, heads, q, ctx, hyp.AttnMod())
    b = run_scored(c, heads, q, ctx, 1.0, None, w)
    s = run_shared(heads, q, c, cu, c.table[:1].contiguous(), torch.zeros(1, dtype=torch.int32, device="cuda"), c.table, ctx)
    for i, l in enumerate(lens):
        if l == 0:
            assert (a[i] == 0).all() and (b[i] == 0).all() and (s[i] == 0).all()
            continue
        want, p, bound, serr = reference(q[i:i + 1].reshape(1, hq, d), c.k[i], c.v[i], torch.ones(1, l, dtype=torch.bool, device="cuda"))
        for o in (a, b, s):
            close(o[i].view(1, hq, d), want, bound, (i, l))
        got = p[:, 0].view(hkv, hq // hkv, l).sum(1)
        assert ((w[i, :, :l].double() - got).abs() <= (2 * serr + 2.0 ** -20) * got).all(), (i, l)
    assert hyp.hyp_device_wait_status() == 0


def partial_rows(heads, n, ng, prefix_pages, own_pages):
    """Partial rows per (sequence, query head) that the scratch of a shared call is made for."""
    return hyp.hyp_op_attn_shared_scratch_bytes(heads, n, ng, prefix_pages, own_pages) // (4 * n * heads[0] * (heads[2] + 2))


def rereads(heads, n, prefix_pages):
    """Bytes of prefix that every sequence would read for itself; row tiles take over above 32 MB (and 8 pages)."""
    return n * heads[1] * prefix_pages * 64 * heads[2]


def check_shared(heads, prefix, sizes, own, c, q, ot):
    n, ng = len(own), len(prefix)
    hq, hkv, d = heads
    cu = torch.tensor([sum(sizes[:i]) for i in range(ng + 1)], dtype=torch.int32, device="cuda")
    ctx = torch.tensor([o - 1 for o in own], dtype=torch.int32, device="cuda")
    out = run_shared(heads, q, c, cu, c.table[:ng].contiguous(), torch.tensor(prefix, dtype=torch.int32, device="cuda"), ot, ctx)
    group = [g for g, size in enumerate(sizes) for _ in range(size)]
    for i in range(n):
        k, v = torch.cat([c.k[group[i]], c.k[ng + i]]), torch.cat([c.v[group[i]], c.v[ng + i]])
        if k.shape[0] == 0:
            assert (out[i] == 0).all()
            continue
        want, _, bound, _ = reference(q[i:i + 1].reshape(1, hq, d), k, v, torch.ones(1, k.shape[0], dtype=torch.bool, device="cuda"))
        close(out[i].view(1, hq, d), want, bound, (i, group[i], own[i]))
    assert hyp.hyp_device_wait_status() == 0


@pytest.mark.parametrize("order", ["growing", "falling", "spread"])
def test_large_scores_through_the_row_tiles_and_their_join(order):
    """Scores far apart, a maximum that moves along the prefix in either direction, shares whose maxima differ by far: enough
    sequences that the prefix goes through row tiles."""
    heads, n, l = (8, 2, 128), 64, 700
    own = [[0, 1, 20, 40][i % 4] for i in range(n)]
    c = Cache([l] + own, 2, 128, seed=61)
    pages, ot = c.table.shape[1], c.table[1:, :4].contiguous()
    assert rereads(heads, n, pages) > 32e6 and partial_rows(heads, n, 1, pages, 4) == 3 + 1      # three shares of the prefix, one own
    scale = {"growing": torch.linspace(0.02, 1.0, l), "falling": torch.linspace(1.0, 0.02, l), "spread": torch.rand(l)}[order]
    c.k[0] = (c.k[0] * scale.cuda().half()[:, None, None]).contiguous()
    for p in range((l + 15) // 16):
        put(c.pool, int(c.table[0, p]), 0, c.k[0][16 * p:16 * p + 16])
    check_shared(heads, [l], [n], own, c, queries(n, 8, 128, seed=62, std=12.0), ot)


@pytest.mark.parametrize("n,ng", [(70, 30), (1000, 2)])
def test_more_row_tiles_than_fit_at_once(n, ng):
    """At most 32 groups, but more (row tile, KV head) pairs than CTAs fit: a fixed number of shares."""
    heads = (40, 10, 128)
    rng = np.random.default_rng(n + ng)
    prefix = [699] + [int(x) for x in rng.integers(0, 700, ng - 1)]
    cuts = [0] + np.sort(rng.integers(0, n + 1, ng - 1)).tolist() + [n]
    sizes = [b - a for a, b in zip(cuts, cuts[1:])]
    own = [int(x) for x in rng.integers(0, 40, n)]
    c = Cache(prefix + own, 10, 128, seed=n)
    pages = c.table.shape[1]
    # even shares would be three of the prefix; every sequence for itself would be one row
    assert (n // 32 + ng) * 10 > 2 * 148 and rereads(heads, n, pages) > 32e6 and partial_rows(heads, n, ng, pages, 4) == 1 + 1
    check_shared(heads, prefix, sizes, own, c, queries(n, 40, 128, seed=63), c.table[ng:, :4].contiguous())


@pytest.mark.parametrize("heads", [(8, 2, 128), (40, 10, 128), (3, 3, 64)])
@pytest.mark.parametrize("m", [dict(window=128, prefix=2000), dict(window=1, prefix=900, cap=20.0), dict(window=300, prefix=2500, slopes=True)])
def test_a_long_visible_prefix_beside_a_window(heads, m):
    """Decode and prompts whose window stands behind, in, or around the end of a long prefix."""
    hq, hkv, d = heads
    lens, new = [2600, 950, 2003, 120], [150, 33, 20, 120]
    c = Cache(lens, hkv, d, seed=64)
    mod, slopes, pre = make_mod(m, hq, len(lens))
    q = queries(len(lens), hq, d, seed=65)
    out = run_decode_mod(c, heads, q, torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda"), mod)
    rows = queries(sum(new), hq, d, seed=66)
    cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    pout = torch.full((sum(new), hq * d), 7.0, dtype=torch.float16, device="cuda")
    hyp.hyp_op_attn_prefill_mod(heads, mod, rows, c.pool, c.table, cu, torch.tensor([l - r for l, r in zip(lens, new)], dtype=torch.int32, device="cuda"),
                                pout)
    torch.cuda.synchronize()
    for i, (l, r) in enumerate(zip(lens, new)):
        mask, bias = mask_and_bias(torch.tensor([l - 1], device="cuda"), l, m, int(pre[i]), slopes)
        want, _, bound, _ = reference(q[i:i + 1].reshape(1, hq, d), c.k[i], c.v[i], mask, m.get("cap", 0.0), bias)
        close(out[i].view(1, hq, d), want, bound, (i, l))
        a, b = int(cu[i]), int(cu[i + 1])
        mask, bias = mask_and_bias(torch.arange(l - r, l, device="cuda"), l, m, int(pre[i]), slopes)
        want, _, bound, _ = reference(rows[a:b].reshape(r, hq, d), c.k[i], c.v[i], mask, m.get("cap", 0.0), bias)
        close(pout[a:b].view(r, hq, d), want, bound, (i, l, r))
    assert hyp.hyp_device_wait_status() == 0


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_tensors_of_another_device_than_the_current_one():
    """The call runs where its tensors are, and reports a wait that ran out to that device's own word."""
    heads, lens = (8, 2, 128), [700, 33]
    c = Cache(lens, 2, 128, seed=71)
    q = queries(2, 8, 128, seed=72)
    ctx = torch.tensor([l - 1 for l in lens], dtype=torch.int32, device="cuda")
    here = run_decode_mod(c, heads, q, ctx, hyp.AttnMod(softcap=20.0))
    other = torch.device("cuda", (torch.cuda.current_device() + 1) % torch.cuda.device_count())
    c.pool, c.table = c.pool.to(other), c.table.to(other)
    out = torch.empty(2, 1024, dtype=torch.float16, device=other)
    scratch = bytes_of(hyp.hyp_op_attn_mod_scratch_bytes(heads, 2, c.table.shape[1])).to(other)
    hyp.hyp_op_attn_decode_mod(heads, hyp.AttnMod(softcap=20.0), q.to(other), c.pool, c.table, ctx.to(other), scratch, out)
    torch.cuda.synchronize(other)
    assert torch.equal(out.cpu(), here.cpu())
    with torch.cuda.device(other):
        assert hyp.hyp_device_wait_status() == 0
