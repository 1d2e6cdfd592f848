"""Operators over the paged key / value cache, as cases that can be timed and compared.

Four operators that a server needs beside plain decode and prefill attention, all on the library's cache layout
(one block's pool fp16 [pages][2 (K, V)][kv heads][16 tokens][head_dim]; inside a token's row the 16-byte chunk c sits at
chunk position c ^ (slot & 7)):

* shared   one new token per sequence, where groups of sequences share a long prefix: the prefix's keys and values are
           kept once per group, every sequence adds pages of its own.
* scored   decode attention that also returns, per KV head and cached position, the running sum of the attention weight
           that position has received (old sum times a decay, plus this step's weights of the group's query heads).
* evict    cuts every sequence's cache to a budget by those sums: the first tokens, the latest tokens and the heaviest of
           the others stay, in their order; keys, values and sums move to a dense place.
* modified attention whose scores are capped by a tanh, get a bias that falls with the distance, and are masked to a
           window behind the query and / or a prefix that every query sees: for prompts (prefill) and single tokens
           (decode).

`run` computes them with elementary torch operations in 32 bits (own = False) or by the library's calls (own = True).
"""
import math
import random

import torch

own = False

PAGE = 16
# (query heads, KV heads, head_dim): the two benchmark models, the small test stage, no sharing, one shared head
HEADS = [(40, 10, 128), (32, 8, 128), (4, 2, 64), (8, 8, 128), (8, 1, 64)]


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def _shared(name, heads, seqs, groups, prefix, own_len, even=False):
    return {"name": name, "op": "shared", "hq": heads[0], "hkv": heads[1], "dim": heads[2], "seqs": seqs, "groups": groups,
            "prefix": prefix, "ctx": own_len, "even": even}


def _scored(name, heads, seqs, ctx, decay, even=False):
    return {"name": name, "op": "scored", "hq": heads[0], "hkv": heads[1], "dim": heads[2], "seqs": seqs, "ctx": ctx,
            "decay": decay, "even": even}


def _evict(name, heads, seqs, ctx, keep, sink, recent, even=False):
    return {"name": name, "op": "evict", "hq": heads[0], "hkv": heads[1], "dim": heads[2], "seqs": seqs, "ctx": ctx,
            "keep": keep, "sink": sink, "recent": recent, "even": even}


def _mod(name, op, heads, seqs, ctx, rows, cap, slopes, window, prefix, even=False):
    return {"name": name, "op": op, "hq": heads[0], "hkv": heads[1], "dim": heads[2], "seqs": seqs, "ctx": ctx, "rows": rows,
            "cap": cap, "slopes": slopes, "window": window, "prefix": prefix, "even": even}


def listed():
    phi, llama, tiny = HEADS[0], HEADS[1], HEADS[2]
    return [
        # three requests on a small stage behind a short common instruction: the latency of the call itself
        _shared("shared_small", tiny, 3, 1, 100, 24),
        # a batch of chats behind one system prompt
        _shared("shared_chat", phi, 32, 1, 2048, 256),
        # the largest decode batch, five tenants with long prompts of different lengths, answers under way
        _shared("shared_tenants", llama, 128, 5, 8192, 1024),
        # the benchmark's decode batch, plain running sums
        _scored("scored_batch8", phi, 8, 1024, 1.0, even=True),
        # long generations with a slowly forgetting sum
        _scored("scored_long", phi, 4, 32768, 0.99),
        # long generation cut back to half its cache
        _evict("evict_half", phi, 4, 4096, 2048, 4, 256, even=True),
        # a ragged batch, some sequences already below the budget
        _evict("evict_ragged", llama, 32, 8191, 1000, 4, 100),
        # one 512-token prompt with capped scores
        _mod("prefill_capped", "prefill", phi, 1, 512, 512, 50.0, False, 0, 0, even=True),
        # chunks of three prompts behind cached tokens, distance bias
        _mod("prefill_distance", "prefill", llama, 3, 2500, 900, 0.0, True, 0, 0),
        # a long prompt with a window, a prefix that all tokens see, and capped scores
        _mod("prefill_window", "prefill", phi, 1, 4096, 4096, 30.0, False, 1024, 200, even=True),
        # the benchmark's decode batch with capped scores
        _mod("decode_capped", "decode", phi, 8, 1024, 1, 30.0, False, 0, 0, even=True),
        # a large ragged batch with a window, a distance bias and a short prefix that stays visible
        _mod("decode_window", "decode", llama, 64, 8192, 1, 0.0, True, 1000, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    op = rng.choice(["shared", "scored", "evict", "prefill", "decode"])
    heads = rng.choice(HEADS)
    even = rng.random() < 0.25
    if op == "shared":
        seqs = _log(rng, 1, 128)
        c = _shared("", heads, seqs, rng.randint(1, min(seqs, 6)), _log(rng, 16, 8192), _log(rng, 1, min(1024, 65536 // seqs)), even)
    elif op == "scored":
        seqs = _log(rng, 1, 64)
        c = _scored("", heads, seqs, _log(rng, 1, max(2, min(32768, 98304 // seqs))), rng.choice([1.0, 0.95, 0.99]), even)
    elif op == "evict":
        seqs = _log(rng, 1, 32)
        ctx = _log(rng, 20, 8191)
        sink, recent = rng.choice([0, 1, 4]), _log(rng, 1, max(1, ctx // 8))
        c = _evict("", heads, seqs, ctx, sink + recent + _log(rng, 1, max(1, ctx // 2)), sink, recent, even)
    else:
        cap = rng.choice([0.0, 30.0, 50.0])
        slopes = rng.random() < 0.4
        window = rng.choice([0, 0, _log(rng, 1, 4096)])
        prefix = rng.choice([0, 0, _log(rng, 1, 512)])
        if op == "prefill":
            seqs = _log(rng, 1, 4)
            rows = _log(rng, 1, 2000 // seqs)
            c = _mod("", op, heads, seqs, rows + rng.choice([0, _log(rng, 1, 1000)]), rows, cap, slopes, window, prefix, even)
        else:
            seqs = _log(rng, 1, 128)
            c = _mod("", op, heads, seqs, _log(rng, 1, min(8192, 98304 // seqs)), 1, cap, slopes, window, prefix, even)
    del c["name"]
    return c


def _spread(case, what, n, top, low=1):
    """n lengths up to `top` (the first one is `top`): all alike, or ragged; they go by the case alone."""
    if case["even"]:
        return [top] * n
    rng = random.Random("%s %d %d %d" % (what, n, top, case["hq"]))
    return [top] + [rng.randint(min(low, top), top) for _ in range(n - 1)]


def _lengths(case):
    """Host lists that belong to a case: tokens visible or cached per sequence, new rows, groups and their prefixes."""
    n = case["seqs"]
    L = {"ctx": _spread(case, "ctx", n, case["ctx"])}
    if case["op"] == "shared":
        g = case["groups"]
        cuts = sorted(random.Random("cuts %d %d" % (n, g)).sample(range(1, n), g - 1)) if g > 1 else []
        L["cu"] = [0] + cuts + [n]
        L["prefix"] = _spread(case, "prefix", g, case["prefix"], low=case["prefix"] // 2)
    if case["op"] == "prefill":
        L["rows"] = [min(r, t) for r, t in zip(_spread(case, "rows", n, case["rows"], low=max(1, case["rows"] // 2)), L["ctx"])]
        L["rows"][0] = min(case["rows"], L["ctx"][0])
    if case["op"] in ("prefill", "decode"):
        L["prefix"] = [max(0, case["prefix"] - i) for i in range(n)]
    return L


def _visible(case, L):
    """(visible query-key pairs, distinct keys read) of a modified-attention case."""
    pairs = keys = 0
    for t, r, p in zip(L["ctx"], L.get("rows", [1] * case["seqs"]), L["prefix"]):
        p = min(p, t)
        pos = torch.arange(t - r, t)
        lo = (pos - case["window"] + 1).clamp(min=0) if case["window"] else torch.zeros_like(pos)
        pairs += int((pos + 1 - lo + (p - pos - 1).clamp(min=0) + torch.minimum(lo, torch.tensor(p))).sum())
        first = int(lo[0])
        keys += t - first + min(p, first)
    return pairs, keys


def work(case):
    L = _lengths(case)
    n, hq, hkv, d = case["seqs"], case["hq"], case["hkv"], case["dim"]
    row = 2 * hkv * d * 2                                  # keys and values of one token
    if case["op"] == "shared":
        sizes = [b - a for a, b in zip(L["cu"], L["cu"][1:])]
        pairs = sum(L["ctx"]) + sum(s * p for s, p in zip(sizes, L["prefix"]))
        return {"bytes": (sum(L["ctx"]) + sum(L["prefix"])) * row + 4 * n * hq * d, "flops": 4 * hq * d * pairs}
    if case["op"] == "scored":
        t = sum(L["ctx"])
        return {"bytes": t * (row + 8 * hkv) + 4 * n * hq * d, "flops": 4 * hq * d * t}
    if case["op"] == "evict":
        kept = sum(min(t, case["keep"]) for t in L["ctx"])
        return {"bytes": 2 * kept * row + sum(L["ctx"]) * 4 * hkv + kept * 8 * hkv, "flops": sum(L["ctx"]) * hkv}
    pairs, keys = _visible(case, L)
    m = sum(L.get("rows", [1] * n))
    return {"bytes": keys * row + 4 * m * hq * d, "flops": 4 * hq * d * pairs}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def prepare(case, seed):
    L = _lengths(case)
    n, hq, hkv, d = case["seqs"], case["hq"], case["hkv"], case["dim"]
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).half()

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    # pages in a shuffled order, as a pool hands them out after some traffic
    width = -(-case["ctx"] // PAGE)
    pwidth = -(-case["prefix"] // PAGE) if case["op"] == "shared" else 0
    n_pages = n * width + (case["groups"] * pwidth if pwidth else 0) + 5
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    s = {"case": case, "shape": (hq, hkv, d), "table": ids[:n * width].view(n, width).contiguous()}
    s["pool"] = torch.empty(n_pages, 2, hkv, PAGE, d, dtype=torch.float16, device="cuda")
    for i in range(0, n_pages, 4096):                       # in parts: the 32-bit normals of a whole pool are large
        s["pool"][i:i + 4096] = normal(*s["pool"][i:i + 4096].shape)
    rows = sum(L.get("rows", [1] * n))
    # queries as they sit in a buffer beside other heads
    s["q"] = normal(rows, (hq + 2 * hkv) * d, std=1.5)[:, :hq * d]
    s["out"] = torch.empty(rows, hq * d, dtype=torch.float16, device="cuda")
    s["longest"] = max(L["ctx"])
    if case["op"] == "shared":
        s["cu"] = ints(L["cu"])
        s["ptable"] = ids[n * width:n * width + case["groups"] * pwidth].view(case["groups"], pwidth).contiguous()
        s["plens"] = ints(L["prefix"])
    if case["op"] in ("shared", "scored", "decode"):
        s["ctx"] = ints([t - 1 for t in L["ctx"]])           # tokens before the new one
    if case["op"] == "scored":
        s["weights"] = torch.rand(n, hkv, width * PAGE, generator=g, device="cuda") * 2.0
        s["weights_out"] = torch.empty_like(s["weights"])
        for i, t in enumerate(L["ctx"]):                     # behind a sequence's end nothing is read or written
            s["weights"][i, :, t:] = 0.0
        s["weights_out"].copy_(s["weights"])
    if case["op"] == "evict":
        s["cached"] = ints(L["ctx"])
        # sums of softmax weights: a few heavy positions, a long light tail, ties among the lightest
        w = torch.rand(n, hkv, width * PAGE, generator=g, device="cuda").pow_(6.0).mul_(8.0)
        s["weights"] = torch.where(w < 1e-4, torch.zeros_like(w), w)
        k = case["keep"]
        kwidth = -(-k // PAGE)
        s["dst"] = torch.zeros(n * kwidth, 2, hkv, PAGE, d, dtype=torch.float16, device="cuda")
        s["dst_table"] = torch.randperm(n * kwidth, generator=g, device="cuda").to(torch.int32).view(n, kwidth).contiguous()
        s["kept"] = torch.empty(n, hkv, k, dtype=torch.int32, device="cuda")
        s["new_lens"] = torch.empty(n, dtype=torch.int32, device="cuda")
        s["weights_out"] = torch.zeros(n, hkv, k, device="cuda")
    if case["op"] == "prefill":
        s["cu"] = ints([sum(L["rows"][:i]) for i in range(n + 1)])
        s["ctx"] = ints([t - r for t, r in zip(L["ctx"], L["rows"])])
        s["most_rows"] = max(L["rows"])
    if case["op"] in ("prefill", "decode"):
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, hq + 1, device="cuda") / hq).float() if case["slopes"] else None
        s["plens"] = ints(L["prefix"]) if case["prefix"] else None
    return s


# ---------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------
def _rows(pool, table):
    """Keys and values behind a table of pages: two fp32 tensors [tables, kv heads, tokens, head_dim]."""
    n, width = table.shape
    hkv, d = pool.shape[2], pool.shape[4]
    slot = torch.arange(PAGE, device=pool.device)[:, None]
    chunk = torch.arange(d // 8, device=pool.device)[None, :] ^ (slot & 7)
    x = pool[table.long()].view(n, width, 2, hkv, PAGE, d // 8, 8)[:, :, :, :, slot, chunk]
    x = x.permute(2, 0, 3, 1, 4, 5, 6).reshape(2, n, hkv, width * PAGE, d).float()
    return x[0], x[1]


def _softmax(s, mask):
    """Weights of the masked scores; a row with nothing to see gets zeros."""
    s = torch.where(mask, s, torch.full_like(s, -math.inf))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def _heads(q, shape):
    hq, hkv, d = shape
    return q.float().reshape(-1, hkv, hq // hkv, d)


def _plain_shared(s):
    hq, hkv, d = s["shape"]
    n = s["ctx"].shape[0]
    group = torch.bucketize(torch.arange(n, device="cuda"), s["cu"][1:].long(), right=True)
    pk, pv = _rows(s["pool"], s["ptable"])
    ok, ov = _rows(s["pool"], s["table"])
    k, v = torch.cat([pk[group], ok], 2), torch.cat([pv[group], ov], 2)
    at = torch.arange(k.shape[2], device="cuda")[None, :]
    split = pk.shape[2]
    mask = torch.where(at < split, at < s["plens"][group][:, None], at - split <= s["ctx"][:, None])
    p = _softmax(_heads(s["q"], s["shape"]) @ k.transpose(2, 3) / math.sqrt(d), mask[:, None, None, :])
    return (p @ v).reshape(n, hq * d).half()


def _plain_scored(s):
    hq, hkv, d = s["shape"]
    n = s["ctx"].shape[0]
    k, v = _rows(s["pool"], s["table"])
    at = torch.arange(k.shape[2], device="cuda")[None, None, :]
    new = s["ctx"][:, None, None]
    p = _softmax(_heads(s["q"], s["shape"]) @ k.transpose(2, 3) / math.sqrt(d), (at <= new)[:, :, None, :])
    w = torch.where(at < new, s["weights"] * s["case"]["decay"], torch.zeros_like(s["weights"])) + p.sum(2)
    return (p @ v).reshape(n, hq * d).half(), torch.where(at <= new, w, s["weights"])


def _plain_evict(s):
    c = s["case"]
    hq, hkv, d = s["shape"]
    w, t, keep = s["weights"], s["cached"].long()[:, None, None], c["keep"]
    at = torch.arange(w.shape[2], device="cuda")[None, None, :].expand_as(w)
    fixed = (at < c["sink"]) | (at >= t - c["recent"])
    rank = torch.where(at < t, torch.where(fixed, 0, 1), 2)
    order = torch.sort(torch.where(torch.isnan(w), torch.full_like(w, -math.inf), w), dim=2, descending=True, stable=True)[1]
    order = torch.gather(order, 2, torch.sort(torch.gather(rank, 2, order), dim=2, stable=True)[1])
    pad = max(0, keep - w.shape[2])
    order = torch.nn.functional.pad(order, (0, pad), value=w.shape[2])[:, :, :keep]
    kept = torch.sort(torch.where(order < t, order, w.shape[2] + 1), dim=2)[0]
    there = torch.arange(keep, device="cuda")[None, None, :] < torch.minimum(t, torch.tensor(keep, device="cuda"))
    src = torch.where(there, kept, torch.zeros_like(kept))
    wout = torch.where(there, torch.gather(w, 2, src), torch.zeros_like(w[:, :, :1]))
    k, v = _rows(s["pool"], s["table"])
    rows = torch.stack([k, v], 2).gather(3, src[:, :, None, :, None].expand(-1, -1, 2, -1, d)).half()   # [n, hkv, 2, keep, d]
    to = torch.arange(keep, device="cuda")
    slot = (to % PAGE)[:, None]
    chunk = torch.arange(d // 8, device="cuda")[None, :] ^ (slot & 7)
    rows = rows.view(*rows.shape[:4], d // 8, 8)[:, :, :, to[:, None], chunk].reshape(rows.shape)
    rows = torch.where(there[:, :, None, :, None], rows, torch.zeros_like(rows))
    n, kwidth = s["dst_table"].shape
    rows = torch.nn.functional.pad(rows, (0, 0, 0, kwidth * PAGE - keep)).view(n, hkv, 2, kwidth, PAGE, d)
    dst = torch.zeros_like(s["dst"])
    dst[s["dst_table"].long()] = rows.permute(0, 3, 2, 1, 4, 5)
    return (torch.where(there, kept, -torch.ones_like(kept)).to(torch.int32), torch.minimum(s["cached"], torch.tensor(keep, device="cuda")).to(torch.int32),
            wout, dst)


def _plain_modified(s):
    c = s["case"]
    hq, hkv, d = s["shape"]
    n = s["ctx"].shape[0]
    k, v = _rows(s["pool"], s["table"])
    q = _heads(s["q"], s["shape"])
    if c["op"] == "decode":
        row = torch.arange(n, device="cuda")[:, None]
        pos = s["ctx"].long()[:, None]
        total = pos + 1
    else:                                                  # every sequence's rows side by side, padded to the longest
        step = torch.arange(s["most_rows"], device="cuda")[None, :]
        count = (s["cu"][1:] - s["cu"][:-1]).long()[:, None]
        row = torch.where(step < count, s["cu"][:-1].long()[:, None] + step, 0)
        pos = s["ctx"].long()[:, None] + step
        total = s["ctx"].long()[:, None] + count
    x = q[row].permute(0, 2, 3, 1, 4)                       # [n, hkv, group, rows, d]
    at = torch.arange(k.shape[2], device="cuda")[None, None, :]
    back = pos[:, :, None] - at                            # distance to the key, negative ahead of the query
    mask = back >= 0
    if c["window"]:
        mask = mask & (back < c["window"])
    if s["plens"] is not None:
        mask = mask | (at < s["plens"][:, None, None])
    mask = mask & (at < total[:, :, None])
    sc = x @ k[:, :, None].transpose(3, 4) / math.sqrt(d)
    if c["cap"]:
        sc = c["cap"] * torch.tanh(sc / c["cap"])
    if s["slopes"] is not None:
        sc = sc - s["slopes"].view(1, hkv, hq // hkv, 1, 1) * back.abs()[:, None, None].float()
    o = _softmax(sc, mask[:, None, None]) @ v[:, :, None]
    o = o.permute(0, 3, 1, 2, 4).reshape(n, -1, hq * d).half()
    if c["op"] == "decode":
        return o[:, 0].contiguous()
    return o[step < count]


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def _library(s):
    """What a user's program sets up once per plan: the binding, a scratch buffer, the score modification."""
    if "lib" not in s:
        from paper_2511_14450_b200 import hyperion as hyp
        c, n = s["case"], s["table"].shape[0]
        nbytes = 0
        if c["op"] == "shared":
            nbytes = hyp.hyp_op_attn_shared_scratch_bytes(s["shape"], n, c["groups"], s["ptable"].shape[1], s["table"].shape[1])
        elif c["op"] == "scored":
            nbytes = hyp.hyp_op_attn_scored_scratch_bytes(s["shape"], n, s["table"].shape[1])
        elif c["op"] in ("prefill", "decode"):
            s["mod"] = hyp.AttnMod(softcap=c["cap"], window=c["window"], slopes=s["slopes"], prefix_lens=s["plens"])
            if c["op"] == "decode":
                nbytes = hyp.hyp_op_attn_mod_scratch_bytes(s["shape"], n, s["table"].shape[1])
        s["scratch"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
        s["lib"] = hyp
    return s["lib"]


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"shared": _plain_shared, "scored": _plain_scored, "evict": _plain_evict}.get(op, _plain_modified)(s)
    hyp = _library(s)
    c = s["case"]
    if op == "shared":
        hyp.hyp_op_attn_decode_shared(s["shape"], s["q"], s["pool"], s["cu"], s["ptable"], s["plens"], s["table"], s["ctx"],
                                      s["scratch"], s["out"])
        return s["out"]
    if op == "scored":
        hyp.hyp_op_attn_decode_scored(s["shape"], s["q"], s["pool"], s["table"], s["ctx"], c["decay"], s["weights"],
                                      s["weights_out"], s["scratch"], s["out"])
        return s["out"], s["weights_out"]
    if op == "evict":
        hyp.hyp_op_kv_evict(s["shape"], s["pool"], s["table"], s["cached"], s["weights"], c["keep"], c["sink"], c["recent"],
                            s["dst"], s["dst_table"], s["kept"], s["new_lens"], s["weights_out"])
        return s["kept"], s["new_lens"], s["weights_out"], s["dst"]
    if op == "decode":
        hyp.hyp_op_attn_decode_mod(s["shape"], s["mod"], s["q"], s["pool"], s["table"], s["ctx"], s["scratch"], s["out"])
    else:
        hyp.hyp_op_attn_prefill_mod(s["shape"], s["mod"], s["q"], s["pool"], s["table"], s["cu"], s["ctx"], s["out"])
    return s["out"]


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits, one sequence and one head at a time
# ---------------------------------------------------------------------------------------------
def _token(pool, pages, kind, head, count):
    """Rows of one KV head, fp64 [count, d], each row put back from its chunk order."""
    d = pool.shape[4]
    slot = torch.arange(count, device="cuda") % PAGE
    raw = pool[pages.long(), kind, head].reshape(-1, d)[:count].double()
    lane = torch.arange(d, device="cuda")
    return raw.gather(1, ((lane // 8) ^ (slot[:, None] & 7)) * 8 + lane % 8)


def exact(case, seed):
    L = _lengths(case)
    pairs = case["hq"] * sum(L["ctx"]) if case["op"] != "prefill" else case["hq"] * _visible(case, L)[0]
    if pairs > 2_000_000_000:
        return None
    s = prepare(case, seed)
    hq, hkv, d = s["shape"]
    group = hq // hkv
    q = s["q"].double()
    if case["op"] == "evict":
        kept = torch.full((case["seqs"], hkv, case["keep"]), -1, dtype=torch.int32)
        wout = torch.zeros(case["seqs"], hkv, case["keep"], dtype=torch.float64)
        dst = torch.zeros(s["dst"].shape, dtype=torch.float16, device="cuda").double()
        w = s["weights"].double().cpu()
        lane = torch.arange(d, device="cuda")
        for b, t in enumerate(L["ctx"]):
            m = min(t, case["keep"])
            fixed = [j for j in range(t) if j < case["sink"] or j >= t - case["recent"]]
            held = set(fixed)
            for h in range(hkv):
                v = w[b, h].tolist()
                rest = sorted((j for j in range(t) if j not in held), key=lambda j: (-v[j], j))
                pick = sorted((fixed + rest)[:m]) if t > case["keep"] else list(range(t))
                kept[b, h, :m] = torch.tensor(pick, dtype=torch.int32)
                wout[b, h, :m] = torch.tensor([v[j] for j in pick], dtype=torch.float64)
                take = torch.tensor(pick, device="cuda")
                slot = torch.arange(m, device="cuda")
                place = ((lane // 8) ^ (slot[:, None] & 7)) * 8 + lane % 8
                for kind in (0, 1):
                    x = _token(s["pool"], s["table"][b], kind, h, t)[take]
                    dst[s["dst_table"][b].long()[slot // PAGE], kind, h, slot % PAGE] = torch.empty_like(x).scatter_(1, place, x)
        return kept, torch.tensor([min(t, case["keep"]) for t in L["ctx"]], dtype=torch.int32), wout.cuda(), dst
    out = torch.zeros(q.shape[0], hq * d, dtype=torch.float64, device="cuda")
    wsum = s["weights"].double() if case["op"] == "scored" else None
    row = 0
    for b, t in enumerate(L["ctx"]):
        rows = L["rows"][b] if case["op"] == "prefill" else 1
        pos = torch.arange(t - rows, t, device="cuda").double()[:, None]
        key = torch.arange(t, device="cuda").double()[None, :]
        seen = key <= pos
        if case.get("window"):
            seen = seen & (key > pos - case["window"])
        if case["op"] in ("prefill", "decode"):
            seen = seen | (key < L["prefix"][b])
        for h in range(hkv):
            k, v = _token(s["pool"], s["table"][b], 0, h, t), _token(s["pool"], s["table"][b], 1, h, t)
            if case["op"] == "shared":
                g = sum(1 for x in L["cu"][1:] if x <= b)
                p = L["prefix"][g]
                k = torch.cat([_token(s["pool"], s["ptable"][g], 0, h, p), k])
                v = torch.cat([_token(s["pool"], s["ptable"][g], 1, h, p), v])
            got = 0.0
            for i in range(h * group, (h + 1) * group):
                x = q[row:row + rows, i * d:(i + 1) * d] @ k.T * d ** -0.5
                if case.get("cap"):
                    x = torch.tanh(x / case["cap"]) * case["cap"]
                if case.get("slopes"):
                    x = x - s["slopes"][i].double() * (pos - key).abs()
                if case["op"] != "shared":
                    x = x.masked_fill(~seen, -math.inf)
                e = torch.softmax(x, -1)
                out[row:row + rows, i * d:(i + 1) * d] = e @ v
                got = got + e[0]
            if case["op"] == "scored":
                wsum[b, h, :t - 1] *= case["decay"]
                wsum[b, h, t - 1] = 0.0
                wsum[b, h, :t] += got
        row += rows
    return out if wsum is None else (out, wsum)
