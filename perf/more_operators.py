"""The 8-bit paged cache, measured: page tables kept on the GPU, the cache that holds
keys and values in 8 bits, and the attention that reads it.

Kinds of cases:

``assign``   page tables from request lengths: pages that no later query sees go
             back to the free list, new tokens get pages, and each token's row
             per head is written down (``moa_paged_assign``).
``append``   new tokens enter the pages: queries and keys are rotated by their
             positions, keys and values stored in 8 bits (``moa_quant_append``).
``prefill``  ragged chunks of new tokens attend to all that their sequences'
             pages hold (``moa_quant_prefill``).
``decode``   one token per sequence (``moa_quant_decode``).
``shared``   the same for a batch whose sequences begin with one long prefix,
             which is read once for all (``moa_quant_decode_shared``).

A page holds ``page`` consecutive positions of one KV head; ``table[b, g, i]`` is the
page of positions ``i * page ..`` of head g of sequence b, negative where there is
none.  Query position p of KV head g sees key j iff j <= p and (j < sink or
p - j < window_g), or with the block band the same in blocks of 64.

Keys and values are e4m3 numbers times a scale of their block of 16 positions: the
smallest power of two 2^e, -117 <= e <= 119, that keeps the block's largest magnitude
within 448.  New tokens behind the first position of a block keep the rows in front of
them: the scale is then the larger of the stored and the needed one, and if that is more
than the stored one the rows in front are rounded to it.

Inputs are N(0, 1); queries share a component with the first four keys, as the sink
tokens of a trained model draw weight from every query, and some channels of the keys
are larger than the rest.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False                # True: the library's kernels; False: plain torch in 32 bits

DEVICE = "cuda"
SINK_TOKENS = 4            # keys that every query leans to
SINK_SHIFT = 0.5           # shared component per dimension
SPAN_INCLUDES_SINKS, BLOCK_BAND, BAND_BLOCK = 1, 2, 64     # plan options
LOWEST, HIGHEST, MOST = -117, 119, 448.0                    # exponents of scales, largest e4m3 number
BLOCK = 16                 # positions of one scale


def _case(kind, b, hq, hkv, d, n, ctx, new=0, page=64, sink=64, mean=0.5, flags=0, rules=1, pad=0, rotary=0,
          interleaved=False, prefix=0, fresh=0):
    """n: the length that the rule is evaluated at.  ctx: the longest cached context (kind shared: the longest
    part behind the prefix).  new: packed new tokens of all sequences, 0 for one token each.  pad: rows behind
    the last sequence, which a call leaves as they are.  fresh: slots whose sequence ended and that get a prompt."""
    return dict(kind=kind, b=b, hq=hq, hkv=hkv, d=d, n=n, ctx=ctx, new=new, page=page, sink=sink, mean=mean, flags=flags,
                rules=rules, pad=pad, rotary=rotary, interleaved=interleaved, prefix=prefix, fresh=fresh)


def listed():
    return [dict(name=name, **case) for name, case in [
        # one step of continuous batching: 45 sequences decode a token, 3 slots get a prompt each
        ("assign-step-gqa8-b48", _case("assign", 48, 64, 8, 128, 16384, 16000, new=1600, page=64, rules=3, fresh=3)),
        # a batch of prompts takes over all slots, small pages
        ("assign-prompts-b5-16k", _case("assign", 5, 32, 32, 128, 8192, 0, new=16000, page=16, rules=4, pad=3, fresh=5)),
        # one decode step's new tokens, one slot idle: latency counts
        ("append-step-gqa4-b16", _case("append", 16, 32, 8, 128, 16384, 16000, rotary=128, rules=3)),
        # a batch of prompts and chunks far into long contexts, pairs side by side, small pages
        ("append-gqa8-8k", _case("append", 5, 64, 8, 128, 32768, 100000, new=8190, page=16, rotary=128, interleaved=True,
                                 pad=2, rules=4)),
        # a short chat prompt
        ("prefill-gqa4-500", _case("prefill", 1, 32, 8, 128, 4096, 0, new=500, rules=2)),
        # continuous batching: short chunks over contexts of up to 16k tokens, small pages
        ("prefill-chunks-b6-16k", _case("prefill", 6, 32, 8, 128, 16384, 16000, new=1507, page=16, pad=5, rules=3)),
        # two whole prompts with the 64-token block band and spans that include the sinks
        ("prefill-b2-12k-block", _case("prefill", 2, 32, 32, 128, 8192, 0, new=12000, page=128, flags=3, rules=4)),
        # interactive decode: one sequence
        ("decode-b1-4k", _case("decode", 1, 32, 32, 128, 4096, 4100, rules=2)),
        # batch decode of a grouped-query model, sequences of 500 to 16,400 tokens, one slot idle
        ("decode-gqa4-b16-16k", _case("decode", 16, 32, 8, 128, 16384, 16400, page=32, rules=3)),
        # a large batch of 8 query heads per KV head, small pages
        ("decode-gqa8-b61-16k", _case("decode", 61, 64, 8, 128, 16384, 16001, page=16, rules=7)),
        # answers of a batch to one long document
        ("shared-gqa4-b16-8k", _case("shared", 16, 32, 8, 128, 16384, 500, prefix=8001, rules=3)),
        # a system prompt of 32k tokens under a large batch
        ("shared-gqa8-b48-32k", _case("shared", 48, 64, 8, 128, 32768, 1000, prefix=32700, page=32, mean=0.25, rules=4)),
    ]]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (query heads, KV heads, head dim): the layers of the configurations, and smaller ones of each group size
_LAYERS = [(32, 32, 128), (32, 8, 128), (64, 8, 128), (16, 8, 128), (32, 8, 64), (16, 16, 64)]


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 8e14)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["assign", "assign", "append", "append", "prefill", "prefill", "decode", "decode", "shared",
                           "shared"])
        hq, hkv, d = rng.choice(_LAYERS)
        b = _log_int(rng, 1, 48)
        ctx = _log_int(rng, 500, 16384)
        new = prefix = fresh = 0
        if kind in ("prefill", "assign") or (kind == "append" and rng.random() < 0.5):
            new = max(b, _log_int(rng, 100, 12000))
            ctx = rng.choice([0, ctx])
        if kind == "assign":
            fresh = b if ctx == 0 else rng.randrange(1, b + 1)
        if kind == "shared":
            b = max(b, 2)
            prefix, ctx = 2 * ctx, _log_int(rng, 1, 1500)
        case = _case(kind, b, hq, hkv, d, max(ctx + new, prefix), ctx, new, rng.choice([16, 32, 64, 128, 256]),
                     rng.choice([0, 4, 64]), rng.choice([0.25, 0.5]), rng.choice([0, 0, 1, 2, 3]),
                     rng.randrange(100, 1000), rng.choice([0, 0, 3]) if new else 0,
                     rng.choice([d, d, d // 2, 0]) if kind == "append" else 0, rng.random() < 0.5, prefix, fresh)
        # the plain form's scores fit the card
        if _cost(case) <= most and (kind != "prefill" or _scores(case) <= 4 << 30):
            return case


# ---------------------------------------------------------------------------
# Windows and lengths (plain arithmetic).
# ---------------------------------------------------------------------------
def _rules(case):
    """(alpha, beta) per KV head with a mean window of case["mean"] of n."""
    rng = np.random.default_rng(case["rules"])
    n, hkv = float(case["n"]), case["hkv"]
    alpha = rng.choice([256.0, 512.0, 1024.0, 2048.0], size=hkv)
    beta = rng.choice([0.0, 0.25, 0.5, 0.75], size=hkv)
    lo, hi = 0.0, 1024.0
    for _ in range(100):
        f = 0.5 * (lo + hi)
        if np.minimum(n, f * (alpha + beta * n)).mean() < case["mean"] * n:
            lo = f
        else:
            hi = f
    return hi * alpha, hi * beta


def _windows(case):
    n, s = float(case["n"]), case["sink"]
    out = []
    for alpha, beta in zip(*_rules(case)):
        x = float(alpha) + float(beta) * n
        if case["flags"] & SPAN_INCLUDES_SINKS:
            out.append(max(int(math.floor(min(max(x, 0.0), n))) - s, 1))
        else:
            out.append(int(math.floor(min(max(x, 1.0), n))))
    return out


def _band_start(case, p, w):
    """First key of position p's band (numbers, arrays or tensors); prompts may count it in blocks."""
    if case["kind"] == "prefill" and case["flags"] & BLOCK_BAND:
        return (p // BAND_BLOCK - -(-w // BAND_BLOCK) + 1) * BAND_BLOCK
    return p - w + 1


def _needed_from(case, p, w):
    """First key behind the sinks that a query at p or later sees, in a prompt or alone."""
    lo = p - w + 1
    if case["flags"] & BLOCK_BAND:
        block = (p // BAND_BLOCK - -(-w // BAND_BLOCK) + 1) * BAND_BLOCK
        lo = lo - (lo > block) * (lo - block)
    return lo


def _sequences(case):
    """(start, count) of each sequence's new tokens: numpy int64 [b], start -1 where idle."""
    rng = np.random.default_rng(case["rules"] + 17)
    b, ctx = case["b"], case["ctx"]
    if case["kind"] == "shared":
        start = case["prefix"] + rng.integers(0, ctx + 1, size=b)
        start[0] = case["prefix"] + ctx
        return start, np.ones(b, dtype=np.int64)
    if case["new"] == 0:
        start = ctx * (2 * np.arange(b) + 1) // (2 * b)
        start[0] = ctx
        if b > 2:
            start[b // 2] = -1
        return start, np.ones(b, dtype=np.int64)
    start = np.floor(ctx * rng.uniform(0.0, 1.0, size=b)).astype(np.int64)
    start[0] = ctx
    many = np.ones(b, dtype=bool)
    if case["kind"] == "assign":
        many = _fresh(case)
        start[many] = 0
    share = rng.uniform(0.2, 1.8, size=b) * many
    count = 1 + np.floor(share / share.sum() * (case["new"] - b)).astype(np.int64)
    count[np.nonzero(many)[0][-1]] += case["new"] - count.sum()
    return start, count


def _fresh(case):
    rng = np.random.default_rng(case["rules"] + 18)
    out = np.zeros(case["b"], dtype=bool)
    out[rng.permutation(case["b"])[:case["fresh"]]] = True
    return out


def _seen(case, w, first, last):
    """Key ranges [(lo, hi), ..] that the queries first .. last of one sequence see."""
    s = min(case["sink"], last + 1)
    lo = max(int(_band_start(case, first, w)), 0)
    return [(0, last + 1)] if lo <= s else [(0, s), (lo, last + 1)]


def _cut(ranges, lo, hi):
    return [(max(a, lo), min(z, hi)) for a, z in ranges if max(a, lo) < min(z, hi)]


def _stored(case, w, start, count):
    """Key ranges of one sequence and head that its own pages have to hold."""
    if start < 0:
        return []
    if case["kind"] == "append":               # the rows in front of the first new one share its scale
        return [(int(start) // BLOCK * BLOCK, int(start + count))]
    return _cut(_seen(case, w, int(start), int(start + count) - 1), case["prefix"], 1 << 40)


def _prefix_stored(case, w):
    """Key ranges of the shared prefix that some sequence sees."""
    start, _ = _sequences(case)
    return _cut(_seen(case, w, int(start.min()), int(start.max())), 0, case["prefix"])


def _pairs(case, w, start, count):
    """Visible (query, key) pairs of one head of one sequence."""
    p = np.arange(start, start + count, dtype=np.int64)
    lo = np.maximum(_band_start(case, p, w), 0)
    return int((p + 1 - lo + np.minimum(lo, case["sink"])).sum())


def _scores(case):
    start, count = _sequences(case)
    return case["b"] * case["hq"] * int(count.max()) * int((start + count).max())


def _width(case):
    start, count = _sequences(case)
    return int(max(start + count)) // case["page"] + 2


def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    start, count = _sequences(case)
    tokens = int(count[start >= 0].sum())
    if case["kind"] == "assign":
        # the entries up to each sequence's end, those of new prompts written and their pages off and on the list; rows
        pages = -(-(start + count) // case["page"])
        moved = int(pages[_fresh(case)].sum()) * hkv
        return {"bytes": 4 * (int(pages.sum()) * hkv + 5 * moved + tokens * hkv + 3 * case["b"]), "flops": 0}
    if case["kind"] == "append":
        return {"bytes": tokens * d * (4 * hq + 6 * hkv), "flops": tokens * 3 * case["rotary"] * (hq + hkv)}
    keys = pairs = 0
    for w in _windows(case):
        for p, c in zip(start, count):
            if p >= 0:
                keys += sum(z - a for a, z in _stored(case, w, p, c))
                pairs += _pairs(case, w, p, c)
        if case["kind"] == "shared":
            keys += sum(z - a for a, z in _prefix_stored(case, w))
    return {"bytes": d * (2 * keys + 4 * tokens * hq) + keys // 2, "flops": 4 * d * pairs * (hq // hkv)}


# ---------------------------------------------------------------------------
# Inputs (plain torch, from the seed alone).
# ---------------------------------------------------------------------------
def _randn(gen, shape):
    """N(0, 1) in fp32, rounded to bf16, drawn in slices of the first axis, so that no large fp32 copy is held."""
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEVICE)
    step = max(1, (1 << 26) // max(1, math.prod(shape[1:])))
    for i in range(0, shape[0], step):
        part = out[i:i + step]
        part.copy_(torch.randn(part.shape, generator=gen, device=DEVICE))
    return out


def _exponent(amax):
    """e of the block's scale 2^e for a largest magnitude (32 bits)."""
    _, k = torch.frexp(amax)                                   # amax = m 2^k, 1/2 <= m < 1
    e = k - 9 + (amax > torch.ldexp(torch.full_like(amax, 0.875), k))
    return torch.where(amax > 0, e, torch.full_like(e, LOWEST)).clamp(LOWEST, HIGHEST)


def _to8(x, e):
    """e4m3 codes of x 2^-e, as bytes."""
    return torch.ldexp(x, -e).clamp(-MOST, MOST).to(torch.float8_e4m3fn).view(torch.uint8)


def _pack(x, page, d):
    """Pages [n, page, d] of bf16 in 8 bits, and their scales [n, page / 16]."""
    codes = torch.empty(x.shape, dtype=torch.uint8, device=DEVICE)
    scale = torch.empty((x.shape[0], page // BLOCK), device=DEVICE)
    step = max(1, (1 << 26) // (page * d))
    for i in range(0, x.shape[0], step):
        part = x[i:i + step].float().view(-1, page // BLOCK, BLOCK * d)
        e = _exponent(part.abs().amax(-1))
        codes[i:i + step] = _to8(part, e[..., None]).view(-1, page, d)
        scale[i:i + step] = torch.ldexp(torch.ones_like(scale[i:i + step]), e)
    return codes.view(torch.float8_e4m3fn), scale


def _tables(case, seed):
    """(table [b, hkv, max_pages], prefix table [hkv, max_pages] or None, number of pages): int32 on the host."""
    rng = np.random.default_rng(seed + 99)
    ps, hkv, b = case["page"], case["hkv"], case["b"]
    start, count = _sequences(case)
    width = _width(case)
    rows = []
    for i in range(b):
        rows += [_stored(case, w, start[i], count[i]) for w in _windows(case)]
    if case["kind"] == "shared":
        rows += [_prefix_stored(case, w) for w in _windows(case)]
    held = np.zeros((len(rows), width), dtype=bool)
    for r, ranges in enumerate(rows):
        for a, z in ranges:
            held[r, a // ps:(z - 1) // ps + 1] = True
    need = int(held.sum())
    table = np.full(held.shape, -1, dtype=np.int32)
    table[held] = rng.permutation(need + 3)[:need]
    own_rows = table[:b * hkv].reshape(b, hkv, width)
    return own_rows, table[b * hkv:] if case["kind"] == "shared" else None, need + 3


def _pool(case, seed):
    """State before an ``assign`` call: (table, free list, counts) on the host.  Each slot holds a sequence whose last
    tokens came in a chunk of their own; slots that get a prompt hold the pages of one that ended."""
    rng = np.random.default_rng(case["rules"] + 19)                # lengths; which page is where goes by the seed
    ps, hkv, b, s = case["page"], case["hkv"], case["b"], case["sink"]
    start, count = _sequences(case)
    fresh, width = _fresh(case), _width(case)
    w = np.array(_windows(case))
    end = np.where(fresh, rng.integers(1, int((start + count).max()) + 1, size=b), start)
    chunk = rng.integers(1, 513, size=b)
    first = np.maximum(_needed_from(case, np.maximum(end - chunk, 0)[:, None], w[None, :]), 0)[..., None]
    i = np.arange(width)
    held = (i * ps < end[:, None, None]) & ((i * ps < s) | ((i + 1) * ps > first))
    after = -(-(start + count) // ps)
    num_pages = int(held.sum() + after[fresh].sum() * hkv + b * hkv) + 5
    order = np.random.default_rng(seed + 99).permutation(num_pages).astype(np.int32)
    table = np.full(held.shape, -1, dtype=np.int32)
    table[held] = order[:held.sum()]
    free = np.full(num_pages, -1, dtype=np.int32)
    left = order[held.sum():]
    free[:len(left)] = left
    return table, free, np.array([len(left), 0], dtype=np.int32)


def _dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEVICE)


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    hq, hkv, d, ps = case["hq"], case["hkv"], case["d"], case["page"]
    start, count = _sequences(case)
    rows = int(count.sum()) + case["pad"]
    x = {"positions": _dev(start.astype(np.int32)), "seq_start": None, "prefix_table": None}
    if case["new"]:
        x["seq_start"] = _dev(np.concatenate([[0], np.cumsum(count)]).astype(np.int32))
    if case["kind"] == "assign":
        table, free, counts = _pool(case, seed)
        x.update(table=_dev(table), free=_dev(free), counts=_dev(counts), fresh=_dev(_fresh(case).astype(np.int32)),
                 slots=torch.full((rows, hkv), -7, dtype=torch.int32, device=DEVICE))
        return x
    table, prefix, pages = _tables(case, seed)
    x["table"] = _dev(table)
    wide = torch.ones(d, device=DEVICE)
    wide[torch.randint(0, d, (4,), generator=gen, device=DEVICE)] = 6.0       # channels of larger keys
    k = _randn(gen, (pages, ps, d)).mul_(wide)
    first = table[:, :, 0]
    if prefix is not None:
        x["prefix_table"] = _dev(prefix)
        first = prefix[:, 0]
    k[_dev(first[first >= 0].astype(np.int64)), :SINK_TOKENS] += SINK_SHIFT
    x["k_pages"], ks = _pack(k, ps, d)
    x["v_pages"], vs = _pack(_randn(gen, (pages, ps, d)), ps, d)
    x["scales"] = torch.stack((ks, vs), -1).contiguous()
    x["q"] = _randn(gen, (rows, hq, d)).add_(SINK_SHIFT)
    if case["kind"] == "append":
        x["k_new"], x["v_new"] = _randn(gen, (rows, hkv, d)).mul_(wide), _randn(gen, (rows, hkv, d))
        half = case["rotary"] // 2
        x["inv_freq"] = None if half == 0 else (
            500000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().to(DEVICE)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    state = dict(x, case=case)
    if case["kind"] != "assign":
        state["out"] = torch.zeros_like(x["q"])
    if own:
        from paper_2406_14909_amd import moa
        alpha, beta = _rules(case)
        state["plan"] = moa.moa_plan(case["hq"], case["hkv"], case["d"], case["sink"], case["n"], "bf16", alpha, beta,
                                     flags=case["flags"])
        if case["kind"] != "append":
            rows = (x["slots"] if case["kind"] == "assign" else x["q"]).shape[0]
            state["workspace"] = moa.new_paged_workspace(state["plan"], case["b"], rows, DEVICE)
    else:
        # what the plain form would otherwise copy from the host or the device in each pass
        start, count = _sequences(case)
        state["windows"] = torch.tensor(_windows(case), device=DEVICE)
        state["longest"], state["most"] = int((start + count).max()), int(count.max())
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(x):
    from paper_2406_14909_amd import moa
    plan, case = x["plan"], x["case"]
    kind = case["kind"]
    if kind == "assign":
        moa.moa_paged_assign(plan, x["table"], x["free"], x["counts"], case["page"], x["positions"], x["workspace"],
                             x["seq_start"], x["fresh"], x["slots"])
        return {"table": x["table"], "free": x["free"], "counts": x["counts"], "slots": x["slots"]}
    cache = (x["k_pages"], x["v_pages"], x["scales"])
    if kind == "append":
        q = moa.moa_quant_append(plan, *cache, x["table"], x["q"], x["k_new"], x["v_new"], x["positions"],
                                  x["seq_start"], x["inv_freq"], case["interleaved"], q_out=x["out"])
        return {"q": q, "k_pages": cache[0], "v_pages": cache[1], "scales": cache[2]}
    if kind == "prefill":
        o = moa.moa_quant_prefill(plan, x["q"], *cache, x["table"], x["positions"], x["seq_start"], x["workspace"],
                                   o=x["out"])
    elif kind == "decode":
        o = moa.moa_quant_decode(plan, x["q"], *cache, x["table"], x["positions"], x["workspace"], o=x["out"])
    else:
        o = moa.moa_quant_decode_shared(plan, x["q"], *cache, x["prefix_table"], case["prefix"], x["table"],
                                         x["positions"], x["workspace"], o=x["out"])
    return {"o": o}


# ---------------------------------------------------------------------------
# Plain forms.
# ---------------------------------------------------------------------------
def _rows(x, n):
    """(sequence, position, whether it is a token of one) of each of the n packed rows."""
    t = torch.arange(n, device=DEVICE)
    if x["seq_start"] is None:
        b, at = t, x["positions"].long()
        return b, at, at >= 0
    ends = x["seq_start"][1:].long()
    b = torch.searchsorted(ends, t, right=True).clamp(max=len(ends) - 1)
    at = x["positions"].long()[b] + t - x["seq_start"].long()[b]
    return b, at, (t < ends[-1]) & (x["positions"][b] >= 0)


def _plain_assign(x):
    case = x["case"]
    ps, s = case["page"], case["sink"]
    table, n_pages = x["table"], x["free"].shape[0]
    start = x["positions"].long()[:, None, None]
    count = (x["seq_start"][1:] - x["seq_start"][:-1]).long()[:, None, None]
    i = torch.arange(table.shape[2], device=DEVICE)
    lo = _needed_from(case, start, x["windows"][None, :, None])
    gone = (table >= 0) & ((x["fresh"] != 0)[:, None, None] | ((start >= 0) & (i * ps >= s) & ((i + 1) * ps <= lo)))
    # given back: behind the free list, in the order of the table
    n = x["counts"][0].long()
    at = torch.where(gone, n + gone.flatten().cumsum(0).view(gone.shape) - 1, n_pages)
    free = torch.cat((x["free"], x["free"][:1])).scatter_(0, at.flatten(), table.flatten())[:n_pages]
    n = n + gone.sum()
    table.masked_fill_(gone, -1)
    # taken: from the end of the list, in the order of the table
    need = (table < 0) & (start >= 0) & (count > 0) & (i >= start // ps) & (i <= (start + count - 1) // ps)
    take = n - need.flatten().cumsum(0).view(need.shape)
    table.copy_(torch.where(need & (take >= 0), free[take.clamp(min=0)], table))
    x["free"].copy_(free)
    total = need.sum()
    x["counts"].copy_(torch.stack(((n - total).clamp(min=0), (total - n).clamp(min=0))))
    # each token's row of the pool, per head
    b, p, real = _rows(x, x["slots"].shape[0])
    page = table[b, :, torch.where(real, p // ps, 0)]
    slot = torch.where(page >= 0, page * ps + (p % ps)[:, None], -1).int()
    x["slots"].copy_(torch.where(real[:, None], slot, x["slots"]))
    return {"table": table, "free": x["free"], "counts": x["counts"], "slots": x["slots"]}


def _turn(x, cos, sin, rotary, interleaved):
    """x [rows, heads, d] in fp32 with its first `rotary` dims turned; cos, sin [rows, 1, rotary / 2]."""
    head, rest = x[..., :rotary], x[..., rotary:]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
    else:
        a, b = head[..., :rotary // 2], head[..., rotary // 2:]
    u, v = a * cos - b * sin, b * cos + a * sin
    head = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((head, rest), -1)


def _store(pages, scale, new, slot):
    """New tokens [rows, heads, d] (32 bits) to the rows `slot` of the pool, and the blocks' scales; a slot past the
    pool's last row is nowhere."""
    n, d = pages.shape[0] * pages.shape[1], pages.shape[2]
    blocks = n // BLOCK
    block = slot // BLOCK
    amax = torch.zeros((blocks + 1,), device=DEVICE).scatter_reduce_(0, block.flatten(), new.abs().amax(-1).flatten(), "amax")
    first = torch.full((blocks + 1,), BLOCK, device=DEVICE).scatter_reduce_(0, block.flatten(), (slot % BLOCK).flatten(), "amin")
    amax, first = amax[:blocks], first[:blocks]
    old = torch.where(scale > 0, torch.frexp(scale)[1] - 1, LOWEST).flatten()       # 0: nothing is stored yet
    e = _exponent(amax)
    e = torch.where(first > 0, torch.maximum(e, old.clamp(LOWEST, HIGHEST)), e)
    e = torch.where(first < BLOCK, e, old)
    # the rows in front of a block's first new one, where its scale grows
    held = pages.view(blocks, BLOCK, d)
    front = (torch.arange(BLOCK, device=DEVICE) < first[:, None]) & (first < BLOCK)[:, None] & (e > old)[:, None]
    grown = _to8(held.float(), (e - old)[:, None, None])
    codes = torch.where(front[..., None], grown, held.view(torch.uint8)).view(n, d)
    codes = torch.cat((codes, codes[:1]))
    codes[slot] = _to8(new, torch.cat((e, e[:1]))[block][..., None])
    pages.view(torch.uint8).copy_(codes[:n].view(pages.shape))
    scale.copy_(torch.where(first < BLOCK, torch.ldexp(torch.ones_like(amax), e), scale.flatten()).view(scale.shape))


def _plain_append(x):
    case = x["case"]
    kp, ps = x["k_pages"], case["page"]
    b, p, real = _rows(x, x["q"].shape[0])
    q, k = x["q"].float(), x["k_new"].float()
    if x["inv_freq"] is not None:
        angle = p[:, None].double() * x["inv_freq"].double()    # far positions need more than 32 bits
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        q = _turn(q, cos, sin, case["rotary"], case["interleaved"])
        k = _turn(k, cos, sin, case["rotary"], case["interleaved"])
    x["out"].copy_(torch.where(real[:, None, None], q.to(torch.bfloat16), x["out"]))
    page = x["table"][b, :, torch.where(real, p // ps, 0)].long()                    # [rows, hkv]
    slot = torch.where(real[:, None] & (page >= 0), page * ps + (p % ps)[:, None], kp.shape[0] * ps)
    _store(kp, x["scales"][..., 0], k, slot)
    _store(x["v_pages"], x["scales"][..., 1], x["v_new"].float(), slot)
    return {"q": x["out"], "k_pages": kp, "v_pages": x["v_pages"], "scales": x["scales"]}


def _values(x, name, i, slot):
    """Rows of the pool as the numbers that they stand for, in 32 bits."""
    codes = x[name].view(torch.uint8).view(-1, x[name].shape[2])[slot].view(torch.float8_e4m3fn)
    return codes.float() * x["scales"].view(-1, 2)[slot // BLOCK, i][..., None]


def _plain_attention(x):
    case = x["case"]
    ps, d, hkv = case["page"], case["d"], case["hkv"]
    group = case["hq"] // hkv
    n = x["q"].shape[0]
    j = torch.arange(x["longest"], device=DEVICE)
    page = x["table"][:, :, j // ps]
    if case["prefix"]:
        page = torch.where(j < case["prefix"], x["prefix_table"][None][:, :, j // ps], page)
    slot = page.clamp(min=0).long() * ps + j % ps
    # the queries of each sequence, padded to the most that one has: [b, hkv, most * group, d]
    first = torch.arange(case["b"], device=DEVICE) if x["seq_start"] is None else x["seq_start"][:-1].long()
    t = torch.arange(x["most"], device=DEVICE)
    rows = (first[:, None] + t).clamp(max=n - 1)
    q = x["q"][rows].float().view(case["b"], x["most"], hkv, group, d).transpose(1, 2).reshape(case["b"], hkv, -1, d)
    p = (x["positions"].long()[:, None] + t)[:, None, :, None]                      # [b, 1, most, 1]
    seen = (j <= p) & ((j < case["sink"]) | (j >= _band_start(case, p, x["windows"][None, :, None, None])))
    seen &= (page >= 0)[:, :, None]
    sc = torch.matmul(q, _values(x, "k_pages", 0, slot).transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d))
    sc.view(case["b"], hkv, x["most"], group, -1).masked_fill_(~seen[:, :, :, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    sc.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = sc.sum(-1, keepdim=True)
    o = torch.matmul(sc, _values(x, "v_pages", 1, slot)) / torch.where(total > 0, total, 1.0)
    o = o.view(case["b"], hkv, x["most"], group, d).transpose(1, 2).reshape(case["b"], x["most"], hkv * group, d)
    b, at, real = _rows(x, n)
    o = o[b, torch.where(real, torch.arange(n, device=DEVICE) - first[b], 0)].to(torch.bfloat16)
    x["out"].copy_(torch.where(real[:, None, None], o, x["out"]))
    return {"o": x["out"]}


def _run_plain(x):
    kind = x["case"]["kind"]
    return _plain_assign(x) if kind == "assign" else _plain_append(x) if kind == "append" else _plain_attention(x)


# ---------------------------------------------------------------------------
# The same in 64 bits.
# ---------------------------------------------------------------------------
def _rotation(positions, inv_freq, rotary, d, interleaved):
    """[rows, d, d] fp64: the rotation of each row's position as a matrix."""
    angle = positions.double()[:, None] * inv_freq.double()
    m = torch.zeros((len(positions), d, d), dtype=torch.float64, device=DEVICE)
    i = torch.arange(rotary // 2, device=DEVICE)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    m[:, a, a], m[:, b, b] = angle.cos(), angle.cos()
    m[:, a, b], m[:, b, a] = -angle.sin(), angle.sin()
    rest = torch.arange(rotary, d, device=DEVICE)
    m[:, rest, rest] = 1.0
    return m


def _scale_of(amax):
    """Scale for the largest magnitude of each row of `amax` (numpy fp64)."""
    e = np.full(amax.shape, LOWEST)
    some = amax > 0
    e[some] = np.clip(np.ceil(np.log2(amax[some] / MOST)), LOWEST, HIGHEST)
    e -= (e > LOWEST) & (amax <= MOST * 2.0 ** (e - 1.0))            # the logarithm's last bits
    e += (e < HIGHEST) & (amax > MOST * 2.0 ** e)
    return 2.0 ** e


def _exact_append(case, x):
    """Codes of new rows are not rounded: what 8 bits make of them is the operator's error."""
    q = torch.zeros(x["q"].shape, dtype=torch.float64, device=DEVICE)
    pages = [x[n].double().view(-1, case["d"]) for n in ("k_pages", "v_pages")]
    scales = x["scales"].double().view(-1, 2)
    ps, hkv, d = case["page"], case["hkv"], case["d"]
    table = x["table"].cpu().numpy()
    row = 0
    for b, (p0, count) in enumerate(zip(*_sequences(case))):
        p0, count = int(p0), int(count)
        row, at = row + count, row
        while p0 >= 0 and at < row:                                   # up to the end of a block of 256 positions
            n = min(row - at, 256 - p0 % 256)
            rows, pos = slice(at, at + n), np.arange(p0, p0 + n)
            turned = [x[i][rows].double() for i in ("q", "k_new")]
            if case["rotary"]:
                m = _rotation(torch.from_numpy(pos).to(DEVICE), x["inv_freq"], case["rotary"], d, case["interleaved"])
                turned = [torch.matmul(t, m.transpose(1, 2).contiguous()) for t in turned]
            q[rows] = turned[0]
            starts = np.unique(np.maximum(pos // BLOCK * BLOCK, p0))
            slot = torch.from_numpy(table[b][:, pos // ps].astype(np.int64) * ps + pos % ps).to(DEVICE)     # [hkv, n]
            for which, new in enumerate((turned[1], x["v_new"][rows].double())):
                amax = np.maximum.reduceat(new.abs().amax(-1).cpu().numpy(), starts - p0, axis=0).T         # [hkv, blocks]
                sc = torch.from_numpy(_scale_of(amax)).to(DEVICE)
                block = slot[:, torch.from_numpy(starts - p0).to(DEVICE)] // BLOCK
                behind = int(starts[0]) % BLOCK                       # rows in front of the first new one
                if behind:
                    old = scales[block[:, 0], which]
                    sc[:, 0] = torch.maximum(sc[:, 0], old)
                    front = block[:, :1] * BLOCK + torch.arange(behind, device=DEVICE)
                    pages[which][front] *= (old / sc[:, 0])[:, None, None]
                scales[block, which] = sc
                pages[which][slot] = new.transpose(0, 1) / scales[slot // BLOCK, which][..., None]
            at, p0 = at + n, p0 + n
    return {"q": q, "k_pages": pages[0].view(x["k_pages"].shape), "v_pages": pages[1].view(x["v_pages"].shape),
            "scales": scales.view(x["scales"].shape)}


def _exact_attention(case, x):
    ps, s, d, hq, hkv = case["page"], case["sink"], case["d"], case["hq"], case["hkv"]
    group = hq // hkv
    o = torch.zeros(x["q"].shape, dtype=torch.float64, device=DEVICE)
    table = x["table"].cpu().numpy()
    shared = None if x["prefix_table"] is None else x["prefix_table"].cpu().numpy()
    scale = x["scales"].view(-1, 2).double()
    codes = [x[n].view(torch.uint8).view(-1, d) for n in ("k_pages", "v_pages")]
    windows = _windows(case)
    row = 0
    for b, (p0, count) in enumerate(zip(*_sequences(case))):
        p0, count = int(p0), int(count)
        for g, w in enumerate(windows if p0 >= 0 else []):
            # the positions that anything here sees, and where they are kept
            pos = np.concatenate([np.arange(a, z) for a, z in _seen(case, w, p0, p0 + count - 1)])
            page = table[b, g, pos // ps]
            if shared is not None:
                page = np.where(pos < case["prefix"], shared[g, pos // ps], page)
            slot = torch.from_numpy(page.astype(np.int64) * ps + pos % ps).to(DEVICE)
            k, v = [c[slot].view(torch.float8_e4m3fn).double() * scale[slot // BLOCK, i][:, None] for i, c in enumerate(codes)]
            kt = k.t().contiguous()
            pos = torch.from_numpy(pos).to(DEVICE)
            for i in range(0, count, 1024):
                p = torch.arange(p0 + i, p0 + min(count, i + 1024), device=DEVICE)[:, None]
                seen = (pos <= p) & ((pos < s) | (pos >= _band_start(case, p, w)))
                rows = slice(row + i, row + i + len(p))
                for h in range(g * group, (g + 1) * group):
                    sc = (x["q"][rows, h].double() @ kt / math.sqrt(d)).masked_fill_(~seen, -math.inf)
                    o[rows, h] = torch.softmax(sc, 1) @ v
        row += count
    return {"o": o}


def exact(case, seed):
    if case["kind"] == "assign":                    # whole numbers only
        return None
    x = _inputs(case, seed)
    return _exact_append(case, x) if case["kind"] == "append" else _exact_attention(case, x)
