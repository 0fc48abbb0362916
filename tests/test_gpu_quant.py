"""The 8-bit paged cache against the fp64 oracle.

Rows that no query sees, unused pages and rows of no sequence hold what is no number, their blocks odd
scales; table entries that no key needs hold numbers out of range or pages with nothing in them."""
import numpy as np
import pytest
import torch

import oracle
from helpers import bits
from oracle import quant_oracle as Q
from paged_cases import attention_bound
from paper_2406_14909_amd import moa as M
from quant_cases import QuantPaged

pytestmark = pytest.mark.gpu


def _say(*a):
    print("[case]", *a, flush=True)


def _u8(t):
    return t.view(torch.uint8).cpu().numpy()


# ---------------------------------------------------------------------------
# Append.
# ---------------------------------------------------------------------------
def _append(d, hq, hkv, positions, counts, page, rotary, interleaved, fused=False, with_q=True, pad=0, lead=0, seed=0,
            size=1.0, again=()):
    """`again`: further calls' counts of each sequence, behind the tokens that are there."""
    plan = M.moa_plan(hq, hkv, d, 4, 100, "bf16", [10.0] * hkv, [0.0] * hkv)
    gen = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    b, positions = len(positions), list(positions)
    steps = [counts, *again]
    total = [1 if counts is None else sum(c[i] for c in steps) for i in range(b)]
    width = max([p + n for p, n in zip(positions, total) if p >= 0] + [1]) // page + 1
    pages = sorted({(i, g, x) for i in range(b) for g in range(hkv) if positions[i] >= 0
                    for x in range(positions[i] // page, (positions[i] + total[i]) // page + 1)})
    lost = pages[2::7]                                # some pages are absent: their tokens are not stored
    n_pages = len(pages) + 2
    table = rng.choice(np.array([-1, -2 ** 31, 2 ** 31 - 1, n_pages], dtype=np.int64).astype(np.int32), (b, hkv, width))
    for where, n in zip(pages, rng.permutation(n_pages)):
        if where not in lost:
            table[where] = n
    # what is there: numbers and scales of all sizes, so that blocks grow and blocks do not
    codes = [rng.integers(0, 256, (n_pages * page, d)).astype(np.uint8) for _ in range(2)]
    scales = [2.0 ** rng.integers(-14, 2, n_pages * page // 16) for _ in range(2)]
    for s in scales:
        s[::5] = 0.0
    at = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    cache = [torch.from_numpy(c.reshape(n_pages, page, d)).cuda().view(torch.float8_e4m3fn) for c in codes]
    cache.append(torch.from_numpy(np.stack(scales, -1).astype(np.float32)).cuda().view(n_pages, page // 16, 2))
    f = None if not rotary else torch.tensor(10000.0 ** (-np.arange(rotary // 2) * 2.0 / rotary), dtype=torch.float32)
    inv = np.zeros(0) if f is None else f.double().numpy()
    for step, count in enumerate(steps):
        seq_start = None if count is None else [lead] + [lead + int(x) for x in np.cumsum(count)]
        rows = b if count is None else seq_start[-1] + pad
        # one row in three is of another size, so that scales differ from block to block
        qkv = (torch.randn(rows, hq + 2 * hkv, d, generator=gen) * size
               * torch.from_numpy(2.0 ** (rng.integers(0, 3, (rows, 1, 1)) * 2 - 2))).bfloat16()
        cut = lambda a, z: qkv[:, a:z] if fused else qkv[:, a:z].contiguous()
        q, k, v = cut(0, hq), cut(hq, hq + hkv), cut(hq + hkv, hq + 2 * hkv)
        dev = qkv.cuda()
        gq, gk, gv = ((dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:]) if fused else (q.cuda(), k.cuda(), v.cuda()))
        out = torch.full((rows, hq, d), 7.0, dtype=torch.bfloat16, device="cuda") if with_q else None
        before = [_u8(c).reshape(-1, d).copy() for c in cache[:2]]
        got = M.moa_quant_append(plan, *cache, at(table), gq if with_q else None, gk, gv, at(positions), at(seq_start),
                                 None if f is None else f.cuda(), interleaved, q_out=out)
        torch.cuda.synchronize()
        assert got is out
        tokens = oracle.token_rows(positions, seq_start)
        turn = lambda x: oracle.rotate_ref(x.double().numpy()[[r for r, _, _ in tokens]], [p for _, _, p in tokens], inv,
                                           interleaved)
        # two products and their sum, of sines and cosines that are rounded: five half steps of both magnitudes
        off = lambda x: 5 * 2.0 ** -24 * 2 * np.abs(x.double().numpy()).max()
        if with_q:
            ref, o = turn(q), out.double().cpu().numpy()
            mine = np.zeros(rows, bool)
            for i, (r, _, _) in enumerate(tokens):
                mine[r] = True
                assert (np.abs(o[r] - ref[i]) <= off(q) + 2.0 ** -8 * np.abs(ref[i])).all(), ("q", r)
                if not rotary:
                    assert torch.equal(bits(out[r]), bits(q[r]))
            assert (o[~mine] == 7.0).all()
        kref = turn(k)
        now, sc = [_u8(c).reshape(-1, d) for c in cache[:2]], cache[2].cpu().double().numpy().reshape(-1, 2)
        for i in range(b):
            mine = [(n, r, p) for n, (r, j, p) in enumerate(tokens) if j == i]
            for g in range(hkv if mine else 0):
                slots = [oracle.slot_ref(table, n_pages, page, i, g, p) for _, _, p in mine]
                for which, new in enumerate((np.stack([kref[n, g] for n, _, _ in mine]),
                                             np.stack([v[r, g].double().numpy() for _, r, _ in mine]))):
                    want, wsc = codes[which].copy(), scales[which].copy()
                    Q.store_ref(want, wsc, new, slots)
                    touched = sorted({s // 16 for s in slots if s >= 0})
                    rotated = rotary and which == 0
                    for s in touched:
                        if rotated and sc[s, which] != wsc[s]:        # the largest one at a scale's border
                            x = np.abs(new[[n for n, t in enumerate(slots) if t >= 0 and t // 16 == s]]).max()
                            assert sc[s, which] in (2.0 ** Q.exponent_ref(x - off(k)), 2.0 ** Q.exponent_ref(x + off(k)))
                            wsc[s] = sc[s, which]
                        assert sc[s, which] == wsc[s], ("scale", i, g, which)
                    if rotated:
                        for n, t in enumerate(slots):
                            if t >= 0:
                                err = np.abs(Q.decode_ref(now[0][t]) * wsc[t // 16] - new[n])
                                assert (err <= np.maximum(2.0 ** -4 * np.abs(new[n]), 2.0 ** -10 * wsc[t // 16])
                                        + 2 * off(k)).all(), ("k", i, g, n)
                                want[t] = now[0][t]
                    codes[which], scales[which] = want, wsc
        for which in range(2):                     # every other row and scale as it was, or as rescaled
            # of a block's rows behind the new ones nothing is said, but they are left as they were here
            x, y = now[which], codes[which]
            nan = (x & 0x7F == 0x7F) & (y & 0x7F == 0x7F)
            assert ((x == y) | nan).all(), ("codes", which, int(((x != y) & ~nan).sum()))
            assert np.array_equal(sc[:, which], scales[which])
        if count is not None:
            positions = [p if p < 0 else p + c for p, c in zip(positions, count)]


@pytest.mark.parametrize("d,hq,hkv", [(64, 3, 3), (128, 8, 2), (128, 64, 8), (64, 1, 1)])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (16, False), (32, True), (64, False), (64, True)])
def test_append_one_token_each(d, hq, hkv, rotary, interleaved):
    _say("append step", d, hq, hkv, rotary, interleaved)
    _append(d, hq, hkv, [0, 15, -1, 16, 4095, 1, 63], None, 16, rotary, interleaved)


@pytest.mark.parametrize("counts", [[1], [5, 0, 1, 33, 0], [0, 0], [400, 1, 300]])
@pytest.mark.parametrize("fused", [False, True])
def test_append_packed_tokens(counts, fused):
    _say("append packed", counts, fused)
    starts = [0, 7, 300, 15, -1][:len(counts)]
    _append(128, 4, 2, starts, counts, 32, 128, False, fused, pad=3, lead=2)
    _append(64, 2, 2, starts, counts, 256, 64, True, fused, with_q=False)
    _append(128, 8, 4, starts, counts, 16, 0, False, fused, lead=17, seed=4)


def test_append_block_by_block():
    """The same sequences token by token and chunk by chunk: scales grow inside blocks."""
    _say("append again")
    _append(128, 2, 2, [3, 0, 14, -1], [2, 1, 1, 0], 16, 0, False, again=[[1, 1, 1, 0], [17, 5, 0, 0], [1, 1, 1, 0], [40, 1, 16, 0]])
    _append(64, 2, 1, [3, 30], [1, 1], 32, 64, False, again=[[1, 3]] * 12)


def test_append_far_positions():
    _say("append far")
    for inter in (False, True):
        _append(128, 2, 1, [1000003, 999990], [3, 20], 256, 128, inter)


def test_append_many_sequences():
    """More sequences than one wave probes at once, most of them empty."""
    _say("append many")
    rng = np.random.default_rng(0)
    counts = rng.choice([0, 0, 0, 1, 2], size=1500)
    starts = [int(x) for x in rng.integers(-3, 20, size=1500)]
    _append(64, 1, 1, starts, counts, 16, 64, False, pad=1)
    _append(64, 1, 1, starts[:3] + [0] * 300 + [5], [100, 0, 70] + [0] * 300 + [40], 16, 0, False)


@pytest.mark.parametrize("size", [2.0 ** -130, 2.0 ** -100, 2.0 ** 100, 2.0 ** 121])
def test_append_sizes(size):
    """Numbers near the ends of bf16: scales at their ends, numbers that become zeros and the largest one."""
    _say("append sizes", size)
    _append(64, 2, 2, [0, 20], [40, 3], 16, 0, False, size=size)


def test_append_what_is_not_finite():
    """NaN and infinities are stored as NaN and do not count for the scale; a growing block keeps them."""
    _say("append not finite")
    plan = M.moa_plan(1, 1, 64, 0, 100, "bf16", [10.0], [0.0])
    kp, vp, sc = M.new_quant_cache(plan, 2, 16)
    table = torch.tensor([[[1, 0]]], dtype=torch.int32, device="cuda")
    at = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    k = torch.zeros((3, 1, 64), dtype=torch.bfloat16, device="cuda")
    k[0, 0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.75])
    M.moa_quant_append(plan, kp, vp, sc, table, None, k, k, at(0), at(0, 3))
    for p, i in ((kp, 0), (vp, 1)):
        x = p.float().cpu()
        assert torch.isnan(x[1, 0, :3]).all() and x[1, 0, 3] == 448 and torch.isfinite(x[1, 1:]).all()
        assert sc[1, 0, i].item() == 2.0 ** -8
    k[0, 0] = 7.0
    M.moa_quant_append(plan, kp, vp, sc, table, None, k[:1], k[:1], at(1), at(0, 1))
    for p, i in ((kp, 0), (vp, 1)):
        x = p.float().cpu()
        assert torch.isnan(x[1, 0, :3]).all() and x[1, 0, 3] == 112 and sc[1, 0, i].item() == 2.0 ** -6
        assert (x[1, 1] == 448).all()


def test_append_in_place_and_past_the_table():
    _say("append in place")
    plan = M.moa_plan(4, 2, 128, 0, 100, "bf16", [10.0] * 2, [0.0] * 2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((3, 4, 128), generator=gen, device="cuda").bfloat16()
    k, v = torch.randn((2, 3, 2, 128), generator=gen, device="cuda").bfloat16()
    f = torch.logspace(0, -3, 64, device="cuda")
    at = torch.tensor([40, 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 2, 2)        # 32 positions
    cache = M.new_quant_cache(plan, 12, 16)
    ref = M.moa_quant_append(plan, *cache, table, q, k, v, at, inv_freq=f)
    hit = (cache[1].float() != 0).any(2).nonzero().tolist()
    assert hit == [[5, 15], [7, 15]]
    same = q.clone()
    assert M.moa_quant_append(plan, *cache, table, same, k, v, at, inv_freq=f, q_out=same) is same
    assert torch.equal(same, ref) and not torch.equal(ref, q)


def test_append_of_rows_in_front_of_the_tensors():
    """A sequence whose first rows are in front of the tensors is stored from row 0 on, like one that starts there."""
    _say("append rows in front")
    plan = M.moa_plan(4, 2, 128, 0, 100, "bf16", [10.0] * 2, [0.0] * 2)
    gen = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn((9, 4, 128), generator=gen, device="cuda").bfloat16()
    k, v = torch.randn((2, 9, 2, 128), generator=gen, device="cuda").bfloat16()
    f = torch.logspace(0, -3, 64, device="cuda")
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 2, 2)
    at = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for p0 in (0, 10, 14):                       # row 0 within a block, and past one's end
        caches = [M.new_quant_cache(plan, 8, 16) for _ in range(2)]
        out = [torch.full_like(q, 7.0) for _ in range(2)]
        M.moa_quant_append(plan, *caches[0], table, q, k, v, at(p0 + 3, 2), at(0, 5, 9), f, q_out=out[0])
        M.moa_quant_append(plan, *caches[1], table, q, k, v, at(p0, 2), at(-3, 5, 9), f, q_out=out[1])
        assert torch.equal(*out) and not (out[0] == 7.0).all(2).any()
        for a, b in zip(*caches):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


# ---------------------------------------------------------------------------
# Attention.
# ---------------------------------------------------------------------------
LAYERS = [(3, 3, 64), (2, 2, 128), (4, 2, 64), (4, 2, 128), (8, 2, 64), (4, 1, 128), (8, 1, 64), (16, 2, 128)]
WINDOWS = [[1, 700, 40], [130, 17], [3000, 64]]


def _windows(hkv, i):
    return (WINDOWS[i % len(WINDOWS)] * 3)[:hkv]


@pytest.mark.parametrize("d", [64, 128])
def test_every_number_and_scale_comes_out_as_it_is(d):
    """With one visible key the output is its value, whatever it is; NaN stays NaN."""
    _say("all codes", d)
    exponents = [-117, -100, -9, -1, 0, 1, 7, 60, 118, 119]
    b = 256 * len(exponents) // d
    plan = M.moa_plan(1, 1, d, 0, 100, "bf16", [1.0], [0.0])
    codes = torch.arange(256, dtype=torch.uint8).repeat(len(exponents)).view(b, 1, d)
    scale = torch.tensor([2.0 ** e for e in exponents]).repeat_interleave(256 // d)
    rows = torch.zeros((b, 16, d), dtype=torch.uint8)
    rows[:, 5] = codes[:, 0]
    sc = torch.ones((b, 1, 2))
    sc[:, 0, 1] = scale
    pages = rows.cuda().view(torch.float8_e4m3fn)
    table = torch.arange(b, dtype=torch.int32, device="cuda").view(b, 1, 1)
    at = torch.full((b,), 5, dtype=torch.int32, device="cuda")
    q = torch.ones((b, 1, d), dtype=torch.bfloat16, device="cuda")
    ws = M.new_paged_workspace(plan, b)
    want = Q.decode_ref(codes[:, 0].numpy()) * scale[:, None].double().numpy()
    zero = torch.zeros((b, 16, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    start = torch.arange(b + 1, dtype=torch.int32, device="cuda")
    for o in (M.moa_quant_decode(plan, q, zero, pages, sc.cuda(), table, at, ws),
              M.moa_quant_prefill(plan, q, zero, pages, sc.cuda(), table, at, start, ws)):
        assert np.array_equal(o[:, 0].double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("i", range(len(LAYERS)))
@pytest.mark.parametrize("page,s", [(16, 0), (64, 4), (256, 70)])
def test_decode(i, page, s):
    hq, hkv, d = LAYERS[i]
    for w in range(2):
        _say("decode", LAYERS[i], page, s, w)
        c = QuantPaged(hq, hkv, d, s, _windows(hkv, i + w), "bf16", [0, 1, -1, 15, 16, 63, 300, 1500, s, 129], page=page, seed=i)
        c.check(f"decode {LAYERS[i]} {page} {s}")


@pytest.mark.parametrize("i", range(len(LAYERS)))
@pytest.mark.parametrize("page,s,flags", [(16, 0, 0), (32, 4, 2), (64, 70, 0), (128, 5, 3), (256, 64, 1)])
def test_prefill(i, page, s, flags):
    hq, hkv, d = LAYERS[i]
    _say("prefill", LAYERS[i], page, s, flags)
    c = QuantPaged(hq, hkv, d, s, _windows(hkv, i), "bf16", [0, 3, 5, 63, 200, -1, 0], [130, 1, 0, 65, 33, 4, 7], page=page,
                   flags=flags, seed=i, pad=3, lead=1)
    c.check(f"prefill {LAYERS[i]} {page} {s} {flags}")


@pytest.mark.parametrize("i", range(len(LAYERS)))
@pytest.mark.parametrize("page,s,prefix", [(16, 0, 100), (64, 4, 1), (32, 70, 64), (256, 70, 500), (16, 4, 1203)])
def test_shared(i, page, s, prefix):
    hq, hkv, d = LAYERS[i]
    _say("shared", LAYERS[i], page, s, prefix)
    where = [prefix, prefix + 1, -1, max(0, prefix - 1), prefix // 2, prefix + 40, 0, prefix + 333, prefix + 16]
    c = QuantPaged(hq, hkv, d, s, _windows(hkv, i), "bf16", where, page=page, prefix_len=prefix, seed=i)
    c.check(f"shared {LAYERS[i]} {page} {s} {prefix}")


def test_shared_by_many_sequences():
    _say("shared many")
    rng = np.random.default_rng(5)
    where = [int(x) for x in 700 + rng.integers(0, 300, size=37)]
    QuantPaged(16, 2, 128, 20, [250, 900], "bf16", where, page=32, prefix_len=700, seed=2).check("shared many")
    QuantPaged(3, 3, 64, 0, [5, 290, 2000], "bf16", where, page=16, prefix_len=700, seed=3).check("shared many mha")


def test_shared_without_a_prefix():
    _say("shared, prefix of 0")
    c = QuantPaged(4, 2, 128, 4, [100, 20], "bf16", [0, 50, 200], seed=1)
    x, ref = c.device(), c.run()
    o = M.moa_quant_decode_shared(c.plan, x["q"], x["k_pages"], x["v_pages"], x["scales"], x["prefix_table"], 0, x["table"],
                                  x["positions"], x["workspace"])
    assert torch.equal(o, ref)


def test_absent_pages_are_not_seen():
    _say("absent")
    gone = [(0, 0, 3), (0, 1, 0), (0, 1, 9)] + [(1, g, x) for g in range(2) for x in range(10)]
    for hq in (2, 8):
        c = QuantPaged(hq, 2, 128, 20, [100, 1000], "bf16", [155, 150, 40], page=16, absent=gone, seed=4)
        o = c.run()
        assert (o[1] == 0).all()
        c.check("absent decode")
        c = QuantPaged(hq, 2, 64, 20, [100, 1000], "bf16", [60, 0, 31], [95, 30, 1], page=16,
                       absent=gone + [(2, 0, 1), (2, 0, 0)], seed=5)
        o = c.run()
        assert (o[95:125] == 0).all()
        c.check("absent prefill")
    c = QuantPaged(8, 2, 128, 4, [2000, 90], "bf16", [300, 331, 302], page=16, prefix_len=300, seed=6)
    c.prefix_table[0, 3:7] = [-1, 2 ** 31 - 1, c.num_pages, -2 ** 31]
    c.prefix_table[1] = -7
    c.check("absent prefix")


def test_long_caches():
    """Lengths whose work is cut into many pieces, for one sequence and several."""
    for hq, hkv, d in ((2, 2, 128), (4, 1, 128), (8, 1, 64)):
        _say("long", hq, hkv, d)
        w = [9000, 5000][:hkv]
        QuantPaged(hq, hkv, d, 33, w, "bf16", [20000, 7003], page=64, seed=7).check("long decode")
        QuantPaged(hq, hkv, d, 33, w, "bf16", [12000, 7003], [9, 40], page=16, seed=8).check("long prefill")
        QuantPaged(hq, hkv, d, 33, w, "bf16", [11003, 11500, 12000], page=128, prefix_len=11000, seed=9).check("long shared")


def test_scale_and_large_scores():
    _say("scale")
    for counts in (None, [40]):
        QuantPaged(4, 2, 64, 3, [60, 300], "bf16", [200], counts, page=32, scale=0.05, seed=10).check("scale")
        c = QuantPaged(4, 2, 64, 3, [60, 300], "bf16", [200], counts, page=32, scale=4.0, seed=11)
        c.q *= 0.25
        c.check("large scores")


def test_positions_past_the_table():
    _say("past the table")
    far = [2 ** 31 - 1, 160, 2 ** 30, 139, 500]
    for counts, prefix in ((None, 0), (None, 100), ([1, 40, 3, 9, 2], 0)):
        c = QuantPaged(4, 2, 64, 20, [50, 130], "bf16", [130, 120, 125, 110, 115], counts, page=16, prefix_len=prefix, seed=12)
        c.width = 9                                # 144 positions, with all of which the pages are filled
        c.table, c.prefix_table = c.table[:, :, :9].copy(), c.prefix_table[:, :9].copy()
        c.table[:, :, :] = np.random.default_rng(13).integers(0, c.num_pages, c.table.shape)
        c.prefix_table[:, :] = c.table[0]
        gen = torch.Generator().manual_seed(14)
        c.k, c.v = (torch.randn(c.k.shape, generator=gen).to(c.dtype) for _ in range(2))
        c.positions = far
        c.check(f"past the table {counts} {prefix}")


# ---------------------------------------------------------------------------
# What is no number reaches the rows that see it, and no other.
# ---------------------------------------------------------------------------
def _poison(c, seed, keys_too):
    rng = np.random.default_rng(seed)
    rows = oracle.token_rows(c.positions, c.seq_start)
    d, block = c.q.shape[2], c.block if c.seq_start is not None else 0
    for i in sorted({b for _, b, _ in rows}):
        own = [p for _, b, p in rows if b == i]
        for g, w in enumerate(c.windows):
            first, last = oracle.visible_set(own[0], w, c.s, block), oracle.visible_set(own[-1], w, c.s, block)
            band = first[first >= c.s]
            picks = {int(own[len(own) // 2]), int(own[-1]), int(rng.choice(first)), int(rng.choice(last))}
            picks |= {int(band[0])} if len(band) else set()
            for n, j in enumerate(sorted(picks)):
                row = oracle.slot_ref(c.table if j >= c.prefix_len else c.prefix_table[None], c.num_pages, c.page,
                                      i if j >= c.prefix_len else 0, g, j)
                if row >= 0:
                    at = (row // c.page, row % c.page)
                    c.v[at][rng.choice(d, 3, replace=False)] = float("nan")
                    if keys_too and n == 1:
                        c.k[at][int(rng.integers(d))] = float("nan")


def _check_values(c):
    got = c.run().double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        ref, a, s = c.reference(keep_nan=True)
    rows = [t for t, _, _ in oracle.token_rows(c.positions, c.seq_start)]
    got, ref, a, s = got[rows], ref[rows], a[rows], s[rows]
    sound = np.isfinite(ref)
    assert not sound.all()
    assert not np.isfinite(got[~sound]).any(), "a row lost what it sees"
    assert np.isfinite(got[sound]).all(), f"{(~np.isfinite(got[sound])).sum()} of {sound.sum()} values are no numbers"
    bound = attention_bound(ref, a, s, c.dtype, c.q.shape[2], max(1, c.width * c.page))
    assert (np.abs(got[sound] - ref[sound]) <= bound[sound]).all()
    return sound.mean()


PREFILL = [
    (1, 1, 128, 4, (40,), (0,), (90,), 16, 0),
    (4, 2, 128, 0, (30, 700), (100, -1, 7), (70, 5, 300), 32, 0),
    (8, 2, 64, 3, (1, 200), (0, 33), (129, 64), 16, 0),
    (8, 1, 128, 16, (1500,), (1700,), (24,), 64, 0),
    (2, 2, 64, 4, (900, 64), (0, 40), (1100, 30), 128, 2),
    (4, 4, 128, 4, (64, 128, 600, 2500), (0,), (2700,), 16, 0),
]


@pytest.mark.parametrize("keys_too", [0, 1])
@pytest.mark.parametrize("n", range(len(PREFILL)))
def test_prefill_values_reach_only_the_rows_that_see_them(n, keys_too):
    hq, hkv, d, s, windows, positions, counts, page, flags = PREFILL[n]
    _say("values", n, keys_too)
    c = QuantPaged(hq, hkv, d, s, windows, "bf16", positions, counts, page, flags, seed=n)
    _poison(c, n, keys_too)
    share = _check_values(c)
    assert share > 0.5 or keys_too       # a key that is NaN takes whole rows, of few rows it may take all


@pytest.mark.parametrize("prefix", [0, 200])
def test_decode_values_reach_only_the_sequences_that_see_them(prefix):
    _say("values", prefix)
    c = QuantPaged(8, 2, 128, 3, (50, 180), "bf16", (230, 199, 210, -1, 120, 330, 205, 60), page=16, prefix_len=prefix, seed=3)
    _poison(c, 5, 0)
    assert _check_values(c) > 0.5
