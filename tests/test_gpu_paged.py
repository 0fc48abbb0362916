"""The paged operators against the fp64 oracle.

Rows that no query sees, unused pages and rows of no sequence hold NaN; table entries that no
key needs hold numbers out of range or pages with nothing in them."""
import numpy as np
import pytest
import torch

import oracle
from helpers import bits
from paged_cases import Paged, rotation_bound
from paper_2406_14909_amd import moa as M

pytestmark = pytest.mark.gpu


def _say(*a):
    print("[case]", *a, flush=True)


# ---------------------------------------------------------------------------
# Append.
# ---------------------------------------------------------------------------
def _append(dt, d, hq, hkv, positions, counts, page, rotary, interleaved, fused=False, with_q=True, pad=0, lead=0, seed=0):
    plan = M.moa_plan(hq, hkv, d, 4, 100, dt, [10.0] * hkv, [0.0] * hkv)
    t = plan.torch_dtype
    gen = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    draw = lambda *shape: torch.randn(shape, generator=gen).to(t)
    b = len(positions)
    seq_start = None if counts is None else [lead] + [lead + int(x) for x in np.cumsum(counts)]
    rows = b if counts is None else seq_start[-1] + pad
    tokens = oracle.token_rows(positions, seq_start)
    width = max([p for _, _, p in tokens] + [0]) // page + 1
    pages = sorted({(i, g, p // page) for _, i, p in tokens for g in range(hkv)})
    lost = pages[2::7]                                # some pages are absent: their tokens are not stored
    n_pages = len(pages) + 2
    table = rng.choice(np.array([-1, -2 ** 31, 2 ** 31 - 1, n_pages], dtype=np.int64).astype(np.int32), (b, hkv, width))
    for where, n in zip(pages, rng.permutation(n_pages)):
        if where not in lost:
            table[where] = n
    kp, vp = draw(n_pages, page, d), draw(n_pages, page, d)
    qkv = draw(rows, hq + 2 * hkv, d)
    cut = lambda a, z: qkv[:, a:z] if fused else qkv[:, a:z].contiguous()
    q, k, v = cut(0, hq), cut(hq, hq + hkv), cut(hq + hkv, hq + 2 * hkv)
    if fused:
        dev = qkv.cuda()
        gq, gk, gv = dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:]
    else:
        gq, gk, gv = q.cuda(), k.cuda(), v.cuda()
    f = None if not rotary else torch.tensor(10000.0 ** (-np.arange(rotary // 2) * 2.0 / rotary), dtype=torch.float32)
    at = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    gkp, gvp = kp.cuda(), vp.cuda()
    out = torch.full((rows, hq, d), 7.0, dtype=t, device="cuda") if with_q else None
    got = M.moa_paged_append(plan, gkp, gvp, at(table), gq if with_q else None, gk, gv, at(positions), at(seq_start),
                             None if f is None else f.cuda(), interleaved, q_out=out)
    torch.cuda.synchronize()
    assert got is out
    inv = np.zeros(0) if f is None else f.double().numpy()
    turn = lambda x: oracle.rotate_ref(x.double().numpy()[[r for r, _, _ in tokens]], [p for _, _, p in tokens], inv,
                                       interleaved)
    mag = lambda x: np.abs(x.double().numpy()).max(axis=2, keepdims=True)
    if with_q:
        ref, o = turn(q), out.double().cpu().numpy()
        mine = np.zeros(rows, bool)
        for i, (r, _, _) in enumerate(tokens):
            mine[r] = True
            assert (np.abs(o[r] - ref[i]) <= rotation_bound(mag(q)[r], mag(q)[r], ref[i], t)).all(), ("q", r)
            if not rotary:
                assert torch.equal(bits(out[r]), bits(q[r]))
        assert (o[~mine] == 7.0).all()
    kref, left = turn(k), torch.ones((n_pages * page,), dtype=torch.bool)
    ko, vo = gkp.cpu().view(-1, d), gvp.cpu().view(-1, d)
    stored = 0
    for i, (r, b_, p) in enumerate(tokens):
        for g in range(hkv):
            slot = oracle.slot_ref(table, n_pages, page, b_, g, p)
            if slot < 0:
                continue
            stored += 1
            left[slot] = False
            assert torch.equal(bits(vo[slot]), bits(v[r, g])), ("v", r, g)
            err = np.abs(ko[slot].double().numpy() - kref[i, g])
            assert (err <= rotation_bound(mag(k)[r, g], mag(k)[r, g], kref[i, g], t)).all(), ("k", r, g)
            if not rotary:
                assert torch.equal(bits(ko[slot]), bits(k[r, g]))
    assert stored or not tokens
    assert torch.equal(bits(ko[left]), bits(kp.view(-1, d)[left])) and torch.equal(bits(vo[left]), bits(vp.view(-1, d)[left]))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,hq,hkv", [(64, 3, 3), (128, 8, 2), (128, 64, 8), (64, 1, 1)])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (16, False), (32, True), (64, False), (64, True)])
def test_append_one_token_each(dt, d, hq, hkv, rotary, interleaved):
    _say("append step", dt, d, hq, hkv, rotary, interleaved)
    _append(dt, d, hq, hkv, [0, 15, -1, 16, 4095, 1, 63], None, 16, rotary, interleaved)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[1], [5, 0, 1, 33, 0], [0, 0], [700, 1, 1400]])
@pytest.mark.parametrize("fused", [False, True])
def test_append_packed_tokens(dt, counts, fused):
    _say("append packed", dt, counts, fused)
    starts = [0, 7, 300, 15, -1][:len(counts)]
    _append(dt, 128, 4, 2, starts, counts, 32, 128, False, fused, pad=3, lead=2)
    _append(dt, 64, 2, 2, starts, counts, 256, 64, True, fused, with_q=False)


def test_append_far_positions():
    """Angles of positions near a million: what fp32 angles would get wrong by a tenth."""
    _say("append far")
    for dt in ("bf16", "f32"):
        for inter in (False, True):
            _append(dt, 128, 2, 1, [1000003, 999990], [3, 20], 256, 128, inter)


def test_append_many_sequences():
    """More sequences than one wave probes at once, most of them empty."""
    _say("append many")
    rng = np.random.default_rng(0)
    counts = rng.choice([0, 0, 0, 1, 2], size=5000)
    _append("bf16", 64, 1, 1, [int(x) for x in rng.integers(-3, 20, size=5000)], counts, 16, 64, False, pad=1)


def test_append_in_place_and_past_the_table():
    _say("append in place")
    plan = M.moa_plan(4, 2, 128, 0, 100, "bf16", [10.0] * 2, [0.0] * 2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn((3, 4, 128), generator=gen, device="cuda").bfloat16()
    k, v = torch.randn((2, 3, 2, 128), generator=gen, device="cuda").bfloat16()
    f = torch.logspace(0, -3, 64, device="cuda")
    at = torch.tensor([40, 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 2, 2)        # 32 positions
    kp, vp = M.new_paged_cache(plan, 12, 16)
    ref = M.moa_paged_append(plan, kp, vp, table, q, k, v, at, inv_freq=f)
    hit = (vp != 0).any(2).nonzero().tolist()
    assert hit == [[5, 15], [7, 15]] and torch.equal(vp[5, 15], v[1, 0])
    same = q.clone()
    assert M.moa_paged_append(plan, kp, vp, table, same, k, v, at, inv_freq=f, q_out=same) is same
    assert torch.equal(same, ref) and not torch.equal(ref, q)


# ---------------------------------------------------------------------------
# Attention.
# ---------------------------------------------------------------------------
LAYERS = [(3, 3, 64), (2, 2, 128), (4, 2, 64), (4, 2, 128), (8, 2, 64), (4, 1, 128), (8, 1, 64), (16, 2, 128)]
WINDOWS = [[1, 700, 40], [130, 17], [3000, 64]]


def _windows(hkv, i):
    return (WINDOWS[i % len(WINDOWS)] * 3)[:hkv]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(LAYERS)))
@pytest.mark.parametrize("page,s", [(16, 0), (64, 4), (256, 70)])
def test_decode(dt, i, page, s):
    hq, hkv, d = LAYERS[i]
    for w in range(2):
        _say("decode", dt, LAYERS[i], page, s, w)
        c = Paged(hq, hkv, d, s, _windows(hkv, i + w), dt, [0, 1, -1, 15, 16, 63, 300, 1500, s, 129], page=page, seed=i)
        c.check(f"decode {dt} {LAYERS[i]} {page} {s}")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(LAYERS)))
@pytest.mark.parametrize("page,s,flags", [(16, 0, 0), (32, 4, 2), (64, 70, 0), (128, 5, 3), (256, 64, 1)])
def test_prefill(dt, i, page, s, flags):
    hq, hkv, d = LAYERS[i]
    _say("prefill", dt, LAYERS[i], page, s, flags)
    c = Paged(hq, hkv, d, s, _windows(hkv, i), dt, [0, 3, 5, 63, 200, -1, 0], [130, 1, 0, 65, 33, 4, 7], page=page,
              flags=flags, seed=i, pad=3, lead=1)
    c.check(f"prefill {dt} {LAYERS[i]} {page} {s} {flags}")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(LAYERS)))
@pytest.mark.parametrize("page,s,prefix", [(16, 0, 100), (64, 4, 1), (32, 70, 64), (256, 70, 500), (16, 4, 1203)])
def test_shared(dt, i, page, s, prefix):
    hq, hkv, d = LAYERS[i]
    _say("shared", dt, LAYERS[i], page, s, prefix)
    where = [prefix, prefix + 1, -1, max(0, prefix - 1), prefix // 2, prefix + 40, 0, prefix + 333, prefix + 16]
    c = Paged(hq, hkv, d, s, _windows(hkv, i), dt, where, page=page, prefix_len=prefix, seed=i)
    c.check(f"shared {dt} {LAYERS[i]} {page} {s} {prefix}")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_shared_by_many_sequences(dt):
    """More query rows than one tile; windows that end in front of the prefix's end for some sequences."""
    _say("shared many", dt)
    rng = np.random.default_rng(5)
    where = [int(x) for x in 700 + rng.integers(0, 300, size=37)]
    Paged(16, 2, 128, 20, [250, 900], dt, where, page=32, prefix_len=700, seed=2).check(f"shared many {dt}")
    Paged(3, 3, 64, 0, [5, 290, 2000], dt, where, page=16, prefix_len=700, seed=3).check(f"shared many mha {dt}")


def test_shared_without_a_prefix():
    _say("shared, prefix of 0")
    c = Paged(4, 2, 128, 4, [100, 20], "bf16", [0, 50, 200], seed=1)
    x, ref = c.device(), c.run()
    o = M.moa_paged_decode_shared(c.plan, x["q"], x["k_pages"], x["v_pages"], x["prefix_table"], 0, x["table"],
                                  x["positions"], x["workspace"])
    r, a, s = c.reference()
    assert np.abs((o - ref).double().cpu().numpy()).max() <= 2.0 ** -6 * np.abs(r).max()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_absent_pages_are_not_seen(dt):
    """A page of a decode's window is gone, all pages of another sequence's heads are; in a
    prefill, pages inside, at the start and at the end of what its rows see."""
    _say("absent", dt)
    gone = [(0, 0, 3), (0, 1, 0), (0, 1, 9)] + [(1, g, x) for g in range(2) for x in range(10)]
    for hq in (2, 8):
        c = Paged(hq, 2, 128, 20, [100, 1000], dt, [155, 150, 40], page=16, absent=gone, seed=4)
        o = c.run()
        assert (o[1] == 0).all()
        c.check(f"absent decode {dt}")
        c = Paged(hq, 2, 64, 20, [100, 1000], dt, [60, 0, 31], [95, 30, 1], page=16,
                  absent=gone + [(2, 0, 1), (2, 0, 0)], seed=5)
        o = c.run()
        assert (o[95:125] == 0).all()
        c.check(f"absent prefill {dt}")


def test_absent_prefix_pages():
    _say("absent prefix")
    for dt in ("bf16", "f32"):
        c = Paged(8, 2, 128, 4, [2000, 90], dt, [300, 331, 302], page=16, prefix_len=300, seed=6)
        c.prefix_table[0, 3:7] = [-1, 2 ** 31 - 1, c.num_pages, -2 ** 31]
        c.prefix_table[1] = -7
        c.check(f"absent prefix {dt}")


def test_long_caches():
    """Lengths whose work is cut into many pieces, for one sequence and several."""
    for dt, hq, hkv, d in (("bf16", 2, 2, 128), ("bf16", 4, 1, 128), ("bf16", 8, 1, 64), ("f32", 2, 1, 64)):
        _say("long", dt, hq, hkv, d)
        w = [9000, 5000][:hkv]
        Paged(hq, hkv, d, 33, w, dt, [20000, 7003], page=64, seed=7).check("long decode")
        Paged(hq, hkv, d, 33, w, dt, [12000, 7003], [9, 40], page=16, seed=8).check("long prefill")
        Paged(hq, hkv, d, 33, w, dt, [11003, 11500, 12000], page=128, prefix_len=11000, seed=9).check("long shared")


def test_scale_and_large_scores():
    """A scale of one's own, and scores whose exponentials overflow without a running maximum."""
    _say("scale")
    for counts in (None, [40]):
        for dt in ("bf16", "f32"):
            c = Paged(4, 2, 64, 3, [60, 300], dt, [200], counts, page=32, scale=0.05, seed=10)
            c.check("scale")
            c = Paged(4, 2, 64, 3, [60, 300], dt, [200], counts, page=32, scale=4.0, seed=11)
            c.q *= 0.25
            c.check("large scores")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_positions_past_the_table(dt):
    """Keys past the table are absent: a row there sees the sinks and what the table holds of its band."""
    _say("past the table", dt)
    far = [2 ** 31 - 1, 160, 2 ** 30, 139, 500]
    for counts, prefix in ((None, 0), (None, 100), ([1, 40, 3, 9, 2], 0)):
        c = Paged(4, 2, 64, 20, [50, 130], dt, [130, 120, 125, 110, 115], counts, page=16, prefix_len=prefix, seed=12)
        c.width = 9                                # 144 positions, with all of which the pages are filled
        c.table, c.prefix_table = c.table[:, :, :9].copy(), c.prefix_table[:, :9].copy()
        c.table[:, :, :] = np.random.default_rng(13).integers(0, c.num_pages, c.table.shape)
        c.prefix_table[:, :] = c.table[0]
        gen = torch.Generator().manual_seed(14)
        c.k, c.v = (torch.randn(c.k.shape, generator=gen).to(c.dtype) for _ in range(2))
        c.positions = far
        c.check(f"past the table {dt} {counts} {prefix}")
