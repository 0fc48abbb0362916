"""What is not finite reaches the outputs that it has a part in, as what it is: a NaN in a key or a query
makes NaN, an infinite value an infinity of its sign, however the keys of a call are cut."""
import numpy as np
import pytest
import torch

import oracle
from paged_cases import Paged, attention_bound

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _slot(c, i, g, j):
    """(page, row) of position j of head g of sequence i."""
    pre = j < c.prefix_len
    row = oracle.slot_ref(c.prefix_table[None] if pre else c.table, c.num_pages, c.page, 0 if pre else i, g, j)
    return row // c.page, row % c.page


def _put(c, kind, i, g, j, dim, sign=1.0):
    """One value of sequence i, head g that is not finite."""
    group = c.q.shape[1] // len(c.windows)
    rows = [t for t, b, _ in oracle.token_rows(c.positions, c.seq_start) if b == i]
    if kind == "query nan":
        c.q[rows[-1], g * group, dim] = NAN
    elif kind == "key nan":
        c.k[_slot(c, i, g, j)][dim] = NAN
    elif kind == "key inf":                     # of the sign of all queries, so that the score is +inf
        heads = c.q[:, g * group:(g + 1) * group, dim]
        heads.copy_(heads.abs() + 0.25)
        c.k[_slot(c, i, g, j)][dim] = INF
    else:
        c.v[_slot(c, i, g, j)][dim] = sign * INF


def _check(c):
    got = c.run().double().cpu().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        ref, a, s = oracle.paged_attention_ref(c.q.double().numpy(), c.k.double().numpy(), c.v.double().numpy(), c.table,
                                               c.positions, c.seq_start, c.windows, c.s, None,
                                               c.block if c.seq_start is not None else 0, c.prefix_table, c.prefix_len)
        bound = attention_bound(ref, a, s, c.dtype, c.q.shape[2], max(1, c.width * c.page))
    rows = [t for t, _, _ in oracle.token_rows(c.positions, c.seq_start)]
    got, ref, bound = got[rows], ref[rows], bound[rows]
    sound = np.isfinite(ref)
    assert not sound.all()
    assert np.array_equal(np.isnan(got), np.isnan(ref)), (np.isnan(got) != np.isnan(ref)).sum()
    assert np.array_equal(np.where(np.isinf(got), np.sign(got), 0), np.where(np.isinf(ref), np.sign(ref), 0))
    assert (np.abs(got[sound] - ref[sound]) <= bound[sound]).all()


# windows of one round, whose cache one work-group has to itself, and ones that are cut over many
@pytest.mark.parametrize("kind", ["query nan", "key nan", "key inf", "value inf"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 128), (4, 2, 64), (8, 2, 128), (8, 1, 64)])
@pytest.mark.parametrize("windows,prefix", [((40, 9), 0), ((3000, 5000), 0), ((40, 3000), 6000)])
def test_decode(kind, dt, hq, hkv, d, windows, prefix):
    print("[case]", kind, dt, hq, hkv, d, windows, prefix, flush=True)
    where = (6100, 6030, -1, 6003)
    c = Paged(hq, hkv, d, 3, windows[:hkv], dt, where, page=32, prefix_len=prefix, seed=1)
    for i, j in ((0, 6100), (3, 6001)):         # sequence 1 is left sound; both are in the narrowest window
        for g in range(hkv):
            if i == 0 or g == 0:
                _put(c, kind, i, g, j, 5 + g, 1.0 if i == 0 else -1.0)
    _check(c)


@pytest.mark.parametrize("kind", ["query nan", "key nan", "value inf"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 2, 128)])
def test_shared_prefix(kind, dt, hq, hkv, d):
    """In the part that is read once for all: it reaches the sequences whose windows go back to it."""
    print("[case]", kind, dt, hq, hkv, d, flush=True)
    where = (3100, 3030, -1, 3003, 2999, 1500)                  # the last two: at the prefix's end, and inside it
    c = Paged(hq, hkv, d, 3, (60, 2500), dt, where, page=32, prefix_len=3000, seed=5)
    _put(c, kind, 3, 0, 2960, 5)
    _put(c, kind, 0, 1, 2999, 9, -1.0)
    _put(c, kind, 1, 1, 1, 11)                                  # a sink
    _check(c)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq", [1, 8])
def test_decode_of_one_key(dt, hq):
    """A cache of the token itself: its value, or NaN where key or query is."""
    for kind in ("query nan", "key nan", "key inf", "value inf"):
        print("[case]", kind, dt, hq, flush=True)
        c = Paged(hq, 1, 64, 0, (1,), dt, (0, 17), page=16, seed=2)
        _put(c, kind, 0, 0, 0, 3)
        _check(c)


# heads, windows, positions, counts: one row tile whole, and ones cut into few and into many pieces
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,windows,positions,counts", [
    (2, 2, (30, 100), (5,), (60,)), (8, 1, (1500,), (1700,), (24,)), (8, 2, (3000, 2000), (2900, 2500), (9, 30)),
    (2, 1, (14000,), (14000,), (20,))])
@pytest.mark.parametrize("kind", ["query nan", "key nan", "value inf"])
def test_prefill(kind, dt, hq, hkv, windows, positions, counts):
    print("[case]", kind, dt, hq, windows, flush=True)
    c = Paged(hq, hkv, 128, 4, windows, dt, positions, counts, page=16, seed=3)
    for i, (p, n) in enumerate(zip(positions, counts)):
        for g in range(hkv):
            _put(c, kind, i, g, p + n // 2, 5 + g)          # a key that some of the sequence's rows see
            if kind == "value inf":
                _put(c, kind, i, g, p + n - 1, 40, -1.0)     # the last key, in the last piece
                _put(c, kind, i, g, max(0, p - 20), 77)      # one that all rows see
    _check(c)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2)])
@pytest.mark.parametrize("counts,prefix", [(None, 0), (None, 51), ((3, 2), 0)])
def test_scores_of_minus_infinity(dt, hq, hkv, counts, prefix):
    """A key of that score weighs nothing; a query with no other gets zeros."""
    print("[case]", dt, hq, counts, prefix, flush=True)
    c = Paged(hq, hkv, 64, 0, (1, 5), dt, (50, 60), counts, page=16, prefix_len=prefix, seed=4)
    heads = c.q[:, :hq // hkv, 7]
    heads.copy_(heads.abs() + 0.25)                             # those of KV head 0, whose window is 1
    c.k[_slot(c, 0, 0, 50)][7] = -INF                           # all that sequence 0's first row sees there
    c.k[_slot(c, 0, 1, 49)][3] = -INF                           # of KV head 1 one of five keys
    c.q[0, hq // hkv:, 3] = c.q[0, hq // hkv:, 3].abs() + 0.25
    if counts is not None:
        c.q[:3, hq // hkv:, 3] = c.q[:3, hq // hkv:, 3].abs() + 0.25
    got = c.run().double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        ref, a, _ = oracle.paged_attention_ref(c.q.double().numpy(), c.k.double().numpy(), c.v.double().numpy(), c.table,
                                               c.positions, c.seq_start, c.windows, c.s, None, 0, c.prefix_table,
                                               c.prefix_len)
    assert np.isnan(ref[0, :hq // hkv]).all() and (got[0, :hq // hkv] == 0.0).all()
    ref[0, :hq // hkv] = 0.0
    # fp32: scores are below 50 in magnitude, of 64 terms; see attention_bound, with 2^-8 for bf16's two roundings
    slack = 8 * 2.0 ** -24 * (12 * 50 + 7) * a + (2.0 ** -8 * (a + 2 * np.abs(ref)) if dt == "bf16" else 2.0 ** -24 * np.abs(ref))
    assert np.isfinite(ref).all() and (np.abs(got - ref) <= slack)[np.isfinite(a)].all()
