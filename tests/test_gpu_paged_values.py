"""Keys and values that are no numbers, at positions that some rows see and others do not: they reach
the rows that see them, and no other."""
import numpy as np
import pytest
import torch

import oracle
from paged_cases import Paged, attention_bound

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _poison(c, seed, keys_too):
    """Puts NaN and infinities into some visible rows of each sequence and head: at the ends of its first
    and last rows' bands, at its own new tokens and at a few others."""
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
                if row < 0:
                    continue
                at = (row // c.page, row % c.page)
                dims = rng.choice(d, 3, replace=False)
                c.v[at][dims] = torch.tensor([NAN, INF, -INF], dtype=c.dtype)[[n % 3, (n + 1) % 3, n % 2]]
                if keys_too and n == 1:
                    c.k[at][int(rng.integers(d))] = NAN


def _check(c):
    got = c.run().double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        ref, a, s = oracle.paged_attention_ref(c.q.double().numpy(), c.k.double().numpy(), c.v.double().numpy(), c.table,
                                               c.positions, c.seq_start, c.windows, c.s, None,
                                               c.block if c.seq_start is not None else 0, c.prefix_table, c.prefix_len)
    rows = [t for t, _, _ in oracle.token_rows(c.positions, c.seq_start)]
    got, ref, a, s = got[rows], ref[rows], a[rows], s[rows]
    sound = np.isfinite(ref)
    assert not sound.all()
    assert not np.isfinite(got[~sound]).any(), "a row lost what it sees"
    assert np.isfinite(got[sound]).all(), f"{(~np.isfinite(got[sound])).sum()} of {sound.sum()} values are no numbers"
    bound = attention_bound(ref, a, s, c.dtype, c.q.shape[2], max(1, c.width * c.page))
    assert (np.abs(got[sound] - ref[sound]) <= bound[sound]).all()
    return sound.mean()


# heads, head_dim, sinks, windows, positions, counts, page, flags: one row tile and few, long ones that are
# cut, two groups of waves and one, blocks, ragged chunks with an idle sequence
PREFILL = [
    (1, 1, 128, 4, (40,), (0,), (90,), 16, 0),
    (4, 2, 128, 0, (30, 700), (100, -1, 7), (70, 5, 300), 32, 0),
    (8, 2, 64, 3, (1, 200), (0, 33), (129, 64), 16, 0),
    (8, 1, 128, 16, (1500,), (1700,), (24,), 64, 0),
    (2, 2, 64, 4, (900, 64), (0, 40), (1100, 30), 128, 2),
    (4, 4, 128, 4, (64, 128, 600, 2500), (0,), (2700,), 16, 0),
]


@pytest.mark.parametrize("keys_too", [0, 1])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("n", range(len(PREFILL)))
def test_prefill_values_reach_only_the_rows_that_see_them(dt, n, keys_too):
    hq, hkv, d, s, windows, positions, counts, page, flags = PREFILL[n]
    print("[case]", dt, n, keys_too, flush=True)
    c = Paged(hq, hkv, d, s, windows, dt, positions, counts, page, flags, seed=n)
    _poison(c, n, keys_too)
    share = _check(c)
    assert share > 0.5 or keys_too       # a key that is NaN takes whole rows, of few rows it may take all


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("prefix", [0, 200])
def test_decode_values_reach_only_the_sequences_that_see_them(dt, prefix):
    print("[case]", dt, prefix, flush=True)
    # over a shared prefix: positions behind it, at its end, inside it, and an idle sequence
    c = Paged(8, 2, 128, 3, (50, 180), dt, (230, 199, 210, -1, 120, 330, 205, 60), page=16, prefix_len=prefix, seed=3)
    _poison(c, 5, 0)
    assert _check(c) > 0.5
