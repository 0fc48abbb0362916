"""Page tables kept on the device against the oracle, entry by entry."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2406_14909_amd import moa as M

pytestmark = pytest.mark.gpu


def _say(*a):
    print("[case]", *a, flush=True)


def _at(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Tables:
    """A layer's tables, the call and the oracle side by side."""

    def __init__(self, hkv, windows, s, page, batch, width, num_pages, flags=0):
        n = max(windows) + s
        self.plan = M.moa_plan(hkv, hkv, 64, s, n, "bf16", [float(w) + (s if flags & 1 else 0) for w in windows], [0.0] * hkv,
                               flags=flags)
        self.windows, self.s, self.page, self.block = [int(w) for w in self.plan.window], s, page, bool(flags & 2)
        self.dev = M.new_page_tables(self.plan, batch, width, num_pages)
        self.ref = [t.cpu().numpy().astype(np.int64) for t in self.dev]
        self.batch, self.hkv = batch, hkv

    def load(self, table=None, free=None, counts=None):
        """Other contents."""
        for i, x in enumerate((table, free, counts)):
            if x is not None:
                self.ref[i] = np.asarray(x, dtype=np.int64)
                self.dev[i].copy_(_at(x))

    def step(self, positions, seq_start=None, fresh=None, rows=None, with_slots=True, stream=None):
        rows = rows if rows is not None else self.batch if seq_start is None else int(max(seq_start))
        slots = torch.full((rows, self.hkv), -7, dtype=torch.int32, device="cuda") if with_slots else None
        ws = M.new_paged_workspace(self.plan, self.batch, max(rows, 1)).fill_(0xFF)
        got = M.moa_paged_assign(self.plan, *self.dev, self.page, _at(positions), ws, _at(seq_start), _at(fresh), slots,
                                 stream=stream)
        torch.cuda.synchronize()
        assert got is slots
        n = rows if with_slots else 1 << 30
        *self.ref, want = Q.assign_ref(*self.ref, self.page, positions, seq_start, fresh, n, self.windows, self.s, self.block)
        for name, a, b in zip(("table", "free", "counts"), self.dev, self.ref):
            assert np.array_equal(a.cpu().numpy(), b), name
        if with_slots:
            full = np.full((rows, self.hkv), -7)
            for at, x in want.items():
                full[at] = x
            assert np.array_equal(slots.cpu().numpy(), full), "slots"


@pytest.mark.parametrize("hkv,windows,s,page,flags", [
    (1, [40], 0, 16, 0), (2, [33, 500], 4, 16, 0), (3, [1, 70, 200], 70, 32, 2), (4, [64, 65, 128, 300], 5, 16, 3),
    (2, [100, 20], 64, 256, 1),
])
def test_steps_of_a_batch(hkv, windows, s, page, flags):
    """Prompts, chunks and single tokens of sequences that come and go."""
    _say("assign", hkv, windows, s, page, flags)
    rng = np.random.default_rng(hkv + page)
    batch, width = 7, 1200 // page + 2
    t = Tables(hkv, windows, s, page, batch, width, batch * hkv * width, flags)
    at = rng.integers(0, 300, batch)
    at[2] = -1
    for step in range(12):
        fresh = (rng.random(batch) < 0.2).astype(int) if step % 3 == 0 else None
        if fresh is not None:
            at = np.where(fresh, rng.choice([0, 0, -1, 5], batch), at)
        if step % 2:
            t.step(at, None, fresh, with_slots=step % 4 == 1)
            at = np.where(at < 0, at, at + 1)
        else:
            count = rng.choice([0, 1, 1, 17, 90], batch)
            start = 3 + np.concatenate([[0], np.cumsum(count)])
            t.step(at, start, fresh, rows=int(start[-1]) + 2)
            at = np.where(at < 0, at, at + count)


def test_a_list_that_runs_out():
    _say("assign short")
    t = Tables(2, [30, 200], 4, 16, 3, 20, 21)
    t.step([0, 0, 0], [0, 100, 200, 300])
    assert t.ref[2].tolist() == [0, 2 * 21 - 21]
    t.step([100, 100, 100], None)                       # what narrow heads give back is given out again
    t.step([-1, 101, -1], None, [1, 0, 1])
    assert t.ref[2][0] > 0
    t.step([0, 102, 40], [0, 30, 31, 32])


def test_whole_release_and_reuse():
    _say("assign reuse")
    t = Tables(3, [50, 60, 70], 0, 16, 4, 40, 4 * 3 * 10)
    t.step([0] * 4, [0, 150, 300, 450, 600])
    t.step([0] * 4, [0, 150, 300, 450, 600], [1] * 4)    # every page goes back and out again
    t.step([-1] * 4, None, [1] * 4)
    assert (t.ref[0] == -1).all() and t.ref[2].tolist() == [120, 0]


@pytest.mark.parametrize("batch,hkv,width", [(1, 1, 1), (33, 64, 5), (700, 3, 70), (5, 2, 3000), (300, 32, 12)])
def test_sizes(batch, hkv, width):
    """Tables of few and many pairs, short and long rows; entries that were never written properly."""
    _say("assign sizes", batch, hkv, width)
    rng = np.random.default_rng(batch)
    windows = [int(x) for x in rng.integers(1, 16 * width + 1, hkv)]
    pages = batch * hkv * width + 10
    t = Tables(hkv, windows, 4, 16, batch, width, pages)
    order = rng.permutation(pages)
    table = np.where(rng.random((batch, hkv, width)) < 0.6, order[:batch * hkv * width].reshape(batch, hkv, width),
                     rng.choice([-1, -2 ** 31, 2 ** 31 - 1, pages], (batch, hkv, width)))
    free = np.setdiff1d(order, table)
    t.load(table, np.concatenate([free, np.full(pages - len(free), -5)]), [len(free), 3])
    at = rng.integers(-1, 16 * width + 40, batch)
    t.step(at, None, (rng.random(batch) < 0.3).astype(int))
    count = rng.integers(0, 40, batch)
    t.step(at, np.concatenate([[0], np.cumsum(count)]), None)


def test_odd_inputs():
    """Counts out of range, rows past the end, positions past the table, no slots: nothing out of bounds."""
    _say("assign odd")
    t = Tables(2, [20, 300], 4, 16, 3, 6, 40)
    t.load(counts=[10 ** 9, 7])
    t.step([0, 90, 2 ** 31 - 1], None)
    t.load(counts=[-5, 0])
    t.step([0, 30, -1], [0, 20, 40, 60], [0, 0, 1])
    t.load(counts=[30, 0])
    t.step([1, 30, 200], [5, 200, 20, 60], rows=100)     # the first runs past the rows, the second backwards
    t.step([1, 30, 200], [0, 10, 20, 30], with_slots=False)
    table = np.full((3, 2, 6), 9)                        # a page that stands in many entries
    t.load(table=table, counts=[38, 0])
    t.step([-1, -1, -1], None, [1, 1, 1])


def test_another_stream():
    _say("assign stream")
    t = Tables(2, [33, 500], 4, 16, 4, 80, 600)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    t.step([0, 3, -1, 0], [0, 100, 150, 150, 400], stream=s)
    t.step([100, 53, 9, 250], None, [0, 0, 1, 0], stream=s)


@pytest.mark.parametrize("batch,hkv,width,count", [(9, 4, 60, 700), (4, 32, 100, 1500), (600, 8, 4, 9), (1500, 3, 6, 4),
                                                   (200, 30, 1500, 25)])
def test_many_tokens_and_pairs(batch, hkv, width, count):
    """Rows by a kernel of their own; more pairs than one work-group adds up; tables larger than the
    workspace holds copies of; sequences without tokens in between."""
    _say("assign many", batch, hkv, width, count)
    rng = np.random.default_rng(batch)
    windows = [int(x) for x in rng.integers(1, 16 * width + 1, hkv)]
    t = Tables(hkv, windows, 7, 16, batch, width, batch * hkv * min(width, count // 4 + 4))
    at = rng.integers(-1, 40, batch)
    counts = rng.integers(0, count, batch) * (rng.random(batch) < 0.7)
    for step in range(2):
        t.step(at, 1 + np.concatenate([[0], np.cumsum(counts)]), rng.random(batch) < 0.2 if step else None,
               rows=int(counts.sum()) + 9)
        at = np.where(at < 0, at, at + counts)
