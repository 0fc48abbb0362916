"""A pool that has no pages left: what the calls do from there on, with the sequences that lacked pages noted."""
import numpy as np
import pytest
import torch

import oracle
from helpers import bits
from oracle import quant_oracle as Q
from paged_cases import attention_bound
from paper_2406_14909_amd import moa as M

pytestmark = pytest.mark.gpu


def _say(*a):
    print("[case]", *a, flush=True)


def _int(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("batch,hkv,width,page,share", [(3, 2, 20, 16, 0.1), (40, 8, 30, 64, 0.1), (700, 8, 6, 256, 0.2),
                                                        (200, 30, 60, 16, 0.05), (1, 1, 4, 32, 0.3)])
@pytest.mark.parametrize("general", [False, True])
def test_tables_against_the_oracle(batch, hkv, width, page, share, general):
    """Few pairs and many; lists that run out in the middle of a sequence, and that get pages again."""
    _say("shortage tables", batch, hkv, width, page, general)
    rng = np.random.default_rng(batch)
    windows = [int(x) for x in rng.integers(1, page * width // 2 + 1, hkv)]
    plan = M.moa_plan(hkv, hkv, 64, 3, max(windows) + 3, "bf16", [float(w) for w in windows], [0.0] * hkv)
    pages = max(2, int(batch * hkv * min(width, 12) * share))
    dev = M.new_page_tables(plan, batch, width, pages)
    ref = [t.cpu().numpy().astype(np.int64) for t in dev]
    lacked, lacked_ref = _int([0] * batch), np.zeros(batch, dtype=np.int64)
    at = rng.integers(-1, 2 * page, batch)
    seen = 0
    for step in range(7):
        counts = rng.integers(0, 3 * page, batch) * (rng.random(batch) < 0.6)
        single = step % 2 == 1
        start = None if single else np.concatenate([[0], np.cumsum(counts)])
        fresh = (rng.random(batch) < 0.3).astype(int) if step > 1 else None
        if fresh is not None:
            at = np.where(fresh, rng.choice([0, 5, -1], batch), at)
        if step == 6:                                    # the caller clears some
            clear = rng.random(batch) < 0.5
            lacked_ref[clear] = 0
            lacked.copy_(_int(lacked_ref))
        n = batch if single else int(start[-1])
        slots = torch.full((n, hkv), -7, dtype=torch.int32, device="cuda")
        ws = M.new_paged_workspace(plan, batch, max(n, 1)).fill_(0xFF)
        M.moa_paged_assign(plan, *dev, page, _int(at), ws, None if single else _int(start), None if fresh is None else _int(fresh),
                           slots, lacked=lacked, stream=torch.cuda.current_stream() if general else None)
        torch.cuda.synchronize()
        *ref, want = Q.assign_ref(*ref, page, at, start, fresh, n, windows, 3, False, lacked_ref)
        for name, a, b in zip(("table", "free", "counts"), dev, ref):
            assert np.array_equal(a.cpu().numpy(), b), (step, name)
        assert np.array_equal(lacked.cpu().numpy(), lacked_ref), step
        full = np.full((n, hkv), -7)
        for where, x in want.items():
            full[where] = x
        assert np.array_equal(slots.cpu().numpy(), full), (step, "slots")
        seen += int(lacked_ref.sum())
        at = np.where(at < 0, at, at + (1 if single else counts))
    assert seen > 0


class Short:
    """Slots over a pool that is too small, whose rows hold NaN until they are written.  kind: f32, bf16 or 8-bit."""

    def __init__(self, kind, hq, d, pages, page=16, windows=(40, 200), batch=4, seed=0):
        self.kind, self.hq, self.hkv, self.d, self.page, self.batch = kind, hq, 2, d, page, batch
        self.plan = M.moa_plan(hq, 2, d, 4, max(windows), "f32" if kind == "f32" else "bf16", [float(w) for w in windows], [0.0] * 2)
        self.windows = [int(w) for w in self.plan.window]
        self.dtype = self.plan.torch_dtype
        self.tables = M.new_page_tables(self.plan, batch, 400 // page, pages)
        self.lacked = _int([0] * batch)
        if kind == "8-bit":
            self.cache = M.new_quant_cache(self.plan, pages, page)
            for c in self.cache[:2]:
                c.view(torch.uint8).fill_(0x7F)
            self.cache[2].fill_(2.0 ** 100)
        else:
            self.cache = M.new_paged_cache(self.plan, pages, page)
            for c in self.cache:
                c.fill_(float("nan"))
        self.ws = M.new_paged_workspace(self.plan, batch, 2000)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.owner = {}                                  # row of the pool: what was stored there last

    def values(self):
        if self.kind != "8-bit":
            return [c.double().cpu().numpy() for c in self.cache]
        return [(c.double() * self.cache[2][..., i].double().repeat_interleave(16, 1)[..., None]).cpu().numpy()
                for i, c in enumerate(self.cache[:2])]

    def step(self, at, start=None, fresh=None):
        n = self.batch if start is None else int(start[-1])
        draw = lambda h: torch.randn((n, h, self.d), generator=self.gen, device="cuda").to(self.dtype)
        q, k, v = draw(self.hq), draw(2), draw(2)
        at_, start_ = _int(at), None if start is None else _int(start)
        slots = torch.full((n, 2), -7, dtype=torch.int32, device="cuda")
        M.moa_paged_assign(self.plan, *self.tables, self.page, at_, self.ws, start_, None if fresh is None else _int(fresh), slots,
                           scales=self.cache[2] if self.kind == "8-bit" else None, lacked=self.lacked)
        table = self.tables[0]
        call = "moa_quant_" if self.kind == "8-bit" else "moa_paged_"
        getattr(M, call + "append")(self.plan, *self.cache, table, None, k, v, at_, start_)
        o = torch.full_like(q, 7.0)
        if start is None:
            getattr(M, call + "decode")(self.plan, q, *self.cache, table, at_, self.ws, o=o)
        else:
            getattr(M, call + "prefill")(self.plan, q, *self.cache, table, at_, start_, self.ws, o=o)
        torch.cuda.synchronize()
        rows, table = oracle.token_rows(at, start), table.cpu().numpy()
        for t, b, p in rows:
            for g in range(2):
                if int(slots[t, g]) >= 0:
                    self.owner[int(slots[t, g])] = (b, g, p)
        # every position that a query sees on a page that is there was stored by its sequence
        n_pages = len(self.tables[1])
        for t, b, p in rows:
            for g, w in enumerate(self.windows):
                for j in oracle.visible_set(p, w, 4).tolist():
                    row = oracle.slot_ref(table, n_pages, self.page, b, g, j)
                    assert row < 0 or self.owner.get(row) == (b, g, j), (t, b, g, p, j)
        got = o.double().cpu().numpy()
        assert np.isfinite(got).all()
        kp, vp = (np.nan_to_num(x) for x in self.values())
        ref, a, s = oracle.paged_attention_ref(q.double().cpu().numpy(), kp, vp, table, at, start, self.windows, 4)
        mine = np.array([t for t, _, _ in rows], dtype=int)
        if len(mine):
            assert (np.abs(got - ref) <= attention_bound(ref, a, s, self.dtype, self.d, 400))[mine].all()
        assert (np.delete(got, mine, 0) == 7.0).all()
        return self.lacked.tolist()


@pytest.mark.parametrize("kind,hq,d", [("bf16", 8, 64), ("f32", 2, 64), ("8-bit", 4, 128)])
def test_no_query_sees_a_row_that_was_not_stored(kind, hq, d):
    _say("shortage", kind)
    sv = Short(kind, hq, d, pages=22)
    # 2 + 2, 4 + 4, 3 + 3 and 1 + 1 pages of 22
    assert sv.step([0, 0, 0, 0], [0, 30, 90, 130, 132]) == [0, 0, 0, 0]
    at = [30, 60, 40, 2]
    for i in range(4):                               # the last two pages go
        lacked = sv.step(at)
        at = [p + 1 for p in at]
    assert sum(lacked) == 0 and int(sv.tables[2][0]) == 0
    seen = [0, 0, 0, 0]
    for i in range(60):                              # narrow heads give pages back all the time, and others want them
        seen = [max(x, y) for x, y in zip(seen, sv.step(at))]
        at = [p + 1 for p in at]
    assert 0 < sum(seen) == sum(sv.lacked.tolist())  # a note stays
    # chunks of all, the sequences that lacked among them, and the last two steps at once
    lacked = sv.step(at, [0, 5, 40, 41, 70])
    at = [p + c for p, c in zip(at, (5, 35, 1, 29))]
    first = lacked.index(1)
    end = [1 if i == first else 0 for i in range(4)]
    at[first] = 0
    other = next(i for i in range(4) if i != first)
    end[other], at[other] = 1, -1                    # one more ends, so that the first has room
    lacked = sv.step(at, [0, 12, 24, 36, 48], end)
    assert lacked[first] == 0 and lacked[other] == 0
    at = [p + 12 if p >= 0 else -1 for p in at]
    for i in range(20):
        sv.step(at)
        at = [p + 1 if p >= 0 else -1 for p in at]


def test_a_note_outlives_the_replays_of_a_captured_step():
    """Tables and positions in one graph; the shortage comes in the middle of the replays."""
    _say("shortage, graph")
    plan = M.moa_plan(2, 2, 64, 0, 200, "bf16", [20.0, 200.0], [0.0] * 2)
    sides = []
    for _ in range(2):
        sides.append(dict(t=M.new_page_tables(plan, 3, 20, 9), ws=M.new_paged_workspace(plan, 3, 3), lacked=_int([0] * 3),
                          at=_int([0, 3, 7]), fresh=_int([0] * 3)))

    def step(x):
        M.moa_paged_assign(plan, *x["t"], 16, x["at"], x["ws"], None, x["fresh"], lacked=x["lacked"])
        x["at"].add_(1)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(sides[1])
    torch.cuda.synchronize()
    short = []
    for i in range(70):
        for x in sides:
            x["fresh"].copy_(_int([i == 50, 0, 0]))
        step(sides[0])
        graph.replay()
        torch.cuda.synchronize()
        a, b = sides
        same = [torch.equal(x, y) for x, y in zip((*a["t"], a["lacked"], a["at"]), (*b["t"], b["lacked"], b["at"]))]
        assert all(same), (i, same)
        short.append((int(a["t"][2][1]), a["lacked"].tolist()))
    first = next(i for i, (n, _) in enumerate(short) if n)
    assert any(n == 0 and any(x) for n, x in short[first + 1:])          # counts forget it, the note does not
    assert bits(sides[0]["lacked"]).tolist() == short[-1][1]


def test_refusals():
    _say("shortage, refused")
    plan = M.moa_plan(2, 2, 64, 0, 200, "f32", [20.0, 200.0], [0.0] * 2)
    t, ws, at = M.new_page_tables(plan, 3, 20, 9), M.new_paged_workspace(plan, 3, 3), _int([0, 1, 2])
    before = [x.clone() for x in t]
    for bad, match in ((_int([0] * 4), "lacked: expected shape"), (_int([0] * 3).long(), "lacked: expected dtype"),
                       (_int([0] * 3).cpu(), "GPU"), (at, "overlaps"), (t[0].view(-1)[:3], "overlaps")):
        with pytest.raises(M.MoaError, match=match):
            M.moa_paged_assign(plan, *t, 16, at, ws, lacked=bad)
    with pytest.raises(M.MoaError, match="bf16"):
        M.moa_paged_assign(plan, *t, 16, at, ws, scales=torch.zeros((9, 1, 2), device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(before, t))
    lacked = _int([0, 1, 0])
    M.moa_paged_assign(plan, *t, 16, at, ws, lacked=lacked)
    assert (t[0][1] == -1).all() and int((t[0] >= 0).sum()) == 4 and lacked.tolist() == [0, 1, 0]
