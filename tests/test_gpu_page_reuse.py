"""Pages of an 8-bit cache that change hands: what a sequence stores does not depend on who had its pages."""
import numpy as np
import pytest
import torch

from helpers import bits
from paper_2406_14909_amd import moa as M

pytestmark = pytest.mark.gpu


def _say(*a):
    print("[case]", *a, flush=True)


def _int(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _u8(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


class Reuse:
    """A pool of which a shared prefix holds some pages and sequences come and go over the others.  `history`: what
    lies there when the sequences behind the prefix begin: nothing, a former owner's large numbers, or an
    allocation that was never written."""

    def __init__(self, history, d=64, hq=8, page=16, prefix=41, batch=4, windows=(64, 300), stream=None, pages=None, seed=0):
        self.hq, self.hkv, self.d, self.page, self.prefix, self.batch, self.kw = hq, 2, d, page, prefix, batch, dict(stream=stream)
        self.plan = M.moa_plan(hq, 2, d, 4, max(windows), "bf16", [float(w) for w in windows], [0.0] * 2)
        self.width = 400 // page + 2
        pages = batch * 2 * self.width if pages is None else pages
        self.tables = M.new_page_tables(self.plan, batch, self.width, pages)
        self.own = -(-prefix // page)
        self.cache = M.new_quant_cache(self.plan, pages + 2 * self.own, page)
        self.prefix_table = torch.full((2, self.width), -1, dtype=torch.int32, device="cuda")
        self.prefix_table[:, :self.own] = pages + torch.arange(2 * self.own, device="cuda").view(2, self.own).int()
        self.ws = M.new_paged_workspace(self.plan, batch, 2000)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        if history == "owner":                       # full tables of large numbers, which all end
            at, start = _int([0] * batch), _int(np.arange(batch + 1) * 400)
            q, k, v = self.tokens(400 * batch)
            self.assign(at, start)
            M.moa_quant_append(self.plan, *self.cache, self.tables[0], None, k * 1e30, v * 1e30, at, start, **self.kw)
            self.assign(_int([-1] * batch), None, _int([1] * batch))
            free = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device="cuda")
            assert int(self.tables[2][0]) == pages and bool((self.tables[0] == -1).all())
            self.tables[1].copy_(free)               # the order of a new list
        if history == "garbage":
            rng = np.random.default_rng(1)
            odd = np.array([np.nan, np.inf, -np.inf, 2.0 ** 119, -3e38, 1.0, 1e-40], dtype=np.float32)
            self.cache[2].copy_(torch.from_numpy(rng.choice(odd, size=tuple(self.cache[2].shape))))
            for c in self.cache[:2]:
                c.view(torch.uint8).copy_(torch.randint(0, 256, c.shape, dtype=torch.uint8, generator=self.gen, device="cuda"))
        self.gen.manual_seed(seed + 5)
        q, k, v = self.tokens(prefix)
        M.moa_quant_append(self.plan, *self.cache, self.prefix_table[None], None, k, v, _int([0]), _int([0, prefix]), **self.kw)

    def tokens(self, n):
        draw = lambda h: torch.randn((n, h, self.d), generator=self.gen, device="cuda").bfloat16()
        return draw(self.hq), draw(2), draw(2)

    def assign(self, at, start=None, fresh=None, slots=None):
        M.moa_paged_assign(self.plan, *self.tables, self.page, at, self.ws, start, fresh, slots, scales=self.cache[2], **self.kw)

    def run(self, steps):
        """Decode steps of sequences behind the prefix: outputs, and what is stored of the new tokens."""
        out = []
        for at, fresh in steps:
            q, k, v = self.tokens(self.batch)
            slots = torch.full((self.batch, 2), -7, dtype=torch.int32, device="cuda")
            self.assign(_int(at), None, None if fresh is None else _int(fresh), slots)
            M.moa_quant_append(self.plan, *self.cache, self.tables[0], None, k, v, _int(at), **self.kw)
            o = M.moa_quant_decode_shared(self.plan, q, *self.cache, self.prefix_table, self.prefix, self.tables[0], _int(at),
                                          self.ws, o=torch.full_like(q, 7.0), **self.kw)     # idle rows stay
            rows = slots.view(-1)[_int(at).repeat_interleave(2) >= 0].long()
            assert bool((rows >= 0).all())
            scales = self.cache[2].view(-1, 2)[rows // 16]
            kept = [_u8(c).view(-1, self.d)[rows] for c in self.cache[:2]]
            for c, x, s in zip(self.cache[:2], (k, v), scales.unbind(-1)):
                x = x.view(-1, self.d)[_int(at).repeat_interleave(2) >= 0].double()
                y = c.view(torch.uint8).view(-1, self.d)[rows].view(torch.float8_e4m3fn).double() * s[:, None].double()
                # half a step of four bits, and below that of the smallest number of the scale
                assert bool(((y - x).abs() <= torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * s[:, None].double())).all())
                # a scale that its block needs: no larger than eight standard deviations would take
                assert bool((s <= 2.0 ** -5).all())
            out += [o, scales.clone(), *kept]
        torch.cuda.synchronize()
        return out


def _steps(prefix, batch):
    at = np.array([prefix, prefix, prefix, -1])[:batch]
    steps = [(at.copy(), None)]
    for _ in range(6):
        at = np.where(at < 0, at, at + 1)
        steps.append((at.copy(), None))
    at[1], at[3] = prefix, prefix                    # one ends and another takes its place; the idle one begins
    steps.append((at.copy(), [0, 1, 0, 1]))
    for _ in range(25):
        at = at + 1
        steps.append((at.copy(), None))
    return steps


@pytest.mark.parametrize("d,hq,page,prefix", [(64, 8, 16, 41), (128, 2, 16, 63), (64, 16, 64, 8), (128, 4, 256, 130), (64, 2, 32, 48)])
@pytest.mark.parametrize("history", ["owner", "garbage"])
def test_a_sequence_that_begins_inside_a_block(history, d, hq, page, prefix):
    _say("reuse", history, d, hq, page, prefix)
    steps = _steps(prefix, 4)
    new = Reuse("nothing", d, hq, page, prefix).run(steps)
    got = Reuse(history, d, hq, page, prefix).run(steps)
    assert len(new) == len(got)
    for i, (a, b) in enumerate(zip(new, got)):
        same = torch.equal(bits(a), bits(b))
        assert same, (i // 4, i % 4)


def test_both_call_paths():
    _say("reuse, paths")
    steps = _steps(41, 4)
    a, b = Reuse("owner").run(steps), Reuse("owner", stream=torch.cuda.current_stream()).run(steps)
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(a, b))


@pytest.mark.parametrize("batch,hkv,width,page", [(3, 2, 20, 16), (40, 8, 30, 64), (700, 8, 6, 256), (200, 30, 1500, 16)])
def test_scales_of_the_pages_given_out_and_of_no_others(batch, hkv, width, page):
    """Few pairs and many, tables that the workspace holds copies of and larger ones."""
    _say("scales", batch, hkv, width, page)
    rng = np.random.default_rng(batch)
    windows = [int(x) for x in rng.integers(1, page * width + 1, hkv)]
    plan = M.moa_plan(hkv, hkv, 64, 3, max(windows) + 3, "bf16", [float(w) for w in windows], [0.0] * hkv)
    pages = batch * hkv * min(width, 9) + 5
    tables = M.new_page_tables(plan, batch, width, pages)
    plain = [t.clone() for t in tables]
    scales = torch.full((pages + 3, page // 16, 2), 7.0, device="cuda")
    ws = M.new_paged_workspace(plan, batch, 2000).fill_(0xFF)
    at = rng.integers(-1, page, batch)
    counts = rng.integers(0, 3 * page, batch)
    for step in range(3):
        start = None if step == 2 else _int(np.concatenate([[0], np.cumsum(counts)]))
        fresh = _int(rng.random(batch) < 0.3) if step else None
        before = [t.clone() for t in tables]
        M.moa_paged_assign(plan, *tables, page, _int(at), ws, start, fresh, scales=scales)
        M.moa_paged_assign(plan, *plain, page, _int(at), ws, start, fresh)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(tables, plain))          # the tables are those of the other call
        want = torch.ones(pages + 3, dtype=torch.bool, device="cuda")
        given = (tables[0] >= 0) & ((tables[0] != before[0]) | (before[0] < 0))
        if fresh is not None:                                                # may get the page that it gave back
            given |= (tables[0] >= 0) & (fresh != 0)[:, None, None]
        want[tables[0][given].long()] = False
        assert torch.equal((scales == 7.0).flatten(1).all(1), want) and bool(((scales == 7.0) | (scales == 0.0)).all())
        scales.fill_(7.0)
        at = np.where(at < 0, at, at + (counts if step == 0 else 1))
    with pytest.raises(M.MoaError, match="scales"):
        M.moa_paged_assign(plan, *tables, page, _int(at), ws, scales=scales[:pages - 1])
    with pytest.raises(M.MoaError, match="scales"):
        M.moa_paged_assign(plan, *tables, page, _int(at), ws, scales=scales[..., 0].contiguous())
    with pytest.raises(M.MoaError, match="scales: expected dtype"):
        M.moa_paged_assign(plan, *tables, page, _int(at), ws, scales=scales.double())


def test_a_captured_step_on_pages_of_a_former_owner():
    """Tables, append and decode in one graph, replayed: as the eager steps, bit for bit."""
    _say("reuse, graph")
    prefix, steps = 41, 30
    sides = [Reuse("owner", prefix=prefix, seed=3) for _ in range(2)]
    state = [dict(r=r, at=_int([prefix] * 4), fresh=_int([0] * 4), o=torch.zeros((4, 8, 64), dtype=torch.bfloat16, device="cuda"),
                  **dict(zip("qkv", r.tokens(4)))) for r in sides]

    def step(x):
        r = x["r"]
        r.assign(x["at"], None, x["fresh"])
        M.moa_quant_append(r.plan, *r.cache, r.tables[0], None, x["k"], x["v"], x["at"])
        M.moa_quant_decode_shared(r.plan, x["q"], *r.cache, r.prefix_table, prefix, r.tables[0], x["at"], r.ws, o=x["o"])
        x["at"].add_(1)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(state[1])
    torch.cuda.synchronize()
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(steps):
        for name in "qkv":
            state[0][name].copy_(torch.randn(state[0][name].shape, generator=gen, device="cuda"))
            state[1][name].copy_(state[0][name])
        for x in state:
            x["fresh"].copy_(_int([0, i == 11, 0, i == 20]))
            if i in (11, 20):
                x["at"][1 if i == 11 else 3] = prefix
        step(state[0])
        graph.replay()
        torch.cuda.synchronize()
        a, b = state
        same = [torch.equal(bits(_u8(x)), bits(_u8(y))) for x, y in zip((a["o"], a["at"], *a["r"].tables, *a["r"].cache),
                                                                       (b["o"], b["at"], *b["r"].tables, *b["r"].cache))]
        assert all(same) and bool(a["o"].any()), (i, same)
