"""The paged operators as a server uses them: together, through both call paths, on other
streams, captured, in large batches and pools, and with arguments that are refused or odd."""
import numpy as np
import pytest
import torch

import oracle
from helpers import bits
from paged_cases import Paged, attention_bound
from paper_2406_14909_amd import moa as M

pytestmark = pytest.mark.gpu


def _say(*a):
    print("[case]", *a, flush=True)


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Server:
    """Sequences that share a prompt of `prefix` tokens; every head has pages of its own."""

    def __init__(self, hq=8, hkv=2, d=64, s=4, windows=(40, 300), dt="bf16", prefix=203, batch=3, most=330, page=16, seed=0):
        self.hq, self.hkv, self.d, self.s, self.windows, self.page, self.prefix = hq, hkv, d, s, list(windows), page, prefix
        self.plan = M.moa_plan(hq, hkv, d, s, max(windows), dt, [float(w) for w in windows], [0.0] * hkv)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.inv_freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().cuda()
        width, shared = -(-most // page), prefix // page                    # whole pages of the prompt are shared
        pages = np.random.default_rng(seed).permutation(hkv * shared + batch * hkv * (width - shared))
        self.table = np.empty((batch, hkv, width), dtype=np.int32)
        self.table[:, :, :shared] = pages[:hkv * shared].reshape(hkv, shared)
        self.table[:, :, shared:] = pages[hkv * shared:].reshape(batch, hkv, width - shared)
        self.table = torch.from_numpy(self.table).cuda()
        self.kp, self.vp = M.new_paged_cache(self.plan, len(pages), page)
        self.ws = M.new_paged_workspace(self.plan, batch, 400)
        self.batch = batch
        self.history = [([], []) for _ in range(batch)]                      # keys and values as the pages hold them

    def tokens(self, n):
        draw = lambda h: torch.randn((n, h, self.d), generator=self.gen, device="cuda").to(self.plan.torch_dtype)
        return draw(self.hq), draw(self.hkv), draw(self.hkv)

    def read(self, b, n):
        """k, v [n, hkv, d] of sequence b, from the pages."""
        at = torch.arange(n, device="cuda")
        page = self.table[b][:, at // self.page].long()
        return [x[page, at % self.page].transpose(0, 1) for x in (self.kp, self.vp)]

    def check(self, o, q, b, first, what):
        """o, q [n, hq, d] of sequence b's tokens from position first on, against the oracle over its pages."""
        n = first + len(q)
        k, v = self.read(b, n)
        w = self.windows
        for i in {0, len(q) // 2, len(q) - 1}:
            ref = oracle.decode_ref(q[i:i + 1], k[None, :first + i + 1], v[None, :first + i + 1], w, self.s)
            err = np.abs(o[i].double().cpu().numpy() - ref[0]).max()
            assert err <= 2.0 ** -6 * float(v.abs().max()), (what, b, i, err)


@pytest.mark.parametrize("dt,d,hq", [("bf16", 64, 8), ("bf16", 128, 2), ("f32", 64, 4)])
def test_a_server(dt, d, hq):
    """The shared prompt in chunks, a question per sequence in one ragged call, then decode steps of
    all, once by way of the shared prefix and once without."""
    _say("server", dt, d, hq)
    sv = Server(dt=dt, d=d, hq=hq)
    done = 0
    for n in (100, 1, sv.prefix - 101):                                       # the prompt, as sequence 0's
        q, k, v = sv.tokens(n)
        at, start, table = _int([done]), _int([0, n]), sv.table[:1].contiguous()
        q = M.moa_paged_append(sv.plan, sv.kp, sv.vp, table, q, k, v, at, start, sv.inv_freq)
        o = M.moa_paged_prefill(sv.plan, q, sv.kp, sv.vp, table, at, start, sv.ws)
        sv.check(o, q, 0, done, "prompt")
        done += n
    # the prompt's last, part-filled page: every sequence has its own copy
    last = (sv.prefix // sv.page)
    for b in range(1, sv.batch):
        for g in range(sv.hkv):
            for x in (sv.kp, sv.vp):
                x[int(sv.table[b, g, last])] = x[int(sv.table[0, g, last])]
    counts = [7, 33, 1]
    start, at = _int([0, 7, 40, 41]), _int([sv.prefix] * 3)
    q, k, v = sv.tokens(41)
    q = M.moa_paged_append(sv.plan, sv.kp, sv.vp, sv.table, q, k, v, at, start, sv.inv_freq)
    o = M.moa_paged_prefill(sv.plan, q, sv.kp, sv.vp, sv.table, at, start, sv.ws)
    for b, (a, z) in enumerate(((0, 7), (7, 40), (40, 41))):
        sv.check(o[a:z], q[a:z], b, sv.prefix, "question")
    at = at + _int(counts)
    for step in range(4):
        q, k, v = sv.tokens(3)
        q = M.moa_paged_append(sv.plan, sv.kp, sv.vp, sv.table, q, k, v, at, inv_freq=sv.inv_freq)
        o = M.moa_paged_decode(sv.plan, q, sv.kp, sv.vp, sv.table, at, sv.ws)
        shared = M.moa_paged_decode_shared(sv.plan, q, sv.kp, sv.vp, sv.table[0], sv.prefix // sv.page * sv.page, sv.table,
                                           at, sv.ws)
        for b in range(3):
            p = int(at[b])
            sv.check(o[b:b + 1], q[b:b + 1], b, p, "decode")
            sv.check(shared[b:b + 1], q[b:b + 1], b, p, "shared")
        at += 1


def test_a_whole_prompt_equals_dense_prefill():
    """moa_paged_prefill over one whole prompt against moa_prefill of the same rows: the same weights
    rounded alike, so within two roundings of bf16."""
    _say("whole prompt")
    for n, flags in ((333, 0), (1500, 2)):
        hq, hkv, d, w = 8, 2, 128, [100, 700]
        plan = M.moa_plan(hq, hkv, d, 10, n, "bf16", [float(x) for x in w], [0.0] * hkv, flags=flags)
        gen = torch.Generator(device="cuda").manual_seed(n)
        q, k, v = (torch.randn((n, h, d), generator=gen, device="cuda").bfloat16() for h in (hq, hkv, hkv))
        dense = M.moa_prefill(plan, q[None], k[None], v[None])[0]
        width = -(-n // 64)
        table = torch.randperm(hkv * width, device="cuda").int().view(1, hkv, width)
        kp, vp = M.new_paged_cache(plan, hkv * width, 64)
        at, start = _int([0]), _int([0, n])
        assert torch.equal(M.moa_paged_append(plan, kp, vp, table, q, k, v, at, start), q)
        o = M.moa_paged_prefill(plan, q, kp, vp, table, at, start, M.new_paged_workspace(plan, 1, n))
        assert float((o.float() - dense.float()).abs().max()) <= 2.0 ** -6 * float(v.abs().max())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_large_batches(dt):
    """More (sequence, head) pairs than threads of a work-group, among them idle sequences and ones without tokens."""
    _say("large batch", dt)
    rng = np.random.default_rng(3)
    where = [int(x) for x in rng.integers(-20, 90, size=700)]
    Paged(4, 2, 64, 3, [9, 50], dt, where, seed=1).check("decode of 700")
    counts = [int(x) for x in rng.choice([0, 1, 2, 17], size=400)]
    Paged(4, 2, 64, 3, [9, 50], dt, where[:400], counts, seed=2, pad=2).check("prefill of 400")
    where = [max(p, -1) if p < 0 else p + 60 for p in where[:300]]
    Paged(4, 2, 64, 3, [9, 100], dt, where, prefix_len=60, seed=4).check("shared by 300")


def test_a_long_sequence_among_many():
    """Pieces of a cut row tile and whole row tiles in one call, with more pairs than threads."""
    _say("long among many")
    rng = np.random.default_rng(5)
    counts = [int(x) for x in rng.choice([1, 3], size=150)]
    where = [int(x) for x in rng.integers(0, 60, size=150)]
    where[70], counts[70] = 9000, 200
    Paged(2, 2, 64, 5, [3000, 8000], "bf16", where, counts, page=64, seed=6).check("long among many")


def test_pools_beyond_32_bit_offsets():
    """Pages more than 4 GiB into their pool."""
    _say("large pool")
    hq, hkv, d, page, n_pages = 4, 2, 128, 256, 70000
    plan = M.moa_plan(hq, hkv, d, 4, 2000, "bf16", [600.0, 2000.0], [0.0] * hkv)
    kp, vp = (torch.empty((n_pages, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert kp.numel() * 2 > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(9)
    n = 700
    q, k, v = (torch.randn((n, h, d), generator=gen, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    table = _int([[[n_pages - 1, n_pages - 5, 66000], [n_pages - 9, 0, 65999]]])
    small = _int([[[0, 1, 2], [3, 4, 5]]])
    ks, vs = M.new_paged_cache(plan, 6, page)
    ws = M.new_paged_workspace(plan, 1, n)
    at, start = _int([0]), _int([0, n])
    out = []
    for a, b, t in ((kp, vp, table), (ks, vs, small)):
        M.moa_paged_append(plan, a, b, t, q, k, v, at, start)
        out.append([M.moa_paged_prefill(plan, q, a, b, t, at, start, ws),
                    M.moa_paged_decode(plan, q[-1:], a, b, t, _int([n - 1]), ws),
                    M.moa_paged_decode_shared(plan, q[-1:], a, b, t[0], 512, t, _int([n - 1]), ws)])
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(*out)) and float(out[0][0].abs().max()) > 0


def test_absent_pages_after_a_call_that_left_nan_in_lds():
    """A tile's rows on an absent page count as zeros, whatever the LDS held before."""
    _say("absent pages, LDS of NaN")
    gone = [(0, 0, 3), (0, 1, 0), (0, 1, 9)]
    for d in (64, 128):
        bad = M.moa_plan(32, 32, d, 0, 512, "bf16", [512.0] * 32, [0.0] * 32)
        x = torch.full((1, 512, 32, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        c = Paged(8, 2, d, 20, [100, 1000], "bf16", [60], [95], page=16, absent=gone, seed=5)
        for _ in range(3):
            M.moa_prefill(bad, x, x, x)
            c.check("absent after NaN")


def test_the_same_call_gives_the_same_bits():
    _say("repeat")
    for kw in (dict(counts=[300, 40, 5]), dict(), dict(prefix_len=250)):
        for dt in ("bf16", "f32"):
            c = Paged(8, 2, 64, 7, [200, 2500], dt, [2100, 900, 260], page=32, seed=8, **kw)
            first = c.run()
            for _ in range(3):
                assert torch.equal(bits(c.run()), bits(first))


# ---------------------------------------------------------------------------
# Call paths, streams, graphs.
# ---------------------------------------------------------------------------
def _everything(stream, dt="bf16"):
    """All four calls once; stream None takes the native path, a stream the general one."""
    sv = Server(dt=dt, seed=4, prefix=0)          # no two tokens go to one row
    q, k, v = sv.tokens(60)
    at, start = _int([0, 5, -1]), _int([0, 30, 58, 60])
    kw = dict(stream=stream)
    out = [M.moa_paged_append(sv.plan, sv.kp, sv.vp, sv.table, q, k, v, at, start, sv.inv_freq, True, torch.zeros_like(q), **kw)]
    out.append(M.moa_paged_prefill(sv.plan, out[0], sv.kp, sv.vp, sv.table, at, start, sv.ws, torch.zeros_like(q), **kw))
    qd, kd, vd = sv.tokens(3)
    at = _int([30, 33, 40])
    M.moa_paged_append(sv.plan, sv.kp, sv.vp, sv.table, None, kd, vd, at, **kw)
    out.append(M.moa_paged_decode(sv.plan, qd, sv.kp, sv.vp, sv.table, at, sv.ws, **kw))
    out.append(M.moa_paged_decode_shared(sv.plan, qd, sv.kp, sv.vp, sv.table[0], 16, sv.table, at, sv.ws, **kw))
    return out + [sv.kp, sv.vp]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_native_path_equals_general_path(dt):
    _say("paths", dt)
    for a, b in zip(_everything(None, dt), _everything(torch.cuda.current_stream(), dt)):
        same = torch.equal(bits(a), bits(b))
        assert same and bool(torch.isfinite(a).all())


def test_native_path_takes_ordinary_calls_and_leaves_the_others():
    _say("native")
    sv = Server()
    q, k, v = sv.tokens(3)
    at, start = _int([0, 1, 2]), _int([0, 1, 2, 3])
    f, p = M._fast, sv.plan._bound
    app = [sv.kp, sv.vp, sv.table, q, k, v, at, start, sv.inv_freq, False, torch.empty_like(q)]
    assert f.paged_append(p, *app) is app[-1]
    assert f.paged_append(p, *app[:-1], None).shape == q.shape
    assert f.paged_append(p, *app[:3], None, k, v, at, None, None, False, None) is True
    pre = [q, sv.kp, sv.vp, sv.table, at, start, sv.ws, torch.empty_like(q)]
    dec = [q, sv.kp, sv.vp, sv.table, at, sv.ws, torch.empty_like(q)]
    sha = [q, sv.kp, sv.vp, sv.table[0], 16, sv.table, at, sv.ws, torch.empty_like(q)]
    for name, args, tensors in (("paged_append", app, range(8)), ("paged_prefill", pre, range(8)),
                                ("paged_decode", dec, range(7)), ("paged_decode_shared", sha, (0, 1, 2, 3, 5, 6, 7, 8))):
        call = getattr(f, name)
        assert call(p, *args) is not None
        for i in tensors:
            t = args[i]
            odd = [t.cpu(), t.unsqueeze(0), torch.stack((t, t), -1)[..., 0]]
            if t.dtype != torch.uint8:
                odd.append(t.long() if t.dtype == torch.int32 else t.double())
            for x in odd:
                if t.dtype == torch.uint8 and x.is_cuda and x.is_contiguous():
                    continue                                     # of a workspace any shape
                bad = list(args)
                bad[i] = x
                assert call(p, *bad) is None, (name, i, tuple(x.shape), x.dtype)
        assert call(p, *args[:-1]) is None and call(None, *args) is None


@pytest.mark.parametrize("change,match", [
    (dict(q=lambda x: x[:, :4]), "q: expected shape"), (dict(k=lambda x: x.float()), "k_new: expected dtype"),
    (dict(v=lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)), "heads must be contiguous"),
    (dict(at=lambda x: x.long()), "positions"), (dict(start=lambda x: x[:-1]), "seq_start: expected shape"),
    (dict(table=lambda x: x[:, :1].contiguous()), "table: expected shape"),
    (dict(table=lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)), "table: must be contiguous"),
    (dict(kp=lambda x: x[:, :, :32].contiguous()), "k_pages: expected shape"), (dict(kp=lambda x: x[0]), "k_pages"),
    (dict(vp=lambda x: x[:2]), "v_pages: expected shape"), (dict(kp=lambda x: x.cpu()), "GPU"),
    (dict(f=lambda x: x.double()), "inv_freq: expected dtype"), (dict(f=lambda x: x[:9]), "rotary_dim"),
    (dict(out=lambda x: x[:1]), "q_out: expected shape"),
])
def test_refusals_of_append(change, match):
    _say("refused", match)
    sv = Server()
    q, k, v = sv.tokens(3)
    x = dict(q=q, k=k, v=v, at=_int([0, 1, 2]), start=_int([0, 1, 2, 3]), table=sv.table, kp=sv.kp, vp=sv.vp, f=sv.inv_freq,
             out=torch.zeros_like(q))
    for name, fn in change.items():
        x[name] = fn(x[name])
    with pytest.raises(M.MoaError, match=match):
        M.moa_paged_append(sv.plan, x["kp"], x["vp"], x["table"], x["q"], x["k"], x["v"], x["at"], x["start"], x["f"],
                           q_out=x["out"])
    assert not sv.kp.any() and not sv.vp.any()


def test_refusals_of_attention():
    _say("refused attention")
    sv = Server()
    q, _, _ = sv.tokens(3)
    at, start = _int([0, 1, 2]), _int([0, 1, 2, 3])
    args = lambda **kw: {**dict(q=q, k_pages=sv.kp, v_pages=sv.vp, table=sv.table, positions=at, workspace=sv.ws), **kw}
    for bad, match in ((dict(workspace=sv.ws[:256]), "workspace"), (dict(workspace=sv.ws.cpu()), "workspace"),
                       (dict(q=q[:2]), "expected shape"), (dict(q=q.float()), "expected dtype"),
                       (dict(positions=at[None]), "positions"), (dict(o=q), "overlaps")):
        with pytest.raises(M.MoaError, match=match):
            M.moa_paged_decode(sv.plan, **args(**bad))
    with pytest.raises(M.MoaError, match="seq_start"):
        M.moa_paged_prefill(sv.plan, seq_start=start[:3], **args())
    with pytest.raises(M.MoaError, match="prefix_table"):
        M.moa_paged_decode_shared(sv.plan, prefix_table=sv.table, prefix_len=16, **args())
    with pytest.raises(M.MoaError, match="prefix_len"):
        M.moa_paged_decode_shared(sv.plan, prefix_table=sv.table[0], prefix_len=10 ** 6, **args())


def test_seq_start_that_is_no_packing_harms_nothing():
    """Sequences that overlap, run backwards or pass the rows: some rows may be written, none outside o."""
    _say("odd seq_start")
    for dt in ("bf16", "f32"):
        sv = Server(dt=dt)
        q, k, v = sv.tokens(40)
        buf = torch.full((60, sv.hq, sv.d), 7.0, dtype=q.dtype, device="cuda")
        for start in ([0, 40, 0, 40], [40, 20, 10, 0], [-5, 10, 30, 40], [0, 10, 30, 100], [0, 2 ** 31 - 1, -2 ** 31, 3]):
            at, ss = _int([0, 0, 0]), _int(start)
            M.moa_paged_append(sv.plan, sv.kp, sv.vp, sv.table, q, k, v, at, ss, sv.inv_freq, q_out=buf[10:50])
            M.moa_paged_prefill(sv.plan, q, sv.kp, sv.vp, sv.table, at, ss, sv.ws, o=buf[10:50])
        assert (buf[:10] == 7.0).all() and (buf[50:] == 7.0).all()


def test_other_streams():
    """Two streams at once, each with a workspace of its own; and tensors used on the current stream only."""
    _say("streams")
    cases = [Paged(8, 2, 128, 4, [900, 60], "bf16", [1200, 777], seed=i) for i in range(2)]
    refs = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    xs = [c.device() for c in cases]
    outs = [torch.zeros_like(x["q"]) for x in xs]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, x, o, s in zip(cases, xs, outs, streams):
            with torch.cuda.stream(s):
                M.moa_paged_decode(c.plan, x["q"], x["k_pages"], x["v_pages"], x["table"], x["positions"], x["workspace"], o=o)
    torch.cuda.synchronize()
    for o, r, c in zip(outs, refs, cases):
        assert torch.equal(bits(o), bits(r))


@pytest.mark.parametrize("shared", [False, True])
def test_a_captured_decode_loop(shared):
    """Append, decode and the next positions in one graph: every replay equals the eager step, bit for bit."""
    _say("graph", shared)
    steps = 6
    sides = [Server(seed=7, prefix=0) for _ in range(2)]
    q, k, v = sides[0].tokens(205 * 3)
    for sv in sides:                                               # every sequence's history
        at, start = _int([0, 0, 0]), _int([0, 205, 410, 615])
        table = sv.table.clone()
        M.moa_paged_append(sv.plan, sv.kp, sv.vp, table, None, k, v, at, start)
    new = [sides[0].tokens(3) for _ in range(steps)]
    state = [dict(q=torch.zeros_like(new[0][0]), k=torch.zeros_like(new[0][1]), v=torch.zeros_like(new[0][2]),
                  at=_int([205, 205, 205]), o=torch.zeros_like(new[0][0]), qr=torch.zeros_like(new[0][0])) for _ in sides]

    def step(sv, x):
        M.moa_paged_append(sv.plan, sv.kp, sv.vp, sv.table, x["q"], x["k"], x["v"], x["at"], inv_freq=sv.inv_freq, q_out=x["qr"])
        if shared:
            M.moa_paged_decode_shared(sv.plan, x["qr"], sv.kp, sv.vp, sv.table[0], 192, sv.table, x["at"], sv.ws, o=x["o"])
        else:
            M.moa_paged_decode(sv.plan, x["qr"], sv.kp, sv.vp, sv.table, x["at"], sv.ws, o=x["o"])
        x["at"].add_(1)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(sides[1], state[1])
    torch.cuda.synchronize()
    for i in range(steps):
        for x in state:
            for name, t in zip("qkv", new[i]):
                x[name].copy_(t)
        step(sides[0], state[0])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(state[0]["o"]), bits(state[1]["o"])) and state[0]["o"].any(), i
        assert torch.equal(bits(sides[0].kp), bits(sides[1].kp)) and torch.equal(state[0]["at"], state[1]["at"])


def test_a_captured_prefill():
    _say("graph of a prefill")
    for dt in ("bf16", "f32"):
        c = Paged(8, 2, 64, 4, [2500, 100], dt, [2300, 10], [90, 200], page=32, seed=12)
        ref, x = c.run(), c.device()
        o = torch.zeros_like(x["q"])
        call = lambda: M.moa_paged_prefill(c.plan, x["q"], x["k_pages"], x["v_pages"], x["table"], x["positions"],
                                           x["seq_start"], x["workspace"], o=o)
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                call()
        for _ in range(3):
            o.zero_()
            x["workspace"].fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(bits(o), bits(ref))
            call()
            torch.cuda.synchronize()
            assert torch.equal(bits(o), bits(ref))
