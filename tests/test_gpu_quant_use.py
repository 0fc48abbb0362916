"""The 8-bit cache and its page tables as a server uses them: together, through both call paths, on
other streams, captured, in large batches and pools, and with arguments that are refused or odd."""
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


def _int(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _same(a, b):
    return all(torch.equal(bits(x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x),
                           bits(y.view(torch.uint8) if y.dtype == torch.float8_e4m3fn else y)) for x, y in zip(a, b))


class Server:
    """Slots for sequences over one pool; the tables are the library's to keep."""

    def __init__(self, batch=4, hq=8, hkv=2, d=64, s=4, windows=(40, 300), page=16, most=400, pages=None, seed=0, flags=0):
        self.hq, self.hkv, self.d, self.s, self.page, self.batch = hq, hkv, d, s, page, batch
        self.plan = M.moa_plan(hq, hkv, d, s, max(windows), "bf16", [float(w) for w in windows], [0.0] * hkv, flags=flags)
        self.windows = [int(w) for w in self.plan.window]
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.inv_freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).float().cuda()
        width = -(-most // page)
        pages = batch * hkv * width if pages is None else pages
        self.tables = M.new_page_tables(self.plan, batch, width, pages)
        self.cache = M.new_quant_cache(self.plan, pages, page)
        self.ws = M.new_paged_workspace(self.plan, batch, 2000)

    def tokens(self, n):
        draw = lambda h: torch.randn((n, h, self.d), generator=self.gen, device="cuda").bfloat16()
        return draw(self.hq), draw(self.hkv), draw(self.hkv)

    def step(self, at, start=None, fresh=None, new=None):
        """One call of all: tables, append, attention; and the attention's outputs against the oracle."""
        at_, start_ = _int(at), None if start is None else _int(start)
        n = self.batch if start is None else int(start[-1])
        q, k, v = new or self.tokens(n)
        slots = torch.full((n, self.hkv), -7, dtype=torch.int32, device="cuda")
        M.moa_paged_assign(self.plan, *self.tables, self.page, at_, self.ws, start_, None if fresh is None else _int(fresh), slots)
        table = self.tables[0]
        q = M.moa_quant_append(self.plan, *self.cache, table, q, k, v, at_, start_, self.inv_freq, q_out=torch.zeros_like(q))
        if start is None:
            o = M.moa_quant_decode(self.plan, q, *self.cache, table, at_, self.ws, o=torch.full_like(q, 7.0))
        else:
            o = M.moa_quant_prefill(self.plan, q, *self.cache, table, at_, start_, self.ws, o=torch.full_like(q, 7.0))
        torch.cuda.synchronize()
        assert self.tables[2].tolist()[1] == 0, "the pool has no pages left"
        kp, vp = ((c.double() * self.cache[2][..., i].double().repeat_interleave(16, 1)[..., None]).cpu().numpy()
                  for i, c in enumerate(self.cache[:2]))
        rows = oracle.token_rows(at, start)
        ref, a, s = oracle.paged_attention_ref(np.nan_to_num(q.double().cpu().numpy()), kp, vp, table.cpu().numpy(), at, start,
                                               self.windows, self.s)
        got = o.double().cpu().numpy()
        mine = np.array([t for t, _, _ in rows], dtype=int)
        if len(mine):
            bound = attention_bound(ref, a, s, torch.bfloat16, self.d, 400)
            assert (np.abs(got - ref) <= bound)[mine].all()
        assert (np.delete(got, mine, 0) == 7.0).all()
        # the rows that the tables name hold the new values
        flat, vs = vp.reshape(-1, self.d), v.double().cpu().numpy()
        for t, b, p in rows:
            for g in range(self.hkv):
                row = int(slots[t, g])
                assert row == oracle.slot_ref(table.cpu().numpy(), len(kp), self.page, b, g, p) >= 0
                step = 2.0 ** -10 * float(self.cache[2].view(-1, 2)[row // 16, 1])
                assert (np.abs(flat[row] - vs[t, g]) <= np.maximum(2.0 ** -4 * np.abs(vs[t, g]), step)).all()
        return o


@pytest.mark.parametrize("d,hq,page", [(64, 8, 16), (128, 2, 32), (128, 16, 64)])
def test_a_server(d, hq, page):
    """Prompts in chunks, decode steps, sequences that end and others that take their place, in a pool
    that holds what the windows need and not what the sequences are long."""
    _say("server", d, hq, page)
    sv = Server(d=d, hq=hq, page=page, most=512, pages=4 * (512 // page + 120 // page + 12))
    at = [0, 0, -1, 0]
    sv.step(at, [0, 100, 230, 230, 231])
    sv.step([100, 130, 0, 1], [0, 57, 58, 200, 333], [0, 0, 1, 0])
    at = [157, 131, 142, 134]
    for i in range(20):
        sv.step(at)
        at = [p + 1 for p in at]
    sv.step([at[0], at[1], 0, -1], [0, 1, 90, 240, 240], [0, 0, 1, 1])
    at = [at[0] + 1, at[1] + 89, 150, -1]
    for i in range(3):
        sv.step(at)
        at = [p + 1 if p >= 0 else p for p in at]
    sv.step([at[0], -1, at[2], 0], [0, 70, 70, 72, 300], [0, 1, 0, 1])
    used = int((sv.tables[0] >= 0).sum())
    assert used + int(sv.tables[2][0]) == len(sv.tables[1])


def test_block_band_prompts_see_all_their_pages():
    """With the block band a prompt's first rows may see further back than the token-exact band, or less far."""
    _say("block band server")
    sv = Server(windows=(70, 129), flags=M.MOA_BLOCK_BAND, page=16)
    at, total = [0, 5, 0, 0], [0, 0, 0, 0]
    for counts in ([64, 65, 1, 130], [70, 1, 63, 3], [1, 100, 64, 64]):
        start = np.concatenate([[0], np.cumsum(counts)])
        ws, n = sv.ws, int(start[-1])
        q, k, v = sv.tokens(n)
        M.moa_paged_assign(sv.plan, *sv.tables, sv.page, _int(at), ws, _int(start))
        q = M.moa_quant_append(sv.plan, *sv.cache, sv.tables[0], q, k, v, _int(at), _int(start), sv.inv_freq)
        o = M.moa_quant_prefill(sv.plan, q, *sv.cache, sv.tables[0], _int(at), _int(start), ws)
        kp, vp = ((c.double() * sv.cache[2][..., i].double().repeat_interleave(16, 1)[..., None]).cpu().numpy()
                  for i, c in enumerate(sv.cache[:2]))
        table = sv.tables[0].cpu().numpy()
        for t, b, p in oracle.token_rows(at, start):             # every key of a row's mask is there
            for g, w in enumerate(sv.windows):
                first = 5 if b == 1 else 0
                for j in oracle.visible_set(p, w, sv.s, 64):
                    assert j < first or oracle.slot_ref(table, len(kp), sv.page, b, g, int(j)) >= 0, (b, g, p, j)
        ref, a, s = oracle.paged_attention_ref(q.double().cpu().numpy(), kp, vp, table, at, start, sv.windows, sv.s, None, 64)
        assert (np.abs(o.double().cpu().numpy() - ref) <= attention_bound(ref, a, s, torch.bfloat16, sv.d, 400)).all()
        at = [p + c for p, c in zip(at, counts)]


def test_the_last_row_of_a_prompt_is_a_decode_step():
    _say("prefill and decode")
    c = QuantPaged(8, 2, 128, 5, [300, 2000], "bf16", [1500, 0], [40, 700], page=32, seed=3)
    x, o = c.device(), c.run()
    last = _int([1539, 699])
    q = x["q"][[39, 739]].contiguous()
    d = M.moa_quant_decode(c.plan, q, x["k_pages"], x["v_pages"], x["scales"], x["table"], last, x["workspace"])
    ref, a, s = (t[[39, 739]] for t in c.reference())          # both are within the bound of the same row
    bound = attention_bound(ref, a, s, c.dtype, 128, c.width * c.page)
    assert (np.abs((d.double() - o[[39, 739]].double()).cpu().numpy()) <= 2 * bound).all()


def test_large_batches():
    _say("large batch")
    rng = np.random.default_rng(3)
    where = [int(x) for x in rng.integers(-20, 90, size=700)]
    QuantPaged(4, 2, 64, 3, [9, 50], "bf16", where, seed=1).check("decode of 700")
    counts = [int(x) for x in rng.choice([0, 1, 2, 17], size=400)]
    QuantPaged(4, 2, 64, 3, [9, 50], "bf16", where[:400], counts, seed=2, pad=2).check("prefill of 400")
    where = [max(p, -1) if p < 0 else p + 60 for p in where[:300]]
    QuantPaged(4, 2, 64, 3, [9, 100], "bf16", where, prefix_len=60, seed=4).check("shared by 300")


@pytest.mark.parametrize("d,hq,prefix", [(64, 2, 0), (128, 4, 0), (64, 8, 100)])
def test_many_caches_of_several_rounds(d, hq, prefix):
    """At least as many caches as workers (two per compute unit, behind a prefix one), of two rounds of 256 keys or
    more on average: starts count in the split.  Idle sequences, short caches and heads, and long ones among them."""
    _say("many caches", d, hq, prefix)
    rng = np.random.default_rng(7)
    b, s, windows = (150 if prefix else 300), 3, [1400, 200]
    where = prefix + rng.integers(1000, 1500, size=b)
    where[rng.permutation(b)[:40]] = prefix + rng.integers(0, 60, size=40)
    where[[0, 17, 18, b - 1]] = -1
    where[[1, b - 2]] = prefix
    own = [sum(-(-min(max(p + 1 - prefix, 0), w + (s if not prefix else 0)) // 256) for p in where) for w in windows]
    assert sum(own) >= 2 * 2 * b
    QuantPaged(hq, 2, d, s, windows, "bf16", [int(x) for x in where], page=32, prefix_len=prefix, seed=8).check("many")


def test_a_long_sequence_among_many():
    _say("long among many")
    rng = np.random.default_rng(5)
    counts = [int(x) for x in rng.choice([1, 3], size=150)]
    where = [int(x) for x in rng.integers(0, 60, size=150)]
    where[70], counts[70] = 9000, 200
    QuantPaged(2, 2, 64, 5, [3000, 8000], "bf16", where, counts, page=64, seed=6).check("long among many")


def test_pools_beyond_32_bit_offsets():
    """Pages more than 4 GiB into their pool."""
    _say("large pool")
    hq, hkv, d, page, n_pages = 4, 2, 128, 256, 140000
    plan = M.moa_plan(hq, hkv, d, 4, 2000, "bf16", [600.0, 2000.0], [0.0] * hkv)
    kp, vp = (torch.empty((n_pages, page, d), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    sc = torch.empty((n_pages, page // 16, 2), device="cuda")
    assert kp.numel() > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(9)
    n = 700
    q, k, v = (torch.randn((n, h, d), generator=gen, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    table = _int([[[n_pages - 1, n_pages - 5, 133000], [n_pages - 9, 0, 132999]]])
    small = _int([[[0, 1, 2], [3, 4, 5]]])
    ws = M.new_paged_workspace(plan, 1, n)
    at, start = _int([0]), _int([0, n])
    out = []
    for cache, t in (((kp, vp, sc), table), (M.new_quant_cache(plan, 6, page), small)):
        M.moa_quant_append(plan, *cache, t, q, k, v, at, start)
        out.append([M.moa_quant_prefill(plan, q, *cache, t, at, start, ws),
                    M.moa_quant_decode(plan, q[-1:], *cache, t, _int([n - 1]), ws),
                    M.moa_quant_decode_shared(plan, q[-1:], *cache, t[0], 512, t, _int([n - 1]), ws)])
    assert _same(*out) and float(out[0][0].abs().max()) > 0


def test_the_same_call_gives_the_same_bits():
    _say("repeat")
    for kw in (dict(counts=[300, 40, 5]), dict(), dict(prefix_len=250)):
        c = QuantPaged(8, 2, 64, 7, [200, 2500], "bf16", [2100, 900, 260], page=32, seed=8, **kw)
        first = c.run()
        for _ in range(3):
            assert torch.equal(bits(c.run()), bits(first))


def test_absent_pages_after_a_call_that_left_nan_in_lds():
    _say("absent pages, LDS of NaN")
    gone = [(0, 0, 3), (0, 1, 0), (0, 1, 9)]
    for d in (64, 128):
        bad = M.moa_plan(32, 32, d, 0, 512, "bf16", [512.0] * 32, [0.0] * 32)
        x = torch.full((1, 512, 32, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        for counts in ([95], None):
            c = QuantPaged(8, 2, d, 20, [100, 1000], "bf16", [60 if counts else 155], counts, page=16, absent=gone, seed=5)
            for _ in range(3):
                M.moa_prefill(bad, x, x, x)
                c.check("absent after NaN")


# ---------------------------------------------------------------------------
# Call paths, streams, graphs.
# ---------------------------------------------------------------------------
def _everything(stream):
    """All five calls once; stream None takes the native path, a stream the general one."""
    sv = Server(seed=4, batch=3)
    q, k, v = sv.tokens(60)
    at, start, kw = _int([0, 5, -1]), _int([0, 30, 58, 60]), dict(stream=stream)
    slots = torch.full((60, 2), -7, dtype=torch.int32, device="cuda")
    got = M.moa_paged_assign(sv.plan, *sv.tables, sv.page, at, sv.ws, start, _int([1, 0, 0]), slots, **kw)
    assert got is slots
    table = sv.tables[0]
    out = [M.moa_quant_append(sv.plan, *sv.cache, table, q, k, v, at, start, sv.inv_freq, True, torch.zeros_like(q), **kw)]
    out.append(M.moa_quant_prefill(sv.plan, out[0], *sv.cache, table, at, start, sv.ws, torch.zeros_like(q), **kw))
    qd, kd, vd = sv.tokens(3)
    at = _int([30, 33, 40])
    assert M.moa_paged_assign(sv.plan, *sv.tables, sv.page, at, sv.ws, **kw) is None
    assert M.moa_quant_append(sv.plan, *sv.cache, table, None, kd, vd, at, **kw) is None
    out.append(M.moa_quant_decode(sv.plan, qd, *sv.cache, table, at, sv.ws, **kw))
    out.append(M.moa_quant_decode_shared(sv.plan, qd, *sv.cache, table[0], 16, table, at, sv.ws, **kw))
    return out + [slots, *sv.tables, *sv.cache]


def test_native_path_equals_general_path():
    _say("paths")
    a, b = _everything(None), _everything(torch.cuda.current_stream())
    assert _same(a, b) and all(bool(torch.isfinite(x.float()).all()) for x in a) and a[0].any() and a[3].any()


def test_native_path_takes_ordinary_calls_and_leaves_the_others():
    _say("native")
    sv = Server(batch=3)
    q, k, v = sv.tokens(3)
    at, start = _int([0, 1, 2]), _int([0, 1, 2, 3])
    f, p, table = M._fast, sv.plan._bound, sv.tables[0]
    slots = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    asg = [*sv.tables, 16, at, sv.ws, start, _int([0, 0, 0]), slots]
    app = [*sv.cache, table, q, k, v, at, start, sv.inv_freq, False, torch.empty_like(q)]
    pre = [q, *sv.cache, table, at, start, sv.ws, torch.empty_like(q)]
    dec = [q, *sv.cache, table, at, sv.ws, torch.empty_like(q)]
    sha = [q, *sv.cache, table[0], 16, table, at, sv.ws, torch.empty_like(q)]
    assert f.quant_append(p, *app[:-1], None).shape == q.shape
    assert f.quant_append(p, *app[:4], None, k, v, at, None, None, False, None) is True
    assert f.paged_assign(p, *asg[:6], None, None, None) is True
    for name, args, tensors in (("paged_assign", asg, (0, 1, 2, 4, 5, 6, 7, 8)), ("quant_append", app, range(9)),
                                ("quant_prefill", pre, range(9)), ("quant_decode", dec, range(8)),
                                ("quant_decode_shared", sha, (0, 1, 2, 3, 4, 6, 7, 8, 9))):
        call = getattr(f, name)
        assert call(p, *args) is not None
        before = [x.clone() for x in (*sv.tables, *sv.cache)]
        for i in tensors:
            t = args[i]
            wide = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
            odd = [t.cpu(), t.unsqueeze(0), torch.stack((wide, wide), -1)[..., 0].view(t.dtype), t.float() if t.dtype != torch.float32 else t.double()]
            for x in odd:
                if t.dtype == torch.uint8 and x.is_cuda and x.is_contiguous():
                    continue                                     # of a workspace any shape and type
                bad = list(args)
                bad[i] = x
                assert call(p, *bad) is None, (name, i, tuple(x.shape), x.dtype)
        assert _same(before, (*sv.tables, *sv.cache))
        assert call(p, *args[:-1]) is None and call(None, *args) is None
    old = [q, sv.cache[0], sv.cache[1], table, at, sv.ws, torch.empty_like(q)]
    assert f.paged_decode(p, *old) is None                       # 8-bit pages are no bf16 ones


@pytest.mark.parametrize("change,match", [
    (dict(q=lambda x: x[:, :4]), "q: expected shape"), (dict(k=lambda x: x.float()), "k_new: expected dtype"),
    (dict(v=lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)), "heads must be contiguous"),
    (dict(at=lambda x: x.long()), "positions"), (dict(start=lambda x: x[:-1]), "seq_start: expected shape"),
    (dict(table=lambda x: x[:, :1].contiguous()), "table: expected shape"),
    (dict(kp=lambda x: x[:, :, :32].contiguous()), "k_pages: expected shape"), (dict(kp=lambda x: x[0]), "k_pages"),
    (dict(kp=lambda x: x.view(torch.uint8)), "k_pages: expected dtype"), (dict(vp=lambda x: x.bfloat16()), "v_pages: expected dtype"),
    (dict(sc=lambda x: x[:, :, 0].contiguous()), "scales: expected shape"), (dict(sc=lambda x: x.double()), "scales: expected dtype"),
    (dict(sc=lambda x: x.cpu()), "GPU"), (dict(sc=lambda x: None), "scales"),
    (dict(f=lambda x: x[:9]), "rotary_dim"), (dict(out=lambda x: x[:1]), "q_out: expected shape"),
])
def test_refusals_of_append(change, match):
    _say("refused", match)
    sv = Server(batch=3)
    q, k, v = sv.tokens(3)
    x = dict(q=q, k=k, v=v, at=_int([0, 1, 2]), start=_int([0, 1, 2, 3]), table=sv.tables[0], f=sv.inv_freq,
             out=torch.zeros_like(q), kp=sv.cache[0], vp=sv.cache[1], sc=sv.cache[2])
    x["table"].copy_(torch.arange(x["table"].numel()).view(x["table"].shape))
    for name, fn in change.items():
        x[name] = fn(x[name])
    with pytest.raises(M.MoaError, match=match):
        M.moa_quant_append(sv.plan, x["kp"], x["vp"], x["sc"], x["table"], x["q"], x["k"], x["v"], x["at"], x["start"], x["f"],
                           q_out=x["out"])
    assert not any(c.view(torch.uint8).any() for c in sv.cache[:2]) and not sv.cache[2].any()


def test_refusals_of_attention_and_tables():
    _say("refused attention")
    sv = Server(batch=3)
    q, k, v = sv.tokens(3)
    at, start = _int([0, 1, 2]), _int([0, 1, 2, 3])
    names = ("k_pages", "v_pages", "scales")
    args = lambda **kw: {**dict(q=q, table=sv.tables[0], positions=at, workspace=sv.ws), **dict(zip(names, sv.cache)), **kw}
    for bad, match in ((dict(workspace=sv.ws[:256]), "workspace"), (dict(workspace=sv.ws.cpu()), "workspace"),
                       (dict(q=q[:2]), "expected shape"), (dict(q=q.float()), "expected dtype"), (dict(o=q), "overlaps"),
                       (dict(positions=at[None]), "positions"), (dict(scales=None), "scales"),
                       (dict(scales=sv.cache[2][:1]), "scales: expected shape")):
        with pytest.raises(M.MoaError, match=match):
            M.moa_quant_decode(sv.plan, **args(**bad))
    with pytest.raises(M.MoaError, match="seq_start"):
        M.moa_quant_prefill(sv.plan, seq_start=start[:3], **args())
    with pytest.raises(M.MoaError, match="prefix_table"):
        M.moa_quant_decode_shared(sv.plan, prefix_table=sv.tables[0], prefix_len=16, **args())
    with pytest.raises(M.MoaError, match="prefix_len"):
        M.moa_quant_decode_shared(sv.plan, prefix_table=sv.tables[0][0], prefix_len=10 ** 6, **args())
    f32 = M.moa_plan(8, 2, 64, 4, 300, "f32", [40.0, 300.0], [0.0] * 2)
    with pytest.raises(M.MoaError, match="bf16"):
        M.moa_quant_decode(f32, **args(q=q.float()))
    t, free, counts = sv.tables
    before = [x.clone() for x in sv.tables]
    for a, match in (((t[:, :1].contiguous(), free, counts, 16, at, sv.ws), "table: expected shape"),
                     ((t, free.long(), counts, 16, at, sv.ws), "free_pages: expected dtype"),
                     ((t, free, counts[:1], 16, at, sv.ws), "counts: expected shape"), ((t, free, counts, 24, at, sv.ws), "page_size"),
                     ((t, free, counts, 16, at.long(), sv.ws), "positions"), ((t, free, counts, 16, at, sv.ws[:512]), "workspace"),
                     ((t, free, counts, 16, at, sv.ws, start[:2]), "seq_start"), ((t, free, counts, 16, at, sv.ws, None, at[:2]), "fresh"),
                     ((t, free, counts, 16, at, sv.ws, None, None, torch.zeros((4, 2), dtype=torch.int32, device="cuda")), "slots: expected shape"),
                     ((t, free, counts, 16, at, sv.ws, None, None, torch.zeros((0, 2), dtype=torch.int32, device="cuda")), "slots: expected shape"),
                     ((t, free, counts, 16, at, sv.ws, start, None, torch.zeros((3, 3), dtype=torch.int32, device="cuda")), "slots"),
                     ((t, t.view(-1), counts, 16, at, sv.ws), "overlaps")):
        with pytest.raises(M.MoaError, match=match):
            M.moa_paged_assign(sv.plan, *a)
    assert _same(before, sv.tables)


def test_seq_start_that_is_no_packing_harms_nothing():
    _say("odd seq_start")
    sv = Server(batch=3)
    q, k, v = sv.tokens(40)
    sv.tables[0].copy_(torch.arange(sv.tables[0].numel()).view(sv.tables[0].shape))
    buf = torch.full((60, sv.hq, sv.d), 7.0, dtype=q.dtype, device="cuda")
    slots = torch.full((60, 2), -7, dtype=torch.int32, device="cuda")
    for start in ([0, 40, 0, 40], [40, 20, 10, 0], [-5, 10, 30, 40], [0, 10, 30, 100], [0, 2 ** 31 - 1, -2 ** 31, 3]):
        at, ss = _int([0, 0, 0]), _int(start)
        M.moa_quant_append(sv.plan, *sv.cache, sv.tables[0], q, k, v, at, ss, sv.inv_freq, q_out=buf[10:50])
        M.moa_quant_prefill(sv.plan, q, *sv.cache, sv.tables[0], at, ss, sv.ws, o=buf[10:50])
        M.moa_paged_assign(sv.plan, *(t.clone() for t in sv.tables), sv.page, at, sv.ws, ss, None, slots[10:50])
    assert (buf[:10] == 7.0).all() and (buf[50:] == 7.0).all() and (slots[:10] == -7).all() and (slots[50:] == -7).all()


def test_outputs_come_from_the_stream_that_writes_them():
    _say("streams' memory")
    c = QuantPaged(8, 2, 128, 4, [100, 700], "bf16", [1400 - i for i in range(40)], page=64, seed=1)
    p = QuantPaged(8, 2, 128, 4, [100, 700], "bf16", [0], [1500], page=64, seed=2)
    x, y = c.device(), p.device()
    plan, cache, pcache = c.plan, (x["k_pages"], x["v_pages"], x["scales"]), (y["k_pages"], y["v_pages"], y["scales"])
    k, v = (torch.randn((1500, 2, 128), device="cuda").bfloat16() for _ in range(2))
    other = [t.clone() for t in pcache]
    side = torch.cuda.Stream()
    for name, call in {
        "append": lambda s: M.moa_quant_append(plan, *other, y["table"], y["q"], k, v, y["positions"], y["seq_start"], stream=s),
        "prefill": lambda s: M.moa_quant_prefill(plan, y["q"], *pcache, y["table"], y["positions"], y["seq_start"], y["workspace"], stream=s),
        "decode": lambda s: M.moa_quant_decode(plan, x["q"], *cache, x["table"], x["positions"], x["workspace"], stream=s),
        "shared": lambda s: M.moa_quant_decode_shared(plan, x["q"], *cache, x["table"][0], 0, x["table"], x["positions"], x["workspace"], stream=s),
    }.items():
        print("[case]", name, flush=True)
        ref = call(None)
        torch.cuda.synchronize()
        held = torch.empty_like(ref)
        at = held.data_ptr()
        del held                                             # the current stream's next block of this size
        out = call(side)
        torch.cuda.synchronize()
        assert out.data_ptr() != at, name
        assert torch.equal(bits(out), bits(ref)) and bool(ref.any()), name


def test_two_streams_at_once():
    _say("two streams")
    cases = [QuantPaged(8, 2, 128, 4, [900, 60], "bf16", [1200, 777], seed=i) for i in range(2)]
    refs, streams, xs = [c.run() for c in cases], [torch.cuda.Stream() for _ in cases], [c.device() for c in cases]
    outs = [torch.zeros_like(x["q"]) for x in xs]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, x, o, s in zip(cases, xs, outs, streams):
            with torch.cuda.stream(s):
                M.moa_quant_decode(c.plan, x["q"], x["k_pages"], x["v_pages"], x["scales"], x["table"], x["positions"], x["workspace"], o=o)
    torch.cuda.synchronize()
    assert _same(outs, refs)


def _captured(call):
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.synchronize()
    return graph


@pytest.mark.parametrize("shared_ws", [False, True])
def test_a_captured_serving_step(shared_ws):
    """Tables, append, decode and the next positions in one graph, of two servers whose graphs may share a
    workspace: every replay equals the eager step, tables and cache included, bit for bit."""
    _say("graph", shared_ws)
    steps = 40
    sides = [[Server(seed=7 + i, windows=(20 + 30 * i, 150)) for i in range(2)] for _ in range(2)]     # eager, captured
    if shared_ws:
        sides[1][1].ws = sides[1][0].ws
    state = []
    for group in sides:
        for sv in group:
            q, k, v = sv.tokens(400)
            at, start = _int([0, 0, 3, 0]), _int([0, 100, 190, 330, 400])
            M.moa_paged_assign(sv.plan, *sv.tables, sv.page, at, sv.ws, start)
            M.moa_quant_append(sv.plan, *sv.cache, sv.tables[0], None, k, v, at, start)
            state.append(dict(sv=sv, q=torch.zeros_like(q[:4]), k=torch.zeros_like(k[:4]), v=torch.zeros_like(v[:4]),
                              at=_int([100, 90, 143, 70]), o=torch.zeros_like(q[:4]), slots=_int(np.zeros((4, 2)))))

    def step(x):
        sv = x["sv"]
        M.moa_paged_assign(sv.plan, *sv.tables, sv.page, x["at"], sv.ws, None, None, x["slots"])
        qr = M.moa_quant_append(sv.plan, *sv.cache, sv.tables[0], x["q"], x["k"], x["v"], x["at"], inv_freq=sv.inv_freq)
        M.moa_quant_decode(sv.plan, qr, *sv.cache, sv.tables[0], x["at"], sv.ws, o=x["o"])
        x["at"].add_(1)

    graphs = [_captured(lambda x=x: step(x)) for x in state[2:]]
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(steps):
        for x in state[:2]:
            for name in "qkv":
                x[name].copy_(torch.randn(x[name].shape, generator=gen, device="cuda"))
        for x, y in zip(state[:2], state[2:]):
            for name in "qkv":
                y[name].copy_(x[name])
        for x in state[:2]:
            step(x)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for x, y in zip(state[:2], state[2:]):
            assert torch.equal(bits(x["o"]), bits(y["o"])) and x["o"].any(), i
            assert _same((x["at"], x["slots"], *x["sv"].tables, *x["sv"].cache), (y["at"], y["slots"], *y["sv"].tables, *y["sv"].cache)), i
    assert int(state[0]["sv"].tables[2][1]) == 0


def test_a_captured_prefill_and_shared_decode():
    _say("graph of a prefill")
    for kw in (dict(positions=[2300, 10], counts=[90, 200]), dict(positions=[2300, 2250], prefix_len=2200)):
        c = QuantPaged(8, 2, 64, 4, [2500, 100], "bf16", page=32, seed=12, **kw)
        ref, x = c.run(), c.device()
        o, cache = torch.zeros_like(x["q"]), (x["k_pages"], x["v_pages"], x["scales"])
        if "counts" in kw:
            call = lambda: M.moa_quant_prefill(c.plan, x["q"], *cache, x["table"], x["positions"], x["seq_start"], x["workspace"], o=o)
        else:
            call = lambda: M.moa_quant_decode_shared(c.plan, x["q"], *cache, x["prefix_table"], 2200, x["table"], x["positions"],
                                                     x["workspace"], o=o)
        graph = _captured(call)
        for _ in range(3):
            o.zero_()
            x["workspace"].fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(bits(o), bits(ref))
            call()
            torch.cuda.synchronize()
            assert torch.equal(bits(o), bits(ref))
