"""The paged operators within the bounds of their roundings, element by element: where sums over many keys are
small against the values, a key too many or too few is far outside them."""
import numpy as np
import pytest
import torch

import oracle
from helpers import bits
from paged_cases import Paged, attention_bound
from paper_2406_14909_amd import moa as M
from test_gpu_paged_use import Server

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _near(o, q, kp, vp, table, at, start, windows, s, block=0, prefix=None, prefix_len=0, what=""):
    """o against the oracle over what the pages hold, each element within attention_bound."""
    f64 = lambda x: x.double().cpu().numpy()
    ref, a, sc = oracle.paged_attention_ref(f64(q), f64(kp), f64(vp), table.cpu().numpy(), at.tolist(),
                                            None if start is None else start.tolist(), windows, s, None, block,
                                            None if prefix is None else prefix.cpu().numpy(), prefix_len)
    mine = ~np.isnan(ref)
    err = np.abs(f64(o) - ref)[mine]
    bound = attention_bound(ref, a, sc, o.dtype, q.shape[2], table.shape[2] * kp.shape[1])[mine]
    assert mine.any() and (err <= bound).all(), (what, float((err / bound).max()))


@pytest.mark.parametrize("dt,d,hq", [("bf16", 64, 8), ("bf16", 128, 2), ("f32", 64, 4), ("f32", 128, 16)])
def test_a_server(dt, d, hq):
    """A prompt in chunks, a question per sequence in one ragged call, decode steps with and without the prefix."""
    print("[case]", dt, d, hq, flush=True)
    sv = Server(dt=dt, d=d, hq=hq, prefix=208)                # whole pages, which all sequences share
    w, s = sv.windows, sv.s
    done = 0
    for n in (100, 1, 107):
        q, k, v = sv.tokens(n)
        at, start, table = _int([done]), _int([0, n]), sv.table[:1].contiguous()
        q = M.moa_paged_append(sv.plan, sv.kp, sv.vp, table, q, k, v, at, start, sv.inv_freq)
        o = M.moa_paged_prefill(sv.plan, q, sv.kp, sv.vp, table, at, start, sv.ws)
        _near(o, q, sv.kp, sv.vp, table, at, start, w, s, what="prompt")
        done += n
    start, at = _int([0, 7, 40, 41]), _int([208] * 3)
    q, k, v = sv.tokens(41)
    q = M.moa_paged_append(sv.plan, sv.kp, sv.vp, sv.table, q, k, v, at, start, sv.inv_freq)
    o = M.moa_paged_prefill(sv.plan, q, sv.kp, sv.vp, sv.table, at, start, sv.ws)
    _near(o, q, sv.kp, sv.vp, sv.table, at, start, w, s, what="question")
    at = at + _int([7, 33, 1])
    for _ in range(3):
        q, k, v = sv.tokens(3)
        q = M.moa_paged_append(sv.plan, sv.kp, sv.vp, sv.table, q, k, v, at, inv_freq=sv.inv_freq)
        o = M.moa_paged_decode(sv.plan, q, sv.kp, sv.vp, sv.table, at, sv.ws)
        _near(o, q, sv.kp, sv.vp, sv.table, at, None, w, s, what="decode")
        o = M.moa_paged_decode_shared(sv.plan, q, sv.kp, sv.vp, sv.table[0], 208, sv.table, at, sv.ws)
        _near(o, q, sv.kp, sv.vp, sv.table, at, None, w, s, 0, sv.table[0], 208, "shared")
        at += 1


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n,flags", [(333, 0), (1500, 2)])
def test_a_whole_prompt(dt, n, flags):
    """A whole prompt, and the dense prefill of the same rows, both within their roundings of the oracle."""
    print("[case]", dt, n, flags, flush=True)
    hq, hkv, d, w = 8, 2, 128, [100, 700]
    plan = M.moa_plan(hq, hkv, d, 10, n, dt, [float(min(x, n)) for x in w], [0.0] * hkv, flags=flags)
    w = [int(x) for x in plan.window]
    gen = torch.Generator(device="cuda").manual_seed(n)
    q, k, v = (torch.randn((n, h, d), generator=gen, device="cuda").to(plan.torch_dtype) for h in (hq, hkv, hkv))
    width = -(-n // 64)
    table = torch.randperm(hkv * width, generator=gen, device="cuda").int().view(1, hkv, width)
    kp, vp = M.new_paged_cache(plan, hkv * width, 64)
    at, start = _int([0]), _int([0, n])
    M.moa_paged_append(plan, kp, vp, table, None, k, v, at, start)
    o = M.moa_paged_prefill(plan, q, kp, vp, table, at, start, M.new_paged_workspace(plan, 1, n))
    _near(o, q, kp, vp, table, at, start, w, 10, 64 if flags & 2 else 0, what="paged")
    dense = M.moa_prefill(plan, q[None], k[None], v[None])[0]
    _near(dense, q, kp, vp, table, at, start, w, 10, 64 if flags & 2 else 0, what="dense")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("counts,prefix", [(None, 0), (None, 150), ((130, 1, 40), 0), ((700, 5, 3), 0)])
def test_tables_made_for_longer_sequences(dt, counts, prefix):
    """A table is as wide as the longest sequence that a server takes; the split goes by its width, too."""
    print("[case]", dt, counts, prefix, flush=True)
    for hq, hkv, d in ((8, 2, 128), (2, 2, 64)):
        c = Paged(hq, hkv, d, 4, [100, 600], dt, [200, 160, 333], counts, page=16, prefix_len=prefix, seed=7, pad=2 if counts else 0)
        c.check("narrow")
        more = 4096 // 16 - c.width
        odd = np.random.default_rng(1).choice(np.array([-1, 0, c.num_pages, 2 ** 31 - 1]), (len(c.positions), hkv, more))
        c.table = np.concatenate([c.table, odd.astype(np.int32)], 2)
        c.prefix_table = np.concatenate([c.prefix_table, odd[0].astype(np.int32)], 1)
        c.check("wide")                  # whose bound is that of the keys there are


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_prefix_of_no_keys(dt):
    """The same bits as the call without one, and the oracle's values."""
    print("[case]", dt, flush=True)
    c = Paged(4, 2, 128, 4, [100, 20], dt, [0, 50, 200, -1], seed=1)
    c.check("decode")
    x, plain = c.device(), c.run()
    o = M.moa_paged_decode_shared(c.plan, x["q"], x["k_pages"], x["v_pages"], x["prefix_table"], 0, x["table"],
                                  x["positions"], x["workspace"], o=torch.full_like(x["q"], 7.0))
    assert torch.equal(bits(o), bits(plain))


def fine_bound(o, a, s, d, n):
    """attention_bound of bf16 where weights keep 16 bits, in two parts of 8: the part that is left over is off by
    2^-8 of itself, so a weight by 2^-16, and the quotient, whose sum is that of the same parts, by at most
    2^-16 (a + |o|); the output is rounded once, 2^-8 |o|."""
    return attention_bound(o, a, s, torch.float32, d, n) + 2.0 ** -16 * (a + np.abs(o)) + 2.0 ** -8 * np.abs(o)


@pytest.mark.parametrize("heads,d", [(2, 128), (2, 64), (1, 128), (3, 64)])
def test_decode_of_single_heads_rounds_its_outputs_and_little_else(heads, d):
    """Whole caches and cut ones, against sums that are small beside the values."""
    print("[case]", heads, d, flush=True)
    c = Paged(heads, heads, d, 4, [100, 2500, 900][-heads:], "bf16", [3000, 90, 700, -1, 2222], page=32, seed=6)
    got = c.run().double().cpu().numpy()
    ref, a, s = c.reference()
    mine = ~np.isnan(ref)
    bound = fine_bound(ref, a, s, d, c.width * c.page)
    worst = np.where(mine, np.abs(got - ref) / bound, 0.0)
    assert worst.max() <= 1.0, (worst.max(), int((worst > 1).sum()), int(mine.sum()))
