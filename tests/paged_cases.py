"""Page pools with scattered pages, and the tolerances of the paged operators."""
import numpy as np
import torch

import oracle
from paper_2406_14909_amd import moa as M


class Paged:
    """A pool whose pages hold the positions that the queries of a call see, in shuffled
    order; all other rows, pages and table entries hold what nothing may look at."""

    def __init__(self, hq, hkv, d, s, windows, dt, positions, counts=None, page=16, flags=0, prefix_len=0, seed=0,
                 pad=0, lead=0, fill=float("nan"), spare=3, absent=(), scale=0.0):
        n = max(windows) + s
        self.plan = M.moa_plan(hq, hkv, d, s, n, dt, [float(w) + (s if flags & 1 else 0) for w in windows], [0.0] * hkv,
                               scale, flags)
        if not flags & 1:
            assert list(self.plan.window) == list(windows)
        self.windows, self.s, self.block = [int(w) for w in self.plan.window], s, 64 if flags & 2 else 0
        self.positions, self.prefix_len, self.page = list(positions), prefix_len, page
        self.dtype = self.plan.torch_dtype
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        draw = lambda *shape: torch.randn(shape, generator=gen).to(self.dtype)
        b = len(positions)
        self.seq_start = None
        rows = b
        block = 0
        if counts is not None:
            self.seq_start = [lead] + [lead + int(x) for x in np.cumsum(counts)]
            rows, block = self.seq_start[-1] + pad, self.block
        seen = {}
        for t, i, p in oracle.token_rows(self.positions, self.seq_start):
            for g, w in enumerate(self.windows):
                seen.setdefault((i, g), set()).update(oracle.visible_set(p, w, s, block).tolist())
        longest = max([max(x) + 1 for x in seen.values() if x] + [prefix_len, 1])
        self.width = -(-longest // page) + 1
        own, pre = set(), set()
        for (i, g), keys in seen.items():
            own |= {(i, g, j // page) for j in keys if j >= prefix_len}
            pre |= {(g, j // page) for j in keys if j < prefix_len}
        wanted = sorted(own) + sorted(pre)
        self.num_pages = len(wanted) + spare
        order = rng.permutation(self.num_pages)[:len(wanted)]
        # entries that no key needs: absent pages and present ones with nothing in them alike
        odd = np.array([-1, -2 ** 31, 2 ** 31 - 1, self.num_pages, 0], dtype=np.int64).astype(np.int32)
        self.table = rng.choice(odd, size=(b, hkv, self.width))
        self.prefix_table = rng.choice(odd, size=(hkv, self.width))
        k = torch.full((self.num_pages, page, d), fill, dtype=self.dtype)
        v = k.clone()
        for where, n_page in zip(wanted, order):
            if len(where) == 3:
                self.table[where] = n_page
            else:
                self.prefix_table[where] = n_page
        for (i, g), keys in seen.items():
            for j in sorted(keys):
                row = int(self.prefix_table[g, j // page] if j < prefix_len else self.table[i, g, j // page])
                if not torch.isfinite(k[row, j % page]).all():
                    k[row, j % page], v[row, j % page] = draw(d) + (0.5 if j < 4 else 0.0), draw(d)
        for i, g, x in absent:                       # pages taken away: numbers out of range of either kind
            self.table[i, g, x] = [-1, self.num_pages, -2 ** 31, 2 ** 31 - 1][(i + g + x) % 4]
        self.k, self.v = k, v
        self.q = torch.full((rows, hq, d), fill, dtype=self.dtype)
        for t, _, _ in oracle.token_rows(self.positions, self.seq_start):
            self.q[t] = draw(hq, d) + 0.5

    def device(self):
        """Arguments of the calls, on the GPU."""
        at = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        return dict(q=self.q.cuda(), k_pages=self.k.cuda(), v_pages=self.v.cuda(), table=at(self.table),
                    positions=at(self.positions), seq_start=None if self.seq_start is None else at(self.seq_start),
                    prefix_table=at(self.prefix_table),
                    workspace=M.new_paged_workspace(self.plan, len(self.positions), self.q.shape[0]).fill_(0xFF))

    def reference(self):
        nan0 = lambda x: torch.nan_to_num(x.float(), nan=0.0).double().numpy()
        return oracle.paged_attention_ref(nan0(self.q), nan0(self.k), nan0(self.v), self.table, self.positions,
                                          self.seq_start, self.windows, self.s,
                                          float(self.plan.desc.softmax_scale) or None,
                                          self.block if self.seq_start is not None else 0, self.prefix_table,
                                          self.prefix_len)

    def run(self, stream=None, o=None):
        """The call of this case, on an output of sevens."""
        x = self.device()
        o = torch.full_like(x["q"], 7.0) if o is None else o
        if self.seq_start is not None:
            M.moa_paged_prefill(self.plan, x["q"], x["k_pages"], x["v_pages"], x["table"], x["positions"],
                                x["seq_start"], x["workspace"], o=o, stream=stream)
        elif self.prefix_len:
            M.moa_paged_decode_shared(self.plan, x["q"], x["k_pages"], x["v_pages"], x["prefix_table"], self.prefix_len,
                                      x["table"], x["positions"], x["workspace"], o=o, stream=stream)
        else:
            M.moa_paged_decode(self.plan, x["q"], x["k_pages"], x["v_pages"], x["table"], x["positions"],
                               x["workspace"], o=o, stream=stream)
        torch.cuda.synchronize()
        return o

    def check(self, what=""):
        got = self.run().double().cpu().numpy()
        ref, a, s = self.reference()
        mine = ~np.isnan(ref)
        assert (got[~mine] == 7.0).all(), f"{what}: rows of no sequence were written"
        err = np.abs(got - ref)
        bound = attention_bound(ref, a, s, self.dtype, self.q.shape[2], max(1, self.width * self.page))
        worst = np.where(mine, err - bound, -np.inf)
        assert np.isfinite(got).all() and (worst <= 0).all(), (
            f"{what}: {int((worst > 0).sum())} of {mine.sum()} off, worst {np.nanmax(err):.3e} at "
            f"{np.unravel_index(np.argmax(worst), worst.shape)}")
        return float(np.nanmax(np.where(mine, err / np.maximum(bound, 1e-30), 0.0)))


def attention_bound(o, a, s, dtype, d, n):
    """How far outputs may be off: a the weighted mean of |v|, s the largest scale * sum |q k| of
    the row, d terms per score, at most n keys.

    fp32: a score's products and sums are off by about sqrt(d) half steps of s, its exponent (in base 2)
    by 4 half steps of s, the exponential by 2 and the sums of n weights by sqrt(n); errors of weights
    count twice (numerator and denominator), four times their size is allowed:
    4 * 2 * 2^-24 * ((sqrt(d) + 4) * s + sqrt(n) + 4) * a.
    bf16 outputs and weights: a weight is rounded once (2^-8 of itself), which moves the quotient by at
    most 2^-8 (a + |o|), and the output once more, 2^-8 |o|."""
    f32 = 8 * 2.0 ** -24 * ((np.sqrt(d) + 4) * s[..., None] + np.sqrt(n) + 4) * a
    if dtype == torch.float32:
        return f32 + 2.0 ** -24 * np.abs(o)
    return f32 + 2.0 ** -8 * (a + 2 * np.abs(o))


def rotation_bound(u, v, out, dtype):
    """u, v: magnitudes of the pair.  fp32 angles in turns are off by 2^-25, their sines and cosines by that
    times 2 pi and a few half steps, 2^-22 in all; products and their sum three half steps; the result is
    rounded once."""
    return (2.0 ** -22 + 3 * 2.0 ** -24) * (u + v) + torch.finfo(dtype).eps / 2 * np.abs(out)
