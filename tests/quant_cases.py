"""8-bit pools for the attention calls, from the bf16 ones of paged_cases."""
import numpy as np
import torch

import oracle
from oracle import quant_oracle as Q
from paged_cases import Paged
from paper_2406_14909_amd import moa as M


def pack(x, rng):
    """(codes uint8, scales fp64 [pages, page / 16], what they stand for) of pages in bf16; scales of blocks
    without a number are what nothing may look at."""
    x = x.double().numpy()
    pages, page, d = x.shape
    blocks = x.reshape(pages, page // 16, 16, d)
    real = np.isfinite(blocks)
    amax = np.where(real, np.abs(blocks), 0.0).max(axis=(2, 3))
    scales = np.array([2.0 ** Q.exponent_ref(a) for a in amax.ravel()]).reshape(amax.shape)
    codes = Q.encode_ref(blocks / scales[..., None, None]).reshape(x.shape)
    values = (Q.decode_ref(codes).reshape(blocks.shape) * scales[..., None, None]).reshape(x.shape)
    odd = rng.choice([np.nan, 0.0, np.inf, -1.0, 1e-45], size=amax.shape)
    return codes, np.where(real.any(axis=(2, 3)), scales, odd), values


class QuantPaged(Paged):
    """The same sequences over an 8-bit cache."""

    def __init__(self, *args, seed=0, **more):
        super().__init__(*args, seed=seed, **more)
        self.seed = seed

    def packed(self):
        """Codes, scales and values of both pools; rows that hold NaN are no numbers in 8 bits either."""
        rng = np.random.default_rng(self.seed + 1)
        return [pack(x, rng) for x in (self.k, self.v)]

    def device(self):
        (kc, ks, _), (vc, vs, _) = self.packed()
        x = super().device()
        x["k_pages"], x["v_pages"] = (torch.from_numpy(c).cuda().view(torch.float8_e4m3fn) for c in (kc, vc))
        x["scales"] = torch.from_numpy(np.stack((ks, vs), -1).astype(np.float32)).cuda()
        return x

    def reference(self, keep_nan=False):
        (_, _, k), (_, _, v) = self.packed()
        zero = (lambda x: x) if keep_nan else (lambda x: np.nan_to_num(x, nan=0.0))
        q = self.q.double().numpy()
        return oracle.paged_attention_ref(zero(q), zero(k), zero(v), self.table, self.positions, self.seq_start,
                                          self.windows, self.s, float(self.plan.desc.softmax_scale) or None,
                                          self.block if self.seq_start is not None else 0, self.prefix_table,
                                          self.prefix_len)

    def run(self, stream=None, o=None):
        x = self.device()
        o = torch.full_like(x["q"], 7.0) if o is None else o
        cache = (x["k_pages"], x["v_pages"], x["scales"])
        if self.seq_start is not None:
            M.moa_quant_prefill(self.plan, x["q"], *cache, x["table"], x["positions"], x["seq_start"], x["workspace"],
                                o=o, stream=stream)
        elif self.prefix_len:
            M.moa_quant_decode_shared(self.plan, x["q"], *cache, x["prefix_table"], self.prefix_len, x["table"],
                                      x["positions"], x["workspace"], o=o, stream=stream)
        else:
            M.moa_quant_decode(self.plan, x["q"], *cache, x["table"], x["positions"], x["workspace"], o=o, stream=stream)
        torch.cuda.synchronize()
        return o
