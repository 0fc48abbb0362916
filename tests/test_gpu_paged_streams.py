"""Outputs of calls on a stream that is not the current one come from that stream's memory: a block that work of
the current stream may still use is not written by them."""
import pytest
import torch

from helpers import bits
from paper_2406_14909_amd import moa as M

pytestmark = pytest.mark.gpu

HQ, HKV, D, N, B = 8, 2, 128, 1500, 40


def _calls():
    """name: a call that makes its output, given its stream."""
    plan = M.moa_plan(HQ, HKV, D, 4, N, "bf16", [100.0, 700.0], [0.0] * HKV)
    gen = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()
    at = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q, k, v = draw(N, HQ, D), draw(N, HKV, D), draw(N, HKV, D)
    width = -(-N // 64)
    table = torch.arange(HKV * width, dtype=torch.int32, device="cuda").view(1, HKV, width)
    kp, vp = M.new_paged_cache(plan, HKV * width, 64)
    ws = M.new_paged_workspace(plan, B, N)
    freq = torch.logspace(0, -3, D // 2, device="cuda")
    zero, start = at([0]), at([0, N])
    M.moa_paged_append(plan, kp, vp, table, None, k, v, zero, start)
    kp2, vp2 = kp.clone(), vp.clone()
    many, wide = at([N - 1 - i for i in range(B)]), table.expand(B, HKV, width).contiguous()
    qd = q[:B].contiguous()
    kc, vc, pc = M.new_cache(plan, B)
    M.moa_kv_append(plan, kc, vc, pc, k[None].expand(B, N, HKV, D).contiguous(), v[None].expand(B, N, HKV, D).contiguous(), 0)
    ws2 = M.new_workspace(plan, B)
    return {
        "paged_append": lambda s: M.moa_paged_append(plan, kp2, vp2, table, q, k, v, zero, start, freq, stream=s),
        "paged_prefill": lambda s: M.moa_paged_prefill(plan, q, kp, vp, table, zero, start, ws, stream=s),
        "paged_decode": lambda s: M.moa_paged_decode(plan, qd, kp, vp, wide, many, ws, stream=s),
        "paged_decode_shared": lambda s: M.moa_paged_decode_shared(plan, qd, kp, vp, table[0], 1000, wide, many, ws, stream=s),
        "prefill": lambda s: M.moa_prefill(plan, q[None], k[None], v[None], stream=s),
        "decode": lambda s: M.moa_decode(plan, qd, kc, vc, N - 1, ws2, stream=s),
        "decode_ragged": lambda s: M.moa_decode_ragged(plan, qd, kc, vc, many, ws2, stream=s),
    }


def test_outputs_come_from_the_stream_that_writes_them():
    side = torch.cuda.Stream()
    for name, call in _calls().items():
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
