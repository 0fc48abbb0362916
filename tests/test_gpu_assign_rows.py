"""Page tables without slots: the number of packed rows says which sequences get pages, as slots do."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q
from paper_2406_14909_amd import moa as M

pytestmark = pytest.mark.gpu


def _int(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("general", [False, True])
@pytest.mark.parametrize("start", [[0, 20, 40, 60], [0, 20, 40, 41], [-1, 20, 30, 40], [0, 20, 20, 20], [5, 50, 30, 40], [0, 39, 40, 2 ** 31 - 1]])
def test_rows_as_with_slots(start, general):
    print("[case] rows", start, general, flush=True)
    plan = M.moa_plan(2, 2, 64, 4, 300, "bf16", [20.0, 300.0], [0.0] * 2)
    kw = dict(stream=torch.cuda.current_stream()) if general else {}
    ws, at, rows = M.new_paged_workspace(plan, 3, 40), [0, 30, 5], 40
    a, b = M.new_page_tables(plan, 3, 8, 48), M.new_page_tables(plan, 3, 8, 48)
    slots = torch.full((rows, 2), -7, dtype=torch.int32, device="cuda")
    M.moa_paged_assign(plan, *a, 16, _int(at), ws, _int(start), None, slots, **kw)
    M.moa_paged_assign(plan, *b, 16, _int(at), ws, _int(start), n_tokens=rows, **kw)
    torch.cuda.synchronize()
    want = Q.assign_ref(*(t.cpu().numpy() for t in M.new_page_tables(plan, 3, 8, 48)), 16, at, start, None, rows, [20, 300], 4, False)
    for x, y, z in zip(a, b, want):
        assert torch.equal(x, y) and np.array_equal(y.cpu().numpy(), z)


def test_rows_that_slots_contradict():
    plan = M.moa_plan(2, 2, 64, 4, 300, "bf16", [20.0, 300.0], [0.0] * 2)
    t, ws, at = M.new_page_tables(plan, 3, 8, 48), M.new_paged_workspace(plan, 3, 40), _int([0, 1, 2])
    before, start = [x.clone() for x in t], _int([0, 1, 2, 3])
    slots = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    for bad in (dict(n_tokens=4, slots=slots), dict(n_tokens=-1), dict(n_tokens=1 << 30)):
        with pytest.raises(M.MoaError, match="n_tokens"):
            M.moa_paged_assign(plan, *t, 16, at, ws, start, **bad)
    assert all(torch.equal(x, y) for x, y in zip(before, t))
    assert M.moa_paged_assign(plan, *t, 16, at, ws, start, None, slots, n_tokens=3) is slots and (t[0][:, :, 0] >= 0).all()


def test_the_native_path_takes_ordinary_calls_and_leaves_the_others():
    plan = M.moa_plan(2, 2, 64, 4, 300, "bf16", [20.0, 300.0], [0.0] * 2)
    t, ws, at, start = M.new_page_tables(plan, 3, 8, 48), M.new_paged_workspace(plan, 3, 40), _int([0, 1, 2]), _int([0, 1, 2, 3])
    slots, scales, lacked = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.zeros((50, 1, 2), device="cuda"), _int([0] * 3)
    args = [*t, 16, at, ws, start, None, slots, scales, lacked, None]
    call = lambda x: M._fast.paged_assign_state(plan._bound, *x)
    assert call(args) is True
    assert call([*args[:8], None, None, None, 3]) is True and call([*args[:8], None, None, None, None]) is True
    before = [x.clone() for x in (*t, slots, scales, lacked)]
    for i, odd in ((9, scales.cpu()), (9, scales.double()), (9, scales[:40]), (9, scales[:, 0]), (9, scales.transpose(0, 2)),
                   (9, torch.zeros((50, 2, 2), device="cuda")), (10, lacked.cpu()), (10, lacked.long()), (10, lacked[:2]),
                   (10, _int([0] * 6)[::2]), (11, 3), (11, 3.0), (11, lacked), (8, slots[:, :1]), (3, 16.0)):
        bad = list(args)
        bad[i] = odd
        assert call(bad) is None, (i, odd)
    assert call(args[:-1]) is None
    assert all(torch.equal(x, y) for x, y in zip(before, (*t, slots, scales, lacked)))
