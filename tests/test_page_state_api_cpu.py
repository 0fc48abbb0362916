"""Argument checks of the page tables with what is kept besides them: they return before anything is launched, so
they run without a GPU.  Addresses here are numbers that nothing reads."""
import ctypes
import os
import re

import pytest

from conftest import ROOT
from paper_2406_14909_amd import moa as M

lib = M.load_library()
A = 1 << 40                                          # distinct regions of 1 TiB
BAD, UNSUP, WS = M.MOA_ERR_INVALID_ARG, M.MOA_ERR_UNSUPPORTED, M.MOA_ERR_WORKSPACE


def assign(p, batch=3, n=3, num_pages=100, page_size=64, max_pages=20, ws_bytes=None, state=True, **over):
    x = dict(dict(table=7 * A, free_pages=15 * A, counts=16 * A, positions=8 * A, seq_start=9 * A, fresh=17 * A, slots=18 * A,
                  workspace=12 * A, scales=14 * A, lacked=19 * A), **over)
    t = M.moa_page_tables_t(x["table"], x["free_pages"], x["counts"], num_pages, page_size, max_pages)
    s = M.moa_page_state_t(**{name: x[name] for name, _ in M.moa_page_state_t._fields_})
    if ws_bytes is None:
        ws_bytes = lib.moa_paged_workspace_bytes(p.handle, batch, max(n, 1))
    return lib.moa_paged_assign_state(p.handle, ctypes.byref(t), ctypes.byref(s) if state else None, x["positions"],
                                      x["seq_start"], x["fresh"], x["slots"], batch, n, x["workspace"], ws_bytes, None)


def plan(dtype="bf16"):
    return M.moa_plan(8, 2, 128, 4, 1000, dtype, [100.0] * 2, [0.0] * 2)


@pytest.mark.parametrize("kw,status", [
    (dict(scales=14 * A + 4), BAD), (dict(scales=7 * A), BAD), (dict(scales=15 * A), BAD), (dict(scales=16 * A), BAD),
    (dict(scales=18 * A), BAD), (dict(scales=8 * A), BAD), (dict(scales=9 * A), BAD), (dict(scales=17 * A), BAD),
    (dict(scales=12 * A), BAD), (dict(scales=15 * A - 100 * 4 * 8 + 8), BAD),
    (dict(lacked=19 * A + 2), BAD), (dict(lacked=7 * A), BAD), (dict(lacked=14 * A), BAD), (dict(lacked=17 * A), BAD),
    (dict(lacked=17 * A - 4), BAD), (dict(lacked=8 * A + 4), BAD), (dict(lacked=12 * A), BAD), (dict(lacked=16 * A + 4), BAD),
    (dict(table=None), BAD), (dict(counts=12 * A), BAD), (dict(workspace=None), WS), (dict(ws_bytes=100), WS),
    (dict(page_size=24), UNSUP), (dict(seq_start=None, n=4), BAD), (dict(n=1 << 30), BAD), (dict(n=1 << 29), UNSUP),
    (dict(n=1 << 29, state=False), UNSUP), (dict(n=1 << 29, scales=None), UNSUP), (dict(table=None, state=False), BAD),
])
def test_refusals(kw, status):
    assert assign(plan(), **kw) == status
    assert lib.moa_last_error().decode().startswith("moa_paged_assign_state")


def test_an_8_bit_cache_takes_bf16_plans():
    assert assign(plan("f32")) == UNSUP and "bf16" in lib.moa_last_error().decode()
    assert assign(plan("f32"), scales=None, n=1 << 29) == UNSUP and "too much" in lib.moa_last_error().decode()


def test_the_struct_is_the_header_s():
    text = open(os.path.join(ROOT, "include", "moa.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\} moa_page_state_t;", text).group(1)
    names = re.findall(r"\*\s*(\w+);", re.sub(r"/\*.*?\*/", "", body, flags=re.S))
    assert names == [name for name, _ in M.moa_page_state_t._fields_]
