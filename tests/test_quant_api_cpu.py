"""Argument checks of the page tables and of the 8-bit cache: they return before anything is launched, so
they run without a GPU.  Addresses here are numbers that nothing reads."""
import ctypes

import pytest

from paper_2406_14909_amd import moa as M

lib = M.load_library()
A = 1 << 40                                          # distinct regions of 1 TiB
BASE = dict(q=1 * A, k_new=2 * A, v_new=3 * A, q_out=4 * A, k_pages=5 * A, v_pages=6 * A, table=7 * A, positions=8 * A,
            seq_start=9 * A, inv_freq=10 * A, o=11 * A, workspace=12 * A, prefix_table=13 * A, scales=14 * A,
            free_pages=15 * A, counts=16 * A, fresh=17 * A, slots=18 * A)
BAD, UNSUP, WS = M.MOA_ERR_INVALID_ARG, M.MOA_ERR_UNSUPPORTED, M.MOA_ERR_WORKSPACE


def plan(hq=8, hkv=2, d=128, dtype="bf16"):
    return M.moa_plan(hq, hkv, d, 4, 1000, dtype, [100.0] * hkv, [0.0] * hkv)


def call(name, p, batch=3, n=3, num_pages=100, page_size=64, max_pages=20, strides=(1024, 256, 256), rope=(64, 0),
         ws_bytes=None, prefix_len=100, **over):
    x = dict(BASE, **over)
    handle = None if p is None else p.handle
    if ws_bytes is None:
        ws_bytes = 0 if p is None else lib.moa_paged_workspace_bytes(handle, batch, n)
    if name == "assign":
        t = M.moa_page_tables_t(x["table"], x["free_pages"], x["counts"], num_pages, page_size, max_pages)
        ref = None if x.get("pages", 1) is None else ctypes.byref(t)
        return lib.moa_paged_assign(handle, ref, x["positions"], x["seq_start"], x["fresh"], x["slots"], batch, n,
                                    x["workspace"], ws_bytes, None)
    pages = M.moa_quant_pages_t(x["k_pages"], x["v_pages"], x["scales"], x["table"], num_pages, page_size, max_pages)
    ref = None if x.get("pages", 1) is None else ctypes.byref(pages)
    if name == "append":
        r = None if rope is None else ctypes.byref(M.moa_rope_t(x["inv_freq"], *rope))
        return lib.moa_quant_append(handle, ref, x["q"], strides[0], x["k_new"], strides[1], x["v_new"], strides[2],
                                    x["q_out"], r, x["positions"], x["seq_start"], batch, n, None)
    if name == "prefill":
        return lib.moa_quant_prefill(handle, ref, x["q"], x["o"], x["positions"], x["seq_start"], batch, n,
                                     x["workspace"], ws_bytes, None)
    if name == "decode":
        return lib.moa_quant_decode(handle, ref, x["q"], x["o"], x["positions"], batch, x["workspace"], ws_bytes, None)
    return lib.moa_quant_decode_shared(handle, ref, x["prefix_table"], prefix_len, x["q"], x["o"], x["positions"], batch,
                                       x["workspace"], ws_bytes, None)


QUANT = ["append", "prefill", "decode", "shared"]
ATTENTION = QUANT[1:]


@pytest.mark.parametrize("name", QUANT + ["assign"])
@pytest.mark.parametrize("kw,status", [
    (dict(pages=None), BAD), (dict(table=None), BAD), (dict(positions=None), BAD), (dict(table=7 * A + 2), BAD),
    (dict(positions=8 * A + 1), BAD), (dict(num_pages=0), BAD), (dict(num_pages=(1 << 25) + 1), BAD),
    (dict(max_pages=0), BAD), (dict(max_pages=(1 << 24) + 1), BAD), (dict(page_size=8), UNSUP), (dict(page_size=48), UNSUP),
    (dict(page_size=512), UNSUP), (dict(page_size=0), UNSUP), (dict(batch=0, n=0), BAD), (dict(batch=65536, n=65536), BAD),
])
def test_refusals_of_every_call(name, kw, status):
    p = plan()
    assert call(name, p, **kw) == status
    assert lib.moa_last_error().decode().startswith("moa_paged_assign" if name == "assign" else "moa_quant_")
    assert call(name, None, **kw) == BAD


@pytest.mark.parametrize("name", QUANT)
@pytest.mark.parametrize("kw,status", [
    (dict(k_pages=None), BAD), (dict(v_pages=None), BAD), (dict(scales=None), BAD), (dict(scales=14 * A + 4), BAD),
    (dict(k_pages=5 * A + 8), BAD), (dict(v_pages=5 * A + 64), BAD), (dict(scales=5 * A + 256), BAD),
    (dict(scales=6 * A), BAD), (dict(q=None), BAD), (dict(q=A + 8), BAD),
])
def test_refusals_of_the_cache(name, kw, status):
    assert call(name, plan(), **kw) == status


@pytest.mark.parametrize("name", QUANT)
def test_fp32_plans_are_refused(name):
    assert call(name, plan(dtype="f32")) == UNSUP
    assert "bf16" in lib.moa_last_error().decode()


@pytest.mark.parametrize("kw,status", [
    (dict(k_new=None), BAD), (dict(q_out=None), BAD), (dict(q_out=14 * A), BAD), (dict(k_new=14 * A), BAD),
    (dict(positions=14 * A), BAD), (dict(table=14 * A + 64), BAD), (dict(rope=(8, 0)), UNSUP), (dict(rope=(64, 2)), BAD),
    (dict(strides=(1024, 255, 256)), BAD), (dict(seq_start=None, n=4), BAD), (dict(n=-1), BAD), (dict(n=1 << 30), BAD),
])
def test_refusals_of_append(kw, status):
    assert call("append", plan(), **kw) == status


@pytest.mark.parametrize("name", ATTENTION)
@pytest.mark.parametrize("kw,status", [
    (dict(o=None), BAD), (dict(o=14 * A), BAD), (dict(workspace=14 * A), BAD), (dict(o=5 * A), BAD),
    (dict(workspace=None), WS), (dict(workspace=12 * A + 128), WS), (dict(o=12 * A), BAD),
])
def test_refusals_of_attention(name, kw, status):
    p = plan()
    assert call(name, p, **kw) == status
    assert call(name, p, ws_bytes=lib.moa_paged_workspace_bytes(p.handle, 3, 3) - 1) == WS


def test_refusals_of_one_call_each():
    p = plan()
    assert call("prefill", p, seq_start=None) == BAD
    assert call("shared", p, prefix_table=None) == BAD
    assert call("shared", p, prefix_len=20 * 64 + 1) == BAD
    assert call("shared", p, prefix_len=-1) == BAD


@pytest.mark.parametrize("kw,status", [
    (dict(free_pages=None), BAD), (dict(counts=None), BAD), (dict(free_pages=15 * A + 2), BAD), (dict(counts=16 * A + 1), BAD),
    (dict(fresh=17 * A + 2), BAD), (dict(slots=18 * A + 2), BAD), (dict(seq_start=9 * A + 2), BAD),
    (dict(seq_start=None, n=4), BAD), (dict(n=-1), BAD), (dict(n=1 << 30), BAD),
    (dict(workspace=None), WS), (dict(workspace=12 * A + 128), WS), (dict(ws_bytes=100), WS),
    (dict(free_pages=7 * A), BAD), (dict(counts=7 * A + 4), BAD), (dict(slots=15 * A), BAD), (dict(positions=7 * A), BAD),
    (dict(seq_start=18 * A), BAD), (dict(fresh=16 * A), BAD), (dict(workspace=7 * A), BAD), (dict(counts=12 * A), BAD),
])
def test_refusals_of_assign(kw, status):
    assert call("assign", plan(), **kw) == status


def test_no_tokens_are_nothing_to_do():
    none = dict(q=None, k_new=None, v_new=None, q_out=None, o=None)
    assert call("append", plan(), n=0, **none) == M.MOA_OK
    assert call("prefill", plan(), n=0, workspace=None, ws_bytes=0, **none) == M.MOA_OK


def test_more_tokens_than_one_launch_takes_are_refused():
    many = 1 << 29
    assert call("append", plan(), n=many) == UNSUP and "too much" in lib.moa_last_error().decode()
    assert call("assign", plan(), n=many) == UNSUP and "too much" in lib.moa_last_error().decode()
