"""Argument checks of the paged entry points: they return before anything is launched,
so they run without a GPU.  Addresses here are numbers that nothing reads."""
import ctypes

import pytest

from paper_2406_14909_amd import moa as M

lib = M.load_library()
A = 1 << 40                                          # distinct regions of 1 TiB
BASE = dict(q=1 * A, k_new=2 * A, v_new=3 * A, q_out=4 * A, k_pages=5 * A, v_pages=6 * A, table=7 * A, positions=8 * A,
            seq_start=9 * A, inv_freq=10 * A, o=11 * A, workspace=12 * A, prefix_table=13 * A)


def plan(hq=8, hkv=2, d=128, dtype="bf16"):
    return M.moa_plan(hq, hkv, d, 4, 1000, dtype, [100.0] * hkv, [0.0] * hkv)


def call(name, p, batch=3, n=3, num_pages=100, page_size=64, max_pages=20, strides=(1024, 256, 256), rope=(64, 0),
         ws_bytes=None, prefix_len=100, **over):
    x = dict(BASE, **over)
    pages = M.moa_pages_t(x["k_pages"], x["v_pages"], x["table"], num_pages, page_size, max_pages)
    if x.get("pages", 1) is None:
        pages = None
    handle = None if p is None else p.handle
    ref = None if pages is None else ctypes.byref(pages)
    if ws_bytes is None:
        ws_bytes = 0 if p is None else lib.moa_paged_workspace_bytes(handle, batch, n)
    if name == "append":
        r = None if rope is None else ctypes.byref(M.moa_rope_t(x["inv_freq"], *rope))
        return lib.moa_paged_append(handle, ref, x["q"], strides[0], x["k_new"], strides[1], x["v_new"], strides[2],
                                    x["q_out"], r, x["positions"], x["seq_start"], batch, n, None)
    if name == "prefill":
        return lib.moa_paged_prefill(handle, ref, x["q"], x["o"], x["positions"], x["seq_start"], batch, n,
                                     x["workspace"], ws_bytes, None)
    if name == "decode":
        return lib.moa_paged_decode(handle, ref, x["q"], x["o"], x["positions"], batch, x["workspace"], ws_bytes, None)
    return lib.moa_paged_decode_shared(handle, ref, x["prefix_table"], prefix_len, x["q"], x["o"], x["positions"], batch,
                                       x["workspace"], ws_bytes, None)


ALL = ["append", "prefill", "decode", "shared"]
ATTENTION = ALL[1:]
BAD, UNSUP, WS = M.MOA_ERR_INVALID_ARG, M.MOA_ERR_UNSUPPORTED, M.MOA_ERR_WORKSPACE


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("kw,status", [
    (dict(k_pages=None), BAD), (dict(v_pages=None), BAD), (dict(table=None), BAD), (dict(positions=None), BAD),
    (dict(pages=None), BAD), (dict(q=None), BAD), (dict(q=A + 8), BAD),
    (dict(k_pages=5 * A + 8), BAD), (dict(v_pages=6 * A + 2), BAD), (dict(table=7 * A + 2), BAD),
    (dict(positions=8 * A + 1), BAD),
    (dict(num_pages=0), BAD), (dict(num_pages=-1), BAD), (dict(num_pages=(1 << 25) + 1), BAD),
    (dict(max_pages=0), BAD), (dict(max_pages=(1 << 24) + 1), BAD),
    (dict(page_size=8), UNSUP), (dict(page_size=48), UNSUP), (dict(page_size=512), UNSUP), (dict(page_size=0), UNSUP),
    (dict(page_size=-16), UNSUP),
    (dict(batch=0, n=0), BAD), (dict(batch=65536, n=65536), BAD),
    (dict(v_pages=5 * A + 64), BAD),                 # the pools overlap
])
def test_refusals_of_every_call(name, kw, status):
    p = plan()
    assert call(name, p, **kw) == status
    assert lib.moa_last_error().decode().startswith("moa_paged_")


@pytest.mark.parametrize("name", ALL)
def test_null_plan(name):
    assert call(name, None) == BAD


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), BAD), (dict(n=0, seq_start=None), BAD), (dict(n=1 << 30), BAD), (dict(k_new=None), BAD), (dict(v_new=None), BAD), (dict(q_out=None), BAD),
    (dict(k_new=2 * A + 4), BAD), (dict(q_out=4 * A + 8), BAD), (dict(seq_start=9 * A + 2), BAD),
    (dict(seq_start=None, n=4), BAD),
    (dict(strides=(1016, 256, 256)), BAD), (dict(strides=(1024, 255, 256)), BAD), (dict(strides=(1024, 256, 260)), BAD),
    (dict(strides=(1024, 256, 1 << 41)), BAD), (dict(strides=(-1024, 256, 256)), BAD),
    (dict(inv_freq=None), BAD), (dict(inv_freq=10 * A + 2), BAD),
    (dict(rope=(0, 0)), UNSUP), (dict(rope=(8, 0)), UNSUP), (dict(rope=(144, 0)), UNSUP), (dict(rope=(-16, 0)), UNSUP),
    (dict(rope=(64, 2)), BAD),
    (dict(q_out=5 * A), BAD), (dict(k_new=5 * A + 64 * 100), BAD), (dict(table=6 * A), BAD), (dict(positions=5 * A), BAD),
    (dict(q=6 * A), BAD), (dict(inv_freq=5 * A), BAD), (dict(seq_start=6 * A + 64), BAD),
    (dict(q_out=2 * A), BAD), (dict(q_out=A + 256), BAD), (dict(q_out=A, strides=(1536, 256, 256)), BAD),
    (dict(q_out=9 * A), BAD),
])
def test_refusals_of_append(kw, status):
    assert call("append", plan(), **kw) == status


@pytest.mark.parametrize("name", ATTENTION)
@pytest.mark.parametrize("kw,status", [
    (dict(o=None), BAD), (dict(o=11 * A + 8), BAD), (dict(workspace=None), WS), (dict(workspace=12 * A + 128), WS),
    (dict(o=A), BAD), (dict(o=5 * A + 256), BAD), (dict(o=6 * A), BAD), (dict(o=7 * A), BAD), (dict(o=8 * A), BAD),
    (dict(o=12 * A), BAD), (dict(workspace=A), BAD), (dict(workspace=5 * A), BAD), (dict(workspace=7 * A), BAD),
    (dict(workspace=8 * A), BAD),
])
def test_refusals_of_attention(name, kw, status):
    assert call(name, plan(), **kw) == status


@pytest.mark.parametrize("name", ATTENTION)
def test_a_small_workspace_is_refused(name):
    p = plan()
    assert call(name, p, ws_bytes=lib.moa_paged_workspace_bytes(p.handle, 3, 3) - 1) == WS


def test_refusals_of_one_call_each():
    p = plan()
    assert call("prefill", p, seq_start=None) == BAD
    assert call("prefill", p, seq_start=9 * A + 1) == BAD
    assert call("prefill", p, n=-1) == BAD
    assert call("prefill", p, n=0, seq_start=None) == BAD
    assert call("prefill", p, o=9 * A) == BAD
    assert call("prefill", p, workspace=9 * A) == BAD
    assert call("shared", p, prefix_table=None) == BAD
    assert call("shared", p, prefix_table=13 * A + 2) == BAD
    assert call("shared", p, prefix_len=-1) == BAD
    assert call("shared", p, prefix_len=20 * 64 + 1) == BAD
    assert call("shared", p, o=13 * A) == BAD
    assert call("shared", p, workspace=13 * A) == BAD


def test_workspace_bytes():
    p = plan()
    assert lib.moa_paged_workspace_bytes(None, 3, 3) == 0
    assert lib.moa_paged_workspace_bytes(p.handle, 0, 3) == 0
    assert lib.moa_paged_workspace_bytes(p.handle, 3, 0) == 0
    sizes = [lib.moa_paged_workspace_bytes(p.handle, b, n) for b, n in ((1, 1), (8, 8), (8, 1000), (65535, 65535))]
    assert sizes == sorted(sizes) and sizes[0] >= 1


def test_no_tokens_are_nothing_to_do():
    none = dict(q=None, k_new=None, v_new=None, q_out=None, o=None)
    assert call("append", plan(), n=0, **none) == M.MOA_OK
    assert call("prefill", plan(), n=0, workspace=None, ws_bytes=0, **none) == M.MOA_OK
