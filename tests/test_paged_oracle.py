"""The paged oracle against the dense one, and rotation against complex numbers."""
import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("block", [0, 64])
@pytest.mark.parametrize("page", [16, 64])
def test_paged_attention_equals_dense_attention(page, block):
    rng = np.random.default_rng(page + block)
    b, n, hq, hkv, d, s, windows = 2, 150, 4, 2, 8, 5, [20, 90]
    q, k, v = rng.normal(size=(b, n, hq, d)), rng.normal(size=(b, n, hkv, d)), rng.normal(size=(b, n, hkv, d))
    width = -(-n // page)
    order = rng.permutation(b * hkv * width)
    table = order.reshape(b, hkv, width).astype(np.int32)
    kp, vp = np.zeros((2, len(order), page, d))
    for i in range(b):
        for g in range(hkv):
            for j in range(n):
                kp[table[i, g, j // page], j % page] = k[i, j, g]
                vp[table[i, g, j // page], j % page] = v[i, j, g]
    dense = oracle.attention_ref(q, k, v, windows, s, block=block)
    got, a, _ = oracle.paged_attention_ref(q.reshape(-1, hq, d), kp, vp, table, [0, 0], [0, n, 2 * n], windows, s,
                                           block=block)
    assert np.allclose(got.reshape(q.shape), dense, rtol=1e-12, atol=1e-12)
    assert (a.reshape(q.shape) >= np.abs(dense) - 1e-12).all()
    if not block:                                    # the last token, as a decode call
        got, _, _ = oracle.paged_attention_ref(q[:, -1], kp, vp, table, [n - 1, -1], None, windows, s)
        assert np.allclose(got[0], dense[0, -1], atol=1e-12) and np.isnan(got[1]).all()
        # keys in front of 77 through one table for all: sequence 0's
        got, _, _ = oracle.paged_attention_ref(q[:, -1], kp, vp, table, [n - 1, n - 1], None, windows, s,
                                               prefix_table=table[0], prefix_len=77)
        mixed = [np.concatenate([x[:1, :77], x[1:, 77:]], 1) for x in (k, v)]
        other = oracle.decode_ref(q[1:, -1], *mixed, windows, s)
        assert np.allclose(got[0], dense[0, -1], atol=1e-12) and np.allclose(got[1], other[0], atol=1e-12)


def test_a_row_without_keys_is_zero_and_absent_pages_are_not_seen():
    kp = np.ones((2, 16, 4))
    table = np.array([[[0, -1, 1]]], dtype=np.int32)
    q = np.ones((1, 1, 4))
    vp = np.arange(2 * 16 * 4, dtype=float).reshape(2, 16, 4)
    o, _, _ = oracle.paged_attention_ref(q, kp, vp, table, [20], None, [8], 0)      # keys 13 .. 20: three are left
    assert np.allclose(o[0, 0], vp[0, 13:].mean(0))
    o, _, _ = oracle.paged_attention_ref(q, kp, vp, table, [28], None, [8], 0)
    assert (o == 0).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, pos, f = rng.normal(size=(3, 2, 12)), [0, 7, 100000], 10.0 ** -np.arange(4.0)
    got = oracle.rotate_ref(x, pos, f, interleaved)
    z = x[..., 0:8:2] + 1j * x[..., 1:8:2] if interleaved else x[..., :4] + 1j * x[..., 4:8]
    z = z * np.exp(1j * np.array(pos)[:, None, None] * f)
    y = got[..., 0:8:2] + 1j * got[..., 1:8:2] if interleaved else got[..., :4] + 1j * got[..., 4:8]
    assert np.allclose(y, z, atol=1e-9) and (got[..., 8:] == x[..., 8:]).all() and (got[0] == x[0]).all()
