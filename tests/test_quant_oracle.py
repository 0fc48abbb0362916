"""Pins of the 8-bit oracle that share none of its code: torch's own e4m3 type, worked examples, and
the page tables of a small step followed by hand."""
import math

import numpy as np
import pytest
import torch

from oracle import quant_oracle as Q


def test_values_are_those_of_the_type():
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).double().numpy(), Q.e4m3_values(), equal_nan=True)


def test_encoding_is_the_nearest_number():
    rng = np.random.default_rng(0)
    v = Q.e4m3_values()[:127]
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(size=4000) * 0.01, (v[1:] + v[:-1]) / 2, v, -v])
    x = torch.from_numpy(x).float()
    assert np.array_equal(Q.encode_ref(x.double().numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert list(Q.encode_ref([449.0, -1e300, math.inf, math.nan])) == [0x7E, 0xFE, 0x7F, 0x7F]


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0001, 1), (224.0, -1), (1.75, -8), (1.76, -7), (0.0, -117),
                                    (2.0 ** -140, -117), (448 * 2.0 ** 119, 119), (3.3e38, 119)])
def test_scales(amax, e):
    assert Q.exponent_ref(amax) == e


def test_a_block_that_grows_takes_its_rows_along():
    codes, scales = np.zeros((32, 2), dtype=np.uint8), np.zeros(2)
    Q.store_ref(codes, scales, [[1.75, -0.5]], [16])
    assert scales[1] == 2.0 ** -8 and list(codes[16]) == [0x7E, 0xF0]       # 448 and -128
    Q.store_ref(codes, scales, [[3.5, 0.0]], [17])
    assert scales[1] == 2.0 ** -7 and list(codes[16]) == [0x76, 0xE8] and list(codes[17]) == [0x7E, 0]
    Q.store_ref(codes, scales, [[0.001, 0.0]], [18])                        # a smaller one leaves it
    assert scales[1] == 2.0 ** -7
    Q.store_ref(codes, scales, [[0.0, 0.875]], [16])                        # the first position begins anew
    assert scales[1] == 2.0 ** -9 and list(codes[16]) == [0, 0x7E] and scales[0] == 0


def test_tables_followed_by_hand():
    # pages of 16, one head, window 20, 4 sinks.  Sequence 0 goes from position 48 on: sees from 29 on,
    # so that entry 1 (16 .. 31) stays; sequence 1 from 64: sees from 45 on, entry 1 goes back; sequence 2 ended.
    table = [[[0, 1, 2, -1, -1]], [[3, 4, 5, 6, -1]], [[7, 99, -1, 8, -1]]]
    t, free, counts, slots = Q.assign_ref(table, [9, 10, 11, 12] + [0] * 9, [4, 0], 16, [48, 64, -1], None, [0, 0, 1], 3,
                                          [20], 4, False)
    # given back 4, 7, 8; taken 8 (sequence 0), 7 (sequence 1)
    assert t.tolist() == [[[0, 1, 2, 8, -1]], [[3, -1, 5, 6, 7]], [[-1, 99, -1, -1, -1]]]
    assert free[:7].tolist() == [9, 10, 11, 12, 4, 7, 8] and counts.tolist() == [5, 0]
    assert slots == {(0, 0): 128, (1, 0): 112}
