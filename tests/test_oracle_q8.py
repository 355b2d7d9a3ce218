"""Pins of the 8-bit cache's oracle (CPU): the code grids against torch's own
8-bit types and brute force, the block orders, ties, windows and eviction."""

import math

import numpy as np
import pytest
import torch

from oracle import q8


def test_orders_are_permutations_in_pieces_of_one_lane():
    for order in (q8.key_order(), q8.value_order()):
        assert sorted(order.reshape(-1).tolist()) == list(range(4096))
    k, v = q8.key_order(), q8.value_order()
    # a 16-byte piece: 16 consecutive channels of one token; two channels 16 apart of 8 tokens
    for piece in range(256):
        t, c = np.nonzero(k // 16 == piece)
        assert len(set(t)) == 1 and sorted(c) == list(range(c[0], c[0] + 16)) and c[0] % 16 == 0
        t, c = np.nonzero(v // 16 == piece)
        assert len(set(c)) == 2 and max(c) - min(c) == 16
        assert len(set(t)) == 8 and len({(x // 4) % 4 for x in t}) == 1


def test_e4m3_values_are_torchs():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(got, q8.e4m3_values(), equal_nan=True)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_codes_are_nearest(fmt):
    rng = np.random.default_rng(1)
    x = torch.tensor(rng.normal(size=(3, 70, 128)) * 5).to(torch.bfloat16).double().numpy()
    codes, s = q8.quantize(x, fmt)
    assert codes.shape == (3, 3, 32, 128) and s.shape == (3, 3)
    got = q8.values(codes, s, fmt)
    assert np.all(got[:, 70:] == 0)
    grid = np.arange(-127, 128.0) if fmt == "int8" else np.unique(q8.e4m3_values()[np.isfinite(q8.e4m3_values())])
    for b in range(3):
        sel = rng.choice(70 * 128, 400, replace=False)
        for i in sel:
            t, c = divmod(int(i), 128)
            err = np.abs(grid * np.float64(s[b, t // 32]) - x[b, t, c])
            assert abs(got[b, t, c] - x[b, t, c]) <= err.min() * (1 + 1e-12)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_ties_to_even_and_extremes(fmt):
    x = np.zeros((32, 128))
    top = q8.QMAX[fmt]
    x[0, 0] = top                                # scale exactly 1
    x[0, 1:5] = [0.5, 1.5, 2.5, -0.5]
    codes, s = q8.quantize(x, fmt)
    assert s[0] == 1.0
    v = q8.values(codes, s, fmt)[0]
    assert v[0] == top
    if fmt == "int8":
        assert v[1:5].tolist() == [0.0, 2.0, 2.0, 0.0]
    else:
        assert v[1:5].tolist() == [0.5, 1.5, 2.5, -0.5]
        x[1, :4] = [17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10]   # between 16 and 18, 18 and 20, the smallest steps
        v = q8.values(*q8.quantize(x, fmt), fmt)[1]
        assert v[:4].tolist() == [16.0, 20.0, 0.0, 2.0 ** -8]
    z = np.full((32, 128), 2.0 ** -97)
    codes, s = q8.quantize(z, fmt)
    assert s[0] == 0 and not codes.any()
    z[3, 5], z[4, 6] = math.nan, math.inf
    z[0, 0] = 1.0
    codes, s = q8.quantize(z, fmt)
    assert s[0] == np.float32(1.0 / top) and not codes[0, 3, 5] and not codes[0, 4, 6]


def test_windows():
    assert q8.visible(10, 0, 0, 0).all()
    assert np.flatnonzero(q8.visible(10, 0, 3, 2)).tolist() == [0, 1, 7, 8, 9]
    assert np.flatnonzero(q8.visible(10, 2, 3, 0)).tolist() == [9]
    assert not q8.visible(10, 5, 3, 0).any()
    assert q8.visible(4, 0, 100, 0).all()


def test_attention_weights_and_empty_rows():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(2, 4, 128)), rng.normal(size=(2, 2, 70, 128)), rng.normal(size=(2, 2, 70, 128))
    out, w = q8.attention(q, k, v, [70, 0], 2, 0.1)
    assert np.allclose(w[0].sum(axis=1), 2) and not out[1].any() and not w[1].any()
    x = np.exp(k[0, 1] @ q[0, 3] * 0.1)
    assert np.allclose(out[0, 3], x @ v[0, 1] / x.sum())


def test_evict_order_ties_and_nan():
    s = [5, 1, 3, 3, 3, 0, math.nan, 9]
    assert q8.evict(s, 8, 8, 0, 1) == list(range(8))
    assert q8.evict(s, 8, 4, 0, 1) == [0, 2, 3, 7]
    assert q8.evict(s, 8, 3, 1, 2) == [0, 6, 7]
    assert q8.evict(s, 8, 7, 0, 1) == [0, 1, 2, 3, 4, 5, 7]
