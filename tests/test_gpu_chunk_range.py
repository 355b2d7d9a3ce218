"""Attention of many queries where sizes are far apart: value blocks of unlike
scales that get next to no weight or are not seen.  Against the formula in 64
bits, within the bound that test_gpu_chunk.py derives: relative to sum a |v|, so
that a block without weight does not widen it."""

import numpy as np
import pytest
import torch

from test_gpu_chunk import DEV, FMTS, LOG2E, _check_all, _filled, _held, _i32, _kv, _q, dq  # noqa: F401

pytestmark = pytest.mark.gpu


def _low(k, q, blocks, down):
    """Keys and queries whose scores (base 2, softmax scale 128^-0.5) of the
    blocks' tokens are about `down` lower than without."""
    k, q = k.clone(), q.clone()
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    for j in blocks:
        k[:, 32 * j:32 * j + 32, :, 0] = -down / (8.0 * 128 ** -0.5 * LOG2E)
    return k, q


# ------------------------------------------------- value blocks of unlike scales

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,T,n,H,G", [(1, 200, 5, 1, 4), (1, 200, 150, 1, 2), (1, 4100, 6, 1, 2), (1, 4100, 150, 1, 1),
                                       (2, 500, 70, 8, 1)])
@pytest.mark.parametrize("up", [17, 24, 30, 60, 90])
def test_large_blocks_without_weight(dq, fmt, B, T, n, H, G, up):
    """Blocks 2^up as large as the others, with weights 2^-(up + 40) of theirs:
    first, last and between."""
    k, v = _kv(T + n, B, T, H)
    q = _q(up, B, n, H * G)
    last = (T - n) // 32 - 1
    for blocks in ([0], [1, last], [last // 2, last]):
        kk, qq = _low(k, q, blocks, up + 40)
        x = v.float()
        for j in blocks:
            x[:, 32 * j:32 * j + 32] *= 2.0 ** up
        x = x.to(torch.bfloat16)
        cache = _filled(dq, fmt, kk, x, H * G)
        out = cache.attend_chunk(qq.to(DEV), _i32([T] * B))
        _check_all(out, qq, _held(kk, fmt), _held(x, fmt), [T] * B, [n] * B)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n", [8, 300])
@pytest.mark.parametrize("window,sinks", [(20, 0), (64, 5), (40, 70)])
def test_large_blocks_outside_the_window(dq, fmt, n, window, sinks):
    """Blocks of sizes between 2^-45 and 2^45, of which a row sees two or three:
    what its tile's other rows see does not touch it."""
    T, H, G = 1000, 1, 2
    k, v = _kv(window + n, 1, T, H)
    q = _q(sinks, 1, n, H * G)
    g = np.random.default_rng(n)
    for order in (np.linspace(45, -45, 32), np.linspace(-45, 45, 32), g.uniform(-45, 45, 32)):
        x = (v.float() * torch.from_numpy(2.0 ** np.repeat(order, 32)[:T]).float()[None, :, None, None]).to(torch.bfloat16)
        cache = _filled(dq, fmt, k, x, H * G)
        out = cache.attend_chunk(q.to(DEV), _i32([T]), window=window, sinks=sinks)
        _check_all(out, q, _held(k, fmt), _held(x, fmt), [T], [n], window=window, sinks=sinks)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n", [30, 200])
@pytest.mark.parametrize("up", [18, 30, 80])
def test_a_large_value_of_a_hidden_token(dq, fmt, n, up):
    """One value of a block is 2^up as large as the others, which its scale rounds
    to zero: rows before it see only the zeros and the blocks before."""
    T, H, G = 512, 1, 2
    k, v = _kv(n, 1, T, H)
    q = _q(up, 1, n, H * G)
    x = v.float()
    for t in (T - n + 20, T - 1):
        x[:, t] *= 2.0 ** up
    x = x.to(torch.bfloat16)
    cache = _filled(dq, fmt, k, x, H * G)
    out = cache.attend_chunk(q.to(DEV), _i32([T]))
    _check_all(out, q, _held(k, fmt), _held(x, fmt), [T], [n])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n", [6, 200])
def test_a_large_block_between_even_ones(dq, fmt, n):
    """A block without weight that is larger, then blocks of the first ones' size
    for long: the sums before and after count alike."""
    T, H, G = 1024, 1, 2
    k, v = _kv(n, 1, T, H)
    q = _q(n, 1, n, H * G)
    for up in (1, 3, 12, 40, 95):
        kk, qq = _low(k, q, [9], up + 40)
        x = v.float()
        x[:, 288:320] *= 2.0 ** up
        x[:, 640:672] *= 2.0 ** -up
        x = x.to(torch.bfloat16)
        cache = _filled(dq, fmt, kk, x, H * G)
        out = cache.attend_chunk(qq.to(DEV), _i32([T]))
        _check_all(out, qq, _held(kk, fmt), _held(x, fmt), [T], [n])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n", [4, 40, 150])
@pytest.mark.parametrize("to", [2.0 ** -88, 2.0 ** -60, 2.0 ** 50, 2.0 ** 90, 2.0 ** 124])
def test_all_values_small_or_large(dq, fmt, n, to):
    """All of a cache's values near the ends of the range, whole and cut."""
    H, G = 1, 2
    for T in (300, 4100):
        k, v = _kv(T + n, 1, T, H)
        q = _q(n, 1, n, H * G)
        x = (v.float() * to).to(torch.bfloat16)
        assert bool(torch.isfinite(x.float()).all())
        cache = _filled(dq, fmt, k, x, H * G)
        out = cache.attend_chunk(q.to(DEV), _i32([T]))
        _check_all(out, q, _held(k, fmt), _held(x, fmt), [T], [n])
