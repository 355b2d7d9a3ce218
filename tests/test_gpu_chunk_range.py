"""Attention of many queries where sizes are far apart: value blocks of unlike
scales that get next to no weight or are not seen, values near the ends of the
range, scores with a large common part.  Against the formula in 64 bits, within
the bound that test_gpu_chunk.py derives: relative to sum a |v|, so that a block
without weight does not widen it, and with the scores' size X in it."""

import math

import numpy as np
import pytest
import torch

from test_gpu_chunk import (DEV, FMTS, LOG2E, _check, _check_all, _check_cross, _cross, _filled, _held, _i32, _kv,  # noqa: F401
                            _q, _visible, dq)

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
@pytest.mark.parametrize("B,T,n,H,G", [(1, 200, 5, 1, 4), (1, 200, 150, 1, 2), (1, 4100, 6, 1, 2), (1, 4100, 150, 1, 1),
                                       (2, 500, 70, 8, 1)])
@pytest.mark.parametrize("up,down", [(12, 10), (30, 28), (60, 63), (100, 90), (110, 112)])
def test_large_blocks_with_little_weight(dq, fmt, B, T, n, H, G, up, down):
    """Blocks 2^up as large as the others, with weights 2^-down of theirs: they make
    a good part of the output, or most of it."""
    k, v = _kv(T + n, B, T, H)
    q = _q(up, B, n, H * G)
    last = (T - n) // 32 - 1
    for blocks in ([0], [1, last], [last // 2, last]):
        kk, qq = _low(k, q, blocks, down)
        x = v.float()
        for j in blocks:
            x[:, 32 * j:32 * j + 32] *= 2.0 ** up
        x = x.to(torch.bfloat16)
        cache = _filled(dq, fmt, kk, x, H * G)
        out = cache.attend_chunk(qq.to(DEV), _i32([T] * B))
        _check_all(out, qq, _held(kk, fmt), _held(x, fmt), [T] * B, [n] * B)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("T,n", [(400, 6), (400, 150), (4100, 100)])
def test_zeros_with_most_of_the_weight(dq, fmt, T, n):
    """First blocks of zeros that get nearly all weight, then values: what their
    small weights leave is the output."""
    k, v = _kv(T + n, 1, T, 1)
    q = _q(n, 1, n, 2)
    for down in (5, 30, 100):
        kk, qq = _low(k, q, range(2, -(-T // 32)), down)
        x = v.clone()
        x[:, :64] = 0
        cache = _filled(dq, fmt, kk, x, 2)
        out = cache.attend_chunk(qq.to(DEV), _i32([T]))
        _check_all(out, qq, _held(kk, fmt), _held(x, fmt), [T], [n])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("T,n", [(600, 6), (600, 150), (4100, 100)])
@pytest.mark.parametrize("size", [0.0, 3000.0, 2.0 ** 14])
def test_zeros_between_values(dq, fmt, T, n, size):
    """Values, zeros that get nearly all weight, then values of the first ones' sizes
    and larger, with small and with large scores."""
    k, v = _kv(T + n, 1, T, 1)
    q = _q(n, 1, n, 2)
    unit = 128 ** -0.5 * LOG2E
    for down in (5, 30, 60):
        kk, qq = _low(k, q, [j for j in range(-(-T // 32)) if j not in (6, 7)], down)
        kk[..., 1], qq[..., 1] = 64.0, size / (64.0 * unit)
        x = v.float()
        x[:, 192:256] = 0
        x[:, 320:352] *= 2.0 ** 20
        x[:, 128:160] *= 2.0 ** 50
        x[:, 384:] *= 2.0 ** 55
        x = x.to(torch.bfloat16)
        cache = _filled(dq, fmt, kk, x, 2)
        out = cache.attend_chunk(qq.to(DEV), _i32([T]))
        _check_all(out, qq, _held(kk, fmt), _held(x, fmt), [T], [n])


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
@pytest.mark.parametrize("n", [8, 150])
@pytest.mark.parametrize("size,up", [(0, 30), (0, 100), (-50, 150), (-80, 200)])
def test_a_large_value_between_the_first_tokens_and_the_window(dq, fmt, n, size, up):
    """First tokens whose block's scale comes from one that no query sees, and rounds
    theirs to zero: the window's values are all there is."""
    T = 300
    k, v = _kv(n, 1, T, 1)
    q = _q(up, 1, n, 2)
    x = v.float() * 2.0 ** size
    x[:, 25] = v[:, 25].float() * 2.0 ** (size + up)
    x = x.to(torch.bfloat16)
    assert bool(torch.isfinite(x.float()).all())
    cache = _filled(dq, fmt, k, x, 2)
    out = cache.attend_chunk(q.to(DEV), _i32([T]), window=64, sinks=20)
    _check_all(out, q, _held(k, fmt), _held(x, fmt), [T], [n], window=64, sinks=20)


@pytest.mark.parametrize("fmt", FMTS)
def test_zeros_beside_a_large_block_of_little_weight(dq, fmt):
    """A large block, blocks 2^-110 of it, then zeros with nearly all weight whose
    scale, from a value that is not seen, is as large: the first block's values are the
    output, after their sums were scaled by 2^110 and back."""
    T, n = 256, 30
    k, v = _kv(n, 1, T, 1)
    q = _q(n, 1, n, 4)
    kk, qq = _low(k, q, [0], 17)
    more, _ = _low(k, q, range(1, 7), 24)
    kk[:, 32:224] = more[:, 32:224]
    x = v.float() * 2.0 ** -55
    x[:, :32] *= 2.0 ** 110
    x[:, 255] *= 2.0 ** 110
    x = x.to(torch.bfloat16)
    cache = _filled(dq, fmt, kk, x, 4)
    out = cache.attend_chunk(qq.to(DEV), _i32([T]))
    _check_all(out, qq, _held(kk, fmt), _held(x, fmt), [T], [n])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("T,n", [(250, 6), (250, 150), (4100, 100)])
def test_small_values_of_little_weight(dq, fmt, T, n):
    """Outputs near the end of the type's range: values of 2^-85 with weights of 2^-38,
    beside zeros."""
    k, v = _kv(T + n, 1, T, 1)
    q = _q(n, 1, n, 2)
    kk, qq = _low(k, q, [j for j in range(-(-T // 32)) if j != 1], 38)
    x = v.float() * 2.0 ** -85
    x[:, 32:64] = 0
    x = x.to(torch.bfloat16)
    cache = _filled(dq, fmt, kk, x, 2)
    out = cache.attend_chunk(qq.to(DEV), _i32([T]))
    _check_all(out, qq, _held(kk, fmt), _held(x, fmt), [T], [n])


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
@pytest.mark.parametrize("B,T,H,n", [(1, 256, 2, 130), (64, 1024, 8, 5)])
@pytest.mark.parametrize("down", [0, 150])
def test_sizes_that_fall_step_by_step(dq, fmt, B, T, H, n, down):
    """Blocks that one wavefront takes one after another, of sizes from 2^60 down to
    2^-60 and up again, with equal weights or with so little of the first ones' that
    the small ones make up the output.  (All sequences share keys and values.)"""
    k, v = _kv(n, 1, T, H)
    q = _q(n, B, n, H)
    blocks = T // 32
    fall = np.linspace(60, -60, blocks)
    for order in (fall, fall[::-1], np.concatenate([fall[::2], fall[1::2][::-1]])):
        kk, qq = _low(k, q, [j for j in range(blocks) if order[j] > 0], down) if down else (k, q)
        x = (v.float() * torch.from_numpy(2.0 ** np.repeat(order, 32)).float()[None, :, None, None]).to(torch.bfloat16)
        cache = dq.Q8KVCache(B, H, H, T, fmt)
        cache.append(*(y.to(DEV).expand(B, -1, -1, -1) for y in (kk, x)), 0)
        out = cache.attend_chunk(qq.to(DEV), _i32([T] * B))
        some = [0, B - 1]
        held = [_held(y, fmt).expand(2, -1, -1, -1) for y in (kk, x)]
        _check_all(out[some], qq[some], *held, [T] * 2, [n] * 2)


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


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("T,n,window", [(300, 200, 0), (200, 8, 36), (200, 40, 36), (4100, 200, 3950), (4100, 200, 3800)])
def test_a_value_scale_that_is_no_number(dq, fmt, T, n, window):
    """NaN for the queries that see the block, as the decode step gives; the others
    are as they were."""
    k, v = _kv(n, 1, T, 1)
    q = _q(n, 1, n, 2)
    see = _visible(T, n, n, True, window, 0)
    sees = see[:, 128:160].any(dim=1)
    rest = (~sees).nonzero()[:, 0]
    assert bool(sees.any()) and (window == 3950 or rest.numel() > 0)
    for what in (math.nan, math.inf):
        cache = _filled(dq, fmt, k, v, 2)
        cache.v_scales[:, :, 4] = what
        out = cache.attend_chunk(q.to(DEV), _i32([T]), window=window)[0]
        assert bool(torch.isnan(out[sees]).all())
        if rest.numel():
            _check(out[rest], q[0, rest.cpu()], _held(k, fmt)[0, :, :T], _held(v, fmt)[0, :, :T], see[rest], 128 ** -0.5, 11)


# ----------------------------------------------------------------- large scores

def _common(seed, T, n, H, G, size, rise, mixed=False):
    """Scores (base 2, softmax scale 128^-0.5) of about `size`, of every row the same
    to a few units; `rise`: how much higher the last token's are than the first's, evenly.
    mixed: every other row's are without the common part, every fourth's negative."""
    k, v = _kv(seed, 1, T, H)
    q = _q(seed, 1, n, H * G)
    unit = 128 ** -0.5 * LOG2E
    k[..., 0], k[..., 1] = 64.0, (torch.arange(T)[:, None] * (60.0 / T)).to(torch.bfloat16)
    part = torch.full((n, 1), size / (64.0 * unit))
    if mixed:
        part[1::2] = 0.0
        part[2::4] *= -1.0
    q[..., 0], q[..., 1] = part.to(torch.bfloat16), rise / (60.0 * unit)
    return k, v, q


SCORES = [(2.0 ** 11, 0), (-2.0 ** 11, 20), (2.0 ** 12, 40), (2.0 ** 13, -40), (-2.0 ** 13, 3), (2.0 ** 14, 300), (1500, 900)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("T,n,G", [(300, 6, 2), (300, 150, 1), (4100, 5, 4), (4100, 200, 1)])
@pytest.mark.parametrize("size,rise", SCORES)
def test_large_scores(dq, fmt, T, n, G, size, rise):
    for mixed in (False, True):
        k, v, q = _common(T + n, T, n, 1, G, size, rise, mixed)
        cache = _filled(dq, fmt, k, v, G)
        out = cache.attend_chunk(q.to(DEV), _i32([T]))
        _check_all(out, q, _held(k, fmt), _held(v, fmt), [T], [n])


@pytest.mark.parametrize("T,n,G", [(300, 6, 2), (300, 150, 1), (4100, 5, 4), (4100, 200, 1)])
@pytest.mark.parametrize("size,rise", SCORES)
def test_large_cross_scores(dq, T, n, G, size, rise):
    for mixed in (False, True):
        k, v, q = _common(T + n, T, n, 1, G, size, rise, mixed)
        _check_cross(_cross(dq, q, k, v), q, k, v, [T], [n])


def _steps(out, q, k, v, see, scale):
    """out [n, 128] of a softmax so steep that it takes the largest score's value:
    rows whose second score (base 2) lies 64 and the two scores' errors further down.
    Every value of theirs is rounded once, 2^-8, the rest adds 2^-60 and the
    quotient's few roundings of 2^-24."""
    q = q.double().to(DEV)
    s = torch.where(see, q @ k.T * (scale * LOG2E), -math.inf)
    X = (q.abs() @ k.abs().T).amax(dim=1) * scale * LOG2E
    best = s.topk(2, dim=1)
    alone = best.values[:, 0] - best.values[:, 1] > 64 + 2 * 14 * 2.0 ** -24 * X
    want = v[best.indices[:, 0]]
    err = (out.double() - want).abs() / want.abs().amax(dim=1, keepdim=True)
    assert int(alone.sum()) >= q.shape[0] // 2
    assert float(err[alone].max()) <= 2.0 ** -8 + 2.0 ** -20


@pytest.mark.parametrize("scale", [1e3, 1e4, 1e6, 1e30])
@pytest.mark.parametrize("T,n", [(1500, 5), (1500, 150), (5000, 40)])
def test_steep_softmax(dq, scale, T, n):
    k, v = _kv(2, 1, T, 1)
    q = _q(2, 1, n, 1)
    see = _visible(T, n, n, True, 0, 0)
    for fmt in FMTS:
        cache = _filled(dq, fmt, k, v, 1)
        out = cache.attend_chunk(q.to(DEV), _i32([T]), softmax_scale=scale)
        _steps(out[0, :, 0], q[0, :, 0], _held(k, fmt)[0, 0, :T], _held(v, fmt)[0, 0, :T], see, scale)
    out = _cross(dq, q, k, v, scale=scale)
    _steps(out[0, :, 0], q[0, :, 0], *(x[0, :, 0].double().to(DEV) for x in (k, v)), torch.ones_like(see), scale)


@pytest.mark.parametrize("scale", [3.4e38, -3.4e38])
@pytest.mark.parametrize("T,n", [(300, 6), (300, 150), (4100, 5)])
def test_the_largest_softmax_scales(dq, scale, T, n):
    """Scores of 0 stay 0, whatever scale is allowed: the mean of the values."""
    k, v = _kv(n, 1, T, 1)
    q = torch.zeros_like(_q(n, 1, n, 2))
    for fmt in FMTS:
        out = _filled(dq, fmt, k, v, 2).attend_chunk(q.to(DEV), _i32([T]), softmax_scale=scale)
        _check_all(out, q, _held(k, fmt), _held(v, fmt), [T], [n], scale=scale)
    _check_cross(_cross(dq, q, k, v, scale=scale), q, k, v, [T], [n], scale=scale)


# -------------------------------------------- bits of the cross attention's weights

@pytest.mark.parametrize("B,T,n,H,G", [(3, 100, 1, 2, 1), (2, 1500, 1, 2, 1), (1, 700, 8, 2, 8), (1, 5000, 2, 1, 3),
                                       (2, 40, 33, 1, 1)])
@pytest.mark.parametrize("spread", [0.05, 0.3])
def test_few_cross_rows_keep_the_weights(dq, B, T, n, H, G, spread):
    """Up to 64 rows: an output is the formula's, rounded once, but for what fp32 and
    weights of two bf16 terms (2^-16) leave of sum a |v|, channel by channel: the
    errors of the scores as in test_gpu_chunk.py and 2^-18 for the sums (1500
    weights and products of one sign each, in parts of at most 2^6 blocks)."""
    k, v = _kv(T, B, T, H)
    q = (_q(n, B, n, H * G).float() * spread).to(torch.bfloat16)
    mask = torch.rand((B, T), generator=torch.Generator().manual_seed(T)) < 0.8
    for m in (None, mask):
        out = _cross(dq, q, k, v, None, m).double()
        for b in range(B):
            for i in range(H * G):
                kk, vv = (y[b, :, i // G].double().to(DEV) for y in (k, v))
                x = q[b, :, i].double().to(DEV)
                s = (x @ kk.T) * 128 ** -0.5
                if m is not None:
                    s[:, ~m[b].to(DEV)] = -math.inf
                a = torch.softmax(s, dim=1)
                ref, size = a @ vv, a @ vv.abs()
                X = float((x.abs() @ kk.abs().T).max()) * 128 ** -0.5 * LOG2E
                tol = 2.0 ** -8 * ref.abs() + (2.0 ** -16 + 2 * math.log(2) * 14 * 2.0 ** -24 * X + 2.0 ** -18) * size
                assert bool(((out[b, :, i] - ref).abs() <= tol).all()), (b, i)
