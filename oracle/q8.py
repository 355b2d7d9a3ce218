"""The 8-bit cache in fp64 (oracle).

TEST INFRASTRUCTURE ONLY -- see the package header.

Definition
----------
* A block is 32 consecutive tokens of one (sequence, KV head), 128 channels.
  Its scale is s = fl32(max |x| / Q), Q = 127 (int8) or 448 (e4m3); a code is
  the type's value nearest to the exact quotient x / s, ties to even; the value
  is s times the code.  A block whose largest magnitude is below 2^-96 is zeros
  with scale 0; infinities and NaN count as zeros.
* The 4096 codes of a block are stored in the order `key_order` / `value_order`
  give (16-byte pieces, 16 channels of one token for keys; two channels of
  eight tokens for values).
* Attention: softmax over the visible tokens of softmax_scale q . k, output
  sum a v; query head i reads KV head i // G.  With a window w, token t of a
  sequence of T cached and e further tokens is visible if t < sinks or
  t >= T + e - w.
* Scores: a block's weight in a step is the sum of a over its tokens and the
  query heads of its KV head.
* Eviction: whole blocks, the partly filled newest one counted as one; the first
  and the newest ones stay, the others are ranked by score, ties to the lower
  index, NaN lowest.
"""

from __future__ import annotations

import math

import numpy as np

BLOCK = 32
D = 128
QMAX = {"int8": 127.0, "e4m3": 448.0}


def key_order():
    """byte position of (t, c) in a block of keys, [32, 128]."""
    t, c = np.meshgrid(np.arange(BLOCK), np.arange(D), indexing="ij")
    return (((t // 16) * 2 + c // 64) * 64 + ((c // 16) % 4) * 16 + t % 16) * 16 + c % 16


def value_order():
    """byte position of (t, c) in a block of values, [32, 128]."""
    t, c = np.meshgrid(np.arange(BLOCK), np.arange(D), indexing="ij")
    return ((c // 32 * 4 + (t // 4) % 4) * 16 + c % 16) * 16 + ((c // 16) % 2) * 8 + (t // 16) * 4 + t % 4


def e4m3_values():
    """The value of each of the 256 patterns (NaN for the two that are none)."""
    out = np.zeros(256)
    for i in range(256):
        e, m = (i >> 3) & 15, i & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if e == 15 and m == 7:
            v = math.nan
        out[i] = -v if i & 128 else v
    return out


def quantize(x, fmt):
    """x fp64 [..., T, 128] (T any) -> (code patterns uint8 [..., nb, 32, 128],
    scales fp32 [..., nb]); the rows behind T are zeros."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isfinite(x), x, 0.0)
    T = x.shape[-2]
    nb = (T + BLOCK - 1) // BLOCK
    y = np.zeros((*x.shape[:-2], nb * BLOCK, D))
    y[..., :T, :] = x
    y = y.reshape(*x.shape[:-2], nb, BLOCK, D)
    top = np.abs(y).max(axis=(-2, -1))
    s = np.where(top >= 2.0 ** -96, (top / QMAX[fmt]).astype(np.float32), np.float32(0.0)).astype(np.float32)
    # fp64 quotients decide exactly: x has 8 significant bits and s 24, so a
    # quotient that is not a border lies 2^-33 of it away from any
    q = y / np.where(s > 0, s, 1.0).astype(np.float64)[..., None, None]
    q = np.where((s > 0)[..., None, None], q, 0.0)
    if fmt == "int8":
        return np.rint(q).astype(np.int8).view(np.uint8), s
    grid = e4m3_values()[:127]
    a = np.abs(q)
    i = np.clip(np.searchsorted(grid, a), 1, 126)
    lo, hi = grid[i - 1], grid[i]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 0))
    p = np.where(up, i, i - 1).astype(np.uint8)
    return p | (np.signbit(q).astype(np.uint8) << 7), s


def values(codes, s, fmt):
    """fp64 values [..., nb * 32, 128]."""
    c = codes.view(np.int8).astype(np.float64) if fmt == "int8" else e4m3_values()[codes]
    v = c * s.astype(np.float64)[..., None, None]
    return v.reshape(*v.shape[:-3], -1, D)


def pack(codes, order):
    """[..., 32, 128] patterns -> [..., 4096] bytes."""
    out = np.zeros((*codes.shape[:-2], BLOCK * D), np.uint8)
    out[..., order.reshape(-1)] = codes.reshape(*codes.shape[:-2], -1)
    return out


def unpack(data, order):
    return data[..., order.reshape(-1)].reshape(*data.shape[:-1], BLOCK, D)


def visible(T, extra, window, sinks):
    t = np.arange(T)
    return np.ones(T, bool) if window <= 0 else (t < sinks) | (t >= T + extra - window)


def attention(q, k, v, lens, G, scale, window=0, sinks=0, extra_k=None, extra_v=None, extra_lens=None):
    """q [B, Hq, 128], k, v [B, H, T, 128] fp64; extra_*: raw tokens [B, H, R, 128]
    behind them, always visible.  Returns (out [B, Hq, 128], block weights
    [B, H, nb])."""
    B, Hq, _ = q.shape
    H = Hq // G
    nb = (k.shape[2] + BLOCK - 1) // BLOCK
    out = np.zeros((B, Hq, D))
    weight = np.zeros((B, H, nb))
    for b in range(B):
        T, e = int(lens[b]), 0 if extra_lens is None else int(extra_lens[b])
        see = visible(T, e, window, sinks)
        for i in range(Hq):
            h = i // G
            kk, vv = k[b, h, :T][see], v[b, h, :T][see]
            if e:
                kk = np.concatenate([kk, extra_k[b, h, :e]])
                vv = np.concatenate([vv, extra_v[b, h, :e]])
            if not len(kk):
                continue
            x = kk @ q[b, i] * scale
            a = np.exp(x - x.max())
            a /= a.sum()
            out[b, i] = a @ vv
            full = np.zeros(nb * BLOCK)
            full[:T][see] = a[:int(see.sum())]
            weight[b, h] += full.reshape(nb, BLOCK).sum(axis=1)
    return out, weight


def evict(scores, nb, keep, first, last):
    """Kept block indexes of one (sequence, head): scores [>= nb], all in blocks."""
    if nb <= keep:
        return list(range(nb))
    s = [-math.inf if math.isnan(x) else x for x in np.asarray(scores[:nb], np.float64)]
    nan = [math.isnan(x) for x in np.asarray(scores[:nb], np.float64)]
    inner = sorted(range(first, nb - last), key=lambda i: (nan[i], -s[i], i))[:keep - first - last]
    return sorted([*range(first), *inner, *range(nb - last, nb)])
