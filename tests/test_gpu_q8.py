"""The 8-bit cache on the GPU against its fp64 oracle (oracle/q8.py): codes,
scales and values bit for bit, attention, block weights and eviction; odd
lengths, strides, windows, pages, empty rows, and the parts together.

Tolerance of the attention outputs, in the 2-norm of a row relative to the
reference's: a score (base 2) is a sum of 128 exact products in fp32, in four
matrix instructions of 32 terms each, and meets four rounded factors; with X
the largest |score| of partial sums that bound it (taken as the sum of |q k|),
its error is at most about (8 + 4) 2^-24 X, and a weight's relative error
ln 2 times that, doubled by the softmax's denominator.  Weights carry 22 bits
(2^-22) and the sums of the values a few roundings more (2^-21 covers them
up to the lengths used here).  `_tol` is that bound."""

import copy
import math

import numpy as np
import pytest
import torch

from oracle import q8

pytestmark = pytest.mark.gpu

DEV = "cuda"
FMTS = ["int8", "e4m3"]


@pytest.fixture(scope="module")
def dq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_19880_amd as mod
    return mod


def _kv(seed, B, T, H, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    k = torch.randn((B, T, H, 128), generator=g) * (0.5 + 1.5 * torch.rand((H, 128), generator=g)) * spread
    k = k + torch.randn((H, 128), generator=g)
    v = torch.randn((B, T, H, 128), generator=g) * spread
    return k.to(torch.bfloat16), v.to(torch.bfloat16)


def _f64(x):
    """[B, T, H, D] bf16 -> fp64 [B, H, T, D]."""
    return x.double().cpu().numpy().transpose(0, 2, 1, 3)


def _held(x, fmt):
    """The values the cache holds of x, fp64 [B, H, nb 32, 128]."""
    codes, s = q8.quantize(_f64(x), fmt)
    return q8.values(codes, s, fmt)


def _tol(q, k, scale):
    """The derived bound of one query head's output."""
    X = float(np.max(np.abs(k) @ np.abs(q))) * abs(scale) * 1.4427 if k.size else 0.0
    return 2 * math.log(2) * 12 * 2.0 ** -24 * X + 2.0 ** -21


def _check_out(got, ref, q, k, lens, G, scale):
    got = got.double().cpu().numpy()
    for b in range(got.shape[0]):
        for i in range(got.shape[1]):
            norm = np.linalg.norm(ref[b, i])
            err = np.linalg.norm(got[b, i] - ref[b, i])
            if norm == 0:
                assert err == 0, (b, i)
            else:
                assert err <= norm * _tol(q[b, i], k[b, i // G, :max(1, int(lens[b]))], scale), (b, i, err / norm)


# ------------------------------------------------------------ encode and read

def _check_bytes(cache, k, v, t0=0):
    n = (k.shape[1] + 31) // 32
    b0 = t0 // 32
    for x, data, scale, order in ((k, cache.k_data, cache.k_scales, q8.key_order()),
                                  (v, cache.v_data, cache.v_scales, q8.value_order())):
        codes, s = q8.quantize(_f64(x), cache.fmt)
        assert np.array_equal(scale[:, :, b0:b0 + n].cpu().numpy(), s)
        got = q8.unpack(data[:, :, b0:b0 + n].cpu().numpy(), order)
        bad = np.argwhere(got != codes)
        # a negative zero's pattern is the encoder's choice: its value is not
        same = q8.values(got, s, cache.fmt) == q8.values(codes, s, cache.fmt)
        assert same.all(), (len(bad), bad[:4])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,T,H", [(1, 1, 1), (2, 31, 3), (1, 32, 8), (3, 33, 2), (2, 200, 5), (1, 1024, 2)])
def test_encode_and_read(dq, fmt, B, T, H):
    k, v = _kv(T, B, T, H)
    cache = dq.Q8KVCache(B, H, H, 1024, fmt)
    cache.k_data.fill_(0x5A)
    cache.v_data.fill_(0x5A)
    cache.append(k.to(DEV), v.to(DEV), 0)
    torch.cuda.synchronize()
    _check_bytes(cache, k, v)
    n = (T + 31) // 32
    assert torch.all(cache.k_data[:, :, n:] == 0x5A) and torch.all(cache.v_data[:, :, n:] == 0x5A)
    assert torch.all(cache.k_scales[:, :, n:] == 0)
    gk, gv = cache.read(0, T)
    for got, x in ((gk, k), (gv, v)):
        codes, s = q8.quantize(_f64(x), fmt)
        c = codes.view(np.int8).astype(np.float32) if fmt == "int8" else q8.e4m3_values()[codes].astype(np.float32)
        want = torch.from_numpy((c * s[..., None, None]).reshape(B, H, -1, 128)[:, :, :T].transpose(0, 2, 1, 3).copy())
        assert torch.equal(got.float().cpu(), want.to(torch.bfloat16).float())
    if T > 64:
        part, _ = cache.read(32, T - 40)
        assert torch.equal(part, gk[:, 32:T - 8])
    assert int(cache.status.item()) == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_every_quotient_rounds_right(dq, fmt):
    """Blocks whose values sweep the bf16 patterns below their largest one, for
    many largest ones: quotients at, next to and between all borders."""
    pats = np.arange(0, 0x7F80, dtype=np.int64)
    blocks = []
    for top in [0x3F80, 0x3FFE, 0x3FFF, 0x4000, 0x42FE, 0x42FD, 0x43E0, 0x43DF, 0x40A5, 0x7F7F, 0x0F90, 0x0FFF, 0x2B31,
                0x6C47]:
        near = pats[(pats <= top) & (pats > top - 4090)]
        near = np.resize(near[::-1], 4096).copy()
        near[1::2] |= 0x8000
        blocks.append(near)
    n = len(blocks)
    bits = torch.from_numpy(np.stack(blocks).astype(np.uint16).view(np.int16)).view(torch.bfloat16)
    x = bits.reshape(1, n * 32, 1, 128).contiguous()
    cache = dq.Q8KVCache(1, 1, 1, 512, fmt)
    cache.append(x.to(DEV), x.flip(3).contiguous().to(DEV), 0)
    torch.cuda.synchronize()
    _check_bytes(cache, x, x.flip(3))


@pytest.mark.parametrize("fmt", FMTS)
def test_encode_odd_inputs(dq, fmt):
    """Zeros, tiny blocks, subnormals, infinities and NaN; the status flag."""
    k, v = _kv(3, 1, 160, 2)
    k[0, :32] = 0
    k[0, 32:64] = 2.0 ** -97
    k[0, 64:96, 0] = 2.0 ** -130
    v[0, :32] = -0.0
    v[0, 32:64] = 2.0 ** -96
    cache = dq.Q8KVCache(1, 2, 2, 256, fmt)
    cache.append(k.to(DEV), v.to(DEV), 0)
    assert int(cache.status.item()) == 0
    _check_bytes(cache, k, v)
    k[0, 5, 1, 7], k[0, 100, 0, 127], v[0, 159, 1, 0] = math.nan, math.inf, -math.inf
    v[0, 64:96] = math.nan
    cache.append(k.to(DEV), v.to(DEV), 0)
    assert int(cache.status.item()) == dq.DQ_STATUS_RANGE
    _check_bytes(cache, k, v)


@pytest.mark.parametrize("fmt", FMTS)
def test_encode_strides_and_offsets(dq, fmt):
    """Slices of a fused projection (rows off 16 bytes among them), a ring's
    transposed view, a batch that is broadcast; appends at offsets."""
    B, T, H = 2, 96, 2
    k, v = _kv(4, B, T, H)
    want = dq.Q8KVCache(B, H, H, 256, fmt)
    want.append(k.to(DEV), v.to(DEV), 0)
    for pad in (0, 1, 8):
        wide = torch.zeros((B, T, H, 2, 128 + pad), dtype=torch.bfloat16, device=DEV)
        wide[..., 0, pad:] = k.to(DEV)
        wide[..., 1, pad:] = v.to(DEV)
        got = dq.Q8KVCache(B, H, H, 256, fmt)
        for t0 in (0, 32):
            got.append(wide[:, t0:t0 + 64, :, 0, pad:], wide[:, t0:t0 + 64, :, 1, pad:], t0)
        for x, y in zip(want.arrays, got.arrays):
            assert torch.equal(x, y), pad
        out = torch.zeros_like(wide)
        dq.dq_q8_decode_kv(fmt, *got.arrays, 0, T, out[..., 0, pad:], out[..., 1, pad:])
        rk, rv = want.read(0, T)
        assert torch.equal(out[..., 0, pad:], rk) and torch.equal(out[..., 1, pad:], rv)
        assert not out[..., :pad].any()
    ring = k.to(DEV).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    got = dq.Q8KVCache(B, H, H, 256, fmt)
    got.append(ring, v[:1].to(DEV).expand(B, T, H, 128), 0)
    assert torch.equal(got.k_data, want.k_data) and torch.equal(got.v_data[1], got.v_data[0])
    assert torch.equal(got.v_data[0], want.v_data[0])
    got.append(k[:, :0].to(DEV), v[:, :0].to(DEV), 0)


# ------------------------------------------------------------------ attention

def _attend_case(dq, fmt, lens, G, H=2, t_cap=1024, window=0, sinks=0, scale=None, scores=False, spread=1.0, seed=7):
    B = len(lens)
    k, v = _kv(seed, B, t_cap, H, spread)
    q = torch.randn((B, H * G, 128), generator=torch.Generator().manual_seed(seed + 1)).to(torch.bfloat16)
    cache = dq.Q8KVCache(B, H, H * G, t_cap, fmt, scores=scores)
    cache.append(k.to(DEV), v.to(DEV), 0)
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = cache.attend(q.to(DEV), seq, softmax_scale=scale, window=window, sinks=sinks)
    torch.cuda.synchronize()
    qf, kf, vf = q.double().numpy(), _held(k, fmt), _held(v, fmt)
    s = 128 ** -0.5 if scale is None else scale
    ref, weight = q8.attention(qf, kf, vf, lens, G, s, window, sinks)
    _check_out(out, ref, qf, kf, lens, G, s)
    return cache, seq, q.to(DEV), out, weight


LENS = [1024, 0, 1, 31, 32, 33, 127, 128, 129, 1000]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("G", [1, 2, 3, 5, 8])
def test_attention_lengths_and_groups(dq, fmt, G):
    _attend_case(dq, fmt, LENS, G)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_attention_scales(dq, fmt, scale):
    _attend_case(dq, fmt, [700, 45], 4, scale=scale)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 0), (32, 4), (33, 40), (100, 128), (500, 600),
                                          (1024, 0), (5000, 7), (2 ** 31 - 1, 2 ** 31 - 1), (64, 1000)])
def test_attention_windows(dq, fmt, window, sinks):
    _attend_case(dq, fmt, LENS, 4, window=window, sinks=sinks)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 33)])
def test_attention_short_sequences(dq, fmt, window, sinks):
    """One launch each: a few short sequences, and many of a few blocks, with their weights."""
    for lens, t_cap in (([1, 256, 37, 0, 129], 256), ([(37 * b) % 385 for b in range(260)], 384)):
        cache, _, _, _, weight = _attend_case(dq, fmt, lens, 3, t_cap=t_cap, window=window, sinks=sinks, scores=True)
        # as in test_scores
        assert np.max(np.abs(cache.scores.double().cpu().numpy() - weight)) <= 3 * 3e-5


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_long_split(dq, fmt):
    """Chunks of many blocks, and the longest split (64 chunks)."""
    _attend_case(dq, fmt, [16384, 9999], 4, H=1, t_cap=16384)
    _attend_case(dq, fmt, [16384, 9999], 8, H=1, t_cap=16384, window=6000, sinks=100)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,t_cap", [(70, 2048), (130, 1024), (300, 640)])
def test_attention_many_sequences(dq, fmt, B, t_cap):
    """More sequences than a wavefront has lanes, of unlike and of like lengths
    (zero and one among them), in one call and as partials."""
    H, G = 1, 2
    k, v = _kv(19, 2, t_cap, H)
    of = torch.arange(B) % 2
    g = torch.Generator().manual_seed(B)
    q = torch.randn((B, H * G, 128), generator=g).to(torch.bfloat16)
    cache = dq.Q8KVCache(B, H, H * G, t_cap, fmt)
    cache.append(k[of].to(DEV), v[of].to(DEV), 0)
    qf, kf, vf = q.double().numpy(), _held(k, fmt)[of.numpy()], _held(v, fmt)[of.numpy()]
    unlike = torch.where(torch.rand(B, generator=g) < 0.8, torch.randint(0, 90, (B,), generator=g), t_cap - 3)
    unlike[:3] = torch.tensor([0, 1, t_cap])
    for lens in (unlike.tolist(), [t_cap - b % 5 for b in range(B)], [0] * B):
        seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
        ref, _ = q8.attention(qf, kf, vf, lens, G, 128 ** -0.5, 0, 0)
        out = torch.full((B, H * G, 128), math.nan, device=DEV)
        cache.attend(q.to(DEV), seq, out=out)
        _check_out(out, ref, qf, kf, lens, G, 128 ** -0.5)
        out.fill_(math.nan)
        cache.partial(q.to(DEV), seq)
        cache.merge(seq, out)
        _check_out(out, ref, qf, kf, lens, G, 128 ** -0.5)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("spread", [1e-20, 1e15])
def test_attention_sizes_of_scores(dq, fmt, spread):
    """Keys and values of any size: finite, and (where the scores are small) right."""
    if spread < 1:
        _attend_case(dq, fmt, [300, 64], 4, spread=spread)
        return
    k, v = _kv(9, 1, 256, 1, spread)
    q = (torch.randn((1, 4, 128), generator=torch.Generator().manual_seed(1)) * spread).to(torch.bfloat16).to(DEV)
    cache = dq.Q8KVCache(1, 1, 4, 256, fmt)
    cache.append(k.to(DEV), v.to(DEV), 0)
    out = cache.attend(q, torch.tensor([256], dtype=torch.int32, device=DEV))
    # one token takes all the weight: its value
    x = _held(k, fmt)[0, 0] @ q[0].double().cpu().numpy().T
    want = _held(v, fmt)[0, 0][np.argmax(x, axis=0)]
    assert np.allclose(out[0].double().cpu().numpy(), want, rtol=1e-6, atol=0)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bits", range(10, 40, 3))
def test_attention_any_size_of_the_largest_score(dq, fmt, bits):
    """Scores about 2^bits whose largest grows from block to block, also where
    fp32 holds no differences of a few units any more."""
    T = 256
    k, v = _kv(19, 1, T, 1)
    k = (k.sign() * (1 + torch.arange(T).view(1, T, 1, 1) / T)).to(torch.bfloat16)
    k[..., 1:] = 0
    q = torch.zeros((1, 2, 128), dtype=torch.bfloat16)
    q[0, 0, 0], q[0, 1, 0] = 2.0 ** bits, -(2.0 ** bits)
    cache = dq.Q8KVCache(1, 1, 2, T, fmt)
    cache.append(k.to(DEV), v.to(DEV), 0)
    out = cache.attend(q.to(DEV), torch.tensor([T], dtype=torch.int32, device=DEV), softmax_scale=1.0)
    kf, vf = _held(k, fmt), _held(v, fmt)
    ref, _ = q8.attention(q.double().numpy(), kf, vf, [T], 2, 1.0)
    # one product and four roundings: a score of at most 2^(bits + 1.6) in base 2
    # is off by 2^(bits - 20), and so is a weight; from 2^16 on the keys with the
    # largest code (equal scores, exactly) share all the weight, since the next
    # code's score lies 2^(bits - 6) below
    tol = (2.0 ** (bits - 19) if bits < 16 else 0.0) + 1e-5
    assert np.max(np.abs(out[0].double().cpu().numpy() - ref[0])) <= tol * np.abs(vf).max()


@pytest.mark.parametrize("fmt", FMTS)
def test_rows_behind_the_length_do_not_matter(dq, fmt):
    """Codes of no number, infinite and NaN scales behind the length; bit for bit."""
    for window, sinks in ((0, 0), (70, 40)):
        cache, seq, q, out, _ = _attend_case(dq, fmt, [130, 999, 32, 0], 4, window=window, sinks=sinks)
        for b, T in enumerate([130, 999, 32, 0]):
            t = T % 32
            if t:
                for data, order in ((cache.k_data, q8.key_order()), (cache.v_data, q8.value_order())):
                    at = torch.from_numpy(order[t:].reshape(-1)).to(DEV)
                    data[b, :, T // 32, at] = 0x7F
            n = (T + 31) // 32
            cache.k_data[b, :, n:] = 0xFF
            cache.v_data[b, :, n:] = 0x7F
            cache.k_scales[b, :, n:] = math.nan
            cache.v_scales[b, :, n:] = math.inf
        assert torch.equal(cache.attend(q, seq, window=window, sinks=sinks), out)


@pytest.mark.parametrize("fmt", FMTS)
def test_query_that_is_no_number(dq, fmt):
    cache, seq, q, out, _ = _attend_case(dq, fmt, [200, 64], 4)
    q = q.clone()
    q[0, 2, 5], q[1, 7, 0] = math.nan, math.inf
    got = cache.attend(q, seq)
    assert torch.isnan(got[0, 2]).all() and torch.isnan(got[1, 7]).all()
    got[0, 2], got[1, 7] = out[0, 2], out[1, 7]
    assert torch.equal(got, out)


@pytest.mark.parametrize("fmt", FMTS)
def test_value_scales_far_apart(dq, fmt):
    """A block of large values without weight beside one of small values with all of it."""
    k, v = _kv(11, 1, 128, 1)
    k[0, :32] = -k[0, 32:33].abs() * 20
    k[0, 32:] = k[0, 32:33].abs()
    v[0, :32] = 2.0 ** 40
    q = (k[0, 32].abs() * 4).reshape(1, 1, 128).to(torch.bfloat16)
    cache = dq.Q8KVCache(1, 1, 1, 128, fmt)
    cache.append(k.to(DEV), v.to(DEV), 0)
    out = cache.attend(q.to(DEV), torch.tensor([128], dtype=torch.int32, device=DEV))
    ref, _ = q8.attention(q.double().numpy(), _held(k, fmt), _held(v, fmt), [128], 1, 128 ** -0.5)
    _check_out(out, ref, q.double().numpy(), _held(k, fmt), [128], 1, 128 ** -0.5)


def _paged(dq, fmt, B, H, mp, page, spare, seed):
    """Pools (0xA5 bytes), and a table of a random permutation of their pages."""
    n = B * mp + spare
    data = [torch.full((n, H, page // 32, 4096), 0xA5, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scale = [torch.full((n, H, page // 32), 3.0, device=DEV) for _ in range(2)]
    bt = torch.from_numpy(np.random.default_rng(seed).permutation(n)[:B * mp].astype(np.int32)).view(B, mp).to(DEV)
    return [data[0], scale[0], data[1], scale[1]], bt


def _from_pages(pool, bt):
    return pool[bt.long()].transpose(1, 2).flatten(2, 3)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("page", [128, 256])
def test_paged(dq, fmt, page):
    """Pages hold what the contiguous cache holds; the step, its window and
    scores are bit-identical; unmapped entries behind the length are not read;
    entries outside the pool are flagged and never written through."""
    B, H, G, t_cap = 3, 2, 4, 1024
    mp = t_cap // page
    pools, bt = _paged(dq, fmt, B, H, mp, page, 3, 5)
    k, v = _kv(13, B, t_cap, H)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ref = dq.Q8KVCache(B, H, H * G, t_cap, fmt, scores=True)
    for t0, n in ((0, 96), (96, 928)):
        ref.append(k[:, t0:t0 + n].to(DEV), v[:, t0:t0 + n].to(DEV), t0)
        dq.dq_q8_encode_kv_paged(fmt, k[:, t0:t0 + n].to(DEV), v[:, t0:t0 + n].to(DEV), t0, bt, *pools, status=status)
    for x, y in zip(ref.arrays, pools):
        assert torch.equal(_from_pages(y, bt), x)
    spare = sorted(set(range(pools[0].shape[0])) - set(bt.flatten().tolist()))
    assert torch.all(pools[0][spare] == 0xA5) and torch.all(pools[3][spare] == 3.0)
    rk, rv = dq.dq_q8_decode_kv_paged(fmt, *pools, bt, 64, 500, status=status)
    assert all(torch.equal(x, y) for x, y in zip((rk, rv), ref.read(64, 500)))
    lens = [1000, 130, 0]
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q = torch.randn((B, H * G, 128), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    cut = bt.clone()
    for b, T in enumerate(lens):
        cut[b, (T + page - 1) // page:] = -1
    for window, sinks in ((0, 0), (200, 33)):
        out = torch.full((B, H * G, 128), math.nan, device=DEV)
        scores = torch.zeros_like(ref.scores)
        ref.scores.zero_()
        lse = torch.empty_like(ref.block_lse)
        dq.dq_q8_decode_attention_paged(fmt, q, *pools, cut, seq, out, ref.workspace, window, sinks, block_lse=lse,
                                        scores=scores, status=status)
        want = ref.attend(q, seq, window=window, sinks=sinks)
        assert torch.equal(out, want) and torch.equal(scores, ref.scores)
        dq.dq_q8_decode_attention_paged_partial(fmt, q, *pools, cut, seq, ref.workspace, window, sinks, status=status)
        dq.dq_decode_attention_merge(B, H * G, H, seq, t_cap, ref.workspace, out)
        # the one-call form cuts the tokens otherwise: the same scores, weights of
        # 22 bits against other maxima (2 x 2^-22), sums over 32 blocks and their
        # parts with a rounding of 2^-24 each (2 x 40 x 2^-24): below 2^-17
        assert ((out - want).norm(dim=2) <= want.norm(dim=2) * 2.0 ** -17).all()
    assert int(status.item()) == 0
    bad = bt.clone()
    bad[0, 0], bad[1, 0] = pools[0].shape[0], -5
    before = [x.clone() for x in pools]
    dq.dq_q8_encode_kv_paged(fmt, k[:, :page].to(DEV) * 2, v[:, :page].to(DEV) * 2, 0, bad, *pools, status=status)
    assert int(status.item()) == dq.DQ_STATUS_PAGE
    for i, (x, y) in enumerate(zip(before, pools)):
        # twice the values: the same codes at twice the scale
        changed = (x != y).flatten(1).any(dim=1).nonzero().flatten().tolist()
        assert changed == ([int(bad[2, 0])] if i in (1, 3) else [])
    status.zero_()
    dq.dq_q8_decode_attention_paged(fmt, q, *pools, bad, seq, out, ref.workspace, status=status)
    assert int(status.item()) == dq.DQ_STATUS_PAGE and torch.isfinite(out).all()


def test_offsets_past_32_bits(dq):
    """A cache of 8.6 GB: the last sequence's blocks lie past 2^32 bytes."""
    B, H, t_cap = 4, 8, 1 << 20
    k, v = _kv(17, 1, 2048, H)
    small = dq.Q8KVCache(1, H, 32, 2048, "int8", scores=True)
    small.append(k.to(DEV), v.to(DEV), 0)
    big = dq.Q8KVCache(B, H, 32, t_cap, "int8", scores=True)
    big.append(k.to(DEV).expand(B, 2048, H, 128), v.to(DEV).expand(B, 2048, H, 128), t_cap - 2048)
    q = torch.randn((1, 32, 128), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    lens = torch.full((B,), t_cap, dtype=torch.int32, device=DEV)
    out = big.attend(q.expand(B, 32, 128).contiguous(), lens, window=2048)
    want = small.attend(q, torch.tensor([2048], dtype=torch.int32, device=DEV))
    assert torch.allclose(out, want.expand_as(out), rtol=0, atol=float(want.abs().max()) * 2.0 ** -20)
    gk, _ = big.read(t_cap - 64, 64)
    assert torch.equal(gk[3:], small.read(2048 - 64, 64)[0])
    kept, lens = big.evict(lens, 2048, 0, 1024)
    assert torch.equal(big.k_data[3, 7, 32:64], small.k_data[0, 7, 32:])


# --------------------------------------------------------- scores and eviction

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("G,window,sinks", [(4, 0, 0), (1, 0, 0), (8, 300, 50), (3, 1, 0)])
def test_scores(dq, fmt, G, window, sinks):
    """A step's block weights: fp32 sums of G numbers below 1 whose exponents
    are differences of logarithms (each rounded at the score's size)."""
    cache, seq, q, _, weight = _attend_case(dq, fmt, LENS, G, window=window, sinks=sinks, scores=True)
    got = cache.scores.double().cpu().numpy()
    assert np.max(np.abs(got - weight)) <= G * 3e-5
    seen = weight > 1e-3
    assert np.max(np.abs(got[seen] / weight[seen] - 1), initial=0) < 3e-5
    assert not got[weight == 0].any()
    total = got.sum(axis=2)
    assert np.allclose(total[np.array(LENS) > 0], G, rtol=3e-5) and not total[1].any()
    first = cache.scores.clone()
    cache.attend(q, seq, window=window, sinks=sinks)
    assert torch.equal(cache.scores, first + first)


@pytest.mark.parametrize("window,sinks", [(0, 0), (7000, 64)])
def test_scores_of_partials(dq, window, sinks):
    """More partials than a wavefront has lanes; the weights of a step's partials
    by a call of their own."""
    cache, seq, q, _, weight = _attend_case(dq, "int8", [16300], 4, H=1, t_cap=16384, window=window, sinks=sinks,
                                            scores=True)
    # as in test_scores
    assert np.max(np.abs(cache.scores.double().cpu().numpy() - weight)) <= 4 * 3e-5
    cache.scores.zero_()
    cache.partial(q, seq, window=window, sinks=sinks)
    cache.add_scores(seq, window, sinks)
    assert np.max(np.abs(cache.scores.double().cpu().numpy() - weight)) <= 4 * 3e-5
    assert np.isclose(float(cache.scores.sum(dtype=torch.float64)), 4, rtol=3e-5)


@pytest.mark.parametrize("lens,G,t_cap", [([1000, 0, 33, 500], 4, 1024), ([16300], 2, 16384), ([300, 1] * 40, 2, 384)])
@pytest.mark.parametrize("raw", [False, True])
def test_merge_scores_is_merge_and_scores(dq, lens, G, t_cap, raw):
    """In one launch what the two give, with and without a residual window (of 0 to 200 tokens)."""
    cache, seq, q, _, _ = _attend_case(dq, "e4m3", lens, G, H=2, t_cap=t_cap, scores=True)
    B = len(lens)
    rk, rv = (x.to(DEV).permute(0, 2, 1, 3).contiguous() for x in _kv(33, B, 256, 2))
    extra = torch.tensor([(200, 0, 7)[b % 3] for b in range(B)], dtype=torch.int32, device=DEV) if raw else None
    both = []
    for one in (False, True):
        out = torch.full((B, 2 * G, 128), math.nan, device=DEV)
        cache.scores.zero_()
        cache.partial(q, seq, extra_lens=extra)
        if raw:
            dq.dq_decode_attention_residual(q, rk, rv, seq, extra, t_cap, cache.workspace)
        if one:
            cache.merge_scores(seq, out, extra_lens=extra)
        else:
            cache.merge(seq, out)
            cache.add_scores(seq, extra_lens=extra)
        both.append((out, cache.scores.clone()))
    (a, sa), (b, sb) = both
    assert torch.equal(sa, sb)
    # the same partials in another order: at most 70 of them, a rounding of 2^-24 for
    # each product and each sum of the output and of its denominator
    assert ((a - b).norm(dim=2) <= a.norm(dim=2) * 4 * 70 * 2.0 ** -24).all()


def _fill(dq, fmt, B, H, t_cap, lens, seed, levels=None):
    k, v = _kv(seed, B, t_cap, H)
    cache = dq.Q8KVCache(B, H, 4 * H, t_cap, fmt, scores=True)
    cache.append(k.to(DEV), v.to(DEV), 0)
    g = torch.Generator().manual_seed(seed)
    s = torch.rand((B, H, t_cap // 32), generator=g)
    if levels:
        s = (s * levels).floor() / levels - 0.5        # ties, zeros of both signs, negatives
    cache.scores.copy_(s)
    return cache, torch.tensor(lens, dtype=torch.int32, device=DEV)


def _check_evict(old, old_scores, lens, to, kept, new_lens, keep, first, last):
    kept_n, scores = kept.cpu().numpy(), old_scores.cpu().numpy()
    for b, T in enumerate(lens):
        nb = (T + 31) // 32
        for h in range(kept.shape[1]):
            want = q8.evict(scores[b, h], nb, keep // 32, first // 32, last // 32)
            n = len(want)
            assert kept_n[b, h, :n].tolist() == want and (kept_n[b, h, n:] == -1).all(), (b, h)
            at = torch.tensor(want, dtype=torch.int64, device=DEV)
            for x, y in zip(old, to.arrays):
                assert torch.equal(x[b, h][at], y[b, h, :n])
            assert torch.equal(to.scores[b, h, :n], old_scores[b, h][at])
            assert not to.scores[b, h, n:min(nb, to.scores.shape[2])].any()
        assert int(new_lens[b]) == T - 32 * (nb - min(nb, keep // 32))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("levels", [None, 1, 3])
@pytest.mark.parametrize("keep,first,last", [(512, 0, 32), (512, 64, 128), (96, 32, 64), (32, 0, 32), (2016, 32, 32)])
def test_evict(dq, fmt, levels, keep, first, last):
    B, H, t_cap = 6, 2, 2048
    lens = [2048, 2047, 0, 96, 513, 1025]
    for into in (False, True):
        cache, seq = _fill(dq, fmt, B, H, t_cap, lens, 21, levels)
        old, old_scores = [x.clone() for x in cache.arrays], cache.scores.clone()
        to = dq.Q8KVCache(B, H, 4 * H, (keep + 127) // 128 * 128, fmt, scores=True) if into else cache
        kept, new_lens = cache.evict(seq, keep, first, last, into=to if into else None)
        torch.cuda.synchronize()
        _check_evict(old, old_scores, lens, to, kept, new_lens, keep, first, last)
        assert torch.equal(seq.cpu(), torch.tensor(lens, dtype=torch.int32))
        if into:
            for x, y in zip(old, cache.arrays):
                assert torch.equal(x, y)
        else:
            # what lies behind the kept blocks stays as it was
            for x, y in zip(old, cache.arrays):
                assert torch.equal(x[:, :, keep // 32:], y[:, :, keep // 32:])
            cache.evict(new_lens, keep, first, last, new_lens=new_lens)      # nothing more to do
            assert [int(x) for x in new_lens] == [T - 32 * max(0, (T + 31) // 32 - keep // 32) for T in lens]


def test_scores_begin_at_zero(dq):
    """Of appended blocks, and behind the kept ones of a cache that held more before."""
    cache, seq = _fill(dq, "int8", 2, 2, 512, [512, 100], 27)
    before = cache.scores.clone()
    k, v = _kv(28, 2, 40, 2)
    cache.append(k.to(DEV), v.to(DEV), 64)
    before[:, :, 2:4] = 0
    assert torch.equal(cache.scores, before)
    to, _ = _fill(dq, "int8", 2, 2, 1024, [1024, 1024], 29)
    cache.evict(seq, 256, 32, 64, into=to)
    assert not to.scores[0, :, 8:].any() and not to.scores[1, :, 4:].any()


def test_evict_nan_scores_and_many_blocks(dq):
    cache, seq = _fill(dq, "int8", 1, 2, 65536, [65536], 23)
    cache.scores[0, 0, 5::7] = math.nan
    cache.scores[0, 1, ::2] = math.inf
    cache.scores[0, 1, 1::2] = -math.inf
    old, old_scores = [x.clone() for x in cache.arrays], cache.scores.clone()
    kept, new_lens = cache.evict(seq, 60000 // 32 * 32, 32, 64)
    for b, h in ((0, 0), (0, 1)):
        want = q8.evict(old_scores[b, h].cpu().numpy(), 2048, 1875, 1, 2)
        assert kept[b, h].tolist() == want
        assert torch.equal(cache.k_data[b, h, :1875], old[0][b, h][torch.tensor(want, device=DEV)])


@pytest.mark.parametrize("into", [False, True])
@pytest.mark.parametrize("blocks", [260, 500, 4100, 9400, 17000])
def test_evict_numbers_of_blocks(dq, blocks, into):
    """Every kind of selection, up to several rounds; ties among them; bytes as they are."""
    B, H, t_cap = 2, 1, blocks * 32
    g = torch.Generator().manual_seed(blocks)
    cache = dq.Q8KVCache(B, H, H, t_cap, scores=True)
    for x in cache.arrays:
        x.copy_(torch.randint(0, 255, x.shape, generator=g, dtype=torch.int32))
    cache.scores.copy_((torch.rand(cache.scores.shape, generator=g) * 50).floor() / 50 - 0.5)
    lens = [t_cap, t_cap - 65]
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    keep = blocks * 2 // 3 // 4 * 128
    to = dq.Q8KVCache(B, H, H, keep, scores=True) if into else cache
    old, old_scores = [x.clone() for x in cache.arrays], cache.scores.clone()
    kept, new_lens = cache.evict(seq, keep, 70, 130, into=to if into else None)
    torch.cuda.synchronize()
    _check_evict(old, old_scores, lens, to, kept, new_lens, keep, 96, 160)


def test_evict_into_another_cache_over_the_old_lengths(dq):
    """The new lengths in the old ones' place, a short and a long cache."""
    for t_cap in (1024, 16384):
        lens = [t_cap, 700, 0, 33]
        cache, seq = _fill(dq, "int8", 4, 2, t_cap, lens, 35)
        to = dq.Q8KVCache(4, 2, 8, 512, scores=True)
        kept, new_lens = cache.evict(seq, 512, 32, 64, into=to, new_lens=seq)
        torch.cuda.synchronize()
        assert new_lens is seq
        _check_evict(cache.arrays, cache.scores, lens, to, kept, seq, 512, 32, 64)


@pytest.mark.parametrize("page", [128, 512])
def test_evict_paged(dq, page):
    B, H, t_cap, keep = 3, 2, 2048, 640
    lens = [2048, 1999, 600]
    ref, seq = _fill(dq, "e4m3", B, H, t_cap, lens, 25, 4)
    mp = t_cap // page
    pools, bt = _paged(dq, "e4m3", B, H, mp, page, 2, 6)
    for x, y in zip(ref.arrays, pools):
        rest = x.shape[3:]
        y[bt.flatten().long()] = x.view(B, H, mp, page // 32, *rest).transpose(1, 2).reshape(B * mp, H, page // 32, *rest)
    scores, status = ref.scores.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
    kept = torch.empty((B, H, keep // 32), dtype=torch.int32, device=DEV)
    new = seq.clone()
    dq.dq_q8_evict_paged(new, new, keep, 32, 64, bt, pools, scores, kept, status)
    want_kept, want_new = ref.evict(seq, keep, 32, 64)
    assert torch.equal(kept, want_kept) and torch.equal(new, want_new) and torch.equal(scores, ref.scores)
    for x, y in zip(ref.arrays, pools):
        assert torch.equal(_from_pages(y, bt)[:, :, :keep // 32], x[:, :, :keep // 32])
    assert int(status.item()) == 0


# ----------------------------------------------------------- the parts together

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5)])
def test_streaming_cache(dq, fmt, window, sinks):
    """Prefill, appends over several flushes, a step over codes and raw tokens
    with scores, an eviction, and steps after it."""
    B, H, G = 2, 2, 4
    k, v = _kv(31, B, 1200, H)
    c = dq.StreamingKVCache(B, H, H * G, 1280, None, None, streams=fmt, scores=True)
    plain = dq.StreamingKVCache(B, H, H * G, 1280, None, None, streams=fmt)
    for x in (c, plain):
        x.prefill(k[:, :900].to(DEV), v[:, :900].to(DEV))
    held_k, held_v = _held(k, fmt), _held(v, fmt)
    raw_k, raw_v = _f64(k), _f64(v)
    score = np.zeros((B, H, 40))
    rows = np.tile(np.arange(c.n_comp), (B, H, 1))           # the token in each compressed row
    for step in range(160):
        t = 900 + step
        for x in (c, plain):
            x.append(k[:, t].to(DEV).contiguous(), v[:, t].to(DEV).contiguous())
        if c.n_comp > rows.shape[2]:
            new = np.arange(t + 1 - c.n_res - 128, t + 1 - c.n_res)
            rows = np.concatenate([rows, np.tile(new, (B, H, 1))], axis=2)
        if step % 40 != 7:
            continue
        q = torch.randn((B, H * G, 128), generator=torch.Generator().manual_seed(step)).to(torch.bfloat16)
        out = c.attend(q.to(DEV), window=window, sinks=sinks)
        n, r = c.n_comp, c.n_res
        kk = np.take_along_axis(held_k, rows[..., None], axis=2)
        vv = np.take_along_axis(held_v, rows[..., None], axis=2)
        first = t + 1 - r
        ref, w = q8.attention(q.double().numpy(), kk, vv, [n] * B, G, 128 ** -0.5, window, sinks,
                              raw_k[:, :, first:t + 1], raw_v[:, :, first:t + 1], [r] * B)
        both = np.concatenate([kk, raw_k[:, :, first:t + 1]], axis=2)
        _check_out(out, ref, q.double().numpy(), both, [n + r] * B, G, 128 ** -0.5)
        score[:, :, :w.shape[2]] += w
        got = c.cache.scores.double().cpu().numpy()
        assert np.max(np.abs(got - score)) < 3e-4
        if step < 100:
            one = plain.attend(q.to(DEV), window=window, sinks=sinks)
            assert torch.allclose(one, out, rtol=0, atol=1e-5 * float(out.abs().max()))
        if step == 87:
            kept = c.evict(400, 32, 64)
            assert (n, c.n_comp, kept.shape[2]) == (768, 512, 16)      # whole rings of 256 tokens leave
            kept = kept.cpu().numpy()
            nb = n // 32
            for b in range(B):
                for h in range(H):
                    assert kept[b, h].tolist() == q8.evict(got[b, h], nb, kept.shape[2], 1, 2)
            tok = (kept[..., None] * 32 + np.arange(32)).reshape(B, H, -1)
            rows = np.take_along_axis(rows, tok, axis=2)
            score = np.take_along_axis(score, kept, axis=2)
            score = np.concatenate([score, np.zeros((B, H, 40 - score.shape[2]))], axis=2)
            assert c.evict(400, 32, 64) is None
    assert int(c.status.item()) == 0
    assert [int(x) for x in c.seq_lens] == [c.n_comp] * B


def test_streaming_refusals(dq):
    c = dq.StreamingKVCache(1, 2, 8, 512, None, None, streams="int8")
    q = torch.zeros((1, 8, 128), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        c.attend(q, window=100)
    with pytest.raises(dq.DqError):
        c.attend(q, sinks=4)
    assert torch.all(c.attend(q) == 0)
    with pytest.raises(ValueError):
        dq.StreamingKVCache(1, 2, 8, 512, None, None, streams="int8").cache.evict(c.seq_lens, 128)


def test_device_refusals(dq):
    cache = dq.Q8KVCache(1, 2, 8, 128)
    q = torch.zeros((1, 8, 128), dtype=torch.bfloat16, device=DEV)
    lens = torch.zeros(1, dtype=torch.int32, device=DEV)
    for bad in (q.cpu(), q.float(), q[:, ::2], q.transpose(1, 2), q[:, :7].contiguous(), q.expand(2, 8, 128)):
        with pytest.raises((ValueError, dq.DqError)):
            cache.attend(bad, lens)
    for bad in (lens.cpu(), lens.long(), torch.zeros(2, dtype=torch.int32, device=DEV)):
        with pytest.raises(ValueError):
            cache.attend(q, bad)
    for kw in (dict(window=-1), dict(window=2 ** 31), dict(sinks=3), dict(out=q), dict(out=q.float().cpu())):
        with pytest.raises((ValueError, dq.DqError)):
            cache.attend(q, lens, **kw)
    with pytest.raises(ValueError):
        cache.attend(q, lens, scores=torch.zeros((1, 2, 4), device=DEV))
    kv = torch.zeros((1, 32, 2, 128), dtype=torch.bfloat16, device=DEV)
    for t0 in (-32, 16, 128, 2 ** 32):
        with pytest.raises((ValueError, dq.DqError)):
            cache.append(kv, kv, t0)
    with pytest.raises(ValueError):
        cache.append(kv, kv[:, :31], 0)


def test_graph_replays(dq):
    """A captured step with scores, replayed with new queries and lengths and
    eager steps between; then a captured eviction."""
    B, H, G = 3, 2, 4
    cache, seq = _fill(dq, "int8", B, H, 2048, [2048, 70, 0], 41)
    q = torch.randn((B, H * G, 128), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).to(DEV)
    out, scores = torch.empty((B, H * G, 128), device=DEV), torch.zeros_like(cache.scores)

    def step():
        cache.attend(q, seq, out=out, scores=scores, window=700, sinks=40)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        q.copy_(torch.randn((B, H * G, 128), generator=torch.Generator().manual_seed(50 + i)).to(torch.bfloat16))
        seq.copy_(torch.tensor([[2048, 1, 33], [0, 2000, 64], [5, 5, 5], [1111, 2047, 31]][i], dtype=torch.int32))
        scores.zero_()
        g.replay()
        torch.cuda.synchronize()
        got, got_scores = out.clone(), scores.clone()
        want_scores = torch.zeros_like(scores)
        want = cache.attend(q, seq, scores=want_scores, window=700, sinks=40)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(got_scores, want_scores), i
    to = dq.Q8KVCache(B, H, H * G, 512, "int8", scores=True)
    kept, new = torch.empty((B, H, 16), dtype=torch.int32, device=DEV), torch.empty_like(seq)

    def cut():
        dq.dq_q8_evict(seq, new, 512, 32, 32, (*cache.arrays, cache.scores), (*to.arrays, to.scores), kept)

    cut()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cut()
    for i in range(3):
        cache.scores.copy_(torch.rand(cache.scores.shape, generator=torch.Generator().manual_seed(i)))
        seq.copy_(torch.tensor([[2048, 1, 33], [0, 2000, 64], [1111, 2047, 512]][i], dtype=torch.int32))
        kept.zero_()
        g.replay()
        torch.cuda.synchronize()
        _check_evict(cache.arrays, cache.scores, seq.tolist(), to, kept, new, 512, 32, 32)


def test_two_streams(dq):
    """Steps of two caches on two streams at once, each with its own workspace."""
    cases = [_attend_case(dq, "e4m3", [1024, 77], 4, seed=s) for s in (61, 62)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        outs = []
        for (cache, seq, q, out, _), s in zip(cases, streams):
            with torch.cuda.stream(s):
                outs.append([cache.attend(q, seq) for _ in range(4)])
        torch.cuda.synchronize()
        for (_, _, _, out, _), got in zip(cases, outs):
            assert all(torch.equal(x, out) for x in got)


def test_graph_of_an_eviction_in_place(dq):
    """A captured eviction in place, lengths included, replayed on new contents."""
    cache, seq = _fill(dq, "e4m3", 2, 2, 1024, [1024, 300], 71)
    arrays = [x.clone() for x in cache.arrays]
    kept = torch.empty((2, 2, 8), dtype=torch.int32, device=DEV)

    def cut():
        own = (*cache.arrays, cache.scores)
        dq.dq_q8_evict(seq, seq, 256, 64, 32, own, own, kept)

    cut()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cut()
    for i in range(3):
        for x, y in zip(arrays, cache.arrays):
            y.copy_(x)
        cache.scores.copy_(torch.rand(cache.scores.shape, generator=torch.Generator().manual_seed(80 + i)))
        lens = [[1024, 0], [999, 256], [257, 1000]][i]
        seq.copy_(torch.tensor(lens, dtype=torch.int32))
        before = cache.scores.clone()
        g.replay()
        torch.cuda.synchronize()
        _check_evict(arrays, before, lens, cache, kept, seq, 256, 64, 32)


def test_read_on_another_stream(dq):
    cache, _ = _fill(dq, "int8", 1, 2, 1024, [1024], 73)
    want = cache.read(32, 900)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = dq.dq_q8_decode_kv("int8", *cache.arrays, 32, 900, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_deep_copy_is_a_cache_of_its_own(dq):
    cache, seq, q, out, _ = _attend_case(dq, "int8", [300, 45], 2, t_cap=384, scores=True)
    other = copy.deepcopy(cache)
    before, scores = [x.clone() for x in cache.arrays], cache.scores.clone()
    assert torch.equal(other.attend(q, seq), out) and torch.equal(other.scores, 2 * scores)
    k, v = _kv(91, 2, 384, 2)
    other.append(k.to(DEV), v.to(DEV), 0)
    other.evict(seq, 128, 32, 32)
    torch.cuda.synchronize()
    assert torch.equal(cache.scores, scores) and all(torch.equal(x, y) for x, y in zip(cache.arrays, before))
    assert torch.equal(cache.attend(q, seq), out)


def test_query_heads_other_than_the_cache_s(dq):
    """The scores' scratch is made for the cache's heads."""
    cache = dq.Q8KVCache(1, 2, 4, 128, scores=True)
    lens = torch.full((1,), 64, dtype=torch.int32, device=DEV)
    q = torch.zeros((1, 16, 128), dtype=torch.bfloat16, device=DEV)
    for call in (lambda: cache.attend(q, lens), lambda: cache.attend(q, lens, scores=cache.scores),
                 lambda: cache.partial(q, lens)):
        with pytest.raises((ValueError, dq.DqError)):
            call()
