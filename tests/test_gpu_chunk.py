"""Attention of many queries (the chunk over the 8-bit cache, cross attention
over BF16 states) on the GPU against the formula in 64 bits: lengths from none
to long, odd sizes, windows, masks, empty rows, pages, strides, values of all
sizes, graphs and streams, and the calls together.

Tolerance of an output row, in its 2-norm.  With a the exact weights and
V = sum a |v| (elementwise):
* the output is rounded to bf16 once: 2^-8 of the row;
* every weight is rounded for the product with the values, to fp16 (2^-11) over
  codes and to bf16 (2^-8) over BF16 states: that much of V;
* a score (base 2) is a sum of 128 exact products in fp32, in eight matrix
  instructions of 16 terms each, and meets up to four rounded factors and the
  rounded maximum: with X the largest sum of |q k| scale log2 e its error is at
  most 14 2^-24 X, a weight's ln 2 times that, twice with the denominator;
* the exponent also takes the logarithm of a block's scale (up to 2^7, three
  roundings of 2^-18), the sums a few roundings more: 2^-15 of V covers both.
A weight below 2^-21 of the row's largest loses up to 2^-32 of that: within the
last term at the lengths used here."""

import copy
import math

import numpy as np
import pytest
import torch

from oracle import q8

pytestmark = pytest.mark.gpu

DEV = "cuda"
FMTS = ["int8", "e4m3"]
LOG2E = 1.4426950408889634


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


def _q(seed, B, n, Hq):
    g = torch.Generator().manual_seed(1000 + seed)
    return torch.randn((B, n, Hq, 128), generator=g).to(torch.bfloat16)


def _held(x, fmt):
    """The values the cache holds of x [B, T, H, 128]: fp64 [B, H, nb 32, 128] on the GPU."""
    codes, s = q8.quantize(x.double().cpu().numpy().transpose(0, 2, 1, 3), fmt)
    return torch.from_numpy(np.ascontiguousarray(q8.values(codes, s, fmt))).to(DEV)


def _visible(T, n, rows, causal, window, sinks):
    """[n, T] truth values of a sequence of T tokens whose queries are n."""
    t = torch.arange(T, device=DEV)[None]
    if not causal:
        return torch.ones((rows, T), dtype=torch.bool, device=DEV)
    p = torch.arange(rows, device=DEV)[:, None] + (T - n)
    see = t <= p
    if window:
        see = see & ((t < sinks) | (t > p - window))
    return see


def _check(got, q, k, v, see, scale, wbits):
    """got [n, Hq, 128] of one sequence against k, v fp64 [H, T, 128]."""
    n, Hq, _ = q.shape
    H, T, _ = k.shape
    G = Hq // H
    got = got.double()
    for i in range(Hq):
        kk, vv = k[i // G], v[i // G]
        x = q[:, i].double().to(DEV)
        s = (x @ kk.T) * scale
        s = torch.where(see, s, -math.inf)
        top = s.amax(dim=1, keepdim=True) if T else s.new_zeros((n, 1))
        empty = ~see.any(dim=1) if T else torch.ones(n, dtype=torch.bool, device=DEV)
        a = torch.exp(s - torch.where(empty[:, None], 0.0, top))
        a = a / a.sum(dim=1, keepdim=True).clamp(min=1e-300)
        ref = a @ torch.where(see.any(dim=0)[:, None], vv, 0.0) if T else torch.zeros((n, 128), dtype=torch.float64, device=DEV)
        spread = a @ torch.where(see.any(dim=0)[:, None], vv.abs(), 0.0) if T else ref
        X = float((x.abs() @ kk.abs().T)[see].max()) * abs(scale) * LOG2E if bool(see.any()) else 0.0
        tol = 2.0 ** -8 * ref.norm(dim=1) + (2.0 ** -wbits + 2 * math.log(2) * 14 * 2.0 ** -24 * X + 2.0 ** -15) * \
            spread.norm(dim=1)
        err = (got[:, i] - ref).norm(dim=1)
        bad = ~(err <= tol)
        assert not bool(bad.any()), (i, int(bad.nonzero()[0]), float(err[bad][0]), float(tol[bad][0]))
        assert bool((got[empty, i] == 0).all()), i


def _check_all(out, q, k, v, lens, new, scale=128 ** -0.5, causal=True, window=0, sinks=0, wbits=11):
    """k, v fp64 [B, H, T', 128]; lens and new per sequence."""
    for b in range(q.shape[0]):
        T, n = int(lens[b]), int(new[b])
        see = _visible(T, n, n, causal, window, sinks)
        _check(out[b, :n], q[b, :n], k[b, :, :T], v[b, :, :T], see, scale, wbits)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _filled(dq, fmt, k, v, Hq, t_cap=None):
    B, T, H, _ = k.shape
    cache = dq.Q8KVCache(B, H, Hq, t_cap or max(1, -(-T // 128)) * 128, fmt)
    cache.append(k.to(DEV), v.to(DEV), 0)
    return cache


# --------------------------------------------------------------- the 8-bit cache

SIZES = [  # B, T, n, H, G
    (1, 1, 1, 1, 1), (2, 33, 5, 2, 4), (1, 64, 64, 1, 1), (3, 200, 200, 2, 3), (1, 300, 17, 8, 8), (2, 513, 129, 1, 2),
    (1, 1111, 300, 2, 4), (1, 4000, 3, 1, 1), (1, 2500, 9, 2, 7), (5, 257, 64, 2, 16), (1, 1025, 1025, 1, 4)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,T,n,H,G", SIZES)
def test_chunk_sizes(dq, fmt, B, T, n, H, G, causal):
    k, v = _kv(T + n, B, T, H)
    q = _q(T, B, n, H * G)
    cache = _filled(dq, fmt, k, v, H * G)
    out = cache.attend_chunk(q.to(DEV), _i32([T] * B), causal=causal)
    assert out.dtype == torch.bfloat16 and out.shape == q.shape
    _check_all(out, q, _held(k, fmt), _held(v, fmt), [T] * B, [n] * B, causal=causal)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,T,n,H,G,cap", [(6, 500, 40, 2, 4, 512), (70, 130, 12, 1, 3, 256), (130, 90, 5, 1, 1, 128),
                                           (4, 3000, 200, 2, 2, 16384), (150, 700, 40, 1, 4, 768),
                                           (140, 300, 70, 8, 1, 384), (9, 2000, 33, 8, 4, 2048),
                                           (70, 1500, 90, 3, 2, 1536)])
def test_ragged(dq, fmt, B, T, n, H, G, cap):
    """Lengths from none up, chunks from none up, chunks longer than their
    sequence (their first rows see nothing); rows behind a chunk stay."""
    k, v = _kv(T, B, T, H)
    q = _q(n, B, n, H * G)
    r = np.random.default_rng(T)
    lens, new = r.integers(0, T + 1, B), r.integers(0, n + 1, B)
    lens[:3], new[:3] = [0, T, 3], [n, n, n]
    new[3], lens[3] = 0, T // 2
    cache = _filled(dq, fmt, k, v, H * G, cap)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    got = cache.attend_chunk(q.to(DEV), _i32(lens.tolist()), q_lens=_i32(new.tolist()), out=out)
    assert got is out
    _check_all(out, q, _held(k, fmt), _held(v, fmt), lens, new)
    for b in range(B):
        assert bool((out[b, int(new[b]):] == 7.0).all())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 1), (32, 0), (33, 37), (100, 4), (128, 128), (5000, 3), (700, 2000)])
def test_window(dq, fmt, window, sinks):
    B, T, n, H, G = 2, 900, 150, 1, 4
    k, v = _kv(window, B, T, H)
    q = _q(sinks, B, n, H * G)
    cache = _filled(dq, fmt, k, v, H * G)
    lens = [900, 611]
    out = cache.attend_chunk(q.to(DEV), _i32(lens), window=window, sinks=sinks)
    _check_all(out, q, _held(k, fmt), _held(v, fmt), lens, [n] * B, window=window, sinks=sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (900, 50)])
@pytest.mark.parametrize("B,T,n,H,G", [(1, 4100, 63, 1, 1), (1, 4100, 64, 8, 1), (1, 4100, 65, 1, 1), (2, 3001, 13, 8, 5),
                                       (2, 3001, 26, 8, 5), (1, 2050, 129, 16, 1), (3, 1999, 43, 5, 3)])
def test_pieces(dq, B, T, n, H, G, window, sinks):
    """Sequences that are cut, of row counts around the variants' borders, heads
    that are and are not a multiple of 8."""
    fmt = FMTS[n % 2]
    k, v = _kv(T + n, B, T, H)
    q = _q(T, B, n, H * G)
    cache = _filled(dq, fmt, k, v, H * G)
    lens = [T - 5 * b for b in range(B)]
    out = cache.attend_chunk(q.to(DEV), _i32(lens), window=window, sinks=sinks)
    _check_all(out, q, _held(k, fmt), _held(v, fmt), lens, [n] * B, window=window, sinks=sinks)


@pytest.mark.parametrize("n,window,sinks", [(3, 64, 4), (300, 64, 40)])
def test_window_of_a_long_sequence(dq, n, window, sinks):
    """Far behind the window nothing is read: what lies there may be anything."""
    T, H, G = 20000, 1, 2
    k, v = _kv(5, 1, T, H)
    q = _q(6, 1, n, H * G)
    cache = _filled(dq, "int8", k, v, H * G)
    kk, vv = _held(k, "int8"), _held(v, "int8")
    cache.k_scales[:, :, 2:T // 32 - 15] = math.nan
    cache.v_scales[:, :, 2:T // 32 - 15] = math.nan
    out = cache.attend_chunk(q.to(DEV), _i32([T]), window=window, sinks=sinks)
    _check_all(out, q, kk, vv, [T], [n], window=window, sinks=sinks)


def _paged(dq, fmt, k, v, page, seed=0, spare=3):
    B, T, H, _ = k.shape
    mp = -(-T // page)
    num = B * mp + spare
    bt = torch.from_numpy(np.random.default_rng(seed).permutation(num)[:B * mp].reshape(B, mp).astype(np.int32)).to(DEV)
    shape = (num, H, page // 32)
    pools = [torch.zeros((*shape, 4096), dtype=torch.uint8, device=DEV), torch.zeros(shape, device=DEV),
             torch.zeros((*shape, 4096), dtype=torch.uint8, device=DEV), torch.zeros(shape, device=DEV)]
    dq.dq_q8_encode_kv_paged(fmt, k.to(DEV), v.to(DEV), 0, bt, *pools)
    return pools, bt


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("page", [128, 512])
@pytest.mark.parametrize("n,window", [(4, 0), (90, 0), (90, 70)])
def test_paged_is_the_contiguous_call(dq, fmt, page, n, window):
    B, T, H, G = 3, 1000, 2, 4
    k, v = _kv(page + n, B, T, H)
    q = _q(n, B, n, H * G).to(DEV)
    pools, bt = _paged(dq, fmt, k, v, page)
    mp = bt.shape[1]
    cache = _filled(dq, fmt, k, v, H * G, mp * page)       # (the same capacity: the same plan)
    lens, new = _i32([1000, 77, 513]), _i32([n, min(n, 50), n])
    a = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    b = torch.zeros_like(a)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    cache.attend_chunk(q, lens, q_lens=new, out=a, window=window)
    dq.dq_q8_chunk_attention_paged(fmt, q, *pools, bt, lens, q_lens=new, out=b, window=window, status=status)
    assert torch.equal(a, b) and int(status) == 0


def test_bad_page(dq):
    """An entry outside the pool: page 0 in its place, and the status bit."""
    k, v = _kv(3, 1, 384, 1)
    q = _q(3, 1, 40, 2).to(DEV)
    pools, bt = _paged(dq, "int8", k, v, 128)
    good = bt.clone()
    for bad in (-1, pools[0].shape[0], 0x7FFFFFFF):
        bt[0, 1], good[0, 1] = bad, 0
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        a = dq.dq_q8_chunk_attention_paged("int8", q, *pools, bt, _i32([384]), status=status)
        b = dq.dq_q8_chunk_attention_paged("int8", q, *pools, good, _i32([384]))
        assert torch.equal(a, b) and int(status) == dq.DQ_STATUS_PAGE
        # behind the length an entry is not looked at
        status.zero_()
        dq.dq_q8_chunk_attention_paged("int8", q, *pools, bt, _i32([128]), status=status)
        assert int(status) == 0


@pytest.mark.parametrize("n", [3, 70])
def test_strides(dq, n):
    """Queries and outputs at other strides and alignments: the same bits."""
    B, T, H, G = 2, 400, 2, 3
    Hq = H * G
    k, v = _kv(n, B, T, H)
    q = _q(n, B, n, Hq).to(DEV)
    cache = _filled(dq, "e4m3", k, v, Hq)
    want = cache.attend_chunk(q, _i32([T] * B))
    heads_first = q.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    wide = torch.zeros((B, n, Hq, 131), dtype=torch.bfloat16, device=DEV)
    wide[..., 1:129] = q
    for x in (heads_first, wide[..., 1:129]):
        for o in (torch.zeros((B, Hq, n, 128), dtype=torch.bfloat16, device=DEV).permute(0, 2, 1, 3),
                  torch.zeros((B, n, Hq, 133), dtype=torch.bfloat16, device=DEV)[..., 3:131], None):
            got = cache.attend_chunk(x, _i32([T] * B), out=o)
            assert torch.equal(got, want)
    frame = torch.full((B, n, Hq, 133), 5.0, dtype=torch.bfloat16, device=DEV)
    cache.attend_chunk(q, _i32([T] * B), out=frame[..., 3:131])
    assert bool((frame[..., :3] == 5).all()) and bool((frame[..., 131:] == 5).all())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 7)])
def test_one_query_is_the_decode_step(dq, fmt, window, sinks):
    B, T, H, G = 3, 700, 2, 4
    k, v = _kv(1, B, T, H)
    q = _q(1, B, 1, H * G).to(DEV)
    cache = _filled(dq, fmt, k, v, H * G)
    lens = _i32([700, 1, 333])
    a = cache.attend_chunk(q, lens, window=window, sinks=sinks)[:, 0].float()
    b = cache.attend(q[:, 0].contiguous(), lens, window=window, sinks=sinks)
    # (two roundings to bf16 and the fp16 weights)
    assert float((a - b).norm() / b.norm()) < 2.0 ** -8 + 2.0 ** -10


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("n", [5, 150])
@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0, 1e4, 1e30])
def test_softmax_scales(dq, fmt, n, scale):
    B, T, H, G = 1, 1500, 1, 2
    k, v = _kv(2, B, T, H)
    q = _q(2, B, n, H * G)
    cache = _filled(dq, fmt, k, v, H * G)
    out = cache.attend_chunk(q.to(DEV), _i32([T]), softmax_scale=scale)
    if abs(scale) < 100:
        _check_all(out, q, _held(k, fmt), _held(v, fmt), [T], [n], scale=scale)
    else:
        # a step function: the largest score's value, where no other is near
        kk, vv = _held(k, fmt), _held(v, fmt)
        s = torch.einsum("nd,td->nt", q[0, :, 0].double().to(DEV), kk[0, 0, :T])
        see = _visible(T, n, n, True, 0, 0)
        best = torch.where(see, s, -math.inf).topk(2, dim=1)
        alone = (best.values[:, 0] - best.values[:, 1]) > 1e-4 * s.abs().amax(dim=1)
        want = vv[0, 0, best.indices[:, 0]]
        err = (out[0, :, 0].double() - want).abs().amax(dim=1) / want.abs().amax(dim=1)
        assert bool(torch.isfinite(out.float()).all())
        if scale >= 1e30:
            assert float(err[alone].max()) < 2.0 ** -8


@pytest.mark.parametrize("fmt", FMTS)
def test_values_of_all_sizes(dq, fmt):
    """Blocks of values between 1e-20 and 1e20, zeros among them, in any order:
    an output is as exact as its largest term."""
    T, n, H, G = 1280, 33, 1, 2
    k, v = _kv(4, 1, T, H, spread=0.3)
    q = _q(4, 1, n, H * G)
    g = np.random.default_rng(4)
    for order in (np.linspace(-20, 20, T // 32), np.linspace(20, -20, T // 32), g.uniform(-20, 20, T // 32)):
        x = v.float() * torch.from_numpy(10.0 ** np.repeat(order, 32)).float()[None, :, None, None]
        x[:, 64:96] = 0
        x = x.to(torch.bfloat16)
        cache = _filled(dq, fmt, k, x, H * G)
        out = cache.attend_chunk(q.to(DEV), _i32([T]))
        _check_all(out, q, _held(k, fmt), _held(x, fmt), [T], [n])


def test_queries_of_all_sizes_and_nan(dq):
    T, n, H, G = 300, 40, 1, 2
    k, v = _kv(8, 1, T, H)
    q = _q(8, 1, n, H * G)
    q[0, :20] = (q[0, :20].float() * torch.logspace(-30, 2, 20)[:, None, None]).to(torch.bfloat16)
    q[0, 21] = 0
    cache = _filled(dq, "int8", k, v, H * G)
    clean = cache.attend_chunk(q.to(DEV), _i32([T]))
    _check_all(clean, q, _held(k, "int8"), _held(v, "int8"), [T], [n])
    for what in (math.nan, math.inf, -math.inf):
        bad = q.clone()
        bad[0, 30, 1, 77] = what
        out = cache.attend_chunk(bad.to(DEV), _i32([T]))
        assert bool(torch.isnan(out[0, 30, 1]).all())
        keep = torch.ones((n, H * G), dtype=torch.bool, device=DEV)
        keep[30, 1] = False
        assert torch.equal(out[0][keep], clean[0][keep])
        # a row that sees nothing is zeros whatever its query holds
        out = cache.attend_chunk(bad.to(DEV), _i32([5]))
        assert bool((out[0, :35] == 0).all()) and bool(torch.isfinite(out[0, 35:].float()).all())


@pytest.mark.parametrize("n,rows", [(2, 2), (80, 80)])
def test_offsets_past_2_31(dq, n, rows):
    """Over 2^31 bytes of codes: one unit of 512 tokens repeated, so that not
    causal the attention is the unit's."""
    T, unit = (1 << 24) + 1024, 512
    k, v = _kv(9, 1, unit, 1)
    q = _q(9, 1, n, 2)
    small = _filled(dq, "int8", k, v, 2)
    cache = dq.Q8KVCache(1, 1, 2, T, "int8")
    for to, x in zip(cache.arrays, small.arrays):
        to.view(1, 1, T // unit, *x.shape[2:])[:] = x[:, :, None]
    out = cache.attend_chunk(q.to(DEV), _i32([T]), causal=False)
    _check_all(out, q, _held(k, "int8"), _held(v, "int8"), [unit], [n], causal=False)
    # the far end, behind a window
    out = cache.attend_chunk(q.to(DEV), _i32([T]), window=unit)
    far = torch.cat([k, k], dim=1), torch.cat([v, v], dim=1)
    _check_all(out, q, _held(far[0], "int8"), _held(far[1], "int8"), [2 * unit], [n], window=unit)


def test_the_same_bits_again(dq):
    k, v = _kv(11, 2, 3000, 2)
    cache = _filled(dq, "int8", k, v, 8)
    for n in (3, 200):
        q = _q(11, 2, n, 8).to(DEV)
        first = cache.attend_chunk(q, _i32([3000, 1200]))
        for _ in range(3):
            assert torch.equal(cache.attend_chunk(q, _i32([3000, 1200])), first)


def test_streams_and_workspaces(dq):
    """Two streams at once, each with its own workspace; one given too small."""
    k, v = _kv(12, 1, 5000, 2)
    cache = _filled(dq, "int8", k, v, 8)
    lens = _i32([5000])
    qs = [_q(i, 1, 6, 8).to(DEV) for i in range(2)]
    want = [cache.attend_chunk(q, lens) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(10):
        for s, q in zip(streams, qs):
            got.append(dq.dq_q8_chunk_attention("int8", q, *cache.arrays, lens, stream=s))
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert torch.equal(x, want[i % 2])
    need = dq.dq_chunk_workspace_bytes(1, 6, 8, 2, cache.t_cap)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    assert torch.equal(cache.attend_chunk(qs[0], lens, workspace=ws), want[0])
    with pytest.raises(dq.DqError):
        cache.attend_chunk(qs[0], lens, workspace=ws[:need - 16])


@pytest.mark.parametrize("n", [4, 130])
def test_graph(dq, n):
    """Captured: new queries, lengths and chunks at every replay, eager work and
    synchronizations between them."""
    k, v = _kv(13, 2, 2000, 1)
    cache = _filled(dq, "e4m3", k, v, 4)
    q = _q(13, 2, n, 4).to(DEV)
    lens, new = _i32([2000, 900]), _i32([n, n])
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(dq.dq_chunk_workspace_bytes(2, n, 4, 1, cache.t_cap), dtype=torch.uint8, device=DEV)
    call = lambda o: cache.attend_chunk(q, lens, q_lens=new, out=o, workspace=ws)  # noqa: E731
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i, (l2, n2) in enumerate([([2000, 900], [n, n]), ([1, 2000], [1, n]), ([0, 64], [n, 2]), ([1999, 33], [3, 0])]):
        q.copy_(_q(20 + i, 2, n, 4))
        lens.copy_(_i32(l2))
        new.copy_(_i32(n2))
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.full_like(out, 3.0)
        call(want)
        assert torch.equal(out, want)


# ------------------------------------------------------------- cross attention

def _cross(dq, q, k, v, lens=None, mask=None, new=None, scale=None, out=None):
    return dq.dq_cross_attention(q.to(DEV), k.to(DEV), v.to(DEV), kv_lens=None if lens is None else _i32(lens),
                                 mask=None if mask is None else mask.to(DEV), q_lens=None if new is None else _i32(new),
                                 softmax_scale=scale, out=out)


def _check_cross(out, q, k, v, lens, new, mask=None, scale=128 ** -0.5):
    kk, vv = (x.double().to(DEV).permute(0, 2, 1, 3) for x in (k, v))
    for b in range(q.shape[0]):
        T, n = int(lens[b]), int(new[b])
        see = torch.ones((n, T), dtype=torch.bool, device=DEV)
        if mask is not None:
            see = see & (mask[b, :T].to(DEV) != 0)[None]
        hidden = ~see.any(dim=0)
        kb, vb = kk[b, :, :T].clone(), vv[b, :, :T].clone()
        kb[:, hidden], vb[:, hidden] = 0.0, 0.0
        _check(out[b, :n], q[b, :n], kb, vb, see, scale, 8)


@pytest.mark.parametrize("B,T,n,H,G", [(1, 1, 1, 1, 1), (2, 31, 5, 2, 1), (1, 33, 64, 1, 4), (3, 64, 1, 2, 8),
                                       (2, 1500, 1, 2, 1), (1, 1500, 70, 2, 3), (1, 5000, 2, 1, 1), (2, 129, 257, 1, 2),
                                       (1, 700, 1025, 1, 1), (40, 100, 1, 2, 1)])
def test_cross_sizes(dq, B, T, n, H, G):
    k, v = _kv(T, B, T, H)
    q = _q(n, B, n, H * G)
    _check_cross(_cross(dq, q, k, v), q, k, v, [T] * B, [n] * B)


@pytest.mark.parametrize("n", [1, 40, 200])
def test_cross_lengths_and_masks(dq, n):
    """Every sequence its own length and mask, none among them; hidden states
    hold NaN and infinities."""
    B, T, H, G = 5, 530, 2, 2
    k, v = _kv(n, B, T, H)
    q = _q(n, B, n, H * G)
    lens, new = [530, 0, 1, 257, 100], [n, n, n, n // 2, n]
    mask = torch.rand((B, T), generator=torch.Generator().manual_seed(3)) < 0.7
    mask[4] = False
    mask[0, 64:128] = False
    dirty_k, dirty_v = k.clone(), v.clone()
    for b in range(B):
        hide = ~mask[b]
        hide[lens[b]:] = True
        at = hide.nonzero()[:, 0]
        for x in (dirty_k, dirty_v):
            x[b, at[0::3]] = math.nan
            x[b, at[1::3]] = math.inf
            x[b, at[2::3]] = -3e38
    for m in (mask, mask.to(torch.uint8) * 5):
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
        got = _cross(dq, q, dirty_k, dirty_v, lens, m, new, out=out)
        _check_cross(got, q, k, v, lens, new, mask)
        for b in range(B):
            assert bool((out[b, new[b]:] == 7.0).all())
    # mask rows of a wider tensor, and no mask
    wide = torch.zeros((B, T + 9), dtype=torch.bool, device=DEV)
    wide[:, 4:T + 4] = mask.to(DEV)
    out2 = torch.full_like(out, 7.0)
    dq.dq_cross_attention(q.to(DEV), dirty_k.to(DEV), dirty_v.to(DEV), kv_lens=_i32(lens), mask=wide[:, 4:T + 4],
                          q_lens=_i32(new), out=out2)
    assert torch.equal(out2, out)
    for x in (dirty_k, dirty_v):
        for b in range(B):
            x[b, :lens[b]] = (k if x is dirty_k else v)[b, :lens[b]]
    got = _cross(dq, q, dirty_k, dirty_v, lens, None, new)
    _check_cross(got, q, k, v, lens, new)


@pytest.mark.parametrize("B,T,n,H,G", [(1, 4100, 64, 8, 1), (1, 4100, 65, 1, 1), (2, 2500, 40, 3, 4)])
def test_cross_pieces(dq, B, T, n, H, G):
    """Sequences that are cut, pieces among them that the mask leaves nothing of."""
    k, v = _kv(n, B, T, H)
    q = _q(n, B, n, H * G)
    mask = torch.rand((B, T), generator=torch.Generator().manual_seed(5)) < 0.5
    mask[0, 300:1900] = False
    lens = [T - 40 * b for b in range(B)]
    for m in (None, mask):
        _check_cross(_cross(dq, q, k, v, lens, m), q, k, v, lens, [n] * B, m)
        _check_cross(_cross(dq, q, k, v, None, m), q, k, v, [T] * B, [n] * B, m)


@pytest.mark.parametrize("B,H,n,new", [(300, 2, 1, False), (90, 8, 2, False), (40, 3, 130, False), (140, 8, 70, True),
                                       (200, 1, 200, True), (520, 1, 3, True)])
def test_cross_one_long_sequence(dq, B, H, n, new):
    """Many short sequences and a few long ones, which are cut."""
    T = 9000
    k, v = _kv(B, 1, T, H)
    q = _q(n, B, n, H)
    r = np.random.default_rng(B)
    lens = r.integers(0, 120, B)
    lens[[3, B // 2, B - 1]] = [T, 5000, 4000]
    news = r.integers(0, n + 1, B) if new else np.full(B, n)
    news[[3, B - 1]] = n
    kd, vd = (x.to(DEV).expand(B, -1, -1, -1) for x in (k, v))
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    dq.dq_cross_attention(q.to(DEV), kd, vd, kv_lens=_i32(lens.tolist()), q_lens=_i32(news.tolist()) if new else None,
                          out=out)
    _check_cross(out, q, k.expand(B, -1, -1, -1), v.expand(B, -1, -1, -1), lens, news)
    for b in range(B):
        assert bool((out[b, int(news[b]):] == 7.0).all())


@pytest.mark.parametrize("n", [2, 90])
def test_cross_strides(dq, n):
    B, T, H, G = 2, 300, 2, 2
    k, v = _kv(n, B, T, H)
    q = _q(n, B, n, H * G).to(DEV)
    k, v = k.to(DEV), v.to(DEV)
    want = dq.dq_cross_attention(q, k, v)
    both = torch.stack([k, v], dim=3)                                    # [B, T, H, 2, 128]
    heads_first = [x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in (k, v)]
    odd = torch.zeros((2, B, T, H, 129), dtype=torch.bfloat16, device=DEV)
    odd[0, ..., 1:], odd[1, ..., 1:] = k, v
    for a, b in ((both[..., 0, :], both[..., 1, :]), heads_first, (odd[0, ..., 1:], odd[1, ..., 1:])):
        assert torch.equal(dq.dq_cross_attention(q, a, b), want)
    # sequences that share states
    shared = dq.dq_cross_attention(q, k[:1].expand(B, -1, -1, -1), v[:1].expand(B, -1, -1, -1))
    assert torch.equal(shared[0], want[0])
    assert torch.equal(shared[1], dq.dq_cross_attention(q[1:], k[:1], v[:1])[0])


def test_cross_extremes(dq):
    B, T, H = 1, 200, 1
    k, v = _kv(1, B, T, H)
    q = _q(1, B, 40, 1)
    none = dq.dq_cross_attention(q.to(DEV), k[:, :0].to(DEV), v[:, :0].to(DEV))
    assert bool((none == 0).all())
    assert dq.dq_cross_attention(q[:, :0].to(DEV), k.to(DEV), v.to(DEV)).shape == (1, 0, 1, 128)
    for scale in (0.0, -0.2, 2.0):
        _check_cross(_cross(dq, q, k, v, scale=scale), q, k, v, [T], [40], scale=scale)
    big = (v.float() * 2.0 ** 76).to(torch.bfloat16)
    out, want = _cross(dq, q, k, big), _cross(dq, q, k, v)
    assert torch.equal(out.float() * 2.0 ** -76, want.float())
    out = _cross(dq, q, k, v, scale=1e30)
    assert bool(torch.isfinite(out.float()).all())
    bad = q.clone()
    bad[0, 3, 0, 5] = math.nan
    out, clean = _cross(dq, bad, k, v), _cross(dq, q, k, v)
    keep = torch.arange(40) != 3
    assert bool(torch.isnan(out[0, 3]).all()) and torch.equal(out[0, keep], clean[0, keep])
    for x, y in ((k, v), (v, k)):
        dirty = x.clone()
        dirty[0, 150, 0, 9] = math.nan
        out = _cross(dq, q, dirty, v) if x is k else _cross(dq, q, k, dirty)
        assert bool(torch.isnan(out[0, :, 0, 9]).all())


@pytest.mark.parametrize("n", [40, 200])
def test_cross_infinities(dq, n):
    """What the formula gives: an infinite query or a score of +infinity NaN, a
    score of -infinity no weight, an infinite value itself."""
    k, v = _kv(1, 1, 200, 1)
    q = _q(1, 1, n, 1)
    q[0, 7, 0, 9] = 0
    clean = _cross(dq, q, k, v)
    for x in (math.inf, -math.inf):
        bad = q.clone()
        bad[0, 3, 0, 5] = x
        out = _cross(dq, bad, k, v)
        keep = torch.arange(n) != 3
        assert bool(torch.isnan(out[0, 3]).all()) and torch.equal(out[0, keep], clean[0, keep])
        zeros = _cross(dq, bad, k, v, [0])
        assert bool((zeros == 0).all())
        key, value = k.clone(), v.clone()
        key[0, 150, 0, 9], value[0, 150, 0, 9] = x, x
        out = _cross(dq, q, key, v)
        without = torch.arange(200)[None] != 150
        hidden = _cross(dq, q, k, v, None, without)
        none = ((q[0, :, 0, 9] * x) < 0)                  # (0 times infinity: NaN)
        assert bool(torch.isnan(out[0][~none]).all())
        # (another maximum than with the token hidden by the mask: close, not equal)
        assert bool(((out[0][none].double() - hidden[0][none].double()).norm(dim=-1)
                     <= 2.0 ** -6 * v.double().norm(dim=-1).max().item()).all())
        out = _cross(dq, q, k, value)
        assert bool((out[0, :, 0, 9] == x).all())
        rest = torch.arange(128) != 9
        assert torch.equal(out[..., rest], clean[..., rest])


def test_cross_graph(dq):
    B, T, n, H = 3, 700, 1, 2
    k, v = (x.to(DEV) for x in _kv(1, B, T, H))
    q = _q(1, B, n, H).to(DEV)
    lens = _i32([700, 20, 333])
    mask = torch.ones((B, T), dtype=torch.bool, device=DEV)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    need = dq.dq_chunk_workspace_bytes(B, n, H, H, T)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    call = lambda o: dq.dq_cross_attention(q, k, v, kv_lens=lens, mask=mask, out=o, workspace=ws)  # noqa: E731
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(4):
        q.copy_(_q(30 + i, B, n, H))
        lens.copy_(_i32([700 - 100 * i, 20 * i, 333 + i]))
        mask.copy_(torch.rand((B, T), device=DEV) < 0.5 + 0.1 * i)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros_like(out)
        call(want)
        assert torch.equal(out, want)


def test_cross_many_sequences_graph(dq):
    """20000 sequences that share states, captured: other lengths at every replay,
    and a workspace that holds NaN."""
    B, T = 20000, 2100
    k, v = _kv(2, 1, T, 1)
    q = _q(2, B, 1, 1)
    kd, vd, qd = k.to(DEV).expand(B, -1, -1, -1), v.to(DEV).expand(B, -1, -1, -1), q.to(DEV)
    kk, vv = (x[0].double().to(DEV).permute(1, 0, 2) for x in (k, v))
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    out = torch.zeros(q.shape, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(dq.dq_chunk_workspace_bytes(B, 1, 1, 1, T), dtype=torch.uint8, device=DEV)
    call = lambda: dq.dq_cross_attention(qd, kd, vd, kv_lens=lens, out=out, workspace=ws)  # noqa: E731
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    r = np.random.default_rng(1)
    for longest, most in ((T, 1), (T, T), (T, 40), (3, 3)):
        now = r.integers(0, most + 1, B)
        now[[0, 63, 64, 9000, B - 1]] = longest
        lens.copy_(_i32(now.tolist()))
        ws.fill_(255)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        see = torch.arange(T, device=DEV)[None] < lens[:, None]
        _check(out[:, 0], q[:, 0], kk, vv, see, 128 ** -0.5, 8)


# ------------------------------------------------------------- together

@pytest.mark.parametrize("fmt", FMTS)
def test_a_prompt_in_pieces_then_decode(dq, fmt):
    """Rotate, append, attend, piece by piece, then one decode step, as an engine
    does: the same as the whole prompt at once, and the formula's."""
    B, T, H, G = 2, 416, 2, 2
    k, v = _kv(17, B, T, H)
    q = _q(17, B, T, H * G)
    rope = dq.RotaryPositions(64, base=5000.0, scaling="linear", factor=2.0)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    cache = dq.Q8KVCache(B, H, H * G, 512, fmt)
    outs, t0 = [], 0
    for n in (160, 96, 32, 128):
        piece = slice(t0, t0 + n)
        qr, kr = rope.apply(q[:, piece].to(DEV), k[:, piece].to(DEV), starts=lens)
        cache.append(kr, v[:, piece].to(DEV), t0)
        lens += n
        outs.append(cache.attend_chunk(qr, lens))
        t0 += n
    qr, kr = rope.apply(q.to(DEV), k.to(DEV))
    whole = dq.Q8KVCache(B, H, H * G, 512, fmt)
    whole.append(kr, v.to(DEV), 0)
    for a, b in zip(cache.arrays, whole.arrays):
        assert torch.equal(a, b)
    out = torch.cat(outs, dim=1)
    _check_all(out, qr.cpu(), _held(kr.cpu(), fmt), _held(v, fmt), [T] * B, [T] * B)
    at_once = whole.attend_chunk(qr, lens)
    assert float((out.float() - at_once.float()).norm() / at_once.float().norm()) < 2.0 ** -7
    step = cache.attend(qr[:, -1].contiguous(), lens)
    assert float((step - out[:, -1].float()).norm() / step.norm()) < 2.0 ** -7
    # and the decoder's cross attention beside it, over states in BF16 and held as codes
    states = _kv(18, B, 100, H)
    a = dq.dq_cross_attention(qr, states[0].to(DEV), states[1].to(DEV))
    held = dq.Q8KVCache(B, H, H * G, 128, fmt)
    held.append(states[0].to(DEV), states[1].to(DEV), 0)
    b = held.attend_chunk(qr, _i32([100] * B), causal=False)
    _check_cross(a, qr.cpu(), *states, [100] * B, [T] * B)
    _check_all(b, qr.cpu(), _held(states[0], fmt), _held(states[1], fmt), [100] * B, [T] * B, causal=False)


def test_a_copied_cache(dq):
    k, v = _kv(19, 1, 200, 1)
    cache = _filled(dq, "int8", k, v, 2)
    q = _q(19, 1, 8, 2).to(DEV)
    want = cache.attend_chunk(q, _i32([200]))
    other = copy.deepcopy(cache)
    cache.k_data.zero_()
    assert torch.equal(other.attend_chunk(q, _i32([200])), want)
