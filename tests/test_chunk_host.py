"""Argument checks of the rotary positions, the chunk attention and the cross
attention, and the frequencies (CPU): every unsupported or inconsistent argument
returns its error code or raises before anything is launched."""

import math

import numpy as np
import pytest
import torch

dq = pytest.importorskip("paper_2609_19880_amd")
from paper_2609_19880_amd import _lib  # noqa: E402

C = _lib._lib
INVALID, WORKSPACE, OK = dq.DQ_ERR_INVALID_ARG, dq.DQ_ERR_WORKSPACE, dq.DQ_OK
P = 4096            # an aligned address that no refused call touches
BIG = 1 << 30       # a workspace size that is enough


def _with(args, changes):
    out = dict(args)
    assert set(changes) <= set(out)
    out.update(changes)
    return list(out.values())


ROPE = dict(layout=0, tr=0, freq=P, mag=1.0, r=128, d=128, B=2, T=5, q=P, qsb=5 * 4096, qst=4096, qsh=128, Hq=32, qo=P,
            qosb=5 * 4096, qost=4096, qosh=128, k=2 * P, ksb=5 * 1024, kst=1024, ksh=128, Hkv=8, ko=2 * P, kosb=5 * 1024,
            kost=1024, kosh=128, pos=None, psb=0, pst=0, starts=None, t0=0, stream=None)


@pytest.mark.parametrize("bad", [
    dict(layout=2), dict(layout=-1), dict(tr=2), dict(tr=-1), dict(freq=None), dict(mag=math.nan), dict(mag=math.inf), dict(r=0),
    dict(r=127), dict(r=130), dict(r=-2), dict(d=126), dict(d=1025), dict(B=-1), dict(T=-1), dict(B=1 << 14, T=1 << 13),
    dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(Hq=-1), dict(Hq=65536), dict(Hkv=0), dict(Hq=0),
    dict(qsb=-1), dict(qst=-1), dict(qsh=-1), dict(ksb=-1), dict(kst=-1), dict(ksh=-1), dict(qosb=-1), dict(kost=-1),
    dict(qosb=0), dict(qost=0), dict(qosh=0), dict(qosh=64), dict(kost=512), dict(kosb=1024), dict(pos=P, starts=P),
    dict(pos=P, t0=1), dict(pos=P, psb=-1), dict(pos=P, pst=-1),
    dict(Hq=0, q=None, qo=None, Hkv=0, k=None, ko=None),
    # a result over the other's input or result
    dict(k=P), dict(ko=P), dict(qo=2 * P), dict(k=3 * P, ko=P), dict(k=P, ko=3 * P),
    # in place the strides have to be the same
    dict(qsh=256, qosh=128), dict(ksb=0, kosb=5 * 1024), dict(qosb=1 << 62)])
def test_rope_refusals(bad):
    assert C.dq_rope(*_with(ROPE, bad)) == INVALID


def test_nothing_to_do_is_ok():
    assert C.dq_rope(*_with(ROPE, dict(B=0))) == OK
    assert C.dq_rope(*_with(ROPE, dict(T=0))) == OK
    assert C.dq_q8_chunk_attention(*_with(CHUNK, dict(B=0))) == OK
    assert C.dq_q8_chunk_attention(*_with(CHUNK, dict(n=0))) == OK
    assert C.dq_cross_attention(*_with(CROSS, dict(B=0))) == OK
    assert C.dq_cross_attention(*_with(CROSS, dict(n=0))) == OK


def _frequencies(**changes):
    a = dict(scaling=4, r=128, base=1e4, factor=4.0, original=8192.0, lo=1.0, hi=32.0)
    freq = np.zeros(512)
    mag = np.zeros(1)
    return C.dq_rope_frequencies(*_with(a, changes), freq.ctypes.data, mag.ctypes.data)


@pytest.mark.parametrize("bad", [
    dict(scaling=5), dict(scaling=-1), dict(r=0), dict(r=3), dict(r=1026), dict(base=0.0), dict(base=-1.0), dict(base=1.0),
    dict(base=math.inf), dict(factor=0.5), dict(factor=math.nan), dict(original=0.0), dict(original=math.inf), dict(lo=0.0),
    dict(lo=32.0), dict(hi=0.5), dict(hi=math.inf), dict(scaling=2, r=2), dict(scaling=3, lo=5.0, hi=4.0),
    dict(scaling=1, factor=0.0)])
def test_frequency_refusals(bad):
    assert _frequencies(**bad) == INVALID


def test_frequency_pointers():
    assert C.dq_rope_frequencies(0, 128, 1e4, 1.0, 0.0, 0.0, 0.0, None, np.zeros(1).ctypes.data) == INVALID
    assert C.dq_rope_frequencies(0, 128, 1e4, 1.0, 0.0, 0.0, 0.0, np.zeros(64).ctypes.data, None) == INVALID


def _close(got, want):
    # (two power functions, each off by an ulp or two of 2^-52, a product and a quotient)
    assert np.allclose(got, want, rtol=2.0 ** -48, atol=0)


@pytest.mark.parametrize("r", [2, 4, 64, 96, 128, 1024])
def test_frequencies(r):
    i = np.arange(r // 2)
    f = 10000.0 ** (-2.0 * i / r)
    got, m = dq.dq_rope_frequencies(r)
    _close(got, f)
    assert m == 1.0
    got, m = dq.dq_rope_frequencies(r, scaling="linear", factor=8.0)
    _close(got, f / 8)
    assert m == 1.0
    if r > 2:
        # by definition the lowest frequency is the linear one, the highest stays
        got, m = dq.dq_rope_frequencies(r, scaling="ntk", factor=8.0)
        assert got[0] == 1.0 and abs(got[-1] / (f[-1] / 8) - 1) < 1e-12 and m == 1.0
    got, m = dq.dq_rope_frequencies(r, scaling="bands", factor=8.0, original=8192, turns=(1.0, 4.0))
    turns = 8192 * f / (2 * math.pi)
    _close(got[turns >= 4], f[turns >= 4])
    _close(got[turns <= 1], f[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 4)
    assert ((got[mid] < f[mid]) & (got[mid] > f[mid] / 8)).all() and m == 1.0
    got, m = dq.dq_rope_frequencies(r, scaling="yarn", factor=8.0, original=8192, turns=(1.0, 32.0))
    assert abs(m - (0.1 * math.log(8.0) + 1)) < 1e-15
    j = lambda n: r * math.log(8192 / (2 * math.pi * n)) / (2 * math.log(10000.0))  # noqa: E731
    lo, hi = math.floor(j(32.0)), math.ceil(j(1.0))
    _close(got[i <= max(lo, 0)], f[i <= max(lo, 0)])
    _close(got[i >= hi], f[i >= hi] / 8)
    assert (np.diff(got / f) <= 1e-15).all()
    # a factor of 1 changes nothing
    for s in ("linear", "bands", "yarn"):
        got, m = dq.dq_rope_frequencies(r, scaling=s, factor=1.0, original=8192)
        _close(got, f)
        assert m == 1.0


CHUNK = dict(f=0, q=P, qsb=16 * 4096, qst=4096, qsh=128, B=2, n=16, Hq=32, H=8, kd=P, ks=P, vd=P, vs=P, qlens=None, lens=P,
             cap=4096, causal=1, window=0, sinks=0, scale=0.1, out=P, osb=16 * 4096, ost=4096, osh=128, ws=P, wsb=BIG,
             stream=None)
STEP = [dict(f=2), dict(f=-1), dict(q=None), dict(qsb=-1), dict(qst=-1), dict(qsh=-1), dict(B=-1), dict(B=65536), dict(n=-1),
        dict(Hq=0), dict(Hq=12), dict(H=0), dict(H=65536, Hq=65536), dict(kd=None), dict(ks=None), dict(vd=None),
        dict(vs=None), dict(kd=P + 8), dict(vd=P + 4), dict(lens=None), dict(causal=2), dict(causal=-1), dict(window=-1),
        dict(sinks=-1, window=4), dict(sinks=1), dict(causal=0, window=8), dict(scale=math.nan), dict(scale=math.inf),
        dict(out=None), dict(osb=-1), dict(ost=-1), dict(osh=-1), dict(osb=0), dict(ost=0), dict(osh=0), dict(osh=127),
        dict(n=1 << 22, Hq=32), dict(B=65535, H=128, Hq=128, n=1, osb=128 * 128, ost=128 * 128), dict(ws=P + 8)]


@pytest.mark.parametrize("bad", STEP + [dict(cap=0), dict(cap=100), dict(cap=-128)])
def test_chunk_refusals(bad):
    assert C.dq_q8_chunk_attention(*_with(CHUNK, bad)) == INVALID


@pytest.mark.parametrize("bad", STEP + [dict(bt=None), dict(mp=0), dict(page=64), dict(page=192), dict(np=0),
                                        dict(mp=1 << 20, page=1 << 12)])
def test_paged_chunk_refusals(bad):
    a = dict(CHUNK)
    keys = list(a)
    at = keys.index("qlens")
    order = keys[:at] + ["bt", "mp", "page", "np"] + [x for x in keys[at:-1] if x != "cap"] + ["status", "stream"]
    a.update(bt=P, mp=32, page=128, np=64, status=None)
    a.update(bad)
    assert C.dq_q8_chunk_attention_paged(*[a[x] for x in order]) == INVALID


CROSS = dict(q=P, qsb=16 * 4096, qst=4096, qsh=128, B=2, n=16, Hq=32, H=8, k=P, ksb=4096 * 1024, kst=1024, ksh=128, v=P,
             vsb=4096 * 1024, vst=1024, vsh=128, T=4096, qlens=None, lens=None, mask=None, msb=0, scale=0.1, out=P,
             osb=16 * 4096, ost=4096, osh=128, ws=P, wsb=BIG, stream=None)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(qsb=-1), dict(qst=-1), dict(qsh=-1), dict(B=-1), dict(B=65536), dict(n=-1), dict(Hq=0), dict(Hq=12),
    dict(H=0), dict(H=65536, Hq=65536), dict(k=None), dict(v=None), dict(ksb=-1), dict(kst=-1), dict(ksh=-1), dict(vsb=-1),
    dict(vst=-1), dict(vsh=-1), dict(T=-1), dict(T=(1 << 30) + 1), dict(mask=P, msb=-1), dict(scale=math.nan), dict(out=None),
    dict(osb=-1), dict(osb=0), dict(ost=0), dict(osh=100), dict(n=1 << 22, Hq=32), dict(ws=P + 4)])
def test_cross_refusals(bad):
    assert C.dq_cross_attention(*_with(CROSS, bad)) == INVALID


def test_workspaces():
    need = C.dq_chunk_workspace_bytes(2, 16, 32, 8, 4096)
    assert need > 0
    for f, a in ((C.dq_q8_chunk_attention, CHUNK), (C.dq_cross_attention, CROSS)):
        assert f(*_with(a, dict(wsb=need - 1))) == WORKSPACE
        assert f(*_with(a, dict(ws=None))) == WORKSPACE
    for args in ((-1, 16, 32, 8, 4096), (2, -1, 32, 8, 4096), (2, 16, 12, 8, 4096), (2, 16, 32, 0, 4096), (2, 16, 32, 8, -1),
                 (0, 16, 32, 8, 4096), (2, 0, 32, 8, 4096), (65536, 16, 32, 8, 4096)):
        assert C.dq_chunk_workspace_bytes(*args) == 0
    # a few MB whatever the sizes are: it holds what the GPU works on at a time
    assert C.dq_chunk_workspace_bytes(64, 4096, 64, 8, 1 << 20) < (1 << 28)
    assert C.dq_chunk_workspace_bytes(1, 1, 8, 8, 128) == 0


def test_binding_checks():
    """What the binding itself refuses needs no GPU: every tensor is on the CPU."""
    q = torch.zeros((1, 4, 8, 128), dtype=torch.bfloat16)
    k = torch.zeros((1, 4, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        dq.dq_cross_attention(q, k, k)
    with pytest.raises(ValueError, match="GPU"):
        dq.dq_rope(torch.ones(64, dtype=torch.float64), q, k)
    with pytest.raises(ValueError, match="layout"):
        dq.dq_rope(torch.ones(64, dtype=torch.float64), q, k, layout="both")
    with pytest.raises(ValueError, match="layout"):
        dq.RotaryPositions(128, layout="both", device="cpu")
    with pytest.raises(ValueError, match="scaling"):
        dq.RotaryPositions(128, scaling="longer", device="cpu")
    with pytest.raises(ValueError, match="rotary_dim"):
        dq.RotaryPositions(0, device="cpu")
    with pytest.raises(dq.DqError):
        dq.RotaryPositions(127, device="cpu")
    rope = dq.RotaryPositions(64, scaling="yarn", factor=4.0, original=4096, device="cpu")
    assert rope.freq.dtype == torch.float64 and rope.freq.shape == (32,) and rope.magnitude > 1
    assert dq.RotaryPositions(64, scaling="yarn", factor=4.0, original=4096, magnitude=1.0, device="cpu").magnitude == 1.0
    cache = dq.Q8KVCache(1, 2, 8, 128, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        cache.attend_chunk(q, torch.zeros(1, dtype=torch.int32))


@pytest.mark.gpu
def test_binding_checks_on_the_gpu():
    dev = "cuda"
    q = torch.zeros((2, 4, 8, 128), dtype=torch.bfloat16, device=dev)
    k = torch.zeros((2, 40, 2, 128), dtype=torch.bfloat16, device=dev)
    lens = torch.full((2,), 40, dtype=torch.int32, device=dev)
    cache = dq.Q8KVCache(2, 2, 8, 128)
    cache.append(k, k, 0)
    for bad in (q.float(), q[0], q[:1], q[..., :64], q.transpose(2, 3), q.cpu(), q[:, :, :7]):
        with pytest.raises(ValueError):
            cache.attend_chunk(bad, lens)
        with pytest.raises(ValueError):
            dq.dq_cross_attention(bad, k, k)
    for bad in (lens.long(), lens[:1], lens.cpu(), lens.repeat(2)[::2]):
        with pytest.raises(ValueError):
            cache.attend_chunk(q, bad)
        with pytest.raises(ValueError):
            cache.attend_chunk(q, lens, q_lens=bad)
        with pytest.raises(ValueError):
            dq.dq_cross_attention(q, k, k, kv_lens=bad)
    for bad in (q.float(), q[:, :3], torch.zeros_like(q).transpose(1, 2), q.cpu()):
        with pytest.raises(ValueError):
            cache.attend_chunk(q, lens, out=bad)
    with pytest.raises(dq.DqError):
        cache.attend_chunk(q, lens, out=torch.zeros((1, 4, 8, 128), dtype=torch.bfloat16, device=dev).expand(2, 4, 8, 128))
    for kw in (dict(window=-1), dict(sinks=-1), dict(window=1 << 31)):
        with pytest.raises(ValueError):
            cache.attend_chunk(q, lens, **kw)
    for kw in (dict(sinks=3), dict(causal=False, window=9), dict(softmax_scale=math.nan)):
        with pytest.raises(dq.DqError):
            cache.attend_chunk(q, lens, **kw)
    for bad in (k.float(), k[:, :39], k[..., :64], k.cpu(), k.transpose(1, 2)):
        with pytest.raises(ValueError):
            dq.dq_cross_attention(q, k, bad)
    for bad in (torch.ones((2, 39), dtype=torch.bool, device=dev), torch.ones((2, 40), device=dev),
                torch.ones((2, 40), dtype=torch.bool), torch.ones((2, 80), dtype=torch.bool, device=dev)[:, ::2]):
        with pytest.raises(ValueError):
            dq.dq_cross_attention(q, k, k, mask=bad)
    rope = dq.RotaryPositions(128)
    pos = torch.zeros((2, 4), dtype=torch.int32, device=dev)
    for a, kw in (((q.float(),), {}), ((None, None), {}), ((q, k), {}), ((q,), dict(positions=pos.long())),
                  ((q,), dict(positions=pos[:, :3])), ((q,), dict(positions=pos, t0=3)),
                  ((q,), dict(positions=pos, starts=lens)), ((q,), dict(starts=lens[:1])), ((q,), dict(q_out=q.float())),
                  ((q,), dict(q_out=q[:, :3])), ((q.transpose(2, 3),), {}), ((q,), dict(t0=1 << 31))):
        with pytest.raises(ValueError):
            rope.apply(*a, **kw)
    # in place needs the same strides, and an output no shared addresses
    with pytest.raises(dq.DqError):
        rope.apply(q.transpose(0, 1)[:2, :2], q_out=q[:, :2])
    with pytest.raises(dq.DqError):
        rope.apply(q, q_out=torch.zeros((1, 4, 8, 128), dtype=torch.bfloat16, device=dev).expand(2, 4, 8, 128))
    with pytest.raises(dq.DqError):
        dq.RotaryPositions(256).apply(q)


@pytest.mark.parametrize("r", [2, 4, 6, 32, 64, 96, 128, 250, 1024])
@pytest.mark.parametrize("base", [1e4, 5e5, 10.0, 0.5])
@pytest.mark.parametrize("factor,original,turns", [(8.0, 8192.0, (1.0, 4.0)), (40.0, 4096.0, (1.0, 32.0)), (1.5, 64.0, (0.25, 30.0)),
                                                   (3.0, 1e6, (2.0, 2.5)), (2.0, 5.0, (1.0, 32.0)), (4.0, 1e9, (1.0, 32.0))])
def test_mixed_frequencies(r, base, factor, original, turns):
    """The two mixtures at every index, from the formulas alone.  A weight's ramp has
    slope up to 1000 in its variable (the ends are at least 0.001 apart), whose
    own error is a few of 2^-53 of numbers up to 2^10 (indexes) or of turns / (high -
    low); both are far below 2^-30."""
    i = np.arange(r // 2)
    f = np.array([base ** (-2.0 * x / r) for x in i])
    low, high = turns
    w = (original * f / (2 * math.pi) - low) / (high - low)
    w = np.where(w < 0, 0.0, np.where(w > 1, 1.0, w))
    got, m = dq.dq_rope_frequencies(r, base=base, scaling="bands", factor=factor, original=original, turns=turns)
    assert m == 1.0 and np.allclose(got, w * f + (1 - w) * f / factor, rtol=2.0 ** -30, atol=0)
    j = lambda n: r * math.log(original / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
    ends = sorted([min(max(math.floor(j(high)), 0), r - 1), min(max(math.ceil(j(low)), 0), r - 1)])
    if j(high) <= j(low):
        got, m = dq.dq_rope_frequencies(r, base=base, scaling="yarn", factor=factor, original=original, turns=turns)
        span = max(ends[1] - ends[0], 0.001)
        w = np.array([1 - min(max((x - ends[0]) / span, 0.0), 1.0) for x in i])
        assert abs(m - (0.1 * math.log(factor) + 1)) < 1e-15
        assert np.allclose(got, w * f + (1 - w) * f / factor, rtol=2.0 ** -30, atol=0)
