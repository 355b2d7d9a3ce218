"""The 8-bit cache's argument checks (CPU): every unsupported or inconsistent
argument returns its error code or raises before anything is launched."""

import ctypes

import pytest
import torch

dq = pytest.importorskip("paper_2609_19880_amd")
from paper_2609_19880_amd import _lib  # noqa: E402

C = _lib._lib
INVALID, WORKSPACE, OK = dq.DQ_ERR_INVALID_ARG, dq.DQ_ERR_WORKSPACE, dq.DQ_OK
P = 4096            # an aligned address that no refused call touches


def _swap(args, changes):
    out = dict(args)
    out.update(changes)
    return list(out.values())


ENC = dict(f=0, k=P, ksb=0, kst=128, ksh=128, v=P, vsb=0, vst=128, vsh=128, B=2, H=8, t0=0, n=64, cap=256, kd=P, ks=P,
           vd=P, vs=P, st=None, stream=None)


@pytest.mark.parametrize("bad", [
    dict(f=2), dict(f=-1), dict(k=None), dict(v=None), dict(ksb=-1), dict(kst=-1), dict(ksh=-1), dict(vsb=-1),
    dict(vst=-1), dict(vsh=-1), dict(B=-1), dict(B=65536), dict(H=0), dict(H=65536), dict(t0=-32), dict(t0=16),
    dict(t0=224, n=33), dict(n=-1), dict(cap=0), dict(cap=96), dict(kd=None), dict(ks=None), dict(vd=None),
    dict(vs=None), dict(kd=P + 8), dict(vd=P + 4), dict(t0=0x7FFFFFE0, n=64)])
def test_encode_refusals(bad):
    assert C.dq_q8_encode_kv(*_swap(ENC, bad)) == INVALID
    a = dict(_swap_dict(ENC, bad))
    order = ["f", "kd", "ks", "vd", "vs", "B", "H", "t0", "n", "cap", "k", "ksb", "kst", "ksh", "v", "vsb", "vst", "vsh"]
    assert C.dq_q8_decode_kv(*[a[x] for x in order], None) == INVALID


def _swap_dict(args, changes):
    out = dict(args)
    out.update(changes)
    return out


def test_nothing_to_do_is_ok():
    assert C.dq_q8_encode_kv(*_swap(ENC, dict(B=0))) == OK
    assert C.dq_q8_encode_kv(*_swap(ENC, dict(n=0))) == OK


PAGES = [dict(bt=None), dict(mp=0), dict(page=64), dict(page=192), dict(page=1 << 21), dict(np=0),
         dict(mp=1 << 20, page=1 << 12)]


@pytest.mark.parametrize("bad", PAGES + [dict(t0=16), dict(t0=256, n=257), dict(f=3), dict(kd=P + 1)])
def test_paged_encode_refusals(bad):
    a = dict(f=0, k=P, ksb=0, kst=128, ksh=128, v=P, vsb=0, vst=128, vsh=128, B=2, H=8, t0=0, n=64, bt=P, mp=4,
             page=128, np=8, kd=P, ks=P, vd=P, vs=P, st=None, stream=None)
    assert C.dq_q8_encode_kv_paged(*_swap(a, bad)) == INVALID


STEP = dict(f=0, q=P, B=2, Hq=32, H=8, kd=P, ks=P, vd=P, vs=P, lens=P, extra=None, cap=256, w=0, s=0, scale=0.1,
            lse=None, ws=P, n=1 << 40, stream=None)


@pytest.mark.parametrize("bad,code", [
    (dict(f=2), INVALID), (dict(q=None), INVALID), (dict(B=0), INVALID), (dict(B=65536), INVALID),
    (dict(Hq=0), INVALID), (dict(Hq=12), INVALID), (dict(Hq=72), INVALID), (dict(H=0), INVALID),
    (dict(H=65536, Hq=65536), INVALID), (dict(kd=None), INVALID), (dict(ks=None), INVALID), (dict(vd=None), INVALID),
    (dict(vs=None), INVALID), (dict(kd=P + 8), INVALID), (dict(lens=None), INVALID), (dict(cap=0), INVALID),
    (dict(cap=160), INVALID), (dict(w=-1), INVALID), (dict(w=5, s=-1), INVALID), (dict(s=4), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(ws=None), WORKSPACE),
    (dict(n=1000), WORKSPACE)])
def test_step_refusals(bad, code):
    assert C.dq_q8_decode_attention_partial(*_swap(STEP, bad)) == code
    a = _swap_dict(STEP, bad)
    one = [a[x] for x in ("f", "q", "B", "Hq", "H", "kd", "ks", "vd", "vs", "lens", "cap", "w", "s", "scale")]
    assert C.dq_q8_decode_attention(*one, P, None, None, a["ws"], a["n"], None) == code
    if set(bad) <= {"B", "Hq", "H", "lens", "cap", "w", "s", "ws", "n"}:
        assert C.dq_q8_add_scores(a["B"], a["Hq"], a["H"], a["lens"], None, a["cap"], a["w"], a["s"], P, a["ws"],
                                  a["n"], P, None) == code


def test_step_needs_outputs():
    a = STEP
    one = [a[x] for x in ("f", "q", "B", "Hq", "H", "kd", "ks", "vd", "vs", "lens", "cap", "w", "s", "scale")]
    assert C.dq_q8_decode_attention(*one, None, None, None, P, 1 << 40, None) == INVALID
    assert C.dq_q8_decode_attention(*one, P, None, P, P, 1 << 40, None) == INVALID      # scores without their scratch
    assert C.dq_q8_add_scores(2, 32, 8, P, None, 256, 0, 0, None, P, 1 << 40, P, None) == INVALID
    assert C.dq_q8_add_scores(2, 32, 8, P, None, 256, 0, 0, P, P, 1 << 40, None, None) == INVALID


@pytest.mark.parametrize("bad", PAGES)
def test_paged_step_refusals(bad):
    a = dict(f=0, q=P, B=2, Hq=32, H=8, kd=P, ks=P, vd=P, vs=P, bt=P, mp=4, page=128, np=8, lens=P, extra=None, w=0,
             s=0, scale=0.1, lse=None, ws=P, n=1 << 40, st=None, stream=None)
    assert C.dq_q8_decode_attention_paged_partial(*_swap(a, bad)) == INVALID


EVICT = dict(B=2, H=8, lens=P, new=P, cap=512, to_cap=512, keep=256, first=32, last=32, kd=P, ks=P, vd=P, vs=P, sc=P,
             tkd=P, tks=P, tvd=P, tvs=P, tsc=P, kept=P, stream=None)
Q = 2 * P


@pytest.mark.parametrize("bad", [
    dict(B=0), dict(B=65536), dict(H=0), dict(lens=None), dict(new=None), dict(cap=0), dict(cap=500),
    dict(to_cap=96), dict(keep=250), dict(keep=0), dict(keep=1024), dict(first=-32), dict(first=16), dict(last=0),
    dict(last=40), dict(first=160, last=128), dict(kd=None), dict(ks=None), dict(vs=None), dict(sc=None),
    dict(tkd=None), dict(tsc=None), dict(kept=None), dict(kd=P + 8, tkd=P + 8),
    # in place only as a whole, and with one capacity
    dict(tkd=Q), dict(tkd=Q, tks=Q, tvd=Q, tvs=Q), dict(to_cap=256), dict(tsc=Q)])
def test_evict_refusals(bad):
    assert C.dq_q8_evict(*_swap(EVICT, bad)) == INVALID


@pytest.mark.parametrize("bad", PAGES + [dict(keep=33), dict(keep=1024), dict(last=0)])
def test_paged_evict_refusals(bad):
    a = dict(B=2, H=8, lens=P, new=P, keep=256, first=32, last=32, bt=P, mp=4, page=128, np=8, kd=P, ks=P, vd=P, vs=P,
             sc=P, kept=P, st=None, stream=None)
    assert C.dq_q8_evict_paged(*_swap(a, bad)) == INVALID


def test_python_refusals():
    """Shapes, types and devices that the binding turns away (host tensors: nothing can be launched)."""
    data, scale = torch.zeros((1, 2, 4, 4096), dtype=torch.uint8), torch.zeros((1, 2, 4))
    kv = torch.zeros((1, 32, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        dq.dq_q8_encode_kv("int4", kv, kv, 0, data, scale, data, scale)
    with pytest.raises(ValueError):
        dq.dq_q8_encode_kv("int8", kv, kv, 0, data, scale, data, scale)          # not on a GPU
    with pytest.raises(ValueError):
        dq.dq_q8_encode_kv("int8", kv, kv, 0, data[:, :, ::2], scale, data, scale)
    with pytest.raises(ValueError):
        dq.Q8KVCache(1, 2, 4, 100)
    with pytest.raises(ValueError):
        dq.Q8KVCache(1, 2, 4, 128, "fp4")
    with pytest.raises(ValueError):
        dq.StreamingKVCache(1, 2, 4, 256, None, None, streams="int4")
    with pytest.raises(ValueError):
        dq.StreamingKVCache(1, 2, 4, 256, object(), None, streams="int8", device="cpu")


def test_cache_on_the_host_keeps_shapes():
    c = dq.Q8KVCache(2, 2, 8, 256, "e4m3", scores=True, device="cpu")
    assert c.k_data.shape == (2, 2, 8, 4096) and c.scores.shape == (2, 2, 8) and c.block_lse.shape == (2, 2, 8, 4)
    assert c.cache_bytes(33) == 2 * 2 * 2 * 2 * 4100
    lens = torch.tensor([256, 256], dtype=torch.int32)
    with pytest.raises(ValueError):
        c.evict(lens, 100)
    with pytest.raises(ValueError):
        dq.Q8KVCache(2, 2, 8, 256, device="cpu").evict(lens, 128)
    assert ctypes.sizeof(ctypes.c_float) == 4


def test_workspace_alignment():
    assert C.dq_q8_decode_attention_partial(*_swap(STEP, dict(ws=P + 8))) == INVALID
    assert C.dq_q8_add_scores(2, 32, 8, P, None, 256, 0, 0, P, P + 4, 1 << 40, P, None) == INVALID


def test_cache_off_the_gpu_is_refused():
    c = dq.Q8KVCache(1, 2, 4, 256, scores=True, device="cpu")
    lens = torch.zeros(1, dtype=torch.int32)
    rows = torch.zeros((1, 32, 2, 128), dtype=torch.bfloat16)
    q = torch.zeros((1, 4, 128), dtype=torch.bfloat16)
    for call in (lambda: c.append(rows, rows, 0), lambda: c.read(0, 32), lambda: c.attend(q, lens),
                 lambda: c.partial(q, lens), lambda: c.evict(lens, 128)):
        with pytest.raises(ValueError, match="GPU"):
            call()


@pytest.mark.parametrize("bad,code", [
    (dict(B=0), INVALID), (dict(Hq=12), INVALID), (dict(H=0), INVALID), (dict(lens=None), INVALID),
    (dict(cap=160), INVALID), (dict(s=3), INVALID), (dict(lse=None), INVALID), (dict(ws=None), WORKSPACE),
    (dict(ws=P + 8), INVALID), (dict(n=1000), WORKSPACE), (dict(out=None), INVALID), (dict(out=P + 4), INVALID),
    (dict(sc=None), INVALID)])
def test_merge_scores_refusals(bad, code):
    a = dict(B=2, Hq=32, H=8, lens=P, extra=None, cap=256, w=0, s=0, lse=P, ws=P, n=1 << 40, out=P, sc=P, stream=None)
    assert C.dq_q8_merge_scores(*_swap(a, bad)) == code
