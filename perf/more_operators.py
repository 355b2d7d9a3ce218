"""From a prompt's projections to its attention, as timed cases: rotary
positions, attention of a chunk of new tokens over the 8-bit cache, and
cross attention.  ``kind`` names the call:

``rope``   queries and keys of a chunk are rotated by their positions: half or
           interleaved pairs, all of the head or its first ``rotary`` channels,
           frequencies scaled for long contexts; or rotated back (``back``).
``chunk``  the last ``new`` of a sequence's ``tokens`` cached tokens attend to
           the tokens up to themselves (``causal``; behind a ``window`` to the
           first ``sinks`` and their own newest ``window`` ones), over int8 or
           e4m3 codes with a scale per 32 tokens, contiguous or in pool pages;
           or (not ``causal``) ``new`` queries attend to all of them, as a
           decoder's tokens do to an encoder's states that the cache holds.
``cross``  ``new`` queries attend to ``tokens`` states of an encoder in BF16,
           each sequence of its own length, with or without a mask.

Head counts, batches and contexts are those of ``dq_workloads``, the tests and
the other timed cases or lie between them; so is the inputs' recipe (keys with
per-channel means, spreads and outlier channels; N(0, 1) queries and values).
"""

from __future__ import annotations

import math
import random

import torch

own = False

D = 128                 # head_dim
BLOCK = 32              # tokens that share a scale
QMAX = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -96       # a block whose largest magnitude is below is stored as zeros
ORIGINAL = 8192         # the context that scaled frequencies extend


def listed():
    return [
        # one decode step of one chat: launches only
        {"name": "rope_b1_n1", "kind": "rope", "batch": 1, "new": 1, "heads": 8, "group": 4, "rotary": 128,
         "layout": "half", "scaling": "none", "at": "starts", "back": False},
        # four long prompts of an odd length, far along in a context extended four times
        {"name": "rope_b4_t8k_yarn", "kind": "rope", "batch": 4, "new": 8171, "heads": 8, "group": 4, "rotary": 128,
         "layout": "half", "scaling": "yarn", "at": "starts", "back": False},
        # a batch of short drafts, every token with a position of its own, half of each head, rotated back
        {"name": "rope_b48_n33_pairs_back", "kind": "rope", "batch": 48, "new": 33, "heads": 8, "group": 4,
         "rotary": 64, "layout": "interleaved", "scaling": "bands", "at": "positions", "back": True},
        # four drafted tokens of one chat are checked
        {"name": "chunk_b1_n4_t4k_paged", "kind": "chunk", "fmt": "int8", "batch": 1, "new": 4, "tokens": 4092,
         "heads": 8, "group": 4, "page": 128, "causal": True},
        # eight beams over long encoder states that the cache holds, a full batch
        {"name": "held_b16_n8_t32k_e4m3", "kind": "chunk", "fmt": "e4m3", "batch": 16, "new": 8, "tokens": 32768,
         "heads": 8, "group": 4, "page": 0, "causal": False},
        # four whole prompts of an odd length
        {"name": "chunk_b4_n8k_t8k", "kind": "chunk", "fmt": "int8", "batch": 4, "new": 8171, "tokens": 8171,
         "heads": 8, "group": 4, "page": 0, "causal": True},
        # the last piece of a long prompt that is read in pieces
        {"name": "chunk_b1_n2k_t34k_paged_e4m3", "kind": "chunk", "fmt": "e4m3", "batch": 1, "new": 2048,
         "tokens": 34816, "heads": 8, "group": 4, "page": 256, "causal": True},
        # continuous batching: single tokens, drafts and pieces of prompts, sequences of every length in pool pages
        {"name": "chunk_b48_n512_t8k_ragged", "kind": "chunk", "fmt": "int8", "batch": 48, "new": 512,
         "tokens": 8192, "heads": 8, "group": 4, "page": 256, "causal": True, "ragged": True},
        # a piece of a long document behind a window, wide GQA
        {"name": "chunk_b2_n1k_t64k_window_e4m3", "kind": "chunk", "fmt": "e4m3", "batch": 2, "new": 1000,
         "tokens": 65473, "heads": 8, "group": 8, "page": 0, "causal": True, "window": 4096, "sinks": 4},
        # a decode step of a batch over its encoders' states, every head its own keys
        {"name": "cross_b32_n1_s1500", "kind": "cross", "batch": 32, "new": 1, "tokens": 1500, "heads": 8,
         "group": 1, "mask": False},
        # the decoder's prompts over states that padding and dropped frames leave holes in
        {"name": "cross_b8_n448_s1500_mask", "kind": "cross", "batch": 8, "new": 448, "tokens": 1500, "heads": 8,
         "group": 1, "mask": True},
        # long targets over long sources of an odd length
        {"name": "cross_b4_n4k_s8k", "kind": "cross", "batch": 4, "new": 4096, "tokens": 8171, "heads": 8,
         "group": 4, "mask": False},
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "chunk", "chunk", "chunk", "cross", "cross"])
    case = {"kind": kind, "heads": rng.choice([1, 2, 4, 8, 8, 8]), "group": rng.choice([1, 2, 3, 4, 4, 4, 6, 7, 8]),
            "batch": _log_int(rng, 1, 64)}
    hq = case["heads"] * case["group"]
    if kind == "rope":
        case["new"] = _log_int(rng, 1, (1 << 15) // case["batch"])
        case.update(rotary=rng.choice([32, 64, 96, 128, 128]), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "ntk", "bands", "yarn"]),
                    at=rng.choice(["starts", "positions"]), back=rng.random() < 0.3)
        return case
    # new x tokens up to a quarter of the largest listed case's
    pairs = (1 << 31) // (case["batch"] * hq)
    if kind == "cross":
        case["tokens"] = _log_int(rng, 1, min(8191, (1 << 18) // case["batch"]))
        case["new"] = _log_int(rng, 1, max(1, min(4096, pairs // case["tokens"], (1 << 17) // case["batch"])))
        case["mask"] = rng.random() < 0.5
        return case
    case["fmt"] = rng.choice(["int8", "e4m3"])
    case["tokens"] = _log_int(rng, 1, min(131072, (1 << 19) // case["batch"]))
    case["new"] = _log_int(rng, 1, max(1, min(8192, case["tokens"], pairs // case["tokens"],
                                              (1 << 17) // case["batch"])))
    case["page"] = rng.choice([0, 128, 256, 512])
    case["causal"] = rng.random() < 0.75
    if case["causal"] and rng.random() < 0.3:
        case["window"] = _log_int(rng, 1, 8192)
        case["sinks"] = rng.choice([0, 1, 4, 37, 64, 128])
    if rng.random() < 0.5:
        case["ragged"] = True
    return case


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Cached tokens and new tokens of each sequence, from the case alone: of a
    ragged batch the lengths are spread evenly up to `tokens`, the numbers of
    new tokens over their logarithm up to `new`."""
    B, T, N = case["batch"], case["tokens"], case["new"]
    if not case.get("ragged") or B == 1:
        return [(T, N)] * B
    out = []
    for b in range(B):
        n = int(round(N ** (((b * 5 + 3) % B) / (B - 1))))
        out.append((max(n, int(round(1 + (T - 1) * b / (B - 1)))), n))
    return out


def _keys(g, batch: int, tokens: int, heads: int) -> torch.Tensor:
    """bf16 [batch, tokens, heads, 128]: per-channel mean and spread, four
    channels of every head eight times as wide."""
    mu = torch.randn((heads, D), generator=g, device="cuda") * math.sqrt(2.0)
    sigma = torch.rand((heads, D), generator=g, device="cuda") * 1.5 + 0.5
    wide = torch.rand((heads, D), generator=g, device="cuda").argsort(dim=1)[:, :4]
    sigma.scatter_(1, wide, sigma.gather(1, wide) * 8.0)
    out = torch.empty((batch, tokens, heads, D), dtype=torch.bfloat16, device="cuda")
    for b in range(batch):
        out[b] = torch.randn((tokens, heads, D), generator=g, device="cuda").mul_(sigma).add_(mu)
    return out


def _normal(g, batch: int, tokens: int, heads: int) -> torch.Tensor:
    out = torch.empty((batch, tokens, heads, D), dtype=torch.bfloat16, device="cuda")
    for b in range(batch):
        out[b] = torch.randn((tokens, heads, D), generator=g, device="cuda")
    return out


def _inputs(case, seed):
    """Everything random of a case, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, N, H, kind = case["batch"], case["new"], case["heads"], case["kind"]
    x = {"q": _normal(g, B, N, H * case["group"])}
    if kind == "rope":
        x["k"] = _keys(g, B, N, H)
        if case["at"] == "starts":
            x["starts"] = torch.randint(4 * ORIGINAL - N, (B,), generator=g, device="cuda", dtype=torch.int32)
        else:
            x["positions"] = torch.randint(4 * ORIGINAL, (B, N), generator=g, device="cuda", dtype=torch.int32)
        return x
    T = case["tokens"]
    x["k"], x["v"] = _keys(g, B, T, H), _normal(g, B, T, H)
    lens = _lengths(case)
    if kind == "cross":
        # states from half of the longest length on, the longest full
        lens = [(T - (T // 2) * b // B, N) for b in range(B)]
        if case["mask"]:
            # dropped frames: one in ten, at random
            x["mask"] = torch.rand((B, T), generator=g, device="cuda") >= 0.1
    x["new"] = [n for _, n in lens]
    x["lens"] = torch.tensor([t for t, _ in lens], dtype=torch.int32, device="cuda")
    x["new_lens"] = torch.tensor(x["new"], dtype=torch.int32, device="cuda")
    if case.get("page"):
        pages = B * -(-T // case["page"])
        # pool pages in the order an engine has handed them out: any
        x["bt"] = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(B, -1).contiguous()
    return x


# ------------------------------------------------------- the plain forms

_BASE = 10000.0
_FACTOR = 4.0
_BANDS = (1.0, 4.0)     # turns over the original context: below the first all scaled, above the second none
_YARN = (1.0, 32.0)     # likewise, the ramp even over the pairs' indexes


def _frequencies(rotary: int, scaling: str):
    """Angles per token fp64 [rotary / 2], and the factor of the rotated values."""
    i = torch.arange(rotary // 2, dtype=torch.float64, device="cuda")
    base = _BASE * _FACTOR ** (rotary / (rotary - 2)) if scaling == "ntk" else _BASE
    f = base ** (-2.0 * i / rotary)
    if scaling == "linear":
        return f / _FACTOR, 1.0
    if scaling == "bands":
        keep = ((ORIGINAL * f / (2.0 * math.pi) - _BANDS[0]) / (_BANDS[1] - _BANDS[0])).clamp(0.0, 1.0)
        return f * keep + f / _FACTOR * (1.0 - keep), 1.0
    if scaling == "yarn":
        # the index of the pair that turns n times over the original context
        lo, hi = (rotary * math.log(ORIGINAL / (n * 2.0 * math.pi)) / (2.0 * math.log(_BASE)) for n in reversed(_YARN))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rotary - 1)
        keep = 1.0 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * keep + f / _FACTOR * (1.0 - keep), 0.1 * math.log(_FACTOR) + 1.0
    return f, 1.0


def _rotate(x, cos, sin, layout):
    """fp32 [B, N, H, D], cos and sin [B, N, rotary / 2]."""
    half = cos.shape[2]
    cos, sin = cos[:, :, None], sin[:, :, None]
    if layout == "half":
        a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], dim=3)
    a, b, rest = x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=4).flatten(3), rest], dim=3)


def _plain_rope(st):
    case = st["case"]
    freq, magnitude = st["freq"]
    if "positions" in st:
        at = st["positions"].double()
    else:
        at = st["starts"].double()[:, None] + torch.arange(case["new"], dtype=torch.float64, device="cuda")
    # angles in 64 bits: in 32 a far position's has lost its fraction
    angle = at[..., None] * freq
    cos, sin = (torch.cos(angle) * magnitude).float(), (torch.sin(angle) * magnitude).float()
    if case["back"]:
        sin = -sin
    return {n: _rotate(st[n].float(), cos, sin, case["layout"]).to(torch.bfloat16) for n in ("q", "k")}


def _quantise(x: torch.Tensor, fmt: str):
    """Codes as bytes [B, H, nb, 32, D] and scales fp32 [B, H, nb] of rows
    [B, T, H, D].  The scale is the block's largest magnitude over the type's,
    rounded to fp32; a code is the type's value nearest to x / scale, ties to
    even.  Both quotients are taken in 64 bits: in 32 they can land on a border
    between two codes."""
    B, T, H, _ = x.shape
    nb = -(-T // BLOCK)
    xb = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, nb * BLOCK - T)).view(B, nb, BLOCK, H, D).permute(0, 3, 1, 2, 4)
    amax = xb.abs().amax(dim=(3, 4)).double()
    scale = torch.where(amax >= TINY, amax / QMAX[fmt], 0.0).float()
    y = xb.double() / torch.where(scale > 0, scale, 1.0).double()[..., None, None]
    y = torch.where((scale > 0)[..., None, None], y, 0.0)
    if fmt == "int8":
        return torch.round(y).to(torch.int8).view(torch.uint8), scale
    # e4m3: three bits behind the leading one, from exponent -6 down steps of 2^-9
    _, e = torch.frexp(y)
    step = ((e.clamp(min=-5).long() + (1023 - 4)) << 52).view(torch.float64)
    return (torch.round(y / step) * step).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _floats(codes: torch.Tensor, scale: torch.Tensor, fmt: str) -> torch.Tensor:
    """fp32 values [..., nb * 32, D] of codes [..., nb, 32, D]."""
    c = codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()
    return (c * scale[..., None, None]).flatten(-3, -2)


def _sees(case, T: int, n: int, lo: int, hi: int, mask):
    """Truth values [hi - lo, T]: what queries lo .. hi of n see of T tokens."""
    t = torch.arange(T, device="cuda")[None]
    if not case.get("causal"):
        seen = t >= 0
        return (seen if mask is None else seen & mask[None, :T]).expand(hi - lo, T)
    p = (torch.arange(lo, hi, device="cuda") + (T - n))[:, None]
    seen = t <= p
    if case.get("window"):
        seen = seen & ((t < case["sinks"]) | (t > p - case["window"]))
    return seen


def _attention(case, q, k, v, mask):
    """fp32 q [n, Hq, D], k and v [H, T, D] -> bf16 [n, Hq, D]; a query that
    sees nothing gives zeros."""
    n, Hq, _ = q.shape
    H, T, _ = k.shape
    G = Hq // H
    out = torch.empty((n, Hq, D), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 29) // (Hq * T))          # rows at a time: 2 GB of scores
    for lo in range(0, n, step):
        hi = min(n, lo + step)
        qs = q[lo:hi].view(hi - lo, H, G, D).permute(1, 2, 0, 3).reshape(H, G * (hi - lo), D)
        seen = _sees(case, T, n, lo, hi, mask).repeat(G, 1)[None]
        s = torch.matmul(qs, k.transpose(1, 2)) * (1.0 / math.sqrt(D))
        s = torch.where(seen, s, -math.inf)
        top = s.amax(dim=2, keepdim=True)
        p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
        p = p / p.sum(dim=2, keepdim=True).clamp(min=1e-30)
        y = torch.matmul(p, v).view(H, G, hi - lo, D).permute(2, 0, 1, 3)
        out[lo:hi] = y.reshape(hi - lo, Hq, D).to(torch.bfloat16)
    return out


def _plain(st):
    case, kind = st["case"], st["case"]["kind"]
    if kind == "rope":
        return _plain_rope(st)
    outs = []
    for b, (T, n) in enumerate(zip(st["host_lens"], st["new"])):
        mask = None
        if kind == "cross":
            k, v = (st[x][b, :T].float().transpose(0, 1).contiguous() for x in ("k", "v"))
            mask = st["mask"][b] if "mask" in st else None
        else:
            kc, ks, vc, vs = st["cache"]
            if "bt" in st:
                bt = st["bt"][b].long()
                kc, ks, vc, vs = (x[bt].transpose(0, 1).flatten(1, 2) for x in (kc, ks, vc, vs))
            else:
                kc, ks, vc, vs = kc[b], ks[b], vc[b], vs[b]
            nb = -(-T // BLOCK)
            k = _floats(kc[:, :nb], ks[:, :nb], case["fmt"])[:, :T]
            v = _floats(vc[:, :nb], vs[:, :nb], case["fmt"])[:, :T]
        outs.append(_attention(case, st["q"][b, :n].float(), k, v, mask))
    return outs


def prepare(case, seed):
    x = _inputs(case, seed)
    kind, B = case["kind"], case["batch"]
    st = {"case": case, **{n: x[n] for n in x if n not in ("k", "v")}}
    if own:
        import paper_2609_19880_amd as dq
        st["dq"] = dq
    if kind == "rope":
        st["k"] = x["k"]
        if own:
            # the plan that a user's program makes once: the table of frequencies
            extra = {"none": {}, "linear": {"factor": _FACTOR}, "ntk": {"factor": _FACTOR},
                     "bands": {"factor": _FACTOR, "original": ORIGINAL, "turns": _BANDS},
                     "yarn": {"factor": _FACTOR, "original": ORIGINAL, "turns": _YARN}}[case["scaling"]]
            st["rope"] = dq.RotaryPositions(case["rotary"], base=_BASE, layout=case["layout"],
                                            scaling=case["scaling"], **extra)
        else:
            st["freq"] = _frequencies(case["rotary"], case["scaling"])
        return st
    st["host_lens"] = x["lens"].tolist()
    if kind == "cross":
        st["k"], st["v"] = x["k"], x["v"]
        return st
    T, H, fmt = case["tokens"], case["heads"], case["fmt"]
    Hq, nb, page = H * case["group"], -(-T // BLOCK), case["page"]
    if own:
        # the cache that a user's program holds before the call, filled by the
        # framework's encoder from the same keys and values
        if page:
            shape = (B * -(-T // page), H, page // BLOCK)
            data = [torch.zeros((*shape, BLOCK * D), dtype=torch.uint8, device="cuda") for _ in range(2)]
            scales = [torch.zeros(shape, dtype=torch.float32, device="cuda") for _ in range(2)]
            dq.dq_q8_encode_kv_paged(fmt, x["k"], x["v"], 0, st["bt"], data[0], scales[0], data[1], scales[1])
            st["pools"] = (data[0], scales[0], data[1], scales[1])
        else:
            st["cache"] = dq.Q8KVCache(B, H, Hq, -(-T // 128) * 128, fmt)
            st["cache"].append(x["k"], x["v"], 0)
        return st
    mp = -(-T // page) if page else 0
    rows = (B * mp, H, page // BLOCK) if page else (B, H, nb)
    cache = [torch.zeros((*rows, *rest), dtype=dtype, device="cuda")
             for rest, dtype in 2 * [((BLOCK, D), torch.uint8), ((), torch.float32)]]
    for b in range(B):
        for i, name in ((0, "k"), (2, "v")):
            for part, to in zip(_quantise(x[name][b:b + 1], fmt), (cache[i], cache[i + 1])):
                if page:
                    full = torch.zeros((H, mp * (page // BLOCK), *part.shape[3:]), dtype=part.dtype, device="cuda")
                    full[:, :nb] = part[0]
                    to[st["bt"][b].long()] = full.unflatten(1, (mp, -1)).transpose(0, 1)
                else:
                    to[b] = part[0]
    st["cache"] = cache
    return st


def run(state):
    if not own:
        return _plain(state)
    case, dq = state["case"], state["dq"]
    kind = case["kind"]
    if kind == "rope":
        q, k = state["rope"].apply(state["q"], state["k"], positions=state.get("positions"),
                                   starts=state.get("starts"), transposed=case["back"])
        return {"q": q, "k": k}
    if kind == "cross":
        out = dq.dq_cross_attention(state["q"], state["k"], state["v"], kv_lens=state["lens"], mask=state.get("mask"))
    else:
        new = state["new_lens"] if case.get("ragged") else None
        see = {"causal": case["causal"], "window": case.get("window", 0), "sinks": case.get("sinks", 0)}
        if case["page"]:
            out = dq.dq_q8_chunk_attention_paged(case["fmt"], state["q"], *state["pools"], state["bt"],
                                                 state["lens"], q_lens=new, **see)
        else:
            out = state["cache"].attend_chunk(state["q"], state["lens"], q_lens=new, **see)
    # a sequence's own rows (those behind them are nobody's)
    return [out[b, :n] for b, n in enumerate(state["new"])]


def work(case):
    B, N, H, kind = case["batch"], case["new"], case["heads"], case["kind"]
    Hq = H * case["group"]
    if kind == "rope":
        n = B * N * (Hq + H)
        return {"bytes": 2 * n * D * 2 + 4 * (B if case["at"] == "starts" else B * N), "flops": n * case["rotary"] * 3}
    nbytes = flops = 0
    if kind == "cross":
        for b in range(B):
            T = case["tokens"] - (case["tokens"] // 2) * b // B
            nbytes += 2 * T * H * D * 2 + (T if case["mask"] else 0) + 2 * N * Hq * D * 2
            flops += N * Hq * T * D * 4 * (0.9 if case["mask"] else 1.0)
        return {"bytes": nbytes, "flops": flops}
    per_token = 2 * H * (D + 4 / BLOCK)          # codes and scales of keys and values
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    for T, n in _lengths(case):
        tokens, pairs = T, n * T
        if case["causal"]:
            pairs = n * T - n * (n - 1) // 2
            if window:
                tokens = min(T, window + n - 1 + sinks)
                pairs = sum(min(p + 1, window + min(sinks, max(0, p + 1 - window))) for p in range(T - n, T))
        nbytes += tokens * per_token + 2 * n * Hq * D * 2
        flops += pairs * Hq * D * 4
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------------- exact
#
# The same in 64 bits, one sequence and head at a time, from the definition:
# a rotation is a complex product, the grid of a type is listed and a code is
# looked up between the midpoints, what a query sees is its list of tokens.

def _grid(fmt: str) -> torch.Tensor:
    if fmt == "int8":
        g = [float(i) for i in range(128)]
    else:
        g = [m * 2.0 ** -9 for m in range(8)]
        g += [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
        g = g[:127]                               # the last pattern is no number
    return torch.tensor(g, dtype=torch.float64, device="cuda")


def _held(x: torch.Tensor, fmt: str):
    """What the cache holds of one sequence x [T, H, D]: values fp64 [H, T, D]."""
    T, H, _ = x.shape
    nb = -(-T // BLOCK)
    y = torch.zeros((H, nb * BLOCK, D), dtype=torch.float64, device="cuda")
    y[:, :T] = x.double().transpose(0, 1)
    y = y.view(H, nb, BLOCK * D)
    top = y.abs().max(dim=2).values
    s = (top / QMAX[fmt]).float().double() * (top >= TINY)
    grid = _grid(fmt)
    mid = (grid[1:] + grid[:-1]) / 2
    for h in range(H):
        z = y[h] / torch.where(s[h] > 0, s[h], 1.0)[:, None]
        a = z.abs()
        lo, hi = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
        # on a midpoint the two differ by one: the even pattern
        y[h] = torch.copysign(grid[torch.where(lo % 2 == 0, lo, hi)], z) * s[h][:, None]
    return y.view(H, nb * BLOCK, D)[:, :T]


def _exact_rope(case, x):
    B, N, r = case["batch"], case["new"], case["rotary"]
    angles, magnitude = [], 1.0
    for i in range(r // 2):
        f = _BASE ** (-2.0 * i / r)
        if case["scaling"] == "linear":
            f /= _FACTOR
        elif case["scaling"] == "ntk":
            f = (_BASE * _FACTOR ** (r / (r - 2.0))) ** (-2.0 * i / r)
        elif case["scaling"] == "bands":
            turns = ORIGINAL * f / (2.0 * math.pi)
            w = min(1.0, max(0.0, (turns - _BANDS[0]) / (_BANDS[1] - _BANDS[0])))
            f = w * f + (1.0 - w) * f / _FACTOR
        elif case["scaling"] == "yarn":
            pair = lambda n: r * math.log(ORIGINAL / (2.0 * math.pi * n)) / (2.0 * math.log(_BASE))  # noqa: E731
            first = max(0, math.floor(pair(_YARN[1])))
            last = min(r - 1, math.ceil(pair(_YARN[0])))
            w = min(1.0, max(0.0, (i - first) / max(last - first, 0.001)))
            f = (1.0 - w) * f + w * f / _FACTOR
            magnitude = 1.0 + 0.1 * math.log(_FACTOR)
        angles.append(f)
    at = x["positions"] if "positions" in x else x["starts"][:, None] + torch.arange(N, device="cuda")
    angle = at.double()[:, :, None] * torch.tensor(angles, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(angle, magnitude), -angle if case["back"] else angle)[:, :, None]
    got = {}
    for name in ("q", "k"):
        y = x[name].double().clone()
        if case["layout"] == "half":
            z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
            y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
        else:
            z = torch.view_as_complex(y[..., :r].unflatten(3, (r // 2, 2)).contiguous()) * turn
            y[..., :r] = torch.view_as_real(z).flatten(3)
        got[name] = y
    return got


def exact(case, seed):
    x = _inputs(case, seed)
    kind = case["kind"]
    if kind == "rope":
        return _exact_rope(case, x)
    outs = []
    H, G = case["heads"], case["group"]
    for b, (T, n) in enumerate(zip(x["lens"].tolist(), x["new"])):
        if kind == "cross":
            k, v = (x[name][b, :T].double().transpose(0, 1) for name in ("k", "v"))
        else:
            # (blocks that end behind the length were encoded with the tokens there)
            k, v = (_held(x[name][b], case["fmt"])[:, :T] for name in ("k", "v"))
        out = torch.zeros((n, H * G, D), dtype=torch.float64, device="cuda")
        step = max(1, (1 << 28) // T)
        for h in range(H):
            for g in range(h * G, (h + 1) * G):
                for lo in range(0, n, step):
                    hi = min(n, lo + step)
                    s = x["q"][b, lo:hi, g].double() @ k[h].T / math.sqrt(D)
                    if kind == "cross" and case["mask"]:
                        s[:, ~x["mask"][b, :T]] = -math.inf
                    if case.get("causal"):
                        t = torch.arange(T, device="cuda")
                        for_row = torch.arange(lo, hi, device="cuda")[:, None] + T - n
                        hidden = t > for_row
                        if case.get("window"):
                            hidden |= (t >= case["sinks"]) & (t <= for_row - case["window"])
                        s[hidden] = -math.inf
                    s = torch.softmax(s, dim=1).nan_to_num(nan=0.0)   # rows that see nothing
                    out[lo:hi, g] = s @ v[h]
        outs.append(out)
    return outs
