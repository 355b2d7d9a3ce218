"""The 8-bit KV cache as timed cases: its encoder, its attention, its eviction.

A block is 32 tokens of one (sequence, KV head): int8 or e4m3 codes of keys and
of values, and one fp32 scale for each.  ``kind`` names the call:

``append``  keys and values encoded into the cache and read back as BF16, as an
            engine does whose prompt attention runs on what the cache will hold.
``attend``  one decode step over the first ``tokens`` tokens.
``paged``   the same over pool pages and a block table, ragged lengths.
``window``  one decode step in which only the first ``sinks`` and the newest
            ``window`` tokens are visible.
``track``   a decode step that also adds every block's attention weight, summed
            over its tokens and the query heads of its KV head, to its score.
``evict``   the first ``sinks`` and newest ``recent`` tokens and the blocks of
            the largest scores, ``keep`` tokens in all, are copied in order to
            a second cache (a branch of the conversation), which is read back.

Head counts, batches and contexts are those of ``dq_workloads``, the tests and
``perf/cases.py`` or lie between them; so is the inputs' recipe (keys with
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


def listed():
    return [
        # a residual window that fills up: 128 tokens of every sequence leave it for the cache
        {"name": "append_b4_window", "kind": "append", "fmt": "int8", "batch": 4, "tokens": 128, "heads": 8},
        # prefill of four prompts of an odd length, as floating point codes
        {"name": "append_b4_t8k_e4m3", "kind": "append", "fmt": "e4m3", "batch": 4, "tokens": 8171, "heads": 8},
        # the first steps of a chat: a few dozen tokens, launches only
        {"name": "attend_b1_t37", "kind": "attend", "fmt": "int8", "batch": 1, "tokens": 37, "heads": 8, "group": 4},
        # the headline shape: a full batch over long contexts
        {"name": "attend_b16_t32k", "kind": "attend", "fmt": "int8", "batch": 16, "tokens": 32768, "heads": 8,
         "group": 4},
        # wide GQA, floating point codes, the largest call
        {"name": "attend_b32_t32k_g8_e4m3", "kind": "attend", "fmt": "e4m3", "batch": 32, "tokens": 32768,
         "heads": 8, "group": 8},
        # continuous batching: sequences of every length in pool pages
        {"name": "paged_b48_t8k_ragged", "kind": "paged", "fmt": "int8", "batch": 48, "tokens": 8192, "heads": 8,
         "group": 4, "page": 256},
        # one long document of an odd length seen through a window
        {"name": "window_b1_t128k_e4m3", "kind": "window", "fmt": "e4m3", "batch": 1, "tokens": 130873, "heads": 8,
         "group": 4, "window": 4096, "sinks": 4},
        # a batch of chats behind a short window
        {"name": "window_b64_t8k", "kind": "window", "fmt": "int8", "batch": 64, "tokens": 8192, "heads": 8,
         "group": 4, "window": 1024, "sinks": 64},
        # a step that keeps the scores up to date: one chat, and a full batch
        {"name": "track_b1_t4k", "kind": "track", "fmt": "int8", "batch": 1, "tokens": 4096, "heads": 8, "group": 4},
        {"name": "track_b16_t8k_e4m3", "kind": "track", "fmt": "e4m3", "batch": 16, "tokens": 8192, "heads": 8,
         "group": 4},
        # a long document cut to half
        {"name": "evict_b1_t128k", "kind": "evict", "fmt": "int8", "batch": 1, "tokens": 131072, "heads": 8,
         "keep": 65536, "sinks": 32, "recent": 1024},
        # a full batch of an odd length cut to a quarter
        {"name": "evict_b16_t8k_e4m3", "kind": "evict", "fmt": "e4m3", "batch": 16, "tokens": 8171, "heads": 8,
         "keep": 2048, "sinks": 64, "recent": 512},
    ]


def _log_int(rng: random.Random, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "paged", "window", "track", "evict"])
    case = {"kind": kind, "fmt": rng.choice(["int8", "e4m3"]), "heads": rng.choice([1, 2, 4, 8, 8, 8]),
            "batch": _log_int(rng, 1, 64)}
    limit = 1 << 15 if kind == "append" else 1 << 18 if kind == "evict" else 1 << 20
    cap = min(131072, limit // case["batch"])
    case["tokens"] = _log_int(rng, 1, cap)
    if kind not in ("append", "evict"):
        case["group"] = rng.choice([1, 2, 3, 4, 4, 4, 6, 7, 8])
    if kind == "paged":
        case["page"] = rng.choice([128, 256, 512])
    if kind == "window":
        case["window"] = _log_int(rng, 1, 8192)
        case["sinks"] = rng.choice([0, 1, 4, 37, 64, 128])
    if kind == "evict":
        case["tokens"] = max(case["tokens"], 4 * BLOCK + 1)
        case["sinks"] = BLOCK * rng.randrange(0, 2)
        case["recent"] = BLOCK * rng.randrange(1, 3)
        case["keep"] = BLOCK * rng.randrange(3, max(4, case["tokens"] // BLOCK))
    return case


# ------------------------------------------------------------------ inputs

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


def _values(g, batch: int, tokens: int, heads: int) -> torch.Tensor:
    out = torch.empty((batch, tokens, heads, D), dtype=torch.bfloat16, device="cuda")
    for b in range(batch):
        out[b] = torch.randn((tokens, heads, D), generator=g, device="cuda")
    return out


def _inputs(case, seed):
    """Everything random of a case, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, T, H, kind = case["batch"], case["tokens"], case["heads"], case["kind"]
    x = {"k": _keys(g, B, T, H), "v": _values(g, B, T, H)}
    if "group" in case:
        x["q"] = torch.randn((B, H * case["group"], D), generator=g, device="cuda").to(torch.bfloat16)
    lens = torch.full((B,), T, dtype=torch.int32, device="cuda")
    if kind == "paged":
        # a running batch: lengths spread over 1 .. T, the longest full
        lens = (torch.rand(B, generator=g, device="cuda") * T).to(torch.int32) + 1
        lens[int(torch.randint(B, (1,), generator=g, device="cuda"))] = T
        pages = B * -(-T // case["page"])
        # pool pages in the order an engine has handed them out: any
        x["bt"] = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(B, -1).contiguous()
    x["lens"] = lens
    if kind in ("track", "evict"):
        # scores of earlier steps: a few blocks hold most of the weight, and some are equal
        z = torch.randn((B, H, -(-T // BLOCK)), generator=g, device="cuda")
        x["scores"] = torch.exp(2.0 * z).mul_(64.0).round_().div_(64.0)
    return x


# ------------------------------------------------------- the plain forms

def _blocks(x: torch.Tensor) -> torch.Tensor:
    """[B, T, H, D] -> [B, H, T / 32 rounded up, 32, D], zeros behind the last token."""
    B, T, H, _ = x.shape
    nb = -(-T // BLOCK)
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, nb * BLOCK - T))
    return x.view(B, nb, BLOCK, H, D).permute(0, 3, 1, 2, 4)


def _quantise(x: torch.Tensor, fmt: str):
    """Codes as bytes [B, H, nb, 32, D] and scales fp32 [B, H, nb].  The scale
    is the block's largest magnitude over the type's, rounded to fp32; a code
    is the type's value nearest to x / scale, ties to even.  Both quotients are
    taken in 64 bits: in 32 they can land on a border between two codes."""
    xb = _blocks(x)
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


def _attention(q, k, v, visible):
    """q [B, Hq, D]; k, v fp32 [B, H, T, D]; visible [B, T].  Output fp32 and
    the weights [B, H, G, T]; a sequence with no visible token gives zeros."""
    B, H, T, _ = k.shape
    qf = q.float().view(B, H, -1, D)
    s = torch.matmul(qf, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    mask = visible[:, None, None, :]
    s = torch.where(mask, s, -math.inf)
    p = torch.where(mask, torch.exp(s - s.amax(dim=3, keepdim=True)), 0.0)
    p = p / p.sum(dim=3, keepdim=True).clamp(min=1e-30)
    return torch.matmul(p, v).view(B, -1, D), p


def _plain(st):
    case, fmt = st["case"], st["case"]["fmt"]
    kind, B, T, H = case["kind"], case["batch"], case["tokens"], case["heads"]
    if kind == "append":
        out = {}
        for name in ("k", "v"):
            codes, out[name + "_scale"] = _quantise(st[name], fmt)
            out[name] = _floats(codes, out[name + "_scale"], fmt)[:, :, :T].transpose(1, 2).to(torch.bfloat16)
        return out
    kc, ks, vc, vs = st["cache"]
    if kind == "evict":
        nb, keep = ks.shape[2], case["keep"] // BLOCK
        n = min(nb, keep)
        at = torch.arange(nb, device="cuda")
        first, last = case["sinks"] // BLOCK, case["recent"] // BLOCK
        rank = torch.where((at < first) | (at >= nb - last), math.inf, st["scores"])
        kept = torch.sort(rank, dim=2, descending=True, stable=True).indices[:, :, :n]
        kept = kept.sort(dim=2).values
        lens = torch.where(st["lens"] > n * BLOCK, st["lens"] - (nb - n) * BLOCK, st["lens"])
        out = {"kept": kept.to(torch.int32), "lens": lens.to(torch.int32), "scores": st["scores"].gather(2, kept)}
        rows = T - (nb - n) * BLOCK
        for name, c, s in (("k", kc, ks), ("v", vc, vs)):
            picked = c.gather(2, kept[..., None, None].expand(-1, -1, -1, BLOCK, D))
            out[name + "_scale"] = s.gather(2, kept)
            x = _floats(picked, out[name + "_scale"], fmt)[:, :, :rows]
            out[name] = x.transpose(1, 2).to(torch.bfloat16)
        return out
    if kind == "paged":
        bt = st["bt"].long()
        kc, vc = (x[bt].transpose(1, 2).flatten(2, 3) for x in (kc, vc))
        ks, vs = (x[bt].transpose(1, 2).flatten(2, 3) for x in (ks, vs))
    k, v = _floats(kc, ks, fmt), _floats(vc, vs, fmt)
    t = torch.arange(k.shape[2], device="cuda")[None]
    visible = t < st["lens"][:, None]
    if kind == "window":
        visible = visible & ((t < case["sinks"]) | (t >= st["lens"][:, None] - case["window"]))
    out, p = _attention(st["q"], k, v, visible)
    if kind != "track":
        return out
    return {"out": out, "scores": st["scores"] + p.sum(dim=2).unflatten(2, (-1, BLOCK)).sum(dim=3)}


def prepare(case, seed):
    x = _inputs(case, seed)
    B, T, H, kind, fmt = case["batch"], case["tokens"], case["heads"], case["kind"], case["fmt"]
    st = {"case": case, **{n: x[n] for n in x if n not in ("k", "v")}}
    if kind == "append":
        st["k"], st["v"] = x["k"], x["v"]
    t_cap = -(-T // 128) * 128
    nb = -(-T // BLOCK)
    if own:
        # the cache that a user's program holds before the call, filled by the
        # framework's encoder from the same keys and values
        import paper_2609_19880_amd as dq
        Hq = H * case.get("group", 1)
        st["dq"] = dq
        if kind == "paged":
            page = case["page"]
            shape = (B * -(-T // page), H, page // BLOCK)
            data = [torch.zeros((*shape, BLOCK * D), dtype=torch.uint8, device="cuda") for _ in range(2)]
            scales = [torch.zeros(shape, dtype=torch.float32, device="cuda") for _ in range(2)]
            dq.dq_q8_encode_kv_paged(fmt, x["k"], x["v"], 0, st["bt"], data[0], scales[0], data[1], scales[1])
            st["pools"] = (data[0], scales[0], data[1], scales[1])
            st["ws"] = torch.empty(dq.dq_decode_workspace_bytes(B, Hq, H, -(-T // page) * page), dtype=torch.uint8,
                                   device="cuda")
            return st
        st["cache"] = dq.Q8KVCache(B, H, Hq, t_cap, fmt, scores=kind in ("track", "evict"))
        if kind == "append":
            return st
        st["cache"].append(x["k"], x["v"], 0)
        if kind == "track":
            st["scores"] = torch.nn.functional.pad(x["scores"], (0, t_cap // BLOCK - nb))
        if kind == "evict":
            st["cache"].scores[:, :, :nb] = x["scores"]
            st["into"] = dq.Q8KVCache(B, H, Hq, -(-case["keep"] // 128) * 128, fmt, scores=True)
        return st
    if kind == "append":
        return st
    if kind == "paged":
        page = case["page"]
        mp = -(-T // page)
        pool = lambda *s, t: torch.zeros((B * mp, H, page // BLOCK, *s), dtype=t, device="cuda")  # noqa: E731
        cache = [pool(BLOCK, D, t=torch.uint8), pool(t=torch.float32), pool(BLOCK, D, t=torch.uint8),
                 pool(t=torch.float32)]
    else:
        new = lambda *s, t: torch.empty((B, H, nb, *s), dtype=t, device="cuda")  # noqa: E731
        cache = [new(BLOCK, D, t=torch.uint8), new(t=torch.float32), new(BLOCK, D, t=torch.uint8),
                 new(t=torch.float32)]
    for b in range(B):
        for i, name in ((0, "k"), (2, "v")):
            for part, to in zip(_quantise(x[name][b:b + 1], fmt), (cache[i], cache[i + 1])):
                if kind == "paged":
                    rows = torch.zeros((H, mp * (page // BLOCK), *part.shape[3:]), dtype=part.dtype, device="cuda")
                    rows[:, :nb] = part[0]
                    to[st["bt"][b].long()] = rows.unflatten(1, (mp, -1)).transpose(0, 1)
                else:
                    to[b] = part[0]
    st["cache"] = cache
    return st


def run(state):
    if not own:
        return _plain(state)
    case, dq = state["case"], state["dq"]
    kind, T = case["kind"], case["tokens"]
    if kind == "paged":
        q, pools, H = state["q"], state["pools"], case["heads"]
        out = torch.empty(q.shape, dtype=torch.float32, device="cuda")
        dq.dq_q8_decode_attention_paged(case["fmt"], q, *pools, state["bt"], state["lens"], out, state["ws"])
        return out
    c = state["cache"]
    if kind == "append":
        c.append(state["k"], state["v"], 0)
        k, v = c.read(0, T)
        nb = -(-T // BLOCK)
        return {"k": k, "v": v, "k_scale": c.k_scales[:, :, :nb], "v_scale": c.v_scales[:, :, :nb]}
    if kind == "attend":
        return c.attend(state["q"], state["lens"])
    if kind == "window":
        return c.attend(state["q"], state["lens"], window=case["window"], sinks=case["sinks"])
    if kind == "track":
        scores = state["scores"].clone()          # this branch's own scores
        out = c.attend(state["q"], state["lens"], scores=scores)
        return {"out": out, "scores": scores[:, :, :-(-T // BLOCK)]}
    to = state["into"]
    kept, lens = c.evict(state["lens"], case["keep"], case["sinks"], case["recent"], into=to)
    nb = -(-T // BLOCK)
    n = min(nb, case["keep"] // BLOCK)
    k, v = to.read(0, T - (nb - n) * BLOCK)
    return {"kept": kept[:, :, :n], "lens": lens, "scores": to.scores[:, :, :n], "k": k, "v": v,
            "k_scale": to.k_scales[:, :, :n], "v_scale": to.v_scales[:, :, :n]}


def work(case):
    B, T, H, kind = case["batch"], case["tokens"], case["heads"], case["kind"]
    per_token = 2 * H * (D + 4 / BLOCK)          # codes and scales of keys and values
    if kind == "append":
        # bf16 in; codes, scales and the values they stand for out
        n = 2 * B * T * H * D
        return {"bytes": n * (2 + 2) + B * T * per_token, "flops": 3 * n}
    if kind == "evict":
        nb = -(-T // BLOCK)
        rows = B * (T - (nb - min(nb, case["keep"] // BLOCK)) * BLOCK)
        return {"bytes": B * H * nb * 4 + rows * (2 * per_token + 2 * H * D * 2), "flops": rows * 2 * H * D}
    tokens = T
    if kind == "paged":
        tokens = (T + 1) / 2                      # lengths are spread evenly over 1 .. T
    if kind == "window":
        tokens = min(T, case["sinks"] + min(case["window"], max(0, T - case["sinks"])))
    Hq = H * case["group"]
    scores = 8 * B * H * -(-T // BLOCK) if kind == "track" else 0
    return {"bytes": B * tokens * per_token + B * Hq * D * (2 + 4) + scores, "flops": B * tokens * Hq * D * 4}


# ------------------------------------------------------------------- exact
#
# The same in 64 bits, one sequence at a time, from the definition: the grid of
# a type is listed, a code is looked up between the midpoints.

def _grid(fmt: str) -> torch.Tensor:
    if fmt == "int8":
        g = [float(i) for i in range(128)]
    else:
        g = [m * 2.0 ** -9 for m in range(8)]
        g += [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)]
        g = g[:127]                               # the last pattern is no number
    return torch.tensor(g, dtype=torch.float64, device="cuda")


def _round_to(grid: torch.Tensor, y: torch.Tensor) -> torch.Tensor:
    mid = (grid[1:] + grid[:-1]) / 2
    a = y.abs()
    lo, hi = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
    # on a midpoint the two differ by one: the even pattern
    return torch.copysign(grid[torch.where(lo % 2 == 0, lo, hi)], y)


def _held(x: torch.Tensor, fmt: str):
    """What the cache holds of one sequence x [T, H, D]: values fp64 [H, T, D]
    and scales [H, nb]."""
    T, H, _ = x.shape
    nb = -(-T // BLOCK)
    y = torch.zeros((H, nb * BLOCK, D), dtype=torch.float64, device="cuda")
    y[:, :T] = x.double().transpose(0, 1)
    y = y.view(H, nb, BLOCK * D)
    top = y.abs().max(dim=2).values
    s = (top / QMAX[fmt]).float().double() * (top >= TINY)
    grid = _grid(fmt)
    for h in range(H):
        d = torch.where(s[h] > 0, s[h], 1.0)[:, None]
        y[h] = _round_to(grid, y[h] / d) * s[h][:, None]
    return y.view(H, nb * BLOCK, D), s


def exact(case, seed):
    x = _inputs(case, seed)
    kind, fmt, B, T, H = case["kind"], case["fmt"], case["batch"], case["tokens"], case["heads"]
    got = {}

    def put(name, value):
        got.setdefault(name, []).append(value)

    for b in range(B):
        k, ks = _held(x["k"][b], fmt)
        v, vs = _held(x["v"][b], fmt)
        if kind == "append":
            for name, y, s in (("k", k, ks), ("v", v, vs)):
                put(name, y[:, :T].transpose(0, 1).contiguous())
                put(name + "_scale", s)
            continue
        if kind == "evict":
            nb = ks.shape[1]
            n = min(nb, case["keep"] // BLOCK)
            lo, hi = case["sinks"] // BLOCK, nb - case["recent"] // BLOCK
            kept = []
            for row in x["scores"][b].tolist():
                inner = sorted(range(lo, hi), key=lambda i: (-row[i], i))[:n - lo - (nb - hi)] if n < nb else range(lo, hi)
                kept.append(sorted([*range(lo), *inner, *range(hi, nb)]))
            at = torch.tensor(kept, device="cuda")
            put("kept", at.to(torch.int32))
            rows = T - (nb - n) * BLOCK
            put("lens", torch.tensor(rows, dtype=torch.int32, device="cuda"))
            put("scores", x["scores"][b].double().gather(1, at))
            for name, y, s in (("k", k, ks), ("v", v, vs)):
                z = y.view(H, nb, BLOCK * D).gather(1, at[:, :, None].expand(-1, -1, BLOCK * D))
                put(name, z.view(H, n * BLOCK, D)[:, :rows].transpose(0, 1).contiguous())
                put(name + "_scale", s.gather(1, at))
            continue
        L, G = int(x["lens"][b]), case["group"]
        at = list(range(L)) if kind != "window" else [*range(min(L, case["sinks"])),
                                                      *range(max(min(L, case["sinks"]), L - case["window"]), L)]
        at = torch.tensor(at, dtype=torch.int64, device="cuda")
        out, weight = [], torch.zeros((H, ks.shape[1] * BLOCK), dtype=torch.float64, device="cuda")
        for h in range(H):
            a = torch.softmax(x["q"][b, h * G:(h + 1) * G].double() @ k[h][at].T / math.sqrt(D), dim=1)
            out.append(a @ v[h][at])
            weight[h, at] = a.sum(dim=0)
        put("out", torch.cat(out))
        if kind == "track":
            put("scores", x["scores"][b].double() + weight.view(H, -1, BLOCK).sum(dim=2))
    got = {name: torch.stack(rows) for name, rows in got.items()}
    return got if kind in ("append", "track", "evict") else got["out"]
