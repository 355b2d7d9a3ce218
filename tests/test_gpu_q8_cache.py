"""The 8-bit cache object on the GPU: what its documents promise of the tokens
that an eviction keeps, of swapped arrays and of query heads, with expectations
from token positions and memory, not from the library's block rules."""

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def dq():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_19880_amd as mod
    return mod


def _kept_tokens(kept, T):
    """Old positions of the tokens that are left, from the list of kept blocks."""
    return {t for blk in kept.tolist() if blk >= 0 for t in range(32 * blk, min(32 * blk + 32, T))}


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65])
def test_evict_keeps_the_newest_tokens_of_every_length(dq, n):
    """recent = n + 31 keeps the newest n tokens, and recent = n, a multiple of
    32, all but 31 of them at least, however full the newest block is; scores
    that fall towards the newest tokens, the first ones' lowest."""
    lens = list(range(257, 257 + 64))
    B, t_cap, keep = len(lens), 384, 192
    cache = dq.Q8KVCache(B, 1, 1, t_cap, scores=True)
    falling = torch.arange(t_cap // 32, 0, -1, dtype=torch.float32, device=DEV)
    falling[:2] = -1.0
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for recent, promised in ((n + 31, n), (n, n - 31)):
        cache.scores.copy_(falling.expand(B, 1, -1))
        into = dq.Q8KVCache(B, 1, 1, 256, scores=True)
        kept, new_lens = cache.evict(seq, keep, 40, recent, into=into)
        for b, T in enumerate(lens):
            left = _kept_tokens(kept[b, 0], T)
            assert left >= set(range(40)) and left >= set(range(T - max(1, promised), T)), (T, recent)
            assert int(new_lens[b]) == len(left) <= keep


def test_evict_of_a_barely_started_block(dq):
    """Four blocks, the newest of one token, the newest but one with the least
    weight: recent = 32 is that one token's block, recent = 63 the 32 newest tokens."""
    cache = dq.Q8KVCache(1, 1, 1, 128, scores=True)
    seq = torch.tensor([97], dtype=torch.int32, device=DEV)
    for recent, want in ((32, [0, 3]), (63, [2, 3])):
        cache.scores.copy_(torch.tensor([5.0, 1.0, 0.0, 9.0]).view(1, 1, 4))
        into = dq.Q8KVCache(1, 1, 1, 128, scores=True)
        kept, new_lens = cache.evict(seq, 64, 0, recent, into=into)
        assert kept.tolist() == [[want]] and int(new_lens[0]) == 33


def _random_cache(dq, seed, t_cap=384, heads=2, group=2):
    g = torch.Generator().manual_seed(seed)
    cache = dq.Q8KVCache(1, heads, heads * group, t_cap, scores=True)
    k, v = (torch.randn((1, t_cap, heads, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    cache.append(k, v, 0)
    q = torch.randn((1, heads * group, 128), generator=g).to(torch.bfloat16).to(DEV)
    return cache, q


def test_arrays_with_other_memory(dq):
    """A cache whose arrays were given other memory works on that memory and
    leaves the old one alone (which this test keeps, so no access can go astray)."""
    a, q = _random_cache(dq, 1)
    b, _ = _random_cache(dq, 2)
    lens = torch.tensor([384], dtype=torch.int32, device=DEV)
    want, want_rows = b.attend(q, lens), b.read(0, 100)
    want_scores = b.scores.clone()
    held = [x.data for x in (*a.arrays, a.scores, a.block_lse)]
    before = [x.clone() for x in held]
    for x, y in zip(a.arrays, b.arrays):
        x.data = y.clone()
    a.scores.data = torch.zeros_like(a.scores)
    a.block_lse.data = torch.empty_like(a.block_lse)
    assert torch.equal(a.attend(q, lens), want) and torch.equal(a.scores, want_scores)
    assert all(torch.equal(x, y) for x, y in zip(a.read(0, 100), want_rows))
    kept, _ = a.evict(lens, 128, 32, 32)
    at = kept[0, 0].long()
    assert torch.equal(a.k_data[0, 0, :4], b.k_data[0, 0][at])
    assert all(torch.equal(x, y) for x, y in zip(held, before))


def test_arrays_that_do_not_fit_are_refused(dq):
    lens = torch.tensor([384], dtype=torch.int32, device=DEV)
    for change in (lambda c: setattr(c.k_data, "data", c.k_data[:, :, :4].contiguous()),
                   lambda c: setattr(c.v_scales, "data", c.v_scales.cpu()),
                   lambda c: c.k_scales.set_(),
                   lambda c: [setattr(x, "data", x[:, :, :8].contiguous()) for x in c.arrays],
                   lambda c: setattr(c.scores, "data", c.scores[:, :1].contiguous())):
        cache, q = _random_cache(dq, 3)
        cache.attend(q, lens)
        change(cache)
        for call in (lambda: cache.attend(q, lens), lambda: cache.partial(q, lens), lambda: cache.read(0, 32),
                     lambda: cache.evict(lens, 128)):
            with pytest.raises(ValueError):
                call()


@pytest.mark.parametrize("scores", [False, True])
def test_partials_of_other_query_heads_are_refused(dq, scores):
    """merge reads the workspace by the cache's own head count."""
    cache = dq.Q8KVCache(1, 2, 8, 256, scores=scores)
    lens = torch.full((1,), 200, dtype=torch.int32, device=DEV)
    for heads in (2, 4, 6, 16):
        with pytest.raises(ValueError):
            cache.partial(torch.zeros((1, heads, 128), dtype=torch.bfloat16, device=DEV), lens)
    with pytest.raises(ValueError):
        cache.partial(torch.zeros((8, 128), dtype=torch.bfloat16, device=DEV), lens)


def test_a_streaming_step_of_fewer_query_heads(dq):
    """Its merge goes by the query's own heads: the first heads of a wider step."""
    g = torch.Generator().manual_seed(5)
    c = dq.StreamingKVCache(1, 2, 8, 512, None, None, streams="int8")
    k, v = (torch.randn((1, 400, 2, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    c.prefill(k, v)
    q = torch.randn((1, 8, 128), generator=g).to(torch.bfloat16).to(DEV)
    some = q.view(1, 2, 4, 128)[:, :, :2].reshape(1, 4, 128).contiguous()
    want = c.attend(q).view(1, 2, 4, 128)[:, :, :2].reshape(1, 4, 128)
    # other head counts cut the tokens otherwise: weights of 22 bits against other
    # maxima (2 x 2^-22), sums of up to 13 blocks and 256 raw tokens: below 2^-15
    assert ((c.attend(some) - want).norm(dim=2) <= want.norm(dim=2) * 2.0 ** -15).all()


def test_what_a_streaming_cache_s_scores_count(dq):
    """Nothing of a prompt, nothing of a block's steps in the ring, all of its
    steps since; without a step an eviction keeps the oldest blocks."""
    g = torch.Generator().manual_seed(6)
    c = dq.StreamingKVCache(1, 2, 4, 1024, None, None, streams="int8", scores=True)
    k, v = (torch.randn((1, 1024, 2, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    q = torch.randn((1, 4, 128), generator=g).to(torch.bfloat16).to(DEV)
    c.prefill(k[:, :768], v[:, :768])                       # 640 encoded, 128 raw
    assert c.n_comp == 640 and not c.cache.scores.any()
    c.attend(q)
    first = c.cache.scores.clone()
    assert (first[:, :, :20] > 0).all() and not first[:, :, 20:].any()
    for t in range(768, 896):
        c.append(k[:, t].contiguous(), v[:, t].contiguous())
    assert c.n_comp == 768 and torch.equal(c.cache.scores, first)      # tokens 640..767: in the ring until now
    c.attend(q)
    assert (c.cache.scores[:, :, 20:24] > 0).all()
    fresh = dq.StreamingKVCache(1, 2, 4, 1024, None, None, streams="int8", scores=True)
    fresh.prefill(k[:, :768], v[:, :768])
    kept = fresh.evict(384, 32, 64)
    assert kept.tolist() == [[[*range(10), 18, 19]] * 2]
