"""The 8-bit cache object's argument checks that need no GPU."""

import pytest
import torch

dq = pytest.importorskip("paper_2609_19880_amd")


@pytest.mark.parametrize("scores", [False, True])
def test_partials_of_other_query_heads_are_refused(scores):
    c = dq.Q8KVCache(1, 2, 8, 256, scores=scores, device="cpu")
    lens = torch.zeros(1, dtype=torch.int32)
    for shape in ((1, 4, 128), (1, 16, 128), (8, 128)):
        with pytest.raises(ValueError, match="q_heads"):
            c.partial(torch.zeros(shape, dtype=torch.bfloat16), lens)


def test_scores_of_a_cache_without_scores_are_refused():
    c = dq.Q8KVCache(1, 2, 8, 256, device="cpu")
    lens = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: c.add_scores(lens), lambda: c.merge_scores(lens, torch.zeros((1, 8, 128)))):
        with pytest.raises(ValueError, match="scores"):
            call()


@pytest.mark.parametrize("kw", [dict(sinks=-1), dict(sinks=-64), dict(recent=-1), dict(recent=-64)])
def test_negative_counts_of_an_eviction_are_refused(kw):
    """Rounded up they would have become 0 and 32."""
    c = dq.Q8KVCache(1, 2, 8, 256, scores=True, device="cpu")
    with pytest.raises(ValueError, match="negative"):
        c.evict(torch.zeros(1, dtype=torch.int32), 128, **kw)
