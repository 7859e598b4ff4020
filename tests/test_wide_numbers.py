"""Whole numbers of more than 32 bits are refused by the calls on bounded caches, not cut to 32 bits: a budget of 2^32 + 10 is not one of 10."""
import pytest
import torch

from paper_2609_35750_b200 import binding as B

WIDE = [2 ** 32 + 5, 2 ** 31, -2 ** 31 - 1, 2 ** 70]


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_35750_b200 import build
    build.build()


@pytest.mark.parametrize("wide", WIDE)
def test_before_anything_else(wide):
    i, f = torch.zeros((1, 4), dtype=torch.int32), torch.zeros((1, 4))
    for at in range(4):
        numbers = [1, 0, 0, 1]
        numbers[at] = wide
        with pytest.raises(ValueError, match="32 bits"):
            B.kvs_cache_evict_lowest(*numbers, i, i[0, :1], i[0], f)
    for drafted, page in ((wide, 1), (1, wide)):
        with pytest.raises(ValueError, match="32 bits"):
            B.kvs_cache_truncate(drafted, i[0, :1], page, i, i[0, :1], i[0])


@pytest.mark.gpu
@pytest.mark.parametrize("wide", WIDE)
def test_attention(wide):
    cache = B.PagedCache(4, 16, 1, 4, 2, 64, track_weights=True)
    kv = torch.ones((1, 3, 2, 64), device="cuda", dtype=torch.bfloat16)
    cache.append_tokens(kv, kv)
    q = torch.ones((1, 1, 4, 64), device="cuda", dtype=torch.bfloat16)
    for how in (dict(window=wide), dict(window=2, sinks=wide), dict(window=2, num_splits=wide), dict(window=2, max_tokens=wide)):
        with pytest.raises(ValueError, match="32 bits"):
            cache.decode_window(q, **how)
    for how in (dict(num_splits=wide), dict(max_tokens=wide)):
        with pytest.raises(ValueError, match="32 bits"):
            cache.decode_weights(q[:, 0], **how)
    assert not cache.token_weight.any()
    assert (cache.decode_window(q, 2 ** 31 - 1, 2 ** 31 - 1, max_tokens=2 ** 31 - 300)[0] == 1).all()
