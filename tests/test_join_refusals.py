"""kvs_cache_append_tokens: which error is told does not depend on which sequence comes first."""
import pytest
import torch

from paper_2609_35750_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S", [4, 1500])                         # by one launch and by two
@pytest.mark.parametrize("top", [0, 8, 99])
def test_a_senseless_length_is_told_before_a_full_table(S, top):
    """Lengths or a stack that make no sense are KVS_ERR_INVALID_ARG, whatever else is short."""
    for bad, full in ((0, 1), (1, 0), (S - 1, 2), (2, S - 1)):
        n = torch.ones(S, dtype=torch.int32, device="cuda")
        n[bad], n[full] = -1, 8
        table = torch.zeros((S, 8), dtype=torch.int32, device="cuda")
        free = torch.zeros(4 + 8, dtype=torch.int32, device="cuda")
        free[0] = top
        kv = torch.zeros((8, 1, 1, 64), device="cuda", dtype=torch.bfloat16)
        new = torch.ones((S, 1, 1, 64), device="cuda", dtype=torch.bfloat16)
        before = n.clone()
        B.kvs_cache_append_tokens(new, new, table, n, free, kv, kv.clone())
        assert free[:2].tolist() == [top, B.KVS_ERR_INVALID_ARG] and torch.equal(n, before) and not kv.any()
    n = torch.ones(S, dtype=torch.int32, device="cuda")
    n[1] = 8                                                      # a full table, and a stack that makes no sense
    free[:2] = torch.tensor([99, 0], dtype=torch.int32)
    B.kvs_cache_append_tokens(new, new, table, n, free, kv, kv.clone())
    assert int(free[1]) == B.KVS_ERR_INVALID_ARG
