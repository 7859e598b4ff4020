"""More rows (sequence, query head) than 2^27: their merge reaches every one of them."""
import pytest
import torch

from paper_2609_35750_b200 import binding as B


@pytest.mark.gpu
def test_the_last_of_more_rows_than_threads_count_in_32_bits():
    S, G, Hkv, d = 65535, 8, 257, 64
    Hq = G * Hkv
    assert S * Hq * 32 > 2 ** 32
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 90e9:
        pytest.skip("needs 90 GB of device memory")
    k, v = (torch.randn((1, 1, Hkv, d), device="cuda").bfloat16() for _ in range(2))
    n = torch.zeros(S, dtype=torch.int32, device="cuda")
    n[0] = n[-1] = 1
    q = torch.empty((S, Hq, d), device="cuda", dtype=torch.bfloat16)
    q[[0, 1, -2, -1]] = torch.randn((4, Hq, d), device="cuda").bfloat16()
    cache = B.PagedCache.__new__(B.PagedCache)
    cache.__dict__.update(Hkv=Hkv, page_size=1, max_pages=1, num_pages=1, block_table=torch.zeros((S, 1), dtype=torch.int32, device="cuda"),
                          n_tokens=n, k_cache=k, v_cache=v)
    out, lse = torch.empty_like(q), torch.empty((S, Hq), device="cuda")
    for s in (0, 1, S - 2, S - 1):
        out[s], lse[s] = 7.0, 7.0
    cache.decode(q, num_splits=1, out=out, lse=lse)
    for s in (0, 1, S - 2, S - 1):
        if int(n[s]):
            assert torch.equal(out[s].view(Hkv, G, d), v[0, 0, :, None].expand(Hkv, G, d))          # one token: its weight is 1
            score = (q[s].view(Hkv, G, d).double() * k[0, 0, :, None].double()).sum(-1).view(-1) * d ** -0.5
            assert (lse[s].double() - score).abs().max() < 1e-4
        else:
            assert not out[s].any() and torch.isneginf(lse[s]).all()
    del q, out, lse, cache
    torch.cuda.empty_cache()
