"""A NaN among the keys that a query sees shows in its log-sum too: -inf is for a query that sees nothing."""
import pytest
import torch

from paper_2609_35750_b200 import binding as B

from .test_window_and_weights import ALL, Cache, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,page", [(8, 2, 128, 16), (8, 2, 128, 1), (4, 2, 64, 16), (2, 2, 128, 1)])
@pytest.mark.parametrize("splits", [1, 3])
def test_a_nan_key_shows_in_out_and_lse(Hq, Hkv, d, page, splits):
    lens = [300, 5, 0, 260]
    c = Cache([Hq, page], lens, page, Hkv, d)
    c.k[c.table[0, 140 // page], 140 % page, 0] = float("nan")              # one KV head of one token
    c.k[c.table[1, 4 // page], 4 % page, 1, 3] = float("nan")               # one number of it
    c.round()
    nan = torch.zeros((4, Hq), dtype=torch.bool)
    G = Hq // Hkv
    nan[0, :G] = nan[1, G:2 * G] = True
    q = queries(1, 4, Hq, d)[0]
    weight = torch.zeros((4, c.table.shape[1] * page), device="cuda")
    cache = B.PagedCache.__new__(B.PagedCache)
    cache.__dict__.update(Hkv=Hkv, page_size=page, max_pages=c.table.shape[1], num_pages=c.gk.shape[0], block_table=c.gt, n_tokens=c.gn, k_cache=c.gk, v_cache=c.gv)
    window = B.kvs_decode_attn_window(q[:, None], *c.args(), ALL, num_splits=splits)
    for out, lse in (cache.decode(q, num_splits=splits), (window[0][:, 0], window[1][:, 0]),
                     B.kvs_decode_attn_weights(q, *c.args(), weight, num_splits=splits)):
        assert torch.equal(torch.isnan(lse).cpu(), nan) and torch.isnan(out).all(dim=-1).cpu().equal(nan)
        assert torch.isneginf(lse[2]).all() and not out[2].any()
        assert torch.isfinite(lse[3]).all() and torch.isfinite(out[3]).all()
    assert torch.isnan(weight[0, :300]).all() and torch.isfinite(weight[2:]).all()
