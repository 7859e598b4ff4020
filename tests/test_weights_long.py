"""kvs_decode_attn_weights at the sizes of full batches and long caches: a CTA of the second launch takes several runs of tokens, and a
head's log-sum is joined from more splits than a warp has lanes."""
import numpy as np
import pytest
import torch

from oracle import bounded_cache as O
from paper_2609_35750_b200 import binding as B

from .test_window_and_weights import Cache, bounds, close, queries

pytestmark = pytest.mark.gpu


def check(c, lens, Hq, Hkv, d, page, **how):
    room = c.table.shape[1] * page
    start = np.random.default_rng(9).random((len(lens), room)).astype(np.float32)
    weight = torch.from_numpy(start).cuda()
    q = queries(3, len(lens), Hq, d)
    out, lse = B.kvs_decode_attn_weights(q[0], *c.args(), weight, **how)
    got = weight.double().cpu().numpy()
    for s, n in enumerate(lens):
        k, v = c.rows(s)
        sees = np.ones((1, n), bool)
        wo, wl, p = O.attention(q[1][s][None], k, v, sees, d ** -0.5)
        bound, delta = bounds(q[1][s][None], k, v, sees, p, wo, d ** -0.5)
        close(out[s][None], wo, bound, (s, "out"))
        close(lse[s][None], wl, delta + 2.0 ** -22 * np.abs(np.where(np.isfinite(wl), wl, 0.0)), (s, "lse"))
        want = start[s].astype(np.float64)
        want[:n] += p[0].sum(axis=0)
        # a head's weight: its score's and the lse's error, exp2 and its argument; then Hq + 1 additions
        tol = np.zeros(room)
        tol[:n] = (p[0] * (2.1 * delta[0][:, None] + 2.0 ** -19)).sum(axis=0) + (Hq + 1) * 2.0 ** -24 * want[:n]
        assert (np.abs(got[s] - want) <= tol).all(), (s, n, (np.abs(got[s] - want) - tol).max())


@pytest.mark.parametrize("S", [70, 130, 250])                     # 2, 4 and 8 runs of 256 tokens a CTA
@pytest.mark.parametrize("Hq,Hkv,d,page", [(4, 2, 64, 16), (4, 1, 128, 1)])
def test_full_batches(S, Hq, Hkv, d, page):
    rng = np.random.default_rng(S)
    lens = rng.integers(0, 200, size=S).tolist()
    lens[1], lens[S // 2], lens[S - 1] = 4096, 4095, 2305
    check(Cache([S, page], lens, page, Hkv, d), lens, Hq, Hkv, d, page, max_tokens=4096)


@pytest.mark.parametrize("Hq,Hkv,d,page", [(4, 1, 64, 16), (8, 1, 128, 16), (7, 1, 128, 1)])
@pytest.mark.parametrize("splits", [0, 33, 64, 100])
def test_more_splits_than_lanes(Hq, Hkv, d, page, splits):
    lens = [5300, 9000]
    if not splits:
        assert B.load().kvs_decode_weights_num_splits(2, Hkv, 9000) > 32
    check(Cache([1, page], lens, page, Hkv, d), lens, Hq, Hkv, d, page, num_splits=splits, max_tokens=9000)
