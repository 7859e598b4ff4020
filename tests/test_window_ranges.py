"""kvs_decode_attn_window: values and scores at the ends of what bf16 holds."""
import numpy as np
import pytest
import torch

from paper_2609_35750_b200 import binding as B

from .test_window_and_weights import ALL, Cache, check_window, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,page,new", [(8, 2, 64, 16, 2), (8, 2, 128, 16, 1), (8, 1, 128, 1, 4)])
@pytest.mark.parametrize("power", [104, -90])
@pytest.mark.parametrize("lean", [0.0, 20.0, -20.0])
def test_values_of_any_size(Hq, Hkv, d, page, new, power, lean):
    """Scores of up to about 30 in base 2, around 0 or to one side of it.  No sum need come near 2^128: 1000 keys, values below 2^107 and
    weights of no more than 2^8 give 2^125; nor do products near 2^-126 count: 2^-90 less the 2^22 that the largest weight may be below 1."""
    c = Cache([d, page], [1000, 700, 128], page, Hkv, d)
    c.k += lean / d
    c.v *= 2.0 ** power
    c.round()
    gq, fq = queries(3, 3, new, Hq, d)
    gq += 2.0
    q = (gq, gq.double().cpu().numpy())
    scale = 2.6 * d ** -0.5
    check_window(c, q, ALL, 0, *B.kvs_decode_attn_window(gq, *c.args(), ALL, softmax_scale=scale, num_splits=2), scale=scale)


def test_scores_far_below_anything_usual():
    """A query whose window begins in its share's second tile, and whose scores are below -1e30: its one visible token has weight 1."""
    S, d, page = 100, 64, 16
    c = Cache(7, [129] * S, page, 1, d)                           # two tiles each, of one CTA: there are more than twice as many as CTAs
    for s in range(S):
        for t in (127, 128):
            c.k[c.table[s, t // page], t % page] = -1e17
    c.round()
    q = torch.full((S, 2, 2, d), 1e17, device="cuda").bfloat16()
    out, lse = B.kvs_decode_attn_window(q, *c.args(), 1, num_splits=1)
    for s in range(S):
        for t in (0, 1):                                           # query t sees token 127 + t alone
            want = c.rows(s)[1][127 + t, 0]
            assert np.array_equal(out[s, t].double().cpu().numpy(), np.broadcast_to(want, (2, d)))
    want = float(q[0, 0, 0, 0]) * float(c.gk[int(c.table[0, 127 // page]), 127 % page, 0, 0]) * d * d ** -0.5
    assert ((lse.double() - want).abs() < 1e-4 * abs(want)).all()
