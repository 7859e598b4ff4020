"""kvs_decode_attn_window: values and scores at the ends of what bf16 holds."""
import numpy as np
import pytest
import torch

from paper_2609_35750_b200 import binding as B

from .test_window_and_weights import Cache

pytestmark = pytest.mark.gpu


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
