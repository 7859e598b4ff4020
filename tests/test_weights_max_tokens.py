"""kvs_decode_attn_weights: `max_tokens` is a bound to the token, not to the tile."""
import pytest
import torch

from paper_2609_35750_b200 import binding as B

from .test_window_and_weights import Cache, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,page", [(8, 2, 128, 16), (8, 2, 128, 1), (4, 2, 64, 16)])
@pytest.mark.parametrize("most", [1, 100, 200])
def test_one_token_more_than_said(Hq, Hkv, d, page, most):
    lens = [most, most + 1, 0, most + 55]
    c = Cache(1, lens, page, Hkv, d)
    q = queries(2, len(lens), Hq, d)[0]
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    weight = torch.zeros((len(lens), c.table.shape[1] * page), device="cuda")
    out, lse = B.kvs_decode_attn_weights(q, *c.args(), weight, max_tokens=most, workspace=ws, num_splits=2)
    assert B.kvs_device_status(ws) == B.KVS_ERR_INVALID_ARG
    assert not weight[1:].any() and abs(float(weight[0].sum()) - Hq) < 1e-4           # the weights of a head add up to 1
    told = torch.zeros_like(weight)
    full, l2 = B.kvs_decode_attn_weights(q, *c.args(), told, max_tokens=most + 55, workspace=ws, num_splits=2)
    assert B.kvs_device_status(ws) == B.KVS_OK
    # The attention itself is theirs all the same.  A split that met an error gives the lowest bit of its sum for the error's kind, so that a
    # sum of weights L may be off by 2^-23 of itself: out by one step of bf16 (2^-7 of itself at most), where it lies next to a border, lse by
    # 2^-23, a step of log L (L < 2^10, log L < 8: 2^-21) and a step of its own (2^-23 of itself).
    dead = torch.isneginf(l2)
    assert torch.equal(torch.isneginf(lse), dead) and ((out - full).abs().float() <= 2.0 ** -7 * full.abs().float()).all()
    assert ((lse - l2).abs() <= 2.0 ** -23 + 2.0 ** -21 + 2.0 ** -23 * l2.abs())[~dead].all()
    assert torch.equal(lse[0], l2[0]) and torch.equal(out[0], full[0])                   # nothing was wrong with this one
    assert torch.equal(told[0], weight[0]) and (told[[1, 3]].sum(dim=1) - Hq).abs().max() < 1e-4
