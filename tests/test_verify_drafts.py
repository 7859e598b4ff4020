"""Verification of drafted tokens: whole numbers, equal to the plain statement in 64 bits; and the distribution it is there for."""
import numpy as np
import pytest
import torch

from oracle import bounded_cache as O
from paper_2609_35750_b200 import binding as B


def case(rng, S, n, V, near=0.5):
    soft = lambda x: np.exp(x - x.max(-1, keepdims=True)) / np.exp(x - x.max(-1, keepdims=True)).sum(-1, keepdims=True)  # noqa: E731
    logits = rng.normal(size=(S, n + 1, V)) * 2
    target = soft(logits).astype(np.float32)
    draft = soft(logits[:, :n] + near * rng.normal(size=(S, n, V))).astype(np.float32)
    x = np.array([[rng.choice(V, p=draft[s, i] / draft[s, i].astype(np.float64).sum()) for i in range(n)] for s in range(S)], np.int32).reshape(S, n)
    return target, draft, x, rng.random((S, n)).astype(np.float32), rng.random(S).astype(np.float32)


def on_gpu(args):
    return B.kvs_verify_drafts(*(torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in args))


def same(args):
    tokens, count = on_gpu(args)
    want, number = O.verify(*args)
    assert np.array_equal(count.cpu().numpy(), number)
    assert np.array_equal(tokens.cpu().numpy(), want)


# ---- CPU ---------------------------------------------------------------------------------------------------------
def test_plain_verification_by_hand():
    target = np.array([[[0.5, 0.25, 0.25, 0.0], [0.25, 0.25, 0.25, 0.25]]], np.float32)
    draft = np.array([[[0.25, 0.5, 0.0, 0.25]]], np.float32)
    go = lambda x, ua, us: [a.tolist() for a in O.verify(target, draft, np.array([[x]]), np.array([[ua]], np.float32), np.array([us], np.float32))]  # noqa: E731
    assert go(0, 0.99, 0.5) == [[[0, 2]], [1]]                  # target 0.5 over draft 0.25: always kept; then the second row
    assert go(1, 0.5, 0.0) == [[[0, -1]], [0]]                  # 0.5 * 0.5 < 0.25 is false: rejected; residual (0.25, 0, 0.25, 0)
    assert go(1, 0.5, 0.5) == [[[2, -1]], [0]]
    assert go(1, 0.49, 0.75) == [[[1, 3]], [1]]
    assert go(3, 0.0, 0.0) == [[[0, -1]], [0]]                  # the target has none of it


def test_plain_verification_keeps_the_target_distribution():
    """Over a grid of random numbers the first token comes out as often as the target says."""
    rng = np.random.default_rng(0)
    target, draft, _, _, _ = case(rng, 1, 1, 5, near=1.5)
    N, freq = 128, np.zeros(5)
    for x in range(5):
        for a in range(N):
            ua = np.float32((a + 0.5) / N)
            us = ((np.arange(N) + 0.5) / N).astype(np.float32)
            rep = lambda t: np.repeat(t, N, axis=0)  # noqa: E731
            tokens, _ = O.verify(rep(target), rep(draft), np.full((N, 1), x), np.full((N, 1), ua, np.float32), us)
            freq += float(draft[0, 0, x]) * np.bincount(tokens[:, 0], minlength=5) / N ** 2
    # both grids place a step to within 1 / (2 N) of where it belongs; five draws of each
    assert np.abs(freq - target[0, 0]).max() <= 2 * 5 / (2 * N)


@pytest.fixture(scope="module")
def lib():
    from paper_2609_35750_b200 import build
    build.build()
    return B.load()


def test_host_refusals_need_no_gpu(lib):
    p = 1 << 20
    go = lambda S=1, n=1, V=4, t=p, d=p, out=p: lib.kvs_verify_drafts(t, d, p, p, p, S, n, V, out, p, None)      # noqa: E731
    assert go(S=-1) == go(n=-1) == go(V=0) == go(t=None) == go(d=None) == go(out=None) == B.KVS_ERR_INVALID_ARG
    assert go(V=(1 << 24) + 1) == go(n=65536) == B.KVS_ERR_UNSUPPORTED
    assert go(t=p + 2) == B.KVS_ERR_ALIGNMENT
    assert go(S=0, t=None) == B.KVS_OK
    f, i = torch.zeros((1, 2, 4)), torch.zeros((1, 1), dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        B.kvs_verify_drafts(f, f[:, :1], i, f[0, :1, :1], f[0, 0, :1])


# ---- GPU ---------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("S,n,V", [(1, 1, 1), (1, 1, 2), (3, 4, 33), (5, 2, 255), (5, 2, 257), (2, 40, 300), (7, 3, 5003), (40, 2, 2049), (700, 1, 100),
                                   (2, 8, 32000), (3, 5, 131071)])
def test_matches_the_plain_statement(S, n, V):
    same(case(np.random.default_rng([S, n, V]), S, n, V))


@pytest.mark.gpu
def test_no_drafts_is_a_plain_draw():
    rng = np.random.default_rng(1)
    target = rng.random((6, 1, 777)).astype(np.float32)                       # rows need not add up to 1
    same((target, np.zeros((6, 0, 777), np.float32), np.zeros((6, 0), np.int32), np.zeros((6, 0), np.float32), rng.random(6).astype(np.float32)))


@pytest.mark.gpu
def test_corners():
    rng = np.random.default_rng(2)
    S, n, V = 14, 3, 1500
    target, draft, x, ua, us = case(rng, S, n, V)
    us[0], us[1] = 0.0, np.nextafter(np.float32(1), np.float32(0))
    ua[2], ua[3] = 0.0, np.nextafter(np.float32(1), np.float32(0))
    x[4, 1], x[5, 0], x[6, 2] = -1, V, 2 ** 31 - 1                           # outside the vocabulary
    draft[7] = target[7, :n]                                                  # the same model: all are kept
    draft[8], ua[8] = target[8, :n] * np.float32(2), 0.75                     # more everywhere: nothing is left of the row
    target[9], target[10, :, :1400] = 0.0, 0.0                                # no probability at all; the last few alone
    target[11, 0, ::3] = np.nan
    draft[12, 0, ::2] = np.nan
    us[13] = 1.0                                                              # outside [0, 1): the last with any weight
    same((target, draft, x, ua, us))
    # one token has it all, wherever it lies
    for k in (0, 1, 255, 256, 1023, 1499):
        target, draft, x, ua, us = case(rng, 3, 2, V)
        target[:], draft[:], ua[:] = 0.0, np.float32(1 / V), 0.5
        target[:, :, k] = 1.0
        us[:] = [0.0, 0.5, np.nextafter(np.float32(1), np.float32(0))]
        same((target, draft, x, ua, us))


@pytest.mark.gpu
def test_shapes_are_checked():
    f, i = torch.zeros((2, 3, 8), device="cuda"), torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    u = torch.zeros((2, 2), device="cuda")
    for args in ((f, f, i, u, u[0]), (f, f[:, :2].contiguous(), i[:1], u, u[0]), (f, f[:, :2], i, u, u[0]), (f.double(), f[:, :2].contiguous(), i, u, u[0]),
                 (f, f[:, :2].contiguous(), i.long(), u, u[0]), (f, f[:, :2].contiguous(), i, u, u)):
        with pytest.raises(ValueError):
            B.kvs_verify_drafts(*args)
