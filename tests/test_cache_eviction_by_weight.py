"""Eviction by accumulated weight, appending and dropping several tokens: whole numbers and moved weights, bit for bit against the
plain statement; refusals on the host; states that make no sense are recorded and left alone."""
import copy

import numpy as np
import pytest
import torch

from oracle import bounded_cache as O
from paper_2609_35750_b200 import binding as B


def make(rng, lens, page, max_pages, spare=3):
    """A cache of these live lengths: scattered pages, weights over many orders of magnitude with ties and zeros."""
    S = len(lens)
    used = [-(-n // page) for n in lens]
    pool = sum(used) + spare
    order = rng.permutation(pool).astype(np.int32)
    table = rng.integers(0, pool, size=(S, max_pages)).astype(np.int32)          # stale entries behind the live ones
    weight, at = np.zeros((S, max_pages * page), np.float32), 0
    for s, n in enumerate(lens):
        table[s, :used[s]] = order[at:at + used[s]]
        at += used[s]
        w = np.exp(rng.normal(size=n) * 4.0).astype(np.float32)
        w[rng.random(n) < 0.3] = 0.0
        w[rng.random(n) < 0.2] = np.float32(0.125)
        weight[s, :n] = w
    free = np.concatenate([[pool - at, 0, 0, 0], order[at:], rng.integers(0, pool, size=at)]).astype(np.int32)
    return dict(table=table, n=np.array(lens, np.int32), free=free, weight=weight)


def on_gpu(c):
    return {k: torch.from_numpy(v.copy()).cuda() for k, v in c.items()}


def same(c, g, what=""):
    for k in c:
        got = g[k].cpu().numpy()
        if k == "free":                       # {top, status, two words of the kernels' own}
            assert got[0] == c[k][0] and got[1] == B.KVS_OK, (what, got[:4], c[k][:4])
            got, want = got[4:], c[k][4:]
        else:
            want = c[k]
        assert got.tobytes() == want.tobytes(), (what, k)


# ---- CPU ---------------------------------------------------------------------------------------------------------
def test_the_plain_eviction_by_hand():
    c = dict(table=np.array([[5, 3, 8, 1, 0]], np.int32), n=np.array([9], np.int32), free=np.array([1, 0, 0, 0, 7] + [0] * 9, np.int32),
             weight=np.array([[9, 9, 1, 1, 0, 2, 0, 1, 4, 0]], np.float32))
    evicted, count = O.evict_lowest(c, 6, 2, 1, 2)            # three pages are candidates: scores 2, 2, 1; two of them leave
    assert evicted.tolist() == [[1, 3, -1, -1, -1]] and count.tolist() == [2] and c["n"].tolist() == [5]
    assert c["table"][0, :3].tolist() == [5, 8, 0] and c["weight"].tolist() == [[9, 9, 0, 2, 4, 0, 0, 0, 0, 0]]
    assert c["free"][0] == 3 and c["free"][4:7].tolist() == [7, 1, 3]
    assert O.append_tokens(c, 4, 2) == {0: [(0, 1), (3, 0), (3, 1), (1, 0)]} and c["free"][0] == 1
    O.truncate(c, 4, [1], 2)
    assert c["n"].tolist() == [6] and c["free"][0] == 3 and c["free"][4:7].tolist() == [7, 1, 3]


@pytest.fixture(scope="module")
def lib():
    from paper_2609_35750_b200 import build
    build.build()
    return B.load()


def test_host_refusals_need_no_gpu(lib):
    p = 1 << 20                                                # an address that is never followed
    ev = lambda budget=1, first=0, recent=0, S=1, page=1, P=4, pool=4, table=p, w=p: lib.kvs_cache_evict_lowest(      # noqa: E731
        budget, first, recent, S, page, P, pool, table, p, p, w, None, p, None)
    assert ev(budget=-1) == ev(first=-1) == ev(recent=-1) == ev(S=-1) == ev(page=0) == ev(P=0) == ev(pool=0) == B.KVS_ERR_INVALID_ARG
    assert ev(table=None) == ev(w=None) == B.KVS_ERR_INVALID_ARG
    assert ev(w=p + 2) == B.KVS_ERR_ALIGNMENT
    assert ev(P=1 << 20) == ev(page=16, P=1 << 16) == ev(page=1 << 16, P=1 << 16) == B.KVS_ERR_UNSUPPORTED
    assert ev(S=0, table=None) == B.KVS_OK
    ap = lambda S=1, new=1, H=1, d=64, page=1, P=4, pool=4, k=p: lib.kvs_cache_append_tokens(k, p, None, S, new, H, d, page, P, pool, p, p, p, p, p, None)      # noqa: E731
    assert ap(S=-1) == ap(new=-1) == ap(H=0) == ap(d=0) == ap(page=0) == ap(P=0) == ap(pool=0) == ap(k=None) == B.KVS_ERR_INVALID_ARG
    assert ap(page=1 << 16, P=1 << 16) == B.KVS_ERR_UNSUPPORTED and ap(k=p + 1) == B.KVS_ERR_ALIGNMENT
    assert ap(S=0) == ap(new=0) == B.KVS_OK
    tr = lambda drafted=1, S=1, page=1, P=4, pool=4, acc=p: lib.kvs_cache_truncate(drafted, acc, S, page, P, pool, p, p, p, None, None)      # noqa: E731
    assert tr(drafted=-1) == tr(S=-1) == tr(page=0) == tr(P=0) == tr(pool=0) == tr(acc=None) == B.KVS_ERR_INVALID_ARG
    assert tr(page=1 << 16, P=1 << 16) == B.KVS_ERR_UNSUPPORTED and tr(acc=p + 1) == B.KVS_ERR_ALIGNMENT
    assert tr(S=0) == tr(drafted=0) == B.KVS_OK


def test_tables_of_more_entries_than_32_bits_count_are_refused(lib):
    p = 1 << 20                                                # an address that is never followed
    for S, P in ((1 << 16, 1 << 15), (1 << 20, 1 << 12), (1 << 24, 128)):
        assert lib.kvs_cache_evict_lowest(1, 0, 0, S, 1, P, 4, p, p, p, p, None, p, None) == B.KVS_ERR_UNSUPPORTED
        assert lib.kvs_cache_append_tokens(p, p, None, S, 1, 1, 64, 1, P, 4, p, p, p, p, p, None) == B.KVS_ERR_UNSUPPORTED
        assert lib.kvs_cache_truncate(1, p, S, 1, P, 4, p, p, p, None, None) == B.KVS_ERR_UNSUPPORTED


def test_host_tensors_are_refused(lib):
    i, f = torch.zeros((1, 4), dtype=torch.int32), torch.zeros((1, 4))
    with pytest.raises(ValueError, match="CUDA"):
        B.kvs_cache_evict_lowest(1, 0, 0, 1, i, i[0, :1], i[0], f)
    with pytest.raises(ValueError, match="CUDA"):
        B.kvs_cache_truncate(1, i[0, :1], 1, i, i[0, :1], i[0])
    kv = torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        B.kvs_cache_append_tokens(kv, kv, i, i[0, :1], i[0], kv, kv)


# ---- GPU ---------------------------------------------------------------------------------------------------------
LENS = [0, 1, 2, 15, 16, 17, 33, 128, 300, 1000]


@pytest.mark.gpu
@pytest.mark.parametrize("page,max_pages", [(1, 1003), (1, 9000), (16, 70), (3, 340), (64, 17), (16, 4000)])
@pytest.mark.parametrize("budget,first,recent", [(0, 0, 0), (100, 4, 32), (16, 20, 1), (5000, 0, 0), (7, 2 ** 31 - 1, 0), (3, 0, 2 ** 31 - 1)])
def test_lowest_pages_leave(page, max_pages, budget, first, recent):
    rng = np.random.default_rng([page, max_pages, budget])
    lens = LENS + ([8191, 9000] if max_pages == 9000 else [50000, 64000] if max_pages == 4000 else [])
    c = make(rng, lens, page, max_pages)
    c["weight"][2, :1] = -0.0
    c["weight"][8, 40:44] = [np.nan, np.inf, -1.0, 1e-42]
    g = on_gpu(c)
    evicted, count = B.kvs_cache_evict_lowest(budget, first, recent, page, g["table"], g["n"], g["free"], g["weight"])
    want, number = O.evict_lowest(c, budget, first, recent, page)
    assert count.cpu().numpy().tolist() == number.tolist()
    assert np.array_equal(evicted.cpu().numpy(), want)
    same(c, g)
    # once more: everything that could leave has left
    before = copy.deepcopy(c)
    _, count = B.kvs_cache_evict_lowest(budget, first, recent, page, g["table"], g["n"], g["free"], g["weight"])
    assert not count.any()
    same(before, g)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[0], [1], [300], [999, 0, 17], [15, 16, 17, 33, 128, 300, 1000, 2], [15, 16, 17, 33, 128, 300, 1000, 2, 400]])
@pytest.mark.parametrize("page,max_pages", [(1, 1003), (16, 70), (5, 400), (1, 2048), (1, 2049), (64, 150)])
def test_few_sequences(lens, page, max_pages):
    """Up to eight small sequences are planned and cut by one launch, more or larger ones by two."""
    c = make(np.random.default_rng([len(lens), page]), lens, page, max_pages)
    c["weight"][:, 5:9] = 3.0
    for s, n in enumerate(lens):
        c["weight"][s, n:] = 0.0
    g = on_gpu(c)
    evicted, count = B.kvs_cache_evict_lowest(20, 3, 5, page, g["table"], g["n"], g["free"], g["weight"])
    want, number = O.evict_lowest(c, 20, 3, 5, page)
    assert np.array_equal(evicted.cpu().numpy(), want) and np.array_equal(count.cpu().numpy(), number)
    same(c, g)


@pytest.mark.gpu
def test_more_sequences_than_the_plan_has_threads_and_equal_scores():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 40, size=2500).tolist()
    c = make(rng, lens, 2, 21)
    c["weight"][c["weight"] > 0] = 1.0                          # mostly ties: the earlier slots leave
    g = on_gpu(c)
    evicted, count = B.kvs_cache_evict_lowest(11, 3, 2, 2, g["table"], g["n"], g["free"], g["weight"])
    want, number = O.evict_lowest(c, 11, 3, 2, 2)
    assert np.array_equal(evicted.cpu().numpy(), want) and np.array_equal(count.cpu().numpy(), number)
    same(c, g)


@pytest.mark.gpu
def test_largest_cache_of_one_token_pages():
    rng = np.random.default_rng(6)
    c = make(rng, [160000, 7], 1, 160000)
    g = on_gpu(c)
    evicted, count = B.kvs_cache_evict_lowest(90001, 4, 1000, 1, g["table"], g["n"], g["free"], g["weight"])
    n, w = 160000, c["weight"][0]
    order = 4 + np.argsort(w[4:n - 1000], kind="stable")[:n - 90001]
    assert np.array_equal(np.sort(order), evicted[0, :n - 90001].cpu().numpy()) and count.tolist() == [n - 90001, 0]
    stay = np.setdiff1d(np.arange(n), order)
    assert np.array_equal(g["table"][0, :90001].cpu().numpy(), c["table"][0, stay])
    assert np.array_equal(g["weight"][0, :90001].cpu().numpy(), w[stay]) and not g["weight"][0, 90001:].any()
    assert g["free"][1] == B.KVS_OK and int(g["free"][0]) == 3 + n - 90001


@pytest.mark.gpu
@pytest.mark.parametrize("more", [0, 9])                         # by one launch and by two
def test_states_that_make_no_sense_are_left_alone(more):
    rng = np.random.default_rng(7)
    c = make(rng, [20, 30] + [4] * more, 2, 16)
    for value in (33, -5):
        bad = copy.deepcopy(c)
        bad["n"][0] = value
        g = on_gpu(bad)
        evicted, count = B.kvs_cache_evict_lowest(10, 0, 0, 2, g["table"], g["n"], g["free"], g["weight"])
        assert int(g["free"][1]) == B.KVS_ERR_INVALID_ARG and count.tolist() == [0, 10] + [0] * more and not (evicted[0] != -1).any()
        assert g["n"].tolist() == [value, 10] + [4] * more and g["table"][0].cpu().numpy().tolist() == bad["table"][0].tolist()
    bad = copy.deepcopy(c)
    bad["free"][0] = len(c["free"]) - 4 - 1                      # more pages would come back than the cache has
    g = on_gpu(bad)
    _, count = B.kvs_cache_evict_lowest(10, 0, 0, 2, g["table"], g["n"], g["free"], g["weight"])
    assert int(g["free"][1]) == B.KVS_ERR_INVALID_ARG and not count.any() and int(g["free"][0]) == bad["free"][0]
    assert g["n"].tolist() == bad["n"].tolist() and np.array_equal(g["table"].cpu().numpy(), bad["table"])


@pytest.mark.gpu
@pytest.mark.parametrize("S,new,Hkv,d", [(128, 3, 1, 64), (129, 3, 1, 64), (300, 1, 2, 128), (2, 300, 4, 128), (1500, 2, 1, 64)])
def test_many_sequences_and_many_tokens_join(S, new, Hkv, d):
    rng = np.random.default_rng([S, new])
    page, lens = 4, rng.integers(0, 30, size=S).tolist()
    c = make(rng, lens, page, (30 + new) // page + 1, spare=S * (new // page + 2))
    g = on_gpu(c)
    kc = torch.zeros((len(c["free"]) - 4, page, Hkv, d), device="cuda", dtype=torch.bfloat16)
    kn = torch.randn((S, new, Hkv, d), device="cuda").bfloat16()
    vc, want = kc.clone(), kc.clone()
    B.kvs_cache_append_tokens(kn, -kn, g["table"], g["n"], g["free"], kc, vc)
    places = O.append_tokens(c, new, page)
    at = torch.tensor([places[s][t] for s in range(S) for t in range(new)], device="cuda")
    want[at[:, 0], at[:, 1]] = kn.view(S * new, Hkv, d)
    same(c, g)
    assert torch.equal(kc, want) and torch.equal(vc, -want)


@pytest.mark.gpu
@pytest.mark.parametrize("page,Hkv,d", [(1, 2, 128), (16, 3, 64), (5, 1, 64), (4, 1, 6)])
@pytest.mark.parametrize("new", [1, 5, 70])
def test_tokens_join_and_leave(page, Hkv, d, new):
    rng = np.random.default_rng([page, new])
    lens = [0, 1, 4, 16, 37, 100, 15]
    S, P = len(lens), -(-(100 + new) // page)
    c = make(rng, lens, page, P, spare=S * (new // page + 2))
    pages = len(c["free"]) - 4
    active = np.array([1, 1, 0, 1, 1, 1, 255], np.uint8)
    g = on_gpu(c)
    kc, vc = (torch.randn((pages, page, Hkv, d), device="cuda").bfloat16() for _ in range(2))
    kn, vn = (torch.randn((S, new, Hkv, d), device="cuda").bfloat16() for _ in range(2))
    wk, wv = kc.clone(), vc.clone()
    B.kvs_cache_append_tokens(kn, vn, g["table"], g["n"], g["free"], kc, vc, active=torch.from_numpy(active).cuda())
    start = copy.deepcopy(c)
    for s, places in O.append_tokens(c, new, page, active).items():
        for t, (pg, row) in enumerate(places):
            wk[pg, row], wv[pg, row] = kn[s, t], vn[s, t]
    same(c, g, "append")
    assert torch.equal(wk, kc) and torch.equal(wv, vc)
    # some stay, the others leave
    accepted = np.where(active, rng.integers(0, new + 1, size=S), new).astype(np.int32)
    c["weight"] += 1.0
    g["weight"] += 1.0
    B.kvs_cache_truncate(new, torch.from_numpy(accepted).cuda(), page, g["table"], g["n"], g["free"], g["weight"])
    O.truncate(c, new, accepted, page)
    same(c, g, "truncate")
    # all join and all leave: as before, but for the stale part of the tables
    g = on_gpu(start)
    B.kvs_cache_append_tokens(kn, vn, g["table"], g["n"], g["free"], kc, vc)
    B.kvs_cache_truncate(new, torch.zeros(S, dtype=torch.int32, device="cuda"), page, g["table"], g["n"], g["free"])
    start["table"] = g["table"].cpu().numpy()
    same(start, g, "there and back")


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 1 << 15])                     # by one launch and by two
def test_tokens_join_all_or_none(d):
    rng = np.random.default_rng(8)
    c = make(rng, [3, 8], 4, 4, spare=4)                        # the call needs 4 pages
    kn = torch.ones((2, 6, 1, d), device="cuda").bfloat16()
    kc = torch.zeros((len(c["free"]) - 4, 4, 1, d), device="cuda").bfloat16()
    for spoil, code in ((lambda x: None, B.KVS_OK), (lambda x: x["free"].__setitem__(0, 3), B.KVS_ERR_WORKSPACE),
                        (lambda x: x["n"].__setitem__(1, 11), B.KVS_ERR_WORKSPACE), (lambda x: x["n"].__setitem__(0, -1), B.KVS_ERR_INVALID_ARG),
                        (lambda x: x["n"].__setitem__(0, 17), B.KVS_ERR_INVALID_ARG), (lambda x: x["free"].__setitem__(0, 99), B.KVS_ERR_INVALID_ARG)):
        bad = copy.deepcopy(c)
        spoil(bad)
        g, k = on_gpu(bad), kc.clone()
        B.kvs_cache_append_tokens(kn, kn, g["table"], g["n"], g["free"], k, k.clone())
        assert int(g["free"][1]) == code
        if code:
            assert not k.any() and int(g["free"][0]) == bad["free"][0]
            assert np.array_equal(g["n"].cpu().numpy(), bad["n"]) and np.array_equal(g["table"].cpu().numpy(), bad["table"])
        else:
            assert g["n"].tolist() == [9, 14] and int(g["free"][0]) == 0


@pytest.mark.gpu
def test_counts_that_make_no_sense_drop_nothing():
    rng = np.random.default_rng(9)
    c = make(rng, [9, 9, 9, 2], 4, 4)
    g = on_gpu(c)
    B.kvs_cache_truncate(3, torch.tensor([-1, 4, 1, 0], dtype=torch.int32, device="cuda"), 4, g["table"], g["n"], g["free"], g["weight"])
    assert int(g["free"][1]) == B.KVS_ERR_INVALID_ARG and g["n"].tolist() == [9, 9, 7, 2] and int(g["free"][0]) == 3 + 1
