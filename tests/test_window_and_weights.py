"""Attention over the paged cache with a window and first tokens that stay visible, and attention that accumulates its weights,
against the plain statements in 64 bits.

Tolerances, per element, from the arithmetic alone.  Scores are sums of d products of bf16 numbers in fp32: off by no more than
d 2^-23 sum |q_c k_c| scale (every addition may cut at the last bit), and a few roundings of the score itself; `delta` is that with
8 roundings.  A softmax weight is then off by a factor of exp(2 delta) at most (its own score's error and the normaliser's), the lse by
delta.  Weights are rounded to bf16 for the second product (off by 2^-8 of themselves), the result once more:
    |out - exact| <= (2^-8 + 2 delta (1 + ...)) sum_j p_j |v_j| + 2^-8 |out|,  written out in `bounds`."""
import numpy as np
import pytest
import torch

from oracle import bounded_cache as O
from paper_2609_35750_b200 import binding as B

ALL = 2 ** 31 - 1


def bounds(q, k, v, sees, p, out, scale):
    """(tolerance of out [new, Hq, d], delta [new, Hq])."""
    G = q.shape[1] // k.shape[1]
    a = np.einsum("thd,jhd->thj", np.abs(q), np.repeat(np.abs(k), G, axis=1)) * scale if k.shape[0] else np.zeros((*q.shape[:2], 1))
    seen = sees[:, None] if k.shape[0] else np.zeros((q.shape[0], 1, 1), bool)
    delta = (np.where(seen, a, 0.0).max(axis=2)) * (q.shape[2] + 8) * 2.0 ** -23 + 2.0 ** -20
    spread = np.einsum("thj,jhd->thd", p, np.repeat(np.abs(v), G, axis=1))
    return (2.0 ** -8 + 2.1 * delta[..., None] * (1 + 2.0 ** -8)) * spread + 2.0 ** -8 * np.abs(out) + 1e-30, delta


class Cache:
    """A cache built by hand: scattered pages, NaN in every row that no token was written to."""

    def __init__(self, seed, lens, page, Hkv, d, spare_pages=1):
        rng = np.random.default_rng(seed)
        S, self.page, self.lens = len(lens), page, lens
        used = [-(-n // page) for n in lens]
        pool = sum(used) + 3
        self.k = np.full((pool, page, Hkv, d), np.nan, np.float32)
        self.v = self.k.copy()
        self.table = rng.integers(0, pool, size=(S, max(used) + spare_pages)).astype(np.int32)
        order, at = rng.permutation(pool), 0
        for s, n in enumerate(lens):
            self.table[s, :used[s]] = order[at:at + used[s]]
            at += used[s]
            t = np.arange(n)
            self.k[self.table[s, t // page], t % page] = rng.normal(size=(n, Hkv, d))
            self.v[self.table[s, t // page], t % page] = rng.normal(size=(n, Hkv, d))
        self.n = np.array(lens, np.int32)
        self.round()

    def round(self):
        """What the library gets, bf16, and the same numbers for the statement."""
        self.gk, self.gv = (torch.from_numpy(x).bfloat16().cuda() for x in (self.k, self.v))
        self.k, self.v = (x.float().cpu().numpy() for x in (self.gk, self.gv))
        self.gt, self.gn = torch.from_numpy(self.table).cuda(), torch.from_numpy(self.n).cuda()

    def rows(self, s):
        return [O.rows_of(x, self.table[s], self.lens[s], self.page).astype(np.float64) for x in (self.k, self.v)]

    def args(self):
        return self.gk, self.gv, self.gt, self.gn


def queries(seed, *shape):
    q = (torch.from_numpy(np.random.default_rng(seed).normal(size=shape).astype(np.float32)) * 1.5).bfloat16()
    return q.cuda(), q.float().numpy().astype(np.float64)


def close(got, want, tol, what):
    got = got.double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), what
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)]), what
    err = np.abs(got - np.where(fine, want, 0.0))[fine]
    over = err - np.broadcast_to(tol, want.shape)[fine]
    assert not over.size or over.max() <= 0, (what, over.max(), err.max())


def check_window(c, q, window, sinks, out, lse, scale=None):
    gq, fq = q
    new = fq.shape[1]
    scale = scale or fq.shape[-1] ** -0.5
    for s, n in enumerate(c.lens):
        k, v = c.rows(s)
        sees = O.visible(n, new, window, sinks)
        wo, wl, p = O.attention(fq[s], k, v, sees, scale)
        tol, delta = bounds(fq[s], np.nan_to_num(k), np.nan_to_num(v), sees, p, np.nan_to_num(wo), scale)
        close(out[s], wo, tol, (s, n, "out"))
        close(lse[s], wl, delta + 2.0 ** -22 * np.abs(np.where(np.isfinite(wl), wl, 0.0)), (s, n, "lse"))


# ---- CPU ---------------------------------------------------------------------------------------------------------
def test_visible_by_hand():
    assert O.visible(6, 2, 3, 1).astype(int).tolist() == [[1, 0, 1, 1, 1, 0], [1, 0, 0, 1, 1, 1]]
    assert O.visible(1, 2, 3, 1).astype(int).tolist() == [[0], [1]]
    assert O.visible(4, 1, ALL, 0).all() and not O.visible(0, 2, 5, 9).size


def test_plain_attention_is_the_trainers_on_a_window_mask():
    """The trainer's mask of the same rule: evict_at[j] = j + window, never for the first ones."""
    from oracle import kvs_oracle as K
    rng = np.random.default_rng(3)
    T, window, sinks = 40, 7, 3
    q, k, v = (rng.normal(size=(T, h, 8)) for h in (4, 2, 2))
    evict = np.where(np.arange(T) < sinks, ALL, np.arange(T) + window).astype(np.int64)
    want, lse = K.dense_fwd(q, k, v, evict, 0.3)
    got, m, _ = O.attention(q, k, v, O.visible(T, T, window, sinks), 0.3)
    assert np.abs(got - want).max() < 1e-12 and np.abs(m.T - lse).max() < 1e-12


@pytest.fixture(scope="module")
def lib():
    from paper_2609_35750_b200 import build
    build.build()
    return B.load()


def test_host_refusals_need_no_gpu(lib):
    p = 1 << 20

    def window(S=1, new=1, Hq=4, Hkv=2, d=64, page=1, P=4, pool=4, scale=0.0, w=5, sinks=0, splits=1, q=p, ws=p, room=1 << 20):
        return lib.kvs_decode_attn_window(q, p, p, p, p, S, new, Hq, Hkv, d, page, P, pool, scale, w, sinks, splits, p, p, ws, room, None)

    assert window(S=-1) == window(new=-1) == window(Hq=0) == window(Hkv=0) == window(page=0) == window(P=0) == window(pool=0) == B.KVS_ERR_INVALID_ARG
    assert window(w=0) == window(sinks=-1) == window(splits=0) == window(scale=-1.0) == window(scale=float("nan")) == window(q=None) == B.KVS_ERR_INVALID_ARG
    assert window(d=96) == window(Hq=5) == window(Hq=130) == window(page=1 << 16, pool=1 << 16) == window(page=1 << 16, P=1 << 16) == B.KVS_ERR_UNSUPPORTED
    assert window(S=1 << 30) == window(new=1 << 29) == B.KVS_ERR_UNSUPPORTED
    assert window(q=p + 8) == window(ws=p + 128) == B.KVS_ERR_ALIGNMENT and window(room=256) == B.KVS_ERR_WORKSPACE
    assert window(S=0, q=None) == window(new=0) == B.KVS_OK

    def weights(S=1, Hq=4, d=64, most=8, w=p, room=1 << 20):
        return lib.kvs_decode_attn_weights(p, p, p, p, p, S, Hq, 2, d, 1, 8, 8, 0.0, 1, most, p, p, w, p, room, None)

    assert weights(most=0) == weights(w=None) == B.KVS_ERR_INVALID_ARG and weights(w=p + 2) == B.KVS_ERR_ALIGNMENT
    assert weights(Hq=1 << 14) == weights(d=80) == B.KVS_ERR_UNSUPPORTED
    assert weights(room=lib.kvs_decode_weights_workspace_bytes(1, 4, 64, 1, 8) - 1) == B.KVS_ERR_WORKSPACE
    assert weights(S=0, w=None) == B.KVS_OK
    assert lib.kvs_decode_weights_workspace_bytes(1, 4, 64, 1, 0) == 0 and lib.kvs_decode_weights_workspace_bytes(1, 0, 64, 1, 5) == 0
    assert lib.kvs_decode_weights_workspace_bytes(3, 8, 128, 2, 129) == lib.kvs_decode_workspace_bytes(3, 8, 128, 2) + 3 * 8 * 256 * 4


def test_split_counts(lib):
    n = lib.kvs_decode_window_num_splits
    assert n(0, 1, 8, 8, 100, 5, 0) == n(1, 1, 8, 8, 100, 0, 0) == n(1, 1, 130, 1, 100, 5, 0) == 1
    for args in ((1, 1, 32, 8, 100000, ALL, 0), (64, 5, 28, 4, 9000, 4096, 4), (4, 1, 16, 2, 700, 256, 4), (1, 8, 64, 1, 300000, ALL, 64)):
        S, new, Hq, Hkv, most, window, sinks = args
        tiles = min(-(-most // 128), -(-sinks // 128) + (window + new + 126) // 128 + 1)
        assert 1 <= n(*args) <= max(1, tiles), args


def test_host_tensors_and_untracked_caches_are_refused(lib):
    kv, i = torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16), torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        B.kvs_decode_attn_window(kv, kv, kv, i, i[0, :1], 4)
    with pytest.raises(ValueError, match="CUDA"):
        B.kvs_decode_attn_weights(kv[0], kv, kv, i, i[0, :1], torch.zeros((1, 4)))
    with pytest.raises(ValueError, match="dimensions"):
        B.kvs_decode_attn_window(kv[0], kv, kv, i, i[0, :1], 4)


# ---- GPU: window -------------------------------------------------------------------------------------------------
SHAPES = [(4, 4, 64, 16, 1), (16, 4, 64, 1, 3), (16, 2, 128, 16, 1), (28, 4, 128, 16, 5), (8, 2, 128, 1, 8), (8, 1, 128, 64, 7), (6, 2, 128, 3, 2), (5, 1, 64, 256, 4),
          (64, 1, 128, 8, 2), (3, 3, 64, 128, 11), (32, 2, 64, 32, 4), (24, 1, 128, 1, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d,page,new", SHAPES)
@pytest.mark.parametrize("window,sinks", [(ALL, 0), (1, 0), (100, 4), (300, 130), (128, 0), (5000, 9)])
def test_window_matches_the_plain_statement(Hq, Hkv, d, page, new, window, sinks):
    lens = [0, 1, 2, 127, 128, 130, 257, 700, 1100]
    c = Cache([Hq, page, new], lens, page, Hkv, d)
    q = queries(1, len(lens), new, Hq, d)
    for splits in (0, 3):
        check_window(c, q, window, sinks, *B.kvs_decode_attn_window(q[0], *c.args(), window, sinks, num_splits=splits))


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d,page,new", [(8, 2, 128, 16, 5), (8, 2, 128, 1, 5), (4, 4, 64, 16, 3), (4, 1, 64, 2, 6), (28, 2, 128, 8, 4)])
@pytest.mark.parametrize("splits", [1, 4])
def test_what_a_query_does_not_see_does_not_reach_it(Hq, Hkv, d, page, new, splits):
    """NaN and infinities outside the window, at its edge, and in the drafted tokens: each query as if the hidden ones were not there."""
    lens, window, sinks = [3, 260, 515, 900], 200, 5
    c = Cache([page, new], lens, page, Hkv, d)
    for s, n in enumerate(lens):
        put = lambda x, t, value: x.__setitem__((c.table[s, t // page], t % page), value)  # noqa: E731
        for t in range(sinks, n - new + 1 - window):                  # seen by none
            put(c.k, t, np.nan if t % 2 else np.inf)
            put(c.v, t, np.nan if t % 3 else -np.inf)
        if n > window + new:
            put(c.v, n - window - 1, np.inf)                          # the window's edge: seen by all but the last
            put(c.v, n - window - 2, -np.inf)
        c.v[c.table[s, (n - 1) // page], (n - 1) % page, :, ::2] = np.nan          # the last token: seen by the last query alone
        if s == 2:
            put(c.k, n - 2, np.nan)
    c.round()
    q = queries(2, len(lens), new, Hq, d)
    out, lse = B.kvs_decode_attn_window(q[0], *c.args(), window, sinks, num_splits=splits)
    for s, n in enumerate(lens):
        # a NaN score makes its whole row NaN, which the statement's sums say too; lse of such a row is not compared
        k, v = c.rows(s)
        sees = O.visible(n, new, window, sinks)
        wo, wl, p = O.attention(q[1][s], k, v, sees, d ** -0.5)
        tol, delta = bounds(q[1][s], np.nan_to_num(k, posinf=0.0), np.nan_to_num(v, posinf=0.0, neginf=0.0), sees, np.nan_to_num(p), np.nan_to_num(wo, posinf=0.0, neginf=0.0), d ** -0.5)
        fine = np.isfinite(wl) | np.isneginf(wl)
        for t in range(new):
            if fine[t].all():
                close(out[s, t], wo[t], tol[t], (s, t))
                close(lse[s, t], wl[t], delta[t] + 1e-6 * np.abs(np.nan_to_num(wl[t], neginf=0.0)), (s, t))
            else:
                assert torch.isnan(out[s, t]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("S,new,Hq,Hkv", [(900, 1, 4, 2), (40, 30, 64, 1)])
def test_more_sequences_and_groups_than_a_cta_has_threads(S, new, Hq, Hkv):
    """The shares are found by several passes over the lengths; most sequences are empty or short, a few are long."""
    rng = np.random.default_rng(S)
    lens = np.where(rng.random(S) < 0.4, 0, rng.integers(1, 60, size=S))
    lens[[0, S // 2, S - 1]] = [0, 400, 150]
    c = Cache(11, lens.tolist(), 8, Hkv, 64)
    q = queries(12, S, new, Hq, 64)
    check_window(c, q, 100, 3, *B.kvs_decode_attn_window(q[0], *c.args(), 100, 3))
    for n in (0, 33):                                           # nothing live anywhere; all alike
        c = Cache(13, [n] * S, 8, Hkv, 64)
        check_window(c, q, 20, 0, *B.kvs_decode_attn_window(q[0], *c.args(), 20))


@pytest.mark.gpu
def test_scores_far_apart_and_scale():
    """References that have to move by hundreds, in both directions, and an explicit scale."""
    c = Cache(5, [640, 333], 16, 2, 128)
    grow = np.linspace(0.1, 12, 640)[:, None, None]
    for s, n in enumerate(c.lens):
        t = np.arange(n)
        c.k[c.table[s, t // 16], t % 16] *= grow[:n] if s == 0 else grow[:n][::-1]
    c.round()
    q = queries(6, 2, 3, 8, 128)
    for window in (ALL, 250):
        check_window(c, q, window, 2, *B.kvs_decode_attn_window(q[0], *c.args(), window, 2, softmax_scale=0.3, num_splits=2), scale=0.3)


@pytest.mark.gpu
def test_window_on_a_trace_is_the_trainers_forward():
    """A trace generated chunk by chunk under a window with sinks has the rows of the trainer's forward under the mask of the same rule."""
    T, new, Hq, Hkv, d, window, sinks = 600, 6, 8, 2, 128, 150, 4
    q, k, v = (torch.randn((T, h, d), device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
    cache = B.PagedCache(40, 16, 1, 40, Hkv, d)
    rows = []
    for t in range(0, T, new):
        cache.append_tokens(k[None, t:t + new], v[None, t:t + new])
        rows.append(cache.decode_window(q[None, t:t + new], window, sinks))
    j = torch.arange(T, device="cuda", dtype=torch.int32)
    evict = torch.where(j < sinks, torch.tensor(ALL, device="cuda", dtype=torch.int32), j + window)
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    out, lse = B.kvs_attn_fwd(q, k, v, B.kvs_mask_meta(evict, cu, T), 1, T)
    got = torch.cat([r[0][0] for r in rows]).float()
    # either is off by 2^-8 of sum p |v| (at most max |v|) and 2^-8 of itself
    assert (got - out.float()).abs().max() <= 4 * 2.0 ** -8 * float(v.float().abs().max())
    assert (torch.cat([r[1][0] for r in rows]).T - lse).abs().max() < 1e-4


@pytest.mark.gpu
def test_bad_pages_are_recorded_and_not_followed():
    c = Cache(7, [300, 40], 16, 2, 128)
    c.gt[0, 3], c.gt[1, 1] = 10 ** 6, -1
    for call in (lambda ws: B.kvs_decode_attn_window(queries(1, 2, 2, 4, 128)[0], *c.args(), 5000, workspace=ws, num_splits=2),
                 lambda ws: B.kvs_decode_attn_weights(queries(1, 2, 4, 128)[0], *c.args(), torch.zeros((2, c.table.shape[1] * 16), device="cuda"), workspace=ws, num_splits=2)):
        ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        call(ws)
        assert B.kvs_device_status(ws) == B.KVS_ERR_INVALID_ARG
        c.gt.copy_(torch.from_numpy(c.table))
        call(ws)
        assert B.kvs_device_status(ws) == B.KVS_OK
        c.gt[0, 3] = -7


# ---- GPU: weights ------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d,page", [(4, 4, 64, 16), (16, 4, 64, 1), (16, 2, 128, 16), (28, 4, 128, 1), (8, 4, 128, 16), (3, 3, 128, 1), (8, 8, 128, 32), (7, 1, 64, 5), (64, 8, 128, 8)])
@pytest.mark.parametrize("splits", [1, 5])
def test_weights_match_the_plain_statement(Hq, Hkv, d, page, splits):
    lens = [0, 1, 15, 128, 129, 1000, 1500]
    c = Cache([Hq, page], lens, page, Hkv, d)
    room = c.table.shape[1] * page
    start = np.random.default_rng(9).random((len(lens), room)).astype(np.float32)
    weight = torch.from_numpy(start).cuda()
    q = queries(3, len(lens), Hq, d)
    out, lse = B.kvs_decode_attn_weights(q[0], *c.args(), weight, num_splits=splits, max_tokens=1500)
    plain = B.PagedCache.__new__(B.PagedCache)                          # the same rows as without weights
    plain.__dict__.update(Hkv=Hkv, page_size=page, max_pages=c.table.shape[1], num_pages=c.gk.shape[0], block_table=c.gt, n_tokens=c.gn, k_cache=c.gk, v_cache=c.gv)
    o2, l2 = plain.decode(q[0], num_splits=splits)
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    want = start.astype(np.float64)
    tol = np.zeros_like(want)
    for s, n in enumerate(lens):
        k, v = c.rows(s)
        sees = np.ones((1, n), bool)
        wo, wl, p = O.attention(q[1][s][None], k, v, sees, d ** -0.5)
        bound, delta = bounds(q[1][s][None], k, v, sees, p, wo, d ** -0.5)
        close(out[s][None], wo, bound, (s, "out"))
        close(lse[s][None], wl, delta + 2.0 ** -22 * np.abs(np.where(np.isfinite(wl), wl, 0.0)), (s, "lse"))
        want[s, :n] += p[0].sum(axis=0)
        # a head's weight: its score's and the lse's error, exp2 and its argument; then Hq + 1 additions
        tol[s, :n] = (p[0] * (2.1 * delta[0][:, None] + 2.0 ** -19)).sum(axis=0) + (Hq + 1) * 2.0 ** -24 * want[s, :n]
    err = np.abs(weight.double().cpu().numpy() - want)
    assert (err <= tol).all(), (err - tol).max()
    # sums in a fixed order: the same bits again
    again = torch.from_numpy(start).cuda()
    B.kvs_decode_attn_weights(q[0], *c.args(), again, num_splits=splits, max_tokens=1500)
    assert torch.equal(again, weight)


@pytest.mark.gpu
@pytest.mark.parametrize("page", [1, 16])
def test_a_sequence_longer_than_said_keeps_its_weights(page):
    c = Cache(4, [200, 1000], page, 2, 128)
    q = queries(4, 2, 8, 128)
    weight = torch.zeros((2, c.table.shape[1] * page), device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    out, _ = B.kvs_decode_attn_weights(q[0], *c.args(), weight, max_tokens=256, workspace=ws, num_splits=2)
    assert B.kvs_device_status(ws) == B.KVS_ERR_INVALID_ARG
    assert not weight[1].any() and abs(float(weight[0].sum()) - 8) < 1e-4
    full, _ = B.kvs_decode_attn_weights(q[0], *c.args(), weight, workspace=ws, num_splits=2)
    assert torch.equal(out, full) and B.kvs_device_status(ws) == B.KVS_OK


@pytest.mark.gpu
@pytest.mark.parametrize("page", [16, 1])
def test_rows_far_into_a_large_cache(page):
    """Rows beyond 2^31 elements: the last pages of a cache of 2.2e9 elements a side, written and read."""
    Hkv, d, n, new = 8, 128, 300, 3
    pages = 2_200_000 // page
    k = torch.zeros((pages, page, Hkv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    need = -(-n // page)
    table = torch.arange(pages - need, pages, dtype=torch.int32, device="cuda").flip(0).view(1, -1).contiguous()
    free = torch.cat((torch.tensor([need, 0, 0, 0], dtype=torch.int32, device="cuda"), table[0].flip(0), torch.zeros(pages - need, dtype=torch.int32, device="cuda")))
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows_k, rows_v = (torch.randn((1, n, Hkv, d), device="cuda").bfloat16() for _ in range(2))
    for a, z in ((0, 290), (290, 297), (297, 300)):               # many rows, few rows
        B.kvs_cache_append_tokens(rows_k[:, a:z].contiguous(), rows_v[:, a:z].contiguous(), table, lens, free, k, v)
    assert lens.tolist() == [n] and free[:2].tolist() == [0, B.KVS_OK]
    q, fq = queries(1, 1, new, 16, d)
    c = Cache.__new__(Cache)
    c.lens, c.page, c.table = [n], page, np.zeros((1, 0))
    c.rows = lambda s: [x[0].float().cpu().numpy().astype(np.float64) for x in (rows_k, rows_v)]
    check_window(c, (q, fq), 200, 4, *B.kvs_decode_attn_window(q, k, v, table, lens, 200, 4))
    weight = torch.zeros((1, need * page), device="cuda")
    out, lse = B.kvs_decode_attn_weights(q[:, -1].contiguous(), k, v, table, lens, weight)
    check_window(c, (q[:, -1:], fq[:, -1:]), ALL, 0, out[:, None], lse[:, None])
    assert abs(float(weight.sum()) - 16) < 1e-3


# ---- GPU: together -----------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("page", [1, 16])
def test_a_rollout_that_evicts_by_weight_is_the_trainers_masked_forward(page):
    """Generate token by token, evict by weight every 32 tokens; the slots that left give the trainer's evict_at, and the masked forward
    on the whole trace has the rollout's rows."""
    T, Hq, Hkv, d, prompt = 448, 8, 2, 128, 64
    q, k, v = (torch.randn((T, h, d), device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
    q[:, :, :8] *= 3
    cache = B.PagedCache(200 // page + 40, page, 1, 320 // page, Hkv, d, track_weights=True)
    with pytest.raises(ValueError, match="evict_lowest"):
        cache.evict(torch.zeros((1, 3), dtype=torch.int32, device="cuda"))
    cache.append_tokens(k[None, :prompt], v[None, :prompt])
    live, evict_at, rows = list(range(prompt)), np.full(T, ALL, np.int64), {}
    for t in range(prompt, T):
        if t % 32 == 0:
            evicted, count = cache.evict_lowest(128, keep_first=16, keep_recent=48)
            gone = [live[i] for sl in evicted[0, :int(count)].tolist() for i in range(sl * page, (sl + 1) * page)]
            evict_at[gone] = t
            live = [j for j in live if evict_at[j] > t]
            assert len(live) == int(cache.n_tokens[0]) and (len(live) <= 128)
        cache.append(k[t:t + 1], v[t:t + 1])
        live.append(t)
        rows[t] = cache.decode_weights(q[t:t + 1])
    assert (evict_at < ALL).sum() > 200 and cache.status()[0] == B.KVS_OK
    assert (cache.token_weight[0, :len(live) - 1] > 0).all() and not cache.token_weight[0, len(live):].any()
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    out, lse = B.kvs_attn_fwd(q, k, v, B.kvs_mask_meta(torch.from_numpy(evict_at.astype(np.int32)).cuda(), cu, T), 1, T)
    for t, (o, m) in rows.items():
        assert (o[0].float() - out[t].float()).abs().max() <= 4 * 2.0 ** -8 * float(v.float().abs().max())
        assert (m[0] - lse[:, t]).abs().max() < 1e-4


@pytest.mark.gpu
def test_rounds_of_drafted_tokens_leave_what_token_by_token_generation_leaves():
    """Drafts join, attend, are verified and the rejected ones leave; a second cache gets the kept tokens one by one."""
    S, n, Hq, Hkv, d, V, page = 3, 4, 4, 2, 64, 50, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    a, b = (B.PagedCache(200, page, S, 60, Hkv, d) for _ in range(2))
    emb_k, emb_v = (torch.randn((V, Hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    last = torch.zeros(S, dtype=torch.int32, device="cuda")
    kept = [[] for _ in range(S)]
    for _ in range(9):
        logits = torch.randn((S, n + 1, V), generator=g, device="cuda") * 2
        target, draft = torch.softmax(logits, -1), torch.softmax(logits[:, :n] + 0.5 * torch.randn((S, n, V), generator=g, device="cuda"), -1)
        drafts = torch.multinomial(draft.view(-1, V), 1, generator=g).view(S, n).int()
        toks = torch.cat((last[:, None], drafts), 1).long()
        a.append_tokens(emb_k[toks], emb_v[toks])
        a.decode_window(torch.randn((S, n + 1, Hq, d), generator=g, device="cuda").bfloat16(), ALL)
        tokens, accepted = B.kvs_verify_drafts(target, draft, drafts, torch.rand((S, n), generator=g, device="cuda"), torch.rand(S, generator=g, device="cuda"))
        a.truncate(n, accepted)
        for s, m in enumerate(accepted.tolist()):
            kept[s] += [int(last[s])] + drafts[s, :m].tolist()
            last[s] = tokens[s, m]
    for t in range(max(map(len, kept))):
        now = torch.tensor([x[min(t, len(x) - 1)] for x in kept], device="cuda")
        b.append(emb_k[now], emb_v[now], torch.tensor([t < len(x) for x in kept], dtype=torch.uint8, device="cuda"))
    assert a.n_tokens.tolist() == b.n_tokens.tolist() == [len(x) for x in kept]
    assert a.status() == (B.KVS_OK, 200 - sum(-(-len(x) // page) for x in kept))
    q = torch.randn((S, 1, Hq, d), generator=g, device="cuda").bfloat16()
    for x, y in zip(a.decode_window(q, 17, 2, num_splits=2), b.decode_window(q, 17, 2, num_splits=2)):
        assert torch.equal(x, y)


@pytest.mark.gpu
def test_a_captured_round_and_a_captured_step_replay():
    """Two graphs of calls with workspaces of their own, replayed in turn; and calls on a given stream."""
    S, n, Hq, Hkv, d, page = 2, 3, 8, 2, 128, 16
    make = lambda: B.PagedCache(60, page, S, 30, Hkv, d, track_weights=True)  # noqa: E731
    k, v = (torch.randn((S, 100, Hkv, d), device="cuda").bfloat16() for _ in range(2))
    q, q1 = torch.randn((S, n, Hq, d), device="cuda").bfloat16(), torch.randn((S, Hq, d), device="cuda").bfloat16()
    none = torch.zeros(S, dtype=torch.int32, device="cuda")

    def round_(c):
        c.append_tokens(k[:, :n].contiguous(), v[:, :n].contiguous())
        got = c.decode_window(q, 60, 4)
        c.truncate(n - 1, none)
        return got

    def step(c):
        got = c.decode_weights(q1)
        return (*got, c.evict_lowest(70, 4, 8)[1])

    caches = [make() for _ in range(3)]
    for c in caches:
        c.append_tokens(k, v)
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                         # the library's first calls, not captured
        round_(caches[1])
        step(caches[1])
    torch.cuda.current_stream().wait_stream(side)
    for f in (round_, step):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(f(caches[0]))
        graphs.append(gr)
    for _ in range(3):
        for gr, f, got in zip(graphs, (round_, step), outs):
            gr.replay()
            want = f(caches[2])
            for x, y in zip(got, want):
                assert torch.equal(x, y)
    for name in ("n_tokens", "token_weight", "free_list"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[2], name)), name
    torch.cuda.synchronize()
    got = caches[0].decode_window(q, 60, 4, stream=side)
    side.synchronize()
    for x, y in zip(got, caches[2].decode_window(q, 60, 4)):
        assert torch.equal(x, y)
    for x, y in zip(got, caches[2].decode_window(q, 60, 4, stream=torch.cuda.default_stream())):
        assert torch.equal(x, y)
