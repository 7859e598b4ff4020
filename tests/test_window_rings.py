"""kvs_decode_attn_window: CTAs that take many tiles, so that every buffer of K and of V is used again and again and a CTA goes from head to head
in mid-ring, in all of its forms: heads of 64 and 128, up to 16, 32 and 64 columns, pages by boxes and rows one by one.  With num_splits = 1
a CTA's share is all tiles of the longest head but one."""
import numpy as np
import pytest
import torch

from oracle import bounded_cache as O
from paper_2609_35750_b200 import binding as B

from .test_window_and_weights import ALL, Cache, bounds, check_window, close, queries

pytestmark = pytest.mark.gpu

COLUMNS = {16: (8, 2, 3), 32: (10, 2, 5), 64: (14, 2, 5)}          # Hq, Hkv, new tokens: 12, 25 and 35 columns


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("columns", COLUMNS)
@pytest.mark.parametrize("page", [16, 1, 3, 128])
@pytest.mark.parametrize("window,sinks", [(ALL, 0), (1500, 200)])
def test_many_tiles_a_cta(d, columns, page, window, sinks):
    Hq, Hkv, new = COLUMNS[columns]
    lens = [3000, 130, 2500, 0, 1153]
    c = Cache([d, columns, page], lens, page, Hkv, d)
    q = queries(1, len(lens), new, Hq, d)
    check_window(c, q, window, sinks, *B.kvs_decode_attn_window(q[0], *c.args(), window, sinks, num_splits=1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("columns", COLUMNS)
@pytest.mark.parametrize("page", [16, 1])
def test_values_that_are_not_finite_in_a_buffer_used_before(d, columns, page):
    """The window's edge and the last tokens lie many tiles into a share: rows that some queries see and others do not are infinite, rows
    behind the window NaN, in the tiles of one head; the other head of the same CTA is finite throughout."""
    Hq, Hkv, new = COLUMNS[columns]
    lens, window, sinks = [2900, 2300], 1700, 3
    c = Cache([d, page], lens, page, Hkv, d)
    for s, n in enumerate(lens):
        at = lambda t: (c.table[s, t // page], t % page, 0)  # noqa: E731
        for t in range(sinks, n - new + 1 - window):
            c.k[at(t)] = np.nan
            c.v[at(t)] = np.inf if t % 2 else np.nan
        c.v[at(n - window - 1)] = np.inf                            # seen by all but the last query
        c.v[at(n - 2)] = -np.inf                                    # seen by the last two
        c.v[at(n - 1)][::2] = np.nan                                # seen by the last alone
    c.round()
    gq, fq = queries(2, 2, new, Hq, d)
    out, lse = B.kvs_decode_attn_window(gq, *c.args(), window, sinks, num_splits=1)
    for s, n in enumerate(lens):
        k, v = c.rows(s)
        sees = O.visible(n, new, window, sinks)
        wo, wl, p = O.attention(fq[s], np.nan_to_num(k), v, sees, d ** -0.5)          # the NaN keys are seen by none
        tame = lambda x: np.nan_to_num(x, posinf=0.0, neginf=0.0)  # noqa: E731
        tol, delta = bounds(fq[s], tame(k), tame(v), sees, p, tame(wo), d ** -0.5)
        close(out[s], wo, tol, (s, n, "out"))
        close(lse[s], wl, delta + 2.0 ** -22 * np.abs(wl), (s, n, "lse"))
        assert np.isinf(wo).any() and np.isnan(wo).any() and np.isfinite(wo[:, Hq // Hkv:]).all()


@pytest.mark.parametrize("Hq,Hkv,new", [(8, 2, 1), (28, 4, 3)])
@pytest.mark.parametrize("page", [16, 1])
def test_more_sequences_than_lanes_with_heads_of_128(Hq, Hkv, new, page):
    """More than 32 sequences: the shares are found by the whole CTA."""
    rng = np.random.default_rng([Hq, page])
    lens = rng.integers(0, 300, size=48).tolist()
    lens[5], lens[40] = 2600, 0
    c = Cache([3, page], lens, page, Hkv, 128)
    q = queries(4, len(lens), new, Hq, 128)
    for splits in (0, 1):
        check_window(c, q, 900, 4, *B.kvs_decode_attn_window(q[0], *c.args(), 900, 4, num_splits=splits))
