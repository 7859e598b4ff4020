"""Plain numpy statements (64 bits) of the rollout engine's operators on bounded caches and drafted tokens.

Test infrastructure: nothing of the library is used here.  A cache is a dict of numpy arrays as the library keeps them:
table int32 [S, P], n int32 [S], free int32 [4 + num_pages] ({top, ...}, then the stack), weight fp32 [S, P * page].
"""
import numpy as np


def visible(n, new, window, sinks):
    """bool [new, n]: which of the n live tokens query t of the `new` last ones sees."""
    at = (n - new + np.arange(new))[:, None]
    j = np.arange(n)[None]
    return (j <= at) & ((j < sinks) | (at - j < window))


def rows_of(pool, table, n, page):
    """The first n live rows [n, Hkv, d] that a table row names."""
    t = np.arange(n)
    return pool[table[t // page], t % page]


def attention(q, k, v, sees, scale):
    """q [new, Hq, d], k, v [n, Hkv, d], sees [new, n] -> (out [new, Hq, d], lse [new, Hq], weights [new, Hq, n]) in float64."""
    new, Hq, d = q.shape
    G = Hq // k.shape[1]
    out, lse, p = np.zeros((new, Hq, d)), np.full((new, Hq), -np.inf), np.zeros((new, Hq, k.shape[0]))
    for t in range(new):
        keys = np.flatnonzero(sees[t])
        if not len(keys):
            continue
        for h in range(Hq):
            s = (k[keys, h // G].astype(np.float64) @ q[t, h].astype(np.float64)) * scale
            top = s.max()
            e = np.exp(s - top)
            lse[t, h] = top + np.log(e.sum())
            p[t, h, keys] = e / e.sum()
            out[t, h] = p[t, h, keys] @ v[keys, h // G].astype(np.float64)
    return out, lse, p


def scores(weight, live, page):
    """Page scores: the tokens' weights added in 64 bits, rounded to 32; NaN above everything."""
    with np.errstate(invalid="ignore"):
        x = weight[:live * page].reshape(live, page).astype(np.float64).sum(axis=1).astype(np.float32)
    return x


def evict_lowest(cache, budget, keep_first, keep_recent, page):
    """In place; returns (evicted int32 [S, P], n_evicted int32 [S])."""
    S, P = cache["table"].shape
    evicted, count, back = np.full((S, P), -1, np.int32), np.zeros(S, np.int32), []
    for s in range(S):
        n = int(cache["n"][s])
        live = -(-n // page)
        may = [i for i in range(live) if i * page >= keep_first and (i + 1) * page <= n - keep_recent]
        take = min(max(0, -(-(n - budget) // page)), len(may))
        x = scores(cache["weight"][s], live, page)
        gone = sorted(sorted(may, key=lambda i: (bool(np.isnan(x[i])), 0.0 if np.isnan(x[i]) else float(x[i]), i))[:take])
        stay = [i for i in range(live) if i not in set(gone)]
        back += [int(cache["table"][s, i]) for i in gone]
        evicted[s, :take], count[s] = gone, take
        rows = cache["weight"][s, :live * page].reshape(live, page)[stay].copy()
        cache["table"][s, :len(stay)] = cache["table"][s, stay]
        cache["weight"][s, :live * page] = 0.0
        cache["weight"][s, :len(stay) * page] = rows.ravel()
        cache["n"][s] = n - take * page
    push(cache, back)
    return evicted, count


def push(cache, pages):
    """Pages back on the stack, the last of the list first."""
    top = int(cache["free"][0])
    cache["free"][4 + top:4 + top + len(pages)] = pages[::-1]
    cache["free"][0] = top + len(pages)


def append_tokens(cache, new, page, active=None):
    """Lengths, tables and stack after `new` tokens joined; returns the (page, row) of every token of every active sequence, or None
    where the call is not begun."""
    S, P = cache["table"].shape
    on = [s for s in range(S) if active is None or active[s]]
    need = [-(-(int(cache["n"][s]) + new) // page) - -(-int(cache["n"][s]) // page) for s in on]
    if sum(need) > int(cache["free"][0]) or any(int(cache["n"][s]) + new > P * page for s in on):
        return None
    places = {}
    for s in on:
        places[s] = []
        for t in range(int(cache["n"][s]), int(cache["n"][s]) + new):
            if t % page == 0:
                cache["free"][0] -= 1
                cache["table"][s, t // page] = cache["free"][4 + cache["free"][0]]
            places[s].append((int(cache["table"][s, t // page]), t % page))
        cache["n"][s] += new
    return places


def truncate(cache, n_drafted, n_accepted, page):
    back = []
    for s in range(len(cache["n"])):
        n, left = int(cache["n"][s]), int(cache["n"][s]) - (n_drafted - int(n_accepted[s]))
        back += [int(x) for x in cache["table"][s, -(-left // page):-(-n // page)]]
        if "weight" in cache:
            cache["weight"][s, left:n] = 0.0
        cache["n"][s] = left
    push(cache, back)


def verify(target, draft, drafted, u_accept, u_sample):
    """Returns (tokens int32 [S, n + 1], n_accepted int32 [S])."""
    S, n, V = draft.shape
    tokens, count = np.full((S, n + 1), -1, np.int32), np.zeros(S, np.int32)
    wide = lambda x: np.asarray(x, dtype=np.float64)  # noqa: E731
    for s in range(S):
        r = 0
        while r < n and 0 <= drafted[s, r] < V and wide(u_accept[s, r]) * wide(draft[s, r, drafted[s, r]]) < wide(target[s, r, drafted[s, r]]):
            r += 1
        own = np.maximum(np.nan_to_num(wide(target[s, r]), nan=0.0), 0.0)
        w = own
        if r < n:
            with np.errstate(invalid="ignore"):
                w = np.maximum(np.nan_to_num(wide(target[s, r]) - wide(draft[s, r]), nan=0.0), 0.0)
            if not w.sum() > 0:
                w = own
        run = np.cumsum(w)
        k = -1
        if run[-1] > 0:
            over = np.flatnonzero((w > 0) & (run > wide(u_sample[s]) * run[-1]))
            k = int(over[0]) if len(over) else int(np.flatnonzero(w > 0)[-1])
        tokens[s, :r], tokens[s, r], count[s] = drafted[s, :r], k, r
    return tokens, count
