"""The operators of the rollout engine's bounded caches and drafted tokens, as cases that can be timed and compared.

A case is a dict of plain values; `kind` says which operator:

  window    attention of one or several new tokens per sequence over the paged cache, with a sliding window and a few first
            tokens that stay visible
  weights   attention of one new token that also adds every live token's softmax weight to its accumulator
  evict     the tokens with the lowest accumulated weight leave the cache, whole pages at a time, until it holds its budget
  verify    which drafted tokens the target's probabilities keep, and the token after them, from given random numbers
  round     a round of drafted tokens as the engine sees it: their K and V rows join the cache, they attend, they leave again

`own` false: elementary torch operations in 32 bits (64 where sums or comparisons need them); `own` true: the library's calls.
Cache lengths are a function of the case; page tables, random numbers and all values are drawn from the seed.
"""
import math

import numpy as np
import torch

own = False

# (query heads, KV heads, head_dim) of the models that the configurations describe, and one small one
HEADS = ((4, 4, 64), (16, 4, 64), (16, 2, 128), (28, 4, 128), (32, 8, 128), (64, 8, 128))
ALL = 2 ** 31 - 1                # a window that hides nothing
MOST_BYTES = 1.7e9               # a drawn case reads no more than the largest listed one


def listed():
    return [
        # one sequence of a windowed layer: latency and launches
        dict(name="window_one", kind="window", seqs=1, shortest=700, longest=700, page=16, Hq=16, Hkv=2, d=128, new=1, window=256, sinks=4),
        # a full rollout batch on a windowed layer, caches up to several windows long
        dict(name="window_batch", kind="window", seqs=64, shortest=2000, longest=30000, page=16, Hq=32, Hkv=8, d=128, new=1, window=4096, sinks=4),
        # four drafted tokens and the one before them on a layer without a window, odd GQA group
        dict(name="window_drafts", kind="window", seqs=24, shortest=3000, longest=16000, page=16, Hq=28, Hkv=4, d=128, new=5, window=ALL, sinks=0),
        # two sequences that generate alone at the end of a batch
        dict(name="weights_few", kind="weights", seqs=2, shortest=900, longest=2500, page=16, Hq=32, Hkv=8, d=128),
        # a full rollout batch with ragged live caches
        dict(name="weights_batch", kind="weights", seqs=48, shortest=1000, longest=16000, page=16, Hq=32, Hkv=8, d=128),
        # the engine with one-token pages on the 7B-class heads, every cache near its budget
        dict(name="weights_token_pages", kind="weights", seqs=64, shortest=6500, longest=7168, page=1, Hq=28, Hkv=4, d=128),
        # a few caches give back what their last turn took
        dict(name="evict_turn", kind="evict", seqs=4, shortest=4000, longest=5000, page=16, leave=0.1, first=64, recent=256),
        # a full batch of caches is cut to half, token by token
        dict(name="evict_half", kind="evict", seqs=64, shortest=16384, longest=32768, page=1, leave=0.5, first=4, recent=1024),
        # a few sequences, a small vocabulary
        dict(name="verify_few", kind="verify", seqs=4, drafts=3, vocab=32000),
        # a full batch, a large vocabulary of odd size (rows that start anywhere)
        dict(name="verify_batch", kind="verify", seqs=128, drafts=5, vocab=131071),
        # a round of five tokens of a medium batch
        dict(name="round_pages", kind="round", seqs=16, shortest=500, longest=6000, page=16, Hq=32, Hkv=8, d=128, new=5, window=ALL, sinks=0),
        # a round of three with one-token pages, small heads, and a window
        dict(name="round_token_pages", kind="round", seqs=40, shortest=800, longest=9000, page=1, Hq=16, Hkv=4, d=64, new=3, window=1500, sinks=16),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        kind = rng.choice(("window", "window", "weights", "weights", "evict", "verify", "round"))
        if kind == "verify":
            return dict(kind=kind, seqs=log(1, 128), drafts=rng.randint(1, 8), vocab=log(1000, 131072))
        longest = log(40, 32768)
        case = dict(kind=kind, seqs=log(1, 64), shortest=max(1, int(longest * rng.uniform(0.1, 1.0))), longest=longest, page=rng.choice((1, 16, 16, 16, 64)))
        if kind == "evict":
            case.update(leave=round(rng.uniform(0.02, 0.9), 3), first=rng.randint(0, 64), recent=log(1, max(2, longest // 4)))
            return case
        Hq, Hkv, d = rng.choice(HEADS)
        case.update(Hq=Hq, Hkv=Hkv, d=d)
        if kind != "weights":
            case.update(new=rng.choice((1, 1, 2, 3, 5, 8)), window=rng.choice((ALL, log(16, 8192))), sinks=rng.choice((0, 1, 4, 64)))
        if work(case)["bytes"] <= MOST_BYTES and case["seqs"] * longest <= 900000:
            return case


def lengths(case):
    """Live lengths: evenly spaced over the case's range, in a fixed shuffled order."""
    n = case["seqs"]
    x = np.linspace(case["shortest"], case["longest"], n + 2)[1:-1] if n > 1 else np.array([case["longest"]], dtype=float)
    return np.random.RandomState(n).permutation(np.maximum(1, np.rint(x)).astype(np.int64))


def budget_of(case):
    return max(1, int(case["longest"] * (1.0 - case["leave"])))


# ---- what a user's program has in hand ---------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["kind"] == "verify":
        S, n, V = case["seqs"], case["drafts"], case["vocab"]
        # next-token logits of a language model spread over several units; the draft model's are near them
        logits = torch.randn((S, n + 1, V), generator=g, device="cuda") * 2.5
        s["target"] = torch.softmax(logits, dim=-1)
        logits = logits[:, :n] + 0.3 * torch.randn((S, n, V), generator=g, device="cuda")
        s["draft"] = torch.softmax(logits, dim=-1)
        s["drafted"] = torch.multinomial(s["draft"].view(S * n, V), 1, generator=g).view(S, n).int()
        s["u_accept"] = torch.rand((S, n), generator=g, device="cuda")
        s["u_sample"] = torch.rand((S,), generator=g, device="cuda")
        return s
    n, page = lengths(case), case["page"]
    new = case["new"] if case["kind"] == "round" else 0
    used = -(-n // page)
    spare = -(-new // page) + 1
    max_pages = int(used.max()) + spare
    pool = int(used.sum()) + spare * len(n)
    # the pages of every sequence are scattered over the pool, as after many evictions
    order = np.random.default_rng([seed, 73]).permutation(pool).astype(np.int32)
    table, at = np.zeros((len(n), max_pages), dtype=np.int32), 0
    for i, u in enumerate(used):
        table[i, :u] = order[at:at + u]
        at += u
    free = np.concatenate([[pool - at, 0, 0, 0], order[at:], np.zeros(at, dtype=np.int32)]).astype(np.int32)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    state = [torch.from_numpy(x).reshape(-1) for x in (table, n.astype(np.int32), free)]
    if case["kind"] in ("evict", "weights"):
        # accumulated weights span orders of magnitude; a tenth of the tokens has drawn none yet
        w = torch.randn((len(n), max_pages * page), generator=g, device="cuda").mul_(2.0).exp_().mul_(0.05)
        w.mul_(torch.rand(w.shape, generator=g, device="cuda") > 0.1)
        w.mul_(torch.arange(w.shape[1], device="cuda") < torch.from_numpy(n).cuda()[:, None])
        state.append(w.view(-1).view(torch.int32).cpu())
    sizes = [len(x) for x in state]
    s["state"] = torch.cat(state).cuda()
    s["kept"] = s["state"].clone()
    parts = s["state"].split(sizes)
    s.update(table=parts[0].view(len(n), max_pages), n_tokens=parts[1], free=parts[2])
    if len(parts) > 3:
        s["weight"] = parts[3].view(torch.float32).view(len(n), max_pages * page)
    s["most"] = int(n.max()) + new
    if case["kind"] == "evict":
        s["budget"] = budget_of(case)
        return s
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    s.update(k_cache=normal(pool, page, Hkv, d), v_cache=normal(pool, page, Hkv, d))
    s["q"] = (normal(len(n), case.get("new", 1), Hq, d).float() * 1.5).bfloat16()
    if case["kind"] == "weights":
        s["q"] = s["q"].squeeze(1)
    if case["kind"] == "round":
        s.update(k_new=normal(len(n), new, Hkv, d), v_new=normal(len(n), new, Hkv, d), accepted=torch.zeros(len(n), dtype=torch.int32, device="cuda"))
    return s


# ---- one pass ------------------------------------------------------------------------------------------

def run(s):
    return {"window": run_window, "weights": run_weights, "evict": run_evict, "verify": run_verify, "round": run_round}[s["kind"]](s)


def run_window(s):
    if own:
        from paper_2609_35750_b200 import binding as B
        return B.kvs_decode_attn_window(s["q"], s["k_cache"], s["v_cache"], s["table"], s["n_tokens"], s["window"], s["sinks"], max_tokens=s["most"])
    return plain_attention(s, s["window"], s["sinks"])[:2]


def run_weights(s):
    """The accumulators go on growing from pass to pass, as they do from token to token."""
    if own:
        from paper_2609_35750_b200 import binding as B
        out, lse = B.kvs_decode_attn_weights(s["q"], s["k_cache"], s["v_cache"], s["table"], s["n_tokens"], s["weight"], max_tokens=s["most"])
        return out, lse, s["weight"]
    out, lse, p = plain_attention(dict(s, q=s["q"].unsqueeze(1)), ALL, 0)
    s["weight"][:, :p.shape[-1]] += p.sum(dim=(1, 2, 3))
    return out.squeeze(1), lse.squeeze(1), s["weight"]


def run_evict(s):
    """Every pass starts from the same full caches: the state (one buffer) is copied back first."""
    s["state"].copy_(s["kept"])
    if own:
        from paper_2609_35750_b200 import binding as B
        evicted, n_evicted = B.kvs_cache_evict_lowest(s["budget"], s["first"], s["recent"], s["page"], s["table"], s["n_tokens"], s["free"], s["weight"])
    else:
        evicted, n_evicted = plain_evict(s)
    return s["table"], s["n_tokens"], s["free"], s["weight"], evicted, n_evicted


def run_verify(s):
    if own:
        from paper_2609_35750_b200 import binding as B
        return B.kvs_verify_drafts(s["target"], s["draft"], s["drafted"], s["u_accept"], s["u_sample"])
    return plain_verify(s)


def run_round(s):
    """All drafted tokens leave again, so that every pass finds the caches as the one before did."""
    if own:
        from paper_2609_35750_b200 import binding as B
        B.kvs_cache_append_tokens(s["k_new"], s["v_new"], s["table"], s["n_tokens"], s["free"], s["k_cache"], s["v_cache"])
        got = B.kvs_decode_attn_window(s["q"], s["k_cache"], s["v_cache"], s["table"], s["n_tokens"], s["window"], s["sinks"], max_tokens=s["most"])
        B.kvs_cache_truncate(s["new"], s["accepted"], s["page"], s["table"], s["n_tokens"], s["free"])
    else:
        plain_append(s)
        got = plain_attention(s, s["window"], s["sinks"])[:2]
        plain_truncate(s)
    return got, s["table"], s["n_tokens"], s["free"]


# ---- the plain forms -------------------------------------------------------------------------------------

def plain_attention(s, window, sinks):
    """q [S, new, Hq, d] against the visible rows of the cache: (out, lse, weights [S, new, Hkv, G, slots])."""
    q, (_, page, Hkv, d), n = s["q"], s["k_cache"].shape, s["n_tokens"].long()
    S, new, Hq, _ = q.shape
    most = s["most"]
    if window + new - 1 + sinks < most:
        # the first tokens, then the windows of all queries; a first token inside a window counts once
        recent = torch.arange(window + new - 1, device=q.device) + n[:, None] - (window + new - 1)
        slot = torch.cat((torch.arange(sinks, device=q.device).expand(S, sinks), recent.masked_fill(recent < sinks, -1)), dim=1)
    else:
        slot = torch.arange(most, device=q.device).expand(S, most)
    there = (slot >= 0) & (slot < n[:, None])
    at = slot.where(there, 0)
    row = torch.gather(s["table"].long(), 1, at // page) * page + at % page
    row = row.where(there, 0)
    position = (n[:, None] - new + torch.arange(new, device=q.device))[:, :, None]
    sees = there[:, None] & (slot[:, None] <= position) & ((slot[:, None] < sinks) | (slot[:, None] > position - window))
    qq = q.float().view(S, new, Hkv, Hq // Hkv, d)
    score = torch.einsum("sthgd,slhd->sthgl", qq, s["k_cache"].view(-1, Hkv, d)[row].float()) * d ** -0.5
    score = score.masked_fill_(~sees[:, :, None, None], -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    p = torch.exp(score.sub_(top.masked_fill(top == -math.inf, 0.0)))
    total = p.sum(dim=-1, keepdim=True)
    lse = (torch.log(total) + top).reshape(S, new, Hq)
    p = p.div_(total.masked_fill(total == 0, 1.0))
    out = torch.einsum("sthgl,slhd->sthgd", p, s["v_cache"].view(-1, Hkv, d)[row].float()).reshape(S, new, Hq, d)
    return out.to(q.dtype), lse, p


def ranks(gone):
    """The place of every page that leaves (sequences in order, slots ascending), and how many there are."""
    order = gone.flatten().long().cumsum(0)
    return (order - 1).view(gone.shape), order[-1]


def push(free, pages, gone):
    """The pages where `gone` holds go back on the free stack, the last one first."""
    rank, total = ranks(gone)
    at = (free[0] + 3 + total - rank).where(gone, len(free))
    padded = torch.cat((free, free.new_zeros(1)))
    padded.scatter_(0, at.flatten(), pages.flatten())
    free.copy_(padded[:-1])
    free[0] += total.int()


def plain_evict(s):
    n, page, weight = s["n_tokens"].long()[:, None], s["page"], s["weight"]
    S, P = s["table"].shape
    slot = torch.arange(P, device=n.device)[None]
    score = weight.view(S, P, page).double().sum(dim=-1).float()
    may = (slot * page >= s["first"]) & ((slot + 1) * page <= n - s["recent"])
    take = torch.minimum(((n - s["budget"]).clamp(min=0) + page - 1) // page, may.sum(dim=1, keepdim=True))
    order = torch.argsort(score.masked_fill(~may, math.inf), dim=1, stable=True)
    rank = torch.empty_like(order).scatter_(1, order, slot.expand(S, P))
    gone = may & (rank < take)
    live = (n + page - 1) // page
    stays = (slot < live) & ~gone
    left = live - take
    source = torch.argsort(~stays, dim=1, stable=True)
    push(s["free"], s["table"], gone)
    table = torch.gather(s["table"], 1, source).where(slot < left, s["table"])
    rows = torch.gather(weight.view(S, P, page), 1, source[..., None].expand(S, P, page))
    weight.copy_(rows.masked_fill_((slot >= left)[..., None], 0.0).view(S, P * page))
    s["table"].copy_(table)
    s["n_tokens"].sub_((take * page).squeeze(1).int())
    evicted = torch.argsort(~gone, dim=1, stable=True).int().where(slot < take, -1)
    return evicted, take.squeeze(1).int()


def plain_verify(s):
    p, q, x = s["target"], s["draft"], s["drafted"].long()[..., None]
    S, n, V = q.shape
    px, qx = torch.gather(p[:, :n], 2, x).squeeze(2).double(), torch.gather(q, 2, x).squeeze(2).double()
    accepted = torch.cumprod((s["u_accept"].double() * qx < px).long(), dim=1).sum(dim=1)
    at = torch.arange(S, device=p.device)
    row = p[at, accepted].double()
    rest = (row - q[at, accepted.clamp(max=n - 1)].double()).clamp(min=0.0)
    rest = rest.where((accepted < n)[:, None] & (rest.sum(dim=1, keepdim=True) > 0), row)
    running = torch.cumsum(rest, dim=1)
    following = (running <= s["u_sample"].double()[:, None] * running[:, -1:]).sum(dim=1).clamp(max=V - 1)
    place = torch.arange(n + 1, device=p.device)[None]
    drafted = torch.cat((s["drafted"], s["drafted"].new_zeros(S, 1)), dim=1)
    tokens = drafted.where(place < accepted[:, None], -1)
    tokens = following.int()[:, None].expand(S, n + 1).where(place == accepted[:, None], tokens)
    return tokens, accepted.int()


def plain_append(s):
    table, n, free, page = s["table"], s["n_tokens"].long(), s["free"], s["page"]
    S, new, Hkv, d = s["k_new"].shape
    live, after = (n + page - 1) // page, (n + new + page - 1) // page
    slot = torch.arange(table.shape[1], device=n.device)[None]
    fresh = (slot >= live[:, None]) & (slot < after[:, None])
    rank, total = ranks(fresh)
    table.copy_(free[(3 + free[0] - rank).where(fresh, 0)].where(fresh, table))
    free[0] -= total.int()
    at = n[:, None] + torch.arange(new, device=n.device)
    row = (torch.gather(table.long(), 1, at // page) * page + at % page).flatten()
    s["k_cache"].view(-1, Hkv, d)[row] = s["k_new"].view(-1, Hkv, d)
    s["v_cache"].view(-1, Hkv, d)[row] = s["v_new"].view(-1, Hkv, d)
    s["n_tokens"] += new


def plain_truncate(s):
    table, n, page = s["table"], s["n_tokens"].long(), s["page"]
    left = n - (s["new"] - s["accepted"].long())
    slot = torch.arange(table.shape[1], device=n.device)[None]
    push(s["free"], table, (slot >= ((left + page - 1) // page)[:, None]) & (slot < ((n + page - 1) // page)[:, None]))
    s["n_tokens"].copy_(left)


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    S = case["seqs"]
    if case["kind"] == "verify":
        # the rows of the target and of the draft at the place that decides; the drafted tokens' own probabilities
        return {"bytes": S * (8 * case["vocab"] + 24 * case["drafts"] + 12), "flops": 4 * S * case["vocab"]}
    n = lengths(case)
    if case["kind"] == "evict":
        tokens, pages = int(n.sum()), int((-(-n // case["page"])).sum())
        return {"bytes": 8 * tokens + 12 * pages, "flops": tokens}
    Hq, Hkv, d, new = case["Hq"], case["Hkv"], case["d"], case.get("new", 1)
    n = n + (new if case["kind"] == "round" else 0)
    rows = int(np.minimum(n, case.get("window", ALL) + new - 1 + case.get("sinks", 0)).sum())
    need = 4 * d * Hkv * rows + S * new * Hq * (4 * d + 4)
    if case["kind"] == "weights":
        need += 8 * int(n.sum())
    if case["kind"] == "round":
        need += 8 * d * Hkv * S * new
    return {"bytes": need, "flops": 4 * d * Hq * new * rows}


# ---- the same outputs in 64 bits --------------------------------------------------------------------------

def exact(case, seed):
    """What run() returns, from the definitions, one sequence after the other in float64."""
    s = prepare(case, seed)
    return {"window": exact_window, "weights": exact_weights, "evict": exact_evict, "verify": exact_verify, "round": exact_round}[case["kind"]](s)


def softmax64(q, k, v, sees):
    """q [new, Hkv, G, d], k, v [Hkv, T, d], sees [new, T]: (out, lse, weights)."""
    score = (q.transpose(0, 1).flatten(1, 2) @ k.transpose(1, 2)).view(k.shape[0], q.shape[0], q.shape[2], -1).transpose(0, 1) / math.sqrt(q.shape[-1])
    score = score.masked_fill(~sees[:, None, None], -math.inf)
    lse = torch.logsumexp(score, dim=-1)
    p = torch.exp(score - lse.masked_fill(lse == -math.inf, 0.0)[..., None])
    return torch.einsum("thgl,hld->thgd", p, v), lse, p


def exact_one(s, b, q, n, window, sinks, more=None):
    """One sequence: the rows that its table names (and `more` behind them)."""
    page = s["page"]
    rows = s["table"][b, :-(-n // page)].long()
    k, v = (c[rows].double().flatten(0, 1)[:n] for c in (s["k_cache"], s["v_cache"]))
    if more is not None:
        k, v = torch.cat((k, more[0].double())), torch.cat((v, more[1].double()))
    new, Hq, d = q.shape
    j = torch.arange(len(k), device=q.device)[None]
    at = torch.arange(len(k) - new, len(k), device=q.device)[:, None]
    sees = (j <= at) & ((j < sinks) | (at - j < window))
    out, lse, p = softmax64(q.double().view(new, k.shape[1], -1, d), k.transpose(0, 1), v.transpose(0, 1), sees)
    return out.reshape(new, Hq, d), lse.reshape(new, Hq), p


def exact_window(s, more=None):
    got = [exact_one(s, b, s["q"][b], n, s["window"], s["sinks"], more and (more[0][b], more[1][b])) for b, n in enumerate(s["n_tokens"].tolist())]
    return torch.stack([g[0] for g in got]), torch.stack([g[1] for g in got])


def exact_weights(s):
    weight, outs, lses = s["weight"].double(), [], []
    for b, n in enumerate(s["n_tokens"].tolist()):
        out, lse, p = exact_one(s, b, s["q"][b][None], n, ALL, 0)
        weight[b, :n] += p.flatten(0, 2).sum(dim=0)
        outs.append(out[0])
        lses.append(lse[0])
    return torch.stack(outs), torch.stack(lses), weight


def exact_evict(s):
    table, n, free = s["table"].cpu().numpy(), s["n_tokens"].cpu().numpy(), s["free"].cpu().numpy()
    weight, page = s["weight"].double().cpu().numpy(), s["page"]
    evicted, counts, back = np.full_like(table, -1), np.zeros_like(n), []
    for b in range(len(n)):
        live = -(-int(n[b]) // page)
        rows = weight[b, :live * page].reshape(live, page).copy()
        lo, hi = -(-s["first"] // page), max(0, int(n[b]) - s["recent"]) // page
        take = min(max(0, -(-(int(n[b]) - s["budget"]) // page)), max(0, hi - lo))
        score = rows[lo:lo + max(0, hi - lo)].sum(axis=1).astype(np.float32)
        gone = np.sort(lo + np.lexsort((np.arange(len(score)), score))[:take])
        stay = np.setdiff1d(np.arange(live), gone)
        back.extend(table[b, gone].tolist())
        evicted[b, :take], counts[b] = gone, take
        table[b, :live - take] = table[b, stay]
        weight[b] = 0.0
        weight[b, :len(stay) * page] = rows[stay].ravel()
        n[b] -= take * page
    top = int(free[0])
    free[4 + top:4 + top + len(back)] = back[::-1]
    free[0] = top + len(back)
    return table, n, free, weight, evicted, counts


def exact_verify(s):
    tokens, counts = [], []
    target, draft, x, ua, us = (s[name].cpu().numpy() for name in ("target", "draft", "drafted", "u_accept", "u_sample"))
    for b in range(len(x)):
        r = 0
        while r < len(x[b]) and np.float64(ua[b, r]) * np.float64(draft[b, r, x[b, r]]) < np.float64(target[b, r, x[b, r]]):
            r += 1
        w = target[b, r].astype(np.float64)
        if r < len(x[b]):
            w = np.maximum(w - draft[b, r].astype(np.float64), 0.0)
        running = np.cumsum(w)
        following = int(np.searchsorted(running, np.float64(us[b]) * running[-1], side="right"))
        tokens.append(x[b, :r].tolist() + [min(following, len(w) - 1)] + [-1] * (len(x[b]) - r))
        counts.append(r)
    return np.array(tokens, dtype=np.int32), np.array(counts, dtype=np.int32)


def exact_round(s):
    """Nothing stays but the pages that were taken, named in the table behind the live ones."""
    got = exact_window(s, (s["k_new"], s["v_new"]))
    table, page = s["table"].cpu().numpy(), s["page"]
    stack = s["free"].cpu().numpy()[4:4 + int(s["free"][0])].tolist()
    for b, n in enumerate(s["n_tokens"].tolist()):
        for t in range(n, n + s["new"]):
            if t % page == 0:
                table[b, t // page] = stack.pop()
    return got, table, s["n_tokens"], s["free"]
