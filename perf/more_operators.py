"""Compression of a per-head cache by accumulated attention weight, as cases that can be timed and checked.

Three operators: `score` adds up the attention weight that the last tokens' queries give every row of the cache; `select` chooses,
for every (sequence, KV head) pair, the rows that stay: protected ones, and the heaviest of the others up to a budget that is a
pair's own or shared by the heads of a sequence; `evict` moves the chosen rows, in their order, into a smaller cache.

Every pair keeps a number of tokens of its own.  A cache is packed (`off`: the first row of every pair) or paged (`pages`: the pages
of every pair in token order, each of `page` rows).  Weights lie as the rows do, one float to a row.  Where `own` is false the
operators run in their plain form: elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
SCALE8 = 0.02                # what a stored byte of an 8-bit K cache is multiplied by, for the first KV head
SPARE = 3                    # rows a pair has to spare behind its last one


def _case(name, op, dtype, B, Hq, Hkv, D, budgets, mean, page=0, **more):
    c = dict(op=op, dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, D=D, budgets=budgets, mean=mean, page=page)
    if op == "score":
        c.update(dict(q_len=1, tree=False, ragged=False, decay=1.0), **more)
    elif op == "select":
        c.update(dict(shared=True, part=0.5, pool=1, sink=4, recent=32), **more)
    else:
        c.update(dict(part=0.5, to_page=0, weights=True), **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The smallest call: one user alone on the GPU, a decode step adds its one token's weights to those of the steps before.
        _case("score_one_bf16", "score", "bf16", 1, 64, 8, 128, "lognormal", 1024),
        # A decode step of a batch over a paged cache of 8-bit floats with a scale per KV head, older steps' weights fading.
        _case("score_step_kv8", "score", "kv8", 64, 64, 8, 128, "lognormal", 1024, page=16, decay=0.95),
        # A verified draft: ragged trees of up to 8 nodes, two heavy KV heads, a paged cache, heads of 64.
        _case("score_tree_paged", "score", "bf16", 32, 40, 8, 64, "heavy", 512, page=16, q_len=8, tree=True, ragged=True),
        # The observation window at the end of long prompts: the last 32 tokens look back over all of them.
        _case("score_window_bf16", "score", "bf16", 8, 64, 8, 128, "equal", 16000, q_len=32, decay=0.0),
        # The largest: chunks of 64 tokens of a batch's prompts, weights added up chunk by chunk.
        _case("score_chunk_bf16", "score", "bf16", 64, 64, 8, 128, "equal", 4096, q_len=64),
        # One user alone: the heads of one sequence share a budget of half its rows.
        _case("select_one", "select", "bf16", 1, 64, 8, 128, "lognormal", 1024),
        # The steady state of a batch at its budget: every pair gives up a few of its rows, a paged cache.
        _case("select_step_paged", "select", "bf16", 128, 64, 8, 128, "lognormal", 1024, page=16, shared=False, part=0.97, recent=64),
        # Long prompts down to a sixteenth, the heads of a sequence sharing, a row's neighbours counting for it.
        _case("select_prompt_shared", "select", "bf16", 16, 64, 8, 128, "equal", 16000, part=0.0625, pool=7),
        # One very long prompt: a million rows that compete with one another.
        _case("select_long_shared", "select", "bf16", 1, 64, 8, 128, "equal", 131072, part=0.02, pool=5, recent=64),
        # One user alone: half of the rows into a smaller cache.
        _case("evict_one_bf16", "evict", "bf16", 1, 64, 8, 128, "lognormal", 1024),
        # Long prompts down to a sixteenth, from where the prompt was run into the pages that decoding uses.
        _case("evict_prompt_bf16", "evict", "bf16", 16, 64, 8, 128, "equal", 16000, part=0.0625, to_page=64),
        # The largest move: a full batch's 8-bit cache halved, from pages into one run of rows per pair.
        _case("evict_large_kv8", "evict", "kv8", 128, 64, 8, 128, "lognormal", 4096, page=16),
    ]


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    op = rng.choice(["score", "score", "select", "evict"])
    dtype = rng.choice(["bf16", "bf16", "kv8", "f32"] if op == "evict" else ["bf16", "bf16", "kv8"] if op == "score" else ["bf16"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    q_len = rng.choice([1, log_int(2, 64), log_int(2, 64)]) if op == "score" else 1
    B = log_int(1, 128)
    budgets = rng.choice(["lognormal", "lognormal", "heavy", "pareto", "equal"])
    # No more bytes, rows and scores than the largest listed cases have, each pair filled up to the longest, as the plain form holds them.
    longest = {"lognormal": 4, "heavy": 11, "pareto": 128, "equal": 1}[budgets]
    row = D * {"bf16": 2, "kv8": 1, "f32": 4}[dtype]
    cells = {"score": 64 * 8 * 4096 * 512, "select": 8 * 131072 * 4, "evict": 800_000_000 // (4 * row)}[op]
    each = longest * Hkv * (max(G * q_len, 16) if op == "score" else 1)
    B = max(1, min(B, cells // (each * 32)))
    mean = 32 if budgets == "pareto" else log_int(24, max(32, min(16000 if B > 1 else 131072, cells // (each * B))))
    if budgets == "heavy":
        mean = max(16, mean // 3)
    page = rng.choice([0, 0, 16, 32, 64, 128])
    if op == "score":
        more = dict(q_len=q_len, tree=rng.random() < 0.5, ragged=rng.random() < 0.4, decay=rng.choice([0.0, 1.0, 0.95]))
    elif op == "select":
        more = dict(shared=rng.random() < 0.5, part=round(rng.choice([rng.uniform(0.02, 0.2), rng.uniform(0.2, 0.98)]), 3), pool=rng.choice([1, 1, 3, 5, 7, 13]),
                    sink=rng.choice([0, 1, 4]), recent=rng.choice([0, 1, 16, 32, 64]))
    else:
        more = dict(part=round(rng.uniform(0.03, 0.98), 3), to_page=rng.choice([0, 16, 32, 64]), weights=rng.random() < 0.7)
    return _case(None, op, dtype, B, G * Hkv, Hkv, D, budgets, mean, page, **more)


# ---- inputs -------------------------------------------------------------------------------------------
def _lens(case, seed):
    """Tokens that every (sequence, KV head) pair keeps, int32 [B][Hkv]: the case's own budgets, so that every seed is the same amount of
    work; the seed says which sequence has which."""
    rng = np.random.default_rng(7)
    deal = np.random.default_rng([int(seed), 11])
    B, H, mean, kind = case["B"], case["Hkv"], case["mean"], case["budgets"]

    def lognormal(m):
        return np.clip(np.rint(m * np.exp(0.6 * rng.standard_normal((B, H)) - 0.18)), 16, 4 * m)

    if kind == "lognormal":
        n = lognormal(mean)
    elif kind == "heavy":                            # every third KV head keeps eight times as much
        n = lognormal(mean)
        n[:, 2::3] = lognormal(8 * mean)[:, 2::3]
    elif kind == "pareto":
        n = np.clip(np.floor(mean * rng.random((B, H)) ** (-1 / 1.2)), mean, 128 * mean)
    else:
        n = np.full((B, H), mean)
    for h in range(H):                               # a heavy head stays heavy
        n[:, h] = deal.permutation(n[:, h])
    return np.ascontiguousarray(n, dtype=np.int32)


def _n_new(case, seed):
    """New tokens of every sequence, int32 [B]."""
    n = np.full(case["B"], case["q_len"])
    if case["ragged"]:
        n = np.random.default_rng(13).integers(1, case["q_len"] + 1, case["B"])
        n = np.random.default_rng([int(seed), 17]).permutation(n)
    return n.astype(np.int32)


def _trees(case, seed):
    """Ancestors of every node with itself as bits, int64 [B][q_len].  A node's parent comes before it."""
    rng = np.random.default_rng([int(seed), 19])
    B, n = case["B"], case["q_len"]
    bits = np.zeros((B, n), dtype=np.uint64)
    for i in range(n):
        parent = rng.integers(-1, i, B) if i else np.full(B, -1)
        bits[:, i] = np.where(parent >= 0, bits[np.arange(B), np.maximum(parent, 0)], 0) | (np.uint64(1) << np.uint64(i))
    return bits.view(np.int64)


def _kept(case, seed, lens):
    """Rows that stay of every pair, as an eviction finds them: heads keep unequal parts; the first rows and the last are among them, the others lie
    anywhere.  int32 [B][Hkv][longest] (ascending, filled up with -1) and their numbers."""
    part = np.random.default_rng(37).random(lens.shape) * 2 * case["part"]
    deal = np.random.default_rng([int(seed), 11])
    for h in range(lens.shape[1]):                   # a sequence's part goes with its length
        part[:, h] = deal.permutation(part[:, h])
    counts = np.clip(np.rint(part * lens), 1, lens).astype(np.int32)
    rng = np.random.default_rng([int(seed), 43])
    keep = np.full(lens.shape + (int(counts.max()),), -1, dtype=np.int32)
    for b in range(lens.shape[0]):
        for h in range(lens.shape[1]):
            n, m = int(counts[b, h]), int(lens[b, h])
            rank = rng.random(m, dtype=np.float32)
            rank[:4], rank[max(0, m - 32):] = -1, -1
            keep[b, h, :n] = np.sort(np.argpartition(rank, n - 1)[:n])
    return keep, counts


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1_000_003 + 4242) & 0x7FFFFFFF)
    return g


def _scales(case):
    return [float(SCALE8 * (1 + 0.1 * i)) for i in range(case["Hkv"])] if case["dtype"] == "kv8" else None


def _on(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _place(lens, page, seed):
    """Where a cache with room for `lens` and a few more rows has them: off, pages, rows in all, room of every pair."""
    room = lens + SPARE
    if not page:
        off = np.concatenate([[0], np.cumsum(room.reshape(-1).astype(np.int64))])
        return _on(off[:-1].reshape(lens.shape)), None, int(off[-1]), _on(room.astype(np.int32))
    need = -(-room // page)                          # pages of a pool that is a quarter larger than it need be, in no order
    pool = int(need.sum()) * 5 // 4 + 1
    order = np.random.default_rng([int(seed), 29]).permutation(pool)[:int(need.sum())]
    pages = np.full((lens.size, int(need.max())), -1, dtype=np.int32)
    pages[np.arange(pages.shape[1])[None, :] < need.reshape(-1, 1)] = order
    return None, _on(pages), pool * page, _on((need * page).astype(np.int32))


def _inputs(case, seed):
    """What a user's program has in hand, as a dict of tensors and numbers."""
    B, Hq, Hkv, D = (case[x] for x in ("B", "Hq", "Hkv", "D"))
    g = _gen(seed)
    op = case["op"]
    n_new = _n_new(case, seed) if op == "score" else np.zeros(B, dtype=np.int32)
    lens = _lens(case, seed) + n_new[:, None]
    s = {"case": case, "longest": int(lens.max()), "lens": _on(lens), "page": case["page"]}
    most = case.get("q_len", 0)                      # of a ragged step's new tokens
    s["off"], s["pages"], rows, s["cap"] = _place(lens - n_new[:, None] + most, case["page"], seed)
    s["scales"] = _scales(case)
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dt)

    def stored(x):
        return (x.float() / SCALE8).clamp(-448, 448).to(torch.float8_e4m3fn) if case["dtype"] == "kv8" else x

    def heavy_tailed(n, each=1.0):                   # weights as attention leaves them
        return torch.exp(2 * torch.randn(n, generator=g, device=DEV)) * each

    if op == "score":
        n = case["q_len"]
        s["k"], s["q"] = stored(randn(rows, D)), randn(B, n, Hq, D)
        s["n_new"] = _on(n_new) if case["ragged"] else None
        s["tree"] = _on(_trees(case, seed)) if case["tree"] else None
        s["weights"], s["weights_out"] = heavy_tailed(rows, n * Hq / Hkv / case["mean"]), torch.zeros(rows, device=DEV)
        # What the attention of the same step left; a sequence at a time, long ones have many scores.
        s["lse"] = torch.zeros(B, n, Hq, device=DEV)
        for b in range(B):
            z = _scores(s, slice(b, b + 1))
            s["lse"][b] = torch.logsumexp(z, -1).permute(0, 2, 1, 3).reshape(n, Hq)
        s["lse"] = torch.where(torch.arange(n, device=DEV)[:, None] < _on(n_new)[:, None, None], s["lse"], torch.zeros((), device=DEV))
    elif op == "select":
        # Heads spread their weight differently; a part of the rows has got nothing at all.
        t = torch.arange(s["longest"], device=DEV)
        z = torch.randn((B, Hkv, s["longest"]), generator=g, device=DEV)
        spread = 0.5 + 2 * torch.rand((B, Hkv, 1), generator=g, device=DEV)
        w = torch.where(z < -1.6, torch.zeros((), device=DEV), torch.exp(spread * z - spread * spread / 2) / s["lens"][:, :, None])
        s["weights"] = torch.zeros(rows, device=DEV)
        live = t < s["lens"][:, :, None]
        s["weights"][_rows(s, torch.minimum(t, s["lens"].long()[:, :, None] - 1))[live]] = w[live]
        budget = np.rint(case["part"] * lens)
        s["budget"] = _on((budget.sum(1) if case["shared"] else budget).astype(np.int32))
        s["keep"] = torch.full((B, Hkv, s["longest"]), -1, dtype=torch.int32, device=DEV)
        s["n_keep"] = torch.zeros((B, Hkv), dtype=torch.int32, device=DEV)
        s["k"] = torch.zeros((rows, D), dtype=torch.bfloat16, device=DEV)      # of no concern here: the cache's handle has it
    else:
        s["k"], s["v"] = stored(randn(rows, D)), stored(randn(rows, D))
        keep, counts = _kept(case, seed, lens)
        s["keep"], s["n_keep"] = _on(keep), _on(counts)
        to = {"page": case["to_page"]}
        to["off"], to["pages"], to_rows, to["cap"] = _place(counts, case["to_page"], seed)
        to["k"], to["v"] = (torch.zeros((to_rows, D), dtype=s["k"].dtype, device=DEV) for _ in range(2))
        s["weights"] = heavy_tailed(rows) if case["weights"] else None
        to["weights"] = torch.zeros(to_rows, device=DEV) if case["weights"] else None
        to["lens"] = torch.zeros_like(s["lens"])
        s["to"] = to
    s.setdefault("v", s["k"])
    return s


def prepare(case, seed):
    return _inputs(case, seed)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the framework's calls -----------------------------------------------------------------------------
def _run_own(s):
    import paper_2502_15804_amd as F

    case = s["case"]
    op = case["op"]
    cache = s.get("cache")
    if cache is None:                                # the handles that a user's program keeps
        def handle(x):
            return F.Cache(x["k"], x["v"], x["cap"], off=x["off"], pages=x["pages"], page_rows=x["page"] or None, k_scale=s["scales"], v_scale=s["scales"])

        cache = s["cache"] = handle(s)
        if op == "evict":
            s["into"] = handle(s["to"])
        if op == "select":
            s["workspace"] = torch.zeros(F.fairkv_select_workspace_bytes(cache, case["shared"]), dtype=torch.uint8, device=DEV)
    if op == "score":
        F.fairkv_attn_weights(cache, s["lens"], s["q"], s["lse"], s["weights"], 1.0 / math.sqrt(case["D"]), tree=s["tree"], n_new=s["n_new"],
                              decay=case["decay"], weights_out=s["weights_out"])
        return s["weights_out"]
    if op == "select":
        F.fairkv_select(cache, s["lens"], s["weights"], s["budget"], s["keep"], s["n_keep"], s["workspace"], pool=case["pool"], sink=case["sink"],
                        recent=case["recent"])
        return s["keep"], s["n_keep"]
    to = s["to"]
    F.fairkv_evict(cache, s["lens"], s["keep"], s["n_keep"], into=s["into"], lens_out=to["lens"], weights=s["weights"], weights_out=to["weights"])
    return to["k"], to["v"], to["lens"], to["weights"]


# ---- the plain forms -----------------------------------------------------------------------------------
def _rows(s, at, which=slice(None)):
    """The cache rows of tokens at [B, Hkv, ...] of every pair (of the sequences `which`)."""
    shape = at.shape[:2] + (1,) * (at.dim() - 2)
    if s["off"] is not None:
        return s["off"][which].reshape(shape) + at
    pages = s["pages"].reshape(*s["cap"].shape, -1)[which].flatten(0, 1)
    return pages.gather(1, (at // s["page"]).reshape(pages.shape[0], -1)).reshape(at.shape).long() * s["page"] + at % s["page"]


def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _scores(s, which=slice(None)):
    """Scaled scores float32 [B, Hkv, n, G, longest], -inf where a node does not see a row."""
    case = s["case"]
    n, Hkv, D = case["q_len"], case["Hkv"], case["D"]
    G = case["Hq"] // Hkv
    lens = s["lens"].long()[which]
    B = lens.shape[0]
    n_new = s["n_new"].long()[which][:, None] if s["n_new"] is not None else torch.full((B, 1), n, device=DEV)
    t = torch.arange(s["longest"], device=DEV)
    k = _bytes(s["k"])[_rows(s, torch.minimum(t, lens[:, :, None] - 1), which)].view(s["k"].dtype).float()
    if s["scales"] is not None:
        k = k * torch.tensor(s["scales"], device=DEV)[:, None, None]
    q = s["q"][which].float().reshape(B, n, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, n * G, D)
    z = (torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)).reshape(B, Hkv, n, G, -1)
    node = t - (lens - n_new)[:, :, None]                                     # of the draft, negative in front of it
    if s["tree"] is not None:
        sees = (s["tree"][which][:, None, :, None] >> node.clamp(0, 63)[:, :, None, :] & 1) != 0
    else:
        sees = node[:, :, None, :] <= torch.arange(n, device=DEV)[:, None]
    sees = ((node < 0)[:, :, None, :] | sees) & (t < lens[:, :, None])[:, :, None, :] & (torch.arange(n, device=DEV) < n_new)[:, None, :, None]
    return z.masked_fill(~sees[:, :, :, None, :], -math.inf)


def _plain_score(s):
    case = s["case"]
    B, n, Hkv = case["B"], case["q_len"], case["Hkv"]
    lens = s["lens"].long()[:, :, None]
    lse = s["lse"].reshape(B, n, Hkv, -1).transpose(1, 2)[..., None]
    w = torch.exp(_scores(s) - lse).sum((2, 3))
    t = torch.arange(s["longest"], device=DEV)
    rows = _rows(s, torch.minimum(t, lens - 1))
    n_new = s["n_new"].long()[:, None, None] if s["n_new"] is not None else n
    if case["decay"]:                                # the new tokens' own rows have no weight from before
        w = w + torch.where(t < lens - n_new, case["decay"] * s["weights"][rows], torch.zeros((), device=DEV))
    live = t < lens
    s["weights_out"][rows[live]] = w[live]


def _plain_select(s):
    case = s["case"]
    B, Hkv, L = s["keep"].shape
    lens = s["lens"].long()[:, :, None]
    t = torch.arange(L, device=DEV)
    live = t < lens
    protected = live & ((t < case["sink"]) | (t >= lens - case["recent"]))
    candidate = live & ~protected
    w = s["weights"][_rows(s, torch.minimum(t, lens - 1))].masked_fill(~candidate, -math.inf)
    half = case["pool"] // 2
    if half:
        edge = torch.full((B, Hkv, half), -math.inf, device=DEV)
        w = torch.cat([edge, w, edge], -1).unfold(-1, case["pool"], 1).amax(-1).masked_fill(~candidate, -math.inf)
    groups = (B, Hkv * L) if case["shared"] else (B * Hkv, L)
    left = (s["budget"].reshape(-1).long() - protected.reshape(groups).sum(1)).clamp(min=0)
    order = torch.sort(w.reshape(groups), dim=1, descending=True, stable=True).indices
    first = torch.arange(groups[1], device=DEV) < left[:, None]
    chosen = torch.zeros(groups, dtype=torch.bool, device=DEV).scatter(1, order, first).reshape(B, Hkv, L)
    stays = protected | (candidate & chosen)
    place = stays.long().cumsum(-1) - 1
    pair = torch.arange(B * Hkv, device=DEV).reshape(B, Hkv, 1).expand(B, Hkv, L)
    s["keep"].view(B * Hkv, L)[pair[stays], place[stays]] = t.to(torch.int32).expand(B, Hkv, L)[stays]
    s["n_keep"].copy_(stays.sum(-1))


def _plain_evict(s):
    to = s["to"]
    i = torch.arange(s["keep"].shape[2], device=DEV)
    last = torch.minimum(i, s["n_keep"].long()[:, :, None] - 1)              # places behind a pair's last write that one's row again
    source, target = _rows(s, s["keep"].long().gather(2, last)), _rows(to, last)
    _bytes(to["k"])[target], _bytes(to["v"])[target] = _bytes(s["k"])[source], _bytes(s["v"])[source]
    if s["weights"] is not None:
        to["weights"][target] = s["weights"][source]
    to["lens"].copy_(s["n_keep"])


def _run_plain(s):
    op = s["case"]["op"]
    if op == "score":
        _plain_score(s)
        return s["weights_out"]
    if op == "select":
        _plain_select(s)
        return s["keep"], s["n_keep"]
    _plain_evict(s)
    return s["to"]["k"], s["to"]["v"], s["to"]["lens"], s["to"]["weights"]


# ---- what a pass cannot do without, and what it should give ----------------------------------------------
def _index_bytes(lens, page):
    """Lengths, and the pages or first rows of the pairs."""
    return lens.size * 4 + (int((-(-lens // page)).sum()) * 4 if page else lens.size * 8)


def work(case):
    D, row = case["D"], case["D"] * {"bf16": 2, "f32": 4, "kv8": 1}[case["dtype"]]
    lens = _lens(case, 0).astype(np.int64)
    if case["op"] == "score":
        n_new = _n_new(case, 0).astype(np.int64)
        rows = lens + n_new[:, None]
        new = int(n_new.sum())
        size = int(rows.sum()) * (row + 4) + (int(lens.sum()) * 4 if case["decay"] else 0) + new * (case["Hq"] * (2 * D + 4) + 8 * bool(case["tree"]))
        return {"bytes": size + _index_bytes(rows, case["page"]), "flops": 2 * int((rows.sum(1) * n_new).sum()) * (case["Hq"] // case["Hkv"]) * D}
    if case["op"] == "select":
        kept = int(np.rint(case["part"] * lens).sum())
        return {"bytes": int(lens.sum()) * 4 + kept * 4 + _index_bytes(lens, case["page"]) + lens.size * 8, "flops": int(lens.sum()) * case["pool"]}
    counts = _kept(case, 0, lens)[1].astype(np.int64)
    return {"bytes": int(counts.sum()) * (4 * row + 4 + 8 * bool(case["weights"])) + lens.size * 8 + _index_bytes(counts, case["to_page"]), "flops": 0}


def _tokens(s, b, h, t):
    """The rows of tokens t (an array) of a pair, on the host."""
    if s["off"] is not None:
        return int(s["off"][b, h]) + t
    return s["pages"].view(*s["cap"].shape, -1)[b, h].cpu().numpy()[t // s["page"]].astype(np.int64) * s["page"] + t % s["page"]


def exact(case, seed):
    s = _inputs(case, seed)
    B, Hq, Hkv, D = (case[x] for x in ("B", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    lens = s["lens"].cpu().numpy().astype(np.int64)
    if case["op"] == "score":
        n_new = _n_new(case, seed)
        see = s["tree"].cpu().numpy() if s["tree"] is not None else None
        out = s["weights_out"].double()
        for b in range(B):
            m = int(n_new[b])
            ones = torch.tril(torch.ones(m, m, dtype=torch.float64)) if see is None else torch.tensor([[float(int(see[b, i]) >> j & 1) for j in range(m)] for i in range(m)], dtype=torch.float64)
            for h in range(Hkv):
                length = int(lens[b, h])
                rows = torch.as_tensor(_tokens(s, b, h, np.arange(length))).to(DEV)
                kd = _bytes(s["k"])[rows].view(s["k"].dtype).double() * (s["scales"][h] if s["scales"] else 1.0)
                cols = s["q"][b, :m, h * G:(h + 1) * G].reshape(m * G, D).double()
                z = kd @ cols.t() / math.sqrt(D) - s["lse"][b, :m, h * G:(h + 1) * G].reshape(m * G).double()
                e = torch.exp(z).reshape(length, m, G).sum(2)
                e[length - m:] *= ones.to(DEV).t()
                w = e.sum(1)
                w[:length - m] += case["decay"] * s["weights"][rows[:length - m]].double()
                out[rows] = w
        return out
    if case["op"] == "select":
        w, budget = s["weights"].cpu().numpy(), s["budget"].cpu().numpy().reshape(-1)
        keep, n_keep = np.full(s["keep"].shape, -1, dtype=np.int64), np.zeros((B, Hkv), dtype=np.int64)
        half, sink, recent = case["pool"] // 2, case["sink"], case["recent"]
        for group in range(budget.size):
            pairs = [(group, h) for h in range(Hkv)] if case["shared"] else [divmod(group, Hkv)]
            value, head, token, free = [], [], [], int(budget[group])
            for b, h in pairs:
                first, end = min(sink, lens[b, h]), max(min(sink, lens[b, h]), lens[b, h] - recent)
                free -= first + lens[b, h] - end
                x = w[_tokens(s, b, h, np.arange(first, end))].astype(np.float64)
                best = x.copy()
                for d in range(1, half + 1):
                    if d < x.size:
                        best[d:] = np.maximum(best[d:], x[:-d])
                        best[:-d] = np.maximum(best[:-d], x[d:])
                value.append(best), head.append(np.full(x.size, h)), token.append(np.arange(first, end))
            value, head, token = (np.concatenate(x) for x in (value, head, token))
            chosen = np.lexsort((token, head, -value))[:max(0, int(free))]
            for b, h in pairs:
                first, end = min(sink, lens[b, h]), max(min(sink, lens[b, h]), lens[b, h] - recent)
                stay = np.concatenate([np.arange(first), np.sort(token[chosen[head[chosen] == h]]), np.arange(end, lens[b, h])])
                keep[b, h, :stay.size], n_keep[b, h] = stay, stay.size
        return _on(keep.astype(np.int32)), _on(n_keep.astype(np.int32))
    to, keep, counts = s["to"], s["keep"].cpu().numpy(), s["n_keep"].cpu().numpy()
    source = np.concatenate([_tokens(s, b, h, keep[b, h, :counts[b, h]].astype(np.int64)) for b in range(B) for h in range(Hkv)])
    target = np.concatenate([_tokens(to, b, h, np.arange(counts[b, h])) for b in range(B) for h in range(Hkv)])
    source, target = torch.as_tensor(source).to(DEV), torch.as_tensor(target).to(DEV)
    k, v = to["k"], to["v"]                          # moved, not computed: as they are stored
    _bytes(k)[target], _bytes(v)[target] = _bytes(s["k"])[source], _bytes(s["v"])[source]
    if case["weights"]:
        to["weights"][target] = s["weights"][source]
    return k, v, to["lens"].copy_(s["n_keep"]), to["weights"]
