"""One step of speculative decoding over a growing per-head cache, as cases that can be timed and checked.

Three operators: `append` normalises the query and key heads of a step's new tokens, rotates them by their positions and
appends the keys and values to the cache; `attend` lets every node of a draft tree attend over the cache and over its
ancestors among the draft's own rows; `accept` moves the rows of the accepted path to the front of the draft's and sets the
lengths (its cases append the draft first, as a step does, so that a pass can be run again on the same state).

Every (sequence, KV head) pair keeps a number of tokens of its own.  A cache is packed (`off`: the first row of every pair) or
paged (`pages`: the pages of every pair in token order, each of `page` rows).  Where `own` is false the operators run in their
plain form: elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
SCALE8 = (0.02, 0.03)        # what a stored byte of an 8-bit K and V cache is multiplied by, for the first KV head
EPS = 1e-6                   # of the norms
N_POS = 32768                # positions in the table of cosines and sines
THETA = 500000.0             # base of the rotation's wavelengths
SPARE = 3                    # rows a pair has to spare behind a step's new ones


def _case(name, op, dtype, B, Hq, Hkv, D, q_len, budgets, mean, page=0, out="bf16", tree=True, norm=False, rot=0, style="half",
          ragged=False, fused=False):
    c = dict(op=op, dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, D=D, q_len=q_len, budgets=budgets, mean=mean, page=page, out=out, tree=tree,
             norm=norm, rot=rot, style=style, ragged=ragged, fused=fused)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The smallest call: one user alone on the GPU, one token of a 70B model's layer with normed heads: launch and latency.
        _case("append_one_bf16", "append", "bf16", 1, 64, 8, 128, 1, "lognormal", 1024, norm=True, rot=128, fused=True),
        # A full batch's decode step into a paged cache of 8-bit floats with a scale per KV head, no norms.
        _case("append_step_kv8", "append", "kv8", 128, 64, 8, 128, 1, "pareto", 32, page=16, rot=128),
        # Accuracy runs in fp32: a small model at an odd batch, drafts of five tokens, half of each head rotated, pairs side by side.
        _case("append_draft_f32", "append", "f32", 13, 32, 8, 64, 5, "lognormal", 700, norm=True, rot=32, style="pairs"),
        # The largest append: chunks of prompts, up to 64 tokens a sequence, from the fused projection into a paged cache.
        _case("append_chunk_bf16", "append", "bf16", 256, 64, 8, 128, 64, "equal", 256, page=64, norm=True, rot=128, ragged=True, fused=True),
        # One user alone on the GPU, a draft tree of 24 nodes: eight pairs for the whole chip.
        _case("tree_one_bf16", "attend", "bf16", 1, 64, 8, 128, 24, "lognormal", 1024),
        # A 70B model's layer at batch 16, trees of 16 nodes (128 columns a pair), outputs in fp32.
        _case("tree_llama70b_bf16", "attend", "bf16", 16, 64, 8, 128, 16, "lognormal", 1024, out="f32"),
        # A 24B model's layer with two heavy KV heads, ragged trees of up to 8 nodes over a paged cache.
        _case("tree_mistral24b_paged", "attend", "bf16", 32, 32, 8, 128, 8, "heavy", 512, page=16, ragged=True),
        # The 70B layer over a paged cache of 8-bit floats.
        _case("tree_llama70b_kv8", "attend", "kv8", 16, 64, 8, 128, 16, "lognormal", 1024, page=64),
        # Plain decoding of a full batch over a paged cache: one token a sequence, many short pairs and a few long ones.
        _case("token_stress_paged", "attend", "bf16", 128, 64, 8, 128, 1, "pareto", 32, page=16, tree=False),
        # The largest: trees of 64 nodes over long equal budgets, bound by the matrix cores.
        _case("tree_large_bf16", "attend", "bf16", 64, 64, 8, 128, 64, "equal", 4096),
        # The end of a step at batch 16: the drafts' rows are appended, the accepted paths kept.
        _case("accept_llama70b_bf16", "accept", "bf16", 16, 64, 8, 128, 16, "lognormal", 1024, rot=128),
        # The same for a full batch of wide trees over a paged cache.
        _case("accept_large_paged", "accept", "bf16", 200, 32, 8, 128, 64, "lognormal", 300, page=32, rot=128),
    ]


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "attend", "attend", "accept"])
    dtype = rng.choice(["bf16", "bf16", "kv8"] if op == "attend" else ["bf16", "bf16", "kv8", "f32"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    q_len = rng.choice([1, log_int(2, 64), log_int(2, 64)])
    B = log_int(1, 200)
    budgets = rng.choice(["lognormal", "lognormal", "heavy", "pareto", "equal"])
    # No more tokens and scores than the largest listed case has, each pair filled up to the longest, as the plain form holds them.
    longest = {"lognormal": 4, "heavy": 11, "pareto": 128, "equal": 1}[budgets]
    cells = 64 * 8 * 4096 * (512 if op == "attend" else 16)
    each = longest * Hkv * (max(G * q_len, 16) if op == "attend" else 16)
    B = max(1, min(B, cells // (each * 32)))
    mean = 32 if budgets == "pareto" else log_int(24, max(32, min(4096, cells // (each * B))))
    if budgets == "heavy":
        mean = max(16, mean // 3)
    page = rng.choice([0, 0, 16, 32, 64, 128])
    rot = rng.choice([D, D, D // 2, 0]) if op != "attend" else 0
    return _case(None, op, dtype, B, G * Hkv, Hkv, D, q_len, budgets, mean, page, rng.choice(["bf16", "bf16", "f32"]) if op == "attend" else "bf16",
                 rng.random() < 0.75, op == "append" and rng.random() < 0.5, rot, rng.choice(["half", "pairs"]), rng.random() < 0.4,
                 op != "attend" and rng.random() < 0.5)


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
    """Parent of every node (int [B][q_len], -1: none) and its ancestors with itself as bits (int64 [B][q_len]).  A node's parent comes before it."""
    rng = np.random.default_rng([int(seed), 19])
    B, n = case["B"], case["q_len"]
    parent = np.full((B, n), -1)
    bits = np.zeros((B, n), dtype=np.uint64)
    for i in range(n):
        if case["tree"]:
            parent[:, i] = rng.integers(-1, i, B) if i else -1
        else:
            parent[:, i] = i - 1
        up = bits[np.arange(B), np.maximum(parent[:, i], 0)]
        bits[:, i] = np.where(parent[:, i] >= 0, up, 0) | (np.uint64(1) << np.uint64(i))
    return parent, bits.view(np.int64)


def _paths(case, seed, n_new, parent):
    """The accepted path of every sequence: the nodes from a root to some node, int32 [B][q_len] (filled up with -1), and their number."""
    rng = np.random.default_rng([int(seed), 23])
    B, n = parent.shape
    path, count = np.full((B, n), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    for b in range(B):
        at, up = int(rng.integers(0, n_new[b])), []
        while at >= 0:
            up.append(at)
            at = int(parent[b, at])
        path[b, :len(up)], count[b] = up[::-1], len(up)
    return path, count


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1_000_003 + 4242) & 0x7FFFFFFF)
    return g


def _scales(case):
    h = np.arange(case["Hkv"])
    return [float(SCALE8[0] * (1 + 0.1 * i)) for i in h], [float(SCALE8[1] * (1 - 0.05 * i)) for i in h]


def _on(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _inputs(case, seed):
    """What a user's program has in hand, as a dict of tensors and numbers."""
    B, Hq, Hkv, D, n, page = (case[x] for x in ("B", "Hq", "Hkv", "D", "q_len", "page"))
    g = _gen(seed)
    before, n_new = _lens(case, seed), _n_new(case, seed)
    attend = case["op"] == "attend"
    lens = before + n_new[:, None] if attend else before
    room = before + n_new[:, None] + SPARE
    s = {"case": case, "n_new": _on(n_new) if case["ragged"] else None, "longest": int((before + n_new[:, None]).max()), "off": None, "pages": None}
    if page:                                         # pages of a pool that is a quarter larger than it need be, in no order
        need = -(-room // page)
        pool = int(need.sum()) * 5 // 4 + 1
        order = np.random.default_rng([int(seed), 29]).permutation(pool)[:int(need.sum())]
        pages = np.full((B * Hkv, int(need.max())), -1, dtype=np.int32)
        pages[np.arange(pages.shape[1])[None, :] < need.reshape(-1, 1)] = order
        s["pages"], rows, room = _on(pages), pool * page, need * page
    else:
        off = np.concatenate([[0], np.cumsum(room.reshape(-1).astype(np.int64))])
        s["off"], rows = _on(off[:-1].reshape(B, Hkv)), int(off[-1])
    s["lens"], s["cap"] = _on(lens), _on(room.astype(np.int32))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dt)

    s["k"], s["v"] = randn(rows, D), randn(rows, D)
    s["k_scale"], s["v_scale"] = _scales(case) if case["dtype"] == "kv8" else (None, None)
    if case["dtype"] == "kv8":
        s["k"], s["v"] = ((x.float() / c).clamp(-448, 448).to(torch.float8_e4m3fn) for x, c in ((s["k"], SCALE8[0]), (s["v"], SCALE8[1])))
    parent, bits = _trees(case, seed)
    if attend:
        s["q"] = randn(B, n, Hq, D)
        s["tree"] = _on(bits) if case["tree"] else None
        s["out"] = torch.zeros((B, n, Hq, D), dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16, device=DEV)
        s["lse"] = torch.zeros((B, n, Hq), dtype=torch.float32, device=DEV)
        return s
    if case["fused"]:                                # slices of what one projection gave
        s["q"], s["k_new"], s["v_new"] = randn(B, n, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], dim=2)
    else:
        s["q"], s["k_new"], s["v_new"] = randn(B, n, Hq, D), randn(B, n, Hkv, D), randn(B, n, Hkv, D)
    s["q_norm"] = s["k_norm"] = s["table"] = s["pos"] = None
    if case["norm"]:
        s["q_norm"], s["k_norm"] = (1 + 0.1 * torch.randn(2, D, generator=g, device=DEV)).unbind(0)
    if case["rot"]:
        half = case["rot"] // 2
        angle = torch.arange(N_POS, dtype=torch.float64, device=DEV)[:, None] * THETA ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        s["table"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
        depth = np.zeros((B, n), dtype=np.int64)
        for i in range(n):
            depth[:, i] = np.where(parent[:, i] >= 0, depth[np.arange(B), np.maximum(parent[:, i], 0)] + 1, 0)
        start = np.random.default_rng([int(seed), 31]).integers(0, N_POS - n, B)
        s["pos"] = _on((start[:, None] + depth).astype(np.int32))
    s["q_out"] = torch.zeros((B, n, Hq, D), dtype=dt, device=DEV)
    s["lens_out"] = torch.zeros_like(s["lens"])
    if case["op"] == "accept":
        path, count = _paths(case, seed, n_new, parent)
        s["path"], s["n_path"] = _on(path), _on(count)
        s["lens_kept"] = torch.zeros_like(s["lens"])
    return s


def prepare(case, seed):
    return _inputs(case, seed)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the framework's calls -----------------------------------------------------------------------------
def _run_own(s):
    import paper_2502_15804_amd as F

    op = s["case"]["op"]
    cache = s.get("cache")
    if cache is None:                                # the handle that a user's program keeps
        cache = s["cache"] = F.Cache(s["k"], s["v"], s["cap"], off=s["off"], pages=s["pages"], page_rows=s["case"]["page"] or None,
                                     k_scale=s["k_scale"], v_scale=s["v_scale"])
        if op == "attend":
            s["workspace"] = torch.zeros(F.fairkv_tree_workspace_bytes(cache, s["case"]["Hq"], s["case"]["q_len"]), dtype=torch.uint8, device=DEV)
    if op == "attend":
        F.fairkv_decode_attn_tree(cache, s["lens"], s["q"], s["workspace"], s["out"], s["lse"], 1.0 / math.sqrt(s["case"]["D"]),
                                  tree=s["tree"], n_new=s["n_new"])
        return s["out"], s["lse"]
    F.fairkv_append_rotated(cache, s["lens"], s["q"], s["k_new"], s["v_new"], s["q_out"], table=s["table"], pos=s["pos"], q_norm=s["q_norm"],
                            k_norm=s["k_norm"], eps=EPS, pairs=s["case"]["style"] == "pairs", n_new=s["n_new"], lens_out=s["lens_out"])
    if op == "append":
        return s["q_out"], s["lens_out"], s["k"], s["v"]
    F.fairkv_accept(cache, s["lens_out"], s["path"], s["n_path"], n_new=s["n_new"], lens_out=s["lens_kept"])
    return s["q_out"], s["lens_kept"], s["k"], s["v"]


# ---- the plain forms -----------------------------------------------------------------------------------
def _rows(s, at):
    """The cache rows of tokens at [B, Hkv, ...] of every pair."""
    shape = at.shape[:2] + (1,) * (at.dim() - 2)
    if s["off"] is not None:
        return s["off"].reshape(shape) + at
    page = s["case"]["page"]
    ids = s["pages"].gather(1, (at // page).reshape(s["pages"].shape[0], -1)).reshape(at.shape)
    return ids.long() * page + at % page


def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _head_scales(scale, like):
    return None if scale is None else torch.tensor(scale, dtype=like.dtype, device=like.device)[:, None]


def _normed_rotated(s, x, weight):
    case = s["case"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    rot = case["rot"]
    if rot:
        cos, sin = s["table"][s["pos"].long()][:, :, None].split(rot // 2, dim=-1)
        if case["style"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
        x = torch.cat([turned, x[..., rot:]], dim=-1)
    return x


def _stored(s, x, scale):
    """New rows [B, n, Hkv, D] in the cache's type."""
    if scale is not None:
        x = (x / _head_scales(scale, x)).clamp(-448, 448)
    return x.to(s["k"].dtype)


def _plain_append(s):
    case = s["case"]
    B, n, Hkv = case["B"], case["q_len"], case["Hkv"]
    i = torch.arange(n, device=DEV)
    n_new = s["n_new"].long() if s["n_new"] is not None else torch.full((B,), n, device=DEV)
    live = i < n_new[:, None]
    q = _normed_rotated(s, s["q"], s["q_norm"]).to(s["q"].dtype)
    s["q_out"].copy_(torch.where(live[:, :, None, None], q, s["q_out"]))
    lens = s["lens"].long()
    # a sequence's tokens behind its last write that one's row again
    last = torch.minimum(i.expand(B, n), n_new[:, None] - 1)
    rows = _rows(s, lens[:, :, None] + last[:, None, :]).transpose(1, 2)
    pick = last[:, :, None, None]
    for_k = _stored(s, _normed_rotated(s, s["k_new"], s["k_norm"]), s["k_scale"])
    for_v = _stored(s, s["v_new"].float(), s["v_scale"])
    _bytes(s["k"])[rows] = _bytes(for_k).gather(1, pick.expand(for_k.shape))
    _bytes(s["v"])[rows] = _bytes(for_v).gather(1, pick.expand(for_v.shape))
    s["lens_out"].copy_(s["lens"] + n_new[:, None].to(torch.int32))


def _plain_accept(s):
    case = s["case"]
    B, n = case["B"], case["q_len"]
    i = torch.arange(n, device=DEV)
    n_new = s["n_new"].long()[:, None] if s["n_new"] is not None else n
    base = (s["lens_out"].long() - n_new)[:, :, None]
    last = torch.minimum(i.expand(B, n), s["n_path"].long()[:, None] - 1)     # at least one node is accepted here
    source = _rows(s, base + s["path"].long().gather(1, last)[:, None, :])
    target = _rows(s, base + last[:, None, :])
    k, v = _bytes(s["k"])[source], _bytes(s["v"])[source]
    _bytes(s["k"])[target], _bytes(s["v"])[target] = k, v
    s["lens_kept"].copy_(s["lens_out"] - n_new + s["n_path"][:, None])


def _plain_attend(s):
    case = s["case"]
    B, n, Hq, Hkv, D = (case[x] for x in ("B", "q_len", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    lens = s["lens"].long()
    n_new = s["n_new"].long()[:, None] if s["n_new"] is not None else torch.full((B, 1), n, device=DEV)
    t = torch.arange(s["longest"], device=DEV)
    rows = _rows(s, torch.minimum(t, lens[:, :, None] - 1))
    k, v = _bytes(s["k"])[rows].view(s["k"].dtype).float(), _bytes(s["v"])[rows].view(s["v"].dtype).float()      # [B, Hkv, longest, D]
    if s["k_scale"] is not None:
        k, v = k * _head_scales(s["k_scale"], k)[..., None], v * _head_scales(s["v_scale"], v)[..., None]
    q = s["q"].float().reshape(B, n, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, n * G, D)
    scores = (torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)).reshape(B, Hkv, n, G, -1)
    node = t - (lens - n_new)[:, :, None]                                     # of the draft, negative in front of it
    if s["tree"] is not None:
        bits = s["tree"][:, None, :, None] >> node.clamp(0, 63)[:, :, None, :] & 1
    else:
        bits = (node[:, :, None, :] <= torch.arange(n, device=DEV)[:, None]).long()
    seen = ((node < 0)[:, :, None, :] | (bits != 0)) & (t < lens[:, :, None])[:, :, None, :]
    scores = scores.masked_fill(~seen[:, :, :, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    w = torch.exp(scores - top)
    total = w.sum(-1, keepdim=True)
    out = (torch.matmul(w.reshape(B, Hkv, n * G, -1), v).reshape(B, Hkv, n, G, D) / total).transpose(1, 2).reshape(B, n, Hq, D)
    lse = (top + total.log()).squeeze(-1).transpose(1, 2).reshape(B, n, Hq)
    live = torch.arange(n, device=DEV) < n_new
    s["out"].copy_(torch.where(live[:, :, None, None], out.to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(live[:, :, None], lse, s["lse"]))


def _run_plain(s):
    op = s["case"]["op"]
    if op == "attend":
        _plain_attend(s)
        return s["out"], s["lse"]
    _plain_append(s)
    if op == "append":
        return s["q_out"], s["lens_out"], s["k"], s["v"]
    _plain_accept(s)
    return s["q_out"], s["lens_kept"], s["k"], s["v"]


# ---- what a pass cannot do without, and what it should give ----------------------------------------------
def work(case):
    B, Hq, Hkv, D, n = (case[x] for x in ("B", "Hq", "Hkv", "D", "q_len"))
    row = D * {"bf16": 2, "f32": 4, "kv8": 1}[case["dtype"]]
    elem = 4 if case["dtype"] == "f32" else 2
    before, n_new = _lens(case, 0).astype(np.int64), _n_new(case, 0).astype(np.int64)
    new = int(n_new.sum())
    if case["op"] == "attend":
        lens = before + n_new[:, None]
        size = 2 * int(lens.sum()) * row + new * Hq * (D * (2 + (4 if case["out"] == "f32" else 2)) + 4) + new * 8 * bool(case["tree"])
        size += (int((-(-lens // case["page"])).sum()) * 4 if case["page"] else B * Hkv * 8) + B * Hkv * 4
        return {"bytes": size, "flops": 4 * int((lens.sum(1) * n_new).sum()) * (Hq // Hkv) * D}
    size = new * ((Hq + 2 * Hkv) * D * elem + Hq * D * elem + 2 * Hkv * row + (case["rot"] * 4 + 4 if case["rot"] else 0)) + B * Hkv * 8
    flops = new * (Hq + Hkv) * D * (3 * bool(case["rot"]) + 4 * bool(case["norm"]))
    if case["op"] == "accept":                       # the rows that move, read and written, and the lengths
        path, count = _paths(case, 0, n_new, _trees(case, 0)[0])
        moved = int(((path != np.arange(n)) & (np.arange(n) < count[:, None])).sum())
        size += moved * Hkv * 4 * row + B * Hkv * 8 + int(count.sum()) * 4
    return {"bytes": size, "flops": flops}


def _turned_exact(case, s, x, weight):
    """float64 [B, n, H, D]: the norm by its sum of squares, the rotation as a product of complex numbers."""
    x = x.double()
    if weight is not None:
        x = x / ((x * x).sum(-1, keepdim=True) / case["D"] + EPS).sqrt() * weight.double()
    if case["rot"]:
        half = case["rot"] // 2
        table = s["table"].double()[s["pos"].long()]
        turn = torch.complex(table[..., :half], table[..., half:])[:, :, None]
        if case["style"] == "half":
            z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * turn
            x = torch.cat([z.real, z.imag, x[..., 2 * half:]], dim=-1)
        else:
            z = torch.view_as_complex(x[..., :2 * half].reshape(*x.shape[:-1], half, 2)) * turn
            x = torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * half:]], dim=-1)
    return x


def _first_row(s, pair, t):
    """The cache row of token t of a pair, on the host."""
    if s["off"] is not None:
        return int(s["host_off"][pair]) + t
    page = s["case"]["page"]
    return s["host_pages"][pair, t // page].astype(np.int64) * page + t % page


def exact(case, seed):
    s = _inputs(case, seed)
    s["host_off"] = s["off"].cpu().numpy().reshape(-1) if s["off"] is not None else None
    s["host_pages"] = s["pages"].cpu().numpy() if s["pages"] is not None else None
    B, n, Hq, Hkv, D = (case[x] for x in ("B", "q_len", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    lens, n_new = s["lens"].cpu().numpy().astype(np.int64), _n_new(case, seed).astype(np.int64)
    ks, vs = _scales(case) if case["dtype"] == "kv8" else ([1.0] * Hkv, [1.0] * Hkv)
    if case["op"] == "attend":
        out, lse = s["out"].double(), s["lse"].double()
        see = None if s["tree"] is None else s["tree"].cpu().numpy()
        for b in range(B):
            m = int(n_new[b])
            own_rows = torch.tril(torch.ones(m, m, dtype=torch.bool)) if see is None else torch.tensor([[bool(int(see[b, i]) >> j & 1) for j in range(m)] for i in range(m)])
            for h in range(Hkv):
                length = int(lens[b, h])
                rows = torch.as_tensor(_first_row(s, b * Hkv + h, np.arange(length))).to(DEV)
                kd, vd = _bytes(s["k"])[rows].view(s["k"].dtype).double() * ks[h], _bytes(s["v"])[rows].view(s["v"].dtype).double() * vs[h]
                cols = s["q"][b, :m, h * G:(h + 1) * G].reshape(m * G, D).double()
                z = (cols @ kd.t() / math.sqrt(D)).reshape(m, G, length)
                z[:, :, length - m:] = z[:, :, length - m:].masked_fill(~own_rows.to(DEV)[:, None, :], -math.inf)
                norm = torch.logsumexp(z, dim=-1)
                out[b, :m, h * G:(h + 1) * G] = (torch.exp(z - norm[..., None]).reshape(m * G, length) @ vd).reshape(m, G, D)
                lse[b, :m, h * G:(h + 1) * G] = norm
        return out, lse
    q, new_k = _turned_exact(case, s, s["q"], s["q_norm"]), _turned_exact(case, s, s["k_new"], s["k_norm"])
    q_out = s["q_out"].double()
    k, v = _bytes(s["k"]).view(s["k"].dtype).double(), _bytes(s["v"]).view(s["v"].dtype).double()
    path = count = None
    if case["op"] == "accept":
        path, count = s["path"].cpu().numpy(), s["n_path"].cpu().numpy()
    for b in range(B):
        m = int(n_new[b])
        q_out[b, :m] = q[b, :m]
        for h in range(Hkv):
            rows = torch.as_tensor(_first_row(s, b * Hkv + h, int(lens[b, h]) + np.arange(m))).to(DEV)
            k[rows], v[rows] = new_k[b, :m, h] / ks[h], s["v_new"][b, :m, h].double() / vs[h]
            if path is not None:
                kept = int(count[b])
                chosen = torch.as_tensor(path[b, :kept].astype(np.int64)).to(DEV)
                k[rows[:kept]], v[rows[:kept]] = k[rows[chosen]], v[rows[chosen]]
    return q_out, None, k, v
