"""The operators of a speculative decoding step, as cases that can be timed and checked.

One step of an engine that drafts a tree of tokens per sequence on a paged cache runs: block tables, slots, positions and
ancestor masks on the GPU (``tables``); in every layer rotary positions on queries and keys and the new rows into the cache
(``append``; ``rope`` is the same rotation on its own, with its gradient for training) and attention of the tree over cache
and tree (``tree``); then the decision which drafts hold (``verify``) and the rows of the accepted path moved to where the
next step expects them (``keep``). A case is one call of one of them (``rope``: the rotation and its gradient). Where ``own``
is false the operators are computed in their plain form.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
MLA = {"Hq": 64, "Hkv": 1, "d_qk": 576, "d_v": 512, "shared": True, "scale": 192 ** -0.5}
D128 = {"Hq": 32, "d_qk": 128, "d_v": 128, "shared": False, "scale": 128 ** -0.5}
# sink blocks, local blocks, block (1: token-granular)
LONG = {"sink": 128, "window": 8192, "block": 1}
SHORT = {"sink": 128, "window": 4096, "block": 1}
PAPER = {"sink": 1, "window": 7, "block": 128}


def listed():
    return [
        # one user's step with a small tree on a long context: launches and latency
        {"name": "tree_mla_paged_b1_n8", "op": "tree", "B": 1, "n": 8, "S_max": 131072, "page": 128, **MLA, **LONG},
        # a serving batch with full trees (40 to 64 nodes each), pages scattered over the pool
        {"name": "tree_mla_paged_b16_n64", "op": "tree", "B": 16, "n": 64, "S_max": 65536, "page": 128, **MLA, **LONG},
        # grouped heads of width 128, trees of odd size, contiguous caches of odd length
        {"name": "tree_gqa128_b8_n37", "op": "tree", "B": 8, "n": 37, "S_max": 32749, "page": 0, "Hkv": 8, **D128, **SHORT},
        # training at 16K tokens: the rotary columns of 64 heads into their place in the wide query rows, and the gradient back out
        {"name": "rope_mla_16k", "op": "rope", "dtype": "bf16", "T": 16384, "H": 64, "d": 64, "d_out": 576, "rot": 64, "interleaved": True, "factor": 32.0},
        # fp32, part of the head, half layout, odd length, no stretched context
        {"name": "rope_f32_half_1021", "op": "rope", "dtype": "f32", "T": 1021, "H": 8, "d": 96, "d_out": 96, "rot": 64, "interleaved": False, "factor": 1.0},
        # the layer-by-layer call of a serving step: rotate queries and latent keys, rows into the pages (1024 tree nodes, some padding)
        {"name": "append_mla_b16_n64", "op": "append", "T": 1024, "Hq": 64, "Hkv": 1, "dq": 64, "dq_out": 576, "d_qk": 576, "d_v": 0, "rot": 64,
         "interleaved": True, "factor": 32.0, "pool": 16384},
        # tables of a batch of trees
        {"name": "tables_tree_b16_n64", "op": "tables", "B": 16, "n": 64, "tree": True, "page": 128, "max_pages": 512},
        # tables of a step of chunked prefill for many requests (rows aligned to the right, not all of them new)
        {"name": "tables_chunk_b512_n200", "op": "tables", "B": 512, "n": 200, "tree": False, "page": 64, "max_pages": 1024},
        # one user's chain of 5 tokens, drafts that are not random (a greedy drafter)
        {"name": "verify_chain_b1_n5", "op": "verify", "B": 1, "n": 5, "V": 32003, "wide": 1, "draft": False},
        # a batch of sampled trees over a large vocabulary
        {"name": "verify_tree_b16_n64", "op": "verify", "B": 16, "n": 64, "V": 131072, "wide": 3, "draft": True},
        # accepted rows of 64 short trees, keys and values of 8 heads, one layer
        {"name": "keep_gqa128_b64_n8", "op": "keep", "B": 64, "n": 8, "layers": 1, "Hkv": 8, "d_qk": 128, "d_v": 128, "pool": 4096},
        # accepted rows of full trees in 28 sparse layers of a stacked latent cache
        {"name": "keep_mla_b16_n64_l28", "op": "keep", "B": 16, "n": 64, "layers": 28, "Hkv": 1, "d_qk": 576, "d_v": 0, "pool": 4096},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("tree", "tree", "rope", "append", "tables", "verify", "keep"))
    if op == "tree":
        wide = rng.random() < 0.6
        head = dict(MLA) if wide else {"Hkv": rng.choice((4, 8, 32)), **D128}
        pat = dict(rng.choice((LONG, PAPER)) if wide else rng.choice((SHORT, PAPER)))
        s, page = _log(rng, 2048, 65536), rng.choice((0, 64, 128))
        if page:
            s = (s + page - 1) // page * page
        return {"op": op, "B": _log(rng, 1, 16), "n": rng.randint(1, 64), "S_max": s, "page": page, **head, **pat}
    if op == "rope":
        d = rng.choice((64, 96, 128))
        return {"op": op, "dtype": rng.choice(("bf16", "f32")), "T": _log(rng, 1, 16384), "H": rng.choice((1, 8, 32, 64)), "d": d,
                "d_out": rng.choice((d, 576)), "rot": rng.choice((32, 64)), "interleaved": rng.random() < 0.5, "factor": rng.choice((1.0, 8.0, 32.0))}
    if op == "append":
        c = {"op": op, "T": _log(rng, 1, 4096), "rot": 64, "interleaved": rng.random() < 0.5, "factor": rng.choice((1.0, 32.0)), "pool": 16384}
        if rng.random() < 0.5:
            return {**c, "Hq": 64, "Hkv": 1, "dq": 64, "dq_out": 576, "d_qk": 576, "d_v": 0}
        return {**c, "Hq": 32, "Hkv": rng.choice((4, 8)), "dq": 128, "dq_out": 128, "d_qk": 128, "d_v": 128, "rot": rng.choice((64, 128))}
    if op == "tables":
        tree = rng.random() < 0.5
        return {"op": op, "B": _log(rng, 1, 512), "n": rng.randint(1, 64) if tree else _log(rng, 1, 512), "tree": tree,
                "page": rng.choice((32, 64, 128)), "max_pages": rng.choice((256, 700))}
    if op == "verify":
        return {"op": op, "B": _log(rng, 1, 16), "n": rng.randint(1, 64), "V": _log(rng, 1000, 131072), "wide": rng.choice((1, 2, 4)),
                "draft": rng.random() < 0.7}
    c = {"op": op, "B": _log(rng, 1, 64), "n": rng.randint(1, 64), "layers": rng.randint(1, 16), "pool": 4096}
    return {**c, **({"Hkv": 1, "d_qk": 576, "d_v": 0} if rng.random() < 0.5 else {"Hkv": rng.choice((2, 8)), "d_qk": 128, "d_v": 128})}


# ---- inputs ------------------------------------------------------------------------------------------

def _normal(gen, dtype, *shape):
    t = torch.empty(shape, dtype=dtype, device=DEV)
    flat = t.view(-1)
    step = 1 << 28
    for a in range(0, flat.numel(), step):
        b = min(flat.numel(), a + step)
        flat[a:b].copy_(torch.randn(b - a, generator=gen, device=DEV, dtype=torch.float32))
    return t


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _parents(rng, B, n, wide):
    """Random trees, parents before their children; node 0 is the root (the token whose row is not in the cache yet)."""
    p = np.full((B, n), -1, dtype=np.int32)
    for r in range(1, n):
        p[:, r] = rng.integers(max(0, (r - 1) // max(1, wide) - 1) if wide > 1 else r - 1, max(1, (r - 1) // max(1, wide) + 1), size=B) if wide > 1 else r - 1
    return p


def _masks(parents, lens):
    B, n = parents.shape
    m = np.zeros((B, n), dtype=np.uint64)
    for r in range(n):
        m[:, r] = np.uint64(1) << np.uint64(r)
        for b in range(B):
            if 0 <= parents[b, r] < r:
                m[b, r] |= m[b, parents[b, r]]
    m[np.arange(n)[None, :] >= np.asarray(lens)[:, None]] = 0
    return m.view(np.int64)


def _freq(c):
    """YaRN: frequencies below one turn of the original context are divided by the factor, those above 32 turns kept, a ramp between."""
    base, s, original = 10000.0, c["factor"], 32768
    f = base ** (-np.arange(0, c["rot"], 2, dtype=np.float64) / c["rot"])
    turns = original * f / (2 * math.pi)
    keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
    m = 0.1 * math.log(s) + 1.0 if s > 1 else 1.0
    return f / s * (1 - keep) + f * keep, m


def _prepare_tree(c, s, gen, rng):
    B, n, S = c["B"], c["n"], c["S_max"]
    lens = rng.integers(max(n, S // 4), S + 1, size=B).astype(np.int32)
    nodes = rng.integers(max(1, (5 * n) // 8), n + 1, size=B).astype(np.int32)
    s["parents_host"], s["lens_host"], s["nodes_host"] = _parents(rng, B, n, 4), lens, nodes
    s["masks"] = _dev(_masks(s["parents_host"], nodes))
    s["lens"], s["nodes"] = _dev(lens), _dev(nodes)
    if c["page"]:
        per = S // c["page"]
        s["table"] = _dev(rng.permutation(B * per).astype(np.int32).reshape(B, per))
        rows = (B * per, c["page"])
    else:
        rows = (B, S)
    bf = torch.bfloat16
    s["q"] = _normal(gen, bf, B, n, c["Hq"], c["d_qk"])
    s["k"] = _normal(gen, bf, *rows, c["Hkv"], c["d_qk"])
    s["v"] = s["k"] if c["shared"] else _normal(gen, bf, *rows, c["Hkv"], c["d_v"])
    s["out"] = torch.empty(B, n, c["Hq"], c["d_v"], dtype=bf, device=DEV)
    s["lse"] = torch.empty(B, c["Hq"], n, dtype=torch.float32, device=DEV)


def _prepare_rope(c, s, gen, rng):
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    start = int(rng.integers(0, 1 << 20))
    s["pos"] = _dev((start + np.arange(c["T"])).astype(np.int32))
    f, s["m"] = _freq(c)
    s["freq"] = _dev(f)
    s["x"] = _normal(gen, dt, c["T"], c["H"], c["d"])
    s["wide"] = torch.zeros(c["T"], c["H"], c["d_out"], dtype=dt, device=DEV)
    s["dwide"] = _normal(gen, dt, c["T"], c["H"], c["d_out"])
    s["y"], s["dy"] = (t[..., c["d_out"] - c["d"]:] for t in (s["wide"], s["dwide"]))
    s["dx"] = torch.empty_like(s["x"])


def _prepare_append(c, s, gen, rng):
    bf, T = torch.bfloat16, c["T"]
    s["pos"] = _dev(rng.integers(0, 1 << 20, size=T).astype(np.int32))
    slots = rng.permutation(c["pool"])[:T].astype(np.int32)
    dead = rng.random(T) < 0.1                      # padding behind the last node of a sequence
    dead[0] = False
    s["pos"][_dev(dead)] = -1
    slots[dead] = -1
    s["slots"] = _dev(slots)
    f, s["m"] = _freq(c)
    s["freq"] = _dev(f)
    s["q"] = _normal(gen, bf, T, c["Hq"], c["dq"])
    s["k"] = _normal(gen, bf, T, c["Hkv"], c["d_qk"])
    s["q_wide"] = _normal(gen, bf, T, c["Hq"], c["dq_out"])
    s["q_out"] = s["q_wide"][..., c["dq_out"] - c["dq"]:]
    s["k_rows"] = _normal(gen, bf, c["pool"], c["Hkv"], c["d_qk"])
    s["v"] = _normal(gen, bf, T, c["Hkv"], c["d_v"]) if c["d_v"] else None
    s["v_rows"] = _normal(gen, bf, c["pool"], c["Hkv"], c["d_v"]) if c["d_v"] else None


def _prepare_tables(c, s, gen, rng):
    B, n, page, most = c["B"], c["n"], c["page"], c["max_pages"]
    cache = rng.integers(0, most * page - n, size=B).astype(np.int32)
    new = (n - rng.integers(0, max(1, n // 2), size=B)).astype(np.int32)
    have = -(-cache // page)
    s["num_pages"] = B * most
    pool = rng.permutation(B * most).astype(np.int32)
    table = np.full((B, most), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, :have[b]] = pool[at:at + have[b]]
        at += int(have[b])
    s["host"] = {"cache": cache, "new": new, "table": table.copy(), "free": pool[at:].copy(), "count": len(pool) - at}
    s["parents_host"] = _parents(rng, B, n, 3) if c["tree"] else None
    s["cache"], s["new"], s["table"], s["free"] = _dev(cache), _dev(new), _dev(table), _dev(pool[at:])
    s["count"] = _dev(np.array([len(pool) - at], dtype=np.int32))
    s["parents"] = _dev(s["parents_host"]) if c["tree"] else None
    i32 = dict(dtype=torch.int32, device=DEV)
    s["granted"], s["seqlens"], s["left"] = torch.empty(B, **i32), torch.empty(B, **i32), torch.empty(1, **i32)
    s["positions"], s["slots"] = torch.empty(B, n, **i32), torch.empty(B, n, **i32)
    s["masks"] = torch.empty(B, n, dtype=torch.int64, device=DEV) if c["tree"] else None


def _prepare_verify(c, s, gen, rng):
    B, n, V = c["B"], c["n"], c["V"]
    parents = _parents(rng, B, n, c["wide"])
    nodes = rng.integers(max(1, n - n // 3), n + 1, size=B).astype(np.int32)
    logits = torch.randn(B, n, V, generator=gen, device=DEV).mul_(3.0)
    s["target"] = torch.softmax(logits, -1)
    # a drafter that is right more often than not: the target's logits with some noise
    draft = torch.softmax(logits.add_(torch.randn(B, n, V, generator=gen, device=DEV), alpha=0.7), -1)
    del logits
    rank = np.zeros((B, n), dtype=np.int64)         # which child of its parent
    for b in range(B):
        seen = {}
        for r in range(1, n):
            rank[b, r] = seen.get(parents[b, r], 0)
            seen[parents[b, r]] = rank[b, r] + 1
    most = int(rank.max()) + 1
    if c["draft"]:
        choice = torch.multinomial(draft.view(B * n, V), most, replacement=True, generator=gen)
    else:
        choice = draft.view(B * n, V).topk(most, -1).indices
    up = _dev(np.maximum(parents, 0).astype(np.int64))
    tok = choice.view(B, n, most)[torch.arange(B, device=DEV)[:, None], up, _dev(rank)].to(torch.int32)
    s["draft"] = draft if c["draft"] else None
    s["tokens"], s["parents"], s["nodes"] = tok, _dev(parents), _dev(nodes)
    s["u_accept"] = torch.rand(B, n, generator=gen, device=DEV)
    s["u_next"] = torch.rand(B, generator=gen, device=DEV)
    s["path"] = torch.empty(B, n, dtype=torch.int32, device=DEV)
    s["path_lens"], s["next"] = (torch.empty(B, dtype=torch.int32, device=DEV) for _ in range(2))


def _prepare_keep(c, s, gen, rng):
    B, n = c["B"], c["n"]
    bf = torch.bfloat16
    s["slots"] = _dev(rng.permutation(c["pool"])[:B * n].astype(np.int32).reshape(B, n))
    path, lens = np.full((B, n), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    for b in range(B):
        # nodes of one path, at most 8 of them, all behind the rows they move to (so that a pass can be repeated)
        a = int(rng.integers(0, min(8, (n + 1) // 2) + 1))
        first = rng.choice(np.arange(a, n), size=max(0, a - 1), replace=False) if a > 1 else np.zeros(0, dtype=np.int64)
        path[b, :a] = ([0] + sorted(int(x) for x in first))[:a]
        lens[b] = a
    s["path"], s["path_lens"] = _dev(path), _dev(lens)
    s["path_host"], s["path_lens_host"] = path, lens
    s["k_rows"] = _normal(gen, bf, c["layers"], c["pool"], c["Hkv"], c["d_qk"])
    s["v_rows"] = _normal(gen, bf, c["layers"], c["pool"], c["Hkv"], c["d_v"]) if c["d_v"] else None


def prepare(case, seed):
    s = {"case": case}
    gen, rng = torch.Generator(device=DEV).manual_seed(seed), np.random.default_rng(seed)
    globals()["_prepare_" + case["op"]](case, s, gen, rng)
    if own:
        import paper_2512_23966_amd as loza
        c = case
        if c["op"] == "tree":
            nb = loza.loza_ssa_extend_tree_workspace_bytes(c["B"], c["Hq"], c["Hkv"], c["S_max"], c["n"], c["d_qk"], c["d_v"], c["sink"], c["window"], c["block"])
            s["ws"] = torch.empty(nb, dtype=torch.uint8, device=DEV)
        if c["op"] == "verify":
            s["ws"] = torch.empty(loza.loza_ssa_verify_tree_workspace_bytes(c["B"], c["n"], c["V"]), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ------------------------------------------------------------------------------------------

def run(s):
    return globals()[("_own_" if own else "_plain_") + s["case"]["op"]](s["case"], s)


def _own_tree(c, s):
    import paper_2512_23966_amd as loza
    loza.loza_ssa_extend_tree(s["q"], s["k"], s["v"], s["lens"], s["nodes"], s["masks"], s["out"], s["lse"], c["sink"], c["window"], c["block"],
                              c["scale"], block_table=s.get("table"), workspace=s["ws"])
    return [s["out"], s["lse"]]


def _own_rope(c, s):
    import paper_2512_23966_amd as loza
    fn = loza.loza_ssa_rope_f32 if c["dtype"] == "f32" else loza.loza_ssa_rope
    fn(s["x"], s["pos"], s["freq"], s["y"], c["d"] - c["rot"], c["interleaved"], s["m"])
    fn(s["dy"], s["pos"], s["freq"], s["dx"], c["d"] - c["rot"], c["interleaved"], s["m"], inverse=True)
    return [s["y"], s["dx"]]


def _own_append(c, s):
    import paper_2512_23966_amd as loza
    loza.loza_ssa_rope_append(s["q"], s["k"], s["v"], s["pos"], s["slots"], s["freq"], s["q_out"], s["k_rows"], s["v_rows"],
                              c["dq"] - c["rot"], c["d_qk"] - c["rot"], c["interleaved"], s["m"])
    return [s["q_wide"], s["k_rows"]] + ([s["v_rows"]] if c["d_v"] else [])


def _own_tables(c, s):
    import paper_2512_23966_amd as loza
    loza.loza_ssa_step_tables(s["cache"], s["new"], s["parents"], s["free"], s["count"], s["table"], s["num_pages"], c["page"],
                              s["granted"], s["seqlens"], s["positions"], s["slots"], s["masks"], s["left"])
    return [s["granted"], s["seqlens"], s["positions"], s["slots"], s["left"], s["table"]] + ([s["masks"]] if c["tree"] else [])


def _own_verify(c, s):
    import paper_2512_23966_amd as loza
    loza.loza_ssa_verify_tree(s["target"], s["draft"], s["tokens"], s["parents"], s["nodes"], s["u_accept"], s["u_next"],
                              s["path"], s["path_lens"], s["next"], s["ws"])
    return [s["path"], s["path_lens"], s["next"]]


def _own_keep(c, s):
    import paper_2512_23966_amd as loza
    loza.loza_ssa_keep_accepted(s["k_rows"], s["v_rows"], s["slots"], s["path"], s["path_lens"])
    return [s["k_rows"]] + ([s["v_rows"]] if c["d_v"] else [])


# ---- plain forms -----------------------------------------------------------------------------------------

def _window_begin(c, i):
    return max(0, (i // c["block"] - c["window"] + 1) * c["block"])


def _popcount(m):
    return ((m[..., None] >> torch.arange(64, device=DEV)) & 1).sum(-1)


def _plain_tree(c, s):
    n, G = c["n"], c["Hq"] // c["Hkv"]
    bit = torch.arange(64, device=DEV)
    for b in range(c["B"]):
        L, nb = int(s["lens_host"][b]), int(s["nodes_host"][b])
        P, sink = L - nb, c["sink"] * c["block"]
        w0 = max(_window_begin(c, P), min(sink, L))
        j = torch.cat([torch.arange(0, min(sink, L), device=DEV), torch.arange(w0, L, device=DEV)])
        if c["page"]:
            at = s["table"][b].long()[j // c["page"]]
            kk, vv = s["k"][at, j % c["page"]], s["v"][at, j % c["page"]]
        else:
            kk, vv = s["k"][b, j], s["v"][b, j]
        m = s["masks"][b]                                                           # [n]
        pos = P + _popcount(m) - 1                                                  # [n]
        seen = ((m[:, None] >> bit) & 1).bool() & (bit[None, :] < nb)               # [n, 64] nodes on the path
        key_pos = torch.where(seen, P + seen.long().cumsum(1) - 1, -1)              # their positions
        a = (j - P).clamp(0, 63)
        at_pos = torch.where((j >= P)[None, :], key_pos[:, a], j[None, :])
        lo = ((pos // c["block"] - c["window"] + 1) * c["block"]).clamp(min=0)
        ok = (at_pos >= 0) & ((at_pos < sink) | (at_pos >= lo[:, None])) & (m != 0)[:, None]
        ok &= (torch.arange(n, device=DEV) < nb)[:, None]
        for g in range(c["Hkv"]):
            hs = slice(g * G, (g + 1) * G)
            q = s["q"][b, :, hs].float().reshape(n * G, -1)
            x = (q @ kk[:, g].float().t()).view(n, G, -1) * c["scale"]
            x = x.masked_fill(~ok[:, None, :], -math.inf)
            top = x.amax(-1, keepdim=True).clamp(min=-1e30)
            p = (x - top).exp()
            den = p.sum(-1, keepdim=True)
            o = (p.view(n * G, -1) @ vv[:, g, : c["d_v"]].float()).view(n, G, -1) / den.clamp(min=1e-30)
            s["out"][b, :, hs] = o.to(torch.bfloat16)
            s["lse"][b, hs] = (top + den.log())[..., 0].t()
    return [s["out"], s["lse"]]


def _rotate(x, pos, freq, m, begin, interleaved, sign=1.0):
    """x [T, H, d] with its columns from `begin` on rotated, in fp32 (the angles in 64 bits)."""
    rot = 2 * freq.numel()
    ang = pos.double()[:, None] * freq[None, :]
    co, si = ((f(ang) * m).float()[:, None, :] for f in (torch.cos, torch.sin))
    y = x.float()
    r = y[..., begin:begin + rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., : rot // 2], r[..., rot // 2:])
    u, w = a * co - sign * b * si, sign * a * si + b * co
    z = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([y[..., :begin], z, y[..., begin + rot:]], -1).to(x.dtype)


def _plain_rope(c, s):
    s["y"].copy_(_rotate(s["x"], s["pos"], s["freq"], s["m"], c["d"] - c["rot"], c["interleaved"]))
    s["dx"].copy_(_rotate(s["dy"], s["pos"], s["freq"], s["m"], c["d"] - c["rot"], c["interleaved"], -1.0))
    return [s["y"], s["dx"]]


def _plain_append(c, s):
    live = s["pos"] >= 0
    q = _rotate(s["q"], s["pos"], s["freq"], s["m"], c["dq"] - c["rot"], c["interleaved"])
    s["q_out"].copy_(torch.where(live[:, None, None], q, s["q_out"]))
    k = _rotate(s["k"], s["pos"], s["freq"], s["m"], c["d_qk"] - c["rot"], c["interleaved"])
    put = live & (s["slots"] >= 0)
    at = s["slots"][put].long()
    s["k_rows"][at] = k[put]
    if c["d_v"]:
        s["v_rows"][at] = s["v"][put]
    return [s["q_wide"], s["k_rows"]] + ([s["v_rows"]] if c["d_v"] else [])


def _plain_tables(c, s):
    B, n, page, most = c["B"], c["n"], c["page"], c["max_pages"]
    cache, new, count = s["cache"].long(), s["new"].long(), s["count"].long()
    have, want = (cache + page - 1) // page, (cache + new + page - 1) // page
    fits = (cache + new <= most * page) & (new >= 0) & (new <= n) & (cache >= 0)
    need = torch.where(fits, want - have, 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= count))
    granted = torch.where(ok, new, 0)
    # entries of the new pages: column have + i of row b takes the page at upto - need + i from the end of the free list
    col = torch.arange(most, device=DEV)[None, :]
    mine = ok[:, None] & (col >= have[:, None]) & (col < want[:, None])
    at = (count - 1 - (upto - need)[:, None] - (col - have[:, None])).clamp(0, max(0, s["free"].numel() - 1))
    if s["free"].numel():
        s["table"].copy_(torch.where(mine, s["free"][at], s["table"]))
    r = torch.arange(n, device=DEV)[None, :]
    if c["tree"]:
        m = torch.zeros(B, n, dtype=torch.int64, device=DEV)
        for i in range(n):
            up = s["parents"][:, i].long()
            above = torch.where((up >= 0) & (up < i), m.gather(1, up.clamp(0, n - 1)[:, None])[:, 0], 0)
            m[:, i] = above | (1 << i if i < 63 else -(1 << 63))
        row, there = cache[:, None] + r, r < granted[:, None]
        s["masks"].copy_(torch.where(there, m, 0))
        pos = cache[:, None] + _popcount(m) - 1
    else:
        row, there = (cache + granted - n)[:, None] + r, r >= n - granted[:, None]
        pos = row
    page_id = s["table"].long().gather(1, (row // page).clamp(0, most - 1))
    slot = torch.where((page_id >= 0) & (page_id < s["num_pages"]), page_id * page + row % page, -1)
    s["granted"].copy_(granted)
    s["seqlens"].copy_(cache + granted)
    s["positions"].copy_(torch.where(there, pos, -1))
    s["slots"].copy_(torch.where(there, slot, -1))
    s["left"].copy_(count - torch.where(ok, upto * (need > 0), 0).amax())
    return [s["granted"], s["seqlens"], s["positions"], s["slots"], s["left"], s["table"]] + ([s["masks"]] if c["tree"] else [])


def _plain_verify(c, s):
    B, n, V = c["B"], c["n"], c["V"]
    row = torch.arange(B, device=DEV)
    f64 = torch.float64
    cur, length = torch.zeros(B, dtype=torch.long, device=DEV), (s["nodes"] > 0).long()
    off, left = torch.zeros(B, dtype=f64, device=DEV), torch.ones(B, dtype=f64, device=DEV)
    gone = torch.zeros(B, V, dtype=torch.bool, device=DEV)      # drafts that are not random: rejected tokens of this node
    s["path"].fill_(-1)
    s["path"][:, 0] = torch.where(s["nodes"] > 0, 0, -1)

    def residual():
        p = s["target"][row, cur].to(f64)
        if s["draft"] is None:
            return p.masked_fill(gone, 0.0)
        return (p - off[:, None] * s["draft"][row, cur].to(f64)).clamp(min=0.0)

    for r in range(1, n):
        test = (s["parents"][:, r] == cur) & (r < s["nodes"]) & (s["tokens"][:, r] >= 0) & (s["tokens"][:, r] < V)
        x = s["tokens"][:, r].long().clamp(0, V - 1)
        p, u = s["target"][row, cur, x].to(f64), s["u_accept"][:, r].to(f64)
        if s["draft"] is None:
            a, q = torch.where(gone[row, x], 0.0, p), torch.ones_like(p)
        else:
            q = s["draft"][row, cur, x].to(f64)
            a = (p - off * q).clamp(min=0.0)
        take = test & (u * q * left < a)
        drop = test & ~take
        if s["draft"] is None:
            left = torch.where(drop, left - a, left)
            gone[row, x] |= drop
            gone &= ~take[:, None]
        else:
            off = torch.where(drop, off + left, off)
            left = torch.where(drop, residual().sum(-1), left)
        off, left = torch.where(take, 0.0, off), torch.where(take, 1.0, left)
        cur = torch.where(take, r, cur)
        s["path"][row, length.clamp(max=n - 1)] = torch.where(take, r, s["path"][row, length.clamp(max=n - 1)])
        length = length + take
    w = residual()
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, s["target"][row, cur].to(f64))
    cum = w.cumsum(-1)
    x = (cum <= s["u_next"].to(f64)[:, None] * cum[:, -1:]).sum(-1).clamp(max=V - 1)
    s["path_lens"].copy_(length)
    s["next"].copy_(torch.where((s["nodes"] > 0) & (cum[:, -1] > 0), x, -1))
    return [s["path"], s["path_lens"], s["next"]]


def _plain_keep(c, s):
    i = torch.arange(c["n"], device=DEV)[None, :]
    src = s["slots"].gather(1, s["path"].long().clamp(0, c["n"] - 1))
    move = (i < s["path_lens"][:, None]) & (s["path"] >= 0) & (src >= 0) & (s["slots"] >= 0)
    a, b = src[move].long(), s["slots"][move].long()
    for t in (s["k_rows"], s["v_rows"]):
        if t is not None:
            t[:, b] = t[:, a]
    return [s["k_rows"]] + ([s["v_rows"]] if c["d_v"] else [])


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "tree":
        row = (c["d_qk"] if c["shared"] else c["d_qk"] + c["d_v"]) * 2
        q_row = (c["d_qk"] + c["d_v"]) * 2 + 4
        at = [max(c["n"], c["S_max"] // 4) + (c["S_max"] - max(c["n"], c["S_max"] // 4)) * (2 * t + 1) // 32 for t in range(16)]
        nodes, deep = (max(1, (5 * c["n"]) // 8) + c["n"]) / 2, math.log2(c["n"] + 1)     # (trees of about that depth)
        live = sum(min(c["sink"] * c["block"], _window_begin(c, x)) + x - _window_begin(c, x) for x in at) / 16
        return {"bytes": c["B"] * (c["Hkv"] * (live + nodes) * row + nodes * c["Hq"] * q_row),
                "flops": c["B"] * c["Hq"] * nodes * (live + deep / 2) * 2 * (c["d_qk"] + c["d_v"])}
    if c["op"] == "rope":
        es, elems = 4 if c["dtype"] == "f32" else 2, c["T"] * c["H"] * c["d"]
        return {"bytes": 4 * elems * es, "flops": 2 * 3 * c["T"] * c["H"] * c["rot"]}
    if c["op"] == "append":
        row = c["Hq"] * c["dq"] + c["Hkv"] * (c["d_qk"] + c["d_v"])
        return {"bytes": 2 * 2 * c["T"] * row, "flops": 3 * c["T"] * (c["Hq"] + c["Hkv"]) * c["rot"]}
    if c["op"] == "tables":
        return {"bytes": c["B"] * (16 + c["n"] * (20 if c["tree"] else 8)), "flops": 0}
    if c["op"] == "verify":
        return {"bytes": c["B"] * c["V"] * 4 * (2 if c["draft"] else 1), "flops": c["B"] * c["V"] * (3 if c["draft"] else 1)}
    rows = c["B"] * max(0.0, min(8, (c["n"] + 1) // 2) / 2 - 1)
    return {"bytes": 2 * rows * c["layers"] * c["Hkv"] * (c["d_qk"] + c["d_v"]) * 2, "flops": 0}


# ---- the same from the definitions, in 64 bits --------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return globals()["_exact_" + case["op"]](case, s)


def _ancestors(parents, r):
    path = [r]
    while parents[path[-1]] >= 0:
        path.append(int(parents[path[-1]]))
    return path[::-1]


def _exact_tree(c, s):
    f64 = torch.float64
    out = torch.zeros(s["out"].shape, dtype=f64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=f64, device=DEV)
    G = c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        L, nb = int(s["lens_host"][b]), int(s["nodes_host"][b])
        P, sink = L - nb, c["sink"] * c["block"]
        first = _window_begin(c, P)
        rows = [j for j in range(0, min(sink, first))] + list(range(first, L))
        j = np.array(rows)
        ok = np.zeros((nb, len(rows)), dtype=bool)
        for r in range(nb):
            path = _ancestors(s["parents_host"][b], r)
            i = P + len(path) - 1
            lo = _window_begin(c, i)
            ok[r] = (j < P) & ((j < sink) | (j >= lo))
            for depth, a in enumerate(path):
                ok[r, len(rows) - nb + a] = P + depth < sink or P + depth >= lo
        if c["page"]:
            at = _dev(s["table"][b].cpu().numpy()[j // c["page"]].astype(np.int64) * c["page"] + j % c["page"])
            kk, vv = (s[x].view(-1, c["Hkv"], s[x].shape[-1])[at] for x in ("k", "v"))
        else:
            kk, vv = s["k"][b, _dev(j)], s["v"][b, _dev(j)]
        bad = ~_dev(ok)
        for g in range(c["Hkv"]):
            hs = slice(g * G, (g + 1) * G)
            kg, vg = kk[:, g].to(f64), vv[:, g, : c["d_v"]].to(f64)
            for a in range(0, nb, 16):
                e = min(nb, a + 16)
                q = s["q"][b, a:e, hs].to(f64)
                x = torch.matmul(q.reshape((e - a) * G, -1), kg.t()).view(e - a, G, -1) * c["scale"]
                x.masked_fill_(bad[a:e, None, :], -math.inf)
                ls = torch.logsumexp(x, -1)
                p = (x - ls[..., None]).exp_()
                out[b, a:e, hs] = torch.matmul(p.view((e - a) * G, -1), vg).view(e - a, G, -1)
                lse[b, hs, a:e] = ls.t()
    return [out, lse]


def _turn(x, pos, freq, m, begin, interleaved, back=False):
    """Every pair as a complex number times m e^(i angle)."""
    k = freq.numel()
    z = x.double().clone()
    first = begin + (2 * torch.arange(k, device=DEV) if interleaved else torch.arange(k, device=DEV))
    second = first + (1 if interleaved else k)
    ang = torch.remainder(pos.double()[:, None] * freq[None, :], 2 * math.pi)
    w = torch.polar(torch.full_like(ang, m), -ang if back else ang)[:, None, :]
    v = torch.complex(z[..., first], z[..., second]) * w
    z[..., first], z[..., second] = v.real, v.imag
    return z


def _exact_rope(c, s):
    at = c["d"] - c["rot"]
    return [_turn(s["x"], s["pos"], s["freq"], s["m"], at, c["interleaved"]), _turn(s["dy"], s["pos"], s["freq"], s["m"], at, c["interleaved"], True)]


def _exact_append(c, s):
    q, rows = s["q_wide"].double(), s["k_rows"].double()
    live = (s["pos"] >= 0).nonzero()[:, 0]
    q[live, :, c["dq_out"] - c["dq"]:] = _turn(s["q"], s["pos"], s["freq"], s["m"], c["dq"] - c["rot"], c["interleaved"])[live]
    at = s["slots"][live].long()
    rows[at] = _turn(s["k"], s["pos"], s["freq"], s["m"], c["d_qk"] - c["rot"], c["interleaved"])[live]
    if not c["d_v"]:
        return [q, rows]
    vals = s["v_rows"].double()
    vals[at] = s["v"][live].double()
    return [q, rows, vals]


def _exact_tables(c, s):
    h, n, page = s["host"], c["n"], c["page"]
    free, left = list(h["free"]), int(h["count"])
    table, B = h["table"].copy(), c["B"]
    granted, seqlens = np.zeros(B, np.int32), np.zeros(B, np.int32)
    positions, slots, masks = (np.full((B, n), -1, np.int32), np.full((B, n), -1, np.int32), np.zeros((B, n), np.uint64))
    for b in range(B):
        cl, m = int(h["cache"][b]), int(h["new"][b])
        first, last = (cl + page - 1) // page, (cl + m + page - 1) // page
        assert last <= c["max_pages"] and last - first <= left
        for i in range(first, last):
            left -= 1
            table[b, i] = free[left]
        granted[b], seqlens[b] = m, cl + m
        for t in range(m):
            r, row = (t, cl + t) if c["tree"] else (n - m + t, cl + t)
            slots[b, r] = table[b, row // page] * page + row % page
            positions[b, r] = row
            if c["tree"]:
                path = _ancestors(s["parents_host"][b], r)
                positions[b, r] = cl + len(path) - 1
                masks[b, r] = sum(1 << a for a in path)
    res = [granted, seqlens, positions, slots, np.array([left], np.int32), table] + ([masks.view(np.int64)] if c["tree"] else [])
    return [_dev(x) for x in res]


def _exact_verify(c, s):
    B, n = c["B"], c["n"]
    path, lens, nxt = np.full((B, n), -1, np.int32), np.zeros(B, np.int32), np.full(B, -1, np.int32)
    tok, par, nodes, ua, un = (s[x].cpu().numpy() for x in ("tokens", "parents", "nodes", "u_accept", "u_next"))
    for b in range(B):
        at, walk = 0, [0]
        while True:
            p = s["target"][b, at].cpu().numpy().astype(np.float64)
            q = None if s["draft"] is None else s["draft"][b, at].cpu().numpy().astype(np.float64)
            total, hit = 1.0, -1
            for r in (r for r in range(at + 1, int(nodes[b])) if par[b, r] == at):
                x = tok[b, r]
                if float(ua[b, r]) * (1.0 if q is None else q[x]) * total < p[x]:
                    hit = r
                    break
                if q is None:
                    total -= p[x]
                    p[x] = 0.0
                else:
                    p = np.maximum(p - total * q, 0.0)     # the residual, not normalised; its sum takes the place of 1
                    total = math.fsum(p)
            if hit < 0:
                break
            at = hit
            walk.append(hit)
        path[b, :len(walk)], lens[b] = walk, len(walk)
        cum = np.cumsum(p)
        nxt[b] = int(np.searchsorted(cum, float(un[b]) * cum[-1], side="right"))
    return [_dev(x) for x in (path, lens, nxt)]


def _exact_keep(c, s):
    res = [s["k_rows"].double()] + ([s["v_rows"].double()] if c["d_v"] else [])
    slots = s["slots"].cpu().numpy()
    for t in res:
        before = t.clone()
        for b in range(c["B"]):
            for i in range(int(s["path_lens_host"][b])):
                t[:, int(slots[b, i])] = before[:, int(slots[b, s["path_host"][b, i]])]
    return res
