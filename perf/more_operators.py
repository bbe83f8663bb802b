"""Operators of a decode step beside its attention, as cases that can be timed and checked.

``norm``: the norm of each head (RMS, with a weight a column) and its rotary positions in one pass, and the gradient of both; ``append``:
the same for the queries and keys of a serving step, whose rows go to the cache; ``probs``: probabilities from logits under penalties for
repeated tokens, biases and grammar masks, for every node of a tree of drafts; ``count``: the record of a request's tokens that those
penalties read; ``pages``: a request's pages shared with its forks, the started page copied, pages of ended requests and of rows that no later
query sees given back; ``compact``: the pages in use moved to the front of the pool. A case is one pass of one of them. Where ``own`` is false the
operators are computed in their plain form.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
F64 = torch.float64
I32 = torch.int32


def listed():
    return [
        # training at 16K tokens: 32 query heads of width 128, normed and rotated as a whole, and the gradient
        {"name": "norm_gqa128_16k", "op": "norm", "dtype": "bf16", "T": 16384, "H": 32, "d": 128, "norm": 128, "rot_begin": 0, "rot": 128,
         "interleaved": False, "factor": 32.0},
        # fp32, an odd number of tokens, a width that is no power of two, part of the columns rotated
        {"name": "norm_f32_1021", "op": "norm", "dtype": "f32", "T": 1021, "H": 8, "d": 96, "norm": 96, "rot_begin": 32, "rot": 64,
         "interleaved": True, "factor": 1.0},
        # one layer of a decode step of 64 requests: queries and keys of width 128 normed and rotated, keys and values into the pages
        {"name": "append_gqa128_b64", "op": "append", "T": 64, "Hq": 32, "Hkv": 8, "dq": 128, "dq_out": 128, "q_norm": 128, "d_k": 128, "k_norm": 128,
         "d_v": 128, "rot": 128, "interleaved": False, "factor": 1.0, "pool": 16384},
        # one layer of chunked prefill at the wide shape: 512 latent columns normed, 64 rotary ones, of 64 heads' queries the rotary columns alone
        {"name": "append_mla_8k", "op": "append", "T": 8192, "Hq": 64, "Hkv": 1, "dq": 64, "dq_out": 576, "q_norm": 0, "d_k": 576, "k_norm": 512,
         "d_v": 0, "rot": 64, "interleaved": True, "factor": 32.0, "pool": 16384},
        # one user's next token: an odd vocabulary, fp32 logits, penalties and a grammar
        {"name": "probs_b1_n1_v32003", "op": "probs", "dtype": "f32", "B": 1, "n": 1, "V": 32003, "bias": 5, "grammar": True, "seen": 3000},
        # a serving batch of full trees over a large vocabulary
        {"name": "probs_tree_b16_n64", "op": "probs", "dtype": "bf16", "B": 16, "n": 64, "V": 131072, "bias": 64, "grammar": True, "seen": 20000},
        # one request of a short prompt arrives
        {"name": "count_b1_500", "op": "count", "B": 1, "n": 500, "V": 32003},
        # 16 requests with long prompts come back after they had to give way
        {"name": "count_b16_100k", "op": "count", "B": 16, "n": 100000, "V": 131072},
        # eight samples of one prompt, one layer of 8 key heads of width 128; another request ends
        {"name": "pages_gqa128_b12", "op": "pages", "B": 12, "forks": 7, "ends": 1, "page": 64, "max_pages": 64, "layers": 1, "Hkv": 8, "d_k": 128, "d_v": 128,
         "sink": 128, "window": 1024},
        # a large batch at the wide shape, four stacked layers of one pool: forks, ends, and windows that leave pages behind
        {"name": "pages_mla_b256", "op": "pages", "B": 256, "forks": 60, "ends": 30, "page": 32, "max_pages": 256, "layers": 4, "Hkv": 1, "d_k": 576, "d_v": 0,
         "sink": 128, "window": 2048},
        # a small pool is tidied
        {"name": "compact_p1500", "op": "compact", "B": 16, "page": 32, "max_pages": 100, "pool": 1500, "used": 0.5, "layers": 1, "Hkv": 2, "d_k": 128, "d_v": 128},
        # half of a large pool is given back to something else
        {"name": "compact_p40000", "op": "compact", "B": 200, "page": 32, "max_pages": 600, "pool": 40000, "used": 0.45, "layers": 1, "Hkv": 1, "d_k": 576, "d_v": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "norm", "append", "append", "probs", "probs", "count", "pages", "pages", "compact"))
    if op == "norm":
        d, norm, at, rot = rng.choice(((64, 64, 0, 64), (96, 96, 32, 64), (128, 128, 0, 128), (128, 128, 64, 64), (128, 64, 64, 64), (576, 512, 512, 64), (80, 80, 0, 80)))
        return {"op": op, "dtype": rng.choice(("bf16", "bf16", "f32")), "T": _log(rng, 1, 16384), "H": 1 if d == 576 else rng.choice((1, 4, 8, 16)), "d": d, "norm": norm,
                "rot_begin": at, "rot": rot, "interleaved": rng.random() < 0.5, "factor": rng.choice((1.0, 8.0, 32.0))}
    if op == "append":
        c = {"op": op, "T": _log(rng, 1, 8192), "interleaved": rng.random() < 0.5, "factor": rng.choice((1.0, 32.0)), "pool": 16384}
        if rng.random() < 0.5:
            return {**c, "Hq": 64, "Hkv": 1, "dq": 64, "dq_out": 576, "q_norm": 0, "d_k": 576, "k_norm": 512, "d_v": 0, "rot": 64}
        return {**c, "Hq": 32, "Hkv": rng.choice((4, 8)), "dq": 128, "dq_out": 128, "q_norm": 128, "d_k": 128, "k_norm": 128, "d_v": 128, "rot": rng.choice((64, 128))}
    if op == "probs":
        V = _log(rng, 1000, 131072)
        n = rng.choice((1, rng.randint(1, 64)))
        return {"op": op, "dtype": rng.choice(("bf16", "f32")), "B": _log(rng, 1, 64 if n == 1 else 14), "n": n, "V": V, "bias": rng.choice((0, 3, 200)),
                "grammar": rng.random() < 0.5, "seen": rng.choice((0, 100, V // 4))}
    if op == "count":
        return {"op": op, "B": _log(rng, 1, 16), "n": _log(rng, 1, 100000), "V": _log(rng, 1000, 131072)}
    heads = {"Hkv": 1, "d_k": 576, "d_v": 0} if rng.random() < 0.5 else {"Hkv": rng.choice((2, 4)), "d_k": 128, "d_v": 128}
    if op == "pages":
        B = _log(rng, 4, 120)
        return {"op": op, "B": B, "forks": rng.randint(0, B // 3), "ends": rng.randint(0, B // 4), "page": rng.choice((32, 64)), "max_pages": rng.choice((64, 200)),
                "layers": rng.choice((1, 2)), **heads, "sink": rng.choice((0, 100, 128)), "window": rng.choice((500, 1024, 4096, 1 << 40))}
    most = rng.choice((50, 200))
    B = _log(rng, 4, 100)
    pool = B * most + rng.randint(0, 500)
    return {"op": op, "B": B, "page": 32, "max_pages": most, "pool": pool, "used": rng.uniform(0.1, 0.9), "layers": 1, **heads}


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


def _i32(*shape):
    return torch.empty(*shape, dtype=I32, device=DEV)


def _freq(c):
    """YaRN: frequencies below one turn of the original context are divided by the factor, those above 32 turns kept, a ramp between."""
    base, s, original = 10000.0, c["factor"], 32768
    f = base ** (-np.arange(0, c["rot"], 2, dtype=np.float64) / c["rot"])
    turns = original * f / (2 * math.pi)
    keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
    m = 0.1 * math.log(s) + 1.0 if s > 1 else 1.0
    return f / s * (1 - keep) + f * keep, m


def _prepare_norm(c, s, gen, rng):
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    start = int(rng.integers(0, 1 << 20))
    s["pos"] = _dev((start + np.arange(c["T"])).astype(np.int32))
    f, s["m"] = _freq(c)
    s["freq"], s["eps"] = _dev(f), 1e-6
    # columns of different size, as projections give them
    size = torch.exp(0.5 * torch.randn(c["d"], generator=gen, device=DEV))
    s["x"] = _normal(gen, dt, c["T"], c["H"], c["d"]).mul_(size.to(dt))
    s["dout"] = _normal(gen, dt, c["T"], c["H"], c["d"])
    s["w"] = 1.0 + 0.2 * torch.randn(c["norm"], generator=gen, device=DEV)
    s["out"], s["dx"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    s["dw"] = torch.empty(c["norm"], device=DEV)


def _prepare_append(c, s, gen, rng):
    bf, T = torch.bfloat16, c["T"]
    pos = rng.integers(0, 1 << 20, size=T).astype(np.int32)
    slots = rng.permutation(c["pool"])[:T].astype(np.int32)
    dead = rng.random(T) < 0.1                      # rows behind the last token of a request
    dead[0] = False
    pos[dead] = -1
    slots[dead] = -1
    s["pos"], s["slots"] = _dev(pos), _dev(slots)
    f, s["m"] = _freq(c)
    s["freq"], s["eps"] = _dev(f), 1e-6
    s["q"], s["k"] = _normal(gen, bf, T, c["Hq"], c["dq"]), _normal(gen, bf, T, c["Hkv"], c["d_k"])
    s["wq"] = 1.0 + 0.2 * torch.randn(c["q_norm"], generator=gen, device=DEV) if c["q_norm"] else None
    s["wk"] = 1.0 + 0.2 * torch.randn(c["k_norm"], generator=gen, device=DEV)
    s["q_wide"] = _normal(gen, bf, T, c["Hq"], c["dq_out"])
    s["q_out"] = s["q_wide"][..., c["dq_out"] - c["dq"]:]
    s["k_rows"] = _normal(gen, bf, c["pool"], c["Hkv"], c["d_k"])
    s["v"] = _normal(gen, bf, T, c["Hkv"], c["d_v"]) if c["d_v"] else None
    s["v_rows"] = _normal(gen, bf, c["pool"], c["Hkv"], c["d_v"]) if c["d_v"] else None


def _words(rng, size, V):
    """Tokens as texts have them: a few of them again and again."""
    return (V * rng.random(size) ** 4).astype(np.int32)


def _prepare_probs(c, s, gen, rng):
    B, n, V = c["B"], c["n"], c["V"]
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    s["logits"] = _normal(gen, dt, B, n, V).mul_(3.0)
    tokens = _words(rng, (B, n), V)
    parents = np.full((B, n), -1)
    masks = np.zeros((B, n), dtype=np.uint64)
    nodes = rng.integers(max(1, n - n // 3), n + 1, size=B).astype(np.int32)
    for b in range(B):
        for r in range(int(nodes[b])):
            parents[b, r] = rng.integers(max(0, (r - 1) // 3 - 1), r) if r else -1
            masks[b, r] = np.uint64(1) << np.uint64(r) | (masks[b, parents[b, r]] if r else np.uint64(0))
    s["tokens"], s["masks"], s["nodes"] = _dev(tokens), _dev(masks.view(np.int64)), _dev(nodes)
    s["masks_host"], s["nodes_host"], s["tokens_host"] = masks, nodes, tokens
    row = (V + 7) // 8 * 8
    seen = np.zeros((B, row), dtype=np.int64)
    if c["seen"]:
        for b in range(B):
            p = np.bincount(_words(rng, c["seen"], V), minlength=row) > 0
            o = np.bincount(_words(rng, 1 + c["seen"] // 8, V), minlength=row)
            seen[b] = p * 32768 + np.minimum(o, 32767)
    s["seen"] = _dev(seen.astype(np.uint16).view(np.int16)) if c["seen"] else None
    f32 = dict(device=DEV, dtype=torch.float32)
    s["rep"] = torch.tensor([(1.0, 1.1, 1.3)[b % 3] for b in range(B)], **f32)
    s["fre"] = torch.tensor([(0.0, 0.25)[b % 2] for b in range(B)], **f32)
    s["pre"] = torch.tensor([(0.5, 0.0)[b % 2] for b in range(B)], **f32)
    s["temp"] = torch.tensor([(0.7, 1.0, 0.0, 0.6)[b % 4] for b in range(B)], **f32)
    s["bt"] = s["bv"] = None
    if c["bias"]:
        s["bt"] = _dev(rng.integers(0, V, size=(B, c["bias"])).astype(np.int32))
        s["bv"] = _dev(rng.normal(0, 4, size=(B, c["bias"])).astype(np.float32))
    s["allowed"] = None
    if c["grammar"]:
        # requests without a grammar allow all, the others a tenth of the words of 32 tokens, with most of their tokens
        words = (V + 31) // 32
        a = rng.integers(-(1 << 31), 1 << 31, size=(B, n, words)).astype(np.int32) | rng.integers(-(1 << 31), 1 << 31, size=(B, n, words)).astype(np.int32)
        a[rng.random((B, n, words)) > 0.1] = 0
        a[..., 0] |= 1
        a[1::2] = -1
        s["allowed"] = _dev(a)
    s["probs"] = torch.zeros(B, n, V, **f32)


def _prepare_count(c, s, gen, rng):
    B, n, V = c["B"], c["n"], c["V"]
    tokens = _words(rng, (B, n), V)
    lens = rng.integers(max(1, n - n // 4), n + 1, size=B).astype(np.int32)
    prompt = (lens * rng.uniform(0.5, 1.0, size=B)).astype(np.int32)
    s["tokens"], s["lens"], s["prompt"] = _dev(tokens), _dev(lens), _dev(prompt)
    s["tokens_host"], s["lens_host"], s["prompt_host"] = tokens, lens, prompt
    s["fresh"] = torch.ones(B, dtype=I32, device=DEV)
    s["seen"] = torch.full((B, (V + 7) // 8 * 8), 77, dtype=torch.int16, device=DEV)


def _pool(c, s, gen, pages):
    bf = torch.bfloat16
    s["k_pages"] = _normal(gen, bf, c["layers"], pages, c["page"], c["Hkv"], c["d_k"])
    s["v_pages"] = _normal(gen, bf, c["layers"], pages, c["page"], c["Hkv"], c["d_v"]) if c["d_v"] else None


def _prepare_pages(c, s, gen, rng):
    B, page, most = c["B"], c["page"], c["max_pages"]
    empty = rng.permutation(B)[: c["forks"]]                # places for the forks
    lens = rng.integers(1, most * page + 1, size=B).astype(np.int32)
    lens[rng.random(B) < 0.2] //= page
    lens[empty] = 0
    live = np.setdiff1d(np.arange(B), empty)
    source = np.full(B, -1, dtype=np.int32)
    some = rng.choice(live, size=max(1, min(len(live), c["forks"] // 4 + 1)), replace=False)
    source[empty] = rng.choice(some, size=len(empty))
    spare = rng.integers(0, 2, size=B)
    pages = (B - c["forks"]) * most * 3 // 5 + c["forks"] + 3
    while True:
        held = np.where(lens > 0, np.minimum(most, -(-lens // page) + spare), 0).astype(np.int32)
        if int(held.sum()) + c["forks"] <= pages:
            break
        lens = np.where(lens > 0, lens * 9 // 10 + 1, 0).astype(np.int32)
    perm = rng.permutation(pages).astype(np.int32)
    table = np.full((B, most), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, : held[b]] = perm[at: at + held[b]]
        at += int(held[b])
    free = np.full(pages, -1, dtype=np.int32)
    free[: pages - at] = perm[at:]
    ending = np.zeros(B, dtype=np.int32)
    ending[rng.choice(live, size=min(len(live), c["ends"]), replace=False)] = 1
    s["host"] = {"source": source, "lens": lens, "held": held, "table": table.copy(), "free": free.copy(), "count": pages - at, "pages": pages, "ending": ending}
    s["source"], s["lens"], s["held"], s["table"], s["free"], s["ending"] = (_dev(x) for x in (source, lens, held, table, free, ending))
    s["count"] = torch.tensor([pages - at], dtype=I32, device=DEV)
    s["free2"] = s["free"].clone()                          # what is given back is put here, so that a pass can be repeated
    s["shared"], s["trimmed"] = torch.zeros(pages, dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV)
    for k in ("forked", "lens1", "held1", "trimmed1", "copy_from", "copy_to", "copy_rows", "lens2", "held2", "trimmed2"):
        s[k] = _i32(B)
    s["left"], s["count2"], s["shared1"], s["shared2"] = _i32(1), _i32(1), _i32(pages), _i32(pages)
    _pool(c, s, gen, pages)


def _prepare_compact(c, s, gen, rng):
    B, most, pool = c["B"], c["max_pages"], c["pool"]
    used = max(1, min(B * most, int(c["used"] * pool)))
    held = rng.multinomial(used, np.ones(B) / B)
    spill = int(np.maximum(held - most, 0).sum())
    held = np.minimum(held, most)
    used -= spill
    perm = rng.permutation(pool).astype(np.int32)
    table = np.full((B, most), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, : held[b]] = perm[at: at + held[b]]
        at += int(held[b])
    shared = np.zeros(pool, dtype=np.int32)
    if held[0] and held[1] < most:                          # a page that two requests share
        table[1, held[1]] = table[0, 0]
        shared[table[0, 0]] = 1
    free = np.full(pool, -1, dtype=np.int32)
    free[: pool - at] = perm[at:]
    s["host"] = {"table": table, "free": free, "count": pool - at, "shared": shared}
    s["table"], s["free"], s["shared"] = _dev(table), _dev(free), _dev(shared)
    s["count"] = torch.tensor([pool - at], dtype=I32, device=DEV)
    s["table2"], s["free2"], s["shared2"], s["count2"], s["copies"] = _i32(B, most), _i32(pool), _i32(pool), _i32(1), _i32(1)
    s["copy_from"], s["copy_to"] = _i32(pool // 2), _i32(pool // 2)
    _pool(c, s, gen, pool)


def prepare(case, seed):
    s = {"case": case}
    gen, rng = torch.Generator(device=DEV).manual_seed(seed), np.random.default_rng(seed)
    globals()["_prepare_" + case["op"]](case, s, gen, rng)
    if own:
        import paper_2512_23966_amd as loza
        c = case
        nbytes = {"norm": lambda: loza.loza_ssa_norm_rope_backward_workspace_bytes(c["T"], c["H"], c["d"], c["norm"]),
                  "probs": lambda: loza.loza_ssa_token_probs_workspace_bytes(c["B"], c["n"], c["V"]),
                  "pages": lambda: loza.loza_ssa_pages_free_workspace_bytes(s["shared"].numel()),
                  "compact": lambda: loza.loza_ssa_pages_compact_workspace_bytes(c["pool"])}.get(c["op"])
        s["ws"] = torch.empty(nbytes(), dtype=torch.uint8, device=DEV) if nbytes else None
    return s


# ---- one pass ------------------------------------------------------------------------------------------

def run(s):
    return globals()[("_own_" if own else "_plain_") + s["case"]["op"]](s["case"], s)


def _own_norm(c, s):
    import paper_2512_23966_amd as loza
    f32 = c["dtype"] == "f32"
    forward = loza.loza_ssa_norm_rope_f32 if f32 else loza.loza_ssa_norm_rope
    backward = loza.loza_ssa_norm_rope_backward_f32 if f32 else loza.loza_ssa_norm_rope_backward
    forward(s["x"], s["w"], s["pos"], s["freq"], s["out"], 0, c["norm"], s["eps"], c["rot_begin"], c["interleaved"], s["m"])
    backward(s["dout"], s["x"], s["w"], s["pos"], s["freq"], s["dx"], s["dw"], 0, c["norm"], s["eps"], c["rot_begin"], c["interleaved"], s["m"], workspace=s["ws"])
    return [s["out"], s["dx"], s["dw"]]


def _own_append(c, s):
    import paper_2512_23966_amd as loza
    loza.loza_ssa_norm_rope_append(s["q"], s["wq"], s["k"], s["wk"], s["v"], s["pos"], s["slots"], s["freq"], s["q_out"], s["k_rows"], s["v_rows"], 0, c["q_norm"],
                                   0, c["k_norm"], s["eps"], c["dq"] - c["rot"], c["d_k"] - c["rot"], c["interleaved"], s["m"])
    return [s["q_wide"], s["k_rows"]] + ([s["v_rows"]] if c["d_v"] else [])


def _own_probs(c, s):
    import paper_2512_23966_amd as loza
    fn = loza.loza_ssa_token_probs_f32 if c["dtype"] == "f32" else loza.loza_ssa_token_probs
    fn(s["logits"], s["probs"], s["ws"], tree_lens=s["nodes"], tokens=s["tokens"], masks=s["masks"], seen=s["seen"], repetition=s["rep"], frequency=s["fre"],
       presence=s["pre"], temperature=s["temp"], bias_tokens=s["bt"], bias_values=s["bv"], allowed=s["allowed"])
    return s["probs"]


def _own_count(c, s):
    import paper_2512_23966_amd as loza
    loza.loza_ssa_count_tokens(s["tokens"], s["lens"], s["seen"], c["V"], prompt_lens=s["prompt"], fresh=s["fresh"])
    return s["seen"]


def _own_pages(c, s):
    import paper_2512_23966_amd as loza
    pages = s["shared"].numel()
    loza.loza_ssa_pages_fork(s["source"], s["lens"], s["held"], s["trimmed"], s["free"], s["count"], s["shared"], s["table"], pages, c["page"], c["sink"], 1, s["forked"],
                             s["lens1"], s["held1"], s["trimmed1"], s["copy_from"], s["copy_to"], s["copy_rows"], s["left"], s["shared1"])
    loza.loza_ssa_pages_copy(s["k_pages"], s["v_pages"], s["copy_from"], s["copy_to"], rows=s["copy_rows"])
    loza.loza_ssa_pages_free(s["ending"], s["lens1"], s["held1"], s["trimmed1"], s["table"], s["shared1"], s["free2"], s["left"], pages, c["page"], c["sink"], c["window"], 1,
                             s["lens2"], s["held2"], s["trimmed2"], s["count2"], s["shared2"], s["ws"])
    return _pages_outputs(s)


def _pages_outputs(s):
    # (what lies behind the valid entries of the free list is nobody's)
    keep = torch.arange(s["free2"].numel(), device=DEV) < s["count2"]
    names = ("forked", "copy_from", "copy_to", "copy_rows", "left", "lens2", "held2", "trimmed2", "count2", "shared2", "table", "k_pages", "v_pages")
    return [torch.where(keep, s["free2"], -1)] + [s[k] for k in names if s[k] is not None]


def _own_compact(c, s):
    import paper_2512_23966_amd as loza
    loza.loza_ssa_pages_compact(s["table"], s["free"], s["count"], s["shared"], c["pool"], s["table2"], s["free2"], s["count2"], s["shared2"], s["copy_from"],
                                s["copy_to"], s["copies"], s["ws"])
    loza.loza_ssa_pages_copy(s["k_pages"], s["v_pages"], s["copy_from"], s["copy_to"], count=s["copies"])
    return [s[k] for k in ("table2", "free2", "count2", "shared2", "copy_from", "copy_to", "copies", "k_pages", "v_pages") if s[k] is not None]


# ---- plain forms -----------------------------------------------------------------------------------------

def _turn(pos, freq, m):
    """m cos, m sin of the tokens' angles [T, 1, rot / 2] (the angles in 64 bits)."""
    ang = pos.double()[:, None] * freq[None, :]
    return ((f(ang) * m).float()[:, None, :] for f in (torch.cos, torch.sin))


def _rotate(y, co, si, begin, interleaved):
    """y [T, H, d] fp32 with its rotary columns rotated."""
    rot = 2 * co.shape[-1]
    r = y[..., begin:begin + rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., : rot // 2], r[..., rot // 2:])
    u, w = a * co - b * si, a * si + b * co
    z = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([y[..., :begin], z, y[..., begin + rot:]], -1)


def _normed(x, w, norm, eps):
    """x fp32 with its first `norm` columns normed, and 1 / their root mean square."""
    r = torch.rsqrt(x[..., :norm].square().mean(-1, keepdim=True) + eps)
    return torch.cat([x[..., :norm] * r * w, x[..., norm:]], -1), r


def _plain_norm(c, s):
    n, x = c["norm"], s["x"].float()
    co, si = _turn(s["pos"], s["freq"], s["m"])
    y, r = _normed(x, s["w"], n, s["eps"])
    s["out"].copy_(_rotate(y, co, si, c["rot_begin"], c["interleaved"]))
    g = _rotate(s["dout"].float(), co, -si, c["rot_begin"], c["interleaved"])
    xn, gn = x[..., :n], g[..., :n]
    h = gn * s["w"]
    dn = r * (h - xn * r.square() * (h * xn).mean(-1, keepdim=True))
    s["dx"].copy_(torch.cat([dn, g[..., n:]], -1))
    s["dw"].copy_((gn * xn * r).sum((0, 1)))
    return [s["out"], s["dx"], s["dw"]]


def _plain_append(c, s):
    live = s["pos"] >= 0
    co, si = _turn(s["pos"], s["freq"], s["m"])
    q = s["q"].float()
    if c["q_norm"]:
        q = _normed(q, s["wq"], c["q_norm"], s["eps"])[0]
    q = _rotate(q, co, si, c["dq"] - c["rot"], c["interleaved"]).to(s["q"].dtype)
    s["q_out"].copy_(torch.where(live[:, None, None], q, s["q_out"]))
    k = _rotate(_normed(s["k"].float(), s["wk"], c["k_norm"], s["eps"])[0], co, si, c["d_k"] - c["rot"], c["interleaved"]).to(s["k"].dtype)
    put = live & (s["slots"] >= 0)
    at = s["slots"][put].long()
    s["k_rows"][at] = k[put]
    if c["d_v"]:
        s["v_rows"][at] = s["v"][put]
    return [s["q_wide"], s["k_rows"]] + ([s["v_rows"]] if c["d_v"] else [])


def _plain_probs(c, s):
    B, n, V = c["B"], c["n"], c["V"]
    node = torch.arange(n, device=DEV)
    for b in range(B):
        on = ((s["masks"][b][:, None] >> node) & 1).bool() & (node < s["nodes"][b])             # [n, n] nodes before each
        x = s["logits"][b].float()
        count = torch.zeros(n, V, device=DEV)
        was = torch.zeros(n, V, dtype=torch.bool, device=DEV)
        if s["seen"] is not None:
            z = s["seen"][b, :V]
            count += (z & 32767).float()
            was |= z < 0
        count.scatter_add_(1, s["tokens"][b].long()[None, :].expand(n, n), on.float())
        there = count > 0
        x = torch.where(was | there, torch.where(x > 0, x / s["rep"][b], x * s["rep"][b]), x)
        x = x - s["fre"][b] * count
        x = x - s["pre"][b] * there.float()
        if s["bt"] is not None:
            x = x + torch.zeros(V, device=DEV).scatter_add_(0, s["bt"][b].long(), s["bv"][b])
        if s["allowed"] is not None:
            ok = ((s["allowed"][b][:, :, None] >> torch.arange(32, device=DEV, dtype=I32)) & 1).bool().flatten(1)[:, :V]
            x = x.masked_fill(~ok, -math.inf)
        x = x.masked_fill(torch.isnan(x), -math.inf)
        top = x.amax(-1, keepdim=True)
        t = s["temp"][b]
        e = torch.where(x == top, 1.0, ((x - top) / t).exp())
        soft = e / e.sum(-1, keepdim=True)
        hard = ((x == top).int().cumsum(-1) == 1) & (x == top)
        p = torch.where(t > 0, soft, hard.float())
        p = torch.where(top == -math.inf, 0.0, p)
        s["probs"][b] = torch.where((node < s["nodes"][b])[:, None], p, s["probs"][b])
    return s["probs"]


def _plain_count(c, s):
    B, n, V = c["B"], c["n"], c["V"]
    row = s["seen"].shape[1]
    i = torch.arange(n, device=DEV)[None, :]
    there, prompt = i < s["lens"][:, None], i < s["prompt"][:, None]
    at = s["tokens"].long()
    p = torch.zeros(B, row, dtype=I32, device=DEV).scatter_add_(1, at, (there & prompt).int())
    o = torch.zeros(B, row, dtype=I32, device=DEV).scatter_add_(1, at, (there & ~prompt).int())
    s["seen"].copy_(torch.where(p > 0, -32768, 0) + o.clamp(max=32767))
    return s["seen"]


def _first_page(c, lens, trimmed):
    """First page behind the sink that a query at position `lens` or later sees, and the number of sink pages."""
    sink = -(-c["sink"] // c["page"])
    begin = (lens.long() - c["window"] + 1).clamp(min=0) // c["page"]
    return torch.maximum(begin, trimmed.long()).clamp(min=sink), sink


def _plain_pages(c, s):
    B, page, most, pages = c["B"], c["page"], c["max_pages"], s["shared"].numel()
    col = torch.arange(most, device=DEV)[None, :]
    sink = -(-c["sink"] // page)
    # forks
    src = s["source"].long()
    lens, held = s["lens"].long(), s["held"].long()
    at = src.clamp(0, B - 1)
    fits = (src >= 0) & (src < B) & (lens == 0) & (held == 0)
    L = torch.where(fits, lens[at], 0)
    need = (fits & (L % page != 0)).long()
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= s["count"]))
    full, have = L // page, (L + page - 1) // page
    rows = s["table"][at]
    new = s["free"][(s["count"].long() - upto).clamp(0, pages - 1)]
    first = torch.where(ok, s["trimmed"][at].long(), 0)
    mine = ok[:, None] & (col < full[:, None]) & ((col < sink) | (col >= first[:, None])) & (rows >= 0) & (rows < pages)
    shared1 = s["shared"].clone()
    shared1.index_add_(0, rows[mine].long(), torch.ones(int(mine.sum()), dtype=I32, device=DEV))
    last = torch.gather(rows, 1, full.clamp(max=most - 1)[:, None])[:, 0]
    started = ok & (need > 0)
    s["copy_from"].copy_(torch.where(started, last, -1))
    s["copy_to"].copy_(torch.where(started, new, -1))
    s["copy_rows"].copy_(torch.where(started, L % page, 0))
    s["forked"].copy_(ok)
    s["left"].copy_((s["count"] - (upto * started).amax()).to(I32))
    table = torch.where(ok[:, None] & (col < full[:, None]), rows, s["table"])
    s["table"].copy_(torch.where(started[:, None] & (col == full[:, None]), new[:, None], table))
    lens1, held1, trimmed1 = torch.where(ok, L, lens), torch.where(ok, have, held), torch.where(ok, first, s["trimmed"].long())
    # started pages
    f, t, r = s["copy_from"][started].long(), s["copy_to"][started].long(), s["copy_rows"][started]
    row = torch.arange(page, device=DEV)[None, :, None, None]
    for x in (s["k_pages"], s["v_pages"]):
        if x is not None:
            for layer in x:
                layer[t] = torch.where(row < r[:, None, None, None], layer[f], layer[t])
    # pages given back
    end = s["ending"] != 0
    now = torch.maximum(held1, (lens1 + page - 1) // page)
    upto1, _ = _first_page(c, lens1, trimmed1)
    begin = trimmed1.clamp(min=sink)
    gone = torch.where(end[:, None], (col < now[:, None]) & ((col < sink) | (col >= begin[:, None])), (col >= begin[:, None]) & (col < torch.minimum(upto1, now)[:, None]))
    gone &= (s["table"] >= 0) & (s["table"] < pages)
    times = torch.zeros(pages, dtype=I32, device=DEV)
    times.index_add_(0, s["table"][gone].long(), torch.ones(int(gone.sum()), dtype=I32, device=DEV))
    back = times > shared1
    s["shared2"].copy_((shared1 - times).clamp(min=0))
    ids = back.nonzero()[:, 0].to(I32)
    k = int(s["left"])
    s["free2"][k:k + ids.numel()] = ids
    s["count2"].copy_(s["left"] + ids.numel())
    s["lens2"].copy_(torch.where(end, 0, lens1))
    s["held2"].copy_(torch.where(end, 0, held1))
    s["trimmed2"].copy_(torch.where(end, 0, torch.maximum(trimmed1, torch.where(upto1 > sink, upto1, 0))))
    return _pages_outputs(s)


def _plain_compact(c, s):
    pool = c["pool"]
    page = torch.arange(pool, device=DEV, dtype=I32)
    is_free = torch.zeros(pool, dtype=torch.bool, device=DEV)
    is_free[s["free"][: int(s["count"])].long()] = True
    frees = int(is_free.sum())
    used = pool - frees
    holes, movers = page[is_free & (page < used)], page[~is_free & (page >= used)]
    k = holes.numel()
    for t, x in ((s["copy_to"], holes), (s["copy_from"], movers)):
        t.fill_(-1)
        t[:k] = x
    s["copies"].fill_(k)
    to = page.clone()
    to[movers.long()] = holes
    t = s["table"]
    s["table2"].copy_(torch.where((t >= 0) & (t < pool), to[t.clamp(0, pool - 1).long()], t))
    s["shared2"].copy_(torch.where(page < used, s["shared"], 0))
    s["shared2"][holes.long()] = s["shared"][movers.long()]
    s["free2"].copy_(torch.where(page < frees, pool - 1 - page, -1))
    s["count2"].fill_(frees)
    for x in (s["k_pages"], s["v_pages"]):
        if x is not None:
            for layer in x:
                layer[holes.long()] = layer[movers.long()]
    return [s[k] for k in ("table2", "free2", "count2", "shared2", "copy_from", "copy_to", "copies", "k_pages", "v_pages") if s[k] is not None]


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "norm":
        es, elems = 4 if c["dtype"] == "f32" else 2, c["T"] * c["H"] * c["d"]
        return {"bytes": 4 * elems * es, "flops": c["T"] * c["H"] * (6 * c["rot"] + 14 * c["norm"])}
    if c["op"] == "append":
        row = c["Hq"] * c["dq"] + c["Hkv"] * (c["d_k"] + c["d_v"])
        return {"bytes": 2 * 2 * c["T"] * row, "flops": c["T"] * (3 * (c["Hq"] + c["Hkv"]) * c["rot"] + 4 * (c["Hq"] * c["q_norm"] + c["Hkv"] * c["k_norm"]))}
    if c["op"] == "probs":
        nodes = c["B"] * (max(1, c["n"] - c["n"] // 3) + c["n"]) / 2
        token = (4 if c["dtype"] == "f32" else 2) + 4 + (0.125 if c["grammar"] else 0)
        return {"bytes": nodes * c["V"] * token + (2 * c["B"] * c["V"] if c["seen"] else 0), "flops": 4 * nodes * c["V"]}
    if c["op"] == "count":
        return {"bytes": c["B"] * (c["n"] * 3.5 + 2 * c["V"]), "flops": 0}
    row = 2 * c["Hkv"] * (c["d_k"] + c["d_v"])
    if c["op"] == "pages":
        return {"bytes": c["forks"] * c["layers"] * c["page"] * row + 4 * c["B"] * (c["max_pages"] / 2 + 12) + 8 * c["B"] * c["max_pages"] / 2, "flops": 0}
    used = min(c["used"] * c["pool"], c["B"] * c["max_pages"])
    moves = used * (1 - used / c["pool"])
    return {"bytes": 2 * moves * c["layers"] * c["page"] * row + 8 * c["B"] * c["max_pages"] + 16 * c["pool"], "flops": 0}


# ---- the same from the definitions, in 64 bits --------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return globals()["_exact_" + case["op"]](case, s)


def _exact_heads(c, x, w, norm, pos, freq, m, eps, begin):
    """Complex numbers in the place of pairs: x [T, H, d] (64 bits), normed and rotated."""
    y = x
    if norm:
        rms = (x[..., :norm] ** 2).sum(-1) / norm + eps
        y = torch.cat((x[..., :norm] / rms.sqrt()[..., None] * w.to(F64), x[..., norm:]), -1)
    k = freq.numel()
    first = begin + (2 * torch.arange(k, device=DEV) if c["interleaved"] else torch.arange(k, device=DEV))
    second = first + (1 if c["interleaved"] else k)
    ang = pos.to(F64)[:, None] * freq
    z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.full_like(ang, m), ang)[:, None, :]
    return y.index_copy(2, first, z.real).index_copy(2, second, z.imag)


def _exact_norm(c, s):
    outs, dxs, dw = [], [], torch.zeros(c["norm"], dtype=F64, device=DEV)
    for a in range(0, c["T"], 4096):
        part = slice(a, a + 4096)
        x = s["x"][part].to(F64).requires_grad_()
        w = s["w"].to(F64).requires_grad_()
        y = _exact_heads(c, x, w, c["norm"], s["pos"][part], s["freq"], s["m"], s["eps"], c["rot_begin"])
        dx, dwp = torch.autograd.grad(y, (x, w), s["dout"][part].to(F64))
        outs.append(y.detach())
        dxs.append(dx)
        dw += dwp
    return [torch.cat(outs), torch.cat(dxs), dw]


def _exact_append(c, s):
    live = (s["pos"] >= 0).nonzero()[:, 0]
    pos = s["pos"][live]
    q_wide, k_rows = s["q_wide"].to(F64), s["k_rows"].to(F64)
    q = _exact_heads(c, s["q"][live].to(F64), s["wq"], c["q_norm"], pos, s["freq"], s["m"], s["eps"], c["dq"] - c["rot"])
    q_wide[live, :, c["dq_out"] - c["dq"]:] = q
    k_rows[s["slots"][live].long()] = _exact_heads(c, s["k"][live].to(F64), s["wk"], c["k_norm"], pos, s["freq"], s["m"], s["eps"], c["d_k"] - c["rot"])
    if not c["d_v"]:
        return [q_wide, k_rows]
    v_rows = s["v_rows"].to(F64)
    v_rows[s["slots"][live].long()] = s["v"][live].to(F64)
    return [q_wide, k_rows, v_rows]


def _exact_probs(c, s):
    B, n, V = c["B"], c["n"], c["V"]
    out = s["probs"].to(F64)
    rep, fre, pre, temp = (s[k].cpu().numpy().astype(np.float64) for k in ("rep", "fre", "pre", "temp"))
    for b in range(B):
        seen = np.zeros(V, dtype=np.int64) if s["seen"] is None else s["seen"][b, :V].cpu().numpy().view(np.uint16).astype(np.int64)
        bias = np.zeros(V)
        if s["bt"] is not None:
            np.add.at(bias, s["bt"][b].cpu().numpy(), s["bv"][b].cpu().numpy().astype(np.float64))
        bias = _dev(bias)
        for r in range(int(s["nodes_host"][b])):
            count = seen % 32768
            for a in range(n):
                if int(s["masks_host"][b, r]) >> a & 1:
                    count[s["tokens_host"][b, a]] += 1
            hit, count = _dev((count > 0) | (seen >= 32768)), _dev(count)
            x = s["logits"][b, r].to(F64)
            x = torch.where(hit, x * torch.where(x > 0, 1.0 / rep[b], rep[b]), x) - fre[b] * count - pre[b] * (count > 0) + bias
            if s["allowed"] is not None:
                bits = np.unpackbits(s["allowed"][b, r].cpu().numpy().view(np.uint8), bitorder="little")[:V]
                x[_dev(bits == 0)] = -math.inf
            if not bool((x > -math.inf).any()):
                out[b, r] = 0.0
            elif temp[b] > 0:
                out[b, r] = torch.softmax(x / temp[b], -1)
            else:
                out[b, r] = 0.0
                out[b, r, (x == x.max()).nonzero()[0]] = 1.0
    return out


def _exact_count(c, s):
    out = np.zeros(tuple(s["seen"].shape), dtype=np.int64)
    for b in range(c["B"]):
        L, P = int(s["lens_host"][b]), int(s["prompt_host"][b])
        said = np.bincount(s["tokens_host"][b, P:L], minlength=out.shape[1])
        out[b] = np.minimum(said, 32767)
        out[b, np.unique(s["tokens_host"][b, :P])] -= 32768
    return _dev(out.astype(np.int16))


def _exact_pages(c, s):
    h = s["host"]
    B, page, most = c["B"], c["page"], c["max_pages"]
    lens, held, table, free = h["lens"].tolist(), h["held"].tolist(), h["table"].copy(), h["free"].tolist()
    holders = np.zeros(h["pages"], dtype=np.int64)
    for b in range(B):
        holders[table[b, : held[b]]] += 1
    list_end = h["count"]
    forked, cf, ct, cr = (np.full(B, x, dtype=np.int32) for x in (0, -1, -1, 0))
    for b in range(B):
        f = int(h["source"][b])
        if f < 0 or h["held"][b]:
            continue
        whole, rest = divmod(int(h["lens"][f]), page)
        if rest and not list_end:
            continue
        forked[b], lens[b], held[b] = 1, int(h["lens"][f]), whole + (rest > 0)
        table[b, :whole] = h["table"][f, :whole]
        holders[table[b, :whole]] += 1
        if rest:
            list_end -= 1
            table[b, whole] = ct[b] = free[list_end]
            cf[b], cr[b] = h["table"][f, whole], rest
            holders[ct[b]] += 1
    pools = [x if x is None else x.clone() for x in (s["k_pages"], s["v_pages"])]
    for b in np.nonzero(cf >= 0)[0]:
        for new, old in zip(pools, (s["k_pages"], s["v_pages"])):
            if new is not None:
                new[:, int(ct[b]), : int(cr[b])] = old[:, int(cf[b]), : int(cr[b])]
    left, trimmed, back = list_end, [0] * B, set()
    sink = -(-c["sink"] // page)
    for b in range(B):
        if h["ending"][b]:
            out, lens[b], held[b] = range(held[b]), 0, 0
        else:
            first = max(0, lens[b] - c["window"] + 1) // page
            out = range(sink, first)
            trimmed[b] = first if first > sink else 0
        for i in out:
            holders[table[b, i]] -= 1
            if holders[table[b, i]] == 0:
                back.add(int(table[b, i]))
    free = free[:left] + sorted(back)
    count2 = len(free)
    free += [-1] * (h["pages"] - count2)
    one = lambda x: _dev(np.array(x, dtype=np.int32))
    return [one(free), one(forked), one(cf), one(ct), one(cr), one([left]), one(lens), one(held), one(trimmed), one([count2]), one(np.maximum(holders - 1, 0)), one(table)] + \
        [x for x in pools if x is not None]


def _exact_compact(c, s):
    h, pool = s["host"], c["pool"]
    free = set(int(x) for x in h["free"][: h["count"]])
    used = pool - len(free)
    move = dict(zip((p for p in range(used, pool) if p not in free), (p for p in range(used) if p in free)))
    table = np.array([[move.get(int(p), int(p)) for p in row] for row in h["table"]], dtype=np.int32)
    shared = np.zeros(pool, dtype=np.int32)
    for p in range(pool):
        if p not in free:
            shared[move.get(p, p)] = h["shared"][p]
    pad = lambda x, k: _dev(np.array(list(x) + [-1] * (k - len(list(x))), dtype=np.int32))
    pools = []
    for x in (s["k_pages"], s["v_pages"]):
        if x is not None:
            y = x.clone()
            y[:, list(move.values())] = x[:, list(move.keys())]
            pools.append(y)
    return [_dev(table), pad(range(pool - 1, used - 1, -1), pool), pad([len(free)], 1), _dev(shared), pad(list(move.keys()), pool // 2), pad(list(move.values()), pool // 2),
            pad([len(move)], 1)] + pools
