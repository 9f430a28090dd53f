"""Speculative decoding and shared blocks on a paged KV cache, as measured: attention of several drafted tokens per request
(a tree or a chain of them) through device tables, the accepted rows moved to their places, requests forked from others with
their blocks shared and freed again, and blocks moved out of ids that are taken away. Plain forms in elementary torch
operations beside the framework's calls.

Cache format (as in the rest of the framework): a block is a K plane [T][Hkv][D] and a V plane of the same shape, 16-bit
elements; inside token row r, within every aligned 64 elements, the unit of 8 elements u is stored at unit u ^ (r & 7). A table
entry e >= 0 names block e of the first arena, e < 0 block ~e of the second one.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # verification of a short chain of drafted tokens for one request: latency alone
        dict(name="tree_1x8", op="tree", n=1, lo=500, hi=500, m_lo=8, m_hi=8, T=16, Hkv=8, G=4, D=128, dtype="bf16", lent=0.25, shape="chain",
             window=0),
        # a running batch, each request with a tree of 24 drafted tokens
        dict(name="tree_64x24", op="tree", n=64, lo=512, hi=4095, m_lo=24, m_hi=24, T=16, Hkv=8, G=4, D=128, dtype="bf16", lent=0.4, shape="tree",
             window=0),
        # few very long requests with large trees of different sizes
        dict(name="tree_5x61", op="tree", n=5, lo=60000, hi=100001, m_lo=29, m_hi=61, T=32, Hkv=8, G=8, D=128, dtype="fp16", lent=0.0, shape="tree",
             window=0),
        # a ragged batch with empty requests, heads without sharing, trees that look back 1000 tokens
        dict(name="tree_window_200", op="tree", n=200, lo=0, hi=5000, m_lo=0, m_hi=9, T=64, Hkv=12, G=1, D=64, dtype="bf16", lent=0.0, shape="tree",
             window=1000),
        # pieces of prompts behind what the cache holds: arithmetic counts
        dict(name="chain_8x2001", op="tree", n=8, lo=0, hi=7000, m_lo=900, m_hi=2001, T=16, Hkv=8, G=4, D=128, dtype="bf16", lent=0.3, shape="chain",
             window=0),
        # the accepted rows of a batch's trees, all layers at once
        dict(name="keep_64x24", op="keep", n=64, lo=100, hi=1000, m=24, most=7, L=8, T=16, Hkv=8, D=128, dtype="bf16", lent=0.4),
        # many short requests, large trees, small heads
        dict(name="keep_700x61", op="keep", n=700, lo=0, hi=300, m=61, most=20, L=2, T=32, Hkv=4, D=64, dtype="fp16", lent=0.0),
        # four samples of one prompt, given up and drawn again: latency
        dict(name="fork_1x4", op="fork", n=1, kids=4, lo=700, hi=700, L=2, T=16, Hkv=8, D=128, dtype="bf16", lent=0.25),
        # a step of beam search: 40 prompts, eight beams each
        dict(name="fork_40x8", op="fork", n=40, kids=8, lo=200, hi=2999, L=8, T=16, Hkv=2, D=128, dtype="bf16", lent=0.4),
        # many short prompts, two samples each, large blocks
        dict(name="fork_500x2", op="fork", n=500, kids=2, lo=0, hi=600, L=4, T=64, Hkv=4, D=64, dtype="fp16", lent=0.0),
        # the lender takes all of its memory back under a running batch
        dict(name="compact_lent_64", op="compact", n=64, lo=512, hi=4095, kids=0, L=2, T=16, Hkv=8, D=128, dtype="bf16", lent=0.4, keep0=1.0, keep1=0.0),
        # the blocks that short requests and their samples hold, moved to the front of both arenas
        dict(name="compact_front_300", op="compact", n=300, lo=1, hi=500, kids=2, L=4, T=32, Hkv=4, D=64, dtype="fp16", lent=0.3, keep0=0.6, keep1=0.6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "tree", "keep", "fork", "compact"])
    T, D, dtype = rng.choice([16, 32, 64]), rng.choice([64, 128, 256]), rng.choice(["bf16", "fp16"])
    lent = rng.choice([0.0, rng.uniform(0.1, 0.9)])
    if op == "tree":
        Hkv, G = rng.randint(1, 12), rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
        shape = rng.choice(["tree", "chain"])
        n = _log(rng, 1, 160)
        most = 6.0e10 / (n * Hkv * G * D)                           # drafted tokens x context of a request: products that keep a pass below the largest listed ones
        m_hi = _log(rng, 1, max(2, min(200 if shape == "tree" else 2000, math.sqrt(most))))
        hi = _log(rng, 10, max(20, min(60000, most / m_hi, 2.0e8 / (n * Hkv * D))))
        return dict(op=op, n=n, lo=rng.choice([0, 1, hi // 3]), hi=hi, m_lo=rng.choice([0, 1, m_hi // 2, m_hi]), m_hi=m_hi, T=T, Hkv=Hkv, G=G, D=D,
                    dtype=dtype, lent=lent, shape=shape, window=rng.choice([0, 0, rng.randint(1, hi + m_hi)]))
    Hkv, L = rng.randint(1, 8), rng.randint(1, 8)
    room = 4.0e8 / (L * Hkv * D)                                   # tokens that all layers' arenas have room for
    n = _log(rng, 1, 800)
    if op == "keep":
        m = _log(rng, 2, 100)
        hi = _log(rng, 5, max(10, min(4000, room / n - m)))
        return dict(op=op, n=n, lo=rng.choice([0, hi // 2]), hi=hi, m=m, most=rng.randint(2, min(m, 20)), L=L, T=T, Hkv=Hkv, D=D, dtype=dtype, lent=lent)
    kids = rng.randint(1, 8) if op == "fork" else rng.randint(0, 3)
    hi = _log(rng, 10, max(20, min(6000, room / (2 * n) - T * kids)))
    case = dict(op=op, n=n, lo=rng.choice([0, 1, hi // 2]), hi=hi, kids=kids, L=L, T=T, Hkv=Hkv, D=D, dtype=dtype, lent=lent)
    if op == "compact":
        case["keep0"], case["keep1"] = rng.choice([(1.0, 0.0), (1.0, rng.uniform(0.1, 0.9)), (0.6, 0.6)])
    return case


def _spread(n, lo, hi):
    """n whole numbers spread evenly over lo..hi: the same for every seed, so that work() knows them."""
    if n == 1:
        return np.array([hi], np.int64)
    return np.floor(lo + (hi - lo) * np.arange(n) / (n - 1) + 0.5).astype(np.int64)


def _drafts(case):
    """Context and drafted tokens of the requests, paired the same for every seed (which orders the pairs)."""
    return _spread(case["n"], case["lo"], case["hi"]), np.random.default_rng(case["n"]).permutation(_spread(case["n"], case["m_lo"], case["m_hi"]))


def _kept(case):
    return np.random.default_rng(case["n"]).permutation(_spread(case["n"], 0 if case["n"] > 1 else 1, case["most"]))


def _limits(case, held, sizes):
    """Ids of each arena that stay, given the blocks held in it and its size: all of it, none, or a share, made to fit."""
    a, b = case["keep0"], case["keep1"]
    first = sizes[0] if a == 1.0 else max(held[0], int(sizes[0] * a))
    second = 0 if b == 0.0 else max(int(sizes[1] * b), min(held[1], sizes[1]) if a != 1.0 else 0)
    return min(first, sizes[0]), min(second, sizes[1])


def work(case):
    T, row = case["T"], case["Hkv"] * case["D"] * 2
    if case["op"] == "tree":
        ctx, m = _drafts(case)
        Hq, D, w = case["Hkv"] * case["G"], case["D"], case["window"]
        read, pairs = 0, 0
        for c, k in zip(ctx.tolist(), m.tolist()):
            back = min(c, w - 1) if w else c
            read += (back + k) if k else 0
            pairs += k * back + (k * (k + 1) // 2 if case["shape"] == "chain" else min(k, 8) * k)
        tokens = int(m.sum())
        words = 8 * -(-case["m_hi"] // 64) if case["shape"] == "tree" else 0
        return {"bytes": read * 2 * row + 4 * read / T + tokens * (Hq * (4 * D + 4) + words), "flops": 4 * pairs * Hq * D}
    if case["op"] == "keep":
        moved = int(np.maximum(_kept(case) - 1, 0).sum())
        return {"bytes": moved * 4 * row * case["L"] + 4 * case["n"], "flops": 0}
    lens = _spread(case["n"], case["lo"], case["hi"])
    blocks = -(-lens // T)
    if case["op"] == "fork":
        # cells of the forks read to be freed, those of their sources read, both written; counts of holders of blocks; rows of the last blocks
        rows = case["kids"] * int((lens % T).sum())
        return {"bytes": rows * 4 * row * case["L"] + 12 * case["kids"] * int(blocks.sum()) + 8 * int((lens // T).sum()), "flops": 0}
    held, sizes = _counts(case)
    first, second = _limits(case, held, sizes)
    moved = held[0] * (1 - first / sizes[0]) + (held[1] * (1 - second / sizes[1]) if sizes[1] else 0)
    cells = int((blocks * (1 + case["kids"])).sum())
    return {"bytes": moved * 4 * row * T * case["L"] + 4 * cells + 4 * (sum(sizes) - sum(held)), "flops": 0}


def _counts(case):
    """Blocks held in either arena and the arenas' sizes, of the cases with a pool."""
    lens = _spread(case["n"], case["lo"], case["hi"])
    T, kids = case["T"], case["kids"]
    blocks = int((-(-lens // T)).sum()) + kids * int((lens % T > 0).sum())
    lent = int(blocks * case["lent"])
    held = (blocks - lent, lent)
    spare = blocks if case["op"] == "compact" else 70             # room for what comes back
    return held, (held[0] + spare, held[1] + (held[1] // 3 + 5 if lent else 0))


# ---------------------------------------------------------------------------------------------- inputs

def _normal(shape, dtype, gen, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=gen, dtype=torch.float32 if math.prod(shape) < (1 << 22) else dtype) * scale).to(dtype)


def _gpu(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


def _ids(rng, count, lent_share):
    """Table entries of `count` blocks in a random order, a share of them in the second arena; and the arenas' sizes."""
    n_lent = int(round(count * lent_share))
    in_lent = rng.permutation(count) < n_lent
    n_local = count - n_lent
    entries = np.empty(count, np.int64)
    entries[~in_lent] = rng.permutation(n_local)
    entries[in_lent] = ~rng.permutation(n_lent)
    return entries, n_local, n_lent


def _arena(s, case, n_local, n_lent, layers, gen):
    """All layers' blocks in one tensor: the first arena's, then the second one's, then one that nobody has (the plain forms write there what is not to be written)."""
    s["arena"] = _normal((layers, n_local + n_lent + 1, 2, case["T"], case["Hkv"], case["D"]), TYPES[case["dtype"]], gen)
    s["local"], s["lent"] = s["arena"][:, :n_local], s["arena"][:, n_local:n_local + n_lent]
    s["n_local"], s["n_lent"] = n_local, n_lent
    if own:
        from paper_2609_27040_b200 import binding as B
        s["caches"] = [B.PagedCache(s["local"][i], s["lent"][i]) for i in range(layers)]
        s["layers"] = B.PagedLayers(s["caches"])


def _rows_of(nb, entries, width):
    tables = np.full((len(nb), width), -1, np.int64)
    tables[np.arange(width)[None, :] < nb[:, None]] = entries
    return tables


def _parents(rng, m):
    """A random tree of m nodes in which a parent comes before its children: -1 for children of the context's last token."""
    up = rng.integers(1, 5, m)
    return np.where(up > np.arange(m), -1, np.arange(m) - up) if m else np.zeros(0, np.int64)


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": dict(case), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    T, n = case["T"], case["n"]
    if case["op"] == "tree":
        order = rng.permutation(n)
        ctx, m = (x[order] for x in _drafts(case))
        lens = np.where(m > 0, ctx + m, ctx)
        nb = -(-lens // T)
        entries, n_local, n_lent = _ids(rng, max(1, int(nb.sum())), case["lent"])
        width = max(1, int(nb.max(initial=1)))
        s["tables"] = _gpu(_rows_of(nb, entries[:int(nb.sum())], width), torch.int32)
        _arena(s, case, n_local, n_lent, 1, gen)
        s["ctx"], s["m"] = ctx, m
        offsets = np.concatenate([[0], np.cumsum(m)])
        tokens = int(offsets[-1])
        s["lens"], s["offsets"] = _gpu(lens, torch.int32), _gpu(offsets, torch.int32)
        words = max(1, -(-case["m_hi"] // 64))
        s["mask"] = s["positions"] = None
        room = max(1, tokens + (5 if n > 1 else 0))                # a captured step has room for a fixed number of tokens
        if case["shape"] == "tree":
            masks, positions = np.zeros((room, words), np.uint64), np.zeros(room, np.int64)
            for i in range(n):
                seen = []
                for j, p in enumerate(_parents(rng, int(m[i])).tolist()):
                    seen.append((seen[p] if p >= 0 else 0) | 1 << j)
                    at = offsets[i] + j
                    positions[at] = ctx[i] + seen[j].bit_count() - 1
                    for w in range(words):
                        masks[at, w] = seen[j] >> (64 * w) & (1 << 64) - 1
            s["mask"] = _gpu(masks.view(np.int64), torch.int64)
            s["positions"] = _gpu(positions, torch.int32) if case["window"] else None
        dtype, Hq, D = TYPES[case["dtype"]], case["Hkv"] * case["G"], case["D"]
        s["q"] = _normal((room, Hq + 2 * case["Hkv"], D), dtype, gen, 1.5)[:, :Hq]   # q of a fused projection
        s["out"] = torch.zeros((room, Hq, D), dtype=dtype, device="cuda")
        s["lse"] = torch.zeros((room, Hq), dtype=torch.float32, device="cuda")
        s["scale"] = D ** -0.5
        if own:
            from paper_2609_27040_b200 import binding as B
            s["work"] = torch.zeros(B.paged_tree_workspace(s["caches"][0], Hq), dtype=torch.uint8, device="cuda")
        return s
    if case["op"] == "keep":
        order = rng.permutation(n)
        ctx, kept = _spread(n, case["lo"], case["hi"])[order], _kept(case)[order]
        nb = -(-(ctx + case["m"]) // T)
        entries, n_local, n_lent = _ids(rng, int(nb.sum()), case["lent"])
        s["tables"], s["lens"] = _gpu(_rows_of(nb, entries, int(nb.max())), torch.int32), _gpu(ctx, torch.int32)
        keep = np.full((n, case["most"]), -1, np.int64)
        for i in range(n):                                         # the first drafted token, then any later ones
            if kept[i]:
                keep[i, 1:kept[i]] = 1 + np.sort(rng.permutation(case["m"] - 1)[:kept[i] - 1])
                keep[i, 0] = 0
        s["keep"], s["counts"] = _gpu(keep, torch.int32), _gpu(kept, torch.int32)
        _arena(s, case, n_local, n_lent, case["L"], gen)
        return s
    # requests and their forks over a pool
    kids = case["kids"]
    lens0 = rng.permutation(_spread(n, case["lo"], case["hi"]))
    held, sizes = _counts(case)
    n_local, n_lent = sizes
    own_blocks = -(-lens0 // T)
    used0, used1 = rng.permutation(n_local), rng.permutation(n_lent)
    used = rng.permutation(np.concatenate([used0[:held[0]], ~used1[:held[1]]]))
    width = max(1, int(own_blocks.max())) + 2
    tables = np.full((n * (1 + kids), width), -1, np.int64)
    tables[:n] = _rows_of(own_blocks, used[:int(own_blocks.sum())], width)
    src = np.repeat(np.arange(n), kids)
    dst = n + rng.permutation(n * kids)
    lens = np.zeros(n * (1 + kids), np.int64)
    lens[:n] = lens0
    refs = [np.zeros(max(1, n_local), np.int64), np.zeros(max(1, n_lent), np.int64)]
    spare = used[int(own_blocks.sum()):]
    if case["op"] == "fork":                                       # the order in which a step frees and takes them: the first arena's first, from the lowest id on
        spare = np.concatenate([np.sort(spare[spare >= 0]), ~np.sort(~spare[spare < 0])])
    for f, k in zip(src, dst):
        whole = int(lens0[f] // T)
        tables[k, :whole] = tables[f, :whole]
        lens[k] = lens0[f]
        if lens0[f] % T:
            tables[k, whole], spare = spare[0], spare[1:]
    for a, sign in ((0, tables), (1, ~tables)):
        width_held = np.arange(width)[None, :] < -(-lens // T)[:, None]
        named = np.bincount(sign[width_held & (sign >= 0)], minlength=len(refs[a]))
        refs[a] = np.maximum(named - 1, 0)
    ids = [np.zeros(max(1, x), np.int64) for x in sizes]
    free = [sizes[0] - held[0], sizes[1] - held[1]]
    ids[0][:free[0]], ids[1][:free[1]] = used0[held[0]:], used1[held[1]:]
    s["src"], s["dst"] = _gpu(src, torch.int32), _gpu(dst, torch.int32)
    # what the calls change, in one piece: a compaction is given the same state in every pass
    parts = dict(tables=tables, refs0=refs[0], refs1=refs[1], ids0=ids[0], ids1=ids[1], free=np.array(free), lens=lens)
    flat = np.concatenate([np.concatenate([x.reshape(-1), np.zeros(-x.size % 4, np.int64)]) for x in parts.values()])
    s["begin"], s["now"] = _gpu(flat, torch.int32), _gpu(flat, torch.int32)
    at = 0
    for name, x in parts.items():
        s[name] = s["now"][at:at + x.size].view(x.shape)
        at += x.size + -x.size % 4
    s["freed"] = s["lens"].clone()
    s["freed"][n:] = 0
    s["limits"] = _gpu(_limits(case, held, sizes) if case["op"] == "compact" else (0, 0), torch.int32)
    s["copies"] = torch.zeros((n * kids if case["op"] == "fork" else sum(held), 3), dtype=torch.int32, device="cuda")
    _arena(s, case, n_local, n_lent, case["L"], gen)
    if own:
        from paper_2609_27040_b200 import binding as B
        s["work"] = torch.zeros(B.PAGED_POOL_WORK_BYTES, dtype=torch.uint8, device="cuda")
        s["share_work"] = torch.zeros(B.paged_shares_workspace(n_local, n_lent), dtype=torch.uint8, device="cuda")
        s["pool"] = B.PagedPool(s["ids0"], s["ids1"] if n_lent else None, s["free"], s["free"], s["work"])
        s["shares"] = B.PagedShares(s["refs0"], s["refs1"] if n_lent else None, s["share_work"])
    return s


# ---------------------------------------------------------------------------------------------- plain forms

def _units(T, device):
    """Row within 8 and stored place of unit u in that row, as index arrays."""
    b = torch.arange(8, device=device)[:, None]
    return b, torch.arange(8, device=device)[None, :] ^ b


def _block(s, e):
    """Index into the arena of both of the blocks that entries name."""
    return torch.where(e >= 0, e, s["n_local"] + ~e)


def _rows(s, lo, hi, blocks):
    """K and V of requests lo..hi - 1, of their first `blocks` blocks, in 32 bits: [n][tokens][Hkv][D]."""
    T, tables = s["case"]["T"], s["tables"][lo:hi, :blocks].long()
    held = torch.arange(blocks, device="cuda")[None, :] * T < s["lens"][lo:hi].long()[:, None]
    x = s["arena"][0, torch.where(held, _block(s, tables), 0)]
    n, w, _, _, Hkv, D = x.shape
    x = x.view(n, w, 2, T // 8, 8, Hkv * D // 64, 8, 8)
    b, u = _units(T, x.device)
    x = x[:, :, :, :, b, :, u]                                     # [row in 8, unit] first, then the others
    x = x.permute(4, 2, 3, 5, 0, 6, 1, 7).reshape(2, n, w * T, Hkv, D)
    return x[0].float(), x[1].float()


def _plain_tree(s):
    c = s["case"]
    T, Hkv, G, D, n = c["T"], c["Hkv"], c["G"], c["D"], c["n"]
    ctx, m = s["ctx"], s["m"]
    lens = np.where(m > 0, ctx + m, 0)
    lo = 0
    while lo < n:                                                  # as many requests at a time as padded scores have room for
        hi, most, long = lo, 0, 0
        while hi < n:
            a, b = max(most, int(m[hi])), max(long, int(lens[hi]))
            if hi > lo and (hi + 1 - lo) * Hkv * G * a * b > 1 << 30:
                break
            most, long, hi = a, b, hi + 1
        if most:
            _plain_part(s, lo, hi, most, -(-long // T))
        lo = hi
    return {"out": s["out"], "lse": s["lse"]}


def _plain_part(s, lo, hi, most, blocks):
    c = s["case"]
    Hkv, G, D, w = c["Hkv"], c["G"], c["D"], c["window"]
    n = hi - lo
    k, v = _rows(s, lo, hi, blocks)
    S = k.shape[1]
    first, end = s["offsets"][lo:hi].long(), s["offsets"][lo + 1:hi + 1].long()
    m = end - first
    begin = (s["lens"][lo:hi].long() - m)[:, None, None]           # where the drafted tokens are
    j = torch.arange(most, device="cuda")
    at = torch.where(j < m[:, None], first[:, None] + j, s["q"].shape[0] - 1)          # [n][most]
    pos = torch.arange(S, device="cuda")[None, None, :]
    place = s["positions"][at].long()[..., None] if s["positions"] is not None else begin + j[None, :, None]
    bit = pos - begin
    context = bit < 0
    if w:
        context = context & (pos > place - w)
    if s["mask"] is not None:
        bits = s["mask"][at]                                       # [n][most][words]
        b = bit.clamp(0, 64 * bits.shape[-1] - 1).expand(n, most, S)
        new = (bits.gather(2, b // 64) >> (b % 64) & 1) == 1
    else:
        new = bit <= j[None, :, None]
        if w:
            new = new & (pos > place - w)
    keep = context | ((bit >= 0) & (bit < m[:, None, None]) & new)
    keep = keep[:, None, None]                                     # [n][1][1][most][S]
    q = s["q"][at].float().reshape(n, most, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * most, D)
    scores = (torch.matmul(q, k.permute(0, 2, 3, 1)) * s["scale"]).view(n, Hkv, G, most, S).masked_fill_(~keep, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp_(scores.sub_(top))
    total = p.sum(-1, keepdim=True)
    held = (pos[0, 0][None, :] < s["lens"][lo:hi].long()[:, None])[..., None, None]
    v = v.masked_fill(~held, 0.0).transpose(1, 2)                  # [n][Hkv][S][D]
    out = torch.matmul(p.view(n, Hkv, G * most, S), v).view(n, Hkv, G, most, D) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).squeeze(-1)                     # [n][Hkv][G][most]
    real = j < m[:, None]
    s["out"].index_put_((at[real],), out.permute(0, 3, 1, 2, 4)[real].reshape(-1, Hkv * G, D).to(s["out"].dtype))
    s["lse"].index_put_((at[real],), lse.permute(0, 3, 1, 2)[real].reshape(-1, Hkv * G))


def _plain_keep(s):
    c = s["case"]
    T, L = c["T"], c["L"]
    keep, counts, lens = s["keep"].long(), s["counts"].long()[:, None], s["lens"].long()[:, None]
    j = torch.arange(keep.shape[1], device="cuda")[None, :]
    real = j < counts
    there, here = lens + torch.where(real, keep, 0), lens + torch.where(real, j, 0)
    tables = s["tables"].long()
    from_block, to_block = (_block(s, tables.gather(1, p // T)) for p in (there, here))
    x = s["arena"][:, from_block, :, there % T]                    # [n][most] first, then layer and plane
    x = x.reshape(x.shape[:4] + (-1, 8, 8))
    unit = torch.arange(8, device="cuda") ^ ((there ^ here) & 7)[..., None]             # a row's units are stored by its place in the block
    x = x.gather(5, unit[:, :, None, None, None, :, None].expand_as(x)).reshape(x.shape[:4] + (c["Hkv"], c["D"]))
    to_block = torch.where(real, to_block, s["n_local"] + s["n_lent"])
    layer, plane = torch.arange(L, device="cuda")[None, None, :, None], torch.arange(2, device="cuda")[None, None, None, :]
    s["arena"].index_put_((layer, to_block[..., None, None], plane, (here % T)[..., None, None]), x)
    return {"local": s["local"], "lent": s["lent"]}


def _copy_blocks(s, copies):
    """The first rows of blocks into others, in all layers."""
    T, copies = s["case"]["T"], copies.long()
    row = torch.arange(T, device="cuda")[None, :]
    on = row < copies[:, 2:]
    src, dst = _block(s, copies[:, :1]).expand_as(on), torch.where(on, _block(s, copies[:, 1:2]), s["n_local"] + s["n_lent"])
    L = s["arena"].shape[0]
    for i in range(0, copies.shape[0], 1 << 14):
        a, b = src[i:i + (1 << 14)], dst[i:i + (1 << 14)]
        for layer in range(L):
            for plane in range(2):
                s["arena"][layer, :, plane].index_put_((b, row), s["arena"][layer, :, plane][a, row])


def _plain_free(s, lens, new_lens):
    T, tables = s["case"]["T"], s["tables"].long()
    j = torch.arange(tables.shape[1], device="cuda")[None, :]
    gone = (j >= ((new_lens.long() + T - 1) // T)[:, None]) & (j < ((lens.long() + T - 1) // T)[:, None])
    top = s["free"].long()
    tops = []
    for a, e in ((0, tables), (1, ~tables)):
        refs, ids = s["refs%d" % a], s["ids%d" % a]
        mine = gone & (e >= 0)
        named = torch.zeros(refs.numel() + 1, dtype=torch.int64, device="cuda")
        named.index_add_(0, torch.where(mine, e, refs.numel()).flatten(), torch.ones_like(e).flatten())
        left = refs.long() - named[:-1]
        freed = (left < 0).flip(0)                                 # pushed from the highest id down
        refs.copy_(left.clamp(min=0))
        at = torch.where(freed, top[a] + freed.long().cumsum(0) - 1, ids.numel())
        values = torch.arange(refs.numel() - 1, -1, -1, device="cuda")
        ids.copy_(torch.cat([ids.long(), ids.new_zeros(1).long()]).index_put((at,), values)[:-1])
        tops.append(top[a] + freed.sum())
    s["free"].copy_(torch.stack(tops))


def _plain_fork(s, lens, new_lens):
    T, tables = s["case"]["T"], s["tables"].long()
    src, dst = s["src"].long(), s["dst"].long()
    length = lens.long()[src]
    whole = length // T
    tail = length % T
    first = (tail > 0).long().cumsum(0) - 1
    top = s["free"].long()
    from0 = s["ids0"].long()[(top[0] - 1 - first).clamp(min=0)]
    from1 = s["ids1"].long()[(top[1] - 1 - (first - top[0])).clamp(0, s["ids1"].numel() - 1)]
    new = torch.where(first < top[0], from0, ~from1)
    j = torch.arange(tables.shape[1], device="cuda")[None, :]
    cells = tables[src]
    old = cells.gather(1, whole[:, None]).squeeze(1)
    shared = j < whole[:, None]
    for a, e in ((0, cells), (1, ~cells)):
        refs = s["refs%d" % a]
        named = torch.zeros(refs.numel() + 1, dtype=torch.int64, device="cuda")
        named.index_add_(0, torch.where(shared & (e >= 0), e, refs.numel()).flatten(), torch.ones_like(e).flatten())
        refs.add_(named[:-1].to(torch.int32))
    after = torch.where(shared, cells, torch.where((j == whole[:, None]) & (tail > 0)[:, None], new[:, None], tables[dst]))
    s["tables"].index_put_((dst,), after.to(torch.int32))
    new_lens.index_put_((dst,), length.to(torch.int32))
    need = (tail > 0).sum()
    popped = torch.minimum(need, top[0])
    s["free"].copy_(torch.stack([top[0] - popped, top[1] - (need - popped)]))
    s["copies"].copy_(torch.where((tail > 0)[:, None], torch.stack([old, new, tail], 1), 0))
    _copy_blocks(s, s["copies"])


def _plain_compact(s):
    T, tables, lens = s["case"]["T"], s["tables"].long(), s["lens"].long()
    j = torch.arange(tables.shape[1], device="cuda")[None, :]
    held = j * T < lens[:, None]
    sizes = (s["n_local"], s["n_lent"])
    moving, eligible = [], []
    for a, e in ((0, tables), (1, ~tables)):
        used = torch.zeros(s["refs%d" % a].numel() + 1, dtype=torch.bool, device="cuda")
        used[torch.where(held & (e >= 0), e, used.numel() - 1).flatten()] = True
        i = torch.arange(used.numel() - 1, device="cuda")
        moving.append(used[:-1] & (i >= s["limits"][a]) & (i < sizes[a]))
        ids = s["ids%d" % a].long()
        k = torch.arange(ids.numel(), device="cuda")
        ok = (k < s["free"][a]) & (ids < s["limits"][a])
        at = torch.where(ok, ok.long().cumsum(0) - 1, ids.numel())
        eligible.append((torch.cat([ids, ids.new_zeros(1)]).index_put((at,), ids)[:-1], ok.sum()))
    (ids0, n0), (ids1, n1) = eligible
    u0 = moving[0].sum()
    need = u0 + moving[1].sum()
    new, copies = [], torch.zeros_like(s["copies"]).long()
    copies = torch.cat([copies, copies.new_zeros((1, 3))])
    rank = torch.cat([moving[0], moving[1]]).long().cumsum(0) - 1
    old = torch.cat([torch.arange(moving[0].numel(), device="cuda"), ~torch.arange(moving[1].numel(), device="cuda")])
    to = torch.where(rank < n0, ids0[(n0 - 1 - rank).clamp(0, ids0.numel() - 1)], ~ids1[(n1 - 1 - (rank - n0)).clamp(0, ids1.numel() - 1)])
    on = torch.cat([moving[0], moving[1]])
    at = torch.where(on, rank, copies.shape[0] - 1)
    copies.index_put_((at,), torch.stack([old, to, torch.full_like(to, T)], 1))
    s["copies"].copy_(copies[:-1])
    # tables and counts of holders
    size0 = moving[0].numel()
    which = torch.where(tables >= 0, tables, size0 + ~tables).clamp(0, on.numel() - 1)
    s["tables"].copy_(torch.where(held & on[which], to[which], tables))
    refs = torch.cat([s["refs0"], s["refs1"]]).long()
    place = torch.where(on, torch.where(to >= 0, to, size0 + ~to), refs.numel())
    after = torch.cat([torch.where(on, 0, refs), refs.new_zeros(1)]).index_put((place,), refs)[:-1]
    s["refs0"].copy_(after[:size0])
    s["refs1"].copy_(after[size0:])
    popped = torch.minimum(need, n0)
    for a, (ids, count) in enumerate(eligible):
        k = torch.arange(ids.numel(), device="cuda")
        s["ids%d" % a].copy_(torch.where(k < count, ids, s["ids%d" % a].long()))
    s["free"].copy_(torch.stack([n0 - popped, n1 - (need - popped)]))
    _copy_blocks(s, s["copies"])


def _state(s):
    return {k: s[k] for k in ("tables", "refs0", "refs1", "ids0", "ids1", "free", "lens", "copies", "local", "lent")}


def run(s):
    c = s["case"]
    if own:
        from paper_2609_27040_b200 import binding as B
        stream = torch.cuda.current_stream()
    if c["op"] == "tree":
        if not own:
            return _plain_tree(s)
        B.paged_tree_attention(s["caches"][0], s["tables"], s["lens"], s["offsets"], s["q"], s["scale"], s["out"], s["work"], mask=s["mask"],
                               lse=s["lse"], window=c["window"], positions=s["positions"], status=s["status"], stream=stream)
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "keep":
        if not own:
            return _plain_keep(s)
        B.paged_keep_rows(s["layers"], s["tables"], s["lens"], s["keep"], s["counts"], status=s["status"], stream=stream)
        return {"local": s["local"], "lent": s["lent"]}
    if c["op"] == "fork":                                          # the forks are freed and made again: the same state before and after
        if not own:
            _plain_free(s, s["lens"], s["freed"])
            _plain_fork(s, s["freed"], s["lens"])
            return _state(s)
        B.paged_free(s["pool"], s["shares"], s["lens"], s["freed"], c["T"], s["tables"], status=s["status"], stream=stream)
        B.paged_fork(s["pool"], s["shares"], s["freed"], s["lens"], s["src"], s["dst"], c["T"], s["tables"], s["copies"], status=s["status"],
                     stream=stream)
        B.paged_copy_blocks(s["layers"], s["copies"], status=s["status"], stream=stream)
        return _state(s)
    s["now"].copy_(s["begin"])
    if not own:
        _plain_compact(s)
        return _state(s)
    B.paged_compact(s["pool"], s["shares"], s["limits"], s["lens"], c["T"], s["tables"], s["copies"], status=s["status"], stream=stream)
    B.paged_copy_blocks(s["layers"], s["copies"], status=s["status"], stream=stream)
    return _state(s)


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits

def _stored(C, row):
    """Place of column c in a row of token index `row` (within its block)."""
    col = torch.arange(C, device="cuda")
    return (col // 64) * 64 + (((col % 64) // 8) ^ (row & 7)[:, None]) * 8 + col % 8


def _exact_tree(case, s):
    T, Hkv, G, D, w = case["T"], case["Hkv"], case["G"], case["D"], case["window"]
    C = Hkv * D
    out, lse = s["out"].double(), s["lse"].double()
    offsets, tables = s["offsets"].tolist(), s["tables"].tolist()
    for i in range(case["n"]):
        m, c = int(s["m"][i]), int(s["ctx"][i])
        if m == 0:
            continue
        p = torch.arange(c + m, device="cuda")
        e = torch.tensor(tables[i], device="cuda")[p // T]
        place = _stored(C, p % T)
        kv = []
        for plane in (0, 1):
            x = torch.empty((c + m, C), device="cuda", dtype=torch.float64)
            for on, arena, ids in ((e >= 0, s["local"], e), (e < 0, s["lent"], ~e)):
                if bool(on.any()):
                    x[on] = arena[0][ids[on], plane, (p % T)[on]].reshape(-1, C).gather(1, place[on]).double()
            kv.append(x.view(-1, Hkv, D).transpose(0, 1))          # [Hkv][tokens][D]
        k, v = kv
        for t0 in range(0, m, 128):
            t1 = min(m, t0 + 128)
            rows = slice(offsets[i] + t0, offsets[i] + t1)
            j = torch.arange(t0, t1, device="cuda")[:, None]
            pos = s["positions"][rows].long()[:, None] if s["positions"] is not None else c + j
            see = (p < c)[None, :].expand(t1 - t0, -1).clone()
            if w:
                see &= p[None, :] >= pos - w + 1
            if s["mask"] is None:
                new = torch.arange(m, device="cuda")[None, :] <= j
                if w:
                    new &= c + torch.arange(m, device="cuda")[None, :] >= pos - w + 1
            else:
                words = s["mask"][rows].cpu().numpy().view(np.uint64)
                new = torch.from_numpy(np.array([[int(r[b // 64]) >> (b % 64) & 1 == 1 for b in range(m)] for r in words])).to("cuda")
            see[:, c:] = new
            q = s["q"][rows].double().reshape(t1 - t0, Hkv, G, D).permute(1, 2, 0, 3)
            z = (q @ k[:, None].transpose(2, 3) * s["scale"]).masked_fill(~see, -math.inf)
            none = ~see.any(1)
            prob = torch.softmax(z, -1).masked_fill(none[:, None], 0.0)
            out[rows] = (prob @ v[:, None]).permute(2, 0, 1, 3).reshape(t1 - t0, Hkv * G, D)
            lse[rows] = torch.logsumexp(z, -1).permute(2, 0, 1).reshape(t1 - t0, Hkv * G)
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    T, C = case["T"], case["Hkv"] * case["D"]
    if case["op"] == "tree":
        return _exact_tree(case, s)
    arena = s["arena"].double()
    flat = arena.view(arena.shape[0], -1, 2, T, C)

    def at(e):
        return e if e >= 0 else s["n_local"] + ~e

    tables = s["tables"].tolist()
    parts = {"local": arena[:, :s["n_local"]], "lent": arena[:, s["n_local"]:s["n_local"] + s["n_lent"]]}
    if case["op"] == "keep":
        lens, keep, counts = s["lens"].tolist(), s["keep"].tolist(), s["counts"].tolist()
        pairs = [(tables[i][(lens[i] + r) // T], (lens[i] + r) % T, tables[i][(lens[i] + j) // T], (lens[i] + j) % T)
                 for i in range(case["n"]) for j, r in enumerate(keep[i][:counts[i]])]
        if pairs:
            e0, r0, e1, r1 = (torch.tensor(x, device="cuda") for x in zip(*[(at(a), b, at(c), d) for a, b, c, d in pairs]))
            plain = flat[:, e0, :, r0].gather(3, _stored(C, r0)[:, None, None].expand(-1, flat.shape[0], 2, -1))
            back = torch.zeros_like(plain).scatter(3, _stored(C, r1)[:, None, None].expand(-1, flat.shape[0], 2, -1), plain)
            flat[:, e1, :, r1] = back
        return parts
    none = {k: None for k in ("tables", "refs0", "refs1", "ids0", "ids1", "free", "lens", "copies")}
    ids = [s["ids0"].tolist()[:int(s["free"][0])], s["ids1"].tolist()[:int(s["free"][1])]]
    lens = s["lens"].tolist()
    if case["op"] == "fork":
        n, moves = case["n"], []
        held = {}
        for i, length in enumerate(lens):
            for b in range(-(-length // T)):
                held.setdefault(tables[i][b], []).append(i)
        gone = [e for e, who in held.items() if all(i >= n for i in who)]
        ids[0] += sorted((e for e in gone if e >= 0), reverse=True)
        ids[1] += sorted((~e for e in gone if e < 0), reverse=True)
        for i in s["src"].tolist():
            if lens[i] % T:
                new = ids[0].pop() if ids[0] else ~ids[1].pop()
                moves.append((tables[i][lens[i] // T], new, lens[i] % T))
    else:
        limits = s["limits"].tolist()
        used = sorted({tables[i][b] for i in range(len(lens)) for b in range(-(-lens[i] // T))}, key=lambda e: (e < 0, at(e)))
        ids = [[x for x in ids[a] if x < limits[a]] for a in (0, 1)]
        moves = [(e, ids[0].pop() if ids[0] else ~ids[1].pop(), T) for e in used if (e if e >= 0 else ~e) >= limits[e < 0]]
    for r in {x[2] for x in moves}:
        e0, e1 = (torch.tensor([at(x[k]) for x in moves if x[2] == r], device="cuda") for k in (0, 1))
        flat[:, e1, :, :r] = flat[:, e0, :, :r]
    return {**none, **parts}
