"""The device-driven serving step of a paged KV cache, as measured: block tables and slot maps built
from request lengths, new K/V rows written through the slot map, attention of one new token per request
read through device-resident tables, and its differential form. Plain forms in elementary torch
operations beside the framework's calls.

Cache format (as in the rest of the framework): a block is a K plane [T][Hkv][D] and a V plane of the
same shape, 16-bit elements; inside token row r, within every aligned 64 elements, the unit of 8
elements u is stored at unit u ^ (r & 7). A table entry e >= 0 names block e of the first arena, e < 0
block ~e of the second one; a slot is block * T + row, or its complement in the second arena.
"""
import math

import numpy as np
import torch

own = False

NO_SLOT = -(1 << 63)
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one decode step of a large running batch: every request grows by its token, some need a block
        dict(name="tables_step_256", op="tables", n=256, T=16, lo=512, hi=4096, add_lo=1, add_hi=1, lent=0.4, back=False),
        # draft tokens of speculative decoding, appended and taken back again: two calls
        dict(name="tables_drafts_97", op="tables", n=97, T=32, lo=1, hi=9000, add_lo=3, add_hi=9, lent=0.0, back=True),
        # admission of prompts next to running requests: about half a million new tokens
        dict(name="tables_prompts_1000", op="tables", n=1000, T=16, lo=0, hi=100, add_lo=1, add_hi=1100, lent=0.5, back=False),
        # the new rows of a decode step whose batch is padded for a captured graph
        dict(name="write_step_250_of_256", op="write", n=250, pad=6, T=16, Hkv=8, D=128, dtype="fp16", lent=0.4),
        # the rows of a long prompt, cut out of a fused projection
        dict(name="write_prompt_131071", op="write", n=131071, pad=0, T=16, Hkv=8, D=128, dtype="bf16", lent=0.4),
        # one short request: latency alone
        dict(name="decode_1x500", op="decode", n=1, lo=500, hi=500, T=16, Hkv=8, G=4, D=128, dtype="bf16", lent=0.25, window=0),
        # the batch of the benchmark: 64 requests of 512 to 4096 tokens, 40 % of their blocks lent
        dict(name="decode_64x4096", op="decode", n=64, lo=512, hi=4095, T=16, Hkv=8, G=4, D=128, dtype="bf16", lent=0.4, window=0),
        # few very long requests: the split over the length carries the work
        dict(name="decode_5x100001", op="decode", n=5, lo=60000, hi=100001, T=32, Hkv=8, G=8, D=128, dtype="fp16", lent=0.0, window=0),
        # a ragged padded batch with empty rows, small heads without sharing, the last 1000 tokens only
        dict(name="decode_window_200", op="decode", n=200, lo=0, hi=5000, T=64, Hkv=12, G=1, D=64, dtype="bf16", lent=0.0, window=1000),
        # differential attention of a few short requests: latency
        dict(name="diff_3x700", op="diff", n=3, lo=1, hi=700, T=16, Hkv=4, G=2, D=128, dtype="fp16", lent=0.0, norm=True),
        # its ordinary batch
        dict(name="diff_48x6000", op="diff", n=48, lo=300, hi=6000, T=16, Hkv=8, G=4, D=128, dtype="bf16", lent=0.3, norm=True),
        # wide heads, long requests
        dict(name="diff_8x40000", op="diff", n=8, lo=9000, hi=40000, T=16, Hkv=4, G=4, D=256, dtype="bf16", lent=0.0, norm=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "write", "decode", "decode", "diff"])
    lent = rng.choice([0.0, rng.uniform(0.1, 0.9)])
    T = rng.choice([16, 32, 64])
    if op == "tables":
        n = _log(rng, 1, 4000)
        add_hi = _log(rng, 1, max(2, min(2000, 400000 // n)))
        return dict(op=op, n=n, T=T, lo=rng.choice([0, 1, 30]), hi=_log(rng, 40, 6000), add_lo=rng.choice([0, 1]), add_hi=add_hi,
                    lent=lent, back=rng.random() < 0.4)
    D = rng.choice([64, 128, 256])
    Hkv = rng.randint(1, 16)
    dtype = rng.choice(["bf16", "fp16"])
    if op == "write":
        return dict(op=op, n=_log(rng, 1, 100000 * 8 * 128 // (max(8, Hkv) * max(128, D))), pad=rng.choice([0, rng.randint(1, 40)]),
                    T=T, Hkv=Hkv, D=D, dtype=dtype, lent=lent)
    n = _log(rng, 1, 160)
    G = rng.choice([1, 2, 3, 4, 5, 7, 8]) if op == "diff" else rng.randint(1, 16)
    most = 300000 * 8 * 128 // (n * Hkv * max(G, 4) // 4 * D)     # tokens per request that keep a pass below the largest listed ones
    hi = _log(rng, 1, max(2, min(100000, most)))
    case = dict(op=op, n=n, lo=rng.choice([0, 1, hi // 3, hi // 2]), hi=hi, T=T, Hkv=Hkv, G=G, D=D, dtype=dtype, lent=lent)
    case.update(dict(window=rng.choice([0, 0, rng.randint(1, hi)])) if op == "decode" else dict(norm=rng.random() < 0.6))
    return case


def _spread(n, lo, hi):
    """n whole numbers spread evenly over lo..hi: the same for every seed, so that work() knows them."""
    if n == 1:
        return np.array([hi], np.int64)
    return np.floor(lo + (hi - lo) * np.arange(n) / (n - 1) + 0.5).astype(np.int64)


def _lengths(case):
    return _spread(case["n"], case["lo"], case["hi"])


def _growth(case):
    """Old and new lengths, paired the same for every seed (which orders the pairs)."""
    old = _lengths(case)
    return old, old + np.random.default_rng(case["n"]).permutation(_spread(case["n"], case["add_lo"], case["add_hi"]))


def work(case):
    if case["op"] == "tables":
        old, new = _growth(case)
        tokens, blocks = int((new - old).sum()), int((-(-new // case["T"]) - -(-old // case["T"])).sum())
        once = 8 * case["n"] + 4 * (case["n"] + 1) + 12 * tokens + 8 * blocks
        return {"bytes": once * (2 if case["back"] else 1), "flops": 0}
    row = case["Hkv"] * case["D"] * 2
    if case["op"] == "write":
        return {"bytes": case["n"] * (4 * row + 8), "flops": 0}
    lens = _lengths(case)
    if case.get("window"):
        lens = np.minimum(lens, case["window"])
    tokens, Hq = int(lens.sum()), case["Hkv"] * case["G"]
    D, n = case["D"], case["n"]
    maps = 2 if case["op"] == "diff" else 1
    # diff: q holds two maps of width D/2 per head; scores 2 * 2 * D/2, values 2 * 2 * D per head and token
    q_out = n * Hq * D * 2 * 2 + (n * Hq * 4 if maps == 1 else 0)
    flops = tokens * Hq * (2 * D + 2 * D * maps)
    return {"bytes": tokens * 2 * row + q_out + 4 * tokens / case["T"], "flops": flops}


# ---------------------------------------------------------------------------------------------- inputs

def _normal(shape, dtype, gen, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=gen, dtype=torch.float32 if math.prod(shape) < (1 << 22) else dtype) * scale).to(dtype)


def _arenas(case, local, lent, gen):
    """Two arenas of random blocks, each with one block more than its cache has (the plain form's writes of padding land there)."""
    shape = (2, case["T"], case["Hkv"], case["D"])
    return _normal((local + 1,) + shape, TYPES[case["dtype"]], gen), _normal((lent + 1,) + shape, TYPES[case["dtype"]], gen)


def _ids(rng, count, lent_share):
    """Table entries of `count` blocks in a random order, a share of them in the second arena; and the arenas' sizes."""
    n_lent = int(round(count * lent_share))
    in_lent = rng.permutation(count) < n_lent
    n_local = count - n_lent
    entries = np.empty(count, np.int64)
    entries[~in_lent] = rng.permutation(n_local)
    entries[in_lent] = ~rng.permutation(n_lent)
    return entries, n_local, n_lent


def _gpu(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": dict(case), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    T = case["T"]
    if case["op"] == "tables":
        n = case["n"]
        order = rng.permutation(n)
        old, new = (x[order] for x in _growth(case))
        ob, nb = -(-old // T), -(-new // T)
        held, need = int(ob.sum()), int((nb - ob).sum())
        n_local = int(round(need * (1 - case["lent"])))
        n_lent = need - n_local
        spare = 64
        # ids 0.. of each arena in a random order: the first ones are held by the requests, the rest are free
        held_lent = int(held * case["lent"])
        ids0 = rng.permutation(held - held_lent + n_local + (0 if n_lent else spare))
        ids1 = rng.permutation(held_lent + n_lent + spare)
        entries = rng.permutation(np.concatenate([ids0[:held - held_lent], ~ids1[:held_lent]]))
        free0, free1 = ids0[held - held_lent:], ids1[held_lent:]
        width = int(nb.max(initial=1)) + 3
        tables = np.full((n, width), -1, np.int64)
        tables[np.arange(width)[None, :] < ob[:, None]] = entries
        s["ids0"], s["ids1"] = (_gpu(np.concatenate([f, np.zeros(len(i) - len(f), np.int64)]), torch.int32) for f, i in ((free0, ids0), (free1, ids1)))
        s["free"] = _gpu([len(free0), len(free1)], torch.int32)
        s["lens"], s["new_lens"], s["tables"] = _gpu(old, torch.int32), _gpu(new, torch.int32), _gpu(tables, torch.int32)
        tokens = int((new - old).sum())
        room = max(1, -(-tokens // 64) * 64)                       # a captured step has room for a fixed number of tokens
        for k in ("", "2"):
            s["free_out" + k] = torch.zeros(2, dtype=torch.int32, device="cuda")
            s["offsets" + k] = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
            s["slots" + k] = torch.zeros(room, dtype=torch.int64, device="cuda")
            s["positions" + k] = torch.zeros(room, dtype=torch.int32, device="cuda")
        if own:
            from paper_2609_27040_b200 import binding as B
            s["work"] = torch.zeros(B.PAGED_POOL_WORK_BYTES, dtype=torch.uint8, device="cuda")
            s["pool"] = B.PagedPool(s["ids0"], s["ids1"], s["free"], s["free_out"], s["work"])
            s["pool2"] = B.PagedPool(s["ids0"], s["ids1"], s["free_out"], s["free_out2"], s["work"])
        return s
    if case["op"] == "write":
        n, Hkv, D = case["n"], case["Hkv"], case["D"]
        blocks = -(-n // T) + 8
        entries, n_local, n_lent = _ids(rng, blocks, case["lent"])
        where = rng.permutation(blocks * T)[:n] if n < 2000 else np.arange(n)   # single rows of many requests, or a prompt's in order
        slots = entries[where // T]
        slots = np.where(slots >= 0, slots * T + where % T, ~(~slots * T + where % T))
        s["slots"] = _gpu(np.concatenate([slots, np.full(case["pad"], NO_SLOT, np.int64)]), torch.int64)
        fused = _normal((n + case["pad"], 6 * Hkv, D), TYPES[case["dtype"]], gen)   # q, k and v of one projection, four query heads to a KV head
        s["k"], s["v"] = fused[:, 4 * Hkv:5 * Hkv], fused[:, 5 * Hkv:]
        s["local"], s["lent"] = _arenas(case, n_local, n_lent, gen)
        s["n_local"], s["n_lent"] = n_local, n_lent
    else:
        n, Hkv, D, Hq = case["n"], case["Hkv"], case["D"], case["Hkv"] * case["G"]
        lens = rng.permutation(_lengths(case))
        nb = -(-lens // T)
        entries, n_local, n_lent = _ids(rng, int(nb.sum()), case["lent"])
        width = max(1, int(nb.max(initial=1)))
        tables = np.full((n, width), -1, np.int64)
        tables[np.arange(width)[None, :] < nb[:, None]] = entries
        s["tables"], s["lens"] = _gpu(tables, torch.int32), _gpu(lens, torch.int32)
        s["local"], s["lent"] = _arenas(case, n_local, n_lent, gen)
        s["n_local"], s["n_lent"] = n_local, n_lent
        dtype = TYPES[case["dtype"]]
        s["scale"] = (D if case["op"] == "decode" else D // 2) ** -0.5
        if case["op"] == "decode":
            s["q"] = _normal((n, Hq + 2 * Hkv, D), dtype, gen, 1.5)[:, :Hq]         # q of a fused projection
            s["lse"] = torch.empty((n, Hq), dtype=torch.float32, device="cuda")
        else:
            s["q"] = _normal((n, 2 * Hq, D // 2), dtype, gen, 1.5)
            s["lam"] = torch.rand(Hq, device="cuda", generator=gen) * 0.6 + 0.2
            s["weight"] = torch.rand(D, device="cuda", generator=gen) + 0.5 if case["norm"] else None
            s["eps"], s["out_scale"] = 1e-5, 0.8 if case["norm"] else 1.0
        s["out"] = torch.empty((n, Hq, D), dtype=dtype, device="cuda")
    if own:
        from paper_2609_27040_b200 import binding as B
        s["cache"] = B.PagedCache(s["local"][:s["n_local"]], s["lent"][:s["n_lent"]])
        if case["op"] != "write":
            s["work"] = torch.zeros(B.paged_decode_workspace(s["cache"], case["Hkv"] * case["G"] * (2 if case["op"] == "diff" else 1)),
                                    dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- plain forms

def _build(T, lens, new_lens, tables, ids0, ids1, free, room):
    """One call: (tables, ids0, ids1, free, offsets, slots, positions) after it."""
    old, new, tables = lens.long(), new_lens.long(), tables.long()
    ids0, ids1, free = ids0.long(), ids1.long(), free.long()
    ob, nb = (old + T - 1) // T, (new + T - 1) // T
    need, add = (nb - ob).clamp(min=0), (new - old).clamp(min=0)
    first = need.cumsum(0) - need
    offsets = torch.cat([add.new_zeros(1), add.cumsum(0)])
    j = torch.arange(tables.shape[1], device=tables.device)[None, :]
    k = first[:, None] + j - ob[:, None]
    popped0 = torch.minimum(need.sum(), free[0])
    popped1 = need.sum() - popped0
    from0 = ids0[(free[0] - 1 - k).clamp(0, ids0.numel() - 1)]
    from1 = ids1[(free[1] - 1 - (k - free[0])).clamp(0, ids1.numel() - 1)]
    after = torch.where((j >= ob[:, None]) & (j < nb[:, None]), torch.where(k < free[0], from0, ~from1), tables)
    t = torch.arange(room, device=tables.device)
    seq = (torch.searchsorted(offsets, t, right=True) - 1).clamp(max=old.numel() - 1)
    real = t < offsets[-1]
    pos = torch.where(real, old[seq] + t - offsets[seq], 0)
    e = after[seq, pos // T]
    slot = torch.where(e >= 0, e * T + pos % T, ~(~e * T + pos % T))
    slots = torch.where(real, slot, NO_SLOT)
    positions = torch.where(real, pos, -1)
    # blocks given back: requests and blocks in descending order, each to its arena's stack
    gone = ((j >= nb[:, None]) & (j < ob[:, None])).flatten().flip(0)
    e = tables.flatten().flip(0)
    g0, g1 = gone & (e >= 0), gone & (e < 0)
    at0 = torch.where(g0, free[0] - popped0 + g0.long().cumsum(0) - 1, ids0.numel())
    at1 = torch.where(g1, free[1] - popped1 + g1.long().cumsum(0) - 1, ids1.numel())
    ids0 = torch.cat([ids0, ids0.new_zeros(1)]).index_put((at0,), e)[:-1]
    ids1 = torch.cat([ids1, ids1.new_zeros(1)]).index_put((at1,), ~e)[:-1]
    free = torch.stack([free[0] - popped0 + g0.sum(), free[1] - popped1 + g1.sum()])
    i32 = torch.int32
    return after.to(i32), ids0.to(i32), ids1.to(i32), free.to(i32), offsets.to(i32), slots, positions.to(i32)


def _units(T, device):
    """Row within 8 and stored place of unit u in that row, as index arrays."""
    b = torch.arange(8, device=device)[:, None]
    return b, torch.arange(8, device=device)[None, :] ^ b


def _rows(s):
    """K and V of every request, padded to its table's width, in 32 bits: [n][tokens][Hkv][D]."""
    T, tables, lens = s["case"]["T"], s["tables"].long(), s["lens"].long()
    held = torch.arange(tables.shape[1], device="cuda")[None, :] * T < lens[:, None]
    e = torch.where(held, tables, 0 if s["n_local"] else -1)
    x = s["local"][e.clamp(min=0)]
    if s["n_lent"]:
        x = torch.where((e >= 0)[..., None, None, None, None], x, s["lent"][(~e).clamp(min=0)])
    n, w, _, _, Hkv, D = x.shape
    x = x.view(n, w, 2, T // 8, 8, Hkv * D // 64, 8, 8)
    b, u = _units(T, x.device)
    x = x[:, :, :, :, b, :, u]                                     # [row in 8, unit] first, then the others
    x = x.permute(4, 2, 3, 5, 0, 6, 1, 7).reshape(2, n, w * T, Hkv, D)
    return x[0].float(), x[1].float()


def _softmax(scores, keep):
    scores = scores.masked_fill(~keep, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    w = torch.exp(scores - top)
    total = w.sum(-1, keepdim=True)
    return w / torch.where(total == 0, 1.0, total), (top + torch.log(total)).squeeze(-1)


def _plain_decode(s):
    c = s["case"]
    k, v = _rows(s)
    n, S, Hkv, D = k.shape
    lens = s["lens"].long()[:, None]
    pos = torch.arange(S, device="cuda")[None, :]
    keep = pos < lens
    if c.get("window"):
        keep &= pos >= lens - c["window"]
    v = v.masked_fill(~keep[..., None, None], 0.0).transpose(1, 2)                  # [n][Hkv][S][D]
    if c["op"] == "decode":
        q = s["q"].float().reshape(n, Hkv, c["G"], D)
        scores = torch.matmul(q, k.permute(0, 2, 3, 1)) * s["scale"]
        w, lse = _softmax(scores, keep[:, None, None, :])
        out = torch.matmul(w, v).reshape(n, Hkv * c["G"], D)
        return {"out": out.to(s["out"].dtype), "lse": lse.reshape(n, -1)}
    q = s["q"].float().reshape(n, Hkv, c["G"], 2, D // 2).transpose(2, 3)          # [n][Hkv][map][G][d]
    k = k.reshape(n, S, Hkv, 2, D // 2).permute(0, 2, 3, 4, 1)
    w, _ = _softmax(torch.matmul(q, k) * s["scale"], keep[:, None, None, None, :])
    lam = s["lam"].reshape(Hkv, c["G"], 1)
    out = torch.matmul(w[:, :, 0], v) - lam * torch.matmul(w[:, :, 1], v)
    if s["weight"] is not None:
        out = out * torch.rsqrt(out.square().mean(-1, keepdim=True) + s["eps"]) * s["weight"]
    return {"out": (out * s["out_scale"]).reshape(n, Hkv * c["G"], D).to(s["out"].dtype)}


def _plain_write(s):
    T, slots = s["case"]["T"], s["slots"]
    first, second = slots >= 0, (slots < 0) & (slots != NO_SLOT)
    at = torch.where(first, slots, torch.where(second, ~slots, 0))
    block, row = at // T, at % T
    token = torch.arange(slots.numel(), device="cuda")[:, None]
    unit = torch.arange(8, device="cuda")[None, :] ^ (row & 7)[:, None]
    for_local, for_lent = torch.where(first, block, s["n_local"]), torch.where(second, block, s["n_lent"])
    k, v = (x.reshape(x.shape[0], -1, 8, 8)[token, :, unit].transpose(1, 2).reshape(x.shape) for x in (s["k"], s["v"]))
    both = torch.stack([k, v], 1)
    plane = torch.arange(2, device="cuda")[None, :]
    s["local"].index_put_((for_local[:, None], plane, row[:, None]), both)
    s["lent"].index_put_((for_lent[:, None], plane, row[:, None]), both)
    return {"local": s["local"][:s["n_local"]], "lent": s["lent"][:s["n_lent"]]}


def run(s):
    c = s["case"]
    if c["op"] == "tables":
        if own:
            from paper_2609_27040_b200 import binding as B
            stream = torch.cuda.current_stream()
            B.paged_build_tables(s["pool"], s["lens"], s["new_lens"], c["T"], s["tables"], s["offsets"], s["slots"], s["positions"],
                                 status=s["status"], stream=stream)
            if c["back"]:
                B.paged_build_tables(s["pool2"], s["new_lens"], s["lens"], c["T"], s["tables"], s["offsets2"], s["slots2"], s["positions2"],
                                     status=s["status"], stream=stream)
            got = (s["tables"], s["ids0"], s["ids1"], s["free_out"], s["offsets"], s["slots"], s["positions"])
            back = (s["tables"], s["ids0"], s["ids1"], s["free_out2"], s["offsets2"], s["slots2"], s["positions2"])
        else:
            room = s["slots"].numel()
            got = _build(c["T"], s["lens"], s["new_lens"], s["tables"], s["ids0"], s["ids1"], s["free"], room)
            back = _build(c["T"], s["new_lens"], s["lens"], *got[:4], room) if c["back"] else None
        names = ("tables", "ids0", "ids1", "free", "offsets", "slots", "positions")
        return {"there": dict(zip(names, got)), "back": dict(zip(names, back))} if c["back"] else dict(zip(names, got))
    if not own:
        return _plain_write(s) if c["op"] == "write" else _plain_decode(s)
    from paper_2609_27040_b200 import binding as B
    stream = torch.cuda.current_stream()
    if c["op"] == "write":
        B.paged_write_kv(s["cache"], s["k"], s["v"], s["slots"], status=s["status"], stream=stream)
        return {"local": s["local"][:s["n_local"]], "lent": s["lent"][:s["n_lent"]]}
    if c["op"] == "decode":
        B.paged_decode_tables(s["cache"], s["tables"], s["lens"], s["q"], s["scale"], s["out"], s["work"], lse=s["lse"],
                              window=c["window"], status=s["status"], stream=stream)
        return {"out": s["out"], "lse": s["lse"]}
    B.paged_decode_diff(s["cache"], s["tables"], s["lens"], s["q"], s["lam"], s["scale"], s["out"], s["work"], norm_weight=s["weight"],
                        eps=s["eps"], out_scale=s["out_scale"], status=s["status"], stream=stream)
    return {"out": s["out"]}


# ---------------------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    if case["op"] == "tables":
        return None                                                # whole numbers throughout
    s = prepare(case, seed)
    T, Hkv, D = case["T"], case["Hkv"], case["D"]
    C = Hkv * D
    col = torch.arange(C, device="cuda")

    def stored(row):                                               # place of column c in a row of token index `row` (within its block)
        return (col // 64) * 64 + (((col % 64) // 8) ^ (row & 7)[:, None]) * 8 + col % 8

    if case["op"] == "write":
        got = {}
        for key, sign in (("local", 1), ("lent", -1)):
            arena = s[key][:s["n_" + key]].double()
            flat = arena.view(-1, C)                               # row (block * 2 + plane) * T + token
            mine = s["slots"] >= 0 if sign > 0 else (s["slots"] < 0) & (s["slots"] > NO_SLOT)
            at = s["slots"][mine] if sign > 0 else ~s["slots"][mine]
            place = stored(at % T)
            for plane, x in ((0, s["k"]), (1, s["v"])):
                rows = (at // T * 2 + plane) * T + at % T
                flat[rows[:, None], place] = x[mine].reshape(-1, C).double()
            got[key] = arena
        return got

    lens, tables = s["lens"].tolist(), s["tables"].tolist()
    outs, lses = [], []
    for i, n in enumerate(lens):
        lo = max(0, n - case["window"]) if case.get("window") else 0
        if n <= lo:
            outs.append(torch.zeros((Hkv * case["G"], D), device="cuda", dtype=torch.float64))
            lses.append(torch.full((Hkv * case["G"],), -math.inf, device="cuda", dtype=torch.float64))
            continue
        p = torch.arange(lo, n, device="cuda")
        e = torch.tensor(tables[i], device="cuda")[p // T]
        place = stored(p % T)
        kv = []
        for plane in (0, 1):
            x = torch.empty((n - lo, C), device="cuda", dtype=torch.float64)
            for m, arena, ids in ((e >= 0, s["local"], e), (e < 0, s["lent"], ~e)):
                x[m] = arena[ids[m], plane, (p % T)[m]].reshape(-1, C).gather(1, place[m]).double()
            kv.append(x.view(-1, Hkv, D).transpose(0, 1))          # [Hkv][tokens][D]
        k, v = kv
        if case["op"] == "decode":
            q = s["q"][i].double().reshape(Hkv, case["G"], D)
            z = q @ k.transpose(1, 2) * s["scale"]
            outs.append((torch.softmax(z, -1) @ v).reshape(-1, D))
            lses.append(torch.logsumexp(z, -1).reshape(-1))
            continue
        q = s["q"][i].double().reshape(Hkv * case["G"], 2, D // 2)
        maps = []
        for m in (0, 1):
            z = q[:, m].reshape(Hkv, case["G"], D // 2) @ k[:, :, m * (D // 2):(m + 1) * (D // 2)].transpose(1, 2) * s["scale"]
            maps.append((torch.softmax(z, -1) @ v).reshape(-1, D))
        o = maps[0] - s["lam"].double()[:, None] * maps[1]
        if s["weight"] is not None:
            o = o / torch.sqrt((o * o).mean(-1, keepdim=True) + s["eps"]) * s["weight"].double()
        outs.append(o * s["out_scale"])
    out = torch.stack(outs)
    return {"out": out, "lse": torch.stack(lses)} if case["op"] == "decode" else {"out": out}
