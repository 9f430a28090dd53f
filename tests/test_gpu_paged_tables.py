"""Block tables and slot maps built on the GPU, and rows written through them, against plain models."""
import numpy as np
import pytest
import torch

from paper_2609_27040_b200 import binding as B
from paper_2609_27040_b200 import build as build_mod
from tests.paged_helpers import NO_SLOT, PoolModel, ceil_div, stored_place

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def gpu(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


class Bench:
    """A pool and its tables on the device beside the model."""

    def __init__(self, n, T, width, blocks0, blocks1, seed, extra=0):
        rng = np.random.default_rng(seed)
        ids0, ids1 = rng.permutation(blocks0).tolist(), rng.permutation(blocks1).tolist()
        self.n, self.T, self.width = n, T, width
        self.model = PoolModel(ids0, ids1)
        self.model.width = width
        self.rows = [{} for _ in range(n)]
        pad = lambda x: gpu(x + [-7] * extra) if x or extra else None   # noqa: E731
        self.ids = [pad(ids0), pad(ids1)]
        self.free = gpu([blocks0, blocks1])
        self.work = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.tables = torch.full((n, width + 3), -99, dtype=torch.int32, device="cuda")[:, :width]     # rows further apart than they are long
        self.status = gpu([0])
        self.lens = [0] * n

    def pool(self, free_out=None):
        return B.PagedPool(self.ids[0], self.ids[1], self.free, self.free if free_out is None else free_out, self.work)

    def call(self, new_lens, max_tokens, stream=None):
        self.offsets = torch.full((self.n + 1,), -5, dtype=torch.int32, device="cuda")
        self.slots = torch.full((max_tokens,), 5, dtype=torch.int64, device="cuda")
        self.positions = torch.full((max_tokens,), 5, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        assert B.paged_build_tables(self.pool(), gpu(self.lens), gpu(new_lens), self.T, self.tables, self.offsets, self.slots,
                                    self.positions, self.status, stream) == B.OK
        torch.cuda.synchronize()

    def step(self, new_lens, max_tokens):
        self.call(new_lens, max_tokens)
        status, offsets, slots, positions = self.model.step(self.T, self.lens, new_lens, self.rows, max_tokens)
        assert int(self.status) == status
        assert self.offsets.tolist() == offsets
        assert self.slots.tolist() == slots
        assert self.positions.tolist() == positions
        self.same_state()
        if status == 0:
            self.lens = list(new_lens)
        self.status.zero_()
        return status

    def same_state(self):
        free = self.free.tolist()
        assert free == [len(s) for s in self.model.stacks]
        for j in (0, 1):
            if self.ids[j] is not None:
                assert self.ids[j][:free[j]].tolist() == self.model.stacks[j]
        want = np.full((self.n, self.width), -99)
        for i, row in enumerate(self.rows):
            for j, e in row.items():
                want[i, j] = e
        assert (self.tables.cpu().numpy() == want).all()
        assert int(self.work) == 0


@pytest.mark.parametrize("n,T,hi,blocks0,blocks1", [
    (1, 16, 40, 3, 0), (1, 64, 64, 0, 1), (5, 16, 100, 10, 30), (33, 32, 700, 200, 600), (512, 16, 60, 900, 2000),
    (513, 16, 60, 3000, 1), (700, 64, 300, 5, 4000), (2500, 16, 50, 5000, 6000), (40, 16, 3000, 500, 8000)])
def test_random_walks_follow_the_model(n, T, hi, blocks0, blocks1):
    rng = np.random.default_rng(n * 7 + T)
    b = Bench(n, T, ceil_div(hi, T) + 1, blocks0, blocks1, n)
    seen = set()
    for k in range(8):
        kind = k % 4
        old = np.array(b.lens)
        if kind == 0:                                            # prompts of all requests that hold nothing, some stay empty
            new = np.where((old == 0) & (rng.random(n) < 0.8), rng.integers(0, hi + 1, n), old)
        elif kind == 1:                                          # one token each, as far as there is room
            new = np.minimum(old + 1, hi)
        elif kind == 2:                                          # some finish, some fall back, some grow
            new = np.where(rng.random(n) < 0.3, 0, np.where(rng.random(n) < 0.5, rng.integers(0, hi + 1, n), old))
        else:
            new = np.where(rng.random(n) < 0.5, rng.integers(0, hi + 1, n), old)
        total = int(np.maximum(new - old, 0).sum())
        seen.add(b.step(new.tolist(), total + int(rng.integers(0, 70)) if k % 3 else max(total, 1)))
    assert 0 in seen


def test_growth_taken_back_restores_the_stacks_exactly():
    b = Bench(90, 16, 30, 200, 900, 3)
    rng = np.random.default_rng(1)
    b.step(rng.integers(0, 200, 90).tolist(), 40000)
    ids = [x.clone() for x in b.ids]
    free, lens = b.free.clone(), list(b.lens)
    b.step([x + int(rng.integers(0, 200)) for x in lens], 40000)
    b.step(lens, 1)
    assert (b.free == free).all() and all((x == y).all() for x, y in zip(ids, b.ids))


@pytest.mark.parametrize("what", ["no space", "no space by one", "too many tokens", "too long", "below zero", "old too long", "top"])
def test_refused_steps_change_nothing(what):
    b = Bench(20, 16, 10, 30, 40, 5)
    assert b.step([50] * 10 + [0] * 10, 500) == 0                 # 40 of 70 blocks
    new, tokens = list(b.lens), 400
    if what == "no space":
        new = [160] * 20
        tokens = 5000
    elif what == "no space by one":
        new[10:] = [48] * 10                                      # 30 more: exactly what is left
        new[0] = 65                                               # and one
        tokens = 5000
    elif what == "too many tokens":
        new[0], tokens = 61, 10
    elif what == "too long":
        new[3] = 161
    elif what == "below zero":
        new[3] = -1
    elif what == "old too long":
        b.lens[15] = 161
    before = [t.clone() for t in (b.tables, b.ids[0], b.ids[1], b.free)]
    if what == "top":
        b.free[0] = 31
        b.call(new, tokens)
        assert int(b.status) == B.EINVAL and b.free.tolist()[0] == 31
        b.free.copy_(before[3])
        assert (b.slots == NO_SLOT).all() and (b.positions == -1).all() and (b.offsets == 0).all()
    else:
        assert b.step(new, tokens) == (B.ENOSPC if "space" in what else B.EINVAL)
    assert all((x == y).all() for x, y in zip(before, (b.tables, b.ids[0], b.ids[1], b.free)))


def test_exactly_all_blocks_and_no_requests():
    b = Bench(3, 16, 4, 4, 3, 2)
    assert b.step([64, 33, 0], 97) == 0 and b.free.tolist() == [0, 0]
    assert b.step([64, 33, 0], 1) == 0
    assert b.step([64, 33, 1], 5) == B.ENOSPC
    assert b.step([0, 0, 0], 1) == 0 and b.free.tolist() == [4, 3]
    empty = Bench(0, 16, 1, 2, 2, 2)
    empty.call([], 70)
    assert empty.offsets.tolist() == [0] and (empty.slots == NO_SLOT).all() and empty.free.tolist() == [2, 2]


def test_pushes_beyond_a_stacks_capacity_are_dropped_and_reported():
    b = Bench(1, 16, 8, 3, 0, 2)
    b.tables[0, :8] = torch.arange(100, 108, dtype=torch.int32)   # blocks that never came from this pool
    b.lens = [128]
    b.call([0], 1)
    assert int(b.status) == B.EINVAL and b.free.tolist() == [3, 0] and int(b.work) == 0


def test_a_separate_count_leaves_the_first_one():
    b = Bench(4, 16, 8, 20, 20, 2)
    out = gpu([-1, -1])
    args = (gpu([0] * 4), gpu([17, 0, 64, 1]), 16, b.tables, gpu([0] * 5), torch.zeros(90, dtype=torch.int64, device="cuda"),
            torch.zeros(90, dtype=torch.int32, device="cuda"))
    for _ in range(2):                                            # the same call again gives the same answer
        assert B.paged_build_tables(b.pool(out), *args) == B.OK
        torch.cuda.synchronize()
        assert b.free.tolist() == [20, 20] and out.tolist() == [13, 20]


def test_a_captured_step_follows_new_lengths():
    """One graph of a build call, replayed with other lengths in the same buffers; many CTAs (large token room)."""
    n, T, room = 300, 16, 30000
    b = Bench(n, T, 20, 2000, 4000, 9)
    lens, new = gpu([0] * n), gpu([0] * n)
    offsets, slots = gpu([0] * (n + 1)), torch.zeros(room, dtype=torch.int64, device="cuda")
    positions, status = gpu([0] * room), gpu([0])
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    pool = b.pool()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            assert B.paged_build_tables(pool, lens, new, T, b.tables, offsets, slots, positions, status, torch.cuda.current_stream()) == B.OK
    rng = np.random.default_rng(4)
    for k in range(12):
        old = b.lens
        want = [int(x) for x in (rng.integers(0, 100, n) if k % 3 == 0 else np.minimum(np.array(old) + 1, 300) if k % 3 == 1
                                 else np.where(rng.random(n) < 0.4, 0, np.minimum(np.array(old) + rng.integers(0, 40, n), 300)))]
        lens.copy_(gpu(old))
        new.copy_(gpu(want))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        st, o, sl, po = b.model.step(T, old, want, b.rows, room)
        assert (int(status), offsets.tolist(), slots.tolist(), positions.tolist()) == (st, o, sl, po)
        b.same_state()
        b.lens = want


# -- rows through the slot map -------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hkv,D,T,n", [(8, 128, 16, 250), (1, 64, 64, 33), (3, 64, 16, 1), (2, 64, 32, 77), (10, 256, 32, 40), (5, 128, 16, 601)])
def test_rows_land_in_their_slots(dtype, Hkv, D, T, n):
    rng = np.random.default_rng(Hkv * D + n)
    blocks = [ceil_div(n, T) + 2, ceil_div(n, T) + 1]
    gen = torch.Generator(device="cuda").manual_seed(n)
    arenas = [torch.randn((b, 3, T, Hkv, D), device="cuda", generator=gen).to(dtype)[:, :2] for b in blocks]   # blocks apart from one another
    fused = torch.randn((n, 4 * Hkv, D), device="cuda", generator=gen).to(dtype)
    k, v = fused[:, Hkv:2 * Hkv], fused[:, 3 * Hkv:]
    slots = rng.permutation(np.concatenate([np.arange(blocks[0] * T), ~np.arange(blocks[1] * T)]))[:n]
    slots[rng.random(n) < 0.1] = NO_SLOT
    want = [a.clone() for a in arenas]
    for t in range(n):
        s = int(slots[t])
        if s == NO_SLOT:
            continue
        a, s = (0, s) if s >= 0 else (1, ~s)
        place = torch.from_numpy(stored_place(s % T, Hkv * D)).cuda()
        for plane, x in ((0, k), (1, v)):
            row = torch.empty(Hkv * D, dtype=dtype, device="cuda")
            row[place] = x[t].reshape(-1)
            want[a][s // T, plane, s % T] = row.view(Hkv, D)
    cache = B.PagedCache(arenas[0], arenas[1])
    status = gpu([0])
    torch.cuda.synchronize()
    assert B.paged_write_kv(cache, k, v, gpu(slots.tolist(), torch.int64), status) == B.OK
    torch.cuda.synchronize()
    assert int(status) == 0
    for a, w in zip(arenas, want):
        assert torch.equal(a.contiguous().view(torch.int16), w.contiguous().view(torch.int16))
    if D == 128 and T == 16:                                      # and what the format's own converter says
        canonical = [B.kv_block_swizzle(a.contiguous().view(torch.int16)).view(dtype) for a in arenas]
        for t in range(n):
            s = int(slots[t])
            if s != NO_SLOT:
                a, s = (0, s) if s >= 0 else (1, ~s)
                assert torch.equal(canonical[a][s // T, 0, s % T], k[t]) and torch.equal(canonical[a][s // T, 1, s % T], v[t])


def test_slots_outside_the_cache_are_skipped_and_reported():
    arenas = [torch.zeros((3, 2, 16, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    guard = [torch.zeros_like(a) for a in arenas]
    k = torch.ones((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    status = gpu([0])
    slots = gpu([48, ~48, (1 << 62), NO_SLOT + 1], torch.int64)
    torch.cuda.synchronize()
    assert B.paged_write_kv(B.PagedCache(*arenas), k, k, slots, status) == B.OK
    torch.cuda.synchronize()
    assert int(status) == B.EINVAL and all(torch.equal(a, g) for a, g in zip(arenas, guard))
    status.zero_()
    assert B.paged_write_kv(B.PagedCache(arenas[0]), k, k, gpu([~0, 5, NO_SLOT, 47], torch.int64), status) == B.OK   # no second arena
    torch.cuda.synchronize()
    assert int(status) == B.EINVAL and float(arenas[0].float().sum()) == 2 * 2 * 2 * 64


def test_tables_and_rows_behind_slow_kernels_and_one_another():
    """Every call waits for what comes before it, eager and captured: inputs are written by a long kernel or a copy right before the
    call, or by a call that lets its successor start early (slots by the tables, rows by attention), and are overwritten right behind it."""
    n, T, Hkv, D, width = 150, 16, 4, 128, 12
    rng = np.random.default_rng(3)
    gen = torch.Generator(device="cuda").manual_seed(3)
    old, new = rng.integers(0, 90, n), rng.integers(90, 180, n)
    room = int((new - old).sum()) + 9
    blocks = int((-(-new // T)).sum())
    bf, i32 = torch.bfloat16, torch.int32
    arena = torch.zeros((blocks + 5, 2, T, Hkv, D), dtype=bf, device="cuda")
    cache = B.PagedCache(arena)
    held = int((-(-old // T)).sum())
    ids = rng.permutation(blocks + 5)
    first = np.full((n, width), -1)
    first[np.arange(width)[None] < (-(-old // T))[:, None]] = ids[:held]
    first, spare = gpu(first.tolist()), gpu(ids[held:].tolist() + [0] * held)
    olds, news, ks, vs = gpu(old.tolist()), gpu(new.tolist()), *(torch.randn((room, Hkv, D), device="cuda", generator=gen).to(bf) for _ in range(2))
    qs = torch.randn((n, Hkv, D), device="cuda", generator=gen).to(bf)
    lens, want = torch.zeros_like(olds), torch.zeros_like(news)
    tables, stack, free, work, status = first.clone(), spare.clone(), gpu([0, 0]), gpu([0]), gpu([0])
    pool = B.PagedPool(stack, None, free, free, work)
    offsets, slots, positions = torch.zeros(n + 1, dtype=i32, device="cuda"), torch.zeros(room, dtype=torch.int64, device="cuda"), torch.zeros(room, dtype=i32, device="cuda")
    k, v, q, out = torch.zeros_like(ks), torch.zeros_like(vs), torch.zeros_like(qs), torch.zeros_like(qs)
    ws = torch.zeros(B.paged_decode_workspace(cache, Hkv), dtype=torch.uint8, device="cuda")
    last = gpu([0], torch.int64).expand(n).contiguous()
    big = torch.ones(100_000_000, device="cuda")                 # a kernel of some 0.1 ms on it
    results = [torch.zeros_like(x) for x in (tables, slots, positions, offsets, free, arena, out, arena)]

    def step():
        s = torch.cuda.current_stream()
        arena.zero_()
        tables.copy_(first)
        stack.copy_(spare)
        lens.fill_(-1)                                           # what a call that came too soon would see: refused
        want.fill_(-1)
        slots.fill_(1 << 40)
        free.copy_(torch_free)
        big.mul_(1.0)
        lens.copy_(olds)
        want.copy_(news)
        assert B.paged_build_tables(pool, lens, want, T, tables, offsets, slots, positions, status, s) == B.OK
        lens.fill_(-1)
        want.fill_(-1)
        k.fill_(9.0)
        v.fill_(9.0)
        big.mul_(1.0)
        k.copy_(ks)
        v.copy_(vs)
        assert B.paged_write_kv(cache, k, v, slots, status, s) == B.OK
        k.fill_(9.0)
        v.fill_(9.0)
        for r, x in zip(results[:6], (tables, slots, positions, offsets, free, arena)):
            r.copy_(x)
        # tables, rows, attention and rows again, back to back: each reads what the one before it writes
        arena.zero_()
        tables.copy_(first)
        free.copy_(torch_free)
        lens.copy_(olds)
        want.copy_(news)
        k.copy_(ks)
        v.copy_(vs)
        q.copy_(qs)
        assert B.paged_build_tables(pool, lens, want, T, tables, offsets, slots, positions, status, s) == B.OK
        assert B.paged_write_kv(cache, k, v, slots, status, s) == B.OK
        assert B.paged_decode_tables(cache, tables, want, q, 0.1, out, ws, status=status, stream=s) == B.OK
        assert B.paged_write_kv(cache, out, out, last, status, s) == B.OK
        results[6].copy_(out)
        results[7].copy_(arena)
        out.fill_(5.0)

    torch_free = gpu([len(ids) - held, 0])
    model = PoolModel(ids[held:].tolist(), [])
    model.width = width
    rows = [dict(enumerate(first[i, :ceil_div(int(old[i]), T)].tolist())) for i in range(n)]
    st, o, sl, po = model.step(T, old.tolist(), new.tolist(), rows, room)
    last.copy_(gpu([int(sl[o[i + 1] - 1]) for i in range(n)], torch.int64))   # each request's last token, distinct
    main = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(main):
        step()
    torch.cuda.synchronize()
    assert st == 0 and int(status) == 0
    assert results[3].tolist() == o and results[1].tolist() == sl and results[2].tolist() == po and results[4].tolist() == [len(model.stacks[0]), 0]
    at = np.array(sl[:o[n]])
    place = torch.from_numpy(np.stack([stored_place(r, Hkv * D) for r in range(T)])).cuda()

    def rows_at(x, where):
        where = torch.from_numpy(np.asarray(where)).cuda()
        return x[where // T, :, where % T].reshape(-1, 2, Hkv * D).gather(2, place[where % T][:, None].expand(-1, 2, -1)).reshape(-1, 2, Hkv, D)

    for j, x in enumerate((ks, vs)):
        assert torch.equal(rows_at(results[5], at)[:, j], x[:o[n]])
        assert torch.equal(rows_at(results[7], last.cpu().numpy())[:, j], results[6])
    assert results[6].any()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        step()
    good = [r.clone() for r in results]
    for rep in range(6):
        for r in results:
            r.fill_(3)
        torch.cuda.synchronize()
        if rep % 2:
            with torch.cuda.stream(main):
                step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, good)) and int(status) == 0 and int(work) == 0


def test_a_call_that_could_not_be_launched_leaves_no_error_to_the_next_one():
    """A stream whose capture has become invalid takes no launch: the call says so, and what the library launches next does not."""
    import ctypes as C
    arena = torch.zeros((3, 2, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    cache, k, slots = B.PagedCache(arena), torch.ones((1, 2, 64), dtype=torch.bfloat16, device="cuda"), gpu([5], torch.int64)
    tables, lens, q = gpu([[0, 1, 2]]), gpu([20]), torch.ones((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    ws, out = torch.zeros(B.paged_decode_workspace(cache, 4), dtype=torch.uint8, device="cuda"), torch.zeros_like(q)
    b = Bench(1, 16, 4, 3, 0, 1)
    args = (gpu([0]), gpu([17]), 16, b.tables, gpu([0, 0]), torch.zeros(17, dtype=torch.int64, device="cuda"), gpu([0] * 17))
    src, dst = torch.arange(64, dtype=torch.int32, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    driver, stream = C.CDLL("libcuda.so.1"), C.c_void_p()

    def calls(s):
        yield B.paged_write_kv(cache, k, k, slots, stream=s)
        yield B.paged_decode_tables(cache, tables, lens, q, 0.1, out, ws, stream=s)
        yield B.paged_decode_diff(cache, tables, lens, q.view(1, 4, 32), torch.ones(2, device="cuda"), 0.1, out, ws, stream=s)
        yield B.paged_build_tables(b.pool(), *args, stream=s)

    assert driver.cuStreamCreate(C.byref(stream), 1) == 0
    try:
        for which in range(4):
            assert driver.cuStreamBeginCapture_v2(stream, 2) == 0
            assert driver.cuStreamSynchronize(stream) != 0       # not allowed there: the capture is invalid
            for i, rc in enumerate(calls(stream.value)):
                if i == which:
                    assert rc == B.ECUDA
                    break
            graph = C.c_void_p()
            assert driver.cuStreamEndCapture(stream, C.byref(graph)) != 0
            dst.zero_()
            torch.cuda.synchronize()
            assert B.lib().slice_copy_blocks(dst.data_ptr(), None, src.data_ptr(), None, 1, 256, 1, 1, None) == B.OK
            torch.cuda.synchronize()
            assert torch.equal(src, dst)
    finally:
        driver.cuStreamDestroy_v2(stream)
    assert [rc for rc in calls(None)] == [B.OK] * 4
    torch.cuda.synchronize()


class Guarded:
    """Arrays that lie in larger ones: what is before and behind them has to stay as it is."""

    def __init__(self):
        self.all = []

    def __call__(self, values, dtype=torch.int32, before=4, behind=600):
        big = torch.full((before + len(values) + behind,), 0x5a5a5a, dtype=dtype, device="cuda")
        part = big[before:before + len(values)]
        part.copy_(gpu(values, dtype))
        self.all.append((big, before, len(values), behind))
        return part

    def untouched(self):
        return all((big[:a] == 0x5a5a5a).all() and (big[a + n:] == 0x5a5a5a).all() for big, a, n, _ in self.all)


@pytest.mark.parametrize("n,T,hi,room,capacity", [
    (1, 16, 128, 1, (3, 2)),                                      # one request gives back more than there is room for
    (7, 16, 100, 333, (9, 5)),
    (40, 32, 900, 2049, (50, 700)),                               # more than one CTA; more blocks than threads come back
    (700, 64, 300, 4097, (1, 800)),
    (300, 16, 200, 60001, (2600, 1)),
    (2100, 16, 40, 2048, (4000, 2000))])                          # more requests than a step lists
def test_nothing_is_written_outside_the_arrays(n, T, hi, room, capacity):
    """Requests grow, and others give back blocks that never came from this pool: those that the stacks have no room for are dropped."""
    rng = np.random.default_rng(n + room)
    width = ceil_div(hi, T)
    guard = Guarded()
    lens = rng.integers(0, hi + 1, n)
    lens[0] = hi
    model = PoolModel(rng.integers(0, 1000, capacity[0] * 2 // 3).tolist(), rng.integers(0, 1000, capacity[1] * 2 // 3).tolist(), capacity)
    model.width = width
    seen = set()
    for kind in ("back", "all back", "grow"):
        if kind == "grow":                                        # as far as the free blocks and the room go
            lens = np.zeros(n, np.int64)
            free = sum(map(len, model.stacks))
            new = np.minimum(rng.integers(0, hi + 1, n), (free // n) * T)
            new[np.cumsum(new) > room] = 0
        else:
            new = np.where(rng.random(n) < 0.5, lens // 3, lens) if kind == "back" else lens * 0
            new[0] = 0
        rows = [{j: int(rng.integers(0, 1000)) if rng.random() < 0.6 else ~int(rng.integers(0, 1000)) for j in range(ceil_div(int(x), T))} for x in lens]
        cells = np.full((n, width + 2), 0x5a5a5a)
        for i, row in enumerate(rows):
            for j, e in row.items():
                cells[i, j] = e
        tables = guard(cells.reshape(-1).tolist())
        tables2 = tables.view(n, width + 2)[:, :width]
        ids = [guard(s + [-7] * (c - len(s))) for s, c in zip(model.stacks, capacity)]
        free, out, work, status = guard([len(s) for s in model.stacks]), guard([-1, -1]), guard([0]), guard([0])
        offsets, slots, positions = guard([-5] * (n + 1)), guard([5] * room, torch.int64), guard([5] * room)
        before = [x.tolist() for x in ids]
        for pool_out in (out, free):
            status.zero_()
            pool = B.PagedPool(ids[0], ids[1], free, pool_out, work)
            a, b = gpu(lens.tolist()), gpu(new.tolist())
            torch.cuda.synchronize()
            if pool_out is free:                                  # again, from the same state
                tables.copy_(gpu(cells.reshape(-1).tolist()))
                for x, y in zip(ids, before):
                    x.copy_(gpu(y))
            assert B.paged_build_tables(pool, a, b, T, tables2, offsets, slots, positions, status) == B.OK
            torch.cuda.synchronize()
            if pool_out is out:
                st, o, sl, po = model.step(T, lens.tolist(), new.tolist(), rows, room)
                seen.add(st)
            assert (int(status), offsets.tolist(), slots.tolist(), positions.tolist(), int(work)) == (st, o, sl, po, 0)
            assert pool_out.tolist() == [len(s) for s in model.stacks]
            for x, s, y in zip(ids, model.stacks, before):
                assert x[:len(s)].tolist() == s and x[len(s):].tolist() == y[len(s):]
            want = cells.copy()
            for i, row in enumerate(rows):
                for j, e in row.items():
                    want[i, j] = e
            assert (tables.cpu().numpy().reshape(n, width + 2) == want).all()
            assert guard.untouched()
        lens = new
    assert seen == {0, B.EINVAL}


def test_a_pool_with_room_to_spare():
    """Stacks whose capacity is above their blocks: the cells behind the tops are left alone."""
    b = Bench(30, 16, 9, 60, 80, 4, extra=50)
    rng = np.random.default_rng(8)
    for _ in range(6):
        assert b.step(rng.integers(0, 80, 30).tolist(), 3000) in (0, B.ENOSPC)
        assert all((x[-50:] == -7).all() for x in b.ids)


def test_rows_that_are_not_written_keep_what_they_hold():
    """Every row of the arenas that no slot names, and what lies behind them."""
    Hkv, D, T, blocks = 3, 64, 16, 5
    gen = torch.Generator(device="cuda").manual_seed(1)
    size = 2 * T * Hkv * D
    bigs = [torch.randn(size * (blocks + 2), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2)]
    before = [x.clone() for x in bigs]
    arenas = [x[size:-size].view(blocks, 2, T, Hkv, D) for x in bigs]
    k, v = (torch.randn((2, Hkv, D), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    slots = gpu([blocks * T - 1, ~0], torch.int64)
    torch.cuda.synchronize()
    assert B.paged_write_kv(B.PagedCache(*arenas), k, v, slots) == B.OK
    torch.cuda.synchronize()
    for x, y, block, row in zip(bigs, before, (blocks, 1), (T - 1, 0)):
        for plane in range(2):
            at = block * size + (plane * T + row) * Hkv * D
            assert not torch.equal(x[at:at + Hkv * D], y[at:at + Hkv * D])
            y[at:at + Hkv * D] = x[at:at + Hkv * D]
        assert torch.equal(x, y)
