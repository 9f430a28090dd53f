"""Shared blocks (forks, freed blocks, compaction), copies of blocks and accepted rows, against models stated one block at a time."""
import numpy as np
import pytest
import torch

from paper_2609_27040_b200 import binding as B
from paper_2609_27040_b200 import build as build_mod
from tests.paged_helpers import ceil_div, logical_rows, stored_place

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
EINVAL, ENOSPC = -1, -2


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def gpu(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


class World:
    """Requests over two arenas on the device, and the same as lists: stacks, one list of entries per request, holders of every entry."""

    def __init__(self, n, T, width, blocks, seed=0, room=None):
        self.rng = np.random.default_rng(seed)
        self.n, self.T, self.width, self.blocks = n, T, width, blocks
        self.stacks = [self.rng.permutation(b).tolist() for b in blocks]
        self.rows = [[] for _ in range(n)]
        self.lens = [0] * n
        self.ids = [gpu(s + [-3] * ((room or 0))) if s else None for s in self.stacks]
        self.free = gpu([len(s) for s in self.stacks])
        self.refs = [torch.zeros(b, dtype=torch.int32, device="cuda") if b else None for b in blocks]
        self.tables = torch.full((n, width + 3), -99, dtype=torch.int32, device="cuda")[:, :width]
        self.pool_work = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.share_work = torch.zeros(B.paged_shares_workspace(*blocks), dtype=torch.uint8, device="cuda")
        self.status = gpu([0])
        self.pool = B.PagedPool(self.ids[0], self.ids[1], self.free, self.free, self.pool_work)
        self.shares = B.PagedShares(self.refs[0], self.refs[1], self.share_work)
        self.held_lens = torch.zeros(n, dtype=torch.int32, device="cuda")

    def pop(self):
        return self.stacks[0].pop() if self.stacks[0] else ~self.stacks[1].pop()

    def holders(self):
        h = {}
        for row in self.rows:
            for e in row:
                h[e] = h.get(e, 0) + 1
        return h

    def grow(self, new_lens):
        room = sum(max(0, b - a) for a, b in zip(self.lens, new_lens))
        i32 = dict(dtype=torch.int32, device="cuda")
        target = gpu(new_lens)
        assert B.paged_build_tables(self.pool, self.held_lens, target, self.T, self.tables, torch.zeros(self.n + 1, **i32),
                                    torch.zeros(max(room, 1), dtype=torch.int64, device="cuda"), torch.zeros(max(room, 1), **i32), self.status) == B.OK
        torch.cuda.synchronize()
        for i, x in enumerate(new_lens):
            while len(self.rows[i]) < ceil_div(x, self.T):
                self.rows[i].append(self.pop())
        self.lens = list(new_lens)
        self.held_lens.copy_(target)

    def fork(self, src, dst, status=0, stream=None, apart=False):
        copies = torch.full((len(src), 3), -7, dtype=torch.int32, device="cuda")
        new_lens = self.held_lens.clone() if apart else self.held_lens
        torch.cuda.synchronize()
        assert B.paged_fork(self.pool, self.shares, self.held_lens, new_lens, gpu(src), gpu(dst), self.T, self.tables, copies, self.status,
                            stream) == B.OK
        torch.cuda.synchronize()
        assert int(self.status) == status
        want = [(0, 0, 0)] * len(src)
        if status == 0:
            for f, (s, d) in enumerate(zip(src, dst)):
                if d < 0:
                    continue
                whole, tail = divmod(self.lens[s], self.T)
                self.rows[d] = self.rows[s][:whole]
                if tail:
                    self.rows[d].append(self.pop())
                    want[f] = (self.rows[s][whole], self.rows[d][-1], tail)
                self.lens[d] = self.lens[s]
        assert [tuple(x) for x in copies.tolist()] == want
        if apart:
            assert self.held_lens.tolist() != self.lens or not any(d >= 0 and self.lens[d] for d in dst) or status
            self.held_lens.copy_(new_lens)
        return want

    def release(self, new_lens, status=0, stream=None):
        torch.cuda.synchronize()
        target = gpu(new_lens)
        assert B.paged_free(self.pool, self.shares, self.held_lens, target, self.T, self.tables, self.status, stream) == B.OK
        torch.cuda.synchronize()
        assert int(self.status) == status
        if status == 0:
            before = set(self.holders())
            for i, x in enumerate(new_lens):
                if x < self.lens[i]:
                    self.rows[i] = self.rows[i][:ceil_div(x, self.T)]
                    self.lens[i] = x
            gone = before - set(self.holders())
            self.stacks[0] += sorted((e for e in gone if e >= 0), reverse=True)
            self.stacks[1] += sorted((~e for e in gone if e < 0), reverse=True)
            self.held_lens.copy_(gpu(self.lens))

    def compact(self, limits, max_copies=None, status=0, stream=None):
        held = self.holders()
        copies = torch.full((len(held) + 2 if max_copies is None else max_copies, 3), -7, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        assert B.paged_compact(self.pool, self.shares, gpu(limits), self.held_lens, self.T, self.tables, copies, self.status, stream) == B.OK
        torch.cuda.synchronize()
        assert int(self.status) == status
        moves = []
        if status == 0:
            old = sorted(e for e in held if e >= limits[0]) + [~x for x in sorted(~e for e in held if e < 0 and ~e >= limits[1])]
            self.stacks = [[x for x in s if x < limits[a]] for a, s in enumerate(self.stacks)]
            moves = [(e, self.pop(), self.T) for e in old]
            to = {a: b for a, b, _ in moves}
            self.rows = [[to.get(e, e) for e in row] for row in self.rows]
        assert [tuple(x) for x in copies.tolist()] == moves + [(0, 0, 0)] * (copies.shape[0] - len(moves))
        return moves

    def same(self):
        assert self.free.tolist() == [len(s) for s in self.stacks]
        for a in (0, 1):
            if self.ids[a] is not None:
                assert self.ids[a].tolist()[:len(self.stacks[a])] == self.stacks[a]
        t = self.tables.tolist()
        for i, row in enumerate(self.rows):
            assert t[i][:len(row)] == row, i
        held = self.holders()
        for a in (0, 1):
            if self.refs[a] is not None:
                assert self.refs[a].tolist() == [max(0, held.get(~b if a else b, 0) - 1) for b in range(self.blocks[a])]
        assert self.held_lens.tolist() == self.lens
        assert int(self.pool_work) == 0
        bits = 4 * (sum(ceil_div(b, 32) for b in self.blocks))
        assert not self.share_work[64:64 + bits].any()
        # nothing is lost: every id is on a stack or held, and not both
        for a in (0, 1):
            mine = {e if a == 0 else ~e for e in held if (e < 0) == bool(a)}
            assert mine.isdisjoint(self.stacks[a]) and len(set(self.stacks[a])) == len(self.stacks[a])


@pytest.mark.parametrize("T,n,width,blocks", [(16, 12, 20, (150, 40)), (32, 5, 9, (0, 60)), (64, 40, 7, (400, 0)), (16, 300, 3, (700, 500))])
def test_runs_of_forks_growth_frees_and_compactions(T, n, width, blocks):
    w = World(n, T, width, blocks, seed=T + n)
    rng = w.rng
    for step in range(25):
        room = len(w.stacks[0]) + len(w.stacks[1])
        what = rng.choice(["grow", "fork", "fork", "free", "compact"])
        if what == "grow":
            # a shared block is whole, so that growth never writes to it
            new = [min(width * T, x + int(rng.integers(0, 2 * T))) if rng.random() < 0.5 else x for x in w.lens]
            while sum(ceil_div(b, T) - ceil_div(a, T) for a, b in zip(w.lens, new)) > room:
                new = [a + (b - a) // 2 for a, b in zip(w.lens, new)]
                if new == w.lens:
                    break
            w.grow(new)
        elif what == "fork":
            empty, full = [i for i in range(n) if w.lens[i] == 0], [i for i in range(n) if w.lens[i]]
            if full and empty:
                k = min(len(empty), int(rng.integers(1, 9)), room)
                dst = rng.permutation(empty)[:k].tolist()
                src = rng.choice(full, k).tolist()
                if rng.random() < 0.5 and k:
                    dst[0] = -1                                  # padding
                w.fork(src, dst, apart=bool(rng.random() < 0.5))
        elif what == "free":
            w.release([0 if rng.random() < 0.3 else x if rng.random() < 0.5 else int(rng.integers(0, x + 1)) if x % T or True else x for x in w.lens])
            # (a request cut inside a block that others hold would share a block that is not full: not from here on)
            held = w.holders()
            w.release([x - x % T if x % T and held[w.rows[i][-1]] > 1 else x for i, x in enumerate(w.lens)])
        else:
            used = [sum(1 for e in w.holders() if (e >= 0) == (a == 0)) for a in (0, 1)]
            free = [len(s) for s in w.stacks]
            limits = [int(rng.integers(0, b + 1)) for b in blocks]
            fits = sum(1 for a in (0, 1) for x in w.stacks[a] if x < limits[a]) >= sum(1 for e in w.holders() if (e if e >= 0 else ~e) >= limits[e < 0])
            if not fits:
                w.compact(limits, status=ENOSPC)
                w.status.zero_()
            else:
                w.compact(limits)
                # the ids come back, so that the run goes on
                for a in (0, 1):
                    back = [x for x in range(limits[a], blocks[a])]
                    w.stacks[a] += back
                    if w.ids[a] is not None:
                        w.ids[a][:len(w.stacks[a])] = gpu(w.stacks[a])
                w.free.copy_(gpu([len(s) for s in w.stacks]))
            assert used and free
        w.same()


def test_a_block_is_freed_by_its_last_holder():
    w = World(6, 16, 8, (30, 0))
    w.grow([100, 0, 0, 0, 0, 0])
    w.fork([0, 0, 0], [1, 2, 3])
    w.same()
    assert w.refs[0].max() == 3
    before = [list(r) for r in w.rows]
    w.release([0, 100, 0, 0, 0, 0])                              # only what the forks had alone comes back
    assert len(w.stacks[0]) == 30 - 7
    w.same()
    w.fork([1, 1], [4, 5])
    w.release([0] * 6)                                           # all holders in one call
    w.same()
    assert sorted(w.stacks[0]) == list(range(30)) and not w.refs[0].any()
    assert before[1][:6] == before[0][:6]


def test_without_sharing_the_ids_are_those_that_build_tables_gives_back():
    a, b = World(9, 16, 30, (200, 100), seed=3), World(9, 16, 30, (200, 100), seed=3)
    lens, less = [400, 17, 0, 480, 16, 33, 100, 5, 300], [0, 17, 0, 100, 1, 0, 400, 0, 290]
    a.grow(lens)
    b.grow(lens)
    a.release(less)
    a.same()
    i32 = dict(dtype=torch.int32, device="cuda")
    assert B.paged_build_tables(b.pool, b.held_lens, gpu([min(x, y) for x, y in zip(lens, less)]), 16, b.tables, torch.zeros(10, **i32),
                                torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, **i32), b.status) == B.OK
    torch.cuda.synchronize()
    for x, y in zip(a.ids, b.ids):
        assert sorted(x.tolist()) == sorted(y.tolist())
    assert a.free.tolist() == b.free.tolist()


def test_more_forks_and_requests_than_threads():
    n = 3000
    w = World(2 * n, 16, 4, (9000, 4000), seed=1)
    w.grow(w.rng.integers(0, 40, n).tolist() + [0] * n)
    w.fork(w.rng.permutation(n).tolist(), (n + w.rng.permutation(n)).tolist())
    w.same()
    w.compact([8000, 2000])
    w.same()
    w.release([0] * (2 * n))
    w.same()


def test_long_rows():
    """More cells than a warp takes at a time."""
    w = World(4, 16, 1000, (2500, 600), seed=2)
    w.grow([15999, 8001, 0, 0])
    w.fork([0, 1], [2, 3])
    w.same()
    w.compact([2400, 100])
    w.same()
    w.release([5000, 0, 15999, 4])
    w.same()


@pytest.mark.parametrize("src,dst", [([0, 0], [2, 2]), ([0, 2], [2, 3]), ([0], [1]), ([4], [2]), ([-1], [2]), ([0], [4]), ([0], [0])])
def test_forks_that_are_refused(src, dst):
    """The same dst twice, a dst that is a src, one that holds tokens, indices out of range: nothing changes."""
    w = World(4, 16, 8, (30, 10))
    w.grow([50, 20, 0, 0])
    tables = w.tables.clone()
    w.fork(src, dst, status=EINVAL)
    w.same()
    assert torch.equal(tables, w.tables)


def test_forks_without_room():
    w = World(4, 16, 8, (5, 1))
    w.grow([50, 17, 0, 0])                                       # six blocks: none is left
    w.fork([0, 1], [2, 3], status=ENOSPC)
    w.same()
    w.status.zero_()
    w.release([48, 17, 0, 0])                                    # whole blocks only: nothing to be popped
    w.fork([0], [2])
    w.same()


def test_lengths_tops_and_limits_out_of_range():
    w = World(3, 16, 8, (30, 10))
    w.grow([50, 20, 0])
    refs = w.refs[0].clone()
    for bad in ([-1, 20, 0], [50, 8 * 16 + 1, 0]):
        w.held_lens.copy_(gpu(bad))
        for call in (lambda: w.release([0, 0, 0], status=EINVAL), lambda: w.fork([0], [2], status=EINVAL), lambda: w.compact([20, 0], status=EINVAL)):
            call()
            w.status.zero_()
            w.held_lens.copy_(gpu(w.lens))
            w.same()
            w.held_lens.copy_(gpu(bad))
    w.held_lens.copy_(gpu(w.lens))
    w.compact([-1, 5], status=EINVAL)
    w.status.zero_()
    w.compact([3, 10], max_copies=1, status=EINVAL)              # more blocks to be moved than copies have room for
    w.status.zero_()
    w.same()
    for bad in ([-1, 10], [31, 10], [3, 11]):
        keep = w.free.clone()
        w.free.copy_(gpu(bad))
        for call in (lambda: w.release([0, 0, 0], status=EINVAL), lambda: w.fork([0], [2], status=EINVAL), lambda: w.compact([20, 0], status=EINVAL)):
            call()
            w.status.zero_()
            assert w.free.tolist() == bad
        w.free.copy_(keep)
    assert torch.equal(refs, w.refs[0])
    w.same()


def test_entries_outside_their_arena():
    w = World(3, 16, 8, (30, 10))
    w.grow([100, 40, 0])
    w.tables[0, 2], w.tables[0, 3] = 30, ~10
    torch.cuda.synchronize()
    assert B.paged_free(w.pool, w.shares, w.held_lens, gpu([0, 40, 0]), 16, w.tables, w.status) == B.OK
    torch.cuda.synchronize()
    assert int(w.status) == EINVAL
    assert w.free.tolist() == [30 - 10 + 5, 10] and not w.refs[0].any()


def test_a_block_that_is_given_up_too_often_is_pushed_once():
    w = World(3, 16, 8, (30, 0))
    w.grow([48, 32, 0])
    w.tables[1, 0] = w.tables[0, 0]                              # nobody has counted this holder
    torch.cuda.synchronize()
    assert B.paged_free(w.pool, w.shares, w.held_lens, gpu([0, 0, 0]), 16, w.tables, w.status) == B.OK
    torch.cuda.synchronize()
    assert int(w.status) == EINVAL
    ids = w.ids[0].tolist()[:int(w.free[0])]
    assert len(set(ids)) == len(ids) == 29 and not w.refs[0].any()


def test_ids_that_a_stack_has_no_room_for_are_dropped():
    w = World(2, 16, 8, (30, 0))
    w.grow([100, 0])
    w.free.copy_(gpu([28, 0]))                                   # seven come back, two fit
    torch.cuda.synchronize()
    assert B.paged_free(w.pool, w.shares, w.held_lens, gpu([0, 0]), 16, w.tables, w.status) == B.OK
    torch.cuda.synchronize()
    assert int(w.status) == EINVAL and w.free.tolist() == [30, 0] and not w.refs[0].any()


def test_ids_beyond_the_limits_and_strange_ones_leave_the_stacks():
    w = World(2, 16, 8, (30, 20))
    w.grow([40, 20])
    w.compact([30, 0])                                           # the lender takes everything: nobody holds any of it
    w.same()
    assert w.stacks[1] == [] and len(w.stacks[0]) == 25
    w.ids[0][3] = 30
    w.stacks[0].pop(3)
    torch.cuda.synchronize()
    copies = torch.zeros((9, 3), dtype=torch.int32, device="cuda")
    assert B.paged_compact(w.pool, w.shares, gpu([30, 20]), w.held_lens, 16, w.tables, copies, w.status) == B.OK
    torch.cuda.synchronize()
    assert int(w.status) == EINVAL and not copies.any()
    w.same()


def test_a_stack_of_nearly_2_to_the_31_ids():
    """Places on a stack are counted without wrapping, in front and at the end of the largest stack that a pool may have."""
    n = 2 ** 31 - 1
    i32 = dict(dtype=torch.int32, device="cuda")
    ids = torch.full((n,), 5, **i32)
    ids[0], ids[n - 2], ids[n - 1] = 1, 2, 0
    free, status = gpu([n, 0]), gpu([0])
    pool = B.PagedPool(ids, None, free, free, torch.zeros(1, **i32))
    shares = B.PagedShares(torch.zeros(6, **i32), None, torch.zeros(B.paged_shares_workspace(6, 0), dtype=torch.uint8, device="cuda"))
    tables, copies = gpu([[4, 3, 0]]), torch.full((3, 3), 7, **i32)
    torch.cuda.synchronize()
    assert B.paged_compact(pool, shares, gpu([4, 0]), gpu([20]), 16, tables, copies, status) == B.OK
    torch.cuda.synchronize()
    assert int(status) == 0 and free.tolist() == [2, 0] and ids[:2].tolist() == [1, 2]
    assert tables.tolist() == [[0, 3, 0]] and copies.tolist() == [[4, 0, 16], [0, 0, 0], [0, 0, 0]]


def test_a_step_of_frees_forks_and_copies_captured_and_replayed():
    """Beams: every replay frees the forks and makes others, from device arrays that change between replays."""
    T, n = 16, 10
    w = World(n, T, 8, (60, 20), seed=5)
    arena = torch.randn((2, 60 + 20, 2, T, 2, 64), device="cuda").to(BF)
    layers = B.PagedLayers([B.PagedCache(arena[i, :60], arena[i, 60:]) for i in range(2)])
    w.grow([90, 33, 0, 0, 0, 0, 0, 0, 0, 0])
    src, dst, left = gpu([0, 1, 0]), gpu([2, 3, 4]), gpu([90, 33] + [0] * 8)
    copies = torch.zeros((3, 3), dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()

    def step():
        assert B.paged_free(w.pool, w.shares, w.held_lens, left, T, w.tables, w.status, s) == B.OK
        with torch.cuda.stream(s):
            w.held_lens.copy_(left)
        assert B.paged_fork(w.pool, w.shares, w.held_lens, w.held_lens, src, dst, T, w.tables, copies, w.status, s) == B.OK
        assert B.paged_copy_blocks(layers, copies, w.status, s) == B.OK

    torch.cuda.synchronize()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for i, d in ((0, 2), (1, 3), (0, 4)):                        # the model follows the first, eager step
        whole, tail = divmod(w.lens[i], T)
        w.rows[d] = w.rows[i][:whole] + ([w.pop()] if tail else [])
        w.lens[d] = w.lens[i]
    w.same()
    for pick in ([(0, 5), (0, 6), (1, 7)], [(1, 2), (0, -1), (1, 9)], [(0, 9), (1, 8), (0, 7)]):
        src.copy_(gpu([a for a, _ in pick]))
        dst.copy_(gpu([b for _, b in pick]))
        before = arena.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert int(w.status) == 0
        gone = set(w.holders()) - {e for r in w.rows[:2] for e in r}
        w.rows[2:], w.lens[2:] = [[] for _ in range(8)], [0] * 8
        w.stacks[0] += sorted((e for e in gone if e >= 0), reverse=True)
        w.stacks[1] += sorted((~e for e in gone if e < 0), reverse=True)
        for i, d in pick:
            if d < 0:
                continue
            whole, tail = divmod(w.lens[i], T)
            w.rows[d] = w.rows[i][:whole] + ([w.pop()] if tail else [])
            w.lens[d] = w.lens[i]
            if tail:
                a, b = (e if e >= 0 else 60 + ~e for e in (w.rows[i][whole], w.rows[d][whole]))
                before[:, b, :, :tail] = before[:, a, :, :tail]
        w.same()
        assert torch.equal(before, arena)


@pytest.mark.parametrize("T,Hkv,D,L,dtype", [(16, 8, 128, 3, BF), (64, 1, 64, 1, HF), (32, 3, 256, 2, BF), (16, 5, 64, 128, HF), (64, 16, 256, 1, BF)])
def test_copies_of_blocks(T, Hkv, D, L, dtype):
    """Any number of rows, both arenas, rows of nothing to copy in between, and nothing else is written."""
    rng = np.random.default_rng(T)
    sizes = (9, 7)
    arena = torch.randint(-30000, 30000, (L, 19, 2, T, Hkv, D), dtype=torch.int16, device="cuda").view(dtype)
    want = arena.view(torch.int16).clone()
    layers = B.PagedLayers([B.PagedCache(arena[i, 1:10], arena[i, 11:18]) for i in range(L)])
    at = lambda e: 1 + e if e >= 0 else 11 + ~e                  # noqa: E731
    entries = rng.permutation(list(range(9)) + [~x for x in range(7)]).tolist()
    rows = [0, 1, T, T - 1, 0, 3, T // 2, 7]
    copies = [(entries[2 * i], entries[2 * i + 1], r) for i, r in enumerate(rows)]
    for a, b, r in copies:
        want[:, at(b), :, :r] = want[:, at(a), :, :r]
    status = gpu([0])
    assert B.paged_copy_blocks(layers, gpu(copies), status) == B.OK
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(arena.view(torch.int16), want)
    for bad in ((sizes[0], 0, 1), (0, ~sizes[1], 1), (0, 1, T + 1), (0, 1, -1)):
        status.zero_()
        assert B.paged_copy_blocks(layers, gpu([bad, (entries[0], entries[0], 2)]), status) == B.OK
        torch.cuda.synchronize()
        assert int(status) == EINVAL and torch.equal(arena.view(torch.int16), want)


def test_many_copies_mostly_empty():
    T, n = 16, 5000
    arena = torch.randn((1, n, 2, T, 1, 64), device="cuda").to(BF)
    want = arena.clone()
    copies = torch.zeros((n // 2, 3), dtype=torch.int32)
    copies[::3] = torch.stack([torch.arange(n // 2), n // 2 + torch.arange(n // 2), torch.full((n // 2,), T)], 1).int()[::3]
    for a, b, r in copies.tolist():
        if r:
            want[:, b] = want[:, a]
    assert B.paged_copy_blocks(B.PagedLayers([B.PagedCache(arena[0])]), copies.cuda()) == B.OK
    torch.cuda.synchronize()
    assert torch.equal(arena, want)


class Rows:
    """Requests with drafted rows in L layers."""

    def __init__(self, lens, m, T, Hkv, D, L, dtype, seed=0, lent=0.4):
        rng = np.random.default_rng(seed)
        self.lens, self.T, self.Hkv, self.D, self.L = lens, T, Hkv, D, L
        nb = [ceil_div(x + m, T) for x in lens]
        count = sum(nb)
        n1 = int(count * lent)
        self.n0 = count - n1 + 1
        self.arena = torch.randint(-30000, 30000, (L, count + 2, 2, T, Hkv, D), dtype=torch.int16, device="cuda").view(dtype)
        ids = rng.permutation(np.concatenate([rng.permutation(self.n0)[:count - n1], ~rng.permutation(n1 + 1)[:n1]]))
        self.table = np.full((len(lens), max(nb) + 1), 0x7fffffff)
        at = 0
        for i, k in enumerate(nb):
            self.table[i, :k] = ids[at:at + k]
            at += k
        self.tables = gpu(self.table.tolist())
        self.layers = B.PagedLayers([B.PagedCache(self.arena[i, :self.n0], self.arena[i, self.n0:]) for i in range(L)])
        self.status = gpu([0])

    def place(self, i, p):
        e = int(self.table[i, p // self.T])
        return (e if e >= 0 else self.n0 + ~e), p % self.T

    def expected(self, keep):
        want, now = self.arena.view(torch.int16).clone(), self.arena.view(torch.int16)
        C = self.Hkv * self.D
        for i, ks in enumerate(keep):
            for j, k in enumerate(ks):
                (a, r), (b, t) = self.place(i, self.lens[i] + k), self.place(i, self.lens[i] + j)
                src = now[:, a, :, r].reshape(self.L, 2, C)[..., torch.from_numpy(stored_place(r, C)).cuda()]
                out = torch.empty_like(src)
                out[..., torch.from_numpy(stored_place(t, C)).cuda()] = src
                want[:, b, :, t] = out.view(self.L, 2, self.Hkv, self.D)
        return want

    def call(self, keep, width, status=0, stream=None):
        k = torch.full((len(keep), width + 2), -9, dtype=torch.int32, device="cuda")[:, :width]
        for i, ks in enumerate(keep):
            if ks:
                k[i, :min(len(ks), width)] = gpu(ks[:width])
        torch.cuda.synchronize()
        assert B.paged_keep_rows(self.layers, self.tables, gpu(self.lens), k, gpu([len(ks) for ks in keep]), self.status, stream) == B.OK
        torch.cuda.synchronize()
        assert int(self.status) == status


@pytest.mark.parametrize("T,Hkv,D,L,dtype", [(16, 8, 128, 2, BF), (64, 1, 64, 5, HF), (32, 3, 256, 1, BF), (16, 3, 64, 128, BF), (64, 40, 256, 1, HF)])
def test_accepted_rows(T, Hkv, D, L, dtype):
    rng = np.random.default_rng(L)
    r = Rows([0, 5, T - 1, T, 100, 33], 40, T, Hkv, D, L, dtype, seed=T)
    keep = [sorted(rng.permutation(40)[:k].tolist()) for k in (1, 0, 9, 40, 17, 6)]
    keep[5] = [34, 35, 36, 37, 38, 39]
    want = r.expected(keep)
    r.call(keep, 40)
    assert torch.equal(r.arena.view(torch.int16), want)


def test_long_lists_of_accepted_rows():
    """More than a stage of them, rows that are read long after rows before them have been written."""
    rng = np.random.default_rng(1)
    r = Rows([7, 100], 900, 16, 2, 64, 2, BF)
    keep = [sorted(rng.permutation(900)[:400].tolist()), list(range(1, 900))]
    want = r.expected(keep)
    r.call(keep, 899)
    assert torch.equal(r.arena.view(torch.int16), want)


@pytest.mark.parametrize("bad", [[3, 3], [4, 2], [-1, 2], [2, 10 ** 6], [0, 1, 2, 3, 4]])
def test_lists_that_are_refused(bad):
    """The same row twice, one that falls, out of range, more than the list's width: the request stays, the others move."""
    r = Rows([20, 30], 12, 16, 2, 64, 2, BF)
    want = r.expected([[], [3, 5]])
    r.call([bad, [3, 5]], 4, status=EINVAL)
    assert torch.equal(r.arena.view(torch.int16), want)


@pytest.mark.parametrize("bad", [[-9, -3], [-2 ** 31, -2 ** 31 + 1, 5], [0, -8, -7], list(range(-60, 0)), [0, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31],
                                 list(range(10)) + [0] + list(range(49)), list(range(60, 0, -1)), [0, 1] * 30])
@pytest.mark.parametrize("at", [0, 1, 36])
def test_lists_whose_entries_pass_one_by_one(bad, at):
    """Entries below 0 that rise, and entries of long lists that are far below their place: none of them leads out of the request's
    cells, with a request at its first row and one that reaches to its table's last cell."""
    r = Rows([at, 30], 12, 16, 2, 64, 2, BF)                       # 48 positions in either row of the table
    r.tables = gpu([row[:3] for row in r.table.tolist()])
    r.tables[r.tables == 0x7fffffff] = 0
    want = r.expected([[], [3, 5]])
    r.call([bad, [3, 5]], 64, status=EINVAL)
    assert torch.equal(r.arena.view(torch.int16), want)


def test_entries_of_accepted_rows_outside_their_arena():
    r = Rows([14, 30], 12, 16, 2, 64, 2, BF)
    want = r.expected([[], [3, 5]])
    r.tables[0, 1] = 10 ** 6
    r.call([[0, 3], [3, 5]], 4, status=EINVAL)
    assert torch.equal(r.arena.view(torch.int16), want)


def test_a_verification_step_with_forks_as_it_is_used():
    """Prompts, forks of them, drafted trees, attention, accepted rows, the rest given back, samples ended, the cache moved to the
    front: every layer's rows and the attention over them are those of a dense copy of each request."""
    T, Hkv, G, D, L, n, width = 16, 2, 4, 64, 2, 6, 20
    w = World(n, T, width, (120, 40), seed=11)
    arena = torch.full((L, 160, 2, T, Hkv, D), float("nan"), device="cuda").to(BF)
    caches = [B.PagedCache(arena[i, :120], arena[i, 120:]) for i in range(L)]
    layers = B.PagedLayers(caches)
    gen = torch.Generator(device="cuda").manual_seed(0)
    i32 = dict(dtype=torch.int32, device="cuda")
    work = torch.empty(B.paged_tree_workspace(caches[0], Hkv * G), dtype=torch.uint8, device="cuda")
    dense = [[torch.zeros((2, 0, Hkv, D), dtype=BF, device="cuda") for _ in range(n)] for _ in range(L)]
    stream = torch.cuda.current_stream()

    def grow(add, room=64):
        """Room for new tokens, rows written; the dense copies grow as well."""
        new = [a + b for a, b in zip(w.lens, add)]
        offsets, positions, slots = torch.zeros(n + 1, **i32), torch.zeros(room, **i32), torch.zeros(room, dtype=torch.int64, device="cuda")
        target = gpu(new)
        assert B.paged_build_tables(w.pool, w.held_lens, target, T, w.tables, offsets, slots, positions, w.status, stream) == B.OK
        for layer in range(L):
            kv = torch.randn((2, room, Hkv, D), device="cuda", generator=gen).to(BF)
            assert B.paged_write_kv(caches[layer], kv[0], kv[1], slots, w.status, stream) == B.OK
            at = 0
            for i, a in enumerate(add):
                dense[layer][i] = torch.cat([dense[layer][i], kv[:, at:at + a]], 1)
                at += a
        w.held_lens.copy_(target)
        for i, x in enumerate(new):
            while len(w.rows[i]) < ceil_div(x, T):
                w.rows[i].append(w.pop())
        w.lens = new
        return offsets

    def same_rows():
        torch.cuda.synchronize()
        assert int(w.status) == 0
        w.same()
        for layer in range(L):
            for i in range(n):
                k, v = logical_rows(arena[layer, :120], arena[layer, 120:], w.rows[i], w.lens[i], T)
                assert torch.equal(torch.stack([k, v]), dense[layer][i].double()), (layer, i)

    grow([40, 21, 0, 0, 0, 0], 64)
    copies = torch.zeros((3, 3), **i32)
    src, dst = [0, 0, 1], [2, 3, 4]
    w.fork(src, dst)
    assert B.paged_fork(w.pool, w.shares, w.held_lens, w.held_lens, gpu([0]), gpu([-1]), T, w.tables, copies[:1], w.status, stream) == B.OK   # padding alone
    for s, d in zip(src, dst):
        for layer in range(L):
            dense[layer][d] = dense[layer][s].clone()
    # the forks' last blocks, from the tables that the model knows
    todo = [(w.rows[s][w.lens[s] // T], w.rows[d][w.lens[s] // T], w.lens[s] % T) for s, d in zip(src, dst)]
    assert B.paged_copy_blocks(layers, gpu(todo), w.status, stream) == B.OK
    same_rows()
    rng = np.random.default_rng(2)
    for step in range(4):
        m = [5, 0, 7, 1, 9, 3]
        offsets = grow(m)
        bits = [[1 << j | (1 << (j - 1) // 2 if j else 0) for j in range(k)] for k in m]   # a parent and itself: any sets will do
        mask = torch.zeros((64, 1), dtype=torch.int64, device="cuda")
        at = 0
        for i, k in enumerate(m):
            for j in range(k):
                mask[at + j, 0] = bits[i][j]
            at += k
        q = torch.randn((64, Hkv * G, D), device="cuda", generator=gen).to(BF)
        out = torch.zeros_like(q)
        for layer in range(L):
            assert B.paged_tree_attention(caches[layer], w.tables, w.held_lens, offsets, q, 0.125, out, work, mask=mask, status=w.status,
                                          stream=stream) == B.OK
            at = 0
            for i, k in enumerate(m):
                kv, c = dense[layer][i].double(), w.lens[i] - k
                for j in range(k):
                    see = torch.tensor([p < c or bits[i][j] >> (p - c) & 1 == 1 for p in range(w.lens[i])], device="cuda")
                    z = torch.einsum("hgd,nhd->hgn", q[at + j].double().view(Hkv, G, D), kv[0]) * 0.125
                    prob = torch.softmax(z.masked_fill(~see, -float("inf")), -1)
                    ref, mean = (torch.einsum("hgn,nhd->hgd", prob, x).reshape(Hkv * G, D) for x in (kv[1], kv[1].abs()))
                    # half a step of the output and of each weight; errors of scores, exponentials and sums are far below 1e-4 here
                    assert bool(((out[at + j].double() - ref).abs() <= torch.finfo(BF).eps / 2 * 1.01 * (ref.abs() + mean) + 1e-4).all())
                at += k
        keep = [sorted(rng.permutation(k)[:int(rng.integers(1, k + 1))].tolist()) if k else [] for k in m]
        kt = torch.zeros((n, 9), **i32)
        for i, ks in enumerate(keep):
            if ks:
                kt[i, :len(ks)] = gpu(ks)
        before = gpu([x - k for x, k in zip(w.lens, m)])
        assert B.paged_keep_rows(layers, w.tables, before, kt, gpu([len(ks) for ks in keep]), w.status, stream) == B.OK
        less = [x - k + len(ks) for x, k, ks in zip(w.lens, m, keep)]
        for layer in range(L):
            for i in range(n):
                c = w.lens[i] - m[i]
                dense[layer][i] = torch.cat([dense[layer][i][:, :c], dense[layer][i][:, [c + k for k in keep[i]]]], 1)
        w.release(less)
        same_rows()
    w.release([w.lens[0], 0, w.lens[2], 0, w.lens[4], 0])
    for i in (1, 3, 5):
        for layer in range(L):
            dense[layer][i] = dense[layer][i][:, :0]
    held = w.holders()
    moves = w.compact([len(held), 0])                            # the lender takes its memory, what is left lies in front
    assert moves
    assert B.paged_copy_blocks(layers, gpu(moves), w.status, stream) == B.OK
    same_rows()
    assert all(0 <= e < len(held) for r in w.rows for e in r)


def test_calls_without_requests():
    """Tops are handed on; a compaction still takes ids off the stacks."""
    w = World(3, 16, 8, (30, 10))
    i32 = dict(dtype=torch.int32, device="cuda")
    none, tables = torch.zeros(0, **i32), torch.zeros((0, 8), **i32)
    assert B.paged_free(w.pool, w.shares, none, none, 16, tables, w.status) == B.OK
    assert B.paged_fork(w.pool, w.shares, none, none, none, none, 16, tables, torch.zeros((0, 3), **i32), w.status) == B.OK
    torch.cuda.synchronize()
    w.same()
    copies = torch.full((2, 3), 7, **i32)
    assert B.paged_compact(w.pool, w.shares, gpu([20, 0]), none, 16, tables, copies, w.status) == B.OK
    torch.cuda.synchronize()
    w.stacks = [[x for x in w.stacks[0] if x < 20], []]
    assert int(w.status) == 0 and not copies.any()
    w.same()


def test_a_request_cut_inside_a_shared_block_is_forked_to_go_on():
    w = World(4, 16, 8, (30, 0))
    w.grow([64, 0, 0, 0])
    w.fork([0], [1])
    w.release([64, 40, 0, 0])                                    # the third block stays shared, eight rows of it are this request's
    assert w.fork([1], [2])[0][2] == 8
    w.release([64, 0, 40, 0])
    w.grow([64, 0, 60, 0])
    w.same()
    assert w.rows[2][2] != w.rows[0][2]
