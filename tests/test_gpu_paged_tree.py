"""Attention of several new tokens per request (trees of drafted tokens, chains) against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2609_27040_b200 import binding as B
from paper_2609_27040_b200 import build as build_mod
from tests.paged_helpers import ceil_div, close, logical_rows, lse_slack, row_error, stored_place

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def gpu(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def tree_bits(rng, m):
    """Who sees whom in a random tree of m nodes, as whole numbers."""
    seen = []
    for j in range(m):
        up = j - int(rng.integers(1, 5))
        seen.append((seen[up] if up >= 0 else 0) | 1 << j)
    return seen


def random_bits(rng, m):
    """Any sets, empty ones among them."""
    return [0 if rng.random() < 0.2 else sum(1 << b for b in range(m) if rng.random() < 0.4) for _ in range(m)]


class Case:
    """Requests of ctx[i] + m[i] tokens in a cache whose rows behind the last token hold `stray`, and their new tokens' queries."""

    def __init__(self, ctx, m, Hkv, G, D, T, dtype, lent=0.0, seed=0, kind="chain", window=0, positions=False, qscale=1.5, stray=math.nan, spare=3):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.m, self.Hkv, self.G, self.D, self.T, self.dtype, self.kind, self.window = list(ctx), list(m), Hkv, G, D, T, dtype, kind, window
        n, lens = len(ctx), [c + k for c, k in zip(ctx, m)]
        self.lens = lens
        nb = [ceil_div(x, T) for x in lens]
        count = sum(nb)
        n_lent = int(round(count * lent))
        sizes = (count - n_lent + 2, n_lent + (1 if lent else 0))
        ids = rng.permutation(np.concatenate([rng.permutation(sizes[0])[:count - n_lent], ~rng.permutation(max(sizes[1], 1))[:n_lent]]))
        randn = lambda *s: torch.randn(s, device="cuda", generator=gen).to(dtype)     # noqa: E731
        self.local, self.lent = randn(sizes[0], 2, T, Hkv, D), randn(sizes[1], 2, T, Hkv, D) if lent else None
        width = max(nb + [1]) + 1
        t = np.full((n, width), 0x7fffffff)                      # cells that are not read hold no valid entry
        at = 0
        for i, k in enumerate(nb):
            t[i, :k] = ids[at:at + k]
            at += k
            if lens[i] % T and stray is not None:
                self.block(int(t[i, k - 1]))[:, lens[i] % T:] = stray
        self.table_np = t
        self.tables = torch.zeros((n, width + 2), dtype=torch.int32, device="cuda")[:, :width]
        self.tables.copy_(torch.from_numpy(t).to(torch.int32))
        self.lens_t, self.off = gpu(lens), np.concatenate([[0], np.cumsum(m)]).tolist()
        self.offsets = gpu(self.off)
        self.tokens = self.off[-1]
        room, Hq = self.tokens + spare, Hkv * G
        self.bits = None
        self.mask = self.positions = None
        if kind != "chain":
            self.bits = [(tree_bits if kind == "tree" else random_bits)(rng, k) for k in m]
            words = max(1, ceil_div(max(list(m) + [1]), 64))
            mask = rng.integers(-1 << 63, (1 << 63) - 1, (room, words + 1))       # bits behind a request's tokens mean nothing
            for i in range(n):
                for j, b in enumerate(self.bits[i]):
                    for w in range(words):
                        low = min(64, max(0, m[i] - 64 * w))
                        junk = int(mask[self.off[i] + j, w]) & ((1 << 64) - 1) & ~((1 << low) - 1)
                        v = (b >> (64 * w) & ((1 << low) - 1)) | junk
                        mask[self.off[i] + j, w] = v - (1 << 64) if v >> 63 else v
            self.mask = torch.from_numpy(mask).to("cuda")[:, :words]
        self.pos = [[c + j for j in range(k)] for c, k in zip(ctx, m)]
        if positions:
            self.pos = [[c + bin(b).count("1") - 1 if self.bits else c + int(rng.integers(0, k)) for b in (self.bits[i] if self.bits else range(k))]
                        for i, (c, k) in enumerate(zip(ctx, m))]
            self.pos = [[max(c, x) for x in row] for c, row in zip(ctx, self.pos)]
            self.positions = gpu([x for row in self.pos for x in row] + [0] * spare)
        self.q = (torch.randn((room, Hq + 2, D), device="cuda", generator=gen) * qscale).to(dtype)[:, :Hq]
        self.scale = D ** -0.5
        self.cache = B.PagedCache(self.local, self.lent)
        self.work = torch.full((B.paged_tree_workspace(self.cache, Hq),), 0xff, dtype=torch.uint8, device="cuda")   # NaN all over
        self.out = torch.full((room, Hq + 1, D), 7.0, dtype=dtype, device="cuda")[:, :Hq]
        self.lse = torch.full((room, Hq), 7.0, device="cuda")
        self.status = gpu([0])

    def block(self, e):
        return self.local[e] if e >= 0 else self.lent[~e]

    def call(self, stream=None, **kw):
        a = dict(mask=self.mask, lse=self.lse, window=self.window, positions=self.positions, status=self.status, stream=stream)
        a.update(kw)
        return B.paged_tree_attention(self.cache, self.tables, self.lens_t, self.offsets, self.q, self.scale, self.out, self.work, **a)

    def run(self, status=0, **kw):
        torch.cuda.synchronize()
        assert self.call(**kw) == B.OK
        torch.cuda.synchronize()
        assert int(self.status) == status
        return self

    def sees(self, i):
        """[m][ctx + m] truth values."""
        c, m = self.ctx[i], self.m[i]
        p, pos = np.arange(c + m)[None, :], np.array(self.pos[i]).reshape(-1, 1)
        see = np.repeat(p < c, m, 0)
        if self.window:
            see &= p > pos - self.window
        if self.bits is None:
            new = np.arange(m)[None, :] <= np.arange(m)[:, None]
            if self.window:
                new &= p[:, c:] > pos - self.window
        else:
            new = np.array([[b >> x & 1 for x in range(m)] for b in self.bits[i]], bool).reshape(m, m)
        see[:, c:] = new
        return see

    def reference(self, i):
        k, v = logical_rows(self.local, self.lent, self.table_np[i], self.lens[i], self.T)
        see = torch.from_numpy(self.sees(i)).to("cuda")
        m, Hkv, G, D = self.m[i], self.Hkv, self.G, self.D
        q = self.q[self.off[i]:self.off[i] + m].double().reshape(m, Hkv, G, D)
        z = torch.einsum("mhgd,nhd->hgmn", q, torch.nan_to_num(k)) * self.scale
        if bool(see.any()):
            size = float((torch.einsum("mhgd,nhd->hgmn", q.abs(), torch.nan_to_num(k).abs()) * abs(self.scale)).masked_fill(~see, 0.0).max())
            vmax = float(v[see.any(0)].abs().max())
        else:
            size = vmax = 0.0
        z = z.masked_fill(~see, -math.inf)
        w = torch.softmax(z, -1).masked_fill(~see.any(1)[:, None], 0.0)
        v = v.masked_fill(~see.any(0)[:, None, None], 0.0)
        out = torch.einsum("hgmn,nhd->mhgd", w, v).reshape(m, Hkv * G, D)
        # A weight is one 16-bit number, off by half a step at most, and the sum of weights is taken before the rounding: an output is
        # off by at most half a step times the weighted sum of magnitudes.
        self.rounded = torch.finfo(self.dtype).eps / 2 * torch.einsum("hgmn,nhd->mhgd", w, v.abs()).reshape(m, Hkv * G, D)
        return out, torch.logsumexp(z, -1).permute(2, 0, 1).reshape(m, -1), size, vmax

    def check(self):
        eps = torch.finfo(self.dtype).eps
        assert (self.out[self.tokens:] == 7.0).all() and (self.lse[self.tokens:] == 7.0).all()
        for i in range(len(self.m)):
            if not self.m[i]:
                continue
            rows = slice(self.off[i], self.off[i + 1])
            ref, lse, size, vmax = self.reference(i)
            n, D = self.lens[i], self.D
            # A step rescales a row's sum and rows when its largest score has grown by 2^4 or more, at most size log2(e) / 2 times (scores lie between -size
            # and size); the factor is the same for both, what is left are two roundings of 2^-24 each time.
            grown = (size * 1.45 / 2 + 2) * 2.0 ** -23
            ok, worst = close(self.out[rows], ref, row_error(n, D, size, vmax) + 2 * grown * vmax + self.rounded, eps)
            assert ok, (i, n, self.m[i], worst)
            none = lse == -math.inf
            assert (self.lse[rows][none] == -math.inf).all() and not self.out[rows][none].any()
            if not bool(none.all()):
                assert float((self.lse[rows].double() - lse)[~none].abs().max()) <= lse_slack(n, D, size) + grown, i
        return self


@pytest.mark.parametrize("D,T,Hkv,G,dtype", [(64, 16, 3, 4, BF), (64, 64, 1, 1, HF), (64, 32, 2, 16, BF), (128, 16, 2, 4, BF), (128, 32, 1, 7, HF),
                                             (128, 64, 3, 8, BF), (256, 16, 2, 4, HF), (256, 64, 1, 3, BF), (256, 32, 2, 16, BF)])
@pytest.mark.parametrize("kind", ["chain", "tree", "any"])
def test_ragged_batches(D, T, Hkv, G, dtype, kind):
    """No context, contexts around the ends of blocks and of steps, requests without new tokens, one token, more than a tile of them."""
    ctx = [0, 0, 1, T - 1, T, 63, 127, 128, 129, 500, 700, 5, 300, 40]
    m = [1, 9, 3, 2, 0, 1, 1, 5, 24, 33, 0, 70, 128 // G + 1, 2 * (128 // G) + 3]
    Case(ctx, m, Hkv, G, D, T, dtype, lent=0.4, seed=D + T, kind=kind).run().check()


@pytest.mark.parametrize("D", [64, 128, 256])
def test_every_number_of_tokens_of_one_request(D):
    for m in (1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129):
        Case([37 * m % 200], [m], 1, 2, D, 16, BF, seed=m, kind="tree" if m % 2 else "any").run().check()


@pytest.mark.parametrize("n,ctx,m,Hkv,G,D,T,dtype", [(1, 30000, 8, 2, 4, 128, 16, BF), (3, 9001, 50, 1, 8, 128, 32, HF), (2, 5003, 17, 3, 2, 256, 16, BF),
                                                    (1, 12007, 5, 8, 1, 64, 64, HF)])
@pytest.mark.parametrize("kind", ["chain", "tree"])
def test_long_contexts_are_cut_and_joined(n, ctx, m, Hkv, G, D, T, dtype, kind):
    Case([ctx - 17 * i for i in range(n)], [m] * n, Hkv, G, D, T, dtype, lent=0.3, seed=m, kind=kind).run().check()


@pytest.mark.parametrize("D,G,dtype", [(64, 4, BF), (128, 4, BF), (128, 1, HF), (256, 2, BF)])
def test_pieces_of_prompts(D, G, dtype):
    """Several items to a request, an odd number of tiles, more items than CTAs."""
    Case([0, 1000, 3, 77], [700, 333, 129, 1], 4, G, D, 16, dtype, seed=3).run().check()


@pytest.mark.parametrize("G,Hkv", [(5, 1), (11, 2), (33, 1), (64, 1), (100, 1), (128, 2)])
def test_groups_that_do_not_divide_a_tile(G, Hkv):
    Case([100, 0, 411], [3, 7, 2], Hkv, G, 128, 16, BF, seed=G, kind="any").run().check()


@pytest.mark.parametrize("kind,positions", [("chain", False), ("chain", True), ("tree", False), ("tree", True), ("any", True)])
@pytest.mark.parametrize("window", [1, 7, 130, 1000])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_windows(D, window, kind, positions):
    Case([0, 5, 129, 900, 2050], [4, 11, 40, 3, 66], 2, 4, D, 16, BF, lent=0.5, seed=window, kind=kind, window=window, positions=positions).run().check()


def test_positions_outside_the_request_are_taken_into_it():
    c = Case([300, 20], [6, 5], 2, 2, 128, 16, BF, kind="tree", window=40, positions=True)
    want = c.run().out.clone()
    c.positions[:11] = gpu([x if 300 < x < 305 else (-5 if x == 300 else 2 ** 31 - 1) for x in c.pos[0]] + [x if 20 < x < 24 else (-9 if x == 20 else 10 ** 6)
                                                                                                      for x in c.pos[1]])
    expect = [[min(max(x, 300), 305) for x in c.positions[:6].tolist()], [min(max(x, 20), 24) for x in c.positions[6:11].tolist()]]
    c.pos = expect
    c.run().check()
    assert c.out.shape == want.shape


@pytest.mark.parametrize("D", [64, 128, 256])
def test_what_nobody_sees_may_hold_anything(D):
    """Rows of V that no token of a request sees, rows of K that a token does not see, behind the last token and before the window."""
    T = 16
    c = Case([200, 90, 513], [9, 70, 3], 2, 4, D, T, BF, seed=1, kind="any", stray=math.inf, window=100)
    for i in range(3):
        see = c.sees(i).any(0)
        for p in np.flatnonzero(~see):
            row = c.block(int(c.table_np[i, p // T]))[:, p % T]
            row[0], row[1] = math.nan, (math.nan, math.inf, -math.inf)[p % 3]
    assert any((~c.sees(i).any(0)).any() for i in range(3))
    c.run().check()


def test_rows_of_k_that_some_do_not_see():
    """A drafted token whose K row is not a number: the tokens that do not see it are as if it were not there."""
    c = Case([130], [6], 1, 4, 128, 16, BF, kind="tree", stray=0.0)
    c.bits = [[1 << j for j in range(6)]]
    c.mask[:6, 0] = gpu([1 << j for j in range(6)], torch.int64)
    row = c.block(int(c.table_np[0, 133 // 16]))[0, 133 % 16]
    row[:] = math.nan
    c.run()
    ref, _, size, vmax = c.reference(0)
    got = c.out[:6].double()
    assert torch.isnan(got[3]).all()
    keep = [0, 1, 2, 4, 5]
    ok, worst = close(got[keep], ref[keep], row_error(136, 128, size, vmax) + 2.0 ** -20 * vmax + c.rounded[keep], torch.finfo(BF).eps)
    assert ok, worst


@pytest.mark.parametrize("scale", [0.0, -0.09, 3.0, 60.0])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_scales(scale, dtype):
    """None, a negative one, scores far apart (weights of 0 and 1, references that grow from step to step)."""
    c = Case([700, 3], [5, 2], 2, 4, 128, 16, dtype, seed=5, kind="tree")
    c.scale = scale
    c.run().check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_references_that_grow_in_every_step(D, dtype):
    """Scores that rise with the position, by 2^3 to 2^30 a step: O is rescaled in some steps, in all of them, and by nearly everything."""
    T = 16
    for rise in (3.0, 5.0, 9.0, 30.0):
        c = Case([1500], [4], 1, 2, D, T, dtype, seed=2)
        c.q[:] = 0.0
        c.q[:, :, 0] = 1.0
        c.scale = 1.0
        k = torch.zeros((1504, D), device="cuda")
        k[:, 0] = torch.arange(1504, device="cuda") * (rise * math.log(2.0) / 128)
        for p in range(1504):
            c.block(int(c.table_np[0, p // T]))[0, p % T, 0] = k[p, torch.from_numpy(np.argsort(stored_place(p % T, D))).to("cuda")].to(dtype)
        c.run().check()


def test_one_token_is_what_decode_gives():
    c = Case([511, 1999, 0, 64], [1, 1, 1, 1], 4, 4, 128, 16, BF, spare=0)
    c.run().check()
    out = torch.empty_like(c.out).contiguous()
    work = torch.zeros(B.paged_decode_workspace(c.cache, 16), dtype=torch.uint8, device="cuda")
    assert B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, out, work) == B.OK
    torch.cuda.synchronize()
    for i in range(4):                                           # half a step of either's result, and of this one's weights
        ref = c.reference(i)[0]
        assert bool(((out[i].double() - c.out[i].double()).abs() <= torch.finfo(BF).eps * 1.01 * ref[0].abs() + c.rounded[0] + 1e-5).all())


def test_results_do_not_depend_on_timing_or_the_workspace():
    c = Case([4000, 100, 7, 9000], [20, 130, 1, 33], 2, 4, 128, 16, BF, seed=9, kind="any")
    first, lse = c.run().out.clone(), c.lse.clone()
    for fill in (0, 0x7f):
        c.work.fill_(fill)
        c.out.zero_()
        c.run()
        assert torch.equal(c.out[:c.tokens], first[:c.tokens]) and torch.equal(c.lse[:c.tokens], lse[:c.tokens])


def test_rows_that_the_offsets_leave_out_are_not_touched():
    c = Case([100, 50, 200], [4, 5, 6], 2, 4, 128, 16, BF, spare=9)
    c.offsets.copy_(gpu([2, 6, 11, 17]))
    c.out.fill_(7.0)
    c.run()
    assert (c.out[:2] == 7.0).all() and (c.out[17:] == 7.0).all() and not (c.out[2:17] == 7.0).all(-1).any()


def test_lengths_and_offsets_out_of_range():
    """The request's rows are zeros, the others as they should be."""
    c = Case([100, 50, 200, 30], [4, 5, 6, 2], 2, 4, 128, 16, BF)
    width = c.tables.shape[1]
    for bad in (-1, width * 16 + 1, 4):                          # the last: fewer positions than new tokens
        c.lens_t.copy_(gpu([104, bad, 206, 32]))
        c.out.fill_(7.0)
        c.status.zero_()
        c.run(status=-1)
        assert not c.out[4:9].any() and (c.lse[4:9] == -math.inf).all()
        for i in (0, 2, 3):
            ref, _, size, vmax = c.reference(i)
            assert close(c.out[c.off[i]:c.off[i + 1]], ref, row_error(c.lens[i], 128, size, vmax) + 2.0 ** -20 * vmax + c.rounded, torch.finfo(BF).eps)[0]
    c.lens_t.copy_(gpu(c.lens))
    for bad in ([0, 4, 3, 15, 17], [-1, 4, 9, 15, 17], [0, 4, 9, 15, 21]):       # falling, below 0, past the token arrays
        c.offsets.copy_(gpu(bad))
        c.status.zero_()
        c.run(status=-1)


def test_entries_outside_their_arena_read_as_zeros():
    c = Case([100, 50], [4, 5], 2, 4, 128, 16, BF, lent=0.5)
    c.tables[0, 1] = 10 ** 6
    c.tables[0, 2] = ~(10 ** 6)
    c.run(status=-1)
    ref, _, size, vmax = c.reference(1)
    assert close(c.out[4:9], ref, row_error(55, 128, size, vmax) + 2.0 ** -20 * vmax + c.rounded, torch.finfo(BF).eps)[0]
    one = Case([100], [4], 2, 4, 128, 16, BF)                    # an arena that the cache does not have
    one.tables[0, 1] = ~3
    one.run(status=-1)


def test_nothing_to_do():
    c = Case([100, 50], [0, 0], 2, 4, 128, 16, BF)
    c.run()
    assert (c.out == 7.0).all()
    empty = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")     # noqa: E731
    assert B.paged_tree_attention(c.cache, empty(0, 3), empty(0), gpu([0]), c.q, c.scale, c.out, c.work) == B.OK
    assert B.paged_tree_attention(c.cache, c.tables, c.lens_t, c.offsets, c.q[:0], c.scale, c.out[:0], c.work) == B.OK
    torch.cuda.synchronize()


def test_many_requests():
    """More than a thread's worth of them each, most without new tokens."""
    rng = np.random.default_rng(0)
    n = 700
    ctx, m = rng.integers(0, 60, n).tolist(), [int(x) if y < 0.5 else 0 for x, y in zip(rng.integers(1, 5, n), rng.random(n))]
    c = Case(ctx, m, 1, 2, 64, 16, BF, kind="tree").run()
    for i in list(range(0, n, 13)):
        if m[i]:
            ref, _, size, vmax = c.reference(i)
            assert close(c.out[c.off[i]:c.off[i + 1]], ref, row_error(c.lens[i], 64, size, vmax) + 2.0 ** -20 * vmax + c.rounded, torch.finfo(BF).eps)[0], i


def test_captured_and_replayed_while_lengths_and_trees_change():
    a = Case([3000, 100, 7, 900], [20, 30, 1, 33], 2, 4, 128, 16, BF, seed=9, kind="any", spare=40)
    s = torch.cuda.Stream()
    a.run(stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        assert a.call(stream=s) == B.OK
    graph.replay()
    torch.cuda.synchronize()
    a.check()
    # other lengths, fewer tokens, another tree: the same graph
    a.ctx, a.m = [2990, 0, 7, 800], [5, 31, 0, 61]
    a.lens, a.off = [c + k for c, k in zip(a.ctx, a.m)], np.concatenate([[0], np.cumsum(a.m)]).tolist()
    rng = np.random.default_rng(4)
    a.bits = [tree_bits(rng, k) for k in a.m]
    a.tokens = a.off[-1]
    a.lens_t.copy_(gpu(a.lens))
    a.offsets.copy_(gpu(a.off))
    for i in range(4):
        for j, b in enumerate(a.bits[i]):
            a.mask[a.off[i] + j, 0] = b - (1 << 64) if b >> 63 else b
    for i in range(4):                                           # what was behind the old lengths is not a number: rows of the new ones are
        for p in range(a.lens[i]):
            a.block(int(a.table_np[i, p // 16]))[:, p % 16].nan_to_num_(0.25)
    a.out.fill_(7.0)
    a.lse.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert int(a.status) == 0
    a.check()


def test_two_streams_with_a_workspace_each():
    cases = [Case([2000 + 100 * x, 50], [20, 7], 2, 4, 128, 16, BF, seed=x, kind="tree") for x in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(cases, streams):
            assert c.call(stream=s) == B.OK
    torch.cuda.synchronize()
    for c in cases:
        assert int(c.status) == 0
        c.check()


def test_a_step_right_behind_the_kernels_that_write_its_inputs():
    c = Case([900, 30], [9, 5], 2, 4, 128, 16, BF, kind="tree")
    want = c.run().out.clone()
    q, lens, offsets, mask = c.q.clone(), c.lens_t.clone(), c.offsets.clone(), c.mask.clone()
    s = torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s):
            c.q.fill_(math.nan)
            c.lens_t.zero_()
            c.offsets.zero_()
            c.mask.zero_()
            torch.cuda._sleep(200000)
            c.q.copy_(q)
            c.lens_t.copy_(lens)
            c.offsets.copy_(offsets)
            c.mask.copy_(mask)
            assert c.call(stream=s) == B.OK
        torch.cuda.synchronize()
        assert torch.equal(c.out[:c.tokens], want[:c.tokens])


def test_blocks_far_behind_the_arenas_start():
    """Block offsets beyond 2^32 bytes."""
    T, Hkv, D = 16, 4, 128
    blocks = (5 << 30) // (2 * T * Hkv * D * 2) + 3
    arena = torch.zeros((blocks, 2, T, Hkv, D), dtype=BF, device="cuda")
    c = Case([150], [6], Hkv, 4, D, T, BF, kind="tree")
    used = c.table_np[0, :10].copy()
    for j, e in enumerate(used):
        arena[blocks - 1 - j] = c.block(int(e))
        c.table_np[0, j] = blocks - 1 - j
    c.local = arena
    c.tables[0, :10] = gpu(c.table_np[0, :10].tolist())
    c.cache = B.PagedCache(arena)
    c.run().check()


@pytest.mark.parametrize("seed", range(12))
def test_mixed_batches(seed):
    """Requests of one tile, of two and of many behind one another in a CTA, padding between them, whatever the shape."""
    rng = np.random.default_rng(1000 + seed)
    D, T, G = int(rng.choice([64, 128, 256])), int(rng.choice([16, 32, 64])), int(rng.choice([1, 2, 4, 7, 16]))
    Hkv = int(rng.integers(1, 5))
    n = int(rng.integers(20, 60))
    tile = 128 // G
    m = [int(x) for x in rng.choice([0, 0, 1, 2, tile - 1, tile, tile + 1, 2 * tile, 2 * tile + 1, 5 * tile + 3], n)]
    ctx = [int(rng.integers(0, 10 ** rng.integers(1, 4))) for _ in range(n)]
    kind = ["chain", "tree", "any"][seed % 3]
    window = int(rng.choice([0, 0, 50, 400]))
    c = Case(ctx, m, Hkv, G, D, T, BF if seed % 2 else HF, lent=0.3, seed=seed, kind=kind, window=window, positions=bool(window and seed % 2))
    c.run().check()


def test_a_batch_that_is_mostly_padding():
    n = 3000
    ctx, m = [0] * n, [0] * n
    for i in (0, 5, 1600, 1601, 2999):
        ctx[i], m[i] = 100 + i // 7, 3
    Case(ctx, m, 2, 4, 128, 16, BF, kind="tree").run().check()


@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_cache_in_the_second_arena_alone(D):
    c = Case([200, 0, 33], [5, 9, 70], 2, 4, D, 16, BF, kind="tree")
    c.local, c.lent = None, c.local
    held = c.table_np < 0x7fffffff
    c.table_np[held] = ~c.table_np[held]
    c.tables.copy_(torch.from_numpy(c.table_np).to(torch.int32))
    c.cache = B.PagedCache(None, c.lent)
    c.run().check()


def test_results_are_the_same_in_a_batch_and_alone():
    """Items that are not cut are computed alike, whoever else is in the batch: here all of them, on both sides."""
    c = Case([40, 90, 17, 60], [3, 5, 2, 7], 2, 4, 128, 16, BF, kind="tree")
    want = c.run().out.clone()
    for i in range(4):
        one = Case([1], [1], 2, 4, 128, 16, BF, spare=0)
        rows = slice(c.off[i], c.off[i + 1])
        out = torch.zeros_like(want[rows]).contiguous()
        assert B.paged_tree_attention(c.cache, c.tables[i:i + 1], c.lens_t[i:i + 1], gpu([0, c.m[i]]), c.q[rows], c.scale, out, one.work,
                                      mask=c.mask[rows]) == B.OK
        torch.cuda.synchronize()
        assert torch.equal(out, want[rows])


@pytest.mark.parametrize("D,G,m,ctx", [(128, 4, [5, 9, 3], [700, 1500, 900]), (128, 3, [42, 37, 40], [800, 513, 2000]), (128, 7, [18, 17, 16], [640, 900, 1300]),
                                       (64, 4, [30, 3, 45], [900, 1500, 700]), (256, 3, [42, 5, 33], [500, 700, 1100]), (128, 33, [3, 1, 2], [700, 800, 1200])])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_results_do_not_depend_on_rows_that_are_nobodys(D, G, m, ctx, dtype):
    """To the bit, with steps that no mask touches: the queries of other requests and of rows that the offsets leave out, and what a
    kernel before has left in shared memory where a group's heads leave rows of a tile free."""
    n = 48                                                         # more items than CTAs: several steps of one lie in a CTA
    c = Case((ctx * n)[:n], (m * n)[:n], 4, G, D, 16, dtype, seed=G + D, kind="tree", spare=9)
    c.offsets.copy_(gpu([x + 4 for x in c.off]))                   # four rows in front, five behind
    c.mask[4:4 + c.tokens] = c.mask[:c.tokens].clone()
    first, lse = c.run().out.clone(), c.lse.clone()
    q = c.q.clone()
    dirt = Case([900] * 40, [50] * 40, 4, 4, 128, 16, dtype, seed=1)
    dirt.q *= 100.0
    for part in range(3):
        mine = torch.cat([torch.arange(4 + c.off[i], 4 + c.off[i + 1]) for i in range(n) if i % 3 == part]).cuda()
        for factor in (100.0, -30.0, 0.0):
            c.q.copy_(q * factor)
            c.q[mine] = q[mine]
            dirt.run()
            c.run()
            assert torch.equal(c.out[mine], first[mine]) and torch.equal(c.lse[mine], lse[mine]), (part, factor)


@pytest.mark.parametrize("D,G,dtype", [(64, 1, BF), (64, 16, HF), (128, 4, BF), (128, 8, HF), (128, 7, BF), (256, 4, BF), (256, 2, HF), (128, 128, BF)])
@pytest.mark.parametrize("kind", ["chain", "tree", "any"])
def test_weights_are_as_exact_as_those_of_single_tokens(D, G, dtype, kind):
    """Requests of up to a tile of rows (128 // G tokens): the bound that single tokens are held to, without an allowance for weights of one
    16-bit number. Few positions with V of 1 and -1 and scores near one another: outputs are small beside what such a weight's rounding
    does to them. With a request of one token more in the batch, which has that allowance."""
    tile = 128 // G
    m = [min(tile, 24), 1, tile, tile + 1, max(1, tile // 2)]
    c = Case([20, 9, 3, 30, 300], m, 2, G, D, 16, dtype, lent=0.3, seed=G, kind=kind, qscale=0.2)
    c.local[:, 1].sign_()
    c.lent[:, 1].sign_()
    c.run().check()
    eps = torch.finfo(dtype).eps
    for i in (0, 1, 2, 4):
        ref, _, size, vmax = c.reference(i)
        grown = (size * 1.45 / 2 + 2) * 2.0 ** -23                 # rescaled, as derived in check
        ok, worst = close(c.out[c.off[i]:c.off[i + 1]], ref, row_error(c.lens[i], D, size, vmax) + 2 * grown * vmax, eps)
        assert ok, (i, worst)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_one_token_and_decode_differ_by_their_own_rounding(dtype):
    c = Case([9, 30, 0, 64, 300], [1] * 5, 4, 4, 128, 16, dtype, spare=0, qscale=0.2)
    c.local[:, 1].sign_()
    c.run()
    out = torch.empty_like(c.out).contiguous()
    work = torch.zeros(B.paged_decode_workspace(c.cache, 16), dtype=torch.uint8, device="cuda")
    assert B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, out, work) == B.OK
    torch.cuda.synchronize()
    for i in range(5):                                             # either is off by half a step and by row_error at most
        ref, _, size, vmax = c.reference(i)
        slack = row_error(c.lens[i], 128, size, vmax)
        far = torch.finfo(dtype).eps * (ref[0].abs() + slack) + 2 * slack + 2.0 ** -24
        assert bool(((out[i].double() - c.out[i].double()).abs() <= far).all()), i


@pytest.mark.parametrize("window", [1, 3, 40])
def test_a_window_and_a_mask(window):
    """Drafts deeper than the window: a chain under a window, the same as a mask whose caller has cleared the ancestors that the window leaves out
    (both: what decoding token by token gives), and as one that names them, which are seen then."""
    ctx, m, bf = [0, 5, 129, 700], [9, 20, 60, 33], torch.finfo(BF).eps
    chain = Case(ctx, m, 2, 2, 128, 16, BF, seed=window, window=window).run().check()
    cleared = Case(ctx, m, 2, 2, 128, 16, BF, seed=window, window=window, kind="tree")
    for name in ("local", "tables", "table_np", "cache", "q"):
        setattr(cleared, name, getattr(chain, name))
    for back in (window, 10 ** 6):
        cleared.bits = [[(1 << j + 1) - 1 & ~((1 << max(0, j + 1 - back)) - 1) for j in range(k)] for k in m]
        cleared.mask[:cleared.tokens, 0] = gpu([b - (1 << 64) if b >> 63 else b for row in cleared.bits for b in row], torch.int64)
        for i in range(4):                                         # a window longer than the chain takes none of it away
            assert np.array_equal(chain.sees(i), cleared.sees(i)) == (back == window or m[i] <= window)
        cleared.run().check()
        if back == window:
            for i in range(4):
                ref, _, size, vmax = chain.reference(i)
                rows = slice(chain.off[i], chain.off[i + 1])
                assert close(cleared.out[rows], ref, row_error(chain.lens[i], 128, size, vmax) + 2.0 ** -20 * vmax + chain.rounded, bf)[0], i


@pytest.mark.parametrize("D,T", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 64), (256, 16), (256, 64)])
@pytest.mark.parametrize("arenas", ["both", "first", "second"])
def test_bad_entries_give_what_blocks_of_zeros_give(D, T, arenas):
    """Entries just and far outside either arena, or of one that the cache does not have, in the context, before a step's end and among the
    new tokens: as if there were a block of zeros."""
    c = Case([700, 50, 3 * T - 2], [4, 5, 9], 2, 4, D, T, BF, lent=0.5 if arenas == "both" else 0.0, seed=T, kind="any")
    zero = next(x for x in range(c.local.shape[0]) if x not in set(c.table_np.flatten().tolist()))
    c.local[zero] = 0.0
    if arenas == "second":
        c.local, c.lent = None, c.local
        held = c.table_np < 0x7fffffff
        c.table_np[held] = ~c.table_np[held]
        c.tables.copy_(torch.from_numpy(c.table_np).to(torch.int32))
        c.cache = B.PagedCache(None, c.lent)
    n0, n1 = (0 if a is None else a.shape[0] for a in (c.local, c.lent))
    bad = [n0, n0 + 1, 2 ** 31 - 1, ~n1, ~(n1 + 1), -2 ** 31]
    last = (c.lens[0] - 1) // T
    cells = [(0, x % last) for x in (0, 3, 5, 7, 9)] + [(0, last), (2, 1), (2, 3)]
    for x, (i, j) in enumerate(cells):
        c.tables[i, j] = bad[x % len(bad)]
        c.table_np[i, j] = ~zero if arenas == "second" else zero
    c.run(status=-1).check()


def test_positions_outside_the_request_give_what_its_first_and_last_give():
    c = Case([300, 20], [6, 5], 2, 2, 128, 16, BF, kind="tree", window=40, positions=True)
    given = [-5, 2 ** 31 - 1, 303, 306, 299, 305, 10 ** 6, -2 ** 31, 22, 25, 19]
    first = [c.ctx[0]] * 6 + [c.ctx[1]] * 5
    last = [305] * 6 + [24] * 5
    outs = []
    for pos in (given, [min(max(x, a), b) for x, a, b in zip(given, first, last)]):
        c.positions[:11] = gpu(pos)
        c.pos = [[min(max(x, 300), 305) for x in pos[:6]], [min(max(x, 20), 24) for x in pos[6:]]]
        outs.append(c.run().check().out.clone())
    assert torch.equal(*outs)
