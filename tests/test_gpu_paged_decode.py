"""Attention through device tables, plain and differential, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2609_27040_b200 import binding as B
from paper_2609_27040_b200 import build as build_mod
from tests.paged_helpers import attend, ceil_div, close, logical_rows, lse_slack, row_error

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def gpu(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


class Case:
    def __init__(self, lens, Hkv, G, D, T, dtype, lent=0.0, seed=0, diff=False, qscale=1.5, stray=None):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.Hkv, self.G, self.D, self.T, self.dtype, self.diff = list(lens), Hkv, G, D, T, dtype, diff
        n, nb = len(lens), [ceil_div(x, T) for x in lens]
        count = sum(nb)
        n_lent = int(round(count * lent))
        self.sizes = (count - n_lent + 2, n_lent + (1 if lent else 0))
        ids = np.concatenate([rng.permutation(self.sizes[0])[:count - n_lent], ~rng.permutation(max(self.sizes[1], 1))[:n_lent]])
        ids = rng.permutation(ids)
        randn = lambda *s: torch.randn(s, device="cuda", generator=gen).to(dtype)     # noqa: E731
        self.local = randn(self.sizes[0], 2, T, Hkv, D)
        self.lent = randn(self.sizes[1], 2, T, Hkv, D) if lent else None
        self.width = max(nb + [1]) + 1
        t = np.full((n, self.width), 0x7fffffff)                 # cells that are not read hold no valid entry
        at = 0
        for i, k in enumerate(nb):
            t[i, :k] = ids[at:at + k]
            at += k
        self.table_np = t
        self.tables = torch.zeros((n, self.width + 2), dtype=torch.int32, device="cuda")[:, :self.width]
        self.tables.copy_(torch.from_numpy(t).to(torch.int32))
        self.lens_t = gpu(self.lens)
        Hq = Hkv * G
        self.q = (torch.randn((n, Hq * (2 if diff else 1) + 3, D // (2 if diff else 1)), device="cuda", generator=gen) * qscale).to(dtype)[:, :-3]
        self.scale = (D // 2 if diff else D) ** -0.5
        self.cache = B.PagedCache(self.local, self.lent)
        self.work = torch.zeros(B.paged_decode_workspace(self.cache, Hq * (2 if diff else 1)), dtype=torch.uint8, device="cuda")
        self.out = torch.full((n + 1, Hq + 2, D), 7.0, dtype=dtype, device="cuda")[:, :Hq]     # rows apart, one more behind the last
        self.lse = torch.full((n + 1, Hq), 7.0, device="cuda")
        self.status = gpu([0])
        self.lam = torch.rand(Hq, device="cuda", generator=gen) * 0.8 + 0.1
        self.weight = torch.rand(D, device="cuda", generator=gen) + 0.5
        if stray is not None:                                    # block tails: bit patterns that may not reach the result
            for i, x in enumerate(lens):
                if x % T:
                    e = int(t[i, x // T])
                    block = self.local[e] if e >= 0 else self.lent[~e]
                    block[:, x % T:] = stray

    def run(self, window=0, stream=None, norm=True, eps=1e-5, out_scale=0.7, lse=True):
        n = len(self.lens)
        self.window, self.norm, self.eps, self.out_scale = window, norm, eps, out_scale
        torch.cuda.synchronize()
        if self.diff:
            rc = B.paged_decode_diff(self.cache, self.tables, self.lens_t, self.q, self.lam, self.scale, self.out[:n], self.work,
                                     norm_weight=self.weight if norm else None, eps=eps, out_scale=out_scale, window=window,
                                     status=self.status, stream=stream)
        else:
            rc = B.paged_decode_tables(self.cache, self.tables, self.lens_t, self.q, self.scale, self.out[:n], self.work,
                                       lse=self.lse[:n] if lse else None, window=window, status=self.status, stream=stream)
        assert rc == B.OK
        torch.cuda.synchronize()
        assert int(self.status) == 0
        assert not self.work[:32768].any()

    def check(self):
        eps = torch.finfo(self.dtype).eps
        n, Hq, D = len(self.lens), self.Hkv * self.G, self.D
        assert (self.out[n] == 7.0).all() and (self.lse[n] == 7.0).all()
        num = den = 0.0
        for i, length in enumerate(self.lens):
            lo = max(0, length - self.window) if self.window else 0
            if length == 0:
                assert not self.out[i].any()
                if not self.diff:
                    assert (self.lse[i] == -math.inf).all()
                continue
            k, v = logical_rows(self.local, self.lent, self.table_np[i], length, self.T)
            k, v, m = k[lo:], v[lo:], length - lo
            vmax = float(v.abs().max())
            q = self.q[i].double()
            if not self.diff:
                ref, lse, size = attend(q, k, v, self.scale)
                slack = row_error(m, D, size, vmax)
                assert float((self.lse[i].double() - lse).abs().max()) <= lse_slack(m, D, size)
            else:
                d = D // 2
                o1, _, s1 = attend(q[0::2], k[..., :d], v, self.scale)
                o2, _, s2 = attend(q[1::2], k[..., d:], v, self.scale)
                x = o1 - self.lam.double()[:, None] * o2
                # both maps' errors, and the subtraction's own rounding
                e = row_error(m, D, s1, vmax) + float(self.lam.max()) * row_error(m, D, s2, vmax) + 2.0 ** -22 * vmax
                if self.norm:
                    rms = torch.sqrt((x * x).mean(-1, keepdim=True) + self.eps)
                    w = self.weight.double()
                    ref = x / rms * w * self.out_scale
                    # x off by e moves x / rms by e / rms, and its norm by at most e / rms of the value; a few f32 roundings
                    slack = float((w.max() * self.out_scale * (e / rms * (1 + x.abs().amax(-1, keepdim=True) / rms))).max()) + 2.0 ** -20 * float(ref.abs().max())
                else:
                    ref, slack = x * self.out_scale, e * self.out_scale
            ok, worst = close(self.out[i], ref, slack, eps)
            assert ok, (i, length, worst, slack)
            num += float((self.out[i].double() - ref).square().sum())
            den += float(ref.square().sum())
        if den:
            assert math.sqrt(num / den) <= eps / 2, math.sqrt(num / den)      # every element is off by half a step at most, plus far less


SHAPES = [(1, 1, 64, 16), (1, 8, 128, 16), (2, 3, 128, 32), (8, 4, 128, 16), (3, 5, 64, 64), (5, 16, 64, 32), (2, 9, 256, 16),
          (1, 16, 256, 64), (4, 1, 256, 32), (7, 2, 128, 64), (12, 12, 128, 16)]


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "fp16"])
@pytest.mark.parametrize("Hkv,G,D,T", SHAPES)
def test_ragged_batches(Hkv, G, D, T, dtype):
    c = Case([1, 0, 17, 16, 64, 65, 500, 3, 0, 129, 1000, 15], Hkv, G, D, T, dtype, lent=0.4, seed=Hkv * D + G, stray=float("nan"))
    c.run()
    c.check()


@pytest.mark.parametrize("lens", [[1], [0], [0, 0, 0], [16], [63], [2047], [5000], [1] * 300, list(range(0, 400)), [4000, 1, 0, 4000], [1, 5000]],
                         ids=lambda x: f"{len(x)}x{max(x)}")
@pytest.mark.parametrize("Hkv,G,D,T", [(8, 4, 128, 16), (1, 2, 64, 64), (2, 12, 256, 32)])
def test_lengths(lens, Hkv, G, D, T):
    c = Case(lens, Hkv, G, D, T, BF, lent=0.2, seed=len(lens), stray=float("inf"))
    c.run()
    c.check()


@pytest.mark.parametrize("window", [1, 15, 16, 17, 33, 500, 10 ** 6])
@pytest.mark.parametrize("Hkv,G,D,T", [(2, 4, 128, 16), (3, 1, 64, 64), (1, 16, 256, 16)])
def test_windows_leave_earlier_blocks_alone(window, Hkv, G, D, T):
    c = Case([700, 1, 0, 16, 40, 333, 1200], Hkv, G, D, T, HF, seed=window, stray=float("nan"))
    for i, n in enumerate(c.lens):                               # what lies before the window: freed blocks, and garbage in its first one
        lo = max(0, n - window)
        c.tables[i, :lo // T] = -5
        if lo % T and lo // T < ceil_div(n, T):
            c.local[int(c.table_np[i, lo // T])][:, :lo % T] = float("nan")
    c.run(window=window)
    c.check()


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "fp16"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("Hkv,G,D,T", [(1, 1, 64, 16), (4, 2, 128, 16), (8, 4, 128, 32), (2, 8, 128, 64), (3, 5, 256, 16), (2, 3, 64, 32), (1, 8, 256, 64)])
def test_differential(Hkv, G, D, T, norm, dtype):
    c = Case([1, 0, 17, 16, 64, 300, 2, 1111, 0], Hkv, G, D, T, dtype, lent=0.3, seed=G * D, diff=True, stray=float("nan"))
    c.run(norm=norm, out_scale=0.7 if norm else 1.0)
    c.check()


@pytest.mark.parametrize("window", [1, 20, 1000])
def test_differential_windows(window):
    c = Case([1, 0, 170, 900, 33], 4, 2, 128, 16, BF, seed=window, diff=True, stray=float("nan"))
    c.run(window=window)
    c.check()


@pytest.mark.parametrize("n,hi,Hkv", [(700, 60, 4), (3000, 70, 4), (400, 300, 8), (900, 400, 3)])
def test_many_short_sequences(n, hi, Hkv):
    lens = np.random.default_rng(n).integers(0, hi, n).tolist()
    for diff in (False, True):
        c = Case(lens, Hkv, 2, 128, 16, BF, lent=0.3, seed=n, diff=diff)
        c.run()
        c.check()


@pytest.mark.parametrize("scale", [0.0, -0.0, -0.11, -3.0, 1e-30])
def test_scales_of_either_sign_and_of_zero(scale):
    for diff in (False, True):
        c = Case([40, 1, 0, 513], 2, 3, 128, 16, BF, seed=11, diff=diff)
        c.scale = scale
        c.run(norm=False)
        c.check()


def test_equal_maps_cancel_exactly():
    """q1 = q2, K1 = K2 and a weight of 1: both maps are the same arithmetic, so nothing is left of any row."""
    c = Case([5, 700, 64], 4, 2, 128, 16, BF, diff=True)
    k = c.local[:, 0].view(-1, 16, 4, 2, 64)
    k[..., 1, :] = k[..., 0, :].clone()
    c.q[:, 1::2] = c.q[:, 0::2].clone()
    c.lam.fill_(1.0)
    c.run(norm=False)
    assert not c.out[:3].any()


def test_peaked_scores_and_large_values():
    """Scores of a few hundred: one key takes all the weight, the others underflow."""
    for diff in (False, True):
        c = Case([900, 33, 1], 2, 4, 128, 16, BF, seed=4, diff=diff, qscale=40.0)
        c.run(norm=False, out_scale=1.0)
        for i, n in enumerate(c.lens):                           # the row of the largest score, unrounded: checked where it leads by far
            k, v = logical_rows(c.local, c.lent, c.table_np[i], n, c.T)
            assert torch.isfinite(c.out[i]).all()
            assert float(c.out[i].double().abs().max()) <= 2 * float(v.abs().max()) * (1 + 2.0 ** -7)
        if not diff:
            c.check()


def test_repeated_calls_are_bit_identical_and_independent_of_the_order_of_ctas():
    c = Case([3000, 77, 1500, 0, 2999], 8, 4, 128, 16, BF, lent=0.5, seed=8)
    c.run()
    first = c.out.clone(), c.lse.clone()
    for _ in range(20):
        c.out.fill_(7.0)
        c.run()
        assert torch.equal(c.out, first[0]) and torch.equal(c.lse, first[1])


def test_one_workspace_serves_calls_of_other_shapes_in_order():
    big = Case([4000, 100, 900], 8, 16, 256, 16, BF, seed=1)
    others = [Case([50, 2000], 2, 1, 64, 32, HF, seed=2), Case([5000], 1, 2, 128, 16, BF, seed=3), Case([700, 700], 4, 8, 256, 16, BF, seed=4, diff=True)]
    for c in others + [big] + others:
        c.work = big.work
        c.out.fill_(7.0)
        c.run()
        c.check()


def test_shared_blocks_of_a_common_prefix():
    """Several sequences read the same blocks."""
    c = Case([640, 10, 10], 2, 4, 128, 16, BF, seed=5)
    c.table_np[1:, :40] = c.table_np[0, :40]
    c.lens = [640, 320, 639]
    c.tables.copy_(torch.from_numpy(c.table_np).to(torch.int32))
    c.lens_t = gpu(c.lens)
    c.run()
    c.check()


def test_a_captured_call_follows_tables_and_lengths():
    c = Case([1500, 800, 3, 0], 4, 4, 128, 16, BF, lent=0.5, seed=6)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            assert B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, c.out[:4], c.work, lse=c.lse[:4], status=c.status,
                                         stream=torch.cuda.current_stream()) == B.OK
    c.window = 0
    for lens in ([1500, 800, 3, 0], [1, 0, 3, 0], [0, 0, 0, 0], [1499, 700, 2, 0], [1500, 800, 3, 0]):
        c.lens_t.copy_(gpu(lens))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        c.lens = lens
        c.check()
        assert int(c.status) == 0 and not c.work[:32768].any()


def test_blocks_apart_and_offsets_beyond_32_bits():
    """A cache of 5 GB in which the sequences' blocks lie at the far end."""
    T, Hkv, D = 16, 8, 128
    blocks = 80000                                               # 64 KB each
    arena = torch.zeros((blocks, 2, T, Hkv, D), dtype=BF, device="cuda")
    c = Case([200, 33], Hkv, 2, D, T, BF, seed=7)
    far = blocks - c.sizes[0]
    arena[far:] = c.local
    c.local, c.table_np = arena, c.table_np + far
    c.table_np[c.table_np > blocks] = 0x7fffffff
    c.tables.copy_(torch.from_numpy(c.table_np).to(torch.int32))
    c.cache = B.PagedCache(arena)
    c.run()
    c.check()
    slots = gpu([(blocks - 1) * T + 3], torch.int64)             # and a row written there
    row = torch.randn((1, Hkv, D), device="cuda").to(BF)
    torch.cuda.synchronize()
    assert B.paged_write_kv(c.cache, row, -row, slots, c.status) == B.OK
    t = np.array([blocks - 1])
    k, v = logical_rows(arena, None, t, 4, T)
    assert torch.equal(k[3], row[0].double()) and torch.equal(v[3], -row[0].double())
    # the same blocks through an arena whose blocks are twice as far apart
    c2 = Case([200, 33], Hkv, 2, D, T, BF, seed=7)
    wide = torch.zeros((c2.sizes[0], 4, T, Hkv, D), dtype=BF, device="cuda")
    wide[:, :2] = c2.local
    wide[:, 2:] = float("nan")
    c2.local = wide[:, :2]
    c2.cache = B.PagedCache(c2.local)
    c2.run()
    c2.check()


def test_lengths_out_of_range_give_empty_rows_and_a_status():
    c = Case([100, 50, 20], 2, 4, 128, 16, BF, seed=9)
    c.run()
    good = c.out[:3].clone()
    c.lens_t.copy_(gpu([100, -3, c.width * 16 + 1]))
    torch.cuda.synchronize()
    assert B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, c.out[:3], c.work, lse=c.lse[:3], status=c.status) == B.OK
    torch.cuda.synchronize()
    assert int(c.status) == B.EINVAL
    assert torch.equal(c.out[0], good[0]) and not c.out[1:3].any() and (c.lse[1:3] == -math.inf).all()


def test_entries_outside_the_cache_read_as_zeros_and_are_reported():
    c = Case([100, 50, 20], 2, 4, 128, 16, BF, lent=0.5, seed=9)
    c.run()
    good = c.out[:3].clone()
    for bad in (c.sizes[0], ~c.sizes[1], 0x7fffffff, -0x80000000):
        c.tables[1, 2] = bad
        c.status.zero_()
        torch.cuda.synchronize()
        assert B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, c.out[:3], c.work, status=c.status) == B.OK
        torch.cuda.synchronize()
        assert int(c.status) == B.EINVAL
        assert torch.equal(c.out[0], good[0]) and torch.equal(c.out[2], good[2]) and torch.isfinite(c.out[1]).all()
    one = Case([100], 2, 4, 128, 16, BF, seed=9)                  # a cache without a second arena
    one.tables[0, 3] = -1
    torch.cuda.synchronize()
    assert B.paged_decode_tables(one.cache, one.tables, one.lens_t, one.q, one.scale, one.out[:1], one.work, status=one.status) == B.OK
    torch.cuda.synchronize()
    assert int(one.status) == B.EINVAL


def test_infinite_scores_of_attended_keys():
    """A key whose score is minus infinity has no weight; where all are, the row is zero and its log-sum-exp minus infinity."""
    c = Case([40, 20], 1, 1, 64, 16, BF, seed=3)
    c.q.abs_()
    e = int(c.table_np[0, 1])
    c.local[e, 0, 3, 0, :] = -float("inf")
    for j in range(2):
        c.local[int(c.table_np[1, j]), 0, :, 0, :] = -float("inf")
    c.run()
    k, v = logical_rows(c.local, None, c.table_np[0], 40, 16)
    ref, lse, _ = attend(c.q[0].double(), k, v, c.scale)
    assert float((c.out[0].double() - ref).abs().max()) <= 2.0 ** -7 and abs(float(c.lse[0, 0]) - float(lse)) < 1e-4
    assert not c.out[1].any() and float(c.lse[1, 0]) == -math.inf


def test_a_serving_loop_of_all_calls_together():
    """Requests come, grow and finish: tables, rows and attention on one stream, against dense 64-bit caches."""
    n, T, Hkv, G, D, width = 6, 16, 2, 3, 64, 20
    rng = np.random.default_rng(0)
    gen = torch.Generator(device="cuda").manual_seed(0)
    arenas = [torch.full((b, 2, T, Hkv, D), float("nan"), dtype=BF, device="cuda") for b in (12, 40)]
    cache = B.PagedCache(*arenas)
    free, work, status = gpu([12, 40]), gpu([0]), gpu([0])
    pool = B.PagedPool(gpu(list(range(12))), gpu(list(range(40))), free, free, work)
    tables = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    ws = torch.zeros(B.paged_decode_workspace(cache, Hkv * G * 2), dtype=torch.uint8, device="cuda")
    lens = [0] * n
    dense = [[] for _ in range(n)]
    s = torch.cuda.Stream()
    for step in range(25):
        new = [0 if (x and rng.random() < 0.1) else x + 1 if x else int(rng.integers(0, 90)) for x in lens]
        grown = sum(max(0, b - a) for a, b in zip(lens, new))
        room = grown + 5
        k = torch.randn((room, Hkv, D), device="cuda", generator=gen).to(BF)
        v = torch.randn((room, Hkv, D), device="cuda", generator=gen).to(BF)
        q = torch.randn((n, Hkv * G * 2, D // 2), device="cuda", generator=gen).to(BF)
        lam = torch.full((Hkv * G,), 0.5, device="cuda")
        offsets, slots, positions = gpu([0] * (n + 1)), torch.zeros(room, dtype=torch.int64, device="cuda"), gpu([0] * room)
        out, out2, lens_t, new_t = (torch.zeros((n, Hkv * G, D), dtype=BF, device="cuda"), torch.zeros((n, Hkv * G, D), dtype=BF, device="cuda"),
                                    gpu(lens), gpu(new))
        q1 = q.reshape(n, Hkv * G, D)
        s.wait_stream(torch.cuda.current_stream())
        assert B.paged_build_tables(pool, lens_t, new_t, T, tables, offsets, slots, positions, status, s) == B.OK
        assert B.paged_write_kv(cache, k, v, slots, status, s) == B.OK
        assert B.paged_decode_tables(cache, tables, new_t, q1, 0.125, out, ws, status=status, stream=s) == B.OK
        assert B.paged_decode_diff(cache, tables, new_t, q, lam, 0.2, out2, ws, status=status, stream=s) == B.OK
        torch.cuda.synchronize()
        assert int(status) == 0
        at = 0
        for i in range(n):
            if new[i] < lens[i]:
                dense[i] = dense[i][:new[i]]
            for _ in range(max(0, new[i] - lens[i])):
                dense[i].append((k[at].double(), v[at].double()))
                at += 1
            if not new[i]:
                assert not out[i].any() and not out2[i].any()
                continue
            kk, vv = torch.stack([x[0] for x in dense[i]]), torch.stack([x[1] for x in dense[i]])
            ref, _, size = attend(q1[i].double(), kk, vv, 0.125)
            ok, worst = close(out[i], ref, row_error(new[i], D, size, float(vv.abs().max())), torch.finfo(BF).eps)
            assert ok, (step, i, worst)
            o1, _, s1 = attend(q[i, 0::2].double(), kk[..., :D // 2], vv, 0.2)
            o2, _, s2 = attend(q[i, 1::2].double(), kk[..., D // 2:], vv, 0.2)
            e = row_error(new[i], D, max(s1, s2), float(vv.abs().max())) * 1.5 + 2.0 ** -22 * float(vv.abs().max())
            ok, worst = close(out2[i], o1 - 0.5 * o2, e, torch.finfo(BF).eps)
            assert ok, (step, i, worst)
        lens = new
    assert free.tolist()[0] + free.tolist()[1] + sum(ceil_div(x, T) for x in lens) == 52


FIRST_CALLS = """
import torch
from paper_2609_27040_b200 import binding as B
i32, bf = torch.int32, torch.bfloat16
dev = "cuda"
gen = torch.Generator(device=dev).manual_seed(1)
arena = torch.zeros((8, 2, 16, 2, 64), dtype=bf, device=dev)
cache = B.PagedCache(arena)
free, free_out, work = torch.tensor([8, 0], dtype=i32, device=dev), torch.zeros(2, dtype=i32, device=dev), torch.zeros(1, dtype=i32, device=dev)
pool = B.PagedPool(torch.arange(8, dtype=i32, device=dev), None, free, free_out, work)
lens, new = torch.zeros(2, dtype=i32, device=dev), torch.tensor([40, 3], dtype=i32, device=dev)
tables, offsets = torch.full((2, 4), -1, dtype=i32, device=dev), torch.zeros(3, dtype=i32, device=dev)
slots, positions = torch.zeros(50, dtype=torch.int64, device=dev), torch.zeros(50, dtype=i32, device=dev)
k, v = (torch.randn((50, 2, 64), device=dev, generator=gen).to(bf) for _ in range(2))
q, q2, lam = torch.randn((2, 4, 64), device=dev, generator=gen).to(bf), torch.randn((2, 8, 32), device=dev, generator=gen).to(bf), torch.full((4,), 0.3, device=dev)
out, out2 = torch.zeros((2, 4, 64), dtype=bf, device=dev), torch.zeros((2, 4, 64), dtype=bf, device=dev)
ws = torch.zeros(B.paged_decode_workspace(cache, 8), dtype=torch.uint8, device=dev)
def step(stream):
    assert B.paged_build_tables(pool, lens, new, 16, tables, offsets, slots, positions, stream=stream) == B.OK
    assert B.paged_write_kv(cache, k, v, slots, stream=stream) == B.OK
    assert B.paged_decode_tables(cache, tables, new, q, 0.125, out, ws, stream=stream) == B.OK
    assert B.paged_decode_diff(cache, tables, new, q2, lam, 0.2, out2, ws, stream=stream) == B.OK
torch.cuda.synchronize()
s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=s):
    step(torch.cuda.current_stream())
torch.cuda.synchronize()
assert not out.any() and not arena.any()
g.replay()
torch.cuda.synchronize()
got = out.clone(), out2.clone(), slots.clone(), arena.clone()
assert out.any() and out2.any() and offsets.tolist() == [0, 40, 43]
for t in (out, out2, slots, arena):
    t.zero_()
step(None)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (out, out2, slots, arena)))
print("the same")
"""


def test_the_very_first_calls_of_a_process_may_be_captured():
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "the same" in r.stdout, r.stderr[-2000:]


def test_two_streams_at_once_with_workspaces_of_their_own():
    cases = [Case([3000, 10, 700], 8, 4, 128, 16, BF, lent=0.4, seed=k) for k in range(2)]
    alone = []
    for c in cases:
        c.run()
        alone.append((c.out.clone(), c.lse.clone()))
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(30):
        for c, s in zip(cases, streams):
            assert B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, c.out[:3], c.work, lse=c.lse[:3], status=c.status, stream=s) == B.OK
    torch.cuda.synchronize()
    for c, (o, l) in zip(cases, alone):
        assert torch.equal(c.out, o) and torch.equal(c.lse, l) and int(c.status) == 0 and not c.work[:32768].any()


def test_one_row_tables_and_queries_of_any_stride():
    """A single sequence: the strides of dimensions of length one mean nothing."""
    c = Case([77], 1, 1, 64, 16, BF, seed=1)
    q = torch.empty((1, 1, 64), dtype=BF, device="cuda").as_strided((1, 1, 64), (7, 3, 1))
    q.copy_(c.q)
    c.q = q
    c.tables = c.tables[:1].as_strided((1, c.width), (1, 1))
    c.tables.copy_(torch.from_numpy(c.table_np).to(torch.int32))
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "fp16"])
@pytest.mark.parametrize("n", [700, 100001])
def test_many_tiny_weights_beside_a_large_one(n, dtype):
    """One token of score 17.53 (bf16: 17.5) and value 0, the others of score 0 (a weight of 2^-25.3 beside it) and value 1. All terms are positive: f32
    sums of n of them are off by n 2^-23 of their size at most (numerator and denominator), a weight by 2^-16 (bf16's two numbers; and
    2^-20 for the score), and the result is rounded once; what fp16 loses below 2^-40 of the largest weight is 2^-14 of the others'."""
    T, D = 64, 64
    local = torch.zeros((ceil_div(n, T), 2, T, 1, D), dtype=dtype, device="cuda")
    local[:, 1] = 1.0
    local[0, 1, 0] = 0.0
    x = 17.53125 if dtype is HF else 17.5                        # as the type has it
    local[0, 0, 0, 0, 0] = x
    q = torch.zeros((1, 1, D), dtype=dtype, device="cuda")
    q[..., 0] = 1.0
    cache, tables = B.PagedCache(local), torch.arange(local.shape[0], dtype=torch.int32, device="cuda")[None]
    work = torch.zeros(B.paged_decode_workspace(cache, 1), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, 1), device="cuda")
    torch.cuda.synchronize()
    assert B.paged_decode_tables(cache, tables, gpu([n]), q, 1.0, out, work, lse=lse) == B.OK
    w = (n - 1) * math.exp(-x)
    ref = w / (1 + w)
    rel = 2 * n * 2.0 ** -23 + 2.0 ** -14 + 2.0 ** -15 + torch.finfo(dtype).eps / 2
    # fp16 below 2^-14 are multiples of 2^-24: there (n = 700, 1.7e-5) the rounding is off by up to 2^-25, whatever the value
    least = 2.0 ** -25 if dtype is HF else 0.0
    assert float((out.double() - ref).abs().max()) <= rel * ref + least, (float(out[0, 0, 0]), ref)
    assert abs(float(lse) - (x + math.log1p(w))) <= lse_slack(n, D, x)


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "fp16"])
@pytest.mark.parametrize("D,T", [(64, 16), (128, 16), (256, 64)])
@pytest.mark.parametrize("n", [1, 100, 3000])
def test_scores_beyond_what_f32_counts_in_ones(n, D, T, dtype):
    """Scores around 2^38, apart by 2^30 and more: the largest has all the weight, exactly."""
    rng = np.random.default_rng(n + D)
    top = 2.0 ** 16 if dtype is BF else 2.0 ** 14
    steps = rng.integers(1, 120, n)                              # of 128: both types have them
    best, least = rng.permutation(n)[:2] if n > 1 else (0, 0)
    steps[least], steps[best] = 0, 127
    nb = ceil_div(n, T)
    rows = torch.zeros(nb * T, dtype=torch.float64)
    rows[:n] = torch.from_numpy(top * (1 + steps / 128))
    local = torch.randn((nb, 2, T, 1, D), device="cuda").to(dtype)
    local[:, 0] = rows.to("cuda").to(dtype).reshape(nb, T, 1, 1)
    cache, tables = B.PagedCache(local), torch.arange(nb, dtype=torch.int32, device="cuda")[None]
    v = logical_rows(local, None, np.arange(nb), n, T)[1]
    q = torch.full((1, 2, D), top, dtype=dtype, device="cuda")
    q[:, 1] = -top
    work = torch.zeros(B.paged_decode_workspace(cache, 2), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, 2), device="cuda")
    if n == 1:
        least = best
    torch.cuda.synchronize()
    for scale, heads in ((1.0, (best, least)), (-1.0, (least, best))):
        assert B.paged_decode_tables(cache, tables, gpu([n]), q, scale, out, work, lse=lse) == B.OK
        for h, t in enumerate(heads):
            assert torch.equal(out[0, h].double(), v[t, 0])
            score = (1 - 2 * h) * scale * D * top * float(rows[t])
            assert abs(float(lse[0, h]) - score) <= 2.0 ** -21 * abs(score)   # log2(e), the product with it and with ln 2: a few roundings
    half = D // 2
    qd = torch.full((1, 2, half), top, dtype=dtype, device="cuda")
    qd[:, 1] = -top
    od, lam = torch.empty((1, 1, D), dtype=dtype, device="cuda"), torch.tensor([0.5], device="cuda")
    torch.cuda.synchronize()
    assert B.paged_decode_diff(cache, tables, gpu([n]), qd, lam, 1.0, od, work) == B.OK
    ref = v[best, 0] - 0.5 * v[least, 0]                         # f32: a rounding of the difference, then the output's
    assert bool(((od[0, 0].double() - ref).abs() <= (torch.finfo(dtype).eps / 2 + 2.0 ** -22) * ref.abs() + 2.0 ** -22 * v.abs().max()).all())


def test_calls_behind_slow_kernels_copies_and_joined_streams():
    """Every call waits for what comes before it, eager and captured: its inputs are written by a long kernel, by a copy, by another
    stream, and what it wrote is read and overwritten right behind it."""
    c = Case([600, 0, 1300], 4, 4, 128, 16, BF, lent=0.3, seed=2)
    c.run()
    want = c.out[:3].clone()
    qs, lens = c.q.clone(), c.lens_t.clone()
    q = torch.zeros_like(qs)
    big = torch.ones(200_000_000, device="cuda")                 # a kernel of some 0.2 ms on it
    out = torch.empty_like(want)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()

    def step(results):
        def decode():
            assert B.paged_decode_tables(c.cache, c.tables, c.lens_t, q, c.scale, out, c.work, status=c.status, stream=torch.cuda.current_stream()) == B.OK
        q.zero_()
        c.lens_t.zero_()
        big.mul_(1.0)
        q.copy_(qs)                                              # a kernel or a copy
        c.lens_t.copy_(lens)
        decode()
        results[0].copy_(out)
        out.fill_(3.0)
        q.zero_()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            big.mul_(1.0)
            q.copy_(qs)
        main.wait_stream(side)                                   # right behind another stream's work
        decode()
        decode()                                                 # and behind itself, with the same workspace
        results[1].copy_(out)
        side.wait_stream(main)                                   # work that overlaps with the next call on the other stream
        with torch.cuda.stream(side):
            big.mul_(1.0)
        c.lens_t.zero_()
        decode()
        results[2].copy_(out)
        c.lens_t.copy_(lens)
        main.wait_stream(side)

    results = [torch.zeros_like(want) for _ in range(3)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(main):
        step(results)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=main):
        step(results)
    for k in range(6):
        if k:
            for r in results:
                r.fill_(-1.0)
            torch.cuda.synchronize()
            if k % 2:
                graph.replay()
            else:
                with torch.cuda.stream(main):
                    step(results)
            torch.cuda.synchronize()
        assert torch.equal(results[0], want) and torch.equal(results[1], want) and not results[2].any()
    assert int(c.status) == 0 and not c.work[:32768].any()


@pytest.mark.parametrize("diff", [False, True], ids=["plain", "diff"])
@pytest.mark.parametrize("lens,Hkv,G,D,T", [
    ([20000], 1, 2, 128, 16),                                    # one item in dozens of parts: more than one level of sums
    ([9000], 3, 8, 64, 64),
    ([3000, 50, 4000, 1, 700, 0, 2500, 390], 1, 3, 128, 32),     # items that end where others begin
    ([384, 385, 383, 400, 767, 768, 769, 1, 5], 2, 1, 128, 16),  # around the least piece and twice that
    ([6000, 40, 5000], 2, 7, 256, 16),
    ([700, 1500, 20, 2600, 0, 0, 1100, 333, 64], 7, 1, 64, 16),
    ([14000, 13000], 8, 1, 256, 64),                             # few items, but long ones: by tickets
])
def test_few_items(lens, Hkv, G, D, T, diff):
    c = Case(lens, Hkv, G, D, T, BF, lent=0.3, seed=sum(lens) % 97, diff=diff, stray=float("nan"))
    c.run()
    c.check()
    again = c.out.clone()
    for _ in range(3):
        c.run()
        assert torch.equal(c.out, again)
    c.run(window=1000)
    c.check()


@pytest.mark.parametrize("seed", range(12))
def test_random_batches_of_few_items(seed):
    rng = np.random.default_rng(1000 + seed)
    n, Hkv = int(rng.integers(1, 25)), int(rng.choice([1, 2, 5, 8]))
    lens = [int(x) for x in rng.integers(0, int(rng.choice([40, 600, 3000, 9000])), n)]
    D, T, diff = int(rng.choice([64, 128, 256])), int(rng.choice([16, 32, 64])), bool(rng.integers(2))
    G = int(rng.integers(1, 9 if diff else 17))
    c = Case(lens, Hkv, G, D, T, [BF, HF][seed % 2], lent=0.25, seed=seed, diff=diff, stray=float("inf"))
    c.run()
    c.check()


@pytest.mark.parametrize("Hkv,n", [(1, 250), (2, 147), (8, 18), (64, 4), (37, 3)])
def test_short_items_on_ctas_of_their_own(Hkv, n):
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 300, n)]
    lens[n // 2] = 1600
    c = Case(lens, Hkv, 1, 64, 16, HF, lent=0.2, seed=n, stray=float("nan"))
    c.run()
    c.check()


@pytest.mark.parametrize("lens,Hkv", [([3000] * 5, 4), ([4000] * 60 + [100, 0, 3900], 8), ([300000, 200000], 4)], ids=str)
def test_a_workspace_is_whole_again_after_lengths_that_changed_under_a_call(lens, Hkv):
    """What such a call answers means nothing (its CTAs may have cut the work differently), but every access stays in bounds, every
    wait ends, and the next call is right. The lengths change around the time at which the CTAs read them."""
    n = len(lens)
    c = Case(lens, Hkv, 1, 128, 16, BF, seed=n)
    c.run()
    good = c.out[:n].clone(), c.lse[:n].clone()
    then = gpu([x // 2 + x // 5 * (i % 3) for i, x in enumerate(lens)])
    lens_t, side = c.lens_t.clone(), torch.cuda.Stream()
    hit = 0
    for k in range(300):
        c.lens_t.copy_(lens_t)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(k * 240)                           # 0 to some 40 us
            c.lens_t.copy_(then)
        assert B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, c.out[:n], c.work, lse=c.lse[:n], status=c.status) == B.OK
        torch.cuda.synchronize()
        assert int(c.status) in (0, B.EINVAL)
        hit += not torch.equal(c.out[:n], good[0])
        c.status.zero_()
        assert not c.work[:32768].any(), k
        c.lens_t.copy_(lens_t)
        c.run()
        assert torch.equal(c.out[:n], good[0]) and torch.equal(c.lse[:n], good[1])
    assert hit                                                   # the lengths did change before or under some of the calls


FIRST_CALLS_OF_THREADS = """
import threading, torch
from tests.test_gpu_paged_decode import B, BF, Case
cases = [Case([900, 33, 0, 700], 2, 3, 128, 16, BF, lent=0.4, seed=k % 2, diff=k % 4 >= 2) for k in range(8)]
streams = [torch.cuda.Stream() for _ in cases]
gate = threading.Barrier(len(cases))
torch.cuda.synchronize()
codes = []
def call(c, s):
    gate.wait()
    for _ in range(20):
        if c.diff:
            codes.append(B.paged_decode_diff(c.cache, c.tables, c.lens_t, c.q, c.lam, c.scale, c.out[:4], c.work, status=c.status, stream=s))
        else:
            codes.append(B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, c.out[:4], c.work, status=c.status, stream=s))
threads = [threading.Thread(target=call, args=x) for x in zip(cases, streams)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert codes == [B.OK] * (20 * len(cases))
for k, c in enumerate(cases):
    assert torch.equal(c.out[:4], cases[k % 4].out[:4]) and c.out[:2].any() and int(c.status) == 0
print("the same")
"""


def test_the_first_calls_of_several_threads():
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS_OF_THREADS], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "the same" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("diff", [False, True], ids=["plain", "diff"])
def test_a_thread_whose_first_use_of_the_gpu_is_the_call(diff):
    import threading
    c = Case([900, 33, 0, 700], 2, 3, 128, 16, BF, lent=0.4, seed=1, diff=diff)
    c.run(norm=False)
    want = c.out[:4].clone()
    c.out.fill_(7.0)
    torch.cuda.synchronize()
    codes = []

    def call():
        for _ in range(2):
            if diff:
                codes.append(B.paged_decode_diff(c.cache, c.tables, c.lens_t, c.q, c.lam, c.scale, c.out[:4], c.work, out_scale=c.out_scale, status=c.status))
            else:
                codes.append(B.paged_decode_tables(c.cache, c.tables, c.lens_t, c.q, c.scale, c.out[:4], c.work, status=c.status))

    t = threading.Thread(target=call)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert codes == [B.OK, B.OK] and torch.equal(c.out[:4], want) and int(c.status) == 0


@pytest.mark.parametrize("T,Hkv,G,D,dtype", [(16, 2, 3, 64, BF), (32, 4, 4, 128, HF), (16, 1, 12, 256, BF)])
def test_a_captured_serving_step_follows_the_requests(T, Hkv, G, D, dtype):
    """One graph of tables, rows, attention of both forms and the new lengths taking the old ones' place, replayed while requests come,
    grow by one or by several, fall back and finish, against dense 64-bit caches."""
    n, width, room = 7, 12, 400
    rng = np.random.default_rng(T + D)
    gen = torch.Generator(device="cuda").manual_seed(D)
    blocks = (20, 40)
    arenas = [torch.full((b, 2, T, Hkv, D), float("nan"), dtype=dtype, device="cuda") for b in blocks]
    cache = B.PagedCache(*arenas)
    free, work, status = gpu(list(blocks)), gpu([0]), gpu([0])
    pool = B.PagedPool(*(gpu(rng.permutation(b).tolist()) for b in blocks), free, free, work)
    tables = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    twice = 2 if G <= 8 else 0                                   # heads of the differential form: none beyond 8 to a KV head
    ws = torch.zeros(B.paged_decode_workspace(cache, Hkv * G * (twice or 1)), dtype=torch.uint8, device="cuda")
    lens_t, new_t, offsets = gpu([0] * n), gpu([0] * n), gpu([0] * (n + 1))
    slots, positions = torch.zeros(room, dtype=torch.int64, device="cuda"), gpu([0] * room)
    k, v = torch.zeros((room, Hkv, D), dtype=dtype, device="cuda"), torch.zeros((room, Hkv, D), dtype=dtype, device="cuda")
    q = torch.zeros((n, Hkv * G, D), dtype=dtype, device="cuda")
    qd, lam = torch.zeros((n, 2 * Hkv * G, D // 2), dtype=dtype, device="cuda"), torch.full((Hkv * G,), 0.5, device="cuda")
    out, out2, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((n, Hkv * G), device="cuda")
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        now = torch.cuda.current_stream()
        assert B.paged_build_tables(pool, lens_t, new_t, T, tables, offsets, slots, positions, status, now) == B.OK
        assert B.paged_write_kv(cache, k, v, slots, status, now) == B.OK
        assert B.paged_decode_tables(cache, tables, new_t, q, 0.125, out, ws, lse=lse, status=status, stream=now) == B.OK
        if twice:
            assert B.paged_decode_diff(cache, tables, new_t, qd, lam, 0.2, out2, ws, status=status, stream=now) == B.OK
        lens_t.copy_(new_t)
    lens, dense = [0] * n, [[] for _ in range(n)]
    finished = fell = 0
    for step in range(30):
        new = []
        for x in lens:
            kind = rng.random()
            new.append(int(rng.integers(0, 50)) if not x else 0 if kind < 0.08 else max(0, x - int(rng.integers(1, 40))) if kind < 0.16 else
                       min(x + (1 if kind < 0.8 else int(rng.integers(1, 9))), 100))
        finished += sum(a > 0 and b == 0 for a, b in zip(lens, new))
        fell += sum(a > b > 0 for a, b in zip(lens, new))
        for x in (k, v, q, qd):
            x.copy_(torch.randn(x.shape, device="cuda", generator=gen))
        new_t.copy_(gpu(new))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0 and lens_t.tolist() == new
        at = 0
        for i in range(n):
            dense[i] = dense[i][:new[i]]
            for _ in range(max(0, new[i] - lens[i])):
                dense[i].append((k[at].double(), v[at].double()))
                at += 1
            if not new[i]:
                assert not out[i].any() and not out2[i].any() and (lse[i] == -math.inf).all()
                continue
            kk, vv = torch.stack([x[0] for x in dense[i]]), torch.stack([x[1] for x in dense[i]])
            top = float(vv.abs().max())
            ref, ref_lse, size = attend(q[i].double(), kk, vv, 0.125)
            ok, worst = close(out[i], ref, row_error(new[i], D, size, top), torch.finfo(dtype).eps)
            assert ok and float((lse[i].double() - ref_lse).abs().max()) <= lse_slack(new[i], D, size), (step, i, worst)
            if twice:
                o1, _, s1 = attend(qd[i, 0::2].double(), kk[..., :D // 2], vv, 0.2)
                o2, _, s2 = attend(qd[i, 1::2].double(), kk[..., D // 2:], vv, 0.2)
                e = row_error(new[i], D, s1, top) + 0.5 * row_error(new[i], D, s2, top) + 2.0 ** -22 * top
                ok, worst = close(out2[i], o1 - 0.5 * o2, e, torch.finfo(dtype).eps)
                assert ok, (step, i, worst)
        assert at == offsets.tolist()[n] and sum(free.tolist()) + sum(ceil_div(x, T) for x in new) == sum(blocks)
        lens = new
    assert finished and fell
