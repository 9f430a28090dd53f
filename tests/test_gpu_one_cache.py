"""The host-planned and the device-driven calls on the same cache: a slice's arenas (layer-major) as PagedCaches, its tables and ids as
device arrays; rows that one path writes are read by the other."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_27040_b200 import binding as B
from paper_2609_27040_b200 import build as build_mod
from paper_2609_27040_b200 import synth
from tests.helpers import Scenario, attention_close
from tests.paged_helpers import attend, close, row_error

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def gpu(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


class Both:
    def __init__(self, wl, seed, **kw):
        from tests.gpu_helpers import GpuScenario
        self.sc = Scenario(wl, seed, slack=40, **kw)
        self.g = GpuScenario(self.sc)
        self.caches = [B.PagedCache(self.g.local[layer].view(BF), self.g.lent[layer].view(BF)) for layer in range(self.sc.L)]
        self.work = torch.zeros(B.paged_decode_workspace(self.caches[0], self.sc.Hq), dtype=torch.uint8, device="cuda")
        self.status = gpu([0])

    def tables(self):
        """The slice's block tables and lengths as device arrays."""
        rows = [self.g.s.slice_get_block_table(i) for i in self.sc.seq_ids]
        t = np.full((len(rows), max(max(len(r[1]) for r in rows), 1)), 0x7fffffff)
        for i, (rc, table, _) in enumerate(rows):
            assert rc == B.OK
            t[i, :len(table)] = table
        return gpu(t.tolist()), gpu([int(r[2]) for r in rows])

    def check(self):
        """Every layer, by both paths, against the 64-bit attention of the oracle's own arenas."""
        sc, g = self.sc, self.g
        tables, lens = self.tables()
        for layer in range(sc.L):
            rc, resolved, _ = sc.orc.gather(layer, sc.seq_ids, sc.lent, sc.staging)
            assert rc == 0
            rc, ref, ref_lse = oracle.paged_attention(sc.q[layer], sc.local[layer], sc.staging[layer % sc.wl.ring_slots], resolved, sc.lengths(),
                                                      sc.Hq, sc.Hkv, sc.D, sc.T, sc.sm_scale)
            assert rc == 0
            q = g.q[layer].view(BF).view(sc.nseq, sc.Hq, sc.D)
            host, device = torch.zeros_like(q), torch.zeros_like(q)
            lse = torch.zeros((2, sc.nseq, sc.Hq), device="cuda")
            assert g.s.prefetch_layer(layer, sc.seq_ids, g.side) == B.OK
            assert g.s.paged_decode(layer, sc.seq_ids, q, sc.Hq, float(sc.sm_scale), host, lse[0], g.main) == B.OK
            assert B.paged_decode_tables(self.caches[layer], tables, lens, q, float(sc.sm_scale), device, self.work, lse=lse[1], status=self.status,
                                         stream=g.main) == B.OK
            torch.cuda.synchronize()
            g.device_ok()
            assert int(self.status) == 0
            for out in (host, device):
                assert attention_close(out.double().cpu().numpy(), ref)[0]
            assert np.abs(lse.double().cpu().numpy() - ref_lse).max() <= 1e-3


WL = synth.Workload("both", 3, 16, 4, 5, 20, 500, 0.4)


@pytest.mark.parametrize("wl", [WL, synth.WORKLOADS["single_layer_mha"]], ids=["gqa", "mha"])
def test_both_paths_read_the_same_cache(wl):
    Both(wl, 3).check()


@pytest.mark.parametrize("writer", ["device", "host"])
def test_rows_that_one_path_writes_are_read_by_the_other(writer):
    b = Both(WL, 4)
    sc, g = b.sc, b.g
    from tests.gpu_helpers import kv_to_host, to_dev
    rng = np.random.default_rng(7)
    for i in sc.seq_ids:                                         # a token more for every sequence
        _, _, n = sc.orc.block_table(i)
        if n % sc.T == 0:
            assert sc.orc.alloc_blocks(i, 1, oracle.AUTO)[0] == 0 and g.s.slice_alloc_blocks(i, 1, B.TIER_AUTO)[0] == 0
        assert sc.orc.set_seq_len(i, n + 1) == 0 and g.s.slice_set_seq_len(i, n + 1) == 0
        sc.pl.lengths[i] = n + 1
    tables, lens = b.tables()
    last = (lens - 1).long()
    e = tables.gather(1, (last // sc.T)[:, None])[:, 0].long()
    slots = torch.where(e >= 0, e * sc.T + last % sc.T, ~(~e * sc.T + last % sc.T))
    assert bool((e >= 0).any()) and bool((e < 0).any())          # some last blocks are lent
    for layer in range(sc.L):
        k, v = (synth.normal_bf16_bits(rng, (sc.nseq, sc.Hkv, sc.D)) for _ in range(2))
        assert sc.orc.append_kv(layer, sc.seq_ids, k, v, sc.Hkv, sc.D, sc.local, sc.lent, None) == 0
        kd, vd = to_dev(k), to_dev(v)
        torch.cuda.synchronize()
        if writer == "device":
            assert B.paged_write_kv(b.caches[layer], kd.view(BF), vd.view(BF), slots, b.status, g.main) == B.OK
        else:
            assert g.s.slice_append_kv(layer, sc.seq_ids, kd, vd, g.main) == B.OK
        torch.cuda.synchronize()
    assert (kv_to_host(g.local) == sc.local).all() and (kv_to_host(g.lent) == sc.lent).all()
    b.check()


def test_requests_on_blocks_that_a_slice_gave_out():
    """Ids of a sequence that was allocated for the purpose are a device pool: requests come, are attended to and go, beside the
    slice's own sequences, and the ids are handed back."""
    b = Both(WL, 5)
    sc, g = b.sc, b.g
    n, T, held, more = 3, sc.T, 100, 6
    stacks = [g.s.slice_get_free_stack(t).tolist() for t in (B.TIER_LOCAL, B.TIER_LENT)]
    rc, _ = g.s.slice_alloc_blocks(held, 20, B.TIER_LOCAL)
    assert rc == B.OK
    assert g.s.slice_alloc_blocks(held, more, B.TIER_LENT)[0] == B.OK
    rc, entries, _ = g.s.slice_get_block_table(held)
    assert rc == B.OK
    ids = [gpu([int(e) for e in entries if e >= 0]), gpu([~int(e) for e in entries if e < 0])]
    count = [sum(e >= 0 for e in entries), sum(e < 0 for e in entries)]
    assert count == [20, more]
    before = [x.clone() for x in ids]
    free, work = gpu(count), gpu([0])
    pool = B.PagedPool(ids[0], ids[1], free, free, work)
    tables, zero, lens = gpu([[-1] * 30] * n), gpu([0] * n), gpu([17, 0, T * (20 + more) - 16 * 2])
    room = int(lens.sum())
    offsets, slots, positions = gpu([0] * (n + 1)), torch.zeros(room, dtype=torch.int64, device="cuda"), gpu([0] * room)
    layer = 1
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((room, sc.Hkv, sc.D), device="cuda", generator=gen).to(BF) for _ in range(2))
    q = torch.randn((n, sc.Hq, sc.D), device="cuda", generator=gen).to(BF)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    assert B.paged_build_tables(pool, zero, lens, T, tables, offsets, slots, positions, b.status, g.main) == B.OK
    assert B.paged_write_kv(b.caches[layer], k, v, slots, b.status, g.main) == B.OK
    assert B.paged_decode_tables(b.caches[layer], tables, lens, q, 0.1, out, b.work, status=b.status, stream=g.main) == B.OK
    torch.cuda.synchronize()
    assert int(b.status) == 0 and free.tolist() == [0, 0]
    at = offsets.tolist()
    for i, x in enumerate(lens.tolist()):
        if not x:
            assert not out[i].any()
            continue
        kk, vv = k[at[i]:at[i + 1]].double(), v[at[i]:at[i + 1]].double()
        ref, _, size = attend(q[i].double(), kk, vv, 0.1)
        assert close(out[i], ref, row_error(x, sc.D, size, float(vv.abs().max())), torch.finfo(BF).eps)[0]
    b.check()                                                    # the slice's own sequences, by both paths: as they were
    assert B.paged_build_tables(pool, lens, zero, T, tables, offsets, slots, positions, b.status, g.main) == B.OK
    torch.cuda.synchronize()
    assert int(b.status) == 0 and free.tolist() == count and all(torch.equal(x[:c], y[:c]) for x, y, c in zip(ids, before, count))
    assert g.s.slice_free_seq(held) == B.OK
    assert [sorted(g.s.slice_get_free_stack(t).tolist()) for t in (B.TIER_LOCAL, B.TIER_LENT)] == [sorted(x) for x in stacks]
