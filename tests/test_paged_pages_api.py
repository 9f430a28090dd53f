"""Refusals of the calls on several new tokens and shared blocks that need no GPU: what the C entry points and the binding check
before anything is enqueued; and that every argument reaches its field."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2609_27040_b200 import binding as B
from paper_2609_27040_b200 import build as build_mod
from tests.test_paged_api import BAD_CACHES, desc


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


P = 1 << 20                                                        # an aligned address that is never touched: these calls are refused first
VP, U64, U32, F32 = C.c_void_p, C.c_uint64, C.c_uint32, C.c_float


class Tree(C.Structure):                                           # the header's argument structs, field by field
    _fields_ = [("cache", VP), ("tables", VP), ("table_stride", U64), ("lens", VP), ("offsets", VP), ("q", VP), ("q_stride", U64), ("out", VP),
                ("out_stride", U64), ("lse", VP), ("mask", VP), ("mask_stride", U64), ("positions", VP), ("work", VP), ("work_bytes", U64),
                ("status", VP), ("nseq", U32), ("max_blocks", U32), ("ntok", U32), ("heads", U32), ("mask_words", U32), ("window", U32), ("scale", F32)]


class Keep(C.Structure):
    _fields_ = [("layers", VP), ("tables", VP), ("table_stride", U64), ("lens", VP), ("keep", VP), ("keep_stride", U64), ("counts", VP),
                ("status", VP), ("nlayers", U32), ("nseq", U32), ("max_blocks", U32), ("max_keep", U32)]


class Copy(C.Structure):
    _fields_ = [("layers", VP), ("copies", VP), ("status", VP), ("nlayers", U32), ("ncopies", U32)]


class Fork(C.Structure):
    _fields_ = [("pool", VP), ("shares", VP), ("lens", VP), ("new_lens", VP), ("tables", VP), ("table_stride", U64), ("src", VP), ("dst", VP),
                ("copies", VP), ("status", VP), ("nseq", U32), ("nfork", U32), ("T", U32), ("max_blocks", U32)]


class Free(C.Structure):
    _fields_ = [("pool", VP), ("shares", VP), ("lens", VP), ("new_lens", VP), ("tables", VP), ("table_stride", U64), ("status", VP), ("nseq", U32),
                ("T", U32), ("max_blocks", U32)]


class Compact(C.Structure):
    _fields_ = [("pool", VP), ("shares", VP), ("limits", VP), ("lens", VP), ("tables", VP), ("table_stride", U64), ("copies", VP), ("status", VP),
                ("nseq", U32), ("max_copies", U32), ("T", U32), ("max_blocks", U32)]


def call(name, args):
    return getattr(B.lib(), name)(C.cast(C.byref(args), C.c_char_p), None)


def tree(d, **kw):
    a = dict(cache=C.addressof(d), tables=P, table_stride=10, max_blocks=10, lens=P, offsets=P, nseq=2, q=P, q_stride=32 * 256, heads=32, scale=1.0,
             out=P, out_stride=32 * 256, work=P, work_bytes=1 << 30, ntok=9)
    a.update(kw)
    return call("paged_tree_attention", Tree(**a))


def pool_desc(**kw):
    d = B.PagedPoolDesc()
    d.ids[0], d.capacity[0], d.free_in, d.free_out, d.work = P, 9, P, P, P
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(d, k)[v[0]] = v[1]
        else:
            setattr(d, k, v)
    return d


def shares_desc(**kw):
    d = B.PagedSharesDesc()
    d.refs[0], d.blocks[0], d.work, d.work_bytes = P, 9, P, 1 << 20
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(d, k)[v[0]] = v[1]
        else:
            setattr(d, k, v)
    return d


def pages(name, cls, pool=None, shares=None, **kw):
    pool, shares = pool or pool_desc(), shares or shares_desc()
    a = dict(pool=C.addressof(pool), shares=C.addressof(shares), lens=P, tables=P, table_stride=10, max_blocks=10, T=16, nseq=3)
    a.update({"paged_fork": dict(new_lens=P, src=P, dst=P, copies=P, nfork=2), "paged_free": dict(new_lens=P),
              "paged_compact": dict(limits=P, copies=P, max_copies=4)}[name])
    a.update(kw)
    return call(name, cls(**a))


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_that_are_refused(bad):
    d = desc(**bad)
    out = C.c_uint64(0)
    assert tree(d) == B.EINVAL
    assert B.lib().paged_tree_workspace(C.byref(d), 32, C.byref(out)) == B.EINVAL
    assert call("paged_copy_blocks", Copy(layers=C.addressof(d), copies=P, nlayers=1, ncopies=1)) == B.EINVAL
    assert call("paged_keep_rows", Keep(layers=C.addressof(d), tables=P, table_stride=9, lens=P, keep=P, keep_stride=4, counts=P, nlayers=1, nseq=1,
                                        max_blocks=9, max_keep=4)) == B.EINVAL


@pytest.mark.parametrize("kw", [dict(cache=None), dict(heads=0), dict(heads=12), dict(heads=8 * 129), dict(tables=None), dict(lens=None), dict(offsets=None),
                                dict(q=None), dict(out=None), dict(work=None), dict(q_stride=32 * 256 - 16), dict(out_stride=32 * 256 + 8), dict(q=P + 8),
                                dict(out=P + 4), dict(work=P + 8), dict(tables=P + 2), dict(offsets=P + 1), dict(lse=P + 2), dict(status=P + 2),
                                dict(positions=P + 2), dict(max_blocks=0), dict(table_stride=9), dict(max_blocks=1 << 28, table_stride=1 << 28), dict(ntok=1 << 31),
                                dict(nseq=(1 << 31) - 1), dict(mask=P), dict(mask=P, mask_words=2, mask_stride=1), dict(mask=P + 4, mask_words=1, mask_stride=1),
                                dict(mask_words=1, mask_stride=1), dict(mask=P, mask_words=1, mask_stride=1 << 40)])
def test_tree_calls_that_are_refused(kw):
    assert tree(desc(), **kw) == B.EINVAL


def test_workspaces():
    d, out = desc(), C.c_uint64(0)
    assert B.lib().paged_tree_workspace(C.byref(d), 32, C.byref(out)) == B.OK
    assert tree(d, work_bytes=out.value - 1) == B.ESCRATCH
    for heads in (0, 12, 8 * 129):
        assert B.lib().paged_tree_workspace(C.byref(d), heads, C.byref(out)) == B.EINVAL
    for b in ((9, 0), (1000, 33), (0, 1)):
        assert B.paged_shares_workspace(*b) >= 4 * sum(b) + sum(-(-x // 32) for x in b) * 4
    s = shares_desc(work_bytes=B.paged_shares_workspace(9, 0) - 1)
    for name, cls in (("paged_fork", Fork), ("paged_free", Free), ("paged_compact", Compact)):
        assert pages(name, cls, shares=s) == B.ESCRATCH
    with pytest.raises(B.SliceError):
        B.paged_shares_workspace(1 << 31, 0)


def test_calls_without_work_are_answered_before_a_device_is_looked_for():
    assert tree(desc(), nseq=0) == B.OK and tree(desc(), ntok=0) == B.OK
    d = desc()
    assert call("paged_copy_blocks", Copy(layers=C.addressof(d), nlayers=1)) == B.OK
    assert call("paged_keep_rows", Keep(layers=C.addressof(d), nlayers=1)) == B.OK


@pytest.mark.parametrize("name,cls", [("paged_fork", Fork), ("paged_free", Free), ("paged_compact", Compact)])
def test_calls_on_shared_blocks_that_are_refused(name, cls):
    for kw in (dict(pool=None), dict(shares=None), dict(lens=None), dict(tables=None), dict(lens=P + 2), dict(tables=P + 1), dict(T=8), dict(T=0),
               dict(max_blocks=0), dict(table_stride=9), dict(max_blocks=1 << 28, table_stride=1 << 28), dict(nseq=(1 << 31) - 1), dict(status=P + 2)):
        if kw in (dict(pool=None), dict(shares=None)):
            a = cls(pool=C.addressof(pool_desc()), shares=C.addressof(shares_desc()), lens=P, tables=P, table_stride=10, max_blocks=10, T=16, nseq=3)
            setattr(a, next(iter(kw)), None)
            assert call(name, a) == B.EINVAL
        else:
            assert pages(name, cls, **kw) == B.EINVAL, kw
    for bad in (dict(free_in=None), dict(free_out=None), dict(work=None), dict(ids=(0, None)), dict(capacity=(1, 4)), dict(free_out=P + 4),
                dict(free_in=P + 2), dict(work=P + 2), dict(capacity=(0, 1 << 31))):
        assert pages(name, cls, pool=pool_desc(**bad)) == B.EINVAL, bad
    for bad in (dict(refs=(0, None)), dict(blocks=(1, 4)), dict(blocks=(0, 1 << 31)), dict(refs=(0, P + 2)), dict(work=None), dict(work=P + 2)):
        assert pages(name, cls, shares=shares_desc(**bad)) == B.EINVAL, bad
    more = {"paged_fork": (dict(new_lens=None), dict(src=None), dict(dst=None), dict(copies=None), dict(copies=P + 2), dict(nseq=262145), dict(nseq=0),
                           dict(nfork=1 << 31)),
            "paged_free": (dict(new_lens=None), dict(new_lens=P + 2)),
            "paged_compact": (dict(limits=None), dict(limits=P + 2), dict(copies=None), dict(copies=P + 1), dict(max_copies=1 << 31))}[name]
    for kw in more:
        assert pages(name, cls, **kw) == B.EINVAL, kw


def test_layers_that_are_refused():
    good = [desc(), desc(base=(0, 2 << 20))]
    bad = [desc(dtype=1), desc(num_kv_heads=4), desc(head_dim=64), desc(block_tokens=32), desc(blocks=(0, 5)), desc(block_stride=(0, 65536 + 16)),
           desc(base=(0, 0))]
    for other in bad:
        arr = (B.PagedCacheDesc * 2)(good[0], other)
        assert call("paged_copy_blocks", Copy(layers=C.addressof(arr), copies=P, nlayers=2, ncopies=1)) == B.EINVAL
    arr = (B.PagedCacheDesc * 129)(*[good[0]] * 129)
    for n in (0, 129):
        assert call("paged_copy_blocks", Copy(layers=C.addressof(arr), copies=P, nlayers=n, ncopies=1)) == B.EINVAL
    for kw in (dict(copies=None), dict(copies=P + 2), dict(status=P + 1), dict(ncopies=1 << 31)):
        assert call("paged_copy_blocks", Copy(**{**dict(layers=C.addressof(arr), copies=P, nlayers=2, ncopies=1), **kw})) == B.EINVAL
    for kw in (dict(tables=None), dict(lens=None), dict(keep=None), dict(counts=None), dict(keep_stride=3), dict(table_stride=8), dict(max_blocks=0),
               dict(max_keep=1 << 31), dict(keep=P + 2), dict(status=P + 2), dict(nseq=1 << 31)):
        a = dict(layers=C.addressof(arr), tables=P, table_stride=9, lens=P, keep=P, keep_stride=4, counts=P, nlayers=2, nseq=1, max_blocks=9, max_keep=4)
        assert call("paged_keep_rows", Keep(**{**a, **kw})) == B.EINVAL, kw


class Caught:
    """Stands in for the library's entry points: keeps the structs that the binding hands over."""

    def __enter__(self):
        self.calls, self.refs = B._torch_calls(), []
        for cls in (Tree, Keep, Copy, Fork, Free, Compact):
            def entry(args, stream, cls=cls):
                self.args, self.stream = cls.from_buffer_copy(C.string_at(args, C.sizeof(cls))), stream
                return 17
            self.refs.append(C.CFUNCTYPE(C.c_int, VP, VP)(entry))
        self.calls.bind_more(*(C.cast(f, VP).value for f in self.refs))
        return self

    def __exit__(self, *_):
        B._calls = None                                            # bound to the library again by the next call


def world():
    bf, i32 = torch.bfloat16, torch.int32
    z = lambda *s: torch.zeros(s, dtype=i32)                       # noqa: E731
    w = dict(arena=torch.zeros((3, 4, 2, 32, 2, 64), dtype=bf), ids=z(9), free=z(2), free_out=z(2), work=z(1), refs=z(4),
             share_work=torch.zeros(B.paged_shares_workspace(4, 0), dtype=torch.uint8), lens=z(3), new=z(3), tables=z(3, 11)[:, :7], offsets=z(4),
             src=z(5), dst=z(5), copies=z(5, 3), status=z(1), limits=z(2), counts=z(3), keep=z(3, 8)[:, :6], positions=z(9))
    w["caches"] = [B.PagedCache(w["arena"][i]) for i in range(3)]
    w["layers"] = B.PagedLayers(w["caches"])
    w["pool"] = B.PagedPool(w["ids"], None, w["free"], w["free_out"], w["work"])
    w["shares"] = B.PagedShares(w["refs"], None, w["share_work"])
    w["q"], w["out"] = torch.zeros((9, 8, 64), dtype=bf)[:, 1:7], torch.zeros((9, 6, 64), dtype=bf)
    w["mask"], w["lse"], w["ws"] = torch.zeros((9, 5), dtype=torch.int64)[:, :2], torch.zeros((9, 6)), torch.zeros(77)
    return w


def test_every_argument_reaches_its_field():
    w = world()
    ptr = {k: v.data_ptr() for k, v in w.items() if isinstance(v, torch.Tensor)}
    common = dict(pool=w["pool"]._addr, shares=w["shares"]._addr, lens=ptr["lens"], tables=ptr["tables"], table_stride=11, max_blocks=7, T=32, nseq=3,
                  status=ptr["status"])

    class Stream:
        cuda_stream = 0x7f0012345678

    def fields(a):
        return {name: getattr(a, name) for name, _ in a._fields_}

    with Caught() as got:
        assert B.paged_tree_attention(w["caches"][0], w["tables"], w["lens"], w["offsets"], w["q"], 0.25, w["out"], w["ws"], mask=w["mask"], lse=w["lse"],
                                      window=9, positions=w["positions"], status=w["status"], stream=Stream()) == 17
        assert fields(got.args) == dict(cache=w["caches"][0]._addr, tables=ptr["tables"], table_stride=11, lens=ptr["lens"], offsets=ptr["offsets"],
                                        q=ptr["q"], q_stride=1024, out=ptr["out"], out_stride=768, lse=ptr["lse"], mask=ptr["mask"], mask_stride=5,
                                        positions=ptr["positions"], work=ptr["ws"], work_bytes=308, status=ptr["status"], nseq=3, max_blocks=7, ntok=9,
                                        heads=6, mask_words=2, window=9, scale=0.25)
        assert got.stream == Stream.cuda_stream
        assert B.paged_tree_attention(w["caches"][0], w["tables"], w["lens"], w["offsets"], w["q"], 1, w["out"], w["ws"]) == 17
        assert (got.args.mask, got.args.mask_words, got.args.lse, got.args.positions, got.args.window, got.args.status, got.stream) == (None, 0, None, None, 0, None, None)
        assert B.paged_keep_rows(w["layers"], w["tables"], w["lens"], w["keep"], w["counts"], w["status"], 5) == 17
        assert fields(got.args) == dict(layers=w["layers"]._addr, nlayers=3, tables=ptr["tables"], table_stride=11, max_blocks=7, lens=ptr["lens"],
                                        keep=ptr["keep"], keep_stride=8, max_keep=6, counts=ptr["counts"], status=ptr["status"], nseq=3)
        assert got.stream == 5
        assert B.paged_copy_blocks(w["layers"], w["copies"], w["status"], 6) == 17
        assert fields(got.args) == dict(layers=w["layers"]._addr, nlayers=3, copies=ptr["copies"], ncopies=5, status=ptr["status"])
        assert B.paged_fork(w["pool"], w["shares"], w["lens"], w["new"], w["src"], w["dst"], 32, w["tables"], w["copies"], w["status"], 7) == 17
        assert fields(got.args) == dict(common, new_lens=ptr["new"], src=ptr["src"], dst=ptr["dst"], copies=ptr["copies"], nfork=5)
        assert B.paged_free(w["pool"], w["shares"], w["lens"], w["new"], 32, w["tables"], w["status"], 8) == 17
        assert fields(got.args) == dict(common, new_lens=ptr["new"])
        assert B.paged_compact(w["pool"], w["shares"], w["limits"], w["lens"], 32, w["tables"], w["copies"], w["status"], 9) == 17
        assert fields(got.args) == dict(common, limits=ptr["limits"], copies=ptr["copies"], max_copies=5)
        assert got.stream == 9
    d = w["layers"].descs
    assert [x.base[0] for x in d] == [w["arena"][i].data_ptr() for i in range(3)]


def test_tensors_that_do_not_fit():
    w = world()
    tree_args = ["tables", "lens", "offsets", "q", "out", "ws", "mask", "lse", "positions", "status"]

    def tree_call(**kw):
        a = {k: kw.get(k, w[k]) for k in tree_args}
        return B.paged_tree_attention(w["caches"][0], a["tables"], a["lens"], a["offsets"], a["q"], 1.0, a["out"], a["ws"], mask=a["mask"], lse=a["lse"],
                                      window=kw.get("window", 0), positions=a["positions"], status=a["status"])

    with Caught():
        assert tree_call() == 17
        for kw in (dict(offsets=w["offsets"][:3]), dict(lens=w["lens"].long()), dict(q=w["q"].float()), dict(q=w["q"][:8]), dict(out=w["out"][..., :32]),
                   dict(out=w["out"].transpose(0, 1)), dict(mask=w["mask"].int()), dict(mask=w["mask"][:8]), dict(mask=w["mask"][:, 0]),
                   dict(mask=w["mask"][:, :0]), dict(mask=torch.zeros((2, 9), dtype=torch.int64).t()), dict(lse=w["lse"][:, :5]), dict(positions=w["positions"][:8]),
                   dict(status=w["status"].long()), dict(window=-1), dict(tables=w["tables"][:2]), dict(tables=None), dict(ws=torch.zeros((4, 4)).t()[1:])):
            with pytest.raises(ValueError):
                tree_call(**kw)
        for args in ((w["keep"].long(), w["counts"]), (w["keep"][:2], w["counts"]), (w["keep"], w["counts"][:2]), (w["keep"][0], w["counts"])):
            with pytest.raises(ValueError):
                B.paged_keep_rows(w["layers"], w["tables"], w["lens"], *args)
        for bad in (w["copies"][:, :2], w["copies"].long(), w["copies"][0], w["copies"].t()):
            with pytest.raises(ValueError):
                B.paged_copy_blocks(w["layers"], bad)
        for src, dst, copies in ((w["src"][:4], w["dst"], w["copies"]), (w["src"], w["dst"].long(), w["copies"]), (w["src"], w["dst"], w["copies"][:4])):
            with pytest.raises(ValueError):
                B.paged_fork(w["pool"], w["shares"], w["lens"], w["new"], src, dst, 32, w["tables"], copies)
        with pytest.raises(ValueError):
            B.paged_free(w["pool"], w["shares"], w["lens"], w["new"][:2], 32, w["tables"])
        with pytest.raises(ValueError):
            B.paged_compact(w["pool"], w["shares"], w["counts"], w["lens"], 32, w["tables"], w["copies"])
        with pytest.raises(ValueError):
            B.paged_free(w["pool"], w["shares"], w["lens"], w["new"], -1, w["tables"])
    with pytest.raises(ValueError):
        B.PagedShares(w["refs"].long(), None, w["share_work"])
    with pytest.raises(ValueError):
        B.PagedLayers([])
    with pytest.raises(ValueError):
        B.PagedLayers([w["caches"][0]] * 129)
    with pytest.raises(ValueError):
        B.PagedLayers([w["caches"][0], B.PagedCache(w["arena"][0][:3])])


def test_kernels_that_start_ahead_read_through_coherent_loads():
    """A kernel launched with programmatic serialisation is there while its inputs are still being written."""
    seen = 0
    for name in os.listdir(build_mod.CSRC):
        with open(os.path.join(build_mod.CSRC, name)) as f:
            text = f.read()
        if "launch_ahead(" in text and name.endswith(".cu"):
            seen += 1
            assert not re.search(r"ld\.global\.nc|__ldg\(|\bld_stream_v4\(", text), name
    assert seen == 2


def test_the_matrix_kernels_fit_their_cta():
    """One CTA of 512 threads to an SM, launched with 128 registers each, which its warps then divide among themselves; nothing spills
    (300 bytes of spills in the softmax loops cost a third of the speed)."""
    res = build_mod.kernel_resources()
    main = {k: v for k, v in res.items() if "paged_tree_kernel" in k}
    assert len(main) == 6
    for name, r in main.items():
        assert r["registers"] == 128 and r["stack"] == r["spill_stores"] == r["spill_loads"] == 0, (name, r)
    for part in ("tree_join_kernel", "fork_kernel", "free_kernel", "compact_plan_kernel", "compact_cells_kernel", "copy_rows_kernel", "keep_rows_kernel"):
        found = [r for k, r in res.items() if part in k]
        assert found and all(r["spill_stores"] == r["spill_loads"] == 0 for r in found), part
