"""Refusals of the device-driven path that need no GPU: what the C entry points and the binding check
before anything is enqueued."""
import ctypes as C

import pytest
import torch

from paper_2609_27040_b200 import binding as B
from paper_2609_27040_b200 import build as build_mod


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_mod.build()


def desc(**kw):
    d = B.PagedCacheDesc()
    d.dtype, d.num_kv_heads, d.head_dim, d.block_tokens = 0, 8, 128, 16
    d.blocks[0], d.base[0] = 4, 1 << 20
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(d, k)[v[0]] = v[1]
        else:
            setattr(d, k, v)
    return d


BAD_CACHES = [dict(dtype=2), dict(num_kv_heads=0), dict(num_kv_heads=65), dict(head_dim=96), dict(head_dim=512), dict(block_tokens=8),
              dict(block_tokens=48), dict(blocks=(0, 0)), dict(base=(0, 0)), dict(base=(0, (1 << 20) + 8)), dict(blocks=(1, 3)),
              dict(block_stride=(0, 65536 - 16)), dict(block_stride=(0, 65536 + 8)), dict(blocks=(0, 0x80000000))]
P = 1 << 20                                                        # an aligned address that is never touched: these calls are refused first


VP, U64, U32, F32 = C.c_void_p, C.c_uint64, C.c_uint32, C.c_float


class Build(C.Structure):                                          # the header's argument structs, field by field
    _fields_ = [("pool", VP), ("lens", VP), ("new", VP), ("tables", VP), ("stride", U64), ("offsets", VP), ("slots", VP), ("positions", VP),
                ("status", VP), ("n", U32), ("T", U32), ("width", U32), ("tokens", U32)]


class Write(C.Structure):
    _fields_ = [("cache", VP), ("k", VP), ("v", VP), ("ks", U64), ("vs", U64), ("slots", VP), ("status", VP), ("ntok", U32)]


class Decode(C.Structure):
    _fields_ = [("cache", VP), ("tables", VP), ("table_stride", U64), ("lens", VP), ("q", VP), ("q_stride", U64), ("out", VP),
                ("out_stride", U64), ("lse", VP), ("lam", VP), ("norm", VP), ("work", VP), ("work_bytes", U64), ("status", VP),
                ("nseq", U32), ("max_blocks", U32), ("heads", U32), ("window", U32), ("scale", F32), ("eps", F32), ("out_scale", F32)]


def call(name, args):
    return getattr(B.lib(), name)(C.cast(C.byref(args), C.c_char_p), None)


def decode(cache, name="paged_decode_tables", **kw):
    a = dict(cache=C.addressof(cache), tables=P, table_stride=10, max_blocks=10, lens=P, nseq=2, q=P, q_stride=32 * 256, heads=32, scale=1.0,
             out=P, out_stride=32 * 256, work=P, work_bytes=1 << 30)
    a.update(kw)
    return call(name, Decode(**a))


def diff(cache, **kw):
    return decode(cache, "paged_decode_diff", **{**dict(lam=P, eps=1e-5, out_scale=1.0), **kw})


def write(cache, **kw):
    a = dict(cache=C.addressof(cache), k=P, ks=2048, v=P, vs=2048, slots=P, ntok=3)
    a.update(kw)
    return call("paged_write_kv", Write(**a))


class Caught:
    """Stands in for the library's entry points: keeps the structs that the binding hands over."""

    def __enter__(self):
        self.calls, self.refs = B._torch_calls(), []
        for cls in (Build, Write, Decode, Decode):
            def entry(args, stream, cls=cls):
                self.args, self.stream = cls.from_buffer_copy(C.string_at(args, C.sizeof(cls))), stream
                return 17
            self.refs.append(C.CFUNCTYPE(C.c_int, VP, VP)(entry))
        self.calls.bind(*(C.cast(f, VP).value for f in self.refs))
        return self

    def __exit__(self, *_):
        B._calls = None                                            # bound to the library again by the next call


def test_every_argument_reaches_its_field():
    bf, i32, i64 = torch.bfloat16, torch.int32, torch.int64
    arena = torch.zeros((4, 2, 32, 2, 64), dtype=bf)
    c = B.PagedCache(arena)
    ids, free, free_out, work = torch.zeros(9, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32)
    pool = B.PagedPool(ids, None, free, free_out, work)
    lens, new, offsets = (torch.zeros(x, dtype=i32) for x in (3, 3, 4))
    tables = torch.zeros((3, 11), dtype=i32)[:, :7]
    slots, positions, status = torch.zeros(5, dtype=i64), torch.zeros(5, dtype=i32), torch.zeros(1, dtype=i32)

    class Stream:
        cuda_stream = 0x7f0012345678

    def fields(a):
        return {name: getattr(a, name) for name, _ in a._fields_}

    with Caught() as got:
        assert B.paged_build_tables(pool, lens, new, 32, tables, offsets, slots, positions, status, stream=Stream()) == 17
        assert fields(got.args) == dict(pool=C.addressof(pool.desc), lens=lens.data_ptr(), new=new.data_ptr(), tables=tables.data_ptr(), stride=11,
                                        offsets=offsets.data_ptr(), slots=slots.data_ptr(), positions=positions.data_ptr(),
                                        status=status.data_ptr(), n=3, T=32, width=7, tokens=5)
        assert got.stream == Stream.cuda_stream
        k, v = torch.zeros((5, 4, 64), dtype=bf)[:, :2], torch.zeros((5, 2, 64), dtype=bf)
        assert B.paged_write_kv(c, k, v, slots) == 17
        assert fields(got.args) == dict(cache=C.addressof(c.desc), k=k.data_ptr(), v=v.data_ptr(), ks=512, vs=256, slots=slots.data_ptr(), status=None,
                                        ntok=5)
        assert got.stream is None
        q, out = torch.zeros((3, 9, 64), dtype=bf)[:, 1:7], torch.zeros((3, 6, 64), dtype=bf)
        lse, ws, lam, weight = torch.zeros((3, 6)), torch.zeros(77), torch.zeros(6), torch.zeros(64)
        assert B.paged_decode_tables(c, tables, lens, q, 0.25, out, ws, lse=lse, window=9, status=status, stream=5) == 17
        common = dict(cache=C.addressof(c.desc), tables=tables.data_ptr(), table_stride=11, lens=lens.data_ptr(), out=out.data_ptr(), out_stride=768,
                      work=ws.data_ptr(), work_bytes=308, nseq=3, max_blocks=7, heads=6)
        assert fields(got.args) == dict(common, q=q.data_ptr(), q_stride=1152, lse=lse.data_ptr(), lam=None, norm=None, status=status.data_ptr(),
                                        window=9, scale=0.25, eps=0.0, out_scale=1.0)
        assert got.stream == 5
        qd = torch.zeros((3, 12, 32), dtype=bf)
        assert B.paged_decode_diff(c, tables, lens, qd, lam, -2, out, ws, norm_weight=weight, eps=0.5, out_scale=3, window=1) == 17
        assert fields(got.args) == dict(common, q=qd.data_ptr(), q_stride=768, lse=None, lam=lam.data_ptr(), norm=weight.data_ptr(), status=None, window=1,
                                        scale=-2.0, eps=0.5, out_scale=3.0)
        # one sequence, none: strides of such dimensions mean nothing
        one = torch.zeros((1, 6, 64), dtype=bf).as_strided((1, 6, 64), (8, 64, 1))
        assert B.paged_decode_tables(c, tables[:1], lens[:1], one, 1.0, out[:1], ws) == 17
        assert (got.args.q_stride, got.args.out_stride, got.args.table_stride, got.args.window, got.args.lse) == (768, 768, 7, 0, None)
        assert B.paged_decode_tables(c, tables[:0], lens[:0], out[:0], 1.0, out[:0], ws) == 17 and got.args.nseq == 0


def test_arguments_that_are_no_tensors_or_numbers():
    bf, i64 = torch.bfloat16, torch.int64
    c = B.PagedCache(torch.zeros((4, 2, 16, 2, 64), dtype=bf))
    k, slots = torch.zeros((5, 2, 64), dtype=bf), torch.zeros(5, dtype=i64)
    for a in ((None, k, slots), (k, 3, slots), (k, k, [1, 2]), (k, k, slots, 0), (k.to_sparse(), k, slots), (k.to("meta"), k, slots),
              (k[0], k, slots)):
        with pytest.raises(ValueError):
            B.paged_write_kv(c, *a)
    with pytest.raises((TypeError, AttributeError)):
        B.paged_write_kv(c, k, k, slots, stream="main")
    q, ws = torch.zeros((3, 4, 64), dtype=bf), torch.zeros(9)
    tables, lens = torch.zeros((3, 5), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError):
        B.paged_decode_tables(c, tables, lens, q, "1", q, ws)
    for kw in (dict(window=-1), dict(window=1 << 40)):
        with pytest.raises(ValueError):
            B.paged_decode_tables(c, tables, lens, q, 1.0, q, ws, **kw)
    with pytest.raises(TypeError):
        B.paged_decode_tables(c, tables, lens, q, 1.0, q, ws, window=1.5)
    with pytest.raises((ValueError, OverflowError)):
        B.paged_decode_tables(c, tables, lens, q, 1.0, q, ws, window=1 << 70)


def test_no_arguments_at_all():
    for name in ("paged_build_tables", "paged_write_kv", "paged_decode_tables", "paged_decode_diff"):
        assert getattr(B.lib(), name)(None, None) == B.EINVAL
        assert getattr(B.lib(), name)(bytes(200), None) == B.EINVAL


@pytest.mark.parametrize("kw", BAD_CACHES, ids=str)
def test_bad_caches_are_refused_everywhere(kw):
    d = desc(**kw)
    n = C.c_uint64(7)
    assert decode(d) == diff(d) == write(d) == B.EINVAL
    assert B.lib().paged_decode_workspace(C.byref(d), 32, C.byref(n)) == B.EINVAL and n.value == 7


@pytest.mark.parametrize("kw", [dict(tables=None), dict(lens=None), dict(q=None), dict(out=None), dict(work=None), dict(max_blocks=0),
                                dict(table_stride=9), dict(max_blocks=1 << 28, table_stride=1 << 28), dict(q_stride=32 * 256 - 16),
                                dict(out_stride=8), dict(q_stride=32 * 256 + 8), dict(q=P + 8), dict(out=P + 2), dict(work=P + 4),
                                dict(tables=P + 2), dict(lens=P + 1), dict(status=P + 1), dict(heads=0), dict(heads=12), dict(heads=136),
                                dict(nseq=0x80000000)], ids=str)
def test_bad_decode_arguments_are_refused(kw):
    assert decode(desc(), **kw) == B.EINVAL
    if kw.get("heads") != 136:
        assert diff(desc(), **kw) == B.EINVAL


def test_bad_differential_arguments_are_refused():
    assert diff(desc(), lam=None) == B.EINVAL
    assert diff(desc(), heads=72) == B.EINVAL                      # nine heads to a KV head
    assert diff(desc(), norm=P, eps=-1.0) == B.EINVAL
    assert diff(desc(), norm=P, eps=float("nan")) == B.EINVAL
    assert diff(desc(), norm=P + 2) == B.EINVAL and diff(desc(), lam=P + 1) == B.EINVAL
    assert diff(desc(), lse=P) == B.EINVAL                         # one call's outputs and weights given to the other
    assert decode(desc(), lam=P) == B.EINVAL and decode(desc(), norm=P) == B.EINVAL and decode(desc(), lse=P + 2) == B.EINVAL


def test_workspace_too_small():
    need = C.c_uint64(0)
    assert B.lib().paged_decode_workspace(C.byref(desc()), 32, C.byref(need)) == B.OK and need.value > 32768
    assert decode(desc(), work_bytes=need.value - 1) == B.ESCRATCH
    more = C.c_uint64(0)
    assert B.lib().paged_decode_workspace(C.byref(desc()), 128, C.byref(more)) == B.OK and more.value > need.value
    assert diff(desc(), heads=64, q_stride=64 * 256, out_stride=64 * 256, work_bytes=need.value) == B.ESCRATCH   # two rows to a head
    for rows in (0, 12, 136):
        assert B.lib().paged_decode_workspace(C.byref(desc()), rows, C.byref(need)) == B.EINVAL
    assert B.lib().paged_decode_workspace(C.byref(desc()), 32, None) == B.EINVAL


def test_nothing_to_do_is_ok():
    assert decode(desc(), nseq=0) == diff(desc(), nseq=0) == write(desc(), ntok=0) == B.OK


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(slots=None), dict(ks=2040), dict(vs=1024), dict(k=P + 8), dict(v=P + 2),
                                dict(slots=P + 4), dict(status=P + 2), dict(ntok=0x80000000)], ids=str)
def test_bad_write_arguments_are_refused(kw):
    assert write(desc(), **kw) == B.EINVAL


def build(pool_kw=None, **kw):
    p = B.PagedPoolDesc()
    p.ids[0], p.capacity[0], p.free_in, p.free_out, p.work = P, 10, P, P, P
    for k, v in (pool_kw or {}).items():
        if isinstance(v, tuple):
            getattr(p, k)[v[0]] = v[1]
        else:
            setattr(p, k, v)
    a = dict(pool=C.addressof(p), lens=P, new=P, n=3, T=16, tables=P, stride=8, width=8, offsets=P, slots=P, positions=P, tokens=100)
    a.update(kw)
    return call("paged_build_tables", Build(**a))


def test_bad_build_arguments_are_refused():
    for kw in (dict(lens=None), dict(new=None), dict(T=0), dict(T=24), dict(T=128), dict(tables=None), dict(stride=7), dict(width=0),
               dict(width=1 << 28, stride=1 << 28), dict(offsets=None), dict(slots=None), dict(positions=None), dict(tokens=0x80000000),
               dict(n=0x7fffffff), dict(slots=P + 4), dict(tables=P + 2), dict(offsets=P + 2), dict(status=P + 3), dict(lens=P + 2)):
        assert build(**kw) == B.EINVAL, kw
    for kw in (dict(ids=(0, None)), dict(capacity=(1, 5)), dict(capacity=(0, 0x80000000)), dict(free_in=None), dict(free_out=None),
               dict(work=None), dict(free_out=P + 4), dict(free_in=P + 4), dict(work=P + 2), dict(ids=(0, P + 2))):
        assert build(kw) == B.EINVAL, kw


def test_binding_refuses_tensors_that_do_not_fit():
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    arena = torch.zeros((4, 2, 16, 2, 64), dtype=bf)
    for bad in (torch.zeros((4, 2, 16, 2, 64)), arena[:, :1], arena.transpose(2, 3), torch.zeros((4, 3, 16, 2, 64), dtype=bf), arena[0],
                arena[:0]):
        with pytest.raises(ValueError):
            B.PagedCache(bad)
    with pytest.raises(ValueError):
        B.PagedCache(arena, torch.zeros((4, 2, 16, 2, 64), dtype=torch.float16))
    with pytest.raises(ValueError):
        B.PagedCache(arena, torch.zeros((4, 2, 32, 2, 64), dtype=bf))
    c = B.PagedCache(arena[::2], arena[1:])
    assert c.desc.block_stride[0] == 2 * 2 * 16 * 2 * 64 * 2 and list(c.desc.blocks) == [2, 3]
    good = dict(tables=torch.zeros((3, 5), dtype=i32), lens=torch.zeros(3, dtype=i32), q=torch.zeros((3, 4, 64), dtype=bf), sm_scale=1.0,
                out=torch.zeros((3, 4, 64), dtype=bf), workspace=torch.zeros(B.paged_decode_workspace(c, 4), dtype=torch.uint8))
    for kw in (dict(tables=good["tables"].long()), dict(tables=good["tables"][:2]), dict(tables=torch.zeros((5, 3), dtype=i32).T),
               dict(lens=torch.zeros(3, dtype=torch.int64)), dict(lens=torch.zeros(6, dtype=i32)[::2]), dict(q=good["q"].half()),
               dict(q=good["q"][:2]), dict(q=torch.zeros((3, 64, 4), dtype=bf).transpose(1, 2)), dict(out=good["out"].float()),
               dict(out=torch.zeros((3, 4, 32), dtype=bf)), dict(lse=torch.zeros((3, 5), dtype=f32)), dict(window=-1),
               dict(status=torch.zeros(2, dtype=i32)), dict(workspace=torch.zeros(64)[::2])):
        with pytest.raises(ValueError):
            B.paged_decode_tables(c, **{**good, **kw})
    d = dict(good, q=torch.zeros((3, 8, 32), dtype=bf), lam=torch.zeros(4))
    for kw in (dict(q=good["q"]), dict(lam=torch.zeros(3)), dict(lam=torch.zeros(4).half()), dict(norm_weight=torch.zeros(32)), dict(window=-3)):
        with pytest.raises(ValueError):
            B.paged_decode_diff(c, **{**d, **kw})
    k = torch.zeros((5, 2, 64), dtype=bf)
    for a in ((k, k[:4], torch.zeros(5, dtype=torch.int64)), (k, k, torch.zeros(5, dtype=i32)), (k.half(), k, torch.zeros(5, dtype=torch.int64)),
              (k, torch.zeros((5, 64, 2), dtype=bf).transpose(1, 2), torch.zeros(5, dtype=torch.int64))):
        with pytest.raises(ValueError):
            B.paged_write_kv(c, *a)
    w = torch.zeros(1, dtype=i32)
    for a in ((torch.zeros(4), None, torch.zeros(2, dtype=i32), torch.zeros(2, dtype=i32), w),
              (torch.zeros(4, dtype=i32), None, torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), w),
              (torch.zeros(4, dtype=i32), None, torch.zeros(2, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(0, dtype=i32))):
        with pytest.raises(ValueError):
            B.PagedPool(*a)


def test_descriptor_sizes_match_the_header():
    assert C.sizeof(B.PagedCacheDesc) == 4 * 4 + 2 * 4 + 2 * 8 + 2 * 8
    assert C.sizeof(B.PagedPoolDesc) == 2 * 8 + 2 * 4 + 3 * 8


def test_memory_that_no_gpu_can_reach_is_refused():
    """Host tensors through the whole binding: every call answers with a code, none launches."""
    arena = torch.zeros((4, 2, 16, 2, 64), dtype=torch.bfloat16)
    c = B.PagedCache(arena)
    k = torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    assert B.paged_write_kv(c, k, k, torch.zeros(5, dtype=torch.int64)) in (B.EINVAL, B.ECUDA)
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    i32 = torch.int32
    assert B.paged_decode_tables(c, torch.zeros((3, 5), dtype=i32), torch.zeros(3, dtype=i32), q, 1.0, q.clone(),
                                 torch.zeros(B.paged_decode_workspace(c, 4), dtype=torch.uint8)) in (B.EINVAL, B.ECUDA)


def test_arenas_whose_blocks_share_memory_are_refused():
    """A first stride of 0 would be the descriptor's "dense": blocks far behind the tensor. Smaller than a block: blocks over one another."""
    one = torch.zeros((1, 2, 16, 2, 64), dtype=torch.bfloat16)
    size = one.numel()
    flat = torch.zeros(4 * size, dtype=torch.bfloat16)
    for bad in (one.expand(64, -1, -1, -1, -1), flat.as_strided((3, 2, 16, 2, 64), (size - 8,) + one.stride()[1:]),
                flat.as_strided((3, 2, 16, 2, 64), (8,) + one.stride()[1:])):
        assert bad[0].is_contiguous()
        with pytest.raises(ValueError):
            B.PagedCache(bad)
        with pytest.raises(ValueError):
            B.PagedCache(one, bad)
    c = B.PagedCache(one.expand(1, -1, -1, -1, -1), flat.as_strided((3, 2, 16, 2, 64), (size + 8,) + one.stride()[1:]))
    assert list(c.desc.blocks) == [1, 3] and list(c.desc.block_stride) == [0, 2 * (size + 8)]


def test_kernels_that_start_early_read_through_coherent_loads():
    """A kernel launched with programmatic serialisation is there while its inputs are still being written: loads of the read-only path
    (ld.global.nc, __ldg) are for data that does not change as long as the kernel lives."""
    import os
    import re
    with open(os.path.join(build_mod.CSRC, "ptx.cuh")) as f:
        wrappers = set(re.findall(r"__forceinline__ \w+ (\w+)\([^{]*\{[^}]*ld\.global\.nc", f.read()))
    assert "ld_stream_v4" in wrappers
    seen = 0
    for name in os.listdir(build_mod.CSRC):
        with open(os.path.join(build_mod.CSRC, name)) as f:
            text = f.read()
        if "launch_early(" in text and name.endswith(".cu"):
            seen += 1
            assert not re.search(r"ld\.global\.nc|__ldg\(|\b(%s)\(" % "|".join(wrappers), text), name
    assert seen == 2


@pytest.mark.parametrize("T,Hkv,D", [(16, 3, 64), (32, 1, 64), (64, 5, 128), (16, 2, 256), (32, 4, 256), (16, 8, 128)])
def test_the_block_formats_converter_takes_every_cache(T, Hkv, D):
    """Unit u of 8 elements of token row r lies at unit u ^ (r & 7) of its 64 elements; its own inverse, for arrays and tensors."""
    from tests.paged_helpers import stored_place
    x = torch.arange(3 * 2 * T * Hkv * D).to(torch.int16).view(3, 2, T, Hkv, D)
    y = B.kv_block_swizzle(x)
    for r in range(T):
        assert torch.equal(y[:, :, r].reshape(3, 2, -1)[..., torch.from_numpy(stored_place(r, Hkv * D))], x[:, :, r].reshape(3, 2, -1))
    assert torch.equal(B.kv_block_swizzle(y), x) and (B.kv_block_swizzle(x.numpy()) == y.numpy()).all()
    for bad in (x[:, :, :8], x[..., :32], x[0, 0, 0]):
        with pytest.raises(ValueError):
            B.kv_block_swizzle(bad)
