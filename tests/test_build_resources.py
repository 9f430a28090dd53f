"""The layer kernel's register budget, checked where it is decided: at build time (no GPU needed).

The kernel runs 352 threads per CTA with 227 KB of shared memory, one CTA per SM, and the compiler
is at the register limit that leaves (168 per thread). Two things have each cost it 4 to 15 % of its
bandwidth without failing any parity test: spills in the streaming loops, and a device function that
takes the ~1 KB parameter block by reference falling out of line, after which every thread keeps a
copy of the block on its stack and reads it from local memory. Both show in what ptxas reports."""
from paper_2609_27040_b200 import build as build_mod


def _layer_kernels():
    res = build_mod.kernel_resources()
    ks = {k: v for k, v in res.items() if "slice_layer_kernel" in k}
    assert len(ks) == 4, sorted(res)                      # tensor-core / f32 tiles x one block or several per stage
    return ks


def test_every_kernel_of_the_library_is_reported():
    res = build_mod.kernel_resources()
    for name in ("slice_layer_kernel", "copy_blocks_bulk", "copy_blocks_vector", "append_kv_kernel", "step_relay_kernel"):
        assert any(name in k for k in res), name
    for k, v in res.items():
        assert {"registers", "stack", "spill_stores", "spill_loads"} <= set(v), k


def test_layer_kernel_fits_one_cta_per_sm_without_a_stack_copy_of_its_parameters():
    for name, r in _layer_kernels().items():
        assert r["registers"] * 352 <= 65536, (name, r)  # one CTA of 352 threads per SM
        # the copy thread's bookkeeping arrays (about 200 bytes) are all the stack there is; a copy of
        # the parameter block would add about 1 KB
        assert r["stack"] <= 320, (name, r)
        assert r["spill_stores"] <= 64 and r["spill_loads"] <= 64, (name, r)


def test_the_benchmarks_variant_does_not_spill_at_all():
    # tensor-core tiles, one block per stage: 5 to 8 KV heads with grouped queries, what bench.py times
    main = [r for k, r in _layer_kernels().items() if "ILb1ELb0E" in k]
    assert len(main) == 1
    assert main[0]["spill_stores"] == 0 and main[0]["spill_loads"] == 0 and main[0]["stack"] <= 256, main[0]


def test_copy_kernels_leave_room_beside_the_layer_kernel():
    # a CTA of the 6-stage bulk gather (32 threads) shares an SM with a CTA of the layer kernel
    res = build_mod.kernel_resources()
    bulk = [r for k, r in res.items() if "copy_blocks_bulkILi6E" in k]
    layer = max(r["registers"] for r in _layer_kernels().values())
    assert len(bulk) == 1
    regs = lambda per_thread, threads: -(-per_thread * 32 // 256) * 256 * (threads // 32)   # allocated per warp, in units of 256
    assert regs(layer, 352) + regs(bulk[0]["registers"], 32) <= 65536


def test_device_driven_kernels_fit_their_cta_and_do_not_spill():
    """One CTA to an SM; no stack and no spills but in the variant of 9 to 16 columns with heads of 256, whose eight consumer warps
    leave 168 registers to a thread (about 20 of a lane's values are kept in local memory)."""
    res = build_mod.kernel_resources()
    decode = {k: v for k, v in res.items() if "paged_decode_kernel" in k}
    assert len(decode) == 12, sorted(res)                 # heads of 64 / 128 / 256 x one group of columns or two x bf16 / fp16
    for name, r in decode.items():
        two = "Lj2E" in name
        warps = (4 * 2 + 1 + 2) if two else (6 + 1 + 1)   # consumers, scheduler, mergers (one group, heads of 256: five consumers)
        if two:                                           # a scheduler's quarter of the registers holds three of the eleven warps
            assert r["registers"] * 32 * -(-warps // 4) <= 16384, (name, r)
        assert r["registers"] <= 255 and r["registers"] * 32 * warps <= 65536, (name, r)
        if two and "Lj256E" in name:
            assert r["stack"] <= 64 and r["spill_stores"] <= 128 and r["spill_loads"] <= 192, (name, r)
        else:
            assert r["stack"] == r["spill_stores"] == r["spill_loads"] == 0, (name, r)
    others = {k: v for k, v in res.items() if "write_kv_kernel" in k or "build_tables_kernel" in k}
    assert len(others) == 3
    for name, r in others.items():
        assert r["stack"] == r["spill_stores"] == r["spill_loads"] == 0, (name, r)
        assert r["registers"] <= (64 if "write_kv" in name else 128), (name, r)   # four CTAs of 256 threads; one of 512


def test_kernels_of_several_new_tokens_and_shared_blocks():
    """paged_tree_kernel moves registers between its warps by setmaxnreg: 168 for the eight softmax warps and 88 for the others are what 512
    threads of 128 have. Launched with fewer, the request for more would wait for good, so the number is exact."""
    res = build_mod.kernel_resources()
    tree = {k: v for k, v in res.items() if "paged_tree_kernel" in k}
    assert len(tree) == 6, sorted(res)                    # heads of 64 / 128 / 256 x bf16 / fp16
    for name, r in tree.items():
        assert r["registers"] == 128 and r["stack"] == r["spill_stores"] == r["spill_loads"] == 0, (name, r)
    join = {k: v for k, v in res.items() if "tree_join_kernel" in k}
    assert len(join) == 6, sorted(res)
    for name, r in join.items():                          # three CTAs of 256 threads to an SM
        assert r["registers"] * 256 * 3 <= 65536 and r["stack"] == r["spill_stores"] == r["spill_loads"] == 0, (name, r)
    # CTAs of 512 threads (two to an SM of the kernel that rewrites cells), of 256 (four) and of 128 (eight)
    for part, most in (("free_kernel", 128), ("fork_kernel", 128), ("compact_plan_kernel", 128), ("compact_cells_kernel", 64), ("copy_rows_kernel", 64),
                       ("keep_rows_kernel", 64)):
        found = [(k, v) for k, v in res.items() if part in k]
        assert len(found) == 1, (part, sorted(res))
        for name, r in found:                             # (8 bytes of stack: the two arenas' limits, indexed by an entry's arena)
            assert r["registers"] <= most and r["stack"] <= 8 and r["spill_stores"] == r["spill_loads"] == 0, (name, r)
