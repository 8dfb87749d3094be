"""The kernels of attention over pages keep their values in registers: a reload from scratch memory waits for every row in flight, and
arrays that the compiler leaves in memory cost several times as much (f32, rows of 512 bytes: 185 us that became 37)."""
from test_kernel_registers_host import _kernels


def test_attention_over_pages_has_no_arrays_in_scratch_memory():
    kernels = {n: k for n, k in _kernels().items() if any(f in n for f in ("paged_tile_kernel", "paged_rows_kernel", "paged_merge_kernel", "rows_kernel"))}
    scratch = {n: k[".private_segment_fixed_size"] for n, k in kernels.items()}
    assert sum("paged_tile_kernel" in n for n in scratch) == 8 and sum("paged_rows_kernel" in n for n in scratch) == 8, sorted(scratch)
    # eight waves of f32 rows of 512 bytes: a few spilled words, outside the sweep
    spilled = {n: x for n, x in scratch.items() if x > (16 if "paged_tile_kernelILi0ELi128ELi8E" in n else 0)}
    assert not spilled, spilled
