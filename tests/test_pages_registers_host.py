"""The kernels of trees, of rows and pages that move and of lists keep their values in registers."""
from test_kernel_registers_host import _kernels


def test_no_arrays_in_scratch_memory():
    names = ("tree_tile_kernel", "tree_rows_kernel", "tree_sees_kernel", "compact_rows_kernel", "copy_pages_kernel", "fork_kernel", "reserve_kernel", "free_kernel")
    scratch = {n: k[".private_segment_fixed_size"] for n, k in _kernels().items() if any(f in n for f in names)}
    for f in names:
        assert any(f in n for n in scratch), f
    # eight waves of f32 rows of 512 bytes: a few spilled words, outside the sweep
    spilled = {n: x for n, x in scratch.items() if x > (16 if "tree_tile_kernelILi0ELi128ELi8E" in n else 0)}
    assert not spilled, spilled
