"""What the compiler says of the kernels of the caches in pages: none spills vector registers (a spilled register's reload waits for all loads that
are under way: chunks of 8192 rows took 3.7 ms in the place of 1.4 with 62 of them)."""
from test_no_spills import needs_tools, spills


@needs_tools
def test_paged_kernels_do_not_spill(tmp_path):
    kernels = {n: s for n, s in spills(tmp_path).items() if "k_paged_" in n or "k_rope_rows" in n}
    # attention: three head sizes and two types of two narrow kernels, a wide one and three joins; append and rope: three types and widths each
    assert len(kernels) == 3 * 2 * 6 + 6 and not any(kernels.values()), kernels
