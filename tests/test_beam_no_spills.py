"""What the compiler says of the kernels of beam search and of pools of pages: none spills vector registers."""
from test_no_spills import needs_tools, spills


@needs_tools
def test_beam_and_pool_kernels_do_not_spill(tmp_path):
    kernels = {n: s for n, s in spills(tmp_path).items() if "k_beam_" in n or "k_pool_" in n}
    # the scan of two types and the join; release, reserve, copy, two forks, compact
    assert len(kernels) == 3 + 6 and not any(kernels.values()), kernels
