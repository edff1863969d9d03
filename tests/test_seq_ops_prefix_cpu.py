"""Who takes a shared prefix, seen from the workspace: prompts that take it in front of their own tokens need none, parts of it do.  On the host, no GPU is needed."""
import pytest

from test_seq_ops_boundary_cpu import lib  # noqa: F401  (the fixture)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_few_prompts_share_out_a_long_prefix(lib, D):  # noqa: F811
    """Tables of 128, 256 and 320 tokens, the last of which is cut in any case: 200 tokens of one sequence after a long text leave most of the GPU idle where each tile walks the whole text alone."""
    need = lambda Bn, new, width, prefix: lib.nvfp4_attn_workspace_bytes(Bn * new, 32, 8, D, 64, Bn, width, prefix)
    for prefix in (4096, 16384, 65536, 1 << 20):
        for Bn, new, width in ((1, 64, 2), (1, 200, 4), (2, 200, 4), (1, 200, 5)):
            assert need(Bn, new, width, prefix) > 0, (Bn, new, width, prefix)
        # as many tiles as the GPU takes at once, or more
        assert need(32, 256, 4, prefix) == 0, prefix
    # a prefix that is short against the partial results, and none
    for prefix in (0, 1, 100):
        assert need(1, 200, 4, prefix) == need(4, 200, 4, prefix) == 0, prefix
