"""Sizes at the ends of their types, and workspaces, of the operators around the quantized linears: on the host, no GPU is needed."""
import ctypes as C

import pytest

from test_block_ops_boundary_cpu import FAKE, SHAPE, ckpt, lib  # noqa: F401  (the fixture)

# N = 0 launches nothing: what is not refused is only reported as good
NEGATIVE = [-1, -64, -(1 << 31), -(1 << 62), -(1 << 63) + 64, -(1 << 63) + 1, -(1 << 63)]


@pytest.mark.parametrize("F", NEGATIVE)
@pytest.mark.parametrize("act", [0, 1])
def test_nonlinearity_refuses_every_negative_width(lib, F, act):  # noqa: F811
    """Also those whose double is not negative in 64 bits."""
    assert lib.nvfp4_act_fwd(FAKE, 0, 1 << 20, 0, F, act, FAKE, 0, 1 << 20, None, None) == SHAPE
    assert lib.nvfp4_act_bwd(FAKE, 0, 1 << 20, FAKE, 0, 1 << 20, 0, F, act, FAKE, 0, 1 << 20, None) == SHAPE
    kept = ckpt(0, F)
    assert lib.nvfp4_act_bwd(FAKE, 0, 1 << 20, C.byref(kept), 3, 0, 0, F, act, FAKE, 0, 1 << 20, None) == SHAPE


def test_norm_workspace_does_not_shrink(lib):  # noqa: F811
    """A workspace for the largest batch and width serves all smaller ones."""
    f = lib.nvfp4_norm_workspace_bytes
    widths = (1, 7, 8, 64, 512, 513, 1000, 1024, 1025, 2048, 2049, 4096, 4100, 8192, 8200, 16384, 16390, 100000)
    batches = list(range(0, 5000)) + [1 << 14, (1 << 14) + 1, 1 << 15, 81000]
    sizes = {D: [f(N, D) for N in batches] for D in widths}
    for D in widths:
        assert sizes[D] == sorted(sizes[D]), D
    for a, b in zip(widths, widths[1:]):
        assert all(x <= y for x, y in zip(sizes[a], sizes[b])), (a, b)
