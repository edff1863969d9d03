"""A cache of no pages, whatever tables and lengths hold: the host decides that there are no tokens, before a kernel could look for them."""
import os
import subprocess
import sys

import pytest

from test_seq_ops_boundary_cpu import lib  # noqa: F401  (the fixture builds the library where it is not built)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIP, WORKSPACE = -7, -4

# In a process that no device is visible to: a call that is not refused ends at its launch, and the addresses are never looked at.
CALL = """
import sys
sys.path[:0] = [%r, %r]
import torch
import test_seq_ops_boundary_cpu as t
import paper_2510_27527_amd.binding as B
pages, N, width, prefix, kind = map(int, sys.argv[1:])
c = t.cache(pages=pages, kind=kind, ke=t.FAKE, ve=t.FAKE)
b = t.batch(Bn=N, width=width, prefix=prefix, prefix_table=t.FAKE)
assert not torch.cuda.is_available()
print(B.lib().nvfp4_attn(t.FAKE, 256, N, 4, c, b, 0.125, t.FAKE, 256, None, 0, None))
""" % (ROOT, os.path.join(ROOT, "tests"))


def attn(*args):
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1", CUDA_VISIBLE_DEVICES="-1")
    r = subprocess.run([sys.executable, "-c", CALL, *map(str, args)], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stderr
    return int(r.stdout)


@pytest.mark.parametrize("N,width,prefix", [(2, 500, 0), (2, 1, 4000), (2, 500, 4000)])
@pytest.mark.parametrize("kind", [0, 1])
def test_a_cache_of_no_pages_has_no_tokens(lib, N, width, prefix, kind):  # noqa: F811
    """Sizes whose tokens would be cut into parts, for which a workspace is asked for: with no page there is nothing to cut, and none is."""
    assert attn(1, N, width, prefix, kind) == WORKSPACE
    assert attn(0, N, width, prefix, kind) == HIP
