"""Sizes at the end of what the losses' C entries accept (CPU only: refusals and workspace sizes, nothing is launched).
The kernels walk rows and columns in 32-bit steps of up to 18944 (the pass over a few tokens) and 8192 (the factors), so a
size has to leave that much room below 2^31."""
import ctypes as C

import pytest

from paper_1901_01544_b200 import binding, build, losses

LARGEST = (1 << 31) - (1 << 16)


@pytest.fixture(scope="module")
def L():
    build.build()
    return losses.lib()


def head(**kw):
    a = losses.HeadArgs(tokens=1, vocab=100, dim=8, dtype=1, hidden=256, hidden_ld=8, weight=256, weight_ld=8, targets=256, top_k=1, lse=256,
                        temperature=1.0, scale=1.0, workspace=256, workspace_bytes=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("which", ["tokens", "vocab", "dim"])
def test_largest_sizes(L, which):
    ld = dict(hidden_ld=LARGEST, weight_ld=LARGEST) if which == "dim" else {}
    assert L.iwp_head_workspace(C.byref(head(**{which: LARGEST}, **ld))) > 0
    assert L.iwp_head_loss(C.byref(head(**{which: LARGEST}, **ld)), None) == binding.IWP_ERR_CAPACITY
    for n in (LARGEST + 1, (1 << 31) - 18944, (1 << 31) - 8192, (1 << 31) - 1024, (1 << 31) - 1):
        a = head(**{which: n}, **({k: n for k in ld}))
        assert L.iwp_head_workspace(C.byref(a)) == -1
        assert L.iwp_head_loss(C.byref(a), None) == binding.IWP_ERR_INVALID
