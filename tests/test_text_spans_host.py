"""CPU-only: buffers of the language-model operators whose rows lie between one another's are refused, as ceca.h says."""
import ctypes
import os

import pytest

import paper_2306_00256_amd as P
from paper_2306_00256_amd import binding as B

A, Bp, Cp, W = (1 << 32) * 256, (1 << 33) * 256, (1 << 34) * 256, (1 << 36) * 256        # stand-ins for device addresses; nothing reads them


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(P.library_path()):
        from paper_2306_00256_amd import build
        build.build_library(verbose=False)
    return P.lib()


def test_interleaved_rows_are_refused(L):
    spec = B.Distill(n=2, T=3, V=100, K=4, type=1, temperature=1.0, hard=0.0, logits=A, ld=200, top=Bp, ids=Bp + 4096)
    assert L.ceca_distill(ctypes.byref(spec), Cp, A + 200, 200, W, 1 << 30, None) == B.CECA_EINVAL          # the gradient beside the logits
    assert L.ceca_embed(A, 60, 12, 1, 5, 6, Bp, 3, 1.0, A + 24, 0, 12, None) == B.CECA_EINVAL               # rows of `out` behind rows of the table
    assert L.ceca_embed_grad(A + 24, 0, 12, Bp, 3, 1.0, 0, A, 60, 12, 1, 5, 6, W, 1 << 30, None) == B.CECA_EINVAL
    assert L.ceca_top_logits(A, 0, 20, 3, 10, 4, A + 40, Cp, W, 1 << 30, None) == B.CECA_EINVAL
