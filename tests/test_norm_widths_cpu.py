"""The widths that dora_residual_norm takes are those that its header states."""
import ctypes
import os
import re

import pytest

import paper_2609_34325_amd as dora
from paper_2609_34325_amd import build

A = 0x10000000          # never dereferenced: no rows, no launch


def call(C, dtype):
    r = [dora.Rows(A + i * (1 << 20), 0, 1, C, C, C, dtype, 0) for i in range(4)]
    v = A + (8 << 20)
    return dora.load_library().dora_residual_norm(*(ctypes.byref(t) for t in r[:2]), v, None, None, None, None, None, 0, 1e-6,
                                                  *(ctypes.byref(t) for t in r[2:]), None)


@pytest.mark.parametrize("dtype,size", [(dora.DORA_BF16, 2), (dora.DORA_F32, 4)])
def test_widths(dtype, size):
    text = open(os.path.join(build.INCLUDE, "dora.h")).read()
    most = int(re.search(r"C at most\s+\*\s+(\d+) and rows a multiple of 16 bytes", text).group(1))
    piece = 16 // size
    for C in (piece, 3 * piece, most - piece, most):
        assert call(C, dtype) == dora.DORA_OK, C
    for C in (1, piece - 1, piece + 1, most + piece, 2 * most):
        assert call(C, dtype) == dora.DORA_ERR_SHAPE, C
