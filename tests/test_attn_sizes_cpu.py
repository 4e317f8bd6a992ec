"""Workspaces of grouped attention on the host: every size that a call may have gets one."""
import ctypes
import random
import subprocess

import pytest

import paper_2609_34325_amd as dora
from paper_2609_34325_amd import build

PROBE = """
#include "grouped_attn_split.h"
// The most keys that one workgroup of a forward call goes over, one after another.
extern "C" long longest(int B, int H, int Hk, int D, int max_q, long total_q, long total_k, int max_k) {
  const dora::Sizes z{B, H, Hk, D, max_q, total_q, total_k};
  const dora::Split p = dora::forward_split(z, max_k);
  const long most = max_k > 0 ? max_k : total_k;
  return p.chunk ? (p.chunk < most ? p.chunk : most) : most / p.splits;
}
"""


@pytest.fixture(scope="module")
def longest(tmp_path_factory):
    d = tmp_path_factory.mktemp("split")
    (d / "probe.hip").write_text(PROBE)
    so = str(d / "probe.so")
    subprocess.run([build.hipcc(), "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", build.INCLUDE, "-I",
                    build.CSRC, str(d / "probe.hip"), "-o", so], check=True, capture_output=True, timeout=300)
    f = ctypes.CDLL(so).longest
    f.argtypes, f.restype = [ctypes.c_int] * 5 + [ctypes.c_long] * 2 + [ctypes.c_int], ctypes.c_long
    return f


def test_one_long_list_among_short_ones(longest):
    """New tokens whose longest list is not known to the call: no workgroup goes over a long one alone."""
    assert longest(501, 32, 8, 128, 1, 501, 60500, 0) <= 1024
    rng = random.Random(4)
    for _ in range(20000):
        Hk, G, B = rng.choice((1, 2, 8, 32)), rng.choice((1, 2, 4, 8)), rng.randint(1, 1000)
        total_k = int(10 ** rng.uniform(0, 6))
        # parts of a fair share of the GPU, 128 keys or more, or all of at most 1024
        fair = max(1024, total_k * Hk // 512 + 64, total_k // B // 32 + 64)
        assert longest(B, Hk * G, Hk, 64, 1, B, total_k, 0) <= min(4096, fair), (B, Hk, G, total_k)
    # known to be short: whole
    assert longest(501, 32, 8, 128, 1, 501, 60500, 256) == 256


@pytest.mark.parametrize("sizes", [(1, 4, 2, 64, 0, 0, 5), (2, 4, 2, 64, 1, 0, 9), (3, 4, 2, 64, 0, 6, 9), (1, 1, 1, 32, 0, 0, 0),
                                   (500, 8, 8, 128, 1, 0, 1 << 20)])
def test_no_queries(sizes):
    """An empty batch against a cache, and one whose sequences all have none."""
    assert dora.dora_grouped_attn_workspace_size(*sizes) >= 256
    assert dora.dora_grouped_attn_backward_workspace_size(*sizes) >= 256


def test_every_size_has_a_workspace():
    rng = random.Random(3)

    def log(lo, hi):
        return int(lo * (hi / lo) ** rng.random())
    for _ in range(20000):
        Hk, D, B = log(1, 32), rng.choice((32, 64, 128)), log(1, 2000)
        H = Hk * rng.choice((1, 2, 4, 5, 8))
        sizes = (B, H, Hk, D, rng.choice((0, 1, log(1, 300))), rng.choice((0, B, log(1, 100000))), rng.choice((0, log(1, 1 << 22))))
        for size in (dora.dora_grouped_attn_workspace_size, dora.dora_grouped_attn_backward_workspace_size):
            n = size(*sizes)
            assert n >= 256 and n % 256 == 0, sizes
