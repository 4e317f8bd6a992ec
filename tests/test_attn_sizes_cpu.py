"""Workspaces of grouped attention on the host: every size that a call may have gets one."""
import random

import pytest

import paper_2609_34325_amd as dora


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
