"""The scratch that the gradient of attention inside packed documents asks for: a program allocates it once, for its longest microbatch."""
import math

import numpy as np
import pytest
import torch

import paper_2507_10392_amd as zs
from docs_reference import Case
from test_attention_docs import Run, say

gpu = pytest.mark.gpu


def test_scratch_of_a_longer_microbatch_serves_shorter_ones():
    """Host only: the bytes never fall as T grows, whatever the launches that a T takes."""
    rng = np.random.default_rng(8)
    shapes = [(dt, nh, nkv, d) for dt in (0, 1, 2) for nh, nkv in ((32, 8), (16, 1), (64, 8), (71, 1), (12, 2), (8, 8), (96, 4), (300, 1), (1, 1)) for d in (8, 128)]
    for dt, nh, nkv, d in shapes:
        last = 0
        for T in sorted({1, 2, 31, 32, 33} | set(range(64, 40000, 997)) | set(int(x) for x in rng.integers(1, 40000, 200)) |
                        {k * n + e for k in (32, 64, 128) for n in range(1, 257) for e in (0, 1)}):
            n = zs.attention_docs_bwd_scratch_bytes(dt, T, nh, nkv, d)
            assert n >= last, (dt, T, nh, nkv, d, n, last)
            last = n


@gpu
def test_one_scratch_for_all_lengths(gpu_device):
    """Allocated for 4096 tokens, whose key heads need no parts, and used for fewer, whose do."""
    nh, nkv, d = 32, 8, 128
    n = zs.attention_docs_bwd_scratch_bytes(1, 4096, nh, nkv, d)
    scratch = torch.full((n // 4,), math.nan, device="cuda")
    for T in (17, 512, 1984):
        say(T)
        r = Run(Case(T, nh, nkv, d, [T - 5]), 1)
        want = r.all()
        r.scratch = scratch
        for a, b in zip(want, r.all()):
            assert torch.equal(a, b)
