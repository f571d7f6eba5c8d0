"""The gated delta rule for keys of unlike length: what the header states of the half precision that inverses, keys and queries are held in.

Bounds, beside those of delta_reference.py.  An element of the inverse is held to 2^-25 absolutely (half of half's least step; larger ones to 2^-22 of themselves),
and multiplies up to 64 values z_j = beta_j (v_j - ..), whose errors have no common sign: 8 2^-25 of the largest z.  With keys between |k| and |k| / r and beta
about 1 / |k|^2, that is r^2 times as large as the values v of the longest keys, whose part of the state it enters; the state itself, of which the
shortest keys have |k| z, is r times as large.  So 2^-22 r of the state's norm; and an element of a key, 2^-28 of the largest one, is 2^-28 r of the
shortest key.  The factor between a result's terms and itself that delta_reference.py counts for gradients is counted here too."""
import math

import numpy as np
import pytest
import torch

from delta_reference import TD, Case, bound, check, reference_of
from test_delta_rule import Run, say

gpu = pytest.mark.gpu


def of_lengths(c, dtype, r):
    """Keys between 1 and 1 / r long, in any order, beta between 0 and 2 over their squares."""
    x, rng = c.inputs(dtype), np.random.default_rng(c.seed)
    length = torch.from_numpy(np.exp2(-rng.uniform(0, math.log2(r), (c.T, c.nk))))
    length[::17], length[5::17] = 1.0, 1.0 / r
    x["k"] = (x["k"] * length[..., None]).to(TD[dtype]).double()
    square = x["k"].square().sum(-1).repeat_interleave(c.nv // c.nk, 1)
    x["beta"] = (torch.from_numpy(rng.uniform(0.1, 1.9, (c.T, c.nv))) / square).float().double()
    x["g"] = x["g"] * 0.05   # states that are kept over a chunk
    return x


@gpu
@pytest.mark.parametrize("dtype,log2r", [(0, 6), (1, 3), (1, 6), (1, 10), (1, 13), (2, 3), (2, 6)])
def test_keys_of_unlike_length(gpu_device, dtype, log2r):
    say("key lengths", dtype, log2r)
    r = 2.0 ** log2r
    c = Case(150, 1, 2, 64, 48, [64, 86], h0=True, ht=True, seed=5, ostd=1.0 if dtype < 2 else 0.125)
    x = of_lengths(c, dtype, r)
    want = reference_of(c, x)
    if dtype == 2:
        assert all(float(want[n].abs().max()) < 65504 for n in ("o", "dq", "dk", "dv"))
    run = Run(c, dtype, x)
    run.all()
    for n in ("o", "ht", "dq", "dk", "dv", "dg", "dbeta", "dh0"):
        b = bound(n, dtype, 2)
        more = 0.0 if dtype == 0 else 2.0 ** -22 * r * math.sqrt(2) * (1 if n in ("o", "ht") else 10)
        check(n, getattr(run, n), want[n], dtype, 2, allow=(b + more) / b)
