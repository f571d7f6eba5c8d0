"""Attention inside packed documents where the blocks are dealt out by their lengths: documents beyond the steps that the lengths are compared in, blocks
that padding begins or ends in.  Every block is computed once (results lie in buffers of NaN) and is right."""
import pytest
import torch

from docs_reference import Case
from test_attention_docs import Run, check_part, chunks, say

gpu = pytest.mark.gpu
CASES = [Case(20000, 16, 16, 64, [60, 17000, 900, 1500]), Case(32768, 8, 8, 32, [2000] * 9 + [3000, 11700]), Case(4096, 32, 32, 128, [2500, 1500]),
         Case(4096, 32, 32, 64, [40, 2900, 1000], first=90, slopes=True), Case(4096, 64, 16, 64, [2000, 1, 1999], prefix=[0, 1, 500], first=33)]


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("c", CASES, ids=str)
def test_blocks_in_the_order_of_their_lengths(gpu_device, c, dtype):
    say(c, dtype)
    r = Run(c, dtype)
    for x in r.all():
        assert not x.isnan().any()
    group = c.nh // c.nkv
    for kv in (0, c.nkv - 1):
        h = slice(kv * group, (kv + 1) * group)
        part = Case(c.T, group, 1, c.d, c.lengths, c.prefix, c.first, scale=c.scale)
        part.slopes = c.slopes[h] if c.slopes else None
        cols, key = slice(h.start * c.d, h.stop * c.d), slice(kv * c.d, (kv + 1) * c.d)
        q, k, v, dout = r.q[:, cols].cuda(), r.k[:, key].cuda(), r.v[:, key].cuda(), r.dout[:, cols].cuda()
        for run in chunks(part):
            check_part(part, dtype, run, q, k, v, dout, r.go[:, cols], r.lse[h], r.dq[:, cols], r.dk[:, key], r.dv[:, key])
        torch.cuda.empty_cache()
