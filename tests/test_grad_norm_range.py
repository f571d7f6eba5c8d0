"""Gradients that are finite and whose norm is beyond fp32: the norm in fp32 is inf, nothing is flagged, and the factor is that of the norm in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2507_10392_amd as zs

gpu = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


@gpu
@pytest.mark.parametrize("dtype,value,n,scale,most", [(torch.float32, 3e38, 1000, 1.0, 1e35), (torch.bfloat16, -3e38, 5000, 1.0, 2e38), (torch.float32, 1e38, 70000, 1024.0, 1.0),
                                                      (torch.float16, 60000.0, 300, 3e38, 1e30), (torch.float32, 3e38, 300000, 3e38, 1.0)], ids=str)
def test_a_norm_beyond_fp32(gpu_device, dtype, value, n, scale, most):
    """factor: one quotient in 64 bits, 2^-53 of itself and of the norm's, rounded to fp32: 2^-24 of itself, or, below 2^-126, half of 2^-149."""
    print("[case] norm beyond fp32", dtype, value, n, flush=True)
    x = torch.full((n,), value, dtype=dtype, device="cuda")
    y = torch.full_like(x, 9.0)
    tensors = zs.tensor_list([x], [y])
    sumsq, norm, factor = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    overflow = torch.zeros(1, dtype=torch.int32, device="cuda")
    zs.grad_norm(stream(), tensors, scale, most, sumsq, norm, factor, overflow, torch.empty(zs.grad_norm_scratch_bytes(tensors), dtype=torch.uint8, device="cuda"))
    zs.grad_scale(stream(), tensors, factor)
    want = float(np.float32(scale)) * abs(float(x[0])) * math.sqrt(n)
    assert want > float(np.finfo(np.float32).max) and float(norm) == math.inf and int(overflow) == 0
    quotient = float(np.float32(most)) / want
    assert abs(float(factor) - quotient) <= 1.01 * 2.0 ** -24 * quotient + 2.0 ** -150
    assert torch.equal(y, (x.float() * factor).to(dtype))
