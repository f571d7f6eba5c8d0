"""The factor in a tensor that is written: workgroups would read it before and after.  In one that is only read it is like any other element."""
import pytest
import torch

import paper_2507_10392_amd as zs
from test_grad_norm import tensors

gpu = pytest.mark.gpu


@pytest.mark.parametrize("rows,factor", [([(4096, 4096, 64, 0)], 4096), ([(4096, 4096, 64, 0)], 4348), ([(4096, 8192, 64, 1)], 8316), ([(4096, 8192, 64, 0), (16384, 16384, 3, 2)], 16388)],
                         ids=str)
def test_a_factor_in_an_output_is_refused(rows, factor):
    assert zs.lib().stage_op_grad_scale(None, len(rows), tensors(*rows), factor) == zs.STAGE_ERR_ARG


def test_a_factor_beside_the_outputs_is_not_refused():
    """On the host: no tensors at all, so that nothing is launched, and elements of none."""
    assert zs.lib().stage_op_grad_scale(None, 0, None, 4096) == zs.STAGE_OK
    assert zs.lib().stage_op_grad_scale(None, 1, tensors((4096, 4096, 0, 0)), 4096) == zs.STAGE_OK


@gpu
def test_a_factor_that_is_one_of_the_gradients(gpu_device):
    print("[case] factor beside outputs", flush=True)
    x = torch.arange(1.0, 5001.0, device="cuda") / 5000
    y = torch.zeros(5002, device="cuda")
    y[5000] = 0.375
    for factor in (x[77:78], y[5000:5001]):   # read as a gradient too; right behind the output
        zs.grad_scale(torch.cuda.current_stream().cuda_stream, zs.tensor_list([x], [y[:5000]]), factor)
        assert torch.equal(y[:5000], x * factor) and float(y[5000]) == 0.375 and float(y[5001]) == 0
