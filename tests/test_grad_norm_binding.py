"""What the Python calls of the gradients' norm refuse before an address of it reaches the library: results of other types (a float32 sum of squares would be
written with 8 bytes), tensors on the host, and tensors on another GPU than the gradients."""
from types import SimpleNamespace

import pytest
import torch

import paper_2507_10392_amd as zs

gpu = pytest.mark.gpu
RESULTS = {"sumsq": torch.float64, "norm": torch.float32, "factor": torch.float32, "overflow": torch.int32}


class Elsewhere:
    """What the checks ask a tensor for; any use of its address fails the test."""

    is_cuda = True

    def __init__(self, dtype=torch.float32, index=0, n=1, contiguous=True):
        self.dtype, self.device, self.n, self.contiguous = dtype, torch.device("cuda", index), n, contiguous

    def get_device(self):
        return self.device.index

    def numel(self):
        return self.n

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        raise AssertionError("the address was taken")


def norm_of(tensors, scratch, **results):
    a = {**dict.fromkeys(RESULTS), **results}
    zs.grad_norm(None, tensors, 1.0, 1.0, a["sumsq"], a["norm"], a["factor"], a["overflow"], scratch)


ON_0 = SimpleNamespace(n=0, c=None, gpu=0)   # a list of tensors on the first GPU


@pytest.mark.parametrize("name", sorted(RESULTS))
def test_results_that_are_refused(name):
    scratch = Elsewhere(torch.uint8, n=256)
    others = [t for t in (torch.float64, torch.float32, torch.int32, torch.int64, torch.bfloat16) if t != RESULTS[name]]
    bad = [Elsewhere(t) for t in others] + [Elsewhere(RESULTS[name], index=1), Elsewhere(RESULTS[name], n=0), torch.zeros(1, dtype=RESULTS[name])]
    for t in bad:
        with pytest.raises(ValueError, match=name):
            norm_of(ON_0, scratch, **{name: t})
    if name == "factor":
        for t in bad:
            with pytest.raises(ValueError, match=name):
                zs.grad_scale(None, ON_0, t)


def test_scratch_that_is_refused():
    for scratch in (torch.zeros(256, dtype=torch.uint8), Elsewhere(torch.uint8, index=1, n=256), Elsewhere(torch.uint8, n=256, contiguous=False)):
        with pytest.raises(ValueError, match="scratch"):
            norm_of(ON_0, scratch)
    with pytest.raises(ValueError, match="scratch"):
        norm_of(zs.tensor_list([]), torch.zeros(256, dtype=torch.uint8))


def test_factors_of_a_stage_that_are_refused():
    stage = object.__new__(zs.Stage)
    stage.h, stage.stream = None, SimpleNamespace(device=torch.device("cuda", 0))
    for t in (torch.zeros(1), Elsewhere(torch.float64), Elsewhere(torch.bfloat16), Elsewhere(index=1), Elsewhere(n=0)):
        with pytest.raises(ValueError):
            stage.set_grad_factor(t)
    assert not hasattr(stage, "_factor")   # a refused one takes no kept one's place
    with pytest.raises(zs.StageError):
        zs.grad_scale(None, ON_0, None)


@gpu
def test_results_on_the_gpu_are_refused_by_type_and_taken_when_right(gpu_device):
    print("[case] binding", flush=True)
    x = [torch.full((100,), 2.0, device="cuda")]
    tensors = zs.tensor_list(x)
    scratch = torch.empty(zs.grad_norm_scratch_bytes(tensors), dtype=torch.uint8, device="cuda")
    right = {n: torch.zeros(1, dtype=t, device="cuda") for n, t in RESULTS.items()}
    for n in RESULTS:
        with pytest.raises(ValueError, match=n):
            norm_of(tensors, scratch, **{**right, n: torch.zeros(1, dtype=torch.float16, device="cuda")})
        with pytest.raises(ValueError, match=n):
            norm_of(tensors, scratch, **{**right, n: right[n].cpu()})
    zs.grad_norm(torch.cuda.current_stream().cuda_stream, tensors, 1.0, 1.0, *right.values(), scratch)
    zs.grad_scale(torch.cuda.current_stream().cuda_stream, tensors, right["factor"])
    assert float(right["sumsq"]) == 400 and float(right["norm"]) == 20 and int(right["overflow"]) == 0
    assert torch.equal(x[0], torch.full((100,), 2.0, device="cuda") * right["factor"])
