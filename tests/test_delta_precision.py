"""What the gated delta rule forms in 32 bits, its last states, dg, dbeta and dh0, against 64 bits, closely enough to tell products of half pairs and of
three bf16 from products of bf16 pairs (delta_precision.py has the bounds).  That these bounds do tell is shown on the CPU, with the mistake in the
64-bit form."""
import pytest
import torch

from delta_precision import bounds, chunked, off, pairs
from delta_reference import Case, reference_of
from test_delta_rule import Run, say

gpu = pytest.mark.gpu

CASES = [
    Case(60, 1, 2, 128, 128, [60], h0=True, ht=True),
    Case(128, 1, 2, 128, 128, [128], h0=True, ht=True, g=lambda rng, T, n: -0.002 * rng.random((T, n))),
    Case(200, 2, 2, 128, 128, [128, 72], h0=True, ht=True, seed=2),
    Case(400, 1, 2, 72, 96, [300, 100], h0=True, ht=True, seed=3),
]
HALF, BF16, THREE = pairs(torch.float16, 2), pairs(torch.bfloat16, 2), pairs(torch.bfloat16, 3)


@pytest.mark.parametrize("case", CASES[:2], ids=str)
def test_the_chunked_form_is_the_rule(case):
    x = case.inputs(1)
    got, want = chunked(case, x)[0], reference_of(case, x)
    for n in got:
        assert off(got[n], want[n]) < 1e-13, n


@pytest.mark.parametrize("case", CASES, ids=str)
def test_operands_as_they_are_held_keep_the_bounds(case):
    """A third of the bounds: the other part is the sums', which are exact here."""
    x = case.inputs(1)
    want, terms = chunked(case, x)
    b, got = bounds(case, want, terms), chunked(case, x, HALF, THREE)[0]
    for n in b:
        assert off(got[n], want[n]) < b[n] / 3, n


@pytest.mark.parametrize("mistake", ["walks", "gradients", "both"])
def test_bf16_pairs_do_not_keep_the_bounds(mistake):
    walk, grad = (HALF if mistake == "gradients" else BF16), (THREE if mistake == "walks" else BF16)
    seen = set()
    for case in (CASES[0], CASES[2]):
        x = case.inputs(1)
        want, terms = chunked(case, x)
        b, got = bounds(case, want, terms), chunked(case, x, walk, grad)[0]
        seen |= {n for n in b if off(got[n], want[n]) > b[n]}
    assert seen == ({"dg", "dbeta"} if mistake == "gradients" else {"ht", "dg", "dbeta", "dh0"})


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_results_of_32_bits(gpu_device, case, dtype):
    say("precision", case, dtype)
    x = case.inputs(dtype)
    want, terms = chunked(case, x)
    b, run = bounds(case, want, terms), Run(case, dtype, x)
    run.all()
    found = {n: off(getattr(run, n), want[n]) for n in b}
    print("  " + "  ".join("%s %.1e of %.1e" % (n, found[n], b[n]) for n in b), flush=True)
    for n in b:
        assert found[n] <= b[n], (n, found[n], b[n])
