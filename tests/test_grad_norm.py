"""The norm of many gradient tensors and their clipping, against sums in 64 bits.

Bounds: an element's square is exact in 64 bits (24 bits times 24), n of them are added with at most n 2^-53 of their sum, whatever the order; the norm
and the factor are rounded to fp32 once, 2^-24 of themselves, after a root and a quotient in 64 bits.  A clipped element is the fp32
product of the element and the factor, rounded to its type: one value, compared bit by bit."""
import math

import numpy as np
import pytest
import torch

import paper_2507_10392_amd as zs

gpu = pytest.mark.gpu
TD = [torch.float32, torch.bfloat16, torch.float16]
E24 = 2.0 ** -24


def say(*a):
    print("[case]", *a, flush=True)


def stream():
    return torch.cuda.current_stream().cuda_stream


def total(tensors):
    return math.fsum(float(x.double().cpu().square().sum()) for x in tensors if x.numel())


class Norm:
    def __init__(self, tensors, outs=None):
        self.list = zs.tensor_list(tensors, outs)
        self.scratch = torch.full((zs.grad_norm_scratch_bytes(self.list) // 8,), math.nan, dtype=torch.float64, device="cuda")
        self.sumsq, self.norm, self.factor = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        self.overflow = torch.zeros(1, dtype=torch.int32, device="cuda")

    def __call__(self, scale=1.0, max_norm=1.0):
        zs.grad_norm(stream(), self.list, scale, max_norm, self.sumsq, self.norm, self.factor, self.overflow, self.scratch)
        return self

    def check(self, tensors, scale=1.0, max_norm=1.0):
        want, n = total(tensors), sum(x.numel() for x in tensors)
        got = float(self.sumsq)
        assert abs(got - want) <= (2 * n + 8) * 2.0 ** -53 * want, (got, want)
        scale, max_norm = float(np.float32(scale)), float(np.float32(max_norm))   # the call's arguments are C floats: 0.005 goes in 2^-25.2 of itself off
        norm = scale * math.sqrt(want)
        # Beyond fp32's range the rounding is to inf (a thousand gradients of 3e38 have the norm 9.5e39), and below 2^-126 its half step is 2^-150
        most = float(np.finfo(np.float32).max)
        assert float(self.norm) == math.inf if norm > most * (1 + E24) else abs(float(self.norm) - norm) <= 1.01 * E24 * norm + 2.0 ** -150
        factor = max_norm / norm if norm > max_norm else 1.0
        assert abs(float(self.factor) - factor) <= 1.01 * E24 * factor + 2.0 ** -150
        assert int(self.overflow) == 0


def draw(rng, n, dtype, shift=0, std=0.01):
    """n values at `shift` elements behind a multiple of 16 bytes."""
    buf = torch.zeros(n + shift + 8, dtype=dtype, device="cuda")
    buf[shift:shift + n] = torch.from_numpy((rng.standard_normal(n) * std).astype(np.float32)).to("cuda").to(dtype)
    return buf[shift:shift + n]


@gpu
@pytest.mark.parametrize("sizes", [[1], [7], [4096], [8191, 1, 0, 3], [16384 * 3 + 5, 65536], [1 << 20, 12345, 0, 0, 2]], ids=str)
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_norm_and_clipping(gpu_device, dtype, sizes):
    say("norm", dtype, sizes)
    rng = np.random.default_rng(len(sizes) + dtype)
    for shift, out_shift in ((0, 0), (1, 1), (3, 0)):
        x = [draw(rng, n, TD[dtype], shift) for n in sizes]
        y = [torch.full((n + out_shift + 1,), 9.0, dtype=TD[dtype], device="cuda") for n in sizes]
        run = Norm(x, [b[out_shift:out_shift + n] for b, n in zip(y, sizes)])
        for scale, most in ((1.0, 0.005), (1.0 / 1024, 1e-6), (2.0, 1e9)):
            run(scale, most).check(x, scale, most)
            zs.grad_scale(stream(), run.list, run.factor)
            for a, b, n in zip(x, y, sizes):
                assert torch.equal(b[out_shift:out_shift + n], (a.float() * run.factor).to(TD[dtype]))
                assert (b[:out_shift] == 9).all() and (b[out_shift + n:] == 9).all()


@gpu
def test_many_tensors_of_all_types_in_place(gpu_device):
    """More than a launch takes, empty ones among them, and pieces larger than the least."""
    say("many")
    rng = np.random.default_rng(3)
    x = [draw(rng, int(rng.integers(0, 3)) * int(rng.integers(1, 5000)) + i % 3, TD[i % 3], int(rng.integers(0, 8))) for i in range(400)]
    x.append(draw(rng, 70_000_001, torch.bfloat16, 1))
    before = [t.clone() for t in x]
    run = Norm(x)(1.0, 0.25)
    run.check(x, 1.0, 0.25)
    first = float(run.sumsq)
    zs.grad_scale(stream(), run.list, run.factor)
    for a, b in zip(before, x):
        assert torch.equal((a.float() * run.factor).to(a.dtype), b)
    for a, b in zip(before, x):
        b.copy_(a)
    assert float(run(1.0, 0.25).sumsq) == first   # the same bits


@gpu
def test_large_small_and_no_gradients(gpu_device):
    say("extremes")
    for value, dtype in ((3e38, torch.float32), (2e-38, torch.float32), (1e-40, torch.float32), (3e38, torch.bfloat16), (60000.0, torch.float16), (6e-8, torch.float16)):
        x = [torch.full((1000,), value, dtype=dtype, device="cuda")]
        Norm(x)(1.0, 1e-30).check(x, 1.0, float(np.float32(1e-30)))
    for x in ([], [torch.zeros(0, device="cuda")], [torch.zeros(5, device="cuda")]):
        run = Norm(x)(1.0, 0.0)
        assert float(run.sumsq) == 0 and float(run.norm) == 0 and float(run.factor) == 1 and int(run.overflow) == 0
        zs.grad_scale(stream(), run.list, run.factor)


@gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_scales_nothing_and_is_told(gpu_device, value):
    say("not finite", value)
    rng = np.random.default_rng(4)
    for dtype in TD:
        x = [draw(rng, 100_000, dtype), draw(rng, 33, dtype, 1)]
        x[1][32] = value
        before = [t.clone() for t in x]
        run = Norm(x)(1.0, 1e-3)
        zs.grad_scale(stream(), run.list, run.factor)
        assert int(run.overflow) == 1 and float(run.factor) == 1 and not math.isfinite(float(run.norm))
        for a, b in zip(before, x):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        run.overflow.fill_(4)
        assert int(run(1.0, 1e-3).overflow) == 5


@gpu
def test_sums_of_shards_make_the_same_factor(gpu_device):
    say("shards")
    rng = np.random.default_rng(5)
    x = [draw(rng, 50_000, torch.float32) for _ in range(4)]
    parts = [Norm([t])() for t in x]
    sums = torch.cat([p.sumsq for p in parts])
    whole = Norm(x)(0.5, 0.125)
    for p in parts:
        p.overflow.zero_()
    p = parts[0]
    zs.ops.grad_factor(stream(), 4, sums, 0.5, 0.125, p.sumsq, p.norm, p.factor, p.overflow)
    p.check(x, 0.5, 0.125)
    assert abs(float(p.factor) - float(whole.factor)) <= 2 * E24 * float(p.factor)
    zs.ops.grad_factor(stream(), 1, sums, 0.5, 0.125, None, None, p.factor, None)


@gpu
def test_replays_of_a_graph(gpu_device):
    """Norm and clipping captured; every replay reads the gradients of its time, with eager work between."""
    say("graph")
    rng = np.random.default_rng(6)
    x = [draw(rng, n, torch.float32) for n in (100_001, 5, 4096)]
    y = [torch.zeros_like(t) for t in x]
    run = Norm(x, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        zs.grad_scale(stream(), run.list, run.factor)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
        zs.grad_scale(stream(), run.list, run.factor)
    for i in range(4):
        for t in x:
            t.copy_(torch.from_numpy((rng.standard_normal(t.numel()) * 10.0 ** -i).astype(np.float32)))
        for t in y:
            t.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        run.check(x)
        for a, b in zip(x, y):
            assert torch.equal(a * run.factor, b)


@gpu
@pytest.mark.parametrize("name", ["C1", "C3t", "C3h"])
def test_the_stage_clips_by_the_factor(gpu_device, name):
    """A step with a device factor is, bit by bit, the step with the product in grad_scale; taken off, it is the step as before."""
    from harness import GpuStage
    from workloads import get_config, make_inputs
    say("stage", name)
    cfg = get_config(name)
    inp = make_inputs(cfg, perturbed=True, num_microbatches=2)
    res = []
    for way in ("plain", "factor", "host", "off"):
        g = GpuStage(cfg, inp, max_microbatches=2)
        g.run_microbatches(inp, M=2)
        run = Norm([g.grad[g.shard[0]:g.shard[1]]])(0.5, 1e-3)
        run.check([g.grad[g.shard[0]:g.shard[1]]], 0.5, float(np.float32(1e-3)))
        assert float(run.factor) < 1
        if way in ("factor", "off"):
            g.stage.set_grad_factor(run.factor)
        if way == "off":
            g.stage.set_grad_factor(None)
        res.append(g.step(1, float(np.float32(0.5) * np.float32(run.factor.item())) if way == "host" else 0.5))
        g.stage.close()
    plain, factor, host, off = res
    for k in ("m", "v", "params", "master"):
        assert np.array_equal(factor[k], host[k]) and np.array_equal(plain[k], off[k]), k
    assert not np.array_equal(plain["m"], factor["m"])


# ---------------------------------------------------------------------------------------------- refusals, on the host
def tensors(*rows):
    from paper_2507_10392_amd.binding import TensorC
    return (TensorC * max(1, len(rows)))(*[TensorC(*r, 0) for r in rows])


@pytest.mark.parametrize("rows", [[(4096, 4096, 8, 3)], [(4096, 4096, -1, 0)], [(None, 4096, 8, 0)], [(4098, 4096, 8, 0)], [(4097, 4096, 8, 1)],
                                  [(4096, 4096, (1 << 50) + 1, 1)], [(4096, 4096, 1 << 50, 0)]], ids=str)
def test_lists_that_are_refused(rows):
    L, t, n = zs.lib(), tensors(*rows), len(rows)
    assert L.stage_op_grad_norm_scratch_bytes(n, t) == -zs.STAGE_ERR_ARG
    assert L.stage_op_grad_norm(None, n, t, 1.0, 1.0, None, None, None, None, 4096, 1 << 20) == zs.STAGE_ERR_ARG
    assert L.stage_op_grad_scale(None, n, t, 4096) == zs.STAGE_ERR_ARG


def test_other_refusals():
    L, t = zs.lib(), tensors((4096, 4096, 8, 0))
    need = L.stage_op_grad_norm_scratch_bytes(1, t)
    assert need > 0 and need % 256 == 0

    def norm(n=1, t=t, scale=1.0, most=1.0, sumsq=None, norm=None, factor=None, overflow=None, scratch=4096, size=need):
        return L.stage_op_grad_norm(None, n, t, scale, most, sumsq, norm, factor, overflow, scratch, size)

    for bad in (dict(n=-1), dict(t=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(most=-1.0), dict(most=math.nan),
                dict(sumsq=4100), dict(norm=4098), dict(factor=4097), dict(overflow=4098)):
        assert norm(**bad) == zs.STAGE_ERR_ARG, bad
    for bad in (dict(scratch=None), dict(scratch=4224), dict(size=need - 1)):
        assert norm(**bad) == zs.STAGE_ERR_WORKSPACE, bad
    assert L.stage_op_grad_scale(None, 1, t, None) == zs.STAGE_ERR_ARG and L.stage_op_grad_scale(None, 1, t, 4098) == zs.STAGE_ERR_ARG
    for rows in ([(4096, None, 8, 0)], [(4096, 4098, 8, 0)]):
        assert L.stage_op_grad_scale(None, 1, tensors(*rows), 4096) == zs.STAGE_ERR_ARG
    for n, p, scale in ((0, 4096, 1.0), (1, None, 1.0), (1, 4100, 1.0), (1, 4096, 0.0)):
        assert L.stage_op_grad_factor(None, n, p, scale, 1.0, None, None, None, None) == zs.STAGE_ERR_ARG
    assert L.stage_set_grad_factor(None, 4096) == zs.STAGE_ERR_ARG


@pytest.mark.parametrize("rows", [[(4096, 4096, 64, 0)] * 2, [(4096, 4096, 64, 0), (4224, 4224, 64, 1)], [(4096, 8192, 64, 0), (16384, 8320, 64, 0)],
                                  [(4096, 8192, 64, 0), (8444, 8444, 64, 0)], [(4096, 4100, 64, 0)], [(4100, 4096, 64, 1)], [(4096, 8192, 64, 0), (8192, 16384, 8, 0)]], ids=str)
def test_scaling_over_another_tensor_is_refused(rows):
    """The same tensor twice, outputs over one another or over inputs; the norm of such lists is fine."""
    L, t = zs.lib(), tensors(*rows)
    assert L.stage_op_grad_scale(None, len(rows), t, 4096) == zs.STAGE_ERR_ARG
    assert L.stage_op_grad_norm_scratch_bytes(len(rows), t) > 0


@gpu
def test_lists_that_share_what_is_only_read(gpu_device):
    """The same input twice, to outputs of its own each, and a tensor that begins where another one ends."""
    say("shared inputs")
    rng = np.random.default_rng(5)
    x = draw(rng, 5000, torch.float32)
    a, b = x[:3000], x[3000:]
    outs = [torch.zeros(3000, device="cuda"), torch.zeros(3000, device="cuda"), b]
    run = Norm([a, a, b], outs)(1.0, 0.01)
    run.check([a, a, b], 1.0, 0.01)
    want = [t * run.factor for t in (a, a, b)]
    zs.grad_scale(stream(), run.list, run.factor)
    assert float(run.factor) < 1
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_lists_of_other_tensors_are_refused():
    x = torch.zeros(4, 4)
    for bad in ([x], [x.to(torch.int32)]):
        with pytest.raises(ValueError):
            zs.tensor_list(bad)
    with pytest.raises(ValueError):
        zs.tensor_list([x], [])


def test_scratch_holds_every_piece():
    """8 bytes for each piece of 16 KB, twice as large until there are 4096, and one for the rest of every tensor."""
    L = zs.lib()
    for rows in ([(4096, None, n, d)] * m for n in (1, 5, 4096, 100_003, 70_000_001, 10 ** 10) for d in (0, 1) for m in (1, 3, 300)):
        size = [4, 2][rows[0][3]] * rows[0][2]
        piece = 16384
        while size * len(rows) // piece > 4096:
            piece *= 2
        need = 8 * len(rows) * -(-size // piece)
        got = L.stage_op_grad_norm_scratch_bytes(len(rows), tensors(*rows))
        assert need <= got <= need + 512, rows[0]
