"""The gated delta rule as a layer's mixer, trained and served: projections, keys and queries of length one, the rule and its gradients, the gradients' norm,
clipping and the optimizer, in fp32, against the same in 64 bits; and a prompt whose last state single tokens go on from.

Bounds: what delta_reference says of the rule's own results, twice.  The rest of a layer adds products of up to 240 terms and the norm's two passes, fp32 all, each
below 2^-20 of its result, which ten to a hundred times that of the rule's bound holds; the gradient of the norm drops its part along the key, one of 32 or more
directions.  The optimizer's first step of a gradient d is lr (d / (|d| + eps)), with eps here above every |d|, so that it is as smooth as d is."""
import math

import numpy as np
import pytest
import torch

import paper_2507_10392_amd as zs
from delta_reference import TD, Case, check, rule
from test_delta_rule import Run, say, step, stream
from test_grad_norm import Norm

gpu = pytest.mark.gpu
LR, B1, B2, EPS_ADAM, EPS_NORM, MAX_NORM = 0.01, 0.9, 0.95, 1.0, 1e-6, 0.05


def weights(c, H, seed):
    rng = np.random.default_rng(seed)
    hold = lambda *s, std=1.0: torch.from_numpy((rng.standard_normal(s) * std).astype(np.float32))
    x = hold(c.T, H)
    w = {"q": hold(H, c.nk * c.dk, std=H ** -0.5), "k": hold(H, c.nk * c.dk, std=H ** -0.5), "v": hold(H, c.nv * c.dv, std=H ** -0.5)}
    gain = torch.full((c.dk,), c.dk ** -0.5) * (1 + 0.02 * hold(c.dk))
    return x, w, gain, hold(c.T, c.nv, c.dv)


def exact(c, x, w, gain, gates, dout):
    """Outputs, the weights' gradients, their norm, and the weights after a clipped step."""
    leaves = {n: t.double().requires_grad_() for n, t in w.items()}
    leaves["gain"] = gain.double().requires_grad_()
    leaves.update({n: t.double().requires_grad_() for n, t in gates.items()})
    heads = lambda y: y / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS_NORM) * leaves["gain"]
    y = {n: x.double() @ leaves[n] for n in "qkv"}
    o, _ = rule(c, {"q": heads(y["q"].view(c.T, c.nk, c.dk)), "k": heads(y["k"].view(c.T, c.nk, c.dk)), "v": y["v"].view(c.T, c.nv, c.dv),
                    "g": leaves["g"], "beta": leaves["beta"], "h0": None})
    grads = dict(zip(leaves, torch.autograd.grad((o * dout.double()).sum(), list(leaves.values()))))
    norm = math.sqrt(sum(float((d * d).sum()) for d in grads.values()))
    clipped = {n: d * min(1.0, MAX_NORM / norm) for n, d in grads.items()}
    stepped = {n: w[n].double() - LR * clipped[n] / (clipped[n].abs() + EPS_ADAM) for n in w}
    return o.detach(), grads, norm, clipped, stepped


def heads_norm(x, gain, out, rstd):
    zs.ops.norm_fwd(stream(), 0, 1, x.numel() // gain.numel(), gain.numel(), x, gain, None, EPS_NORM, out, rstd, None)


class Layer:
    """The layer's buffers; forward, backward, clipping and the optimizer's step enqueue all their work on the current stream."""

    def __init__(self, c, x, w, gain, gates, dout):
        self.c, self.H = c, x.shape[1]
        self.x, self.w, self.gain = x.cuda(), {n: t.cuda() for n, t in w.items()}, gain.cuda()
        self.y = {n: torch.empty(c.T, t.shape[1], device="cuda") for n, t in w.items()}
        zeros = {"q": torch.zeros(c.T, c.nk, c.dk), "k": torch.zeros(c.T, c.nk, c.dk), "v": torch.zeros(c.T, c.nv, c.dv), "h0": None, "dht": None, "dout": dout, **gates}
        self.run = Run(c, 0, zeros)
        self.run.dh0 = None
        self.rstd = {n: torch.empty(c.T * c.nk, device="cuda") for n in "qk"}
        self.dw = {n: torch.zeros_like(t) for n, t in self.w.items()}
        self.dy = {n: torch.empty_like(self.y[n]) for n in "qk"}
        self.parts = {n: torch.empty(8, c.dk, device="cuda") for n in "qk"}
        self.dgain = torch.empty(c.dk, device="cuda")
        self.leaves = [*self.dw.values(), self.dgain, self.run.dg, self.run.dbeta]
        self.norm = Norm(self.leaves)
        self.m, self.v2 = ({n: torch.zeros_like(t) for n, t in self.w.items()} for _ in range(2))

    def product(self, ta, M, N, K, a, lda, b, ldb, out, accumulate):
        zs.ops.gemm(stream(), 0, ta, 0, M, N, K, a, lda, b, ldb, out, N, accumulate, None, None, 0, 1, 0, 0, 0, 0, 0, 0, 0)

    def gradients(self):
        c, r = self.c, self.run
        for n, w in self.w.items():
            self.product(0, c.T, w.shape[1], self.H, self.x, self.H, w, w.shape[1], self.y[n], 0)
        heads_norm(self.y["q"], self.gain, r.q, self.rstd["q"])
        heads_norm(self.y["k"], self.gain, r.k, self.rstd["k"])
        r.v = self.y["v"]
        r.table().fwd().bwd()
        for n, d in (("q", r.dq), ("k", r.dk)):
            zs.ops.norm_bwd(stream(), 0, 1, c.T * c.nk, c.dk, d, self.y[n], self.gain, self.rstd[n], None, None, self.dy[n], self.parts[n], None, 8)
            self.product(1, self.H, c.nk * c.dk, c.T, self.x, self.H, self.dy[n], c.nk * c.dk, self.dw[n], 1)
        self.product(1, self.H, c.nv * c.dv, c.T, self.x, self.H, r.dv, c.nv * c.dv, self.dw["v"], 1)
        torch.sum(torch.cat((self.parts["q"], self.parts["k"])), 0, out=self.dgain)
        return self

    def update(self):
        self.norm(1.0, MAX_NORM)
        zs.grad_scale(stream(), self.norm.list, self.norm.factor)
        clipped = [t.clone() for t in self.leaves]
        for n, w in self.w.items():
            zs.ops.adamw(stream(), 0, w.numel(), 0, w, None, self.dw[n], self.m[n], self.v2[n], LR, B1, B2, EPS_ADAM, 0.0, 1, 1.0)
        return clipped


LAYERS = [(Case(150, 2, 4, 32, 40, [70, 1, 64], first=5), 48), (Case(240, 1, 1, 64, 64, [240]), 64), (Case(130, 2, 2, 128, 32, [3, 126]), 40)]


@gpu
@pytest.mark.parametrize("case,H", LAYERS, ids=lambda x: str(x))
def test_a_step_of_training(gpu_device, case, H):
    say(case, H)
    c = case
    x, w, gain, dout = weights(c, H, 7)
    hidden = torch.ones(c.T, dtype=torch.bool)
    hidden[c.offsets[0]:c.offsets[-1]] = False
    i = c.inputs(0)
    gates = {n: i[n].float() for n in ("g", "beta")}
    dout[hidden] = 0.0
    want, grads, norm, clipped, stepped = exact(c, x, w, gain, gates, dout)
    layer = Layer(c, x, w, gain, gates, dout).gradients()
    chunks = -(-max(c.lengths) // 64)
    check("o", layer.run.o, want, 0, chunks, 2)
    for n in "qkv":
        check("d" + n, layer.dw[n], grads[n], 0, chunks, 2)
    check("dgain", layer.dgain, grads["gain"], 0, chunks, 2)
    check("dg", layer.run.dg, grads["g"], 0, chunks, 2)
    check("dbeta", layer.run.dbeta, grads["beta"], 0, chunks, 2)
    before = [t.clone() for t in layer.leaves]
    got = layer.update()
    layer.norm.check(before, 1.0, MAX_NORM)
    assert norm > MAX_NORM and abs(float(layer.norm.norm) - norm) <= 200 * math.sqrt(chunks) * 2.0 ** -20 * norm
    for t, b in zip(got, before):
        assert torch.equal(t, b * layer.norm.factor)
    for n in "qkv":
        moved = stepped[n] - w[n].double()
        # weights are below 1: a half step of fp32 beside the bound of what moves them
        d = layer.w[n].double().cpu() - w[n].double() - moved
        assert float(d.norm()) <= 400 * math.sqrt(chunks) * 2.0 ** -20 * float(moved.norm()) + 2.0 ** -24 * math.sqrt(d.numel()), n
        assert (layer.dw[n] == 0).all()


@gpu
def test_steps_of_training_in_a_graph(gpu_device):
    """Captured once, replayed over eager work in between: every replay is the eager step, bit by bit."""
    say("graph")
    c, H = LAYERS[0]
    i = c.inputs(0)
    x, w, gain, dout = weights(c, H, 7)
    args = (c, x, w, gain, {n: i[n].float() for n in ("g", "beta")}, dout)
    layer = Layer(*args)
    state = lambda a: [t for t in (*a.w.values(), *a.m.values(), *a.v2.values(), *a.dw.values(), a.run.dg, a.run.dbeta, a.norm.norm)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def once(a):
        a.gradients()
        a.update()

    with torch.cuda.stream(side):
        once(layer)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        once(layer)
    eager = Layer(*args)
    once(eager)   # as the layer's own one before the capture, which runs nothing
    for _ in range(4):
        once(eager)
        g.replay()
        torch.cuda.synchronize()
        for p, q in zip(state(eager), state(layer)):
            assert torch.equal(p, q)


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_a_prompt_and_the_tokens_behind_it(gpu_device, dtype):
    """Prompts in one call, then tokens one by one on their last states."""
    say("serving", dtype)
    prompts, more = [70, 0, 129, 1], 3
    whole = Case(sum(prompts) + more * len(prompts), 2, 4, 64, 72, [p + more for p in prompts], h0=True)
    x = whole.inputs(dtype)
    want, states = rule(whole, x)
    part = Case(sum(prompts), 2, 4, 64, 72, prompts, h0=True, seed=1)
    of = torch.cat([torch.arange(whole.offsets[n], whole.offsets[n] + p) for n, p in enumerate(prompts)])
    rows_of = lambda v: v[of] if v is not None and v.shape[0] == whole.T else v
    r = Run(part, dtype, {n: rows_of(v) if n != "h0" else v for n, v in x.items()}).table().fwd()
    check("o", r.o, want[of], dtype, 3)
    full = Run(whole, dtype, x)
    state, slots = r.ht, [2, 0, 3, 1]
    for i in range(more):
        at = torch.tensor([whole.offsets[n] + prompts[n] + i for n in slots])
        o = step(full, at, slots, state)
        check("o", o, want[at], dtype, 3)
    check("ht", state, states, dtype, 3)
