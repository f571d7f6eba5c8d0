"""The gated delta rule in 64 bits, token after token as its definition says, with gradients by automatic differentiation of that; and how far a correct
kernel may be off it.

Bounds.  With keys of length one and 0 <= beta <= 2 a step changes a state by a factor of norm at most one, so an error made in a chunk is carried to the end without
growing.  A chunk makes about ten products (of the state with keys and queries, of the triangular matrices, of what is written), each with
an error of at most EPS of its size: bf16 pairs leave 2^-18 of a value and drop a product of 2^-18, together at most 2^-16; half pairs 2^-22, and their fp32
sums of 128 terms, like those of fp32, 128 2^-24 at most, sqrt(128) 2^-24 = 2^-20.5 as a rule.  Errors of different places have no common sign, so over n
chunks they grow as sqrt(n): relative to the 2-norm of a result, 10 sqrt(n) EPS.  Gradients go through both walks, and dbeta and dg are differences of sums: ten
times that.  A 16-bit result is rounded once: u = finfo.eps / 2 of itself.  Single values: forty times the bound, relative to the larger of themselves and
the result's root mean square."""
import math

import numpy as np
import torch

TD = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}
EPS = {0: 2.0 ** -20, 1: 2.0 ** -16, 2: 2.0 ** -20}


class Case:
    def __init__(self, T, nk, nv, dk, dv, lengths, first=0, h0=False, ht=False, scale=None, seed=0, g=None, beta=None, keys="unit", vstd=1.0, ostd=1.0):
        self.T, self.nk, self.nv, self.dk, self.dv, self.lengths, self.first, self.has_h0, self.has_ht = T, nk, nv, dk, dv, lengths, first, h0, ht
        self.scale = float(np.float32(dk ** -0.5 if scale is None else scale))
        self.offsets = [first + sum(lengths[:i]) for i in range(len(lengths) + 1)]
        assert self.offsets[-1] <= T
        self.seed, self.g_is, self.beta_is, self.keys, self.vstd, self.ostd = seed, g, beta, keys, vstd, ostd

    def __str__(self):
        return "%d-%d.%d-%d.%d-%s%s%s" % (self.T, self.nk, self.nv, self.dk, self.dv, "+".join(map(str, self.lengths[:6])), "-h0" * self.has_h0, "-ht" * self.has_ht)

    def inputs(self, dtype):
        """Values that the type holds, as float64 on the CPU."""
        rng = np.random.default_rng(1000 + self.seed)
        T, nk, nv, dk, dv, n = self.T, self.nk, self.nv, self.dk, self.dv, len(self.lengths)
        hold = lambda x, t=TD[dtype]: torch.from_numpy(np.asarray(x, dtype=np.float32)).to(t).double()
        unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)
        x = {"q": unit(rng.standard_normal((T, nk, dk))), "k": unit(rng.standard_normal((T, nk, dk)) + rng.standard_normal((1, nk, dk)))}
        if self.keys == "same":
            x["k"] = np.broadcast_to(x["k"][:1], x["k"].shape).copy()
        x = {a: hold(b) for a, b in x.items()}
        x["v"] = hold(rng.standard_normal((T, nv, dv)) * self.vstd)
        g = -np.exp(rng.uniform(math.log(1e-3), math.log(3.0), (1, nv))) * np.log1p(np.exp(rng.standard_normal((T, nv))))
        x["g"] = hold(g if self.g_is is None else self.g_is(rng, T, nv), torch.float32)
        x["beta"] = hold(1 / (1 + np.exp(-rng.standard_normal((T, nv)))) if self.beta_is is None else self.beta_is(rng, T, nv), torch.float32)
        x["h0"] = hold(rng.standard_normal((n, nv, dk, dv)) * 0.3 * self.vstd, torch.float32) if self.has_h0 else None
        x["dout"] = hold(rng.standard_normal((T, nv, dv)) * self.ostd)
        x["dht"] = hold(rng.standard_normal((n, nv, dk, dv)) * self.ostd, torch.float32) if self.has_ht else None
        return x


def rule(c, x):
    """-> o [T, nv, dv] and the last states, from the definition."""
    group = c.nv // c.nk
    o, last = [torch.zeros(c.nv, c.dv, dtype=torch.float64)] * c.T, []
    for n, length in enumerate(c.lengths):
        S = torch.zeros(c.nv, c.dk, c.dv, dtype=torch.float64) if x["h0"] is None else x["h0"][n]
        for t in range(c.offsets[n], c.offsets[n + 1]):
            q, k = x["q"][t].repeat_interleave(group, 0), x["k"][t].repeat_interleave(group, 0)
            S = torch.exp(x["g"][t])[:, None, None] * S
            u = x["beta"][t][:, None] * (x["v"][t] - (S * k[:, :, None]).sum(1))
            S = S + k[:, :, None] * u[:, None]
            o[t] = c.scale * (S * q[:, :, None]).sum(1)
        last.append(S)
    return torch.stack(o), torch.stack(last)


NAMES = ("q", "k", "v", "g", "beta", "h0")


def reference(c, dtype):
    x = c.inputs(dtype)
    return x, reference_of(c, x)


def reference_of(c, x):
    leaves = {n: x[n].clone().requires_grad_() for n in NAMES if x[n] is not None}
    o, ht = rule(c, {**x, **leaves})
    loss = (o * x["dout"]).sum()
    if x["dht"] is not None:
        loss = loss + (ht * x["dht"]).sum()
    grads = torch.autograd.grad(loss, list(leaves.values()))
    return {"o": o.detach(), "ht": ht.detach(), **{"d" + n: d for n, d in zip(leaves, grads)}}


def bound(name, dtype, chunks):
    u = torch.finfo(TD[dtype]).eps / 2 if name in ("o", "dq", "dk", "dv") and dtype else 2.0 ** -24
    return u + 10 * math.sqrt(max(1, chunks)) * EPS[dtype] * (1 if name in ("o", "ht") else 10)


def check(name, got, want, dtype, chunks, allow=1.0):
    got, want = got.double().cpu().reshape(-1), want.reshape(-1)
    assert got.shape == want.shape and torch.isfinite(got).all(), name
    d, norm = got - want, float(want.norm())
    b = bound(name, dtype, chunks) * allow
    rel = float(d.norm()) / norm if norm else float(d.norm())
    big = float((d.abs() / want.abs().clamp(min=norm / math.sqrt(max(1, want.numel())) or 1.0)).max()) if want.numel() else 0.0
    print("  %-6s rel %.2e of %.2e, max %.2e" % (name, rel, b, big), flush=True)
    assert rel <= b and big <= 40 * b, (name, rel, big, b)
