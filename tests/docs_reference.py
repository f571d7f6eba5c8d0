"""Attention inside packed documents in 64 bits (on the device of its inputs), and how far a correct kernel may be off it.

The bounds are worst cases of the roundings that the kernels make, element by element:
- scores: sums of d exact products in fp32, (d + 8) 2^-24 of the sum of absolute values; the cap, the bias and the change to powers of two,
  a few 2^-24 of their magnitudes.  An absolute error e of a score is a relative one of its weight.
- weights and their derivatives go into the second product in the tensors' type: half a step, u = finfo.eps / 2, of each, and in half
  never less than half the smallest subnormal step, 2^-25.  In fp32 and bf16 a weight below the smallest normal number, 2^-126, may become zero
  (exp(-87.4) = 2^-126.1 does on the hardware): off by up to 2^-126, times what the weight is multiplied by.
- that product's sums of n terms in fp32: (n + 8) 2^-24 of the sum of absolute values.
- the result: u of itself."""
import math

import numpy as np
import torch

TD = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}
E24 = 2.0 ** -24


def draw(rng, shape, dtype, std=1.0):
    """Values that the tensors' type holds, as float64."""
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(TD[dtype]).double()


def offsets_of(lengths, first=0):
    return [first + sum(lengths[:i]) for i in range(len(lengths) + 1)]


def visible(T, offsets, prefix):
    """numpy bool [T, T]."""
    m = np.zeros((T, T), dtype=bool)
    for n in range(len(offsets) - 1):
        b, e = offsets[n], offsets[n + 1]
        p = min(prefix[n], e - b) if prefix else 0
        m[b:e, b:e] = np.tril(np.ones((e - b, e - b), dtype=bool))
        m[b:e, b:b + p] = True
    return m


def ranges_of(T, offsets, prefix):
    """What stage_op_doc_ranges leaves, from the mask."""
    m = visible(T, offsets, prefix)
    r = np.zeros((T, 4), dtype=np.int32)
    for t in range(T):
        if m[t].any():
            j, i = np.flatnonzero(m[t]), np.flatnonzero(m[:, t])
            assert len(j) == j[-1] - j[0] + 1 and len(i) == i[-1] - i[0] + 1
            r[t] = (j[0], j[-1] + 1, i[0], i[-1] + 1)
    return torch.from_numpy(r)


class Case:
    def __init__(self, T, nh, nkv, d, lengths, prefix=None, first=0, softcap=0.0, slopes=False, scale=None):
        self.T, self.nh, self.nkv, self.d, self.lengths, self.prefix, self.first = T, nh, nkv, d, lengths, prefix, first
        self.softcap, self.scale = softcap, float(np.float32(scale or 1 / math.sqrt(d)))
        self.slopes = [float(np.float32(2.0 ** (-8.0 * (h + 1) / nh))) for h in range(nh)] if slopes else None
        self.offsets = offsets_of(lengths, first)

    def __str__(self):
        docs = "+".join(map(str, self.lengths)) if len(self.lengths) < 9 else "%ddocs" % len(self.lengths)
        return "T%d_h%dof%d_d%d_%s%s%s%s%s" % (self.T, self.nkv, self.nh, self.d, docs, "_prefix" if self.prefix else "",
                                               "_from%d" % self.first if self.first else "", "_cap%g" % self.softcap if self.softcap else "",
                                               "_bias" if self.slopes else "")


def heads(x, n):
    """[T, n*d] -> [n, T, d]"""
    return x.reshape(x.shape[0], n, -1).transpose(0, 1)


def rows(x):
    return x.transpose(0, 1).reshape(x.shape[1], -1)


def scores(c, q, k):
    """float64 [nh, T, T]: the scores, their derivative to scale q.k, a bound on the kernel's error, and the mask."""
    g = c.nh // c.nkv
    Q, K = heads(q, c.nh), heads(k, c.nkv).repeat_interleave(g, 0)
    u = c.scale * Q @ K.transpose(1, 2)
    err = c.scale * (Q.abs() @ K.abs().transpose(1, 2)) * (c.d + 8) * E24
    s, ds = u, torch.ones_like(u)
    if c.softcap > 0:
        t = torch.tanh(u / c.softcap)
        s, ds = c.softcap * t, 1 - t * t
        err = err + 16 * c.softcap * E24
    if c.slopes:
        at = torch.arange(c.T, device=q.device).double()
        bias = torch.tensor(c.slopes, dtype=torch.float64, device=q.device)[:, None, None] * (at[:, None] - at[None, :]).abs()
        s = s - bias
        err = err + 4 * bias * E24
    return s, ds, err + 8 * (s.abs() + 8) * E24, torch.from_numpy(visible(c.T, c.offsets, c.prefix)).to(q.device)


def forward(c, q, k, v):
    """o [T, nh*d], lse [nh, T]."""
    s, _, _, m = scores(c, q, k)
    s = s.masked_fill(~m, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(m, torch.exp(s - torch.where(lse.isinf(), 0.0, lse)[..., None]), 0.0)
    return rows(p @ heads(v, c.nkv).repeat_interleave(c.nh // c.nkv, 0)), lse


def round_step(dtype):
    """Half a step of the type relative to a value, and half the smallest step there is."""
    return torch.finfo(TD[dtype]).eps / 2, {0: 2.0 ** -126, 1: 2.0 ** -126, 2: 2.0 ** -25}[dtype]


def forward_bounds(c, dtype, q, k, v):
    """How far o and lse may be off."""
    u, tiny = round_step(dtype)
    s, _, err, m = scores(c, q, k)
    p = torch.softmax(s.masked_fill(~m, -1e300), -1) * m
    V = heads(v, c.nkv).repeat_interleave(c.nh // c.nkv, 0)
    pv, n = p @ V.abs(), m.sum(1).double()
    e = (err * m).amax(-1) + (n + 8) * E24       # of a weight, relative; the row sum's too
    up = 0.0 if dtype == 0 else u
    ob = (2 * e[..., None] + up + (n[:, None] + 8) * E24) * pv + tiny * (m.double() @ V.abs())
    ob = ob + u * ((p @ V).abs() + ob) + tiny
    lse = torch.logsumexp(s.masked_fill(~m, -1e300), -1)
    return rows(ob), e + 4 * lse.abs() * E24 * (n > 0)


def backward(c, q, k, v, o, lse, dout):
    """dq, dk, dv from what the call gets."""
    return _backward(c, None, q, k, v, o, lse, dout)


def backward_bounds(c, dtype, q, k, v, o, lse, dout):
    return _backward(c, dtype, q, k, v, o, lse, dout)


def _backward(c, dtype, q, k, v, o, lse, dout):
    g = c.nh // c.nkv
    s, slope, err, m = scores(c, q, k)
    p = torch.where(m, torch.exp(s - torch.where(lse.isinf(), 0.0, lse)[..., None]), 0.0)
    Q, K, V = heads(q, c.nh), heads(k, c.nkv).repeat_interleave(g, 0), heads(v, c.nkv).repeat_interleave(g, 0)
    O, D = heads(o, c.nh), heads(dout, c.nh)
    dp, delta = D @ V.transpose(1, 2), (D * O).sum(-1, keepdim=True)
    shared = lambda x: rows(x.reshape(c.nkv, g, c.T, c.d).sum(1))
    ds = p * (dp - delta) * slope
    if dtype is None:
        return rows(ds @ K) * c.scale, shared(ds.transpose(1, 2) @ Q) * c.scale, shared(p.transpose(1, 2) @ D)
    u, tiny = round_step(dtype)
    up, t = 0.0 if dtype == 0 else u, tiny
    e = err + 8 * E24
    # of ds: the weight's error, that of dp - delta (sums of d products), that of the slope
    size = D.abs() @ V.abs().transpose(1, 2) + (D.abs() * O.abs()).sum(-1, keepdim=True)
    dds = ds.abs() * (e + 8 * E24) + p * slope * size * (c.d + 8) * E24 + p * (dp - delta).abs() * 8 * E24 * (c.softcap > 0) + 2.0 ** -126 * size
    n = float(max(c.lengths, default=0))
    sums = lambda terms, errs: errs + terms * (up + (n + 8) * E24)
    # in half, ds is rounded in steps that may be as coarse as 2^-25 of the largest magnitude that its rows' gradient has
    ds_t = t * D.abs().amax().clamp(min=1.0)
    bq = (sums(ds.abs() @ K.abs(), dds @ K.abs()) + ds_t * m.double() @ K.abs()) * c.scale
    mt = m.double().t()
    bk = (sums(ds.abs().transpose(1, 2) @ Q.abs(), dds.transpose(1, 2) @ Q.abs()) + ds_t * mt @ Q.abs()) * c.scale
    bv = sums(p.transpose(1, 2) @ D.abs(), (p * e).transpose(1, 2) @ D.abs()) + t * mt @ D.abs()
    dq, dk, dv = rows(ds @ K) * c.scale, shared(ds.transpose(1, 2) @ Q) * c.scale, shared(p.transpose(1, 2) @ D)
    bq, bk, bv = rows(bq), shared(bk) * 1.01, shared(bv) * 1.01
    last = lambda b, x: b + u * (x.abs() + b) + tiny
    return last(bq, dq), last(bk, dk), last(bv, dv)


def within(got, want, bound, what):
    """got may be off want by bound, element by element."""
    got, want = got.double().to(want.device), want.double()
    same = (got == want) | (got.isnan() & want.isnan())   # infinities
    off = torch.where(same, 0.0, (got - want).abs() / bound)
    assert not off.isnan().any() and off.max() <= 1.0, "%s: %.2f of its bound, at %s" % (what, off.nan_to_num(math.inf).max(), tuple(np.unravel_index(int(off.nan_to_num(math.inf).argmax()), off.shape)))
    return float(off.max())
