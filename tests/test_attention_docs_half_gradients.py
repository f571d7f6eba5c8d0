"""Half gradients inside packed documents where dout differs in size: between documents, along a document, between the query heads of a key head, and far
below 1.  Score gradients go into their second product as halves, in units that follow dout; what a unit may follow is what the bounds here say:
dq_i the largest |dout| of row i, dk_j the largest of the rows that see key j.  Half a step, 2^-25 of that, is the most that a score gradient is off by."""
import numpy as np
import pytest
import torch

import docs_reference as ref
from docs_reference import Case, E24
from test_attention_docs import Run, say

gpu = pytest.mark.gpu
HALF = 2
DOCS = [17, 300, 1, 190]
# each launch of the backward: both kernels in one, eight waves on 64 keys, four on 64, four on 128
SHAPES = [(2, 1, 128), (4, 4, 64), (32, 8, 64), (32, 4, 128), (80, 80, 64), (205, 205, 72)]


def bounds(c, q, k, v, o, lse, dout):
    """dq, dk (float64) and how far they may be off, of one key head and its query heads: the terms of docs_reference, with the step of a score gradient as
    above."""
    s, slope, err, m = ref.scores(c, q, k)
    m = m.double()
    p = torch.where(m > 0, torch.exp(s - torch.where(lse.isinf(), 0.0, lse)[..., None]), 0.0)
    Q, K, V, O, D = ref.heads(q, c.nh), ref.heads(k, 1), ref.heads(v, 1), ref.heads(o, c.nh), ref.heads(dout, c.nh)
    dp, delta = D @ V.transpose(1, 2), (D * O).sum(-1, keepdim=True)
    ds = p * (dp - delta) * slope
    u, tiny = ref.round_step(HALF)
    size = D.abs() @ V.abs().transpose(1, 2) + (D.abs() * O.abs()).sum(-1, keepdim=True)
    off = ds.abs() * (err + 16 * E24) + p * slope * size * (c.d + 8) * E24 + p * (dp - delta).abs() * 8 * E24 * (c.softcap > 0) + 2.0 ** -126 * size
    off = off + ds.abs() * (u + (max(c.lengths) + 8) * E24)
    row = D.abs().amax(-1)                                        # [nh, T]
    key = (m[None] * row[..., None]).amax((0, 1))                 # [T]
    dq, bq = ds @ K * c.scale, (off + 2.0 ** -25 * row[..., None] * m) @ K.abs() * c.scale
    dk = (ds.transpose(1, 2) @ Q).sum(0) * c.scale
    bk = ((off + 2.0 ** -25 * key * m).transpose(1, 2) @ Q.abs()).sum(0) * c.scale * 1.01
    last = lambda b, x: b + u * (x.abs() + b) + tiny
    return ref.rows(dq), last(ref.rows(bq), ref.rows(dq)), dk, last(bk, dk)


def sizes(kind, c):
    """A power of two for dout's [T, nh]."""
    e = torch.zeros(c.T, c.nh)
    at = 0
    for n, length in enumerate(c.lengths):
        rows = slice(at, at + length)
        at += length
        if kind == "documents":
            e[rows] = [10.0, -10.0, 8.0, -8.0][n]
        elif kind == "rising":
            e[rows] = torch.linspace(-10, 8, length).round()[:, None]
        elif kind == "falling":
            e[rows] = torch.linspace(8, -10, length).round()[:, None]
    if kind == "small":
        e[:] = -13.0
    if kind == "heads":
        e[:] = torch.tensor([-8.0, 4.0, -2.0, 7.0])[torch.arange(c.nh) % 4]
    x = 2.0 ** e
    if kind == "zeros":
        x[5:40] = 0
        x[100:200] = 0
        x[sum(DOCS[:3]):sum(DOCS[:3]) + 30] = 0
    return x


@gpu
@pytest.mark.parametrize("wide", ["q", "k"])
@pytest.mark.parametrize("kind", ["documents", "rising", "falling", "small", "heads", "zeros"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_sizes_of_dout(gpu_device, shape, kind, wide):
    """wide: q (which dk is made of) or k (dq) is 16 times its size and the other a 16th, so that the results stay above half's subnormal numbers."""
    nh, nkv, d = shape
    c = Case(sum(DOCS) + 12, nh, nkv, d, DOCS, softcap=20.0 if nkv == 8 else 0.0, slopes=nkv == 4)
    say(c, kind, wide)
    r = Run(c, HALF)
    for name, f in (("q", 16.0 if wide == "q" else 1 / 16), ("k", 16.0 if wide == "k" else 1 / 16)):
        x = (getattr(r, name) * f).half()
        setattr(r, name, x.double())
        getattr(r, "g" + name).copy_(x)
    x = (r.dout.reshape(c.T, nh, d) * sizes(kind, c)[..., None]).reshape(c.T, -1).half()
    r.dout = x.double()
    r.gdout.copy_(x)
    first = r.all()
    group = nh // nkv
    for kv in sorted({0, nkv // 2, nkv - 1}):
        part = Case(c.T, group, 1, d, c.lengths, softcap=c.softcap, scale=c.scale)
        part.slopes = c.slopes[kv * group:(kv + 1) * group] if c.slopes else None
        cols, key = slice(kv * group * d, (kv + 1) * group * d), slice(kv * d, (kv + 1) * d)
        dq, bq, dk, bk = bounds(part, r.q[:, cols].cuda(), r.k[:, key].cuda(), r.v[:, key].cuda(), r.go[:, cols].double(),
                                r.lse[kv * group:(kv + 1) * group].double(), r.dout[:, cols].cuda())
        ref.within(r.dq[:, cols], dq, bq, "dq")
        ref.within(r.dk[:, key], dk, bk, "dk")
    for a, b in zip(first, r.all()):
        assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_a_document_does_not_change_with_its_neighbours_dout(gpu_device, shape):
    """The second document's gradients with small and with large dout in the documents around it: the same bits."""
    nh, nkv, d = shape
    c = Case(sum(DOCS) + 12, nh, nkv, d, DOCS)
    say(c)
    r = Run(c, HALF)
    rows = slice(DOCS[0], DOCS[0] + DOCS[1])
    got = []
    for factor in (2.0 ** -6, 2.0 ** 15):
        x = r.dout * factor
        x[rows] = r.dout[rows] * 2.0 ** -6
        r.gdout.copy_(x.clamp(-60000, 60000).half())
        r.all()
        got.append([g[rows].clone() for g in (r.dq, r.dk, r.dv)])
    for a, b in zip(*got):
        assert torch.equal(a, b)
