"""inf and NaN inside packed documents on every launch of the attention: what does not see them, and what is not seen by what sees them, gets what the formulas
give without them.  Their blocks' rows and keys are computed again row by row, with the launch's own numbering of rows, heads and parts."""
import math

import numpy as np
import pytest
import torch

import docs_reference as ref
from docs_reference import Case, TD
from test_attention_docs import Run, say, check_part

gpu = pytest.mark.gpu
DOCS = [200, 1, 350, 64, 30, 410]
# Forward: four waves on 32 rows, eight on 64 (two heads; one), eight on 128 (four heads; two), four on 128 (four, two, one), more blocks than are ordered.
# Backward: both in one launch, eight waves on 64 keys (whole, in parts), four on 64, four on 128.
CASES = [Case(300, 8, 2, 128, [70, 50, 160], slopes=True), Case(500, 32, 8, 128, [100, 300, 90], slopes=True), Case(500, 32, 32, 64, [100, 310, 80], softcap=20.0),
         Case(1000, 32, 8, 80, DOCS[:4] + [300]), Case(1000, 32, 16, 128, [300, 77, 600], softcap=10.0, slopes=True),
         Case(1100, 64, 16, 128, DOCS, prefix=[50, 1, 0, 64, 0, 100], softcap=30.0), Case(1100, 64, 32, 64, DOCS, slopes=True),
         Case(1100, 64, 64, 96, DOCS, first=17), Case(1500, 64, 1, 128, [700, 33, 600]), Case(900, 132, 132, 128, [333, 66, 400], softcap=25.0),
         Case(9000, 8, 1, 64, [60, 3000, 900] + [500] * 10)]


def key_heads(c):
    return sorted({0, c.nkv // 2, c.nkv - 1})


def one_head(c, kv):
    """The case of a key head and its query heads, their columns in q and in k, and the heads."""
    group = c.nh // c.nkv
    h = slice(kv * group, (kv + 1) * group)
    part = Case(c.T, group, 1, c.d, c.lengths, c.prefix, c.first, c.softcap, scale=c.scale)
    part.slopes = c.slopes[h] if c.slopes else None
    return part, slice(h.start * c.d, h.stop * c.d), slice(kv * c.d, (kv + 1) * c.d), h


def check_documents(r, clean, bad, t, name):
    """The documents beside the one with the bad token t, as they are, and the rows and keys of its own that have nothing to do with it."""
    c = r.c
    n = max(i for i, b in enumerate(c.offsets[:-1]) if b <= t)
    pre = c.prefix or [0] * len(c.lengths)
    for kv in key_heads(c):
        part, cols, key, h = one_head(c, kv)
        q, k, v, dout = r.q[:, cols].cuda(), r.k[:, key].cuda(), r.v[:, key].cuda(), r.dout[:, cols].cuda()
        o, lse, dq, dk, dv = bad[0][:, cols], bad[1][h], bad[2][:, cols], bad[3][:, key], bad[4][:, key]
        for i in (n - 1, n + 1):
            run = (c.offsets[i], c.offsets[i + 1], c.lengths[i:i + 1], pre[i:i + 1])
            check_part(part, r.dtype, run, q, k, v, dout, o, lse, dq, dk, dv)
        s, length, at = slice(c.offsets[n], c.offsets[n + 1]), c.lengths[n], t - c.offsets[n]
        own = Case(length, part.nh, 1, c.d, [length], [pre[n]], 0, c.softcap, scale=c.scale)
        own.slopes = part.slopes
        x = (q[s], k[s], v[s])
        m = torch.from_numpy(ref.visible(length, own.offsets, own.prefix)).cuda()
        rows = torch.zeros(length, dtype=torch.bool, device="cuda")   # rows whose scores, result or gradient the bad token enters
        if name in ("k", "v"):
            rows = m[:, at].clone()
        else:
            rows[at] = True
        ok, keys = ~rows, ~(m & rows[:, None]).any(0)
        fwd = ok if name != "dout" else torch.ones_like(ok)
        want, wl = ref.forward(own, *x)
        bo, bl = ref.forward_bounds(own, r.dtype, *x)
        ref.within(o[s][fwd], want[fwd], bo[fwd], "o")
        ref.within(lse[:, s][:, fwd], wl[:, fwd], bl[:, fwd], "lse")
        saved = (torch.where(fwd[:, None], o[s], clean[0][s, cols]).double(), torch.where(fwd, lse[:, s], clean[1][h, s]).double())
        want, bounds = ref.backward(own, *x, *saved, dout[s]), ref.backward_bounds(own, r.dtype, *x, *saved, dout[s])
        for got, w, b, which, what in ((dq, want[0], bounds[0], ok, "dq"), (dk, want[1], bounds[1], keys, "dk"), (dv, want[2], bounds[2], keys, "dv")):
            if which.any():
                ref.within(got[s][which], w[which], b[which], what)


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("c", CASES, ids=str)
def test_non_finite_values_on_every_launch(gpu_device, c, dtype):
    r = Run(c, dtype)
    clean = r.all()
    n = 2 if len(c.lengths) > 3 else 1
    for t in (c.offsets[n] + 3, c.offsets[n + 1] - 2):         # near the document's begin, among its neighbour's rows and keys, and near its end
        for name in ("q", "k", "v", "dout"):
            g = getattr(r, "g" + name)
            held = g[t].clone()
            for value in (math.inf, math.nan):
                say(c, dtype, t, name, value)
                g[t] = value
                bad = r.all()
                check_documents(r, clean, bad, t, name)
                if math.isnan(value):                          # what it reaches is not hidden
                    assert (bad[4] if name == "dout" else bad[0])[t].isnan().all()
            g[t] = held
    for a, b in zip(clean, r.all()):
        assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("c", CASES, ids=str)
def test_padding_on_every_launch(gpu_device, c, dtype):
    """Tokens of no document hold NaN or inf: the same bits."""
    say(c, dtype)
    r = Run(c, dtype)
    clean = r.all()
    t = np.ones(c.T, dtype=bool)
    t[c.first:c.offsets[-1]] = False
    t = torch.from_numpy(t).cuda()
    for value in (math.nan, math.inf, -torch.finfo(TD[dtype]).max):
        for g in (r.gq, r.gk, r.gv, r.gdout):
            g[t] = value
        for a, b in zip(clean, r.all()):
            assert torch.equal(a, b), value


@gpu
@pytest.mark.parametrize("dtype", [1, 2])
def test_nan_throughout_does_not_take_long(gpu_device, dtype):
    """A step that has overflowed: every row is NaN, and no row's walk goes on once it is.  Walks to their ends take 200 times a finite call's time, as they are 5 to 9."""
    c = Case(4096, 32, 8, 128, [4096])
    r = Run(c, dtype)

    def took(f):
        ms = []
        for _ in range(3):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            f()
            b.record()
            torch.cuda.synchronize()
            ms.append(a.elapsed_time(b))
        return min(ms)

    r.all()
    fwd, bwd = took(r.fwd), took(r.bwd)
    r.gdout.fill_(math.nan)
    say(c, dtype, "dout")
    assert took(r.bwd) < 40 * bwd
    assert all(x.isnan().all() for x in (r.dq, r.dk, r.dv))
    r.gq.fill_(math.nan)
    say(c, dtype, "q")
    assert took(r.fwd) < 40 * fwd
    assert r.go.isnan().all() and r.lse.isnan().all()
    assert took(r.bwd) < 40 * bwd
