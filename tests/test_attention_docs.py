"""Attention inside packed documents (stage_op_doc_ranges, stage_op_attention_docs_fwd / _bwd) against the formulas in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import docs_reference as ref
import paper_2507_10392_amd as zs
from docs_reference import Case, TD

gpu = pytest.mark.gpu
CASES = [
    Case(1, 1, 1, 8, [1]),                                                  # one token
    Case(5, 2, 1, 16, [2, 0, 3], prefix=[1, 0, 9], softcap=2.0, slopes=True),   # an empty document, a prefix past its end
    Case(9, 3, 1, 24, []),                                                  # no document at all
    Case(64, 4, 4, 64, [64]),
    Case(65, 4, 2, 80, [33, 31], slopes=True),                              # a last token of no document
    Case(127, 2, 2, 128, [60, 1, 66], prefix=[7, 1, 0]),
    Case(130, 6, 2, 96, [1, 1, 1, 100, 20], prefix=[0, 1, 0, 64, 20], first=3),
    Case(257, 3, 3, 40, [31, 33, 128], first=5, softcap=5.0),
    Case(300, 4, 1, 128, [150, 140], prefix=[0, 70], softcap=30.0, slopes=True),
    Case(200, 8, 1, 64, [3] * 60),                                          # every tile holds many documents
    Case(385, 5, 5, 128, [384], slopes=True),
    Case(700, 8, 2, 128, [513, 187]),
    Case(777, 16, 4, 64, [777], prefix=[300], softcap=50.0),
    Case(640, 2, 1, 72, [129, 383, 128], slopes=True),
    Case(1100, 3, 1, 112, [1100], softcap=1.0, scale=0.5),                  # scores at the cap
]


def stream():
    return torch.cuda.current_stream().cuda_stream


def vec(dtype):
    return 4 if dtype == 0 else 8


class Run:
    """A case's buffers on the GPU: q, k, v columns of one buffer whose rows have spare columns, results in buffers of NaN."""

    def __init__(self, c, dtype, seed=0, std=1.0):
        self.c, self.dtype = c, dtype
        rng = np.random.default_rng(seed + 7 * c.T + c.d)
        T, Q, K = c.T, c.nh * c.d, c.nkv * c.d
        self.q, self.k, self.v = (ref.draw(rng, (T, n), dtype, std) for n in (Q, K, K))
        self.dout = ref.draw(rng, (T, Q), dtype, 0.5)
        dt, pad = TD[dtype], vec(dtype)
        self.qkv = torch.full((T, Q + 2 * K + pad), math.nan, dtype=dt, device="cuda")
        self.gq, self.gk, self.gv = self.qkv[:, :Q], self.qkv[:, Q:Q + K], self.qkv[:, Q + K:Q + 2 * K]
        for g, x in ((self.gq, self.q), (self.gk, self.k), (self.gv, self.v)):
            g.copy_(x.to(dt))
        self.gdout = torch.full((T, Q + pad), math.nan, dtype=dt, device="cuda")[:, :Q]
        self.gdout.copy_(self.dout.to(dt))
        self.go_all = torch.full((T, Q + pad), math.nan, dtype=dt, device="cuda")
        self.go = self.go_all[:, :Q]
        self.lse = torch.full((c.nh, T), math.nan, device="cuda")
        self.grads_all = torch.full((T, Q + 2 * K + pad), math.nan, dtype=dt, device="cuda")
        self.dq, self.dk, self.dv = self.grads_all[:, :Q], self.grads_all[:, Q:Q + K], self.grads_all[:, Q + K:Q + 2 * K]
        n = zs.attention_docs_bwd_scratch_bytes(dtype, T, c.nh, c.nkv, c.d)
        self.scratch = torch.full((n // 4,), math.nan, device="cuda")
        self.slopes = torch.tensor(c.slopes, device="cuda") if c.slopes else None
        self.offsets = torch.tensor(c.offsets, dtype=torch.int32, device="cuda")
        self.prefix = torch.tensor(c.prefix, dtype=torch.int32, device="cuda") if c.prefix else None
        self.ranges = torch.full((T, 4), -1, dtype=torch.int32, device="cuda")

    def find(self):
        zs.ops.doc_ranges(stream(), self.c.T, len(self.c.lengths), self.offsets, self.prefix, self.ranges)

    def fwd(self):
        c = self.c
        zs.ops.attention_docs_fwd(stream(), self.dtype, c.T, c.nh, c.nkv, c.d, self.gq, self.gq.stride(0), self.gk, self.gv, self.gk.stride(0),
                                  self.ranges, c.scale, c.softcap, self.slopes, self.go, self.go.stride(0), self.lse)

    def bwd(self):
        c = self.c
        zs.ops.attention_docs_bwd(stream(), self.dtype, c.T, c.nh, c.nkv, c.d, self.gq, self.gq.stride(0), self.gk, self.gv, self.gk.stride(0),
                                  self.ranges, c.scale, c.softcap, self.slopes, self.go, self.gdout, self.go.stride(0), self.lse, self.dq,
                                  self.dq.stride(0), self.dk, self.dv, self.dk.stride(0), self.scratch, 4 * self.scratch.numel())

    def all(self):
        self.find()
        self.fwd()
        self.bwd()
        torch.cuda.synchronize()
        return [x.clone() for x in (self.go, self.lse, self.dq, self.dk, self.dv)]

    def check(self, x=None):
        """Every result against 64 bits; x: the inputs where they are not the drawn ones."""
        c, (q, k, v, dout) = self.c, x or (self.q, self.k, self.v, self.dout)
        o, lse = ref.forward(c, q, k, v)
        bo, bl = ref.forward_bounds(c, self.dtype, q, k, v)
        ref.within(self.go, o, bo, "o")
        ref.within(self.lse, lse, bl, "lse")
        saved = (self.go.double().to(q.device), self.lse.double().to(q.device))
        want = ref.backward(c, q, k, v, *saved, dout)
        bounds = ref.backward_bounds(c, self.dtype, q, k, v, *saved, dout)
        for name, got, w, b in zip(("dq", "dk", "dv"), (self.dq, self.dk, self.dv), want, bounds):
            ref.within(got, w, b, name)


def say(*what):
    print("[case]", *what, flush=True)


@gpu
@pytest.mark.parametrize("c", CASES, ids=str)
def test_ranges(gpu_device, c):
    r = Run(c, 1)
    r.find()
    assert torch.equal(r.ranges.cpu(), ref.ranges_of(c.T, c.offsets, c.prefix))


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("c", CASES, ids=str)
def test_forward_and_gradients_match_64_bits(gpu_device, c, dtype):
    say(c, dtype)
    r = Run(c, dtype)
    first = r.all()
    r.check()
    for x in (r.go_all, r.grads_all):                 # nothing outside the heads' columns
        assert x[:, -vec(dtype):].isnan().all()
    again = r.all()
    for a, b in zip(first, again):                    # and the same bits from a second call
        assert torch.equal(a, b)


DOCS = [200, 1, 350, 64, 30, 410]   # 1055 tokens
LARGE = [Case(500, 32, 8, 128, [100, 300, 90], slopes=True), Case(500, 32, 32, 64, [480], prefix=[70], softcap=20.0),     # 512 groups of 32 rows
         Case(1000, 32, 8, 80, DOCS[:4] + [300]), Case(1000, 32, 16, 128, [1000], softcap=10.0, slopes=True),             # 1024
         Case(1100, 64, 16, 128, DOCS, prefix=[50, 1, 0, 64, 0, 100], softcap=30.0), Case(1100, 64, 64, 128, DOCS, first=17),   # 2240
         Case(1100, 64, 32, 64, [1090], slopes=True), Case(1100, 64, 64, 96, DOCS, prefix=[0, 0, 350, 0, 0, 0], softcap=30.0, slopes=True),
         Case(1500, 64, 1, 128, [700, 33, 600]),                                                                          # one key head, its query heads in parts
         Case(900, 132, 132, 128, [333, 66, 500], softcap=25.0), Case(2050, 64, 64, 64, [40] * 50, slopes=True),   # 1056 and 1088 blocks of 128 keys
         Case(9000, 8, 1, 64, [60, 3000, 900] + [500] * 10), Case(9001, 8, 8, 128, [2900] + [100] * 61)]                   # more than 256 blocks of rows


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("c", LARGE, ids=str)
def test_larger_launches_match_64_bits(gpu_device, c, dtype):
    """Launches of hundreds and thousands of groups of rows; the 64-bit side on the GPU, head by head."""
    say(c, dtype)
    r = Run(c, dtype)
    first = r.all()
    group = c.nh // c.nkv
    for kv in sorted({0, c.nkv // 2, c.nkv - 1}):        # three key heads with their query heads
        h = slice(kv * group, (kv + 1) * group)
        part = Case(c.T, group, 1, c.d, c.lengths, c.prefix, c.first, c.softcap, scale=c.scale)
        part.slopes = c.slopes[h] if c.slopes else None
        cols, key = slice(h.start * c.d, h.stop * c.d), slice(kv * c.d, (kv + 1) * c.d)
        q, k, v, dout = r.q[:, cols].cuda(), r.k[:, key].cuda(), r.v[:, key].cuda(), r.dout[:, cols].cuda()
        for rows in chunks(part):
            check_part(part, dtype, rows, q, k, v, dout, r.go[:, cols], r.lse[h], r.dq[:, cols], r.dk[:, key], r.dv[:, key])
    for a, b in zip(first, r.all()):
        assert torch.equal(a, b)


def chunks(c):
    """Runs of whole documents of up to 3000 tokens: (first token, end, lengths, prefix)."""
    runs, at = [], c.first
    for n, length in enumerate(c.lengths):
        p = c.prefix[n] if c.prefix else 0
        if not runs or runs[-1][1] - runs[-1][0] + length > 3000:
            runs.append([at, at, [], []])
        runs[-1][1] += length
        runs[-1][2].append(length)
        runs[-1][3].append(p)
        at += length
    return runs


def check_part(c, dtype, run, q, k, v, dout, o, lse, dq, dk, dv):
    first, end, lengths, prefix = run
    t = slice(first, end)
    part = Case(end - first, c.nh, 1, c.d, lengths, prefix, 0, c.softcap, scale=c.scale)
    part.slopes = c.slopes
    x = (q[t], k[t], v[t])
    want, wl = ref.forward(part, *x)
    bo, bl = ref.forward_bounds(part, dtype, *x)
    ref.within(o[t], want, bo, "o")
    ref.within(lse[:, t], wl, bl, "lse")
    saved = (o[t].double(), lse[:, t].double())
    want = ref.backward(part, *x, *saved, dout[t])
    for name, got, w, b in zip(("dq", "dk", "dv"), (dq[t], dk[t], dv[t]), want, ref.backward_bounds(part, dtype, *x, *saved, dout[t])):
        ref.within(got, w, b, name)


@gpu
@pytest.mark.parametrize("dtype", [1, 2])
def test_many_tiles(gpu_device, dtype):
    """Rows with thousands of keys, several blocks of rows and of keys."""
    c = Case(2600, 2, 1, 128, [100, 2300], prefix=[0, 500])
    say(c, dtype)
    r = Run(c, dtype)
    r.all()
    r.check()


def with_values(r, t, value, names):
    """Puts value into token t's q, k, v or dout, on both sides; the inputs in 64 bits."""
    x = {n: getattr(r, n).clone() for n in ("q", "k", "v", "dout")}
    for n in names:
        x[n][t] = value
        getattr(r, "g" + n)[t] = value
    return [x[n] for n in ("q", "k", "v", "dout")]


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("d", [64, 128])
def test_what_padding_holds_reaches_nothing(gpu_device, dtype, d):
    c = Case(200, 4, 2, d, [90, 85], first=5)
    say(c, dtype)
    r = Run(c, dtype)
    clean = r.all()
    for value in (math.nan, math.inf, -torch.finfo(TD[dtype]).max):
        for t in (0, 4, 180, 199):
            with_values(r, t, value, ("q", "k", "v", "dout"))
        got = r.all()
        for a, b in zip(clean, got):
            assert torch.equal(a, b), value


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("name", ["k", "v", "q", "dout"])
def test_non_finite_values_stay_in_their_document(gpu_device, dtype, value, name):
    """Token 60 of a document 40 .. 139 holds inf or NaN.  Rows that do not see it, and keys that it does not see, get what they get without it."""
    c = Case(200, 2, 1, 64, [40, 100, 60], softcap=20.0)
    say(c, dtype, value, name)
    r = Run(c, dtype)
    clean = [x.double().cpu() for x in r.all()]
    with_values(r, 60, value, (name,))
    o, lse, dq, dk, dv = [x.double().cpu() for x in r.all()]
    hidden = torch.arange(200)
    rows = (hidden < 60) | (hidden >= 140)                # rows that do not see token 60
    if name in ("q", "dout"):
        rows = hidden != 60                               # only its own row takes part in the forward
    want, wl = ref.forward(c, r.q, r.k, r.v)
    bo, bl = ref.forward_bounds(c, dtype, r.q, r.k, r.v)
    ref.within(o[rows], want[rows], bo[rows], "o")
    ref.within(lse[:, rows], wl[:, rows], bl[:, rows], "lse")
    # the gradients' formulas with what this run saved: a row that was computed again may have an o that rounds otherwise
    saved = (torch.where(rows[:, None], o, clean[0]), torch.where(rows, lse, clean[1]))
    want, bounds = (f(*x, r.q, r.k, r.v, *saved, r.dout) for f, x in ((ref.backward, (c,)), (ref.backward_bounds, (c, dtype))))
    ref.within(dq[rows], want[0][rows], bounds[0][rows], "dq")
    # keys whose rows are all fine: after a bad key or value, those of the rows that see it are not
    keys = (hidden < 40) | (hidden >= 140)
    if name in ("q", "dout"):
        keys = (hidden < 40) | (hidden > 60)
    ref.within(dk[keys], want[1][keys], bounds[1][keys], "dk")
    ref.within(dv[keys], want[2][keys], bounds[2][keys], "dv")
    if math.isnan(value):                                 # and what it reaches is not hidden
        bad = {"k": o, "v": o, "q": o, "dout": dv}[name]
        assert bad[60].isnan().any() and (name not in ("k", "v") or bad[139].isnan().any())


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_large_scores(gpu_device, dtype):
    """Scores in the thousands: one key takes all the weight, the others none."""
    c = Case(150, 2, 2, 64, [150], scale=8.0)
    say(c, dtype)
    r = Run(c, dtype, std=4.0)
    r.all()
    r.check()


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_capped_gradients_of_small_weights(gpu_device, dtype):
    """Scores of a few times their usual size: most weights, and their score gradients, lie far below the largest, in half among its subnormal numbers,
    whose step a factor left out of the rounded value would coarsen."""
    c = Case(1138, 6, 3, 80, [339, 0, 0, 0, 167, 615, 0, 1, 16], softcap=50.0)
    say(c, dtype)
    r = Run(c, dtype, seed=66, std=2.0)
    r.all()
    r.check()


@gpu
@pytest.mark.parametrize("dtype,softcap", [(0, 1e6), (0, 1024.0), (1, 1024.0), (2, 1024.0)])
def test_caps_far_above_the_scores(gpu_device, dtype, softcap):
    """Such a cap changes nothing that the type shows.  Scores of up to about 5 differ from uncapped ones by s^3 / (3 softcap^2) < 2^-14, and are off by
    up to 2^-22 softcap = 2^-12 in 16 bits (fp32: 2^-21 of themselves): weights by twice that, relative, and so o, against the largest |v|; then the
    roundings of P and o."""
    say(dtype, softcap)
    c = Case(200, 4, 2, 64, [150, 50], softcap=softcap)
    r = Run(c, dtype)
    r.all()
    plain = Case(200, 4, 2, 64, [150, 50])
    u = ref.scores(plain, r.q, r.k)[0].abs().max()
    assert u < 6, u
    o, lse = ref.forward(plain, r.q, r.k, r.v)
    off = float(u) ** 3 / (3 * softcap ** 2) + (2.0 ** -21 * 6 if dtype == 0 else 2.0 ** -22 * softcap) + 72 * 2.0 ** -24 * 64
    half = torch.finfo(ref.TD[dtype]).eps / 2
    assert (r.lse.double().cpu() - lse).abs().max() <= off + 2.0 ** -16   # the sum: 158 x 2^-24
    assert (r.go.double().cpu() - o).abs().max() <= (2 * off + (2 if dtype else 1) * half + 2.0 ** -16) * r.v.abs().max()


@gpu
def test_rows_that_are_far_apart(gpu_device):
    """Rows whose byte offsets pass 32 bits."""
    T, ld = 600, 1 << 22
    c = Case(T, 1, 1, 64, [300, 300])
    r = Run(c, 1)
    want = r.all()
    buf = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")        # 5 GB
    wide = [torch.as_strided(buf, (T, 64), (ld, 1), 1024 * i) for i in range(8)]
    for w, x in zip(wide, (r.gq, r.gk, r.gv, r.gdout)):
        w.copy_(x)
    r.gq, r.gk, r.gv, r.gdout, r.go, r.dq, r.dk, r.dv = wide
    for a, b in zip(want, r.all()):
        assert torch.equal(a, b)


@gpu
def test_side_stream_and_graph(gpu_device):
    """All three calls captured together, replayed on new inputs with eager work in between."""
    c = Case(333, 4, 2, 128, [200, 100], prefix=[50, 0], softcap=30.0)
    r = Run(c, 1)
    other = Run(c, 1, seed=5)
    want = other.all()
    r.all()
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        r.find()
        r.fwd()
        r.bwd()
    for _ in range(3):
        r.qkv.copy_(other.qkv)
        r.gdout.copy_(other.gdout)
        for x in (r.go, r.lse, r.dq, r.dk, r.dv):
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (r.go, r.lse, r.dq, r.dk, r.dv)):
            assert torch.equal(a, b)
        other.all()


@gpu
def test_two_streams(gpu_device):
    """Calls that run side by side, each with a scratch of its own."""
    c = Case(500, 16, 4, 64, [300, 150], slopes=True)
    runs = [Run(c, 2, seed=s) for s in (1, 2)]
    want = [r.all() for r in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(5):
        for r in runs:
            for x in (r.go, r.lse, r.dq, r.dk, r.dv):
                x.zero_()
        torch.cuda.synchronize()
        for r, s in zip(runs, streams):
            with torch.cuda.stream(s):
                r.fwd()
                r.bwd()
        torch.cuda.synchronize()
        for r, w in zip(runs, want):
            for a, b in zip(w, (r.go, r.lse, r.dq, r.dk, r.dv)):
                assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_every_length_around_the_blocks(gpu_device, dtype):
    """One document of every length up to 70, and around 128, alone and behind another one."""
    for n in list(range(1, 71)) + [95, 96, 97, 127, 128, 129, 130]:
        for c in (Case(n, 2, 1, 32, [n]), Case(n + 33, 1, 1, 32, [n, 33], prefix=[n // 2, 5], softcap=8.0)):
            r = Run(c, dtype)
            r.all()
            r.check()


@gpu
def test_gradients_against_differences(gpu_device):
    """sum(o * w) of the fp32 forward, differenced along random directions."""
    c = Case(24, 2, 1, 16, [10, 12], prefix=[4, 0], softcap=3.0, slopes=True)
    r = Run(c, 0)
    r.all()
    w = r.gdout.double()
    rng = np.random.default_rng(3)
    for name, grad in (("gq", r.dq), ("gk", r.dk), ("gv", r.dv)):
        x = getattr(r, name)
        base, d = x.clone(), torch.from_numpy(rng.standard_normal(tuple(x.shape)).astype(np.float32)).cuda()
        h, loss = 2.0 ** -7, []
        for s in (h, -h):
            x.copy_(base + s * d)
            r.fwd()
            torch.cuda.synchronize()
            loss.append(float((r.go.double() * w).sum()))
        x.copy_(base)
        want = float((grad.double() * d.double()).sum())
        # the difference's own error: h^2 / 6 times a third derivative of order 10, and fp32 rounding of 400 outputs over 2 h
        assert abs((loss[0] - loss[1]) / (2 * h) - want) <= 2e-3 * (1 + abs(want)), name


@gpu
def test_documents_of_wrong_offsets_stay_inside(gpu_device):
    """Offsets that the interface does not allow: the table's ranges stay inside [0, T]."""
    T = 300
    for offsets, prefix in (([-5, 900, 20, 301], [4, -3, 999]), ([200, 100, 0], [2**31 - 1, 5]), ([-2**31, 2**31 - 1], None)):
        o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        p = torch.tensor(prefix, dtype=torch.int32, device="cuda") if prefix else None
        r = torch.full((T, 4), -1, dtype=torch.int32, device="cuda")
        zs.ops.doc_ranges(stream(), T, len(offsets) - 1, o, p, r)
        r = r.cpu()
        assert (r >= 0).all() and (r <= T).all() and (r[:, 0] <= r[:, 1]).all() and (r[:, 2] <= r[:, 3]).all()


@gpu
def test_more_documents_than_two_numbers_of_them_add_up_to(gpu_device):
    """2^30 + 4 empty documents before the one that has the tokens: the sum of two documents' numbers passes 31 bits."""
    n, T = (1 << 30) + 5, 5
    o = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    o[n] = T
    r = torch.full((T, 4), -1, dtype=torch.int32, device="cuda")
    zs.ops.doc_ranges(stream(), T, n, o, None, r)
    assert r.cpu().tolist() == [[0, t + 1, t, T] for t in range(T)]


# ---------------------------------------------------------------------------------------------- no GPU
GOOD = dict(dtype=1, T=16, nh=4, nkv=2, d=64, q=4096, ldq=256, k=4096, v=4096, ldkv=128, ranges=4096, scale=0.125, softcap=0.0, slopes=None,
            o=4096, ldo=256, lse=4096)
BAD = [dict(dtype=3), dict(dtype=-1), dict(T=-1), dict(nh=0), dict(nkv=0), dict(nh=5), dict(d=0), dict(d=60), dict(d=136), dict(q=None), dict(k=None),
       dict(v=None), dict(ranges=None), dict(ranges=4100), dict(o=None), dict(lse=None), dict(lse=4098), dict(q=4104), dict(k=4098), dict(v=4104),
       dict(o=4104), dict(ldq=255), dict(ldq=248), dict(ldq=260), dict(ldkv=120), dict(ldkv=132), dict(ldo=248), dict(ldo=(1 << 22) + 8),
       dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(softcap=-1.0), dict(softcap=math.nan),
       dict(softcap=math.inf), dict(softcap=1025.0), dict(dtype=2, softcap=2048.0), dict(softcap=1e-31), dict(softcap=1e31), dict(scale=1e31), dict(scale=1e10, softcap=1e-25),
       dict(slopes=4097), dict(T=1 << 29), dict(T=(1 << 30) + 1, nh=1, nkv=1),
       dict(T=(1 << 28) + 1)]


def fwd_code(a):
    return zs.lib().stage_op_attention_docs_fwd(None, a["dtype"], a["T"], a["nh"], a["nkv"], a["d"], a["q"], a["ldq"], a["k"], a["v"], a["ldkv"],
                                                a["ranges"], a["scale"], a["softcap"], a["slopes"], a["o"], a["ldo"], a["lse"])


def bwd_code(a, **more):
    b = dict(dict(dout=4096, dq=4096, lddq=256, dk=4096, dv=4096, lddkv=128, scratch=4096, bytes=1 << 40), **more)
    return zs.lib().stage_op_attention_docs_bwd(None, a["dtype"], a["T"], a["nh"], a["nkv"], a["d"], a["q"], a["ldq"], a["k"], a["v"], a["ldkv"],
                                                a["ranges"], a["scale"], a["softcap"], a["slopes"], a["o"], b["dout"], a["ldo"], a["lse"], b["dq"],
                                                b["lddq"], b["dk"], b["dv"], b["lddkv"], b["scratch"], b["bytes"])


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_refusals(bad):
    assert fwd_code(dict(GOOD, **bad)) == zs.STAGE_ERR_ARG
    assert bwd_code(dict(GOOD, **bad)) == zs.STAGE_ERR_ARG


@pytest.mark.parametrize("bad", [dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dq=4104), dict(dk=4104), dict(dv=4104),
                                 dict(dout=4104), dict(lddq=248), dict(lddkv=120), dict(lddkv=132)], ids=str)
def test_refusals_of_the_backward(bad):
    assert bwd_code(GOOD, **bad) == zs.STAGE_ERR_ARG


def test_scratch_of_the_backward():
    n = zs.attention_docs_bwd_scratch_bytes(1, 16, 4, 2, 64)
    assert n >= 16 * 4 * 4
    for bad in (dict(scratch=None), dict(scratch=4096 + 128), dict(bytes=n - 1), dict(bytes=0)):
        assert bwd_code(GOOD, **bad) == zs.STAGE_ERR_WORKSPACE
    for shape in ((3, 16, 4, 2, 64), (1, -1, 4, 2, 64), (1, 16, 4, 3, 64), (1, 16, 4, 2, 60), (1, 16, 4, 2, 136), (1, 16, 0, 0, 64)):
        with pytest.raises(zs.StageError):
            zs.attention_docs_bwd_scratch_bytes(*shape)


def test_no_tokens():
    assert fwd_code(dict(GOOD, T=0)) == zs.STAGE_OK and bwd_code(dict(GOOD, T=0)) == zs.STAGE_OK
    assert zs.lib().stage_op_doc_ranges(None, 0, 1, 4096, None, 4096) == zs.STAGE_OK
    empty = dict(GOOD, T=0, q=None, k=None, v=None, o=None, lse=None, ranges=None)   # an empty tensor's address
    assert fwd_code(empty) == zs.STAGE_OK and bwd_code(empty, dout=None, dq=None, dk=None, dv=None, scratch=None, bytes=0) == zs.STAGE_OK
    assert zs.lib().stage_op_doc_ranges(None, 0, 0, None, None, None) == zs.STAGE_OK
    assert fwd_code(dict(GOOD, T=0, nh=5)) == zs.STAGE_ERR_ARG


@pytest.mark.parametrize("args", [(-1, 1, 4096, None, 4096), (8, -1, 4096, None, 4096), (8, 1, None, None, 4096), (8, 1, 4096, None, None),
                                  (8, 1, 4096, None, 4104), ((1 << 30) + 1, 1, 4096, None, 4096), (8, 1, 4097, None, 4096), (8, 1, 4096, 4097, 4096)], ids=str)
def test_refusals_of_ranges(args):
    assert zs.lib().stage_op_doc_ranges(None, *args) == zs.STAGE_ERR_ARG
