"""The gated delta rule inside packed documents against its definition in 64 bits (delta_reference.py), forward, backward and for single tokens."""
import math

import numpy as np
import pytest
import torch

import paper_2507_10392_amd as zs
from delta_reference import TD, Case, check, reference, reference_of, rule

gpu = pytest.mark.gpu


def say(*a):
    print("[case]", *a, flush=True)


def stream():
    return torch.cuda.current_stream().cuda_stream


def rows(x, dtype, pad=0, lead=0):
    """[T, heads, d] as rows on the GPU with `pad` elements of NaN behind each, `lead` before."""
    T = x.shape[0]
    w = x.reshape(T, -1).to(TD[dtype]).cuda()
    buf = torch.full((T, lead + w.shape[1] + pad), math.nan, dtype=TD[dtype], device="cuda")
    buf[:, lead:lead + w.shape[1]] = w
    return buf[:, lead:lead + w.shape[1]]


class Run:
    """A program's buffers; results and scratch hold NaN before the calls."""

    def __init__(self, c, dtype, x, packed=False, pad=0):
        self.c, self.dtype = c, dtype
        n, f = len(c.lengths), lambda t: None if t is None else t.float().cuda()
        hidden = torch.ones(c.T, dtype=torch.bool)
        hidden[c.offsets[0]:c.offsets[-1]] = False   # rows of no document
        y = {k: (v.clone() if v is not None else None) for k, v in x.items()}
        for k in ("q", "k", "v", "g", "beta", "dout"):
            y[k][hidden] = math.nan
        if packed:
            qkv = torch.cat([y[k].reshape(c.T, -1) for k in "qkv"], 1).to(TD[dtype]).cuda()
            a, b = c.nk * c.dk, 2 * c.nk * c.dk
            self.q, self.k, self.v = qkv[:, :a], qkv[:, a:b], qkv[:, b:]
        else:
            self.q, self.k, self.v = (rows(y[k], dtype, pad) for k in "qkv")
        self.dout = rows(y["dout"], dtype, pad)
        self.g, self.beta, self.h0, self.dht = f(y["g"]), f(y["beta"]), f(y["h0"]), f(y["dht"])
        self.offsets = torch.tensor(c.offsets, dtype=torch.int32, device="cuda")
        self.chunks = torch.full((zs.delta_chunks_ints(c.T, n),), -7, dtype=torch.int32, device="cuda")
        new = lambda *s, dt=torch.float32: torch.full(s, math.nan, dtype=dt, device="cuda")
        Q, V, td = c.nk * c.dk, c.nv * c.dv, TD[dtype]
        self.o = new(c.T, V + pad, dt=td)[:, :V]
        self.dq, self.dk, self.dv = new(c.T, Q + pad, dt=td)[:, :Q], new(c.T, Q + pad, dt=td)[:, :Q], new(c.T, V + pad, dt=td)[:, :V]
        self.ht, self.dh0 = new(n, c.nv, c.dk, c.dv), new(n, c.nv, c.dk, c.dv)
        self.dg, self.dbeta = new(c.T, c.nv), new(c.T, c.nv)
        sizes = (dtype, c.T, n, c.nk, c.nv, c.dk, c.dv)
        self.fwd_scratch = torch.full((zs.delta_fwd_scratch_bytes(*sizes) // 4,), math.nan, device="cuda")
        self.bwd_scratch = torch.full((zs.delta_bwd_scratch_bytes(*sizes) // 4,), math.nan, device="cuda")

    def table(self):
        zs.ops.delta_chunks(stream(), self.c.T, len(self.c.lengths), self.offsets, self.chunks)
        return self

    def head(self):
        c = self.c
        return (stream(), self.dtype, c.T, c.nk, c.nv, c.dk, c.dv, self.q, self.q.stride(0), self.k, self.k.stride(0), self.v, self.v.stride(0), self.g,
                self.beta, len(c.lengths), self.chunks, c.scale, self.h0)

    def fwd(self):
        zs.ops.delta_fwd(*self.head(), self.o, self.o.stride(0), self.ht, self.fwd_scratch, self.fwd_scratch.numel() * 4)
        return self

    def bwd(self):
        zs.ops.delta_bwd(*self.head(), self.dout, self.dout.stride(0), self.dht, self.dq, self.dq.stride(0), self.dk, self.dk.stride(0), self.dv,
                         self.dv.stride(0), self.dg, self.dbeta, self.dh0, self.bwd_scratch, self.bwd_scratch.numel() * 4)
        return self

    def all(self):
        self.table().fwd().bwd()
        return [t.clone() for t in (self.o, self.ht, self.dq, self.dk, self.dv, self.dg, self.dbeta, self.dh0)]

    def check(self, want, allow=1.0):
        chunks = -(-max(self.c.lengths + [1]) // 64)
        for n in ("o", "ht", "dq", "dk", "dv", "dg", "dbeta") + (("dh0",) if "dh0" in want else ()):
            check(n, getattr(self, n), want[n], self.dtype, chunks, allow)
        hidden = torch.ones(self.c.T, dtype=torch.bool, device="cuda")
        hidden[self.c.offsets[0]:self.c.offsets[-1]] = False
        for n in ("o", "dq", "dk", "dv", "dg", "dbeta"):
            assert (getattr(self, n)[hidden] == 0).all(), n


CASES = [
    Case(1, 1, 1, 8, 8, [1]),
    Case(3, 1, 2, 64, 16, [1, 0, 2], h0=True, ht=True),
    Case(64, 2, 2, 128, 128, [64]),
    Case(150, 2, 2, 128, 128, [63, 65], first=11, ht=True),
    Case(260, 1, 4, 32, 40, [2, 1, 0, 130, 64, 0], first=1, h0=True, ht=True),
    Case(333, 2, 4, 96, 64, [200, 128], h0=True),
    Case(400, 1, 1, 72, 256, [400], ht=True),
    Case(129, 3, 3, 128, 136, [129], h0=True, ht=True),
    Case(200, 5, 5, 40, 88, [1] * 40 + [100], h0=True),
]


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_rule_and_gradients(gpu_device, case, dtype):
    say(case, dtype)
    x, want = reference(case, dtype)
    for packed, pad in ((False, 0), (True, 0), (False, 8)):
        r = Run(case, dtype, x, packed, pad)
        r.all()
        r.check(want)


GATES = {
    "keeps": Case(300, 1, 1, 64, 32, [300], g=lambda r, T, n: np.zeros((T, n)), h0=True, ht=True),
    "forgets": Case(300, 1, 2, 64, 32, [170, 130], g=lambda r, T, n: np.where(r.random((T, n)) < 0.1, -1e4, -0.01), h0=True, ht=True),
    "writes": Case(200, 1, 1, 64, 32, [200], beta=lambda r, T, n: np.ones((T, n))),
    "reflects": Case(200, 1, 1, 128, 32, [200], beta=lambda r, T, n: np.full((T, n), 2.0), g=lambda r, T, n: np.full((T, n), -0.02)),
    "nothing": Case(100, 1, 1, 64, 32, [100], beta=lambda r, T, n: np.where(r.random((T, n)) < 0.5, 0.0, 0.7), h0=True),
    "one key": Case(260, 1, 1, 64, 64, [260], keys="same", h0=True, ht=True, beta=lambda r, T, n: np.full((T, n), 1.5)),
}


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("name", sorted(GATES))
def test_gates_and_keys_at_their_ends(gpu_device, name, dtype):
    """dg of a token that forgets everything is a difference of sums that cancel: against what it stands beside, as the 2-norm has it."""
    say(name, dtype)
    x, want = reference(GATES[name], dtype)
    r = Run(GATES[name], dtype, x)
    r.all()
    r.check(want)


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_minus_infinity_forgets(gpu_device, dtype):
    """A document whose token t has g = -inf goes on as one that begins there."""
    say("-inf", dtype)
    c = Case(200, 1, 2, 64, 32, [200], h0=True, ht=True, seed=3)
    x = c.inputs(dtype)
    x["g"][100] = -math.inf
    r = Run(c, dtype, x)
    r.all()
    y = {k: (v.clone() if v is not None else None) for k, v in x.items()}
    y["g"][100] = -1e5
    want = reference_of(c, y)
    for n in ("o", "ht", "dq", "dk", "dv", "dg", "dbeta", "dh0"):
        check(n, getattr(r, n), want[n], dtype, 4)


@gpu
@pytest.mark.parametrize("vstd,ostd", [(2000.0, 1e-4), (1e-3, 500.0), (1.0, 1e-6)])
def test_half_of_any_size(gpu_device, vstd, ostd):
    """States and gradients far from one: operands of the products follow their sizes.  Results below half's normal numbers are off by half a step of these, 2^-25,
    which is counted as well."""
    say("half", vstd, ostd)
    c = Case(200, 1, 2, 96, 48, [70, 130], h0=True, ht=True, vstd=vstd, ostd=ostd)
    x, want = reference(c, 2)
    r = Run(c, 2, x)
    r.all()
    for n in ("ht", "dg", "dbeta", "dh0"):
        check(n, getattr(r, n), want[n], 2, 3)
    for n in ("o", "dq", "dk", "dv"):
        got, w = getattr(r, n).double().cpu().reshape(-1), want[n].reshape(-1)
        rms = float(w.norm()) / math.sqrt(w.numel())
        assert ((got - w).abs() <= 2.0 ** -11 * w.abs() + 2.0 ** -25 + 40 * 100 * math.sqrt(3) * 2.0 ** -20 * w.abs().clamp(min=rms)).all(), n


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("sizes", [(4, 8, 128, 64), (8, 8, 72, 48), (4, 12, 64, 40)], ids=str)
def test_many_documents(gpu_device, sizes, dtype):
    """Enough of the states for workgroups of 32 columns, the last of them with 16 or 8."""
    say("many", sizes, dtype)
    c = Case(420, *sizes, [1, 64, 0, 7, 65] + [9] * 28 + [20], first=2, h0=True, ht=True)
    x, want = reference(c, dtype)
    r = Run(c, dtype, x)
    r.all()
    r.check(want)


@gpu
@pytest.mark.parametrize("kscale,qscale,vstd,ostd", [(1.0, 2.0 ** 40, 1e6, 1e-30), (2.0 ** -30, 1.0, 1e-20, 1e20), (2.0 ** -4, 2.0 ** -40, 1.0, 1e-25)])
def test_bfloat16_of_any_size(gpu_device, kscale, qscale, vstd, ostd):
    """What a half would not hold: keys, queries, values and gradients of other sizes, times powers of two so that they stay what the type holds."""
    say("bf16", kscale, qscale, vstd, ostd)
    c = Case(200, 2, 4, 96, 48, [70, 130], h0=True, ht=True, vstd=vstd, ostd=ostd)
    x = c.inputs(1)
    x["k"], x["q"] = x["k"] * kscale, x["q"] * qscale
    r = Run(c, 1, x)
    r.all()
    r.check(reference_of(c, x))


@gpu
def test_rows_far_apart(gpu_device):
    """Rows at the largest stride, their last ones behind 2^32 elements: the bits of rows that lie together."""
    say("far")
    c = Case(1200, 1, 2, 64, 32, [3, 70, 64], first=1000, h0=True, ht=True)
    x = c.inputs(1)
    near = Run(c, 1, x)
    want, ld = near.all(), 1 << 22
    far = Run(c, 1, x)
    buf = torch.empty(c.T * ld, dtype=torch.bfloat16, device="cuda")
    assert c.offsets[0] * ld < 1 << 32 < (c.offsets[0] + 30) * ld
    at = 0
    for n in ("q", "k", "v", "dout", "o", "dq", "dk", "dv"):
        t = getattr(far, n)
        w = torch.as_strided(buf, t.shape, (ld, 1), at)
        w.copy_(t)
        setattr(far, n, w)
        at += t.shape[1]
    for p, q in zip(want, far.all()):
        assert torch.equal(p, q)


@gpu
def test_calls_repeat_their_bits_and_streams_do_not_meet(gpu_device):
    say("streams")
    c = Case(700, 2, 4, 128, 128, [300, 64, 336], h0=True, ht=True)
    x = c.inputs(1)
    a, b = Run(c, 1, x), Run(c, 1, x)
    want = a.all()
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    for r, st in zip((a, b), s):
        with torch.cuda.stream(st):
            for _ in range(3):
                got = r.all()
            r.got = got
    torch.cuda.synchronize()
    for r in (a, b):
        for p, q in zip(want, r.got):
            assert torch.equal(p, q)


@gpu
def test_replays_of_a_graph(gpu_device):
    say("graph")
    c = Case(300, 2, 2, 64, 64, [130, 90, 80], h0=True, ht=True)
    r = Run(c, 1, c.inputs(1)).table()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.fwd().bwd()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.table().fwd().bwd()
    other = Run(c, 1, c.inputs(1))
    for i in range(4):
        c.seed = i
        x = c.inputs(1)
        for n in "qkv":
            getattr(r, n).copy_(rows(x[n], 1))
        r.dout.copy_(rows(x["dout"], 1))
        for n in ("g", "beta", "h0", "dht"):
            getattr(r, n).copy_(x[n].float().cuda())
        other = Run(c, 1, x)
        want = other.all()
        g.replay()
        torch.cuda.synchronize()
        for p, q in zip(want, (r.o, r.ht, r.dq, r.dk, r.dv, r.dg, r.dbeta, r.dh0)):
            assert torch.equal(p, q)


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_not_finite_tokens_stay_in_their_document(gpu_device, dtype):
    say("not finite", dtype)
    c = Case(320, 2, 2, 64, 64, [100, 120, 100], h0=True, ht=True)
    x = c.inputs(dtype)
    want = Run(c, dtype, x).all()
    for name, value in (("q", math.nan), ("k", math.inf), ("v", math.nan), ("g", math.nan), ("beta", math.inf), ("dout", math.inf)):
        y = {k: (v.clone() if v is not None else None) for k, v in x.items()}
        y[name][150] = value
        got = Run(c, dtype, y).all()
        for p, q in zip(want, got):
            if p.shape[0] == c.T:
                assert torch.equal(p[:100], q[:100]) and torch.equal(p[220:], q[220:]), name
            else:
                assert torch.equal(p[[0, 2]], q[[0, 2]]), name


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_a_document_in_two_calls(gpu_device, dtype):
    """The last state of the first part begins the second; its gradient ends the first part's."""
    say("two calls", dtype)
    c = Case(230, 1, 2, 128, 64, [230], h0=True, ht=True)
    x, want = reference(c, dtype)
    a, b = Case(100, 1, 2, 128, 64, [100], h0=True, ht=True), Case(130, 1, 2, 128, 64, [130], h0=True, ht=True)
    part = lambda lo, hi: {k: (v[lo:hi] if k in ("q", "k", "v", "g", "beta", "dout") else v) for k, v in x.items()}
    ra, rb = Run(a, dtype, part(0, 100)).table().fwd(), Run(b, dtype, part(100, 230)).table()
    rb.h0 = ra.ht
    rb.fwd().bwd()
    ra.dht = rb.dh0
    ra.bwd()
    for n in ("o", "dq", "dk", "dv", "dg", "dbeta"):
        check(n, torch.cat((getattr(ra, n), getattr(rb, n))), want[n], dtype, 4)
    check("ht", rb.ht, want["ht"], dtype, 4)
    check("dh0", ra.dh0, want["dh0"], dtype, 4)


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_results_that_are_not_wanted(gpu_device, dtype):
    """No last states, no gradient of the first: the others keep their bits, but for results of bf16 beside last states, which are of finer products; either way
    they keep their bound."""
    say("not wanted", dtype)
    c = Case(200, 1, 1, 64, 64, [90, 110])
    x, exact = reference(c, dtype)
    r = Run(c, dtype, x)
    want = r.all()
    r.ht = r.dh0 = None
    r.fwd().bwd()
    for p, n in zip((want[0],) + tuple(want[2:7]), ("o", "dq", "dk", "dv", "dg", "dbeta")):
        assert torch.equal(p, getattr(r, n)) or (dtype == 1 and n == "o")
        check(n, getattr(r, n), exact[n], dtype, 2)


@gpu
@pytest.mark.parametrize("case", [CASES[2], CASES[4], CASES[6], CASES[7]], ids=str)
def test_results_of_bfloat16_without_last_states(gpu_device, case):
    say("no states", case)
    x, want = reference(case, 1)
    r = Run(case, 1, x)
    r.ht = None
    r.table().fwd()
    check("o", r.o, want["o"], 1, -(-max(case.lengths) // 64))


@gpu
def test_many_documents_without_last_states(gpu_device):
    say("many, no states")
    c = Case(420, 4, 8, 128, 64, [1, 64, 0, 7, 65] + [9] * 28 + [20], first=2, h0=True)
    x, want = reference(c, 1)
    r = Run(c, 1, x)
    r.ht = None
    r.table().fwd()
    check("o", r.o, want["o"], 1, 2)


@gpu
def test_as_many_documents_as_there_may_be(gpu_device):
    """2^18 walks, the first and the last one with tokens: states of the others pass through, tokens have the bits of two documents by themselves."""
    say("most")
    n = 1 << 18
    few = Case(65, 1, 1, 8, 256, [64, 1], h0=True, ht=True)
    x = few.inputs(1)
    want = Run(few, 1, x).all()
    many = Case(65, 1, 1, 8, 256, [64])
    many.lengths, many.offsets = [64] + [0] * (n - 2) + [1], [0] + [64] * (n - 1) + [65]
    r = Run(many, 1, {**x, "h0": None, "dht": None})
    r.h0, r.dht = (torch.full((n, 1, 8, 256), v, device="cuda") for v in (0.5, -0.25))
    for state, name in ((r.h0, "h0"), (r.dht, "dht")):
        state[[0, n - 1]] = x[name].float().cuda()
    got = r.all()
    for p, q in zip(want, got):
        assert torch.equal(p, q[[0, n - 1]] if q.shape[0] == n else q)
    assert (got[1][1:n - 1] == 0.5).all() and (got[7][1:n - 1] == -0.25).all()


@gpu
def test_no_documents_and_no_tokens(gpu_device):
    say("nothing")
    c = Case(70, 1, 1, 64, 64, [])
    r = Run(c, 1, Case(70, 1, 1, 64, 64, [70]).inputs(1))
    r.table().fwd().bwd()
    for t in (r.o, r.dq, r.dk, r.dv, r.dg, r.dbeta):
        assert (t == 0).all()
    c = Case(5, 1, 1, 64, 64, [0, 0], first=2, h0=True, ht=True)   # documents without tokens pass their states on
    x = c.inputs(1)
    r = Run(c, 1, x)
    r.all()
    assert torch.equal(r.ht, r.h0) and torch.equal(r.dh0, r.dht) and (r.o == 0).all()


# ---------------------------------------------------------------------------------------------- the table
def table_of(c):
    n, room = len(c.lengths), zs.delta_chunks_ints(c.T, len(c.lengths)) // 4
    t = np.zeros((room, 4), dtype=np.int64)
    t[0] = (0, c.offsets[0], c.offsets[-1], 0)
    first = np.concatenate(([0], np.cumsum([-(-m // 64) for m in c.lengths])))
    order = sorted(range(n), key=lambda d: (-c.lengths[d], d)) if n <= 1024 else range(n)
    for place, d in enumerate(order):
        t[1 + place] = (c.offsets[d], c.lengths[d], first[d], d)
    at = 1 + n
    for d in range(n):
        for i in range(-(-c.lengths[d] // 64)):
            t[at] = (c.offsets[d] + 64 * i, min(64, c.lengths[d] - 64 * i), d, i)
            at += 1
    return t


@gpu
@pytest.mark.parametrize("lengths,first,T", [([1], 0, 1), ([64, 0, 65, 1000, 3], 5, 1200), ([7] * 1024, 0, 7168), (list(range(0, 1500)), 3, 1124253)], ids=["one", "few", "1024", "1500"])
def test_table(gpu_device, lengths, first, T):
    say("table", len(lengths))
    c = Case(T, 1, 1, 8, 8, lengths, first)
    out = torch.full((zs.delta_chunks_ints(T, len(lengths)),), -7, dtype=torch.int32, device="cuda")
    zs.ops.delta_chunks(stream(), T, len(lengths), torch.tensor(c.offsets, dtype=torch.int32, device="cuda"), out)
    assert np.array_equal(out.cpu().numpy().reshape(-1, 4), table_of(c))


@gpu
def test_table_of_offsets_that_fall_or_leave_the_tokens(gpu_device):
    """Whatever they are, every row of the table stays inside the tokens and inside the table, and the calls end."""
    say("bad offsets")
    rng = np.random.default_rng(9)
    for T, n in ((100, 3), (1000, 50), (700, 1), (64, 200)):
        room = zs.delta_chunks_ints(T, n) // 4 - 1 - n
        for _ in range(5):
            offsets = rng.integers(-2 * T, 3 * T, n + 1)
            out = torch.full((4 * (1 + n + room),), -7, dtype=torch.int32, device="cuda")
            zs.ops.delta_chunks(stream(), T, n, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out)
            t = out.cpu().numpy().reshape(-1, 4)
            docs, chunks = t[1:1 + n], t[1 + n:]
            assert 0 <= t[0, 1] <= t[0, 2] <= T
            assert (docs[:, 0] >= 0).all() and (docs[:, 1] >= 0).all() and (docs[:, 0] + docs[:, 1] <= T).all() and sorted(docs[:, 3]) == list(range(n))
            busy = docs[:, 1] > 0
            assert (docs[busy, 2] >= 0).all() and (docs[busy, 2] + -(-docs[busy, 1] // 64) <= room).all()
            assert (chunks[:, 0] >= 0).all() and (chunks[:, 1] >= 0).all() and (chunks[:, 1] <= 64).all() and (chunks[:, 0] + chunks[:, 1] <= T).all()


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_a_table_of_anything(gpu_device, dtype):
    """Results are unspecified then; what lies beside and behind them keeps its values, and calls with a right table theirs."""
    say("any table", dtype)
    c = Case(200, 1, 2, 64, 32, [90, 0, 110], h0=True, ht=True)
    x = c.inputs(dtype)
    want = Run(c, dtype, x).all()
    rng = np.random.default_rng(9)
    for most in (300, 2 ** 31 - 1):
        r = Run(c, dtype, x, pad=8)
        r.chunks.copy_(torch.from_numpy(rng.integers(-most, most, r.chunks.numel(), dtype=np.int64).astype(np.int32)))
        outs = [t._base for t in (r.o, r.dq, r.dk, r.dv)]
        r.fwd().bwd()
        torch.cuda.synchronize()
        for t in outs:
            assert torch.isnan(t[:, -8:]).all()
        for p, q in zip(want, Run(c, dtype, x).all()):
            assert torch.equal(p, q)


# ---------------------------------------------------------------------------------------------- single tokens
def step(r, rows_, slots, state, o=None):
    c = r.c
    n = len(rows_)
    q, k, v, g, beta = (t[rows_].contiguous() for t in (r.q, r.k, r.v, r.g, r.beta))
    o = torch.full((n, c.nv * c.dv), math.nan, dtype=TD[r.dtype], device="cuda") if o is None else o
    s = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
    zs.ops.delta_step(stream(), r.dtype, n, c.nk, c.nv, c.dk, c.dv, q, q.stride(0), k, k.stride(0), v, v.stride(0), g, beta, s, c.scale, state.shape[0], state,
                      o, o.stride(0))
    return o


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("sizes", [(1, 1, 8, 8), (2, 4, 128, 128), (1, 3, 72, 40), (2, 2, 96, 256)], ids=str)
def test_single_tokens(gpu_device, sizes, dtype):
    """Three sequences of 5 tokens, a token of each at a time, against the definition; the other states keep their bits."""
    say("step", sizes, dtype)
    nk, nv, dk, dv = sizes
    c = Case(15, nk, nv, dk, dv, [5, 5, 5], h0=True, ht=True)
    x, want = reference(c, dtype)
    r = Run(c, dtype, x)
    state = torch.randn(7, nv, dk, dv, device="cuda")
    slots = [4, 0, 6]
    state[slots] = r.h0
    before = state.clone()
    out = torch.empty(15, nv * dv, dtype=TD[dtype], device="cuda")
    for t in range(5):
        out[[t, 5 + t, 10 + t]] = step(r, [t, 5 + t, 10 + t], slots, state)
    # fp32 throughout, whatever the tensors' type: 5 steps of two sums of dk terms
    check("o", out, want["o"], dtype, 1)
    check("ht", state[slots], want["ht"], 0, 1)
    for i in (1, 2, 3, 5):
        assert torch.equal(state[i], before[i])
    # without slots, and all tokens of a sequence in one call
    state = r.h0.clone()
    first = step(r, [0, 5, 10], None, state)
    assert torch.equal(first, out[[0, 5, 10]])
    state = before.clone()
    order = [0, 5, 1, 10, 2, 6, 3, 7, 4, 8, 9, 11, 12, 13, 14]
    mixed = step(r, order, [slots[t // 5] for t in order], state)
    assert torch.equal(mixed, out[order])
    check("ht", state[slots], want["ht"], 0, 1)


@gpu
def test_a_state_far_behind(gpu_device):
    """States behind 2^32 bytes and 2^31 elements: the bits of the first ones."""
    say("far state")
    c = Case(3, 4, 16, 128, 128, [3], h0=True)
    r = Run(c, 1, c.inputs(1))
    states = 2 ** 31 // (16 * 128 * 128) + 2
    state = torch.empty(states, 16, 128, 128, device="cuda")
    slots = [states - 1, 0, states - 2]
    state[slots] = r.h0[0]
    near = r.h0.expand(3, -1, -1, -1).contiguous()
    o, want = step(r, [0, 1, 2], slots, state), step(r, [0, 1, 2], None, near)
    assert torch.equal(o, want) and torch.equal(state[slots], near)


@gpu
def test_slots_outside_the_states(gpu_device):
    say("slots")
    c = Case(4, 1, 2, 64, 40, [4])
    r = Run(c, 1, c.inputs(1))
    state = torch.randn(3, 2, 64, 40, device="cuda")
    before = state.clone()
    o = step(r, [0, 1, 2, 3], [-1, 3, 1, 2 ** 31 - 1], state)
    assert (o[[0, 1, 3]] == 0).all() and o[2].abs().max() > 0
    assert torch.equal(state[[0, 2]], before[[0, 2]]) and not torch.equal(state[1], before[1])


@gpu
def test_many_tokens_of_a_state_in_one_call(gpu_device):
    """More tokens than a workgroup looks through at once."""
    say("many tokens")
    c = Case(600, 1, 1, 32, 32, [300, 300], h0=True)
    x, want = reference(c, 0)
    r = Run(c, 0, x)
    state = torch.zeros(2, 1, 32, 32, device="cuda")
    state.copy_(r.h0)
    order = [t // 2 + 300 * (t % 2) for t in range(600)]
    o = step(r, order, [t % 2 for t in range(600)], state)
    check("o", o, want["o"][order], 0, 5)
    check("ht", state, want["ht"], 0, 5)


# ---------------------------------------------------------------------------------------------- the reference, on the CPU
def test_reference_gradients_are_differences():
    c = Case(7, 1, 2, 3, 2, [4, 3], h0=True, ht=True)
    x = c.inputs(0)
    names = [n for n in ("q", "k", "v", "g", "beta", "h0")]
    leaves = [x[n].clone().requires_grad_() for n in names]
    assert torch.autograd.gradcheck(lambda *a: rule(c, {**x, **dict(zip(names, a))}), leaves)


# ---------------------------------------------------------------------------------------------- refusals, on the host
P = 4096   # an aligned address that nothing reads


def call(which, **change):
    a = dict(stream=None, dtype=1, T=128, nk=2, nv=4, dk=64, dv=64, q=P, ldq=128, k=P, ldk=128, v=P, ldv=256, g=P, beta=P, ndocs=3, chunks=P, scale=0.125, h0=None,
             o=P, ldo=256, ht=None, dht=None, dq=P, lddq=128, dkey=P, lddk=128, dval=P, lddv=256, dg=P, dbeta=P, dh0=None, scratch=P, size=1 << 40, n=8,
             slots=None, nstates=8, state=P)
    a.update(change)
    head = [a[k] for k in "stream dtype T nk nv dk dv q ldq k ldk v ldv g beta".split()]
    L = zs.lib()
    if which == "step":
        head[2] = a["n"]
        return L.stage_op_delta_step(*head, *[a[k] for k in "slots scale nstates state o ldo".split()])
    head += [a[k] for k in "ndocs chunks scale h0 o ldo".split()]
    if which == "fwd":
        return L.stage_op_delta_fwd(*head, *[a[k] for k in "ht scratch size".split()])
    return L.stage_op_delta_bwd(*head, *[a[k] for k in "dht dq lddq dkey lddk dval lddv dg dbeta dh0 scratch size".split()])


SHARED = [dict(dtype=3), dict(dtype=-1), dict(nk=0), dict(nk=3), dict(nv=0), dict(nk=8), dict(nk=2, nv=4098), dict(dk=0), dict(dk=4), dict(dk=12), dict(dk=136, ldq=272, ldk=272),
          dict(dv=0), dict(dv=12), dict(dv=264, ldv=1056, ldo=1056), dict(q=None), dict(k=None), dict(v=None), dict(g=None), dict(beta=None), dict(o=None), dict(q=P + 8), dict(k=P + 2),
          dict(v=P + 4), dict(o=P + 8), dict(g=P + 2), dict(beta=P + 1), dict(ldq=120), dict(ldk=132), dict(ldv=248), dict(ldo=255), dict(ldq=(1 << 22) + 8), dict(scale=math.inf),
          dict(scale=math.nan)]


@pytest.mark.parametrize("which", ["fwd", "bwd", "step"])
@pytest.mark.parametrize("bad", SHARED, ids=str)
def test_refusals(which, bad):
    assert call(which, **bad) == zs.STAGE_ERR_ARG


@pytest.mark.parametrize("which", ["fwd", "bwd"])
def test_refusals_of_documents(which):
    for bad in (dict(T=-1), dict(T=(1 << 26) + 1), dict(T=1 << 26, nv=32, ldv=2048, ldo=2048, lddv=2048), dict(ndocs=-1), dict(ndocs=(1 << 20) + 1), dict(ndocs=(1 << 18) + 1),
                dict(chunks=None), dict(chunks=P + 4), dict(h0=P + 4)):
        assert call(which, **bad) == zs.STAGE_ERR_ARG, bad
    for bad in (dict(scratch=None), dict(scratch=P + 128), dict(size=1000)):
        assert call(which, **bad) == zs.STAGE_ERR_WORKSPACE, bad
    assert call(which, T=0, ndocs=0, q=None, k=None, v=None, g=None, beta=None, o=None, chunks=None, scratch=None) == zs.STAGE_OK


def test_other_refusals():
    for bad in (dict(ht=P + 8),):
        assert call("fwd", **bad) == zs.STAGE_ERR_ARG
    for bad in (dict(dht=P + 8), dict(dh0=P + 8), dict(dq=None), dict(dkey=None), dict(dval=None), dict(dg=None), dict(dbeta=None), dict(dg=P + 2), dict(lddq=120), dict(lddk=120),
                dict(lddv=248), dict(dq=P + 8)):
        assert call("bwd", **bad) == zs.STAGE_ERR_ARG, bad
    for bad in (dict(n=-1), dict(n=65536, nstates=1 << 20), dict(n=9), dict(nstates=-1), dict(state=None), dict(state=P + 8), dict(slots=P + 2)):
        assert call("step", **bad) == zs.STAGE_ERR_ARG, bad
    assert call("step", n=0, q=None, k=None, v=None, state=None) == zs.STAGE_OK
    L = zs.lib()
    for T, n in ((-1, 1), (1, -1), ((1 << 26) + 1, 1), (1, (1 << 20) + 1)):
        assert L.stage_op_delta_chunks_ints(T, n) == -zs.STAGE_ERR_ARG and L.stage_op_delta_chunks(None, T, n, P, P) == zs.STAGE_ERR_ARG
    for offsets, chunks in ((None, P), (P, None), (P + 2, P), (P, P + 8)):
        assert L.stage_op_delta_chunks(None, 10, 1, offsets, chunks) == zs.STAGE_ERR_ARG
    for f in (L.stage_op_delta_fwd_scratch_bytes, L.stage_op_delta_bwd_scratch_bytes):
        assert f(1, 10, 1, 2, 3, 64, 64) == -zs.STAGE_ERR_ARG


def test_the_most_documents():
    L = zs.lib()
    for f in (L.stage_op_delta_fwd_scratch_bytes, L.stage_op_delta_bwd_scratch_bytes):
        assert f(1, 10, 1 << 16, 4, 4, 64, 64) > 0 and f(1, 10, (1 << 16) + 1, 4, 4, 64, 64) == -zs.STAGE_ERR_ARG
        assert f(1, 10, 1 << 18, 1, 1, 64, 64) > 0 and f(1, 10, (1 << 18) + 1, 1, 1, 64, 64) == -zs.STAGE_ERR_ARG


def test_scratch_and_table_never_shrink():
    for f in (zs.delta_fwd_scratch_bytes, zs.delta_bwd_scratch_bytes):
        last = 0
        for T in (0, 1, 63, 64, 65, 128, 1000, 4096, 8191, 100000):
            n = f(1, T, 7, 2, 4, 128, 128)
            assert n >= last
            last = n
        assert f(1, 1000, 8, 2, 4, 128, 128) >= f(1, 1000, 7, 2, 4, 128, 128)
    rng = np.random.default_rng(1)
    for _ in range(300):   # room for any cut of T tokens
        lengths = rng.integers(0, int(rng.integers(2, 300)), int(rng.integers(1, 40)))
        T = int(lengths.sum())
        assert zs.delta_chunks_ints(T, len(lengths)) >= 4 * (1 + len(lengths) + int((-(-lengths // 64)).sum()))
