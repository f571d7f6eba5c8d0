"""A recurrent token mixer and what bounds the step that trains it, as a program that builds a layer from single operators calls them:
the gated delta rule inside packed documents (`delta_fwd`), its gradient (`delta_bwd`), its form for single tokens over kept states
(`delta_step`), and the global norm of many gradient tensors (`grad_norm`) with their clipping (`grad_scale`).

listed() gives the cases by name, draw() more of the same ranges, prepare() the buffers that such a program holds, run() one pass
(in plain torch, or with `own` through the framework), exact() the same results in 64 bits, work() what a pass cannot do without.
"""
import math
from types import SimpleNamespace

import torch

own = False

F32, BF16, F16 = 0, 1, 2
TORCH = {F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16}
BYTES = {F32: 4, BF16: 2, F16: 2}
CHUNK = 64   # tokens that the plain form works on at a time


def delta(kind, name, dtype, T, nk, nv, dk, dv, lengths, states=False, packed=False):
    """nk heads of q and k, dk wide, nv heads of v, dv wide.  lengths: of the documents, which begin at token 0; tokens behind the last one
    are padding.  states: documents begin with a state that they are given, and their last one comes back (backward: its gradient
    goes in, the first one's comes back).  packed: q, k and v are columns of one buffer."""
    c = dict(kind=kind, dtype=dtype, T=T, nk=nk, nv=nv, dk=dk, dv=dv, lengths=lengths, states=states, packed=packed)
    return dict(c, name=name) if name else c


def step(name, dtype, n, nk, nv, dk, dv, slots):
    """n sequences take one token each; their states are n of `slots` that are kept."""
    c = dict(kind="step", dtype=dtype, n=n, nk=nk, nv=nv, dk=dk, dv=dv, slots=slots)
    return dict(c, name=name) if name else c


def grads(kind, name, types, sizes, scale, max_norm, packed=False):
    """types: of the tensors, in turn; sizes: their elements, "n*times".  packed: the tensors of a type follow one another without gaps."""
    c = dict(kind=kind, types=types, sizes=sizes, scale=scale, max_norm=max_norm, packed=packed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One short microbatch of a small bf16 model: three documents, one of them a single token.
        delta("fwd", "fwd_bf16_small", BF16, 256, 4, 4, 128, 128, "100 1 155", packed=True),
        # A 7B-class layer over packed documents, padding at the end.
        delta("fwd", "fwd_bf16_docs", BF16, 4096, 16, 16, 128, 128, "1531 64 700 1289 300 150"),
        # One long document, two value heads to a key head: the largest amount of work.
        delta("fwd", "fwd_bf16_long", BF16, 8192, 16, 32, 128, 128, "8192"),
        # Prompts that go on from kept states, in half, with heads of other widths.
        delta("fwd", "fwd_f16_states", F16, 2000, 8, 8, 96, 192, "333 80 512 17 250 808", states=True, packed=True),
        # fp32, as a user checks a setup.
        delta("bwd", "bwd_f32_states", F32, 1000, 4, 8, 64, 64, "400 7 350 200", states=True),
        # The gradients of the same layers.
        delta("bwd", "bwd_bf16_small", BF16, 256, 4, 4, 128, 128, "100 1 155", packed=True),
        delta("bwd", "bwd_bf16_docs", BF16, 4096, 16, 16, 128, 128, "1531 64 700 1289 300 150"),
        # Decoding: one sequence, and a batch of them over a larger store of states.
        step("step_bf16_one", BF16, 1, 16, 32, 128, 128, 8),
        step("step_bf16_batch", BF16, 48, 16, 32, 128, 128, 64),
        # The norm of a small fp32 model's gradients: a launch and little else.
        grads("norm", "norm_f32_small", "f32", "196608*2 65536*2 262144*4 1024*4 256*14", 1.0, 1.0),
        # Clipping all gradients of two 7B-class layers, which are segments of one accumulator.
        grads("clip", "clip_f32_layers", "f32", "4096*2 16777216*4 45088768*3 4096*2 16777216*4 45088768*3", 0.0625, 1.0, packed=True),
        # Many tensors of two types, matrices in bf16 and gains in fp32, of odd sizes.
        grads("clip", "clip_mixed_many", "bf16 f32", "1048577*40 777*40 262143*60 1*20 4096*140", 1.0, 1.0),
    ]


def log_int(rng, lo, hi, multiple=1):
    """A whole number between lo and hi, spread over the logarithm, a multiple of `multiple`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    most = max(work(c)["bytes"] for c in listed() if c["kind"] == "fwd")
    while True:
        kind = rng.choice(["fwd", "fwd", "bwd", "bwd", "step", "norm", "clip"])
        dtype = rng.choice([F32, BF16, BF16, F16])
        nk = log_int(rng, 1, 16)
        nv = nk * rng.choice([1, 1, 2, 4])
        dk, dv = rng.choice([32, 64, 72, 96, 128, 128]), rng.choice([32, 64, 88, 128, 128, 192, 256])
        if kind == "step":
            n = log_int(rng, 1, 96)
            c = step(None, dtype, n, nk, nv, dk, dv, n + rng.randint(0, 16))
            if work(c)["bytes"] <= most:
                return c
            continue
        if kind in ("norm", "clip"):
            sizes = " ".join("%d*%d" % (log_int(rng, 1, 2e7), log_int(rng, 1, 40)) for _ in range(rng.randint(1, 6)))
            c = grads(kind, None, rng.choice(["f32", "f32", "bf16", "f16", "bf16 f32", "f16 f32"]), sizes, rng.choice([1.0, 1.0 / 1024]),
                      rng.choice([1.0, 0.1, 1e6]), rng.random() < 0.5)
            if work(c)["bytes"] <= max(work(d)["bytes"] for d in listed() if d["kind"] == "clip"):
                return c
            continue
        T = log_int(rng, 16, 2048 if dtype == F32 else 8192)
        left, lengths = T - rng.choice([0, 0, rng.randint(0, T // 4)]), []
        mean = log_int(rng, 32, 4096)
        while left > 0:
            lengths.append(min(left, 1 + int(rng.expovariate(1.0 / mean))))
            left -= lengths[-1]
        c = delta(kind, None, dtype, T, nk, nv, dk, dv, " ".join(map(str, lengths)), rng.random() < 0.4, rng.random() < 0.5)
        # the plain form pads the documents to the longest
        if work(c)["bytes"] <= most and len(lengths) * max(lengths) * nv <= 2 ** 18 and T * nv <= (2 ** 16 if kind == "bwd" else 2 ** 18):
            return c


def ints(text):
    return [int(x) for x in text.split()]


def scale_of(c):
    return float(torch.tensor(c["dk"] ** -0.5, dtype=torch.float32))


# ---------------------------------------------------------------------------------------------- inputs
class Draw:
    """Normal deviates on the GPU from one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float32)

    def uniform(self, lo, hi, *shape):
        return lo + (hi - lo) * torch.rand(*shape, generator=self.g, device="cuda", dtype=torch.float32)


def rows_of(c, r, T):
    """q [T, nk*dk] and k, whose heads have length one, as the rule wants them, v [T, nv*dv], g [T, nv] and beta [T, nv] in fp32."""
    dt, nk, nv, dk, dv = TORCH[c["dtype"]], c["nk"], c["nv"], c["dk"], c["dv"]
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)
    q, k = unit(r.normal(T, nk, dk)).reshape(T, -1).to(dt), unit(r.normal(T, nk, dk) + 0.5 * r.normal(1, nk, dk)).reshape(T, -1).to(dt)
    v = r.normal(T, nv * dv).to(dt)
    # heads that forget within a few tokens to some that keep thousands
    g = -torch.exp(r.uniform(math.log(1e-3), math.log(2.0), 1, nv)) * torch.nn.functional.softplus(r.normal(T, nv))
    beta = torch.sigmoid(r.normal(T, nv))
    return q, k, v, g, beta


def inputs(c, seed):
    r = Draw(seed)
    s = SimpleNamespace(c=c)
    if c["kind"] in ("norm", "clip"):
        return grad_inputs(s, r)
    if c["kind"] == "step":
        s.q, s.k, s.v, s.g, s.beta = rows_of(c, r, c["n"])
        s.slots = torch.randperm(c["slots"], generator=r.g, device="cuda")[:c["n"]].to(torch.int32)
        s.state = 0.3 * r.normal(c["slots"], c["nv"], c["dk"], c["dv"])
        return s
    q, k, v, s.g, s.beta = rows_of(c, r, c["T"])
    if c["packed"]:
        qkv = torch.cat((q, k, v), 1)
        q, k, v = qkv[:, :q.shape[1]], qkv[:, q.shape[1]:2 * q.shape[1]], qkv[:, 2 * q.shape[1]:]
    s.q, s.k, s.v = q, k, v
    s.lengths = ints(c["lengths"])
    n = len(s.lengths)
    s.offsets = torch.tensor([sum(s.lengths[:i]) for i in range(n + 1)], dtype=torch.int32, device="cuda")
    shape = (n, c["nv"], c["dk"], c["dv"])
    s.h0 = 0.3 * r.normal(*shape) if c["states"] else None
    if c["kind"] == "bwd":
        s.dout = (r.normal(c["T"], c["nv"] * c["dv"]) * 1e-2 * (256.0 if c["dtype"] == F16 else 1.0)).to(TORCH[c["dtype"]])
        s.dht = 1e-2 * r.normal(*shape) if c["states"] else None
    return s


def grad_inputs(s, r):
    """The tensors as pieces of one buffer for each type; those of packed buffers follow one another at once."""
    types = s.c["types"].split()
    sizes = [int(n) for part in s.c["sizes"].split() for n in [part.split("*")[0]] * int(part.split("*")[1])]
    at, places = {t: 0 for t in types}, []
    for i, n in enumerate(sizes):
        t = types[i % len(types)]
        places.append((t, at[t], n))
        at[t] += n if s.c["packed"] else -(-n // 128) * 128
    dts = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
    s.flat = {t: (0.01 * r.normal(max(1, at[t]))).to(dts[t]) for t in sorted(at)}
    s.tensors = [s.flat[t][a:a + n] for t, a, n in places]
    if not s.c["packed"]:
        for t, a, n in places:
            s.flat[t][a + n:a + -(-n // 128) * 128] = 0
    s.places = places
    return s


def prepare(case, seed):
    s = inputs(case, seed)
    c = s.c
    if not own:
        return s
    import paper_2507_10392_amd as zs
    s.zs = zs
    empty = lambda *shape, dtype: torch.empty(*shape, dtype=dtype, device="cuda")
    if c["kind"] in ("norm", "clip"):
        s.flat_out = {t: torch.zeros_like(x) for t, x in s.flat.items()}
        s.list = zs.tensor_list(s.tensors, [s.flat_out[t][a:a + n] for t, a, n in s.places])
        s.scratch = empty(zs.grad_norm_scratch_bytes(s.list), dtype=torch.uint8)
        s.sumsq, s.norm, s.factor = empty(1, dtype=torch.float64), empty(1, dtype=torch.float32), empty(1, dtype=torch.float32)
        return s
    dt = TORCH[c["dtype"]]
    if c["kind"] == "step":
        s.o = empty(c["n"], c["nv"] * c["dv"], dtype=dt)
        return s
    # The documents' chunks are a table that a program makes once per microbatch and keeps for all layers, forward and backward.
    T, n, sizes = c["T"], len(s.lengths), (c["dtype"], c["T"], len(s.lengths), c["nk"], c["nv"], c["dk"], c["dv"])
    s.chunks = empty(zs.delta_chunks_ints(T, n), dtype=torch.int32)
    zs.ops.delta_chunks(torch.cuda.current_stream().cuda_stream, T, n, s.offsets, s.chunks)
    if c["kind"] == "fwd":
        s.o = empty(T, c["nv"] * c["dv"], dtype=dt)
        s.ht = torch.empty_like(s.h0) if c["states"] else None
        s.scratch = empty(zs.delta_fwd_scratch_bytes(*sizes), dtype=torch.uint8)
    else:
        s.dq, s.dk, s.dv = (empty(T, x.shape[1], dtype=dt) for x in (s.q, s.k, s.v))
        s.dg, s.dbeta = torch.empty_like(s.g), torch.empty_like(s.beta)
        s.dh0 = torch.empty_like(s.h0) if c["states"] else None
        s.scratch = empty(zs.delta_bwd_scratch_bytes(*sizes), dtype=torch.uint8)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return {"fwd": own_fwd, "bwd": own_bwd, "step": own_step, "norm": own_norm, "clip": own_clip}[state.c["kind"]](state)
    return {"fwd": plain_fwd, "bwd": plain_bwd, "step": plain_step, "norm": plain_norm, "clip": plain_clip}[state.c["kind"]](state)


def stream():
    return torch.cuda.current_stream().cuda_stream


def with_states(s, res, **more):
    return dict(res, **more) if s.c["states"] else res


def own_fwd(s):
    c = s.c
    s.zs.ops.delta_fwd(stream(), c["dtype"], c["T"], c["nk"], c["nv"], c["dk"], c["dv"], s.q, s.q.stride(0), s.k, s.k.stride(0), s.v, s.v.stride(0),
                       s.g, s.beta, len(s.lengths), s.chunks, scale_of(c), s.h0, s.o, s.o.stride(0), s.ht, s.scratch, s.scratch.numel())
    return with_states(s, {"o": s.o}, ht=s.ht)


def own_bwd(s):
    c = s.c
    s.zs.ops.delta_bwd(stream(), c["dtype"], c["T"], c["nk"], c["nv"], c["dk"], c["dv"], s.q, s.q.stride(0), s.k, s.k.stride(0), s.v, s.v.stride(0),
                       s.g, s.beta, len(s.lengths), s.chunks, scale_of(c), s.h0, s.dout, s.dout.stride(0), s.dht, s.dq, s.dq.stride(0), s.dk,
                       s.dk.stride(0), s.dv, s.dv.stride(0), s.dg, s.dbeta, s.dh0, s.scratch, s.scratch.numel())
    return with_states(s, {"dq": s.dq, "dk": s.dk, "dv": s.dv, "dg": s.dg, "dbeta": s.dbeta}, dh0=s.dh0)


def own_step(s):
    c = s.c
    s.zs.ops.delta_step(stream(), c["dtype"], c["n"], c["nk"], c["nv"], c["dk"], c["dv"], s.q, s.q.stride(0), s.k, s.k.stride(0), s.v, s.v.stride(0),
                        s.g, s.beta, s.slots, scale_of(c), c["slots"], s.state, s.o, s.o.stride(0))
    return {"o": s.o, "state": s.state}


def own_norm(s):
    s.zs.grad_norm(stream(), s.list, s.c["scale"], s.c["max_norm"], s.sumsq, s.norm, s.factor, None, s.scratch)
    return {"sumsq": s.sumsq, "norm": s.norm, "factor": s.factor}


def own_clip(s):
    s.zs.grad_norm(stream(), s.list, s.c["scale"], s.c["max_norm"], s.sumsq, s.norm, s.factor, None, s.scratch)
    s.zs.grad_scale(stream(), s.list, s.factor)
    return {"norm": s.norm, "clipped": s.flat_out}


def plain_norm(s):
    # squares in 64 bits: those of large and of small gradients do not fit 32
    sumsq = sum(x.double().square().sum() for x in s.flat.values()).reshape(1)
    norm = (s.c["scale"] * sumsq.sqrt()).float()
    return {"sumsq": sumsq, "norm": norm, "factor": torch.where(norm > s.c["max_norm"], s.c["max_norm"] / norm, 1.0)}


def plain_clip(s):
    n = plain_norm(s)
    return {"norm": n["norm"], "clipped": {t: (x.float() * n["factor"]).to(x.dtype) for t, x in s.flat.items()}}


def plain_step(s):
    c = s.c
    group = c["nv"] // c["nk"]
    at = s.slots.long()
    q, k = (x.float().reshape(c["n"], c["nk"], c["dk"]).repeat_interleave(group, 1) for x in (s.q, s.k))
    v = s.v.float().reshape(c["n"], c["nv"], c["dv"])
    h = s.state[at] * s.g.exp()[..., None, None]
    u = (v - (h * k[..., None]).sum(2)) * s.beta[..., None]
    h = h + k[..., None] * u[:, :, None]
    s.state[at] = h
    o = (h * q[..., None]).sum(2) * scale_of(c)
    return {"o": o.reshape(c["n"], -1).to(s.v.dtype), "state": s.state}


def chunked(s):
    """The documents side by side, padded to whole chunks of the longest with tokens that change nothing: x [tokens, heads * d] ->
    [chunks, documents * value heads, CHUNK, d], and back."""
    c = s.c
    n, chunks = len(s.lengths), -(-max(s.lengths) // CHUNK)
    at = torch.arange(chunks * CHUNK, device="cuda")
    length = s.offsets[1:] - s.offsets[:-1]
    live = at[None] < length[:, None]
    token = (s.offsets[:-1, None] + at[None]).clamp(max=c["T"] - 1).long()

    def split(x, heads):
        y = x.float()[token] * live[..., None]
        y = y.reshape(n, chunks, CHUNK, heads, -1).repeat_interleave(c["nv"] // heads, 3)
        return y.permute(1, 0, 3, 2, 4).reshape(chunks, n * c["nv"], CHUNK, -1)

    def join(y, heads):
        d = y.shape[-1]
        y = y.reshape(chunks, n, heads, c["nv"] // heads, CHUNK, d).sum(3)
        x = torch.zeros(c["T"], heads * d, device="cuda")
        x[token[live]] = y.permute(1, 0, 3, 2, 4).reshape(n, chunks * CHUNK, heads * d)[live]
        return x

    return split, join


def t_(x):
    return x.transpose(-1, -2).contiguous()


def plain_forward(s):
    """Every chunk's matrices at once, then its state from the one before."""
    c = s.c
    split, join = chunked(s)
    f = SimpleNamespace(join=join)
    f.q, f.k, f.v = split(s.q, c["nk"]), split(s.k, c["nk"]), split(s.v, c["nv"])
    G = split(s.g, c["nv"]).double().cumsum(2)              # angles of the decay: sums of many small logarithms
    f.beta = split(s.beta, c["nv"])
    low = torch.ones(CHUNK, CHUNK, device="cuda").tril()
    f.decay = torch.exp(((G - t_(G)) * low).float()) * low  # of j's share up to i
    f.since, f.until, f.whole = torch.exp(G).float(), torch.exp(G[:, :, -1:] - G).float(), torch.exp(G[:, :, -1:]).float()
    f.kk = torch.matmul(f.k, t_(f.k)) * f.decay.tril(-1)
    A = (f.beta * f.kk).double()
    f.inv = torch.eye(CHUNK, device="cuda", dtype=torch.float64) - A
    for _ in range(5):                                      # 1 / (1 + A) = (1 - A)(1 + A^2)(1 + A^4)... , and A^CHUNK = 0
        A = torch.matmul(A, A)
        f.inv = f.inv + torch.matmul(f.inv, A)
    f.inv = f.inv.float()
    f.p = torch.matmul(f.q, t_(f.k)) * f.decay
    h = torch.zeros(f.q.shape[1], c["dk"], c["dv"], device="cuda") if s.h0 is None else s.h0.reshape(-1, c["dk"], c["dv"])
    f.h, f.u = [], []
    for i in range(f.q.shape[0]):
        f.h.append(h)
        f.u.append(torch.matmul(f.inv[i], f.beta[i] * (f.v[i] - f.since[i] * torch.matmul(f.k[i], h))))
        h = f.whole[i] * h + torch.matmul(t_(f.k[i]), f.until[i] * f.u[i])
    f.h, f.u, f.last = torch.stack(f.h), torch.stack(f.u), h
    return f


def plain_fwd(s):
    c = s.c
    f = plain_forward(s)
    o = (f.since * torch.matmul(f.q, f.h) + torch.matmul(f.p, f.u)) * scale_of(c)
    return with_states(s, {"o": f.join(o, c["nv"]).to(s.v.dtype)}, ht=f.last.reshape(len(s.lengths), c["nv"], c["dk"], c["dv"]))


def plain_bwd(s):
    c = s.c
    f = plain_forward(s)
    split, join = chunked(s)
    do = split(s.dout, c["nv"]) * scale_of(c)
    pt, invt, kt, qt = t_(f.p), t_(f.inv), t_(f.k), t_(f.q)
    dh = torch.zeros_like(f.last) if s.dht is None else s.dht.reshape(f.last.shape)
    dhs, ys = [], []
    for i in reversed(range(f.q.shape[0])):
        dhs.append(dh)
        du = torch.matmul(pt[i], do[i]) + f.until[i] * torch.matmul(f.k[i], dh)
        ys.append(torch.matmul(invt[i], du))
        dh = f.whole[i] * dh + torch.matmul(qt[i], f.since[i] * do[i]) - torch.matmul(kt[i], f.beta[i] * f.since[i] * ys[-1])
    dhs, y = torch.stack(dhs[::-1]), torch.stack(ys[::-1])
    ht = t_(f.h)
    dp, da = torch.matmul(do, t_(f.u)), -torch.matmul(y, t_(f.u))
    ep, ea = dp * f.p, da * (f.beta * f.kk)                 # by the decay's logarithm
    mp, ma = dp * f.decay, da * f.beta * f.decay.tril(-1)
    q_state, k_state, k_next = f.since * torch.matmul(do, ht), -f.since * torch.matmul(y, ht), f.until * torch.matmul(f.u, t_(dhs))
    dq = q_state + torch.matmul(mp, f.k)
    dk = f.beta * k_state + k_next + torch.matmul(t_(mp), f.q) + torch.matmul(ma + t_(ma), f.k)
    dbeta = (y * f.v).sum(-1) + (f.k * k_state).sum(-1) + (da * f.kk).sum(-1)
    e, next_ = ep + ea, (f.k * k_next).sum(-1)
    dG = e.sum(-1) - e.sum(-2) + (f.q * q_state).sum(-1) + f.beta[..., 0] * (f.k * k_state).sum(-1) - next_
    dG[..., -1] += next_.sum(-1) + (f.whole * f.h * dhs).sum((-1, -2))
    dg = dG.flip(-1).cumsum(-1).flip(-1)
    dt = s.v.dtype
    res = {"dq": join(dq, c["nk"]).to(dt), "dk": join(dk, c["nk"]).to(dt), "dv": join(f.beta * y, c["nv"]).to(dt), "dg": join(dg[..., None], c["nv"]),
           "dbeta": join(dbeta[..., None], c["nv"])}
    return with_states(s, res, dh0=dh.reshape(len(s.lengths), c["nv"], c["dk"], c["dv"]))


# ---------------------------------------------------------------------------------------------- work
def work(c):
    if c["kind"] in ("norm", "clip"):
        types, sizes = c["types"].split(), [int(n) for part in c["sizes"].split() for n in [part.split("*")[0]] * int(part.split("*")[1])]
        n = sum(m * (4 if types[i % len(types)] == "f32" else 2) for i, m in enumerate(sizes))
        return {"bytes": n * (2 if c["kind"] == "clip" else 1), "flops": sum(sizes) * (3 if c["kind"] == "clip" else 2)}
    E, Q, V, H = BYTES[c["dtype"]], c["nk"] * c["dk"], c["nv"] * c["dv"], c["nv"] * c["dk"] * c["dv"]
    if c["kind"] == "step":
        return {"bytes": c["n"] * (2 * E * (Q + V) + 8 * c["nv"] + 8 * H), "flops": 7 * c["n"] * H}
    lengths = ints(c["lengths"])
    tokens, states = sum(lengths), len(lengths) * H * 8 if c["states"] else 0
    if c["kind"] == "fwd":   # a token reads its state along k, adds to it, reads it along q
        return {"bytes": 2 * E * c["T"] * (Q + V) + 8 * c["T"] * c["nv"] + states, "flops": 6 * tokens * H}
    return {"bytes": E * c["T"] * (4 * Q + 3 * V) + 16 * c["T"] * c["nv"] + 2 * states, "flops": 16 * tokens * H}   # the states again, then their gradients


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = inputs(case, seed)
    if case["kind"] in ("norm", "clip"):
        return exact_grads(s)
    return {"fwd": exact_fwd, "bwd": exact_bwd, "step": exact_step}[case["kind"]](s)


def exact_grads(s):
    total = math.fsum(float(torch.dot(x.double(), x.double())) for x in s.tensors)
    norm = s.c["scale"] * math.sqrt(total)
    factor = min(1.0, s.c["max_norm"] / norm) if norm else 1.0
    one = lambda v: torch.tensor([v], dtype=torch.float64, device="cuda")
    if s.c["kind"] == "norm":
        return {"sumsq": one(total), "norm": one(norm), "factor": one(factor)}
    return {"norm": one(norm), "clipped": {t: x.double() * factor for t, x in s.flat.items()}}


def heads64(s, x, n):
    return x.double().reshape(x.shape[0], n, -1).repeat_interleave(s.c["nv"] // n, 1)


def exact_step(s):
    c = s.c
    q, k, v = heads64(s, s.q, c["nk"]), heads64(s, s.k, c["nk"]), heads64(s, s.v, c["nv"])
    state = s.state.double()
    old = torch.exp(s.g.double())[..., None, None] * state[s.slots.long()]
    new = old + torch.einsum("nhk,nhv->nhkv", k, s.beta.double()[..., None] * (v - torch.einsum("nhk,nhkv->nhv", k, old)))
    state[s.slots.long()] = new
    return {"o": torch.einsum("nhk,nhkv->nhv", q, new).reshape(c["n"], -1) * scale_of(c), "state": state}


def exact_states(s, first, n, h, keep):
    """Token after token of one document: its outputs, what each writes, the last state, and (keep) the decayed state before each."""
    c = s.c
    rows = slice(first, first + n)
    q, k, v = (heads64(s, x[rows], m) for x, m in ((s.q, c["nk"]), (s.k, c["nk"]), (s.v, c["nv"])))
    a, beta = torch.exp(s.g[rows].double()), s.beta[rows].double()
    o, u, kept = torch.empty_like(v), torch.empty_like(v), []
    for t in range(n):
        h = a[t][:, None, None] * h
        if keep:
            kept.append(h)
        u[t] = beta[t][:, None] * (v[t] - torch.bmm(k[t][:, None], h)[:, 0])
        h = torch.baddbmm(h, k[t][:, :, None], u[t][:, None])
        o[t] = torch.bmm(q[t][:, None], h)[:, 0] * scale_of(c)
    return SimpleNamespace(q=q, k=k, v=v, a=a, beta=beta, o=o, u=u, h=h, kept=kept)


def first_state(s, i):
    c = s.c
    return torch.zeros(c["nv"], c["dk"], c["dv"], dtype=torch.float64, device="cuda") if s.h0 is None else s.h0[i].double()


def exact_fwd(s):
    c = s.c
    o, last, first = torch.zeros(c["T"], c["nv"], c["dv"], dtype=torch.float64, device="cuda"), [], 0
    for i, n in enumerate(s.lengths):
        d = exact_states(s, first, n, first_state(s, i), False)
        o[first:first + n] = d.o
        last.append(d.h)
        first += n
    return with_states(s, {"o": o.reshape(c["T"], -1)}, ht=torch.stack(last))


def exact_bwd(s):
    """The transposed recurrence, from the last token to the first."""
    c = s.c
    new = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")
    T, nv, dk, dv = c["T"], c["nv"], c["dk"], c["dv"]
    dq, dkey, dval, dg, dbeta, dh0, first = new(T, nv, dk), new(T, nv, dk), new(T, nv, dv), new(T, nv), new(T, nv), [], 0
    for i, n in enumerate(s.lengths):
        h0 = first_state(s, i)
        d = exact_states(s, first, n, h0, True)
        do = s.dout[first:first + n].double().reshape(n, nv, dv) * scale_of(c)
        e = new(nv, dk, dv) if s.dht is None else s.dht[i].double()
        for t in reversed(range(n)):
            at, before = first + t, d.kept[t]
            after = torch.baddbmm(before, d.k[t][:, :, None], d.u[t][:, None])
            dq[at] = torch.bmm(after, do[t][:, :, None])[..., 0]
            e = torch.baddbmm(e, d.q[t][:, :, None], do[t][:, None])
            du = torch.bmm(d.k[t][:, None], e)[:, 0]
            dval[at] = d.beta[t][:, None] * du
            dbeta[at] = (du * d.u[t]).sum(-1) / d.beta[t]
            dkey[at] = torch.bmm(e, d.u[t][:, :, None])[..., 0] - torch.bmm(before, dval[at][:, :, None])[..., 0]
            e = torch.baddbmm(e, d.k[t][:, :, None], dval[at][:, None], alpha=-1)
            dg[at] = (e * before).sum((-1, -2))
            e = d.a[t][:, None, None] * e
        dh0.append(e)
        first += n
    share = lambda x: x.reshape(T, c["nk"], -1, dk).sum(2).reshape(T, -1)
    res = {"dq": share(dq), "dk": share(dkey), "dv": dval.reshape(T, -1), "dg": dg, "dbeta": dbeta}
    return with_states(s, res, dh0=torch.stack(dh0))
