"""The operators for packed sequences (several documents behind one another in a microbatch), as a training program calls them:
rotary positions with several axes on the heads of q and k (`rope_axes`), attention inside the documents with capped scores, a
bias that falls with distance, bidirectional prefixes and shared key heads (`attention_docs_fwd`), and its gradient
(`attention_docs_bwd`).

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
ROPE_BASE = 10000.0


def rope(name, dtype, T, nh, nkv, d, sections, own_spectrum=False, start=0, sign=1, packed=False):
    """sections: pairs of a head's d/2 that each axis turns.  start: the first position of the first axis.  packed: q and k are
    columns of one [q | k | v] buffer."""
    c = dict(kind="rope", dtype=dtype, T=T, nh=nh, nkv=nkv, d=d, sections=sections, own_spectrum=own_spectrum, start=start, sign=sign,
             packed=packed)
    return dict(c, name=name) if name else c


def attention(kind, name, dtype, T, nh, nkv, d, lengths, prefix="", softcap=0.0, slopes=False, packed=False):
    """lengths: of the documents, which begin at token 0; tokens behind the last one are padding.  prefix: tokens at each document's
    begin that all its tokens see, none if empty."""
    c = dict(kind=kind, dtype=dtype, T=T, nh=nh, nkv=nkv, d=d, lengths=lengths, prefix=prefix, softcap=softcap, slopes=slopes, packed=packed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # Heads of the small fp32 stage, text positions only on one axis: a launch and little else.
        rope("rope_f32_small", F32, 256, 4, 4, 64, "32"),
        # A 7B-class layer on video tokens: time, height and width, 8 key heads.
        rope("rope_bf16_video", BF16, 4096, 32, 8, 128, "16 24 24", start=100000),
        # Gradients of an image encoder's heads (height and width, a spectrum each), odd number of tokens, inside a packed buffer.
        rope("rope_f16_image_back", F16, 9001, 16, 16, 80, "20 20", own_spectrum=True, sign=-1, packed=True),
        # One short microbatch of a small bf16 model: three documents, one of them a single token.
        attention("fwd", "fwd_bf16_small", BF16, 256, 4, 4, 128, "100 1 139", packed=True),
        # A 7B-class layer over packed documents with capped scores and 8 key heads, padding at the end.
        attention("fwd", "fwd_bf16_capped", BF16, 4096, 32, 8, 128, "1531 64 700 1289 300 150", softcap=50.0),
        # One long document after a bidirectional prefix: the largest amount of work.
        attention("fwd", "fwd_bf16_prefix_long", BF16, 8192, 32, 8, 128, "8192", prefix="1024"),
        # Many short documents with a distance bias instead of positions, heads of 64, in fp16.
        attention("fwd", "fwd_f16_bias_short", F16, 4000, 16, 16, 64, "333 80 512 17 250 61 400 129 200 350 90 611 5 400 262 300",
                  slopes=True, packed=True),
        # fp32, everything at once, as a user checks a setup.
        attention("fwd", "fwd_f32_all", F32, 1000, 8, 2, 64, "400 7 350 200", prefix="100 0 350 13", softcap=30.0, slopes=True),
        # The gradients of the same layers.
        attention("bwd", "bwd_bf16_small", BF16, 256, 4, 4, 128, "100 1 139", packed=True),
        attention("bwd", "bwd_bf16_capped", BF16, 4096, 32, 8, 128, "1531 64 700 1289 300 150", prefix="256 64 0 0 100 0", softcap=50.0),
        attention("bwd", "bwd_f16_bias_short", F16, 4000, 16, 16, 64, "333 80 512 17 250 61 400 129 200 350 90 611 5 400 262 300",
                  slopes=True, packed=True),
        attention("bwd", "bwd_f32_all", F32, 1000, 8, 2, 64, "400 7 350 200", prefix="100 0 350 13", softcap=30.0, slopes=True),
    ]


def log_int(rng, lo, hi, multiple=1):
    """A whole number between lo and hi, spread over the logarithm, a multiple of `multiple`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["rope", "fwd", "fwd", "bwd", "bwd"])
        dtype = rng.choice([F32, BF16, BF16, F16])
        nkv = log_int(rng, 1, 8)
        nh = nkv * rng.choice([1, 1, 2, 4])
        d = rng.choice([64, 80, 96, 128, 128])
        packed = rng.random() < 0.5
        if kind == "rope":
            axes = rng.randint(1, 3)
            cuts = sorted(rng.randint(1, d // 2 - 1) for _ in range(axes - 1))
            sections = [b - a for a, b in zip([0] + cuts, cuts + [d // 2])]
            return rope(None, dtype, log_int(rng, 64, 9000), nh, nkv, d, " ".join(map(str, sections)), rng.random() < 0.5,
                        log_int(rng, 1, 200000), rng.choice([1, -1]), packed)
        T = log_int(rng, 64, 1024 if dtype == F32 else 6000)
        left, lengths = T - rng.choice([0, 0, rng.randint(0, T // 4)]), []
        mean = log_int(rng, 32, 4096)
        while left > 0:
            lengths.append(min(left, 1 + int(rng.expovariate(1.0 / mean))))
            left -= lengths[-1]
        prefix = [rng.randint(0, n) for n in lengths] if rng.random() < 0.3 else []
        c = attention(kind, None, dtype, T, nh, nkv, d, " ".join(map(str, lengths)), " ".join(map(str, prefix)),
                      rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.4, packed)
        if work(c)["flops"] <= (2e10 if dtype == F32 else most):
            return c


def ints(text):
    return [int(x) for x in text.split()]


def scale_of(c):
    return float(torch.tensor(1.0 / math.sqrt(c["d"]), dtype=torch.float32))


# ---------------------------------------------------------------------------------------------- inputs
class Draw:
    """Normal deviates on the GPU from one seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, shape, std, dtype):
        return (torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32) * std).to(dtype)

    def whole(self, top):
        return int(torch.randint(0, top, (1,), generator=self.g, device="cuda"))


def heads(c, r):
    """q [T, nh*d] and k, v [T, nkv*d]: columns of one buffer, or three buffers."""
    T, Q, K, dt = c["T"], c["nh"] * c["d"], c["nkv"] * c["d"], TORCH[c["dtype"]]
    if c["packed"]:
        qkv = r.normal((T, Q + 2 * K), 1.0, dt)
        return qkv[:, :Q], qkv[:, Q:Q + K], qkv[:, Q + K:]
    return r.normal((T, Q), 1.0, dt), r.normal((T, K), 1.0, dt), r.normal((T, K), 1.0, dt)


def positions(c, r):
    """int32 [axes, T]: the cells of a grid in their order, width changing fastest; one axis: text.  The grid's origin is the seed's."""
    axes, T = len(ints(c["sections"])), c["T"]
    t = torch.arange(T, device="cuda", dtype=torch.int64)
    first = c["start"] + r.whole(64)
    width, height = 24, 20
    rows = {1: [t + first], 2: [t // width + first, t % width], 3: [t // (width * height) + first, t // width % height, t % width]}[axes]
    return torch.stack(rows).to(torch.int32)


def inputs(c, seed):
    r = Draw(seed)
    s = SimpleNamespace(c=c)
    s.q, s.k, s.v = heads(c, r)
    if c["kind"] == "rope":
        s.positions = positions(c, r)
        return s
    lengths, prefix = ints(c["lengths"]), ints(c["prefix"])
    s.offsets = torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")
    s.prefix = torch.tensor(prefix, dtype=torch.int32, device="cuda") if prefix else None
    nh = c["nh"]
    s.slopes = (2.0 ** (-8.0 * torch.arange(1, nh + 1, device="cuda", dtype=torch.float32) / nh)) if c["slopes"] else None
    if c["kind"] == "bwd":   # what the forward pass left: its result in the tensors' type, and the rows' logarithms
        s.dout = r.normal((c["T"], nh * c["d"]), 1e-2 * (256.0 if c["dtype"] == F16 else 1.0), TORCH[c["dtype"]])
        s.o, s.lse = plain_fwd(s)
    return s


def prepare(case, seed):
    s = inputs(case, seed)
    c, dt = s.c, TORCH[case["dtype"]]
    T, Q, K = c["T"], c["nh"] * c["d"], c["nkv"] * c["d"]
    if not own:
        return s
    import paper_2507_10392_amd as zs
    s.zs = zs
    empty = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device="cuda")
    if c["kind"] == "rope":
        s.q_out, s.k_out = empty(T, Q), empty(T, K)
        return s
    # The documents' ranges are a table that a program makes once per microbatch and keeps for all layers, forward and backward.
    s.ranges = empty(T, 4, dtype=torch.int32)
    zs.ops.doc_ranges(torch.cuda.current_stream().cuda_stream, T, len(ints(c["lengths"])), s.offsets, s.prefix, s.ranges)
    if c["kind"] == "fwd":
        s.o, s.lse = empty(T, Q), empty(c["nh"], T, dtype=torch.float32)
    else:
        s.dqkv = empty(T, Q + 2 * K)
        n = zs.attention_docs_bwd_scratch_bytes(c["dtype"], T, c["nh"], c["nkv"], c["d"])
        s.scratch = empty(n, dtype=torch.uint8)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return {"rope": own_rope, "fwd": own_fwd, "bwd": own_bwd}[state.c["kind"]](state)
    if state.c["kind"] == "rope":
        return plain_rope(state)
    if state.c["kind"] == "fwd":
        o, lse = plain_fwd(state)
        return {"o": o, "lse": lse}
    return plain_bwd(state)


def own_rope(s):
    c, st = s.c, torch.cuda.current_stream().cuda_stream
    s.zs.rope_axes(st, c["dtype"], c["T"], c["nh"], c["nkv"], c["d"], s.q, s.q.stride(0), s.k, s.k.stride(0), s.positions,
                   ints(c["sections"]), c["own_spectrum"], ROPE_BASE, c["sign"], s.q_out, s.q_out.stride(0), s.k_out, s.k_out.stride(0))
    return {"q": s.q_out, "k": s.k_out}


def own_fwd(s):
    c, st = s.c, torch.cuda.current_stream().cuda_stream
    s.zs.ops.attention_docs_fwd(st, c["dtype"], c["T"], c["nh"], c["nkv"], c["d"], s.q, s.q.stride(0), s.k, s.v, s.k.stride(0), s.ranges,
                                scale_of(c), c["softcap"], s.slopes, s.o, s.o.stride(0), s.lse)
    return {"o": s.o, "lse": s.lse}


def own_bwd(s):
    c, st = s.c, torch.cuda.current_stream().cuda_stream
    Q, K = c["nh"] * c["d"], c["nkv"] * c["d"]
    dq, dk, dv = s.dqkv[:, :Q], s.dqkv[:, Q:Q + K], s.dqkv[:, Q + K:]
    s.zs.ops.attention_docs_bwd(st, c["dtype"], c["T"], c["nh"], c["nkv"], c["d"], s.q, s.q.stride(0), s.k, s.v, s.k.stride(0), s.ranges,
                                scale_of(c), c["softcap"], s.slopes, s.o, s.dout, s.o.stride(0), s.lse, dq, dq.stride(0), dk, dv,
                                dk.stride(0), s.scratch, s.scratch.numel())
    return {"dq": dq, "dk": dk, "dv": dv}


def plain_rope(s):
    c = s.c
    sections, d = ints(c["sections"]), c["d"]
    freq, axis = [], []
    for a, n in enumerate(sections):
        first = sum(sections[:a])
        freq += [ROPE_BASE ** (-j / n) if c["own_spectrum"] else ROPE_BASE ** (-2.0 * (first + j) / d) for j in range(n)]
        axis += [a] * n
    angle = s.positions.double()[axis].t() * torch.tensor(freq, dtype=torch.float64, device="cuda") * c["sign"]
    cs, sn = angle.cos().float()[:, None], angle.sin().float()[:, None]
    out = []
    for x in (s.q, s.k):
        p = x.float().reshape(c["T"], -1, d // 2, 2)
        u, w = p[..., 0], p[..., 1]
        out.append(torch.stack((u * cs - w * sn, u * sn + w * cs), -1).reshape(c["T"], -1).to(x.dtype))
    return {"q": out[0], "k": out[1]}


def visible(s):
    """bool [T, T]: row i sees key j."""
    T = s.c["T"]
    t = torch.arange(T, device="cuda")
    doc = (s.offsets[None, 1:] <= t[:, None]).sum(1)
    n = s.offsets.numel() - 1
    inside = (t >= s.offsets[0]) & (doc < n)
    doc = doc.clamp(max=n - 1)
    sees = t[None, :] <= t[:, None]
    if s.prefix is not None:
        sees = sees | (t < s.offsets[doc] + s.prefix[doc])[None, :]
    return sees & (doc[None, :] == doc[:, None]) & inside[None, :] & inside[:, None]


def head_groups(c):
    """Slices of the key heads whose score matrices are worked on at a time: about 2^28 scores."""
    step = max(1, min(c["nkv"], (1 << 28) // (c["T"] * c["T"] * (c["nh"] // c["nkv"]))))
    return [slice(i, min(i + step, c["nkv"])) for i in range(0, c["nkv"], step)]


def split(s, x, n):
    """[T, n*d] -> float [n, T, d]."""
    return x.float().reshape(s.c["T"], n, s.c["d"]).transpose(0, 1).contiguous()


def plain_scores(s, q, k, group, h0):
    """Capped and biased scores [heads, T, T] of the key heads k, and what the cap's derivative needs."""
    c = s.c
    z = torch.matmul(q, k.repeat_interleave(group, 0).transpose(1, 2).contiguous()) * scale_of(c)
    t = None
    if c["softcap"] > 0:
        t = torch.tanh(z / c["softcap"])
        z = c["softcap"] * t
    if s.slopes is not None:
        at = torch.arange(c["T"], device="cuda", dtype=torch.float32)
        z = z - s.slopes[h0:h0 + z.shape[0], None, None] * (at[:, None] - at[None, :]).abs()
    return z, t


def plain_fwd(s):
    c = s.c
    T, nh, group = c["T"], c["nh"], c["nh"] // c["nkv"]
    sees = visible(s)
    empty = ~sees.any(1)
    q, k, v = split(s, s.q, nh), split(s, s.k, c["nkv"]), split(s, s.v, c["nkv"])
    o, lse = torch.empty(nh, T, c["d"], device="cuda"), torch.empty(nh, T, device="cuda")
    for g in head_groups(c):
        h = slice(g.start * group, g.stop * group)
        z, _ = plain_scores(s, q[h], k[g], group, h.start)
        z = torch.where(sees, z, -math.inf)
        m = torch.where(empty, 0.0, z.max(-1).values)
        p = torch.exp(z - m[..., None])
        l = p.sum(-1)
        o[h] = torch.matmul(p, v[g].repeat_interleave(group, 0)) / torch.where(empty, 1.0, l)[..., None]
        lse[h] = m + torch.log(l)
    return o.transpose(0, 1).reshape(T, -1).to(s.q.dtype), lse


def plain_bwd(s):
    c = s.c
    T, nh, nkv, d, group = c["T"], c["nh"], c["nkv"], c["d"], c["nh"] // c["nkv"]
    sees = visible(s)
    q, k, v = split(s, s.q, nh), split(s, s.k, nkv), split(s, s.v, nkv)
    o, dout = split(s, s.o, nh), split(s, s.dout, nh)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    for g in head_groups(c):
        h = slice(g.start * group, g.stop * group)
        z, t = plain_scores(s, q[h], k[g], group, h.start)
        p = torch.where(sees, torch.exp(z - s.lse[h][..., None]), 0.0)
        dp = torch.matmul(dout[h], v[g].repeat_interleave(group, 0).transpose(1, 2).contiguous())
        ds = p * (dp - (dout[h] * o[h]).sum(-1, keepdim=True))
        if t is not None:
            ds = ds * (1 - t * t)
        ds = ds * scale_of(c)
        dq[h] = torch.matmul(ds, k[g].repeat_interleave(group, 0))
        dk[g] = torch.matmul(ds.transpose(1, 2).contiguous(), q[h]).reshape(-1, group, T, d).sum(1)
        dv[g] = torch.matmul(p.transpose(1, 2).contiguous(), dout[h]).reshape(-1, group, T, d).sum(1)
    return {n: x.transpose(0, 1).reshape(T, -1).to(s.q.dtype) for n, x in (("dq", dq), ("dk", dk), ("dv", dv))}


# ---------------------------------------------------------------------------------------------- work
def pairs(c):
    """Pairs of a row and a key that it sees, in one head."""
    prefix = ints(c["prefix"]) or [0] * len(ints(c["lengths"]))
    return sum(n * (n + 1) // 2 + min(p, n) * (min(p, n) - 1) // 2 for n, p in zip(ints(c["lengths"]), prefix))


def work(c):
    E, T, Q, K = BYTES[c["dtype"]], c["T"], c["nh"] * c["d"], c["nkv"] * c["d"]
    if c["kind"] == "rope":
        return {"bytes": 2 * E * T * (Q + K) + 4 * T * len(ints(c["sections"])), "flops": 3 * T * (Q + K)}
    stats = 4 * c["nh"] * T
    if c["kind"] == "fwd":
        return {"bytes": E * T * (2 * Q + 2 * K) + stats, "flops": 4 * pairs(c) * Q}
    return {"bytes": E * T * (4 * Q + 4 * K) + stats, "flops": 10 * pairs(c) * Q}   # five products; the scores are not kept


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = inputs(case, seed)
    return exact_rope(s) if case["kind"] == "rope" else exact_attention(s)


def exact_rope(s):
    """Every pair as a complex number, turned by exp(i * angle)."""
    c = s.c
    sections, d = ints(c["sections"]), c["d"]
    turn, i = [], 0
    for a, n in enumerate(sections):
        for j in range(n):
            exponent = 2.0 * j / (2 * n) if c["own_spectrum"] else 2.0 * i / d
            turn.append(s.positions[a].double() * math.exp(-exponent * math.log(ROPE_BASE)))
            i += 1
    angle = c["sign"] * torch.stack(turn, 1)
    factor = torch.complex(angle.cos(), angle.sin())[:, None, :]
    res = {}
    for name, x in (("q", s.q), ("k", s.k)):
        z = torch.view_as_complex(x.double().reshape(c["T"], -1, d // 2, 2).contiguous())
        res[name] = torch.view_as_real(z * factor).reshape(c["T"], -1)
    return res


def exact_attention(s):
    """Head after head and document after document; the gradients from the formulas with the saved rows that the call gets."""
    c = s.c
    T, nh, nkv, d = c["T"], c["nh"], c["nkv"], c["d"]
    lengths = ints(c["lengths"])
    prefix = ints(c["prefix"]) or [0] * len(lengths)
    new = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")
    bwd = c["kind"] == "bwd"
    o, lse = new(T, nh, d), torch.full((nh, T), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = new(T, nh, d), new(T, nkv, d), new(T, nkv, d)
    Q, K, V = (x.double().reshape(T, -1, d) for x in (s.q, s.k, s.v))
    first = 0
    for n, pre in zip(lengths, prefix):
        rows = slice(first, first + n)
        first += n
        at = torch.arange(n, device="cuda")
        hidden = (at[None, :] > at[:, None]) & (at[None, :] >= pre)
        far = (at[None, :] - at[:, None]).abs().double()
        for h in range(nh):
            kv = h // (nh // nkv)
            q, k, v = Q[rows, h], K[rows, kv], V[rows, kv]
            z = scale_of(c) * (q @ k.t())
            slope = torch.ones_like(z)
            if c["softcap"] > 0:
                slope = 1 / torch.cosh(z / c["softcap"]).square()
                z = c["softcap"] * torch.tanh(z / c["softcap"])
            if s.slopes is not None:
                z = z - s.slopes[h].double() * far
            z = z.masked_fill(hidden, -math.inf)
            if not bwd:
                lse[h, rows] = torch.logsumexp(z, -1)
                o[rows, h] = torch.softmax(z, -1) @ v
                continue
            do = s.dout.reshape(T, nh, d)[rows, h].double()
            p = torch.exp(z - s.lse[h, rows].double()[:, None])
            delta = (do * s.o.reshape(T, nh, d)[rows, h].double()).sum(1)
            dz = p * (do @ v.t() - delta[:, None]) * slope * scale_of(c)
            dq[rows, h] = dz @ k
            dk[rows, kv] += dz.t() @ q
            dv[rows, kv] += p.t() @ do
    if bwd:
        return {"dq": dq.reshape(T, -1), "dk": dk.reshape(T, -1), "dv": dv.reshape(T, -1)}
    return {"o": o.reshape(T, -1), "lse": lse}
