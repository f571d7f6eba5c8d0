"""Rotary positions with several axes (stage_op_rope_axes) against complex numbers in 64 bits, and a layer's attention over packed tokens as a
whole: rotation, attention inside the documents, its gradient and the rotation back."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import docs_reference as ref
import paper_2507_10392_amd as zs
from docs_reference import TD
from test_attention_docs import Run

gpu = pytest.mark.gpu
# (T, nq, nk, d, sections, own spectrum)
CASES = [(1, 1, 0, 8, [4], 0), (3, 1, 1, 8, [0, 4], 1), (64, 4, 4, 64, [32], 0), (77, 5, 1, 80, [10, 15, 15], 0), (256, 4, 2, 128, [16, 24, 24], 0),
         (301, 3, 3, 96, [24, 24], 1), (1030, 2, 1, 256, [128], 0), (2100, 8, 1, 40, [4, 0, 6, 10], 1), (9000, 1, 2, 128, [20, 22, 22], 1)]


def spectrum(d, sections, own, base):
    f, axis = [], []
    for a, n in enumerate(sections):
        for j in range(n):
            f.append(base ** -(j / n if own else 2.0 * len(f) / d))
            axis.append(a)
    return torch.tensor(f, dtype=torch.float64), axis


def rotated(x, positions, d, sections, own, base, sign):
    """float64 [T, n*d]."""
    f, axis = spectrum(d, sections, own, base)
    angle = sign * positions.double()[axis].t() * f
    z = torch.view_as_complex(x.reshape(x.shape[0], -1, d // 2, 2).contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.view_as_real(z).reshape(x.shape)


def bound(x, want, dtype, angle_error):
    """Half a step of the type, four roundings of the pair's products in fp32, and the pair's length times the angle's error."""
    pair = x.reshape(x.shape[0], -1, 2).norm(dim=-1).repeat_interleave(2, -1)
    return torch.finfo(TD[dtype]).eps / 2 * want.abs() * 1.01 + pair * (6 * 2.0 ** -24 + angle_error) + (2.0 ** -25 if dtype == 2 else 1e-38)


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_matches_64_bits(gpu_device, case, dtype):
    T, nq, nk, d, sections, own = case
    print("[case]", case, dtype, flush=True)
    rng = np.random.default_rng(T + d)
    base = 10000.0
    pos = torch.from_numpy(rng.integers(-300, 200000, (len(sections), T)).astype(np.int32))
    pad = 4 if dtype == 0 else 8
    q, k = ref.draw(rng, (T, nq * d), dtype), ref.draw(rng, (T, nk * d), dtype)
    both = torch.cat([q, k, torch.zeros(T, pad).double()], 1).to(TD[dtype]).cuda()
    gq, gk = both[:, :nq * d], both[:, nq * d:(nq + nk) * d] if nk else None
    out = torch.full((T, (nq + nk) * d + pad), math.nan, dtype=TD[dtype], device="cuda")
    oq, ok = out[:, :nq * d], out[:, nq * d:(nq + nk) * d] if nk else None
    st = torch.cuda.current_stream().cuda_stream
    for sign in (1, -1):
        zs.rope_axes(st, dtype, T, nq, nk, d, gq, both.stride(0), gk, both.stride(0), pos.cuda(), sections, own, base, sign, oq, out.stride(0), ok,
                     out.stride(0))
        for x, got in ((q, oq),) + (((k, ok),) if nk else ()):
            want = rotated(x, pos, d, sections, own, base, sign)
            ref.within(got, want, bound(x, want, dtype, 4 * 2.0 ** -24), "sign %d" % sign)
        assert out[:, -pad:].isnan().all()
    first = out.clone()
    zs.rope_axes(st, dtype, T, nq, nk, d, gq, both.stride(0), gk, both.stride(0), pos.cuda(), sections, own, base, -1, gq, both.stride(0), gk,
                 both.stride(0))                                                 # in place: the same bits
    assert torch.equal(both[:, :-pad], first[:, :-pad])


@gpu
def test_far_positions(gpu_device):
    """Positions up to the ends of their type: the angle stays good to 2^-20."""
    T, d = 64, 128
    rng = np.random.default_rng(1)
    pos = torch.from_numpy(rng.integers(-2**31, 2**31, (2, T)).astype(np.int32))
    q = ref.draw(rng, (T, d), 0)
    out = torch.empty(T, d, device="cuda")
    zs.rope_axes(torch.cuda.current_stream().cuda_stream, 0, T, 1, 0, d, q.float().cuda(), d, None, 0, pos.cuda(), [30, 34], 0, 500000.0, 1, out, d, None, 0)
    f, axis = spectrum(d, [30, 34], 0, 500000.0)
    want = rotated(q, pos, d, [30, 34], 0, 500000.0, 1)
    # 64 bits on this side too: a frequency's and a product's rounding, 2^-53 of up to 2^31, on both sides
    ref.within(out, want, bound(q, want, 0, 2.0 ** -20), "far")


@gpu
def test_one_axis_is_the_rotation_of_the_stage(gpu_device):
    """Positions 0 .. T-1 on one axis: what stage_op_rope does, up to the rounding of its table."""
    T, n, d = 200, 3, 64
    rng = np.random.default_rng(2)
    x = ref.draw(rng, (T, n * d), 0).float().cuda()
    y, table, out = x.clone(), torch.empty(T, d // 2, 2, device="cuda"), torch.empty_like(x)
    st = torch.cuda.current_stream().cuda_stream
    zs.ops.rope(st, 0, T, T, n * d, d, y, n * d, 10000.0, 1.0, table)
    zs.rope_axes(st, 0, T, n, 0, d, x, n * d, None, 0, torch.arange(T, dtype=torch.int32, device="cuda")[None], [d // 2], 0, 10000.0, 1, out, n * d, None, 0)
    want = y.double().cpu()
    ref.within(out, want, 2 * bound(x.double().cpu(), want, 0, 4 * 2.0 ** -24), "stage")


@gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_a_layer_over_packed_tokens(gpu_device, dtype):
    """q, k turned by (time, height, width) positions that begin anew in every document, attention with a bidirectional prefix, capped
    scores and shared key heads, its gradient, and the gradients of the unrotated q and k, against automatic differentiation in 64 bits."""
    c = ref.Case(260, 4, 2, 64, [120, 9, 111], prefix=[40, 0, 111], softcap=20.0)
    sections, base = [8, 12, 12], 10000.0
    r = Run(c, dtype)
    at = np.concatenate([np.arange(n) for n in c.lengths] + [np.zeros(c.T - sum(c.lengths), int)])
    pos = torch.from_numpy(np.stack([at // 30, at // 6 % 5, at % 6]).astype(np.int32))
    st, gpos = torch.cuda.current_stream().cuda_stream, pos.cuda()

    def turn(q, k, sign):
        zs.rope_axes(st, dtype, c.T, c.nh, c.nkv, c.d, q, q.stride(0), k, k.stride(0), gpos, sections, 0, base, sign, q, q.stride(0), k, k.stride(0))

    turn(r.gq, r.gk, 1)
    r.find()
    r.fwd()
    r.bwd()
    turn(r.dq, r.dk, -1)
    torch.cuda.synchronize()
    q, k, v = (x.clone().requires_grad_() for x in (r.q, r.k, r.v))
    o, lse = ref.forward(c, rotated(q, pos, c.d, sections, 0, base, 1), rotated(k, pos, c.d, sections, 0, base, 1), v)
    (o * r.dout).sum().backward()
    # roundings to the type on the way to a gradient: q, k, o, P, dS, the gradient and its rotation, a norm-wise half step each, of which none
    # is amplified by more than the scores' size (about 4): 8 x 4 half steps of the norm are never reached
    u = torch.finfo(TD[dtype]).eps / 2
    for name, got, want in (("o", r.go, o.detach()), ("dq", r.dq, q.grad), ("dk", r.dk, k.grad), ("dv", r.dv, v.grad)):
        err = (got.double().cpu() - want).norm() / want.norm()
        assert err <= 32 * u, (name, float(err))


# ---------------------------------------------------------------------------------------------- no GPU
def code(**change):
    a = dict(dict(dtype=1, T=4, nq=2, nk=1, d=64, q=4096, ldq=128, k=4096, ldk=64, positions=4096, sections=[12, 20], own=0, base=10000.0, sign=1,
                  qo=4096, ldqo=128, ko=4096, ldko=64, naxes=None), **change)
    s = None if a["sections"] is None else (C.c_int32 * max(1, len(a["sections"])))(*a["sections"])
    n = a["naxes"] if a["naxes"] is not None else len(a["sections"] or [])
    return zs.lib().stage_op_rope_axes(None, a["dtype"], a["T"], a["nq"], a["nk"], a["d"], a["q"], a["ldq"], a["k"], a["ldk"], a["positions"], n, s,
                                       a["own"], a["base"], a["sign"], a["qo"], a["ldqo"], a["ko"], a["ldko"])


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(T=-1), dict(nq=0), dict(nk=-1), dict(d=60), dict(d=0), dict(d=264, sections=[132]), dict(q=None),
                                 dict(k=None), dict(qo=None), dict(ko=None), dict(positions=None), dict(positions=4098), dict(q=4104), dict(k=4104),
                                 dict(qo=4098), dict(ko=4104), dict(ldq=120), dict(ldk=60), dict(ldqo=130), dict(ldko=56), dict(sections=[12, 21]),
                                 dict(sections=[-1, 33]), dict(sections=[]), dict(sections=[8, 8, 8, 4, 4]), dict(sections=None, naxes=1),
                                 dict(base=0.0), dict(base=-1.0), dict(base=math.nan), dict(base=math.inf), dict(sign=0), dict(sign=2), dict(T=(1 << 26) + 1)], ids=str)
def test_refusals(bad):
    assert code(**bad) == zs.STAGE_ERR_ARG


def test_no_tokens():
    assert code(T=0, q=None, k=None, qo=None, ko=None, positions=None) == zs.STAGE_OK and code(T=0, sections=[3]) == zs.STAGE_ERR_ARG
    assert code(T=0) == zs.STAGE_OK and code(T=0, nk=0, k=None, ko=None) == zs.STAGE_OK
