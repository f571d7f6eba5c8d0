"""The chunked form of the gated delta rule and of its gradient in 64 bits, with operands held as a kernel would hold them, and how far results of
such a kernel may be off.

Bounds, as root mean squares over many values, relative to the 2-norm of a product's terms.  A half pair leaves up to 2^-23 of a value (11 bits, and 11 of what
these leave), 0.31 2^-23 as a mean; two of them drop a product of (2^-11)^2 / 3, 0.33 2^-23 of the values'; fp32 sums of 128 terms, 32 to an instruction, three
products, are twelve roundings of 2^-24 / sqrt(3): 2^-23.  Together 1.14 2^-23; with a quarter for chance, 2^-22.5.  fp32 products and three bf16
terms are off by less.  A state goes, per chunk, through ten results of this kind: K K^T, four levels of the inverse, two decays, K S, T Z and K^T U.  Their
errors have no common sign: sqrt(10 n) 2^-22.5 of its norm over n chunks.  STATE(n) is that; the gradient's walk, which also takes P, adds as many again for
results that need both walks, sqrt(2) STATE(n).

dg and dbeta are sums whose terms cancel: the same share, of the 2-norm of the terms that a value is the sum of, which the 64-bit form gives: for
dg a token's terms and those of all tokens behind it in its chunk, which are summed."""
import math

import torch

CHUNK = 64
STATE = lambda n: math.sqrt(10 * n) * 2.0 ** -22.5


def pairs(dtype, terms):
    """x as the sum of so many values of the type; half: times a power of two per column that brings its largest to 2^13 .. 2^14."""
    def hold(x):
        unit = 1.0
        if dtype == torch.float16:
            most = x.abs().amax(-2, keepdim=True).clamp(min=1e-30)
            unit = torch.exp2(13 - torch.floor(torch.log2(most)))
        y, out = x * unit, torch.zeros_like(x)
        for _ in range(terms):
            part = (y - out).to(dtype).double()
            out = out + part
        return out / unit
    return hold


def exact(x):
    return x


def chunked(c, x, walk=exact, grad=exact):
    """-> ht, dg, dbeta, dh0, and the 2-norms of the terms of dg and dbeta.  walk: what holds the operands of both walks; grad: those of a chunk's gradients."""
    group, heads = c.nv // c.nk, range(c.nv)
    ht, dh0 = torch.zeros(len(c.lengths), c.nv, c.dk, c.dv, dtype=torch.float64), torch.zeros(len(c.lengths), c.nv, c.dk, c.dv, dtype=torch.float64)
    dg, dbeta, tg, tb = (torch.zeros(c.T, c.nv, dtype=torch.float64) for _ in range(4))
    for d, length in enumerate(c.lengths):
        for h in heads:
            S = torch.zeros(c.dk, c.dv, dtype=torch.float64) if x["h0"] is None else x["h0"][d, h]
            kept = []
            for t0 in range(c.offsets[d], c.offsets[d + 1], CHUNK):
                r = slice(t0, min(t0 + CHUNK, c.offsets[d + 1]))
                K, Q, V, beta = x["k"][r, h // group], x["q"][r, h // group], x["v"][r, h], x["beta"][r, h][:, None]
                G = x["g"][r, h].cumsum(0)
                D = torch.exp((G[:, None] - G[None]).tril()).tril()
                inverse = torch.linalg.inv(torch.eye(len(G), dtype=torch.float64) + (beta * (K @ K.t()) * D).tril(-1))
                since, until, whole = torch.exp(G)[:, None], torch.exp(G[-1] - G)[:, None], torch.exp(G[-1])
                U = walk(inverse) @ walk(beta * (V - since * (K @ walk(S))))
                kept.append((r, K, Q, V, beta, D, inverse, since, until, whole, S, U))
                S = whole * S + K.t() @ walk(until * U)
            ht[d, h] = S
            dS = torch.zeros(c.dk, c.dv, dtype=torch.float64) if x["dht"] is None else x["dht"][d, h]
            for r, K, Q, V, beta, D, inverse, since, until, whole, S, U in reversed(kept):
                dO = x["dout"][r, h]
                Y = walk(inverse).t() @ walk(c.scale * walk((Q @ K.t()) * D).t() @ dO + until * (K @ walk(dS)))
                gS, gdS, gU, gY = grad(S), grad(dS), grad(U), grad(Y)
                m, a = c.scale * D * (dO @ gU.t()), -(gY @ gU.t()).tril(-1) * D
                kk = K @ K.t()
                e = m * (Q @ K.t()) + beta * a * kk
                q_state, k_state, k_next = c.scale * since * (dO @ gS.t()), -since * (gY @ gS.t()), until * (gU @ gdS.t())
                of_dG = [e, -e.t(), Q * q_state, beta * K * k_state, -K * k_next]   # a token's row of each
                last = torch.cat(((K * k_next).reshape(-1), whole * (S * dS).reshape(-1)))
                dG, squares = sum(t.sum(1) for t in of_dG), sum(t.square().sum(1) for t in of_dG)
                dG[-1] += last.sum()
                squares[-1] += last.square().sum()
                dg[r, h], tg[r, h] = dG.flip(0).cumsum(0).flip(0), squares.flip(0).cumsum(0).flip(0).sqrt()
                of_beta = [Y * V, K * k_state, a * kk]
                dbeta[r, h], tb[r, h] = sum(t.sum(1) for t in of_beta), sum(t.square().sum(1) for t in of_beta).sqrt()
                dS = whole * dS + Q.t() @ walk(c.scale * since * dO) - K.t() @ walk(beta * since * Y)
            dh0[d, h] = dS
    return {"ht": ht, "dg": dg, "dbeta": dbeta, "dh0": dh0}, {"dg": tg, "dbeta": tb}


def bounds(c, want, terms):
    """Relative to a result's 2-norm."""
    n = max(1, -(-max(c.lengths) // CHUNK))
    both = math.sqrt(2) * STATE(n)
    return {"ht": STATE(n), "dh0": both, **{k: both * float(terms[k].norm() / want[k].norm()) for k in ("dg", "dbeta")}}


def off(got, want):
    return float((got.double().cpu().reshape(-1) - want.reshape(-1)).norm() / want.norm())
