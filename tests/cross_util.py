"""Cross attention of a pack from its definition, in 64 bits, with element-wise bounds for bf16 kernels."""
import math

import torch

HALF = 2.0 ** -8   # half a step of bf16, relative
F32 = 2.0 ** -24


def inputs(ql, kl, hq, hkv, d, e, seed, sigma=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *shape: (torch.randn(shape, generator=g, device="cuda") * sigma).to(torch.bfloat16)  # noqa: E731
    return new(sum(ql), hq, d), new(sum(kl), hkv, d), new(sum(kl), hkv, e), new(sum(ql), hq, e)


def exact(ql, kl, q, k, v, d_o, scale=None):
    """{name: (value, bound)} of O, LSE, dQ, dK, dV.  Bounds, with A = sum_k P |V| >= |O|:
      probabilities are fp32 up to `p` (the scores' fp32 sums, exp2 and the fp32 LSE), rounded to bf16 in front of the products;
      O    (half a step of P and of O): (2 HALF + p) A
      D    = sum dO O of the stored O:  sum |dO| bound(O)
      dS   rounded to bf16: HALF |dS| + P bound(D) + p (|dS| + P (|dO||V| + |D|)), P |dO||V| with fp32 sums of dP
      dQ, dK: scale * bound(dS) through the products, and half a step of themselves; dV: (2 HALF + p) sum P |dO|"""
    hq, d, hkv, e = q.shape[1], q.shape[2], k.shape[1], v.shape[2]
    c, g = scale or 1 / math.sqrt(d), hq // hkv
    out = {n: [torch.zeros(s, dtype=torch.float64, device="cuda") for _ in range(2)] for n, s in
           (("o", d_o.shape), ("lse", (hq, q.shape[0])), ("dq", q.shape), ("dk", k.shape), ("dv", v.shape))}
    out["lse"][0].fill_(-math.inf)
    q0 = k0 = 0
    for a, b in zip(ql, kl):
        rows, cols = slice(q0, q0 + a), slice(k0, k0 + b)
        q0, k0 = q0 + a, k0 + b
        if a == 0 or b == 0:
            continue
        for h in range(hq):
            Q, K, V, dO = (x.double() for x in (q[rows, h], k[cols, h // g], v[cols, h // g], d_o[rows, h]))
            S = c * Q @ K.t()
            size = float((c * Q.abs() @ K.abs().t()).max())
            p = 4 * (d + 8) * F32 * size + 1e-6
            lse = torch.logsumexp(S, 1)
            P = torch.exp(S - lse[:, None])
            O, A = P @ V, P @ V.abs()
            D = (dO * O).sum(1, keepdim=True)
            bO = (2 * HALF + HALF ** 2 + p) * A + 1e-30
            bD = (dO.abs() * bO).sum(1, keepdim=True) + 2 * e * F32 * (dO.abs() * A).sum(1, keepdim=True)
            dP, dPa = dO @ V.t(), dO.abs() @ V.abs().t()
            dS = P * (dP - D)
            bS = HALF * (dS.abs() + P * bD) + P * bD + p * (P * (dPa + D.abs())) + 2 * e * F32 * P * dPa
            half = lambda x, bx: bx + HALF * (x.abs() + bx) + 1e-30  # noqa: E731
            out["o"][0][rows, h], out["o"][1][rows, h] = O, bO
            out["lse"][0][h, rows] = lse
            out["lse"][1][h, rows] = 2 * (d + 8) * F32 * size + 4 * F32 * lse.abs() + (b ** 0.5 + 8) * F32
            out["dq"][0][rows, h], out["dq"][1][rows, h] = c * dS @ K, half(c * dS @ K, c * bS @ K.abs())
            out["dk"][0][cols, h // g] += c * dS.t() @ Q
            out["dk"][1][cols, h // g] += c * bS.t() @ Q.abs()
            out["dv"][0][cols, h // g] += P.t() @ dO
            out["dv"][1][cols, h // g] += (HALF + p) * (P.t() @ dO.abs())
    for n in ("dk", "dv"):
        x, bx = out[n]
        out[n][1] = bx + HALF * (x.abs() + bx) + 1e-30
    return out


def check(got, want, names):
    for n in names:
        value, bound = want[n]
        x = got[n].double()
        none = torch.isinf(value)
        assert torch.equal(none, torch.isinf(x)) and bool((x[none] < 0).all()), n
        err = torch.where(none, torch.zeros_like(x), (x - value).abs())
        err[none] = 0
        assert bool((err <= bound).all()), (n, float((err / bound.clamp_min(1e-300)).max()))
        both = torch.nan_to_num(value, neginf=0.0).norm()
        if float(both) > 0 and n != "lse":
            print("  %s rel 2-norm %.2e, largest error / bound %.2f" % (n, float((x - value)[~none].norm() / both), float((err / bound.clamp_min(1e-300)).max())))
