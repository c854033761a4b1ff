"""Exact attention of one sequence in 64 bits, with the error that the types
allow, element by element.

Half a step of rounding is u = eps / 2 relative: 2^-8 (bf16), 2^-11 (fp16),
2^-24 (fp32).  What a kernel that works in fp32 and rounds the weights P and
dS to the element type may be off by:

  O      u |O| + (u + e) A                     A = P |V|
  delta  D = sum_c |dO_c| (u |O_c| + (u + e) A_c)      (delta = sum_c dO_c O_c)
  dS     u |dS| + e P (|dP| + |delta|) + P D
  dQ     u |dQ| + s E |K|                      E: the error of dS, row by row
  dK     u |dK| + s E^T |Q|
  dV     u |dV| + (u + e) P^T |dO|

(fp32 does not round P and dS: u is 0 there inside the sums).  e is the fp32
arithmetic: a score is a sum of d products, whose rounding errors shift it by
at most (d + 4) 2^-24 s |q|.|k|, which is the relative error of its weight; a
sum over n terms adds n 2^-24 of the sum of their magnitudes; exp2 and the
reciprocal add a few steps.  Both are worst cases and every factor is applied
once, not squared.
"""
import math

import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def attention(q, k, v, causal, shift=0, g=None):
    """q [n, Hq, d], k, v [L, Hkv, d] of one sequence; row i sees keys 0..i + shift
    (all, if not causal).  Returns {name: (value, bound)} of out, lse and, with
    g = dL/dout, of dq, dk, dv, in float64."""
    dtype = q.dtype
    u = torch.finfo(dtype).eps / 2
    w = 0.0 if dtype == torch.float32 else u
    n, Hq, d = q.shape
    L, Hkv, _ = k.shape
    G, s = Hq // Hkv, 1.0 / math.sqrt(d)
    q, k, v = q.double(), k.double(), v.double()
    res = {"out": torch.zeros_like(q), "lse": torch.full((Hq, n), -math.inf, dtype=torch.float64, device=q.device)}
    tol = {"out": torch.zeros_like(q), "lse": torch.zeros_like(res["lse"])}
    if g is not None:
        g = g.double()
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            res[name], tol[name] = torch.zeros_like(like), torch.zeros_like(like)
    see = torch.ones(n, L, dtype=torch.bool, device=q.device)
    if causal:
        see = torch.arange(L, device=q.device)[None] <= torch.arange(n, device=q.device)[:, None] + shift
    some = see.any(1)
    for h in range(Hq if L else 0):
        qh, kh, vh = q[:, h], k[:, h // G], v[:, h // G]
        sc = torch.where(see, s * qh @ kh.T, -math.inf)
        lse = torch.logsumexp(sc, 1)
        p = torch.where(some[:, None], torch.exp(sc - torch.where(some, lse, 0.0)[:, None]), 0.0)
        size = torch.where(see, s * qh.abs() @ kh.abs().T, 0.0).amax(1)  # s |q|.|k|
        e = ((d + 4) * size + L + 16)[:, None] * 2.0 ** -24
        A = p @ vh.abs()
        o = p @ vh
        res["out"][:, h], tol["out"][:, h] = o, u * o.abs() + (w + e) * A
        res["lse"][h], tol["lse"][h] = lse, e[:, 0] + 2.0 ** -22 * torch.where(some, lse, 0.0).abs()
        if g is None:
            continue
        gh = g[:, h]
        dp = gh @ vh.T
        delta = (gh * o).sum(1, keepdim=True)
        D = (gh.abs() * (u * o.abs() + (w + e) * A)).sum(1, keepdim=True) + (d * 2.0 ** -24) * (gh * o).abs().sum(1, keepdim=True)
        dp_size = gh.abs() @ vh.abs().T  # dP is a sum of d products
        ds = p * (dp - delta)
        E = w * ds.abs() + p * (e * (dp.abs() + delta.abs()) + D + (d * 2.0 ** -24) * dp_size)
        sums = n * 2.0 ** -24
        x = s * ds @ kh
        res["dq"][:, h], tol["dq"][:, h] = x, u * x.abs() + s * (E + sums * ds.abs()) @ kh.abs()
        res["dk"][:, h // G] += s * ds.T @ qh
        tol["dk"][:, h // G] += s * (E + sums * ds.abs()).T @ qh.abs()
        res["dv"][:, h // G] += p.T @ gh
        tol["dv"][:, h // G] += ((w + e + sums) * p).T @ gh.abs()
    if g is not None:
        for name in ("dk", "dv"):
            tol[name] += u * res[name].abs()
    tiny = torch.finfo(dtype).smallest_normal * u  # half a step of the numbers below the normal ones
    return {x: (res[x], tol[x] + (tiny if x != "lse" else 0.0)) for x in res}


def worst(got, want, bound):
    """The largest error in units of its bound (inf where one side is finite and the other is not)."""
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, 0.0, (got - want).abs() / bound.clamp(min=1e-300))
    off = torch.where(torch.isnan(off), math.inf, off)
    return float(off.max()) if off.numel() else 0.0


def starts(lens, device, first=0):
    return torch.tensor([first] + list(lens), device=device).cumsum(0).to(torch.int32)
