"""Plain 64-bit forms of the training operators, and bounds of what rounding may
do to each output value.

Every bound counts roundings of at most u = eps / 2 of a type (bf16 2^-8, fp32
2^-24) through the formulas, element by element, with the sums of absolute
values that they act on:

  logit      fp32 sum of d_h products, scaled:   dt = (d_h + 8) u32 (scale |q|.|k| + |bias|)
  P          relative rp = 2 max_j dt + (n + 16) u32   (exponentials, sum, lse)
  out        (u_p + rp + n u32) P |v| + u |out|, u_p the rounding of P for the product (bf16 only)
  D          sum_f |dO| (bound of out) + d_h u32 |dO| |out|    (D is taken from the rounded out)
  dS         dds = P (D's bound + (rp + (d_h + 8) u32) (|dO||v| + |D|))
  dq, dk     scale (dds + u_p |dS| + n u32 |dS|) |k| (|q|) + u |value|
  dv         (u_p + rp + n u32) P^T |dO| + u |dv|
  drel       sum of dds over the bucket's pairs + pairs u32 |dS| + u |drel|; the last bucket is minus the sum of
             the others, whose bounds it inherits
"""
from __future__ import annotations

import math

import numpy as np
import torch

U32 = 2.0 ** -24


def unit(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def attention(q, k, v, groups, rel=None, scale=None, dout=None):
    """groups: list of (query rows, key rows, limits): index ranges (a, b), (c, d)
    and the number of visible keys of each query row (at most d - c). Causal
    bias of distance (row in group) - (key in group). Returns {name: (value,
    bound)} in float64 on the CPU; what a bound does not cover (a NaN) is NaN."""
    dt = q.dtype
    u = unit(dt)
    up = u if dt == torch.bfloat16 else 0.0
    Q, K, V = (x.detach().cpu().double() for x in (q, k, v))
    dO = dout.detach().cpu().double() if dout is not None else None
    M, H, dh = Q.shape
    N, G = K.shape[:2]
    sc = 1.0 / math.sqrt(dh) if scale is None else scale
    per = H // G
    z = lambda *s: torch.zeros(*s, dtype=torch.float64)
    out, out_b, lse, lse_b = z(M, H, dh), z(M, H, dh), torch.full((H, M), -math.inf, dtype=torch.float64), z(H, M)
    dq, dq_b, dk, dk_b, dv, dv_b = z(M, H, dh), z(M, H, dh), z(N, G, dh), z(N, G, dh), z(N, G, dh), z(N, G, dh)
    R = rel.shape[1] if rel is not None else 0
    drel, drel_b = z(H, max(R, 1)), z(H, max(R, 1))
    B = rel.detach().cpu().double() if rel is not None else None
    for (a, b), (c, d), lim in groups:
        n, m = b - a, d - c
        if n == 0 or m == 0:
            continue
        j = torch.arange(m)[None, :]
        seen0 = j < torch.as_tensor(lim)[:, None]
        dist = torch.arange(n)[:, None] - j
        for h in range(H):
            g = h // per
            qs, ks, vs = Q[a:b, h], K[c:d, g], V[c:d, g]
            seen = seen0.clone()
            t = sc * (qs @ ks.T)
            mag = sc * (qs.abs() @ ks.abs().T)
            if R:
                bias = B[h][dist.clamp(0, R - 1)]
                seen &= bias > -1e30
                t, mag = t + torch.where(seen, bias, 0.0), mag + torch.where(seen, bias.abs(), 0.0)
            some = seen.any(1)
            tm = t.masked_fill(~seen, -math.inf)
            top = torch.where(some, torch.nan_to_num(tm, nan=-math.inf).max(1).values, 0.0)
            e = torch.where(seen, torch.exp(tm - top[:, None]), 0.0)
            tot = e.sum(1)
            P = torch.where(some[:, None], e / torch.where(some, tot, 1.0)[:, None], 0.0)
            lse[h, a:b] = torch.where(some, top + torch.log(torch.where(some, tot, 1.0)), -math.inf)
            dlogit = (dh + 8) * U32 * torch.where(seen, mag, 0.0).max(1).values
            rp = 2 * dlogit + (m + 16) * U32
            lse_b[h, a:b] = rp + 8 * U32 * (1 + lse[h, a:b].abs().nan_to_num(posinf=0.0))
            # masked pairs are left out of the sums, whatever their values are
            def pv(X, Y):
                bad = ~torch.isfinite(Y)
                r = X @ torch.where(bad, 0.0, Y)
                return torch.where((seen.double() @ bad.double()) > 0, math.nan, r)

            def ptv(X, Y):
                bad = ~torch.isfinite(Y)
                r = X.T @ torch.where(bad, 0.0, Y)
                return torch.where((seen.double().T @ bad.double()) > 0, math.nan, r)
            o = pv(P, vs)
            ob = (up + rp + m * U32)[:, None] * pv(P, vs.abs()) + u * o.abs()
            out[a:b, h], out_b[a:b, h] = o, ob
            if dO is None:
                continue
            gs = dO[a:b, h]
            D = torch.where(some, (gs * o).sum(1), 0.0)
            D_b = torch.where(some, (gs.abs() * ob).sum(1) + dh * U32 * (gs.abs() * o.abs()).sum(1), 0.0)
            dS = torch.where(seen, P * (gs @ vs.T - D[:, None]), 0.0)
            absdp = gs.abs() @ vs.abs().T + D.abs()[:, None]
            dds = torch.where(seen, P * (D_b[:, None] + (rp + (dh + 8) * U32)[:, None] * absdp), 0.0)
            w = dds + (up + (m + n) * U32) * dS.abs()
            x = sc * pv(dS, ks)
            dq[a:b, h] = x
            dq_b[a:b, h] = sc * pv(w, ks.abs()) + u * x.abs()
            dk[c:d, g] += sc * ptv(dS, qs)
            dk_b[c:d, g] += sc * ptv(w, qs.abs())
            dv[c:d, g] += ptv(P, gs)
            dv_b[c:d, g] += ptv(P * (up + rp + (m + n) * U32)[:, None], gs.abs())
            if R:
                wr = dds + (m + n) * U32 * dS.abs()
                for bkt in range(R - 1):
                    dg = torch.diagonal(dS, -bkt) if bkt < n else None
                    if dg is not None:
                        drel[h, bkt] += dg.sum()
                        drel_b[h, bkt] += torch.diagonal(wr, -bkt).sum()
    res = {"out": (out, out_b), "lse": (lse, lse_b)}
    if dO is not None:
        res.update(dq=(dq, dq_b), dk=(dk, dk_b + u * dk.abs()), dv=(dv, dv_b + u * dv.abs()))
        if R:
            # each row's dS adds up to zero
            drel[:, R - 1] = -drel[:, :R - 1].sum(1)
            drel_b[:, R - 1] = drel_b[:, :R - 1].sum(1)
            res["drel"] = (drel, drel_b + u * drel.abs())
    return res


def sequences(offsets):
    """groups of packed causal sequences"""
    o = [int(x) for x in offsets]
    return [((a, b), (a, b), np.arange(1, b - a + 1)) for a, b in zip(o, o[1:])]


def events(key_offsets, event_offsets, query_offsets, prefix):
    """groups of event_attention, a user each"""
    res = []
    for u in range(len(key_offsets) - 1):
        e0, e1 = int(event_offsets[u]), int(event_offsets[u + 1])
        a, b = int(query_offsets[e0]), int(query_offsets[e1])
        lim = np.concatenate([np.full(int(query_offsets[e + 1] - query_offsets[e]), int(prefix[e]), dtype=np.int64)
                              for e in range(e0, e1)] + [np.zeros(0, dtype=np.int64)])
        res.append(((a, b), (int(key_offsets[u]), int(key_offsets[u + 1])), lim))
    return res


def check(got: dict, want: dict, skip=()):
    """Every value within its bound (1 % for the bounds' own higher orders);
    infinities and NaN where the formula has them."""
    worst = {}
    for name, (ref, bound) in want.items():
        if name in skip or name not in got:
            continue
        x = got[name].detach().cpu().double()
        assert x.shape == ref.shape, (name, x.shape, ref.shape)
        fin = torch.isfinite(ref)
        assert torch.equal(torch.isnan(x), torch.isnan(ref)), \
            f"{name}: NaN at {(torch.isnan(x) ^ torch.isnan(ref)).nonzero()[:5].tolist()}"
        assert torch.equal(x[~fin & ~torch.isnan(ref)], ref[~fin & ~torch.isnan(ref)]), name
        tiny = 1e-30
        err = (x[fin] - ref[fin]).abs() / (1.01 * bound[fin] + tiny)
        worst[name] = float(err.max()) if err.numel() else 0.0
        assert worst[name] <= 1.0, f"{name}: {worst[name]:.3f} times its bound"
    return worst
