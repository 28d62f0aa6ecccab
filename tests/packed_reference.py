"""Plain 64-bit forms of what the calls on packed batches compute, sequence by sequence and head by head, with bounds on what the
kernels' roundings may amount to.  Half a step of bf16 is 2^-8 of a value.  (On the device the tensors are on)"""
import math

import torch

HALF = 2.0 ** -8


def norm_rope(x, gain, positions, dim, eps, theta):
    n, half = x.shape[0], dim // 2
    z = x.double().view(n, -1, dim)
    z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt()
    if gain is not None:
        z = z * gain.double()
    ang = positions.double()[:, None, None] * theta ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    a, b = z[..., :half], z[..., half:]
    return torch.cat((a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()), -1).flatten(1)


def seen(nq, nk, causal, device):
    if not causal:
        return torch.ones(nq, nk, dtype=torch.bool, device=device)
    i, j = torch.arange(nq, device=device)[:, None], torch.arange(nk, device=device)[None, :]
    return j <= i + nk - nq


def attention(q, k, v, cu_q, cu_k, dim, scale=None, causal=True, dout=None):
    """{out, lse (, dq, dk, dv)} and the same keys + "_off": bounds of the absolute error.  Rows of no sequence are NaN."""
    scale = dim ** -0.5 if scale is None else scale
    dev = q.device
    q, k, v = (t.double().view(t.shape[0], -1, dim) for t in (q, k, v))
    H, KV = q.shape[1], k.shape[1]
    nan = lambda like: torch.full_like(like, math.nan)
    r = {"out": nan(q), "lse": torch.full(q.shape[:2], math.nan, dtype=torch.float64, device=dev)}
    r["out_off"] = nan(q)
    if dout is not None:
        dout = dout.double().view_as(q)
        for n, t in (("dq", q), ("dk", k), ("dv", v)):
            r[n], r[n + "_off"] = nan(t), nan(t)
    for b in range(len(cu_q) - 1):
        qs, ks = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        nq, nk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        if dout is not None:
            for n in ("dk", "dk_off", "dv", "dv_off"):
                r[n][ks] = 0.0
        vis = seen(nq, nk, causal, dev)
        any_ = vis.any(1, keepdim=True)
        lonely = vis.sum(1, keepdim=True) == 1          # one key: probability 1, whatever the scores
        for h in range(H):
            g = h * KV // H
            s = (q[qs, h] @ k[ks, g].T) * scale
            s = torch.where(vis, s, -math.inf)
            lse = torch.logsumexp(s, 1, keepdim=True) if nk else torch.full((nq, 1), -math.inf, dtype=torch.float64, device=dev)
            p = torch.where(any_ & vis, (s - torch.where(any_, lse, 0.0)).exp(), 0.0)
            # (masked places have no part, whatever they hold)
            vz = torch.where(vis.any(0)[:, None], v[ks, g], 0.0)
            out = p @ vz
            mag = p @ vz.abs()
            r["out"][qs, h], r["lse"][qs, h] = out, lse[:, 0]
            r["out_off"][qs, h] = HALF * (mag + out.abs()) + 1e-5 * mag
            if dout is None:
                continue
            d = dout[qs, h]
            out_off = r["out_off"][qs, h]
            dp = d @ vz.T
            delta = (d * out).sum(1, keepdim=True)
            delta_off = (d.abs() * out_off).sum(1, keepdim=True) + 1e-5 * (d.abs() * mag).sum(1, keepdim=True)
            ds = torch.where(vis & ~lonely, p * (dp - delta), 0.0)
            # scores in fp32: 1e-5 of a probability and of the products
            ds_off = torch.where(vis & ~lonely, HALF * ds.abs() + p * (delta_off + 1e-5 * (d.abs() @ vz.abs().T)) + 3e-5 * ds.abs(), 0.0)
            r["dq"][qs, h] = scale * ds @ k[ks, g]
            r["dq_off"][qs, h] = scale * ds_off @ k[ks, g].abs()
            r["dk"][ks, g] += scale * ds.T @ q[qs, h]
            r["dk_off"][ks, g] += scale * ds_off.T @ q[qs, h].abs()
            r["dv"][ks, g] += p.T @ d
            r["dv_off"][ks, g] += (HALF + 1e-5) * (p.T @ d.abs())
    if dout is not None:
        for n in ("dq", "dk", "dv"):
            r[n + "_off"] += HALF * r[n].abs()
    return {n: (t if n == "lse" else t.flatten(1)) for n, t in r.items()}


def rows_in(cu, total, device):
    """Which rows belong to a sequence."""
    m = torch.zeros(total, dtype=torch.bool, device=device)
    m[cu[0]:cu[-1]] = True
    return m
