"""Plain 64-bit forms of what the calls on a cache in pages compute, sequence by sequence, with bounds on what the kernels' roundings may amount to.  Half a step of
bf16 is 2^-8 of a value, of fp32 2^-24."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def frequencies(r, device):
    """of agzo_rope's fields"""
    p = torch.arange(r.rot_dim // 2, device=device, dtype=torch.float64)
    f = float(r.theta) ** (-2 * p / r.rot_dim)
    if r.scaling == 0:
        m = torch.ones_like(f)
    elif r.scaling == 1:
        m = torch.zeros_like(f)
    elif r.scaling == 2:
        m = ((r.original * f / (2 * math.pi) - r.low) / (r.high - r.low)).clamp(0, 1)
    else:
        pair = lambda turns: r.rot_dim * math.log(r.original / (2 * math.pi * turns)) / (2 * math.log(r.theta))
        first, last = max(math.floor(pair(r.high)), 0), min(math.ceil(pair(r.low)), r.rot_dim - 1)
        m = 1 - ((p - first) / max(last - first, 0.001)).clamp(0, 1)
    return f if r.scaling == 0 else f * (m + (1 - m) / r.factor)


def rotate(x, positions, r, dim, back=False):
    """x [n][heads * dim] in fp64 -> (result, bound of the fp32 arithmetic's error): angles are off by 2^-21 and 2^-50 of a position, products and sums by 2^-22"""
    n, rot = x.shape[0], r.rot_dim
    z = x.double().reshape(n, -1, dim).clone()
    ang = positions.double()[:, None, None] * frequencies(r, x.device)
    cos, sin = ang.cos() * r.magnitude, ang.sin() * (-r.magnitude if back else r.magnitude)
    ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if r.interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = z[..., ia].clone(), z[..., ib].clone()
    z[..., ia], z[..., ib] = a * cos - b * sin, b * cos + a * sin
    off = torch.zeros_like(z)
    off[..., ia] = off[..., ib] = (2.0 ** -20 + 2.0 ** -50 * positions.double().abs()[:, None, None]) * abs(r.magnitude) * (a.abs() + b.abs())
    return z.reshape(n, -1), off.reshape(n, -1)


def norm(x, gain, dim, eps):
    z = x.double().reshape(x.shape[0], -1, dim)
    z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt()
    return (z if gain is None else z * gain.double()).reshape(x.shape[0], -1)


def places(cu, k_len, room):
    """(sequence, row of it, place) of each new token"""
    for s in range(len(cu) - 1):
        m, have = cu[s + 1] - cu[s], min(max(k_len[s], 0), room)
        for i in range(m):
            yield s, i, have - m + i


def slot(table, page_size, n_pages, s, place):
    """(page, slot) or None"""
    if place < 0 or place >= len(table[s]) * page_size:
        return None
    page = table[s][place // page_size]
    return (page, place % page_size) if 0 <= page < n_pages else None


def gather(cache, table, page_size, s, n):
    """the first n places of a sequence, [n][key heads][dim]; ids that are no page's are the nearest"""
    at = torch.arange(n, device=cache.device)
    ids = torch.tensor(table[s], device=cache.device, dtype=torch.long).clamp(0, cache.shape[0] - 1) if len(table[s]) else torch.zeros(0, dtype=torch.long, device=cache.device)
    return cache[ids[at // page_size], at % page_size]


def seen(m, n, bits, device):
    """[m][n]: which of a sequence's n places its m new tokens see; bits: [m] python ints or None"""
    i, j = torch.arange(m, device=device)[:, None], torch.arange(n, device=device)[None, :]
    rel = j - (n - m)
    if bits is None:
        return rel <= i
    own = torch.tensor([[bool(b >> t & 1) for t in range(m)] for b in bits], dtype=torch.bool, device=device).reshape(m, m)
    return (rel < 0) | own.gather(1, rel.clamp(0, max(m - 1, 0)).expand(m, n))


def attention(q, kc, vc, table, page_size, k_len, cu, dim, scale=None, bits=None):
    """{out, lse, out_off} of the new tokens' rows; rows of no sequence are NaN.  bits: a python int for each row"""
    scale = dim ** -0.5 if scale is None else scale
    dev, room = q.device, len(table[0]) * page_size if table else 0
    q = q.double().view(q.shape[0], -1, dim)
    heads, kv = q.shape[1], kc.shape[2]
    out, off = torch.full_like(q, math.nan), torch.full_like(q, math.nan)
    lse = torch.full(q.shape[:2], math.nan, dtype=torch.float64, device=dev)
    for s in range(len(cu) - 1):
        m, n = cu[s + 1] - cu[s], min(max(k_len[s], 0), room)
        if m == 0:
            continue
        rows = slice(cu[s], cu[s + 1])
        vis = seen(m, n, None if bits is None else bits[rows], dev)
        any_ = vis.any(1, keepdim=True)
        k, v = gather(kc, table, page_size, s, n).double(), gather(vc, table, page_size, s, n).double()
        for h in range(heads):
            g = h * kv // heads
            z = torch.where(vis, (q[rows, h] @ torch.where(vis.any(0)[:, None], k[:, g], 0.0).T) * scale, -math.inf)
            top = torch.logsumexp(z, 1, keepdim=True) if n else torch.full((m, 1), -math.inf, dtype=torch.float64, device=dev)
            p = torch.where(any_ & vis, (z - torch.where(any_, top, 0.0)).exp(), 0.0)
            vz = torch.where(vis.any(0)[:, None], v[:, g], 0.0)
            bad = ~torch.isfinite(vz)
            if bad.any():
                # (what a row does not see has no part, whatever it is)
                o = torch.stack([(p[i][vis[i]][:, None] * vz[vis[i]]).sum(0) for i in range(m)])
                mag = torch.where(torch.isfinite(o), p @ torch.where(bad, 0.0, vz).abs(), 0.0)
            else:
                o, mag = p @ vz, p @ vz.abs()
            out[rows, h], lse[rows, h] = o, top[:, 0]
            # probabilities and the result rounded, scores in fp32
            off[rows, h] = HALF[torch.bfloat16] * (mag + o.abs()) + 1e-5 * mag
    return {"out": out.flatten(1), "lse": lse, "out_off": off.flatten(1)}


def verify(p, q, tokens, uniforms, cu, parents=None):
    """(out_tokens, out_rows, n_accepted) as lists, the first two with None where nothing is written.  p, q: fp64 tensors on the CPU"""
    n, vocab = p.shape
    good = lambda t: torch.where(t > 0, t, torch.zeros_like(t))
    out_tokens, out_rows, accepted = [None] * n, [None] * n, []
    for s in range(len(cu) - 1):
        r0, rows = cu[s], cu[s + 1] - cu[s]
        if rows == 0:
            accepted.append(0)
            continue
        up = [i - 1 if parents is None else parents[r0 + i] for i in range(rows)]
        at, path, refused = 0, [], []
        while True:
            mine, refused, left, nxt = good(p[r0 + at]), [], 1.0, None
            for i in range(at + 1, rows):
                if up[i] != at:
                    continue
                x = tokens[r0 + i]
                inside = 0 <= x < vocab
                mass = float(mine[x]) if inside and x not in [tokens[r0 + j] for j in refused] else 0.0
                if q is None and not inside:
                    mass = 0.0
                if q is not None:
                    yes = inside and mass > 0 and uniforms[r0 + i] * float(good(q[r0 + i])[x]) < mass
                else:
                    yes = mass > 0 and uniforms[r0 + i] * left < mass
                if yes:
                    nxt = i
                    break
                refused.append(i)
                left -= mass
            if nxt is None:
                break
            path.append(nxt)
            at = nxt
        w = good(p[r0 + at]).clone()
        if q is not None and refused:
            w = good(w - good(q[r0 + refused[-1]]))
        elif refused:
            for j in refused:
                if 0 <= tokens[r0 + j] < vocab:
                    w[tokens[r0 + j]] = 0.0
        if not bool((w > 0).any()):
            w = good(p[r0 + at])
        live = (w > 0).nonzero()[:, 0]
        if live.numel() == 0:
            follows = -1
        else:
            sums = w[live].cumsum(0)
            above = (sums > uniforms[r0] * sums[-1]).nonzero()[:, 0]
            follows = int(live[above[0]] if above.numel() else live[-1])
        for i in range(rows):
            out_tokens[r0 + i] = tokens[r0 + path[i]] if i < len(path) else follows if i == len(path) else -1
            out_rows[r0 + i] = path[i] if i < len(path) else -1
        accepted.append(len(path))
    return out_tokens, out_rows, accepted
