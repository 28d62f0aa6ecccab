"""Operators of a decoder that is trained or evaluated on packed batches, as cases that can be timed and whose outputs can be compared.

  norm_rope   norms of queries and keys for each head, a gain for each of a head's dims, and the rotation by the token's position in one pass;
              and its gradient
  attention   causal attention with grouped heads over packed sequences of different lengths: whole prompts, single new tokens behind the
              keys that are there already, and a training pass with the gradients of q, k and v
  head        softmax cross-entropy of an LM head without keeping the logits, and its gradient for the head's inputs and weights

With own = False the plain form of each, in elementary torch operations; with own = True the library's calls.
"""
import math
import random

import torch

own = False

EPS, THETA = 1e-6, 1.0e6


def listed():
    return [
        # one new token for each of 16 sequences: latency is all there is
        {"name": "norm_rope_single", "kind": "norm_rope", "grad": False, "tokens": 16, "heads": 16, "kv": 8, "dim": 128, "far": 32768},
        # a packed prompt batch of the 8B-sized layer
        {"name": "norm_rope_prompt", "kind": "norm_rope", "grad": False, "tokens": 16384, "heads": 32, "kv": 8, "dim": 128, "far": 4096},
        # the gradient for a batch of no round size
        {"name": "norm_rope_grad", "kind": "norm_rope", "grad": True, "tokens": 15001, "heads": 32, "kv": 8, "dim": 128, "far": 4096},
        # a handful of short sentences, packed, with 64-wide heads
        {"name": "attention_sentences", "kind": "attention", "form": "prompt", "seqs": 37, "tokens": 1501, "heads": 14, "kv": 2, "dim": 64, "split": 1},
        # packed prompts of the 8B-sized layer, from a few tokens to a few thousand
        {"name": "attention_prompts", "kind": "attention", "form": "prompt", "seqs": 16, "tokens": 16384, "heads": 32, "kv": 8, "dim": 128, "split": 2},
        # one long document
        {"name": "attention_document", "kind": "attention", "form": "prompt", "seqs": 1, "tokens": 16001, "heads": 16, "kv": 8, "dim": 128, "split": 3},
        # one new token for each of 64 sequences, behind the keys that they have
        {"name": "attention_single", "kind": "attention", "form": "single", "seqs": 64, "tokens": 200000, "heads": 32, "kv": 8, "dim": 128, "split": 4},
        # training on short sentences
        {"name": "attention_train_short", "kind": "attention", "form": "train", "seqs": 16, "tokens": 1001, "heads": 16, "kv": 8, "dim": 128, "split": 5},
        # training on a packed batch, the decoder configuration's heads and tokens
        {"name": "attention_train", "kind": "attention", "form": "train", "seqs": 8, "tokens": 8192, "heads": 16, "kv": 8, "dim": 128, "split": 6},
        # the answers of a handful of tokens scored: the head's weights are read once
        {"name": "head_few", "kind": "head", "grad": False, "tokens": 7, "d": 2048, "vocab": 32000},
        # a batch without padding, a vocabulary that no tile divides
        {"name": "head_train_ragged", "kind": "head", "grad": True, "tokens": 3001, "d": 2048, "vocab": 32011},
        # the 8B-sized layer's width, a large vocabulary
        {"name": "head_train", "kind": "head", "grad": True, "tokens": 8192, "d": 4096, "vocab": 131072},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case over the ranges that the listed ones span."""
    kind = rng.choice(("norm_rope", "attention", "attention", "attention", "head"))
    if kind == "head":
        grad = rng.random() < 0.7
        return {"kind": "head", "grad": grad, "tokens": _log_int(rng, 1, 6000), "d": 8 * _log_int(rng, 32, 512), "vocab": _log_int(rng, 1000, 100000)}
    kv = rng.choice((1, 2, 4, 8))
    heads, dim = kv * rng.choice((1, 2, 3, 4, 7)), rng.choice((64, 128, 128))
    if kind == "norm_rope":
        return {"kind": "norm_rope", "grad": rng.random() < 0.5, "tokens": _log_int(rng, 1, 14000), "heads": heads, "kv": kv, "dim": dim, "far": _log_int(rng, 64, 200000)}
    form = rng.choice(("prompt", "single", "train"))
    while True:
        seqs = _log_int(rng, 1, 128)
        tokens = _log_int(rng, max(seqs, 16), 200000 if form == "single" else 12000)
        case = {"kind": "attention", "form": form, "seqs": seqs, "tokens": tokens, "heads": heads, "kv": kv, "dim": dim, "split": rng.randint(10, 1 << 20)}
        longest = max(_lengths(case))
        # (scores of a padded batch, in 32 bits: what the plain form holds)
        if seqs * heads * longest * (1 if form == "single" else longest) <= (1 << 30):
            return case


def _lengths(case):
    """How the tokens are dealt to the sequences: unevenly, at least one each."""
    rng, n, total = random.Random(case["split"]), case["seqs"], case["tokens"]
    share = [rng.lognormvariate(0.0, 0.8) for _ in range(n)]
    free, whole = total - n, sum(share)
    lens = [1 + int(free * s / whole) for s in share]
    lens[share.index(max(share))] += total - sum(lens)
    return lens


# ---- inputs ------------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", dtype=torch.float32, generator=gen)


def _unit(x):
    return x / x.square().mean(-1, keepdim=True).sqrt()


def _offsets(lens):
    return torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    bf = torch.bfloat16
    s = dict(case)
    if case["kind"] == "head":
        n, d, v = case["tokens"], case["d"], case["vocab"]
        w = _normal(gen, v, d) * 0.02
        ids = torch.randint(0, v, (n,), device="cuda", generator=gen).to(torch.int32)
        # inputs that know something of their targets: a mean loss of some two thirds of the untrained one
        x = _unit(_normal(gen, n, d) + 8.0 / math.sqrt(0.02 * d) * _unit(w[ids.long()]) * torch.rand(n, 1, device="cuda", generator=gen) * 0.1)
        ids[torch.rand(n, device="cuda", generator=gen) < 0.1] = -1      # prompt tokens, which are not learnt
        s.update(w=w.to(bf), x=x.to(bf), ids=ids, loss=torch.zeros(1, dtype=torch.float64, device="cuda"), lse=torch.empty(n, device="cuda"))
        if case["grad"]:
            s.update(dx=torch.empty(n, d, dtype=bf, device="cuda"), dw=torch.empty(v, d, dtype=bf, device="cuda"))
        return s
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    if case["kind"] == "norm_rope":
        n = case["tokens"]
        s.update(q=(_normal(gen, n, heads * dim) * 0.7).to(bf), k=(_normal(gen, n, kv * dim) * 1.3).to(bf),
                 q_gain=1.0 + 0.1 * _normal(gen, dim), k_gain=1.0 + 0.1 * _normal(gen, dim),
                 positions=torch.randint(0, case["far"], (n,), device="cuda", generator=gen).to(torch.int32),
                 qo=torch.empty(n, heads * dim, dtype=bf, device="cuda"), ko=torch.empty(n, kv * dim, dtype=bf, device="cuda"))
        if case["grad"]:
            s.update(dqo=_normal(gen, n, heads * dim).to(bf), dko=_normal(gen, n, kv * dim).to(bf),
                     dq_gain=torch.empty(dim, device="cuda"), dk_gain=torch.empty(dim, device="cuda"))
        return s
    lens, single = _lengths(case), case["form"] == "single"
    qlens = [1] * len(lens) if single else lens
    nq, nk = sum(qlens), sum(lens)
    # queries and keys as their norms leave them, with directions that a head's tokens share
    common = _normal(gen, 1, kv, dim)
    k = _unit(_normal(gen, nk, kv, dim) + 0.5 * common)
    q = _unit(_normal(gen, nq, heads, dim) + 0.5 * common.repeat_interleave(heads // kv, 1))
    s.update(q=(1.3 * q).reshape(nq, -1).to(bf), k=(1.3 * k).reshape(nk, -1).to(bf), v=_normal(gen, nk, kv * dim).to(bf),
             cu_q=_offsets(qlens), cu_k=_offsets(lens), max_q=max(qlens), max_k=max(lens),
             out=torch.empty(nq, heads * dim, dtype=bf, device="cuda"))
    if case["form"] == "train":
        s.update(dout=_normal(gen, nq, heads * dim).to(bf), lse=torch.empty(nq, heads, device="cuda"),
                 dq=torch.empty(nq, heads * dim, dtype=bf, device="cuda"), dk=torch.empty(nk, kv * dim, dtype=bf, device="cuda"),
                 dv=torch.empty(nk, kv * dim, dtype=bf, device="cuda"))
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------
def _angles(s):
    half = s["dim"] // 2
    inv = THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    a = s["positions"].double()[:, None, None] * inv
    return torch.cos(a).float(), torch.sin(a).float()


def _norm_rope(x, gain, s, cs):
    half = s["dim"] // 2
    x = x.float().view(x.shape[0], -1, s["dim"])
    x = gain * x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    a, b = x[..., :half], x[..., half:]
    return torch.cat((a * cs[0] - b * cs[1], b * cs[0] + a * cs[1]), -1).flatten(1).to(torch.bfloat16)


def _norm_rope_grad(x, dy, gain, s, cs):
    half = s["dim"] // 2
    x, dy = x.float().view(x.shape[0], -1, s["dim"]), dy.float().view(x.shape[0], -1, s["dim"])
    a, b = dy[..., :half], dy[..., half:]
    dn = torch.cat((a * cs[0] + b * cs[1], b * cs[0] - a * cs[1]), -1)
    scale = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    unit = x * scale
    dgain = (dn * unit).sum((0, 1), dtype=torch.float64).float()
    dn = dn * gain
    dx = scale * (dn - unit * (dn * unit).mean(-1, keepdim=True))
    return dx.flatten(1).to(torch.bfloat16), dgain


def _padded(x, cu, longest):
    """[tokens][heads * dim] -> [sequence][position][heads * dim] in 32 bits, and which positions are there."""
    start, length = cu[:-1].long()[:, None], (cu[1:] - cu[:-1]).long()[:, None]
    at = torch.arange(longest, device="cuda")[None, :]
    there = at < length
    return x.float()[torch.where(there, start + at, 0)], there


def _rows(x, kv, dim):
    """-> [sequence][kv head][its heads x position][dim]"""
    b, t = x.shape[:2]
    return x.view(b, t, kv, -1, dim).permute(0, 2, 3, 1, 4).reshape(b, kv, -1, dim)


def _packed(x, heads, t, there):
    """The inverse of _rows(_padded()), for the positions that are there."""
    b, kv, _, dim = x.shape
    return x.view(b, kv, heads // kv, t, dim).permute(0, 3, 1, 2, 4).reshape(b, t, heads * dim)[there]


def _attention(s):
    heads, kv, dim = s["heads"], s["kv"], s["dim"]
    q, q_there = _padded(s["q"], s["cu_q"], s["max_q"])
    k, k_there = _padded(s["k"], s["cu_k"], s["max_k"])
    v, _ = _padded(s["v"], s["cu_k"], s["max_k"])
    q, k, v = _rows(q, kv, dim), _rows(k, kv, dim), _rows(v, kv, dim)
    scale = 1.0 / math.sqrt(dim)
    before = (s["cu_k"][1:] - s["cu_k"][:-1]) - (s["cu_q"][1:] - s["cu_q"][:-1])      # keys in front of the queries
    seen = torch.arange(s["max_k"], device="cuda")[None, None, :] <= (torch.arange(s["max_q"], device="cuda")[:, None] + before[:, None, None])
    hidden = (~(seen & k_there[:, None, :]))[:, None, None]                  # [sequence][1][1][query][key]
    p = q @ k.transpose(-1, -2)
    grid = (p.shape[0], kv, heads // kv, s["max_q"], s["max_k"])
    p.mul_(scale).view(grid).masked_fill_(hidden, -math.inf)
    top = p.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0, 1.0, total))
    out = _packed(p @ v, heads, s["max_q"], q_there).to(torch.bfloat16)
    if s["form"] != "train":
        return out
    dout, _ = _padded(s["dout"], s["cu_q"], s["max_q"])
    dout = _rows(dout * q_there[..., None], kv, dim)
    dv = p.transpose(-1, -2) @ dout
    lse = _packed(top + total.log(), heads, s["max_q"], q_there)
    ds = dout @ v.transpose(-1, -2)
    ds.sub_((p * ds).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = ds @ k, ds.transpose(-1, -2) @ q
    bf = torch.bfloat16
    return {"out": out, "lse": lse, "dq": _packed(dq, heads, s["max_q"], q_there).to(bf),
            "dk": _packed(dk, kv, s["max_k"], k_there).to(bf), "dv": _packed(dv, kv, s["max_k"], k_there).to(bf)}


def _head(s):
    x, w = s["x"].float(), s["w"].float()
    p = x @ w.T
    top = p.amax(-1, keepdim=True)
    counted = s["ids"] >= 0
    ids = torch.where(counted, s["ids"], 0).long()[:, None]
    hit = p.gather(1, ids)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = top + total.log()
    count = counted.sum().clamp(min=1)
    loss = (torch.where(counted[:, None], lse - hit, 0.0).sum(dtype=torch.float64) / count).float()
    if not s["grad"]:
        return {"loss": loss, "lse": lse[:, 0]}
    p.div_(total)
    p.scatter_add_(1, ids, torch.full_like(hit, -1.0))
    p.mul_((counted / count)[:, None])
    return {"loss": loss, "lse": lse[:, 0], "dx": (p @ w).to(torch.bfloat16), "dw": (p.T @ x).to(torch.bfloat16)}


# ---- the library's calls -----------------------------------------------------------------------------------------
_context = None


def _library():
    global _context
    from paper_2601_17261_amd import binding
    if _context is None:
        _context = binding.Context()
    return binding, _context


def _own(s):
    binding, ctx = _library()
    if s["kind"] == "norm_rope":
        if s["grad"]:
            ctx.glue_qk_norm_rope_backward(s["q"], s["k"], s["positions"], s["dqo"], s["dko"], s["qo"], s["ko"], s["dim"], s["q_gain"], s["k_gain"],
                                           s["dq_gain"], s["dk_gain"], EPS, THETA)
            return {"dq": s["qo"], "dk": s["ko"], "dq_gain": s["dq_gain"], "dk_gain": s["dk_gain"]}
        ctx.glue_qk_norm_rope(s["q"], s["k"], s["positions"], s["qo"], s["ko"], s["dim"], s["q_gain"], s["k_gain"], EPS, THETA)
        return {"q": s["qo"], "k": s["ko"]}
    if s["kind"] == "attention":
        if s["form"] != "train":
            ctx.glue_attention_packed(s["q"], s["k"], s["v"], s["out"], s["cu_q"], s["cu_k"], s["dim"])
            return s["out"]
        ctx.glue_attention_packed(s["q"], s["k"], s["v"], s["out"], s["cu_q"], s["cu_k"], s["dim"], lse=s["lse"])
        ctx.glue_attention_packed_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"], s["cu_q"], s["cu_k"], s["dim"])
        return {"out": s["out"], "lse": s["lse"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    layer, target = binding.make_layer(s["w"], s["x"]), binding.make_loss(s["ids"], binding.LOSS_CE)
    ctx.ce_forward(layer, s["w"], s["x"], target, s["loss"], s["lse"])
    if not s["grad"]:
        return {"loss": s["loss"][0].float(), "lse": s["lse"]}
    ctx.ce_backward(layer, s["w"], s["x"], target, s["lse"], s["dx"], s["dw"])
    return {"loss": s["loss"][0].float(), "lse": s["lse"], "dx": s["dx"], "dw": s["dw"]}


def run(state):
    s = state
    if own:
        return _own(s)
    if s["kind"] == "norm_rope":
        cs = _angles(s)
        if not s["grad"]:
            return {"q": _norm_rope(s["q"], s["q_gain"], s, cs), "k": _norm_rope(s["k"], s["k_gain"], s, cs)}
        dq, dq_gain = _norm_rope_grad(s["q"], s["dqo"], s["q_gain"], s, cs)
        dk, dk_gain = _norm_rope_grad(s["k"], s["dko"], s["k_gain"], s, cs)
        return {"dq": dq, "dk": dk, "dq_gain": dq_gain, "dk_gain": dk_gain}
    return _attention(s) if s["kind"] == "attention" else _head(s)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "head":
        n, d, v = case["tokens"], case["d"], case["vocab"]
        rw = 2 * (n * d + v * d)
        return {"bytes": (2 * rw if case["grad"] else rw) + 8 * n, "flops": 2.0 * n * v * d * (3 if case["grad"] else 1)}
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    if case["kind"] == "norm_rope":
        n = case["tokens"] * (heads + kv) * dim
        return {"bytes": 2 * n * (3 if case["grad"] else 2) + 4 * case["tokens"], "flops": n * (14.0 if case["grad"] else 6.0)}
    lens, single, train = _lengths(case), case["form"] == "single", case["form"] == "train"
    pairs = sum(lens) if single else sum(n * (n + 1) // 2 for n in lens)
    q, k = (len(lens) if single else sum(lens)) * heads * dim, sum(lens) * kv * dim
    # (training: q, k, v, dout in; out, dq, dk, dv and the sums' logarithms out)
    moved = 2 * (4 * q + 4 * k) + 4 * q // dim if train else 2 * (2 * q + 2 * k)
    return {"bytes": moved, "flops": pairs * heads * dim * (14.0 if train else 4.0)}


# ---- from the definition, in 64 bits -----------------------------------------------------------------------------
def _exact_norm_rope(x, gain, pos, dim, dy):
    n, half = x.shape[0], dim // 2
    z = x.double().reshape(n, -1, 2, half)
    rms = (z.pow(2).sum((2, 3), keepdim=True) / dim + EPS).sqrt()
    g = gain.double().view(2, half)
    turn = torch.exp(torch.arange(half, device="cuda", dtype=torch.float64) * (-2.0 / dim * math.log(THETA))) * pos.double()[:, None]
    rot = torch.polar(torch.ones_like(turn), turn)[:, None]
    if dy is None:
        y = torch.complex(z[:, :, 0] / rms[:, :, 0] * g[0], z[:, :, 1] / rms[:, :, 0] * g[1]) * rot
        return torch.stack((y.real, y.imag), 2).reshape(n, -1), None
    d = dy.double().reshape(n, -1, 2, half)
    back = torch.complex(d[:, :, 0], d[:, :, 1]) * rot.conj()
    d = torch.stack((back.real, back.imag), 2)
    dgain = (d * z / rms).sum((0, 1)).reshape(dim)
    d = d * g
    dz = d / rms - z * (d * z).sum((2, 3), keepdim=True) / (dim * rms.pow(3))
    return dz.reshape(n, -1), dgain


def _exact_attention(case, s):
    heads, kv, dim, train = case["heads"], case["kv"], case["dim"], case["form"] == "train"
    q, k, v = (s[n].double().view(s[n].shape[0], -1, dim) for n in ("q", "k", "v"))
    out, lse = torch.zeros_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    d = s["dout"].double().view_as(q) if train else None
    cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
    for b in range(case["seqs"]):
        qs, ks = slice(cq[b], cq[b + 1]), slice(ck[b], ck[b + 1])
        nq, nk = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
        future = torch.ones(nq, nk, dtype=torch.bool, device="cuda").triu(nk - nq + 1)
        for h in range(heads):
            g = h * kv // heads
            a = torch.mm(q[qs, h], k[ks, g].t().contiguous()) / math.sqrt(dim)
            a = a.masked_fill(future, -math.inf)
            lse[qs, h] = a.logsumexp(1)
            a = (a - lse[qs, h, None]).exp()
            out[qs, h] = a @ v[ks, g]
            if train:
                dv[ks, g] += a.t() @ d[qs, h]
                da = d[qs, h] @ v[ks, g].t()
                da = a * (da - (d[qs, h] * out[qs, h]).sum(1, keepdim=True)) / math.sqrt(dim)
                dq[qs, h] = da @ k[ks, g]
                dk[ks, g] += da.t() @ q[qs, h]
    if not train:
        return out.flatten(1)
    return {"out": out.flatten(1), "lse": lse, "dq": dq.flatten(1), "dk": dk.flatten(1), "dv": dv.flatten(1)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm_rope":
        grad = case["grad"]
        q, q_gain = _exact_norm_rope(s["q"], s["q_gain"], s["positions"], case["dim"], s["dqo"] if grad else None)
        k, k_gain = _exact_norm_rope(s["k"], s["k_gain"], s["positions"], case["dim"], s["dko"] if grad else None)
        return {"dq": q, "dk": k, "dq_gain": q_gain, "dk_gain": k_gain} if grad else {"q": q, "k": k}
    if case["kind"] == "attention":
        return _exact_attention(case, s)
    x, w, ids = s["x"].double(), s["w"].double(), s["ids"].long()
    rows = (ids >= 0).nonzero()[:, 0]
    logits = torch.mm(x, w.t())
    lse = logits.logsumexp(1)
    n = max(1, rows.numel())
    loss = (lse[rows] - logits[rows, ids[rows]]).sum() / n
    if not case["grad"]:
        return {"loss": loss, "lse": lse}
    d = torch.zeros_like(logits)
    d[rows] = (logits[rows] - lse[rows, None]).exp() / n
    d[rows, ids[rows]] -= 1.0 / n
    return {"loss": loss, "lse": lse, "dx": torch.mm(d, w), "dw": torch.mm(d.t(), x)}
