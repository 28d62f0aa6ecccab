"""Operators of a decoder that serves from a cache in pages and drafts tokens ahead, as cases that can be timed and whose outputs can be compared.

  rope        rotation of queries and keys by the token's position: pairs half a head apart or side by side, part of the head, frequencies
              scaled for contexts longer than the trained one; and its gradient
  append      new tokens on their way into the cache: norms and rotation of queries and keys, keys and values written to their pages
  attention   attention over the cache: single new tokens, trees of drafted tokens, further pieces of long prompts
  verify      drafted tokens accepted or refused by the target's probabilities and given random numbers, and the token that follows
  keep        the accepted tokens of a tree moved together in the cache

With own = False the plain form of each, in elementary torch operations; with own = True the library's calls.
"""
import math
import random

import torch

own = False

EPS, THETA = 1e-6, 1.0e6
SCALED = {"plain": {}, "linear": {"factor": 4.0}, "turns": {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192.0},
          "dims": {"factor": 4.0, "low": 1.0, "high": 32.0, "original": 32768.0, "magnitude": 0.1 * math.log(4.0) + 1.0}}


def listed():
    return [
        # a packed prompt batch of the 8B-sized layer, four times the context that it was trained on
        {"name": "rope_prompt", "kind": "rope", "grad": False, "type": "bf16", "tokens": 16384, "heads": 32, "kv": 8, "dim": 128, "rot": 128, "inter": False, "scaling": "dims", "far": 131072},
        # the gradient for a batch of no round size, half of each head rotated, pairs side by side
        {"name": "rope_grad", "kind": "rope", "grad": True, "type": "bf16", "tokens": 15001, "heads": 16, "kv": 8, "dim": 128, "rot": 64, "inter": True, "scaling": "plain", "far": 4096},
        # one new token for each of 64 sequences: latency is all there is
        {"name": "append_single", "kind": "append", "form": "single", "seqs": 64, "tokens": 64, "before": 20000, "page": 16, "heads": 32, "kv": 8, "dim": 128, "norm": True, "inter": False, "split": 1},
        # prompts of the 8B-sized layer, from a few tokens to a few thousand
        {"name": "append_prompt", "kind": "append", "form": "chunk", "seqs": 16, "tokens": 16384, "before": 100, "page": 16, "heads": 32, "kv": 8, "dim": 128, "norm": True, "inter": False, "split": 2},
        # the first tokens of a few conversations: latency again
        {"name": "attention_start", "kind": "attention", "form": "single", "seqs": 4, "tokens": 700, "new": 4, "page": 16, "heads": 16, "kv": 8, "dim": 128, "split": 3},
        # one new token for each of 64 sequences, behind the keys that they have
        {"name": "attention_single", "kind": "attention", "form": "single", "seqs": 64, "tokens": 200000, "new": 64, "page": 16, "heads": 32, "kv": 8, "dim": 128, "split": 4},
        # trees of up to 48 drafted tokens
        {"name": "attention_tree", "kind": "attention", "form": "tree", "seqs": 12, "tokens": 60000, "new": 48, "page": 64, "heads": 32, "kv": 8, "dim": 128, "split": 5},
        # the next pieces of a few long prompts
        {"name": "attention_chunk", "kind": "attention", "form": "chunk", "seqs": 3, "tokens": 20001, "new": 2500, "page": 32, "heads": 32, "kv": 8, "dim": 128, "split": 6},
        # chains of eight drafted tokens, a large vocabulary
        {"name": "verify_chain", "kind": "verify", "form": "chain", "type": "f32", "seqs": 64, "nodes": 9, "vocab": 131072, "split": 7},
        # trees of drafts that are proposed for certain, a vocabulary that no tile divides
        {"name": "verify_tree", "kind": "verify", "form": "tree", "type": "f32", "seqs": 12, "nodes": 48, "vocab": 32011, "split": 8},
        # what is accepted of one tree
        {"name": "keep_tree", "kind": "keep", "seqs": 1, "nodes": 48, "before": 5000, "page": 16, "kv": 8, "dim": 128, "split": 9},
        # ... and of the trees of a full batch
        {"name": "keep_trees", "kind": "keep", "seqs": 256, "nodes": 64, "before": 50000, "page": 16, "kv": 8, "dim": 128, "split": 10},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case over the ranges that the listed ones span."""
    kind = rng.choice(("rope", "append", "attention", "attention", "attention", "verify", "verify", "keep"))
    kv = rng.choice((1, 2, 4, 8))
    heads, dim = kv * rng.choice((1, 2, 3, 4, 7)), rng.choice((64, 128, 128))
    page, split = rng.choice((1, 12, 16, 16, 32, 64, 256)), rng.randint(11, 1 << 20)
    if kind == "rope":
        dim = rng.choice((64, 80, 96, 128, 128, 256))
        heads = min(heads, 4096 // dim)
        return {"kind": "rope", "grad": rng.random() < 0.5, "type": rng.choice(("bf16", "bf16", "f32")), "tokens": _log_int(rng, 1, 8000), "heads": heads, "kv": kv, "dim": dim,
                "rot": 16 * rng.randint(1, dim // 16), "inter": rng.random() < 0.5, "scaling": rng.choice(sorted(SCALED)), "far": _log_int(rng, 64, 1000000)}
    if kind == "append":
        form, seqs = rng.choice(("single", "tree", "chunk")), _log_int(rng, 1, 128)
        tokens = seqs if form == "single" else seqs * rng.randint(2, 64) if form == "tree" else _log_int(rng, seqs, 12000)
        return {"kind": "append", "form": form, "seqs": seqs, "tokens": tokens, "before": _log_int(rng, seqs, 20000), "page": page, "heads": heads, "kv": kv, "dim": dim,
                "norm": rng.random() < 0.5, "inter": rng.random() < 0.5, "split": split}
    if kind == "keep":
        seqs = _log_int(rng, 1, 200)
        return {"kind": "keep", "seqs": seqs, "nodes": rng.randint(2, 64), "before": _log_int(rng, seqs, 40000), "page": page, "kv": kv, "dim": dim, "split": split}
    if kind == "verify":
        vocab, nodes = _log_int(rng, 500, 130000), rng.randint(2, 60)
        form = rng.choice(("chain", "tree"))
        nodes = min(nodes, 17) if form == "chain" else nodes
        return {"kind": "verify", "form": form, "type": rng.choice(("f32", "bf16")), "seqs": _log_int(rng, 1, max(2, min(64, 50000000 // (nodes * vocab)))), "nodes": nodes, "vocab": vocab,
                "split": split}
    form = rng.choice(("single", "tree", "chunk"))
    while True:
        seqs = _log_int(rng, 1, 100 if form == "single" else 24)
        tokens = _log_int(rng, max(seqs * 64, 200), 180000 if form == "single" else 60000 if form == "tree" else 20000)
        new = seqs if form == "single" else rng.randint(2, 64) if form == "tree" else min(tokens, _log_int(rng, 2 * seqs, 2500))
        case = {"kind": "attention", "form": form, "seqs": seqs, "tokens": tokens, "new": new, "page": page, "heads": heads, "kv": kv, "dim": dim, "split": split}
        qlens, klens = _lengths(case)
        # (scores of a padded batch, in 32 bits: what the plain form holds)
        if seqs * heads * max(qlens) * max(klens) <= (1 << 29):
            return case


# ---- how the tokens lie ------------------------------------------------------------------------------------------
def _deal(rng, total, n):
    """total tokens dealt to n sequences: unevenly, at least one each"""
    share = [rng.lognormvariate(0.0, 0.8) for _ in range(n)]
    free, whole = total - n, sum(share)
    lens = [1 + int(free * s / whole) for s in share]
    lens[share.index(max(share))] += total - sum(lens)
    return lens


def _tree(rng, n):
    """parents of the n nodes of a tree: its likeliest chain first, branches behind it"""
    chain = min(n - 1, 8)
    parents, depth = [-1] + list(range(chain)), list(range(chain + 1))
    for i in range(chain + 1, n):
        p = rng.randrange(i)
        while depth[p] >= 8:
            p = rng.randrange(i)
        parents.append(p)
        depth.append(depth[p] + 1)
    return parents, depth


def _lengths(case):
    """new tokens and keys (the new ones among them) of each sequence"""
    rng, n, form = random.Random(case["split"]), case["seqs"], case.get("form", "tree")
    if form == "single":
        new = [1] * n
    elif form == "tree":
        most = case["nodes"] if "nodes" in case else case["new"] if case["kind"] == "attention" else case["tokens"] // n
        new = [rng.randint((most + 1) // 2, most) if case["kind"] == "attention" else most for _ in range(n)]
    else:
        new = _deal(rng, case["new"] if case["kind"] == "attention" else case["tokens"], n)
    if case["kind"] == "attention":
        have = [max(h, q) for h, q in zip(_deal(rng, case["tokens"], n), new)]
    else:
        have = [h + q for h, q in zip(_deal(rng, case["before"], n), new)]
    return new, have


def _trees(case, new):
    rng = random.Random(case["split"] + 1)
    return [_tree(rng, n) for n in new]


# ---- inputs ------------------------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", dtype=torch.float32, generator=gen)


def _unit(x):
    return x / x.square().mean(-1, keepdim=True).sqrt()


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _offsets(lens):
    return _ints([0] + lens).cumsum(0).to(torch.int32)


def _pages(case, have, gen):
    """a table of pages in no order, and how many there are"""
    page = case["page"]
    need = [(h + page - 1) // page for h in have]
    total = sum(need) + 3
    order = torch.randperm(total, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros(len(need), max(need), dtype=torch.int32, device="cuda")
    at = torch.arange(max(need), device="cuda")
    there = at[None, :] < _ints(need)[:, None]
    table[there] = order[:sum(need)]
    return table, total


def _bits(trees, new):
    """for each new token a bit for each one of its sequence that it sees: itself and those above it"""
    words = (max(new) + 31) // 32
    rows = []
    for parents, _ in trees:
        masks = []
        for i, p in enumerate(parents):
            masks.append((masks[p] if p >= 0 else 0) | 1 << i)
        for m in masks:
            w = [m >> (32 * j) & 0xFFFFFFFF for j in range(words)]
            rows.append([x - (1 << 32) if x >> 31 else x for x in w])
    return _ints(rows)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s, kind = dict(case), case["kind"]
    if kind == "verify":
        return _prepare_verify(s, gen)
    kv, dim = case["kv"], case["dim"]
    bf = torch.bfloat16
    if kind == "rope":
        n, dtype = case["tokens"], bf if case["type"] == "bf16" else torch.float32
        for name, width in (("q", case["heads"] * dim), ("k", kv * dim)):
            s[name] = _normal(gen, n, width).to(dtype)
            s[name + "o"] = torch.empty_like(s[name])
        s["positions"] = torch.randint(0, case["far"], (n,), device="cuda", generator=gen).to(torch.int32)
        return s
    new, have = _lengths(case)
    n = sum(new)
    table, pages = _pages(case, have, gen)
    k_len, cu = _ints(have), _offsets(new)
    s.update(table=table, k_len=k_len, cu=cu, max_new=max(new), max_have=max(have))
    # keys as their norms leave them, with directions that a head's tokens share
    s["kc"] = (1.3 * _unit(_normal(gen, pages, case["page"], kv, dim) + 0.5 * _normal(gen, 1, 1, kv, dim))).to(bf)
    s["vc"] = _normal(gen, pages, case["page"], kv, dim).to(bf)
    trees = _trees(case, new) if case.get("form", "tree") == "tree" else None
    if kind == "keep":
        # (a path from the root to a leaf of each tree, as far as it is accepted)
        rng = random.Random(int(seed))
        rows, kept = [], []
        for parents, depth in trees:
            path, i = [], rng.randrange(len(parents))
            while i > 0:
                path.insert(0, i)
                i = parents[i]
            rows += path + [-1] * (len(parents) - len(path))
            kept.append(len(path))
        s.update(rows=_ints(rows), kept=_ints(kept))
        return s
    heads = case["heads"]
    if kind == "append":
        s.update(q=(_normal(gen, n, heads * dim) * 0.7).to(bf), k=(_normal(gen, n, kv * dim) * 1.3).to(bf), v=_normal(gen, n, kv * dim).to(bf),
                 qo=torch.empty(n, heads * dim, dtype=bf, device="cuda"), q_gain=None, k_gain=None, positions=None)
        if case["norm"]:
            s.update(q_gain=1.0 + 0.1 * _normal(gen, dim), k_gain=1.0 + 0.1 * _normal(gen, dim))
        if trees:
            # a drafted token's position goes by its depth
            s["positions"] = torch.cat([torch.tensor(depth) + h - m for (_, depth), h, m in zip(trees, have, new)]).to(torch.int32).cuda()
        return s
    s.update(q=(1.3 * _unit(_normal(gen, n, heads, dim) + 0.5)).reshape(n, -1).to(bf), out=torch.empty(n, heads * dim, dtype=bf, device="cuda"),
             tree=_bits(trees, new) if trees else None)
    return s


def _prepare_verify(s, gen):
    n, nodes, vocab = s["seqs"], s["nodes"], s["vocab"]
    dtype = torch.bfloat16 if s["type"] == "bf16" else torch.float32
    logits = 2.5 * _normal(gen, n * nodes, vocab)
    s.update(p=torch.softmax(logits, -1).to(dtype), q=None, parents=None, cu=_offsets([nodes] * n),
             uniforms=torch.rand(n * nodes, device="cuda", generator=gen), out_tokens=torch.empty(n * nodes, dtype=torch.int32, device="cuda"),
             out_rows=torch.empty(n * nodes, dtype=torch.int32, device="cuda"), accepted=torch.empty(n, dtype=torch.int32, device="cuda"))
    logits += 0.7 * _normal(gen, n * nodes, vocab)                 # the draft's
    if s["form"] == "chain":
        # a row's token is drawn from the draft's probabilities behind the row before it
        logits = logits.roll(1, 0)
        s["tokens"] = (logits - _normal(gen, n * nodes, vocab).uniform_(1e-20, 1.0, generator=gen).log_().neg_().log_()).argmax(-1).to(torch.int32)
        s["q"] = torch.softmax(logits, -1).to(dtype)
        return s
    trees = _trees(s, [nodes] * n)
    parents, child = [], []
    for of, _ in trees:
        seen = [0] * nodes
        for p in of:
            parents.append(p)
            child.append(seen[p] if p >= 0 else 0)
            seen[p] += p >= 0
    s["parents"] = _ints(parents)
    # a node's children are its likeliest tokens by the draft
    best = logits.topk(max(child) + 1, -1).indices
    row = torch.arange(n * nodes, device="cuda") // nodes * nodes + s["parents"].clamp(min=0)
    s["tokens"] = best[row, _ints(child).long()].to(torch.int32)
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------
def _frequencies(rot, theta, scaling):
    """angle of a position's step for each pair, as the far context has it"""
    half, a = rot // 2, SCALED[scaling]
    i = torch.arange(half, device="cuda", dtype=torch.float64)
    f = theta ** (-i / half)
    if scaling == "linear":
        return f / a["factor"]
    if scaling == "turns":
        keep = ((a["original"] / (2 * math.pi) * f - a["low"]) / (a["high"] - a["low"])).clamp(0, 1)
        return f * (keep + (1 - keep) / a["factor"])
    if scaling == "dims":
        at = lambda turns: rot * math.log(a["original"] / (2 * math.pi * turns)) / (2 * math.log(theta))
        lo, hi = max(math.floor(at(a["high"])), 0), min(math.ceil(at(a["low"])), rot - 1)
        keep = 1 - ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (keep + (1 - keep) / a["factor"])
    return f


def _rotate(x, positions, dim, rot, inter, scaling, back=False):
    """[n][heads * dim] in 32 bits, turned"""
    magnitude = SCALED[scaling].get("magnitude", 1.0)
    a = positions.double()[:, None, None] * _frequencies(rot, THETA, scaling)
    cos, sin = torch.cos(a).float() * magnitude, torch.sin(a).float() * (-magnitude if back else magnitude)
    x = x.view(x.shape[0], -1, dim)
    t = x[..., :rot]
    u, w = (t[..., 0::2], t[..., 1::2]) if inter else (t[..., :rot // 2], t[..., rot // 2:])
    u, w = u * cos - w * sin, w * cos + u * sin
    t = torch.stack((u, w), -1).flatten(-2) if inter else torch.cat((u, w), -1)
    return torch.cat((t, x[..., rot:]), -1).flatten(1)


def _norm(x, gain, dim):
    x = x.view(x.shape[0], -1, dim)
    return (gain * x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)).flatten(1)


def _places(s):
    """which sequence each new token is of, and its place in it"""
    n = s["q"].shape[0] if "q" in s else s["rows"].shape[0]
    tok = torch.arange(n, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["cu"], tok, right=True) - 1
    return seq, tok - s["cu"][seq + 1] + s["k_len"][seq]


def _page_rows(s, seq, place):
    return s["table"][seq, (place // s["page"]).long()].long() * s["page"] + place % s["page"]


def _append(s):
    q, k, dim = s["q"].float(), s["k"].float(), s["dim"]
    seq, place = _places(s)
    if s["norm"]:
        q, k = _norm(q, s["q_gain"], dim), _norm(k, s["k_gain"], dim)
    pos = place if s["positions"] is None else s["positions"]
    q, k = (_rotate(x, pos, dim, dim, s["inter"], "plain").to(torch.bfloat16) for x in (q, k))
    rows = _page_rows(s, seq, place)
    s["kc"].view(-1, k.shape[1])[rows] = k
    s["vc"].view(-1, k.shape[1])[rows] = s["v"]
    return {"q": q, "k": s["kc"], "v": s["vc"]}


def _keep(s):
    seq, _ = _places(s)
    j = torch.arange(seq.shape[0], device="cuda", dtype=torch.int32) - s["cu"][seq]
    base = s["k_len"][seq] - (s["cu"][seq + 1] - s["cu"][seq])
    moved = j < s["kept"][seq]
    # (those that are not moved: each place onto itself)
    last = s["cu"][seq + 1] - s["cu"][seq] - 1
    to = torch.where(moved, j + 1, torch.where(j + 1 > last, 0, j + 1))
    source = _page_rows(s, seq, base + torch.where(moved, s["rows"], to))
    to = _page_rows(s, seq, base + to)
    for c in (s["kc"], s["vc"]):
        flat = c.view(-1, s["kv"] * s["dim"])
        flat[to] = flat[source]
    return {"k": s["kc"], "v": s["vc"]}


def _attention(s):
    heads, kv, dim, n_seq = s["heads"], s["kv"], s["dim"], s["seqs"]
    mq, mk = s["max_new"], s["max_have"]
    new = s["cu"][1:] - s["cu"][:-1]
    at_q, at_k = torch.arange(mq, device="cuda"), torch.arange(mk, device="cuda")
    q_there, k_there = at_q[None, :] < new[:, None], at_k[None, :] < s["k_len"][:, None]
    q_rows = torch.where(q_there, s["cu"][:-1, None].long() + at_q, 0)
    k_rows = torch.where(k_there, _page_rows(s, torch.arange(n_seq, device="cuda")[:, None], at_k[None, :]), 0)
    q = s["q"].float()[q_rows].view(n_seq, mq, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(n_seq, kv, -1, dim)
    k, v = (c.view(-1, kv, dim)[k_rows].float().permute(0, 2, 1, 3).contiguous() for c in (s["kc"], s["vc"]))
    before = s["k_len"] - new
    rel = at_k[None, :] - before[:, None]                                     # [sequence][key]: which new token it is
    if s["tree"] is None:
        seen = rel[:, None, :] <= at_q[None, :, None]
    else:
        words = s["tree"][q_rows]                                             # [sequence][query][word]
        r = rel.clamp(0, 32 * words.shape[2] - 1)
        word = words.gather(2, (r // 32)[:, None, :].expand(-1, mq, -1))
        seen = (rel < 0)[:, None, :] | ((word >> (r % 32)[:, None, :]) & 1).bool()
    hidden = (~(seen & k_there[:, None, :]))[:, None, None]                   # [sequence][1][1][query][key]
    p = q @ k.transpose(-1, -2).contiguous()
    p.mul_(dim ** -0.5).view(n_seq, kv, heads // kv, mq, mk).masked_fill_(hidden, -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0, 1.0, total))
    out = (p @ v).view(n_seq, kv, heads // kv, mq, dim).permute(0, 3, 1, 2, 4).reshape(n_seq, mq, heads * dim)
    return out[q_there].to(torch.bfloat16)


def _verify(s):
    p, n_seq, nodes = s["p"], s["seqs"], s["nodes"]
    start = s["cu"][:-1].long()
    seqs = torch.arange(n_seq, device="cuda")
    tokens = s["tokens"].long()
    at = torch.zeros(n_seq, dtype=torch.long, device="cuda")                  # the node that has been reached
    left = torch.ones(n_seq, dtype=torch.float64, device="cuda")              # what is left of its probabilities
    count = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    refused = torch.zeros(n_seq, dtype=torch.long, device="cuda")             # a chain's row that was
    out_tokens = torch.full((n_seq, nodes), -1, dtype=torch.int32, device="cuda")
    out_rows = torch.full((n_seq, nodes), -1, dtype=torch.int32, device="cuda")
    gone = torch.zeros(n_seq, s["vocab"], dtype=torch.bool, device="cuda")    # the reached node's refused tokens
    for i in range(1, nodes):
        tok = tokens[start + i]
        parent = torch.full_like(at, i - 1) if s["parents"] is None else s["parents"][start + i].long()
        tried = parent == at
        u, target = s["uniforms"][start + i].double(), p[start + at, tok].double()
        if s["q"] is not None:
            yes = tried & (u * s["q"][start + i, tok].double() < target)
            refused = torch.where(tried & ~yes, i, refused)
        else:
            target = torch.where(gone[seqs, tok], 0.0, target)
            yes = tried & (u * left < target)
            left = torch.where(yes, 1.0, torch.where(tried, left - target, left))
            gone = gone & ~yes[:, None]
            gone[seqs, tok] = gone[seqs, tok] | (tried & ~yes)
        spot = count.long()
        out_tokens[seqs, spot] = torch.where(yes, tok.int(), out_tokens[seqs, spot])
        out_rows[seqs, spot] = torch.where(yes, i, out_rows[seqs, spot])
        count = count + yes
        at = torch.where(yes, i, at)
    whole = p[start + at].double()
    w = whole
    if s["q"] is not None:
        w = torch.where((refused > 0)[:, None], (whole - s["q"][start + refused].double()).clamp(min=0), whole)
    else:
        w = torch.where(gone, 0.0, whole)
    w = torch.where((w.sum(-1, keepdim=True) > 0), w, whole)
    sums = w.cumsum(-1)
    above = sums > s["uniforms"][start].double()[:, None] * sums[:, -1:]
    # the first that is above, of those that have any weight; else the last that has
    able = w > 0
    first = (above & able).int().argmax(-1)
    last = s["vocab"] - 1 - able.flip(-1).int().argmax(-1)
    token = torch.where((above & able).any(-1), first, torch.where(able.any(-1), last, -1))
    out_tokens[seqs, count.long()] = token.int()
    return {"tokens": out_tokens.view(-1), "rows": out_rows.view(-1), "accepted": count}


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
    kind = s["kind"]
    if kind == "rope":
        scalings = {"plain": binding.ROPE_PLAIN, "linear": binding.ROPE_LINEAR, "turns": binding.ROPE_TURNS, "dims": binding.ROPE_DIMS}
        rope = binding.make_rope(s["rot"], THETA, interleaved=s["inter"], scaling=scalings[s["scaling"]], **SCALED[s["scaling"]])
        (ctx.glue_rope_backward if s["grad"] else ctx.glue_rope)(rope, s["q"], s["k"], s["positions"], s["qo"], s["ko"], s["dim"])
        return {"q": s["qo"], "k": s["ko"]}
    if kind == "verify":
        ctx.verify_drafts(s["p"], s["q"], s["tokens"], s["uniforms"], s["cu"], s["out_tokens"], s["out_rows"], s["accepted"], parents=s["parents"])
        return {"tokens": s["out_tokens"], "rows": s["out_rows"], "accepted": s["accepted"]}
    cache = binding.make_cache(s["kc"], s["vc"], s["table"], s["k_len"])
    if kind == "append":
        ctx.glue_cache_append(cache, binding.make_rope(s["dim"], THETA, interleaved=s["inter"]), s["q"], s["k"], s["v"], s["qo"], s["cu"], positions=s["positions"],
                              q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS if s["norm"] else None)
        return {"q": s["qo"], "k": s["kc"], "v": s["vc"]}
    if kind == "keep":
        ctx.glue_cache_keep(cache, s["cu"], s["rows"], s["kept"])
        return {"k": s["kc"], "v": s["vc"]}
    ctx.glue_attention_paged(cache, s["q"], s["out"], s["cu"], tree=s["tree"])
    return s["out"]


def run(state):
    s = state
    if own:
        return _own(s)
    if s["kind"] == "rope":
        return {n: _rotate(s[n].float(), s["positions"], s["dim"], s["rot"], s["inter"], s["scaling"], s["grad"]).to(s[n].dtype) for n in ("q", "k")}
    return {"append": _append, "keep": _keep, "attention": _attention, "verify": _verify}[s["kind"]](s)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "verify":
        # one row of probabilities for each sequence, and of the draft's
        n = case["seqs"] * case["vocab"] * (2 if case["form"] == "chain" else 1)
        return {"bytes": n * (4 if case["type"] == "f32" else 2) + 20 * case["seqs"] * case["nodes"], "flops": 2.0 * n}
    kv, dim = case["kv"], case["dim"]
    if kind == "rope":
        n = case["tokens"] * (case["heads"] + kv)
        return {"bytes": 2 * n * dim * (2 if case["type"] == "bf16" else 4) + 4 * case["tokens"], "flops": 3.0 * n * case["rot"]}
    if kind == "keep":
        # (half of a tree's depth is accepted, half of it from branches)
        moved = case["seqs"] * min(4, case["nodes"]) / 2
        return {"bytes": int(moved * 2 * kv * dim * 2 * 2) + 8 * case["seqs"], "flops": 0.0}
    new, have = _lengths(case)
    n, heads = sum(new), case["heads"]
    if kind == "append":
        return {"bytes": 2 * 2 * n * (heads + 2 * kv) * dim + 8 * len(new), "flops": n * (heads + kv) * dim * (6.0 if case["norm"] else 3.0)}
    if case["form"] == "tree":
        pairs = sum(q * (k - q) + sum(d + 1 for d in depth) for q, k, (_, depth) in zip(new, have, _trees(case, new)))
    else:
        pairs = sum(q * (k - q) + q * (q + 1) // 2 for q, k in zip(new, have))
    return {"bytes": 2 * (2 * n * heads * dim + 2 * sum(have) * kv * dim) + 4 * case["seqs"] * (2 + max(have) // case["page"]), "flops": 4.0 * pairs * heads * dim}


# ---- from the definition, in 64 bits -----------------------------------------------------------------------------
def _exact_rotation(x, positions, dim, rot, inter, scaling, sign):
    n, half, a = x.shape[0], rot // 2, SCALED[scaling]
    steps = []
    for i in range(half):
        f = math.exp(-2.0 * i / rot * math.log(THETA))
        if scaling == "plain":
            m = 1.0
        elif scaling == "linear":
            m = 0.0
        elif scaling == "turns":
            m = (a["original"] * f / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])
        else:
            lo, hi = (rot / 2 * (math.log(a["original"]) - math.log(2 * math.pi * t)) / math.log(THETA) for t in (a["high"], a["low"]))
            lo, hi = max(0, math.floor(lo)), min(rot - 1, math.ceil(hi))
            m = 1.0 - (i - lo) / max(hi - lo, 0.001)
        m = min(1.0, max(0.0, m))
        steps.append(f * m + f * (1 - m) / a.get("factor", 1.0))
    turn = sign * positions.double()[:, None] * torch.tensor(steps, device="cuda", dtype=torch.float64)
    by = torch.polar(torch.full_like(turn, a.get("magnitude", 1.0)), turn)[:, None]
    y = x.double().reshape(n, -1, dim).clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, half), slice(half, rot))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * by
    y[..., first], y[..., second] = z.real, z.imag
    return y.reshape(n, -1)


def _exact_rows(case, s):
    """for each sequence the rows of its keys in the cache's pages"""
    table, out = s["table"].tolist(), []
    for t, h in zip(table, s["k_len"].tolist()):
        ids = torch.tensor(t, device="cuda")[:, None] * case["page"] + torch.arange(case["page"], device="cuda")
        out.append(ids.flatten()[:h])
    return out


def _exact_verify(case, s):
    n_seq, nodes = case["seqs"], case["nodes"]
    p, q = s["p"], s["q"]
    tokens, u = s["tokens"].tolist(), s["uniforms"].double().tolist()
    parents = None if s["parents"] is None else s["parents"].tolist()
    idx = torch.arange(n_seq * nodes, device="cuda")
    above = idx - 1 if parents is None else idx // nodes * nodes + s["parents"].long()
    target = p[above.clamp(min=0), s["tokens"].long()].double().tolist()       # what its parent's row has for each token
    draft = None if q is None else q[idx, s["tokens"].long()].double().tolist()
    out_tokens, out_rows, accepted = [-1] * (n_seq * nodes), [-1] * (n_seq * nodes), []
    for b in range(n_seq):
        r0, at, n, refused, spent = b * nodes, 0, 0, [], 0.0
        more = True
        while more:
            more = False
            refused, spent = [], 0.0
            for i in range(at + 1, nodes):
                if (i - 1 if parents is None else parents[r0 + i]) != at:
                    continue
                r = r0 + i
                mass = 0.0 if tokens[r] in [tokens[r0 + j] for j in refused] else target[r]
                if u[r] * (1.0 - spent if draft is None else draft[r]) < mass:
                    out_tokens[r0 + n], out_rows[r0 + n] = tokens[r], i
                    n, at, more = n + 1, i, True
                    break
                refused.append(i)
                spent += mass
        w = p[r0 + at].double()
        if refused and draft is not None:
            w = torch.relu(w - q[r0 + refused[-1]].double())
        elif refused:
            w = w.index_fill(0, torch.tensor([tokens[r0 + j] for j in refused], device="cuda"), 0.0)
        if not float(w.sum()) > 0:
            w = p[r0 + at].double()
        live = w.nonzero()[:, 0]
        sums = w[live].cumsum(0)
        hit = torch.searchsorted(sums, (u[r0] * sums[-1:]).contiguous(), right=True).clamp(max=live.numel() - 1)
        out_tokens[r0 + n] = int(live[hit])
        accepted.append(n)
    return {"tokens": _ints(out_tokens), "rows": _ints(out_rows), "accepted": _ints(accepted)}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "verify":
        return _exact_verify(case, s)
    dim, kv = case["dim"], case["kv"]
    if kind == "rope":
        return {n: _exact_rotation(s[n], s["positions"], dim, case["rot"], case["inter"], case["scaling"], -1.0 if case["grad"] else 1.0) for n in ("q", "k")}
    rows, cu = _exact_rows(case, s), s["cu"].tolist()
    new = [b - a for a, b in zip(cu, cu[1:])]
    if kind == "keep":
        kc, vc = s["kc"].clone(), s["vc"].clone()
        at, kept = s["rows"].tolist(), s["kept"].tolist()
        for b, r in enumerate(rows):
            r = r[len(r) - new[b]:]
            path = torch.tensor(at[cu[b]:cu[b] + kept[b]], device="cuda", dtype=torch.long)
            for to, of in ((kc, s["kc"]), (vc, s["vc"])):
                to.view(-1, kv * dim)[r[1:1 + kept[b]]] = of.view(-1, kv * dim)[r[path]]
        return {"k": kc, "v": vc}
    if kind == "append":
        place = torch.cat([torch.arange(len(r) - n, len(r), device="cuda") for r, n in zip(rows, new)])
        pos = place if s["positions"] is None else s["positions"]
        res = {}
        for name in ("q", "k"):
            x = s[name].double().reshape(len(place), -1, dim)
            if case["norm"]:
                x = x * s[name + "_gain"].double() / (x.pow(2).sum(-1, keepdim=True) / dim + EPS).sqrt()
            res[name] = _exact_rotation(x.flatten(1), pos, dim, dim, case["inter"], "plain", 1.0)
        to = torch.cat([r[len(r) - n:] for r, n in zip(rows, new)])
        kc, vc = s["kc"].double(), s["vc"].double()
        kc.view(-1, kv * dim)[to], vc.view(-1, kv * dim)[to] = res["k"], s["v"].double()
        return {"q": res["q"], "k": kc, "v": vc}
    heads = case["heads"]
    group = heads // kv
    out = torch.zeros(cu[-1], heads, dim, dtype=torch.float64, device="cuda")
    trees = _trees(case, new) if case["form"] == "tree" else None
    for b, r in enumerate(rows):
        n, before = new[b], len(r) - new[b]
        seen = torch.ones(n, n, dtype=torch.bool).tril()
        if trees:
            seen = torch.zeros(n, n, dtype=torch.bool)
            for i in range(n):
                j = i
                while j >= 0:
                    seen[i, j] = True
                    j = trees[b][0][j]
        hidden = torch.cat((torch.zeros(n, before, dtype=torch.bool), ~seen), 1).cuda()
        for g in range(kv):
            k, v = (c.view(-1, kv, dim)[r, g].double() for c in (s["kc"], s["vc"]))
            x = s["q"].view(-1, heads, dim)[cu[b]:cu[b + 1], g * group:(g + 1) * group].double().transpose(0, 1).reshape(-1, dim)
            z = (torch.mm(x, k.t()) / math.sqrt(dim)).view(group, n, -1).masked_fill(hidden, -math.inf)
            y = torch.mm(torch.softmax(z, -1).view(group * n, -1), v)
            out[cu[b]:cu[b + 1], g * group:(g + 1) * group] = y.view(group, n, dim).transpose(0, 1)
    return out.flatten(1)
