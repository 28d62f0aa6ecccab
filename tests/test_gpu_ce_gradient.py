"""Token cross-entropy with the sums' logarithms, and its gradient for inputs and weights, against a 64-bit form with element-wise bounds."""
import pytest
import torch

from paper_2601_17261_amd import binding

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


def make(seed, n, d, v, ignored=0.2, dtype=torch.bfloat16, pad=0, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn(v, d + pad, device="cuda", generator=gen) * std / d ** 0.5).to(dtype)[:, :d]
    x = torch.randn(n, d + pad, device="cuda", generator=gen).to(dtype)[:, :d]
    ids = torch.randint(0, v, (n,), device="cuda", generator=gen)
    ids[torch.rand(n, device="cuda", generator=gen) < ignored] = -1
    return w, x, ids.int()


def exact(w, x, ids, g=1.0):
    w, x, ids = w.double(), x.double(), ids.long()
    y = x @ w.T
    lse = y.logsumexp(1)
    rows = ((ids >= 0) & (ids < w.shape[0])).nonzero()[:, 0]
    count = max(1, rows.numel())
    d = torch.zeros_like(y)
    d[rows] = (y[rows] - lse[rows, None]).exp()
    d[rows, ids[rows]] -= 1.0
    d *= g / count
    loss = (lse[rows] - y[rows, ids[rows]]).sum() / count
    return {"loss": loss, "lse": lse, "d": d, "dx": d @ w, "dw": d.T @ x,
            # half a step of D and of the result; fp32 logits and sums
            "dx_off": (HALF + 4e-5) * (d.abs() @ w.abs()) + HALF * (d @ w).abs(), "dw_off": (HALF + 4e-5) * (d.abs().T @ x.abs()) + HALF * (d.T @ x).abs()}


def run(ctx, w, x, ids, g=None, dx=True, dw=True):
    L, loss = binding.make_layer(w, x), binding.make_loss(ids, binding.LOSS_CE)
    r = {"loss": torch.full((1,), 7.0, dtype=torch.float64, device="cuda"), "lse": torch.full((x.shape[0],), 7.0, device="cuda")}
    ctx.ce_forward(L, w, x, loss, r["loss"], r["lse"])
    if dx or dw:
        r["dx"], r["dw"] = torch.full_like(x, 7.0) if dx else None, torch.full_like(w, 7.0) if dw else None
        ctx.ce_backward(L, w, x, loss, r["lse"], r["dx"], r["dw"], g)
    return r


def check(got, want):
    assert abs(float(got["loss"]) - float(want["loss"])) <= 2e-6 * max(1.0, abs(float(want["loss"])))
    assert (got["lse"].double() - want["lse"]).abs().max() <= 2e-6 * max(1.0, float(want["lse"].abs().max()))
    for n in ("dx", "dw"):
        if got.get(n) is not None:
            bad = ~((got[n].double() - want[n]).abs() <= want[n + "_off"] + 1e-30)
            assert not bad.any(), (n, int(bad.sum()), bad.nonzero()[:3].tolist(), got[n][bad][:3].tolist(), want[n][bad][:3].tolist())


@pytest.mark.parametrize("n,d,v,pad", [
    (1, 8, 1, 0), (1, 64, 2, 0), (3, 40, 7, 8), (7, 2048, 999, 0), (63, 72, 64, 0), (64, 64, 65, 16), (65, 136, 257, 0), (200, 256, 1000, 0),
    (256, 128, 256, 0), (257, 264, 4097, 8), (256, 256, 512, 0), (512, 128, 768, 0), (300, 512, 12345, 0), (1000, 1024, 5000, 0), (5, 16, 140000, 0), (70, 8, 300001, 0),
    # blocks of 32 tokens, the last outputs and tokens alone
    (33, 72, 1000, 0), (96, 264, 1025, 8), (129, 512, 2000, 0), (255, 1000, 7000, 0), (255, 128, 7300, 0), (161, 2488, 4588, 0),
    # several pieces of the outputs
    (2049, 64, 70001, 0), (40, 8192, 33000, 0)])
def test_loss_and_gradients(n, d, v, pad):
    ctx = binding.Context()
    w, x, ids = make(n + v, n, d, v, pad=pad)
    if n > 2:
        ids[1] = v + 3                      # no output: not counted
    check(run(ctx, w, x, ids), exact(w, x, ids))


def test_one_of_the_gradients_and_an_upstream_one():
    ctx = binding.Context()
    w, x, ids = make(4, 300, 256, 2000)
    g = torch.tensor([-0.75], dtype=torch.float64, device="cuda")
    want = exact(w, x, ids, -0.75)
    both = run(ctx, w, x, ids, g)
    check(both, {**want})
    for kw in (dict(dx=False), dict(dw=False)):
        r = run(ctx, w, x, ids, g, **kw)
        assert all(torch.equal(r[n], both[n]) for n in ("dx", "dw") if r[n] is not None)


@pytest.mark.parametrize("n,d,v,pad", [(1, 1, 1, 0), (3, 5, 7, 2), (33, 65, 129, 1), (200, 100, 1001, 0), (700, 384, 5000, 4),
                                       # several pieces of the outputs
                                       (3, 40, 7000001, 0)])
def test_layers_in_fp32(n, d, v, pad):
    ctx = binding.Context()
    w, x, ids = make(n + v, n, d, v, dtype=torch.float32, pad=pad)
    ids[0] = v - 1
    if n > 2:
        ids[1] = v + 3
    want, got = exact(w, x, ids), run(ctx, w, x, ids)
    # steps of 2^-24: a logit's, lse's, their difference's and the exponential's to D, three of the results' and one a piece
    u, W, X = 2.0 ** -24, w.double().abs(), x.double().abs()
    y = x.double() @ w.double().T
    p = torch.where(want["d"] != 0, (y - want["lse"][:, None]).exp(), 0.0)
    count = max(1, int(((ids >= 0) & (ids < v)).sum()))
    off = u * (p * (2 * y.abs() + 2 * want["lse"].abs()[:, None] + 8) / count + 2 * want["d"].abs())
    assert abs(float(got["loss"]) - float(want["loss"])) <= 2e-6 * max(1.0, abs(float(want["loss"])))
    for name, bound in (("dx", off @ W + 6 * u * (want["d"].abs() @ W)), ("dw", off.T @ X + 6 * u * (want["d"].abs().T @ X))):
        bad = ~((got[name].double() - want[name]).abs() <= bound + 1e-37)
        assert not bad.any(), (name, int(bad.sum()), float(((got[name].double() - want[name]).abs() - bound).max()))


def test_fp32_rows_that_are_not_counted_one_gradient_and_refusals():
    ctx = binding.Context()
    w, x, ids = make(6, 50, 33, 90, dtype=torch.float32)
    ids[7] = -1
    both = run(ctx, w, x, ids)
    assert (both["dx"][7] == 0).all()
    y = x.clone()
    y[7] = float("nan")
    L, loss = binding.make_layer(w, y), binding.make_loss(ids, binding.LOSS_CE)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ctx.ce_backward(L, w, y, loss, both["lse"], dx, dw)
    assert torch.equal(dw, both["dw"]) and torch.equal(dx, both["dx"])
    for kw in (dict(dx=False), dict(dw=False)):
        r = run(ctx, w, x, ids, **kw)
        assert all(torch.equal(r[n], both[n]) for n in ("dx", "dw") if r[n] is not None)
    L = binding.make_layer(w, x)
    with pytest.raises(TypeError):
        ctx.ce_backward(L, w, x, loss, both["lse"], dx.bfloat16(), dw)
    with pytest.raises(binding.AgzoError):
        ctx.ce_backward(L, w, x, loss, both["lse"], x, dw)
    with pytest.raises(binding.AgzoError):
        ctx.ce_backward(L, w, x, loss, both["lse"], dw[:50], dw)


def test_no_row_counted():
    ctx = binding.Context()
    w, x, ids = make(5, 40, 64, 300)
    ids[:] = -1
    r = run(ctx, w, x, ids)
    assert float(r["loss"]) == 0.0 and not r["dx"].any() and not r["dw"].any()
    assert (r["lse"].double() - (x.double() @ w.double().T).logsumexp(1)).abs().max() < 1e-5


def test_rows_that_are_not_counted_have_no_part():
    """NaN and infinities in the inputs of rows that are not counted show in their lse alone."""
    ctx = binding.Context()
    w, x, ids = make(6, 300, 128, 700)
    ids[17], ids[250] = -1, 700
    clean = run(ctx, w, x, ids)
    x2 = x.clone()
    x2[17], x2[250] = float("nan"), float("inf")
    got = run(ctx, w, x2, ids)
    assert not got["dx"][17].any() and all(torch.equal(got[n], clean[n]) for n in ("dx", "dw", "loss"))
    there = torch.ones(300, dtype=torch.bool, device="cuda")
    there[[17, 250]] = False
    assert torch.equal(got["lse"][there], clean["lse"][there])


def test_confident_rows_and_large_logits():
    """Logits of some hundreds: one-hot softmaxes, of which some are right (the gradient is 0) and some wrong."""
    ctx = binding.Context()
    w, x, ids = make(7, 280, 256, 600, std=30.0)
    y = x.double() @ w.double().T
    ids[:140] = y[:140].argmax(1).int()
    want = exact(w, x, ids)
    got = run(ctx, w, x, ids)
    # fp32 logits of up to some 150 are off by 150 * 2^-20, and so are probabilities
    for n, m in (("dx", want["d"].abs() @ w.double().abs()), ("dw", want["d"].abs().T @ x.double().abs())):
        want[n + "_off"] = want[n + "_off"] + 3e-4 * m
    p = (want["d"].abs() * 0 + (y - want["lse"][:, None]).exp()) * (ids >= 0)[:, None] / (ids >= 0).sum()
    want["dx_off"] = want["dx_off"] + 3e-4 * (p @ w.double().abs())
    want["dw_off"] = want["dw_off"] + 3e-4 * (p.T @ x.double().abs())
    assert abs(float(got["loss"]) - float(want["loss"])) <= 1e-5 * float(want["loss"])
    got["loss"] = want["loss"]
    want["lse"] = got["lse"].double() + (want["lse"] - got["lse"].double()) * ((want["lse"] - got["lse"].double()).abs() > 3e-4)
    check(got, want)


def test_the_loss_is_the_forwards_bit_for_bit():
    ctx = binding.Context()
    for n, d, v, dtype in ((300, 256, 1000, torch.bfloat16), (1024, 512, 2048, torch.bfloat16), (40, 64, 90, torch.float32)):
        w, x, ids = make(8, n, d, v, dtype=dtype)
        L, loss = binding.make_layer(w, x), binding.make_loss(ids, binding.LOSS_CE)
        a, b = (torch.zeros(1, dtype=torch.float64, device="cuda") for _ in range(2))
        ctx.layer_forward_sketch(L, w, x, None, binding.SKETCH_NONE, None, 0, None, loss, a)
        lse = torch.empty(n, device="cuda")
        ctx.ce_forward(L, w, x, loss, b, lse)
        assert torch.equal(a, b)
        assert (lse.double() - (x.double() @ w.double().T).logsumexp(1)).abs().max() < 1e-5
        ctx.ce_forward(L, w, x, loss, b)
        assert torch.equal(a, b)


def test_gradient_against_differences():
    ctx = binding.Context()
    w, x, ids = make(9, 90, 128, 500)
    got = run(ctx, w, x, ids)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for name, t in (("dx", x), ("dw", w)):
        way = torch.randn(t.shape, device="cuda", generator=gen).double()
        f = [exact(w.double() + (s * 1e-4 * way if name == "dw" else 0), x.double() + (s * 1e-4 * way if name == "dx" else 0), ids)["loss"] for s in (1, -1)]
        slope, mine = (f[0] - f[1]) / 2e-4, (got[name].double() * way).sum()
        assert (slope - mine).abs() <= 4 * HALF * (got[name].double() * way).norm() + 1e-5 * slope.abs(), name


def test_repeated_captured_and_on_another_stream():
    st = torch.cuda.Stream()
    w, x, ids = make(10, 400, 256, 3000)
    first = run(binding.Context(), w, x, ids)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        ctx = binding.Context(stream=st)
        r = run(ctx, w, x, ids)
        assert all(torch.equal(r[n], first[n]) for n in r)
        L, loss = binding.make_layer(w, x), binding.make_loss(ids, binding.LOSS_CE)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            ctx.ce_forward(L, w, x, loss, r["loss"], r["lse"])
            ctx.ce_backward(L, w, x, loss, r["lse"], r["dx"], r["dw"])
        for seed in range(3):
            w2, x2, ids2 = make(20 + seed, 400, 256, 3000)
            for a, b in ((w, w2), (x, x2), (ids, ids2)):
                a.copy_(b)
            graph.replay()
            st.synchronize()
            got = {n: t.clone() for n, t in r.items()}
            want = run(ctx, w, x, ids)
            run(ctx, *make(40 + seed, 500 * (seed + 1), 256, 4000))
            assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("n,d,v,dtype", [(1, 64, 500, torch.bfloat16), (29, 264, 3001, torch.bfloat16), (50, 128, 900, torch.bfloat16), (200, 256, 5000, torch.bfloat16), (70, 256, 30000, torch.bfloat16), (127, 512, 2000, torch.bfloat16),
                                         (600, 200, 700, torch.bfloat16), (60, 50, 333, torch.float32)])
def test_every_way_is_captured_and_repeats(n, d, v, dtype):
    st = torch.cuda.Stream()
    w, x, ids = make(n, n, d, v, dtype=dtype)
    w2, x2, ids2 = make(n + 1, n, d, v, dtype=dtype)
    plain = binding.Context()
    first, second = run(plain, w, x, ids), run(plain, w2, x2, ids2)
    assert all(torch.equal(first[k], t) for k, t in run(plain, w, x, ids).items())
    torch.cuda.synchronize()
    ctx = binding.Context(st)
    wc, xc, idc = w.clone(), x.clone(), ids.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        r = run(ctx, wc, xc, idc)
        L, loss = binding.make_layer(wc, xc), binding.make_loss(idc, binding.LOSS_CE)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            ctx.ce_forward(L, wc, xc, loss, r["loss"], r["lse"])
            ctx.ce_backward(L, wc, xc, loss, r["lse"], r["dx"], r["dw"])
    for data, want in (((w2, x2, ids2), second), ((w, x, ids), first), ((w2, x2, ids2), second)):
        for a, b in zip((wc, xc, idc), data):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(r[k], want[k]) for k in want)
        run(plain, w, x, ids)


def test_two_contexts_on_two_streams_at_once():
    sets = [make(50 + i, 7 + 200 * i, 1024, 9000) for i in range(2)]
    want = [run(binding.Context(), *s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    contexts = [binding.Context(s) for s in streams]
    outs = [[], []]
    for _ in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                outs[i].append(run(contexts[i], *sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for got in outs[i]:
            assert all(torch.equal(got[k], want[i][k]) for k in got)


def test_refusals():
    ctx = binding.Context()
    w, x, ids = make(11, 32, 64, 100)
    L, loss = binding.make_layer(w, x), binding.make_loss(ids, binding.LOSS_CE)
    out, lse = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(32, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    with pytest.raises(binding.AgzoError):
        ctx.ce_forward(L, w, x, binding.make_loss(None), out, lse)
    with pytest.raises(binding.AgzoError):
        ctx.ce_forward(L, w, x, loss, None, lse)
    with pytest.raises(ValueError):
        ctx.ce_forward(L, w, x, loss, out, lse[:8])
    with pytest.raises(TypeError):
        ctx.ce_forward(L, w, x, loss, out.float(), lse)
    with pytest.raises(binding.AgzoError):
        ctx.ce_backward(L, w, x, loss, None, dx, dw)
    with pytest.raises(binding.AgzoError):
        ctx.ce_backward(L, w, x, loss, lse, None, None)
    with pytest.raises(binding.AgzoError):
        ctx.ce_backward(L, w, x, loss, lse, x, dw)
    with pytest.raises(binding.AgzoError):
        ctx.ce_backward(L, w, x, loss, lse, dw[:32], dw)
    with pytest.raises(ValueError):
        ctx.ce_backward(L, w, x, loss, lse, dx[:5], dw)
    with pytest.raises(TypeError):
        ctx.ce_backward(L, w, x, loss, lse, dx.float(), dw)
