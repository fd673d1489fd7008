"""The loss over a vocabulary and its gradients against the definition in 64
bits, at sizes, strides, masks and values where they can go wrong."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # unit roundoff of the outputs
# of a softmax entry on its way into the gradient products: the numerator's rounding and the entry's (binary32: 22 bits)
UD = {"f32": 2.0 ** -20, "bf16": 2.0 ** -11 + 2.0 ** -8, "f16": 2 * 2.0 ** -11}
IGNORE = -100


@pytest.fixture(scope="module")
def head(tc):
    from paper_2401_07788_amd import head
    yield head
    head.free_workspaces()
    assert tc.device_errors() == 0


def inputs(n, v, h, dt, seed=0, scale=1.0, padx=0, padw=0, shift=0, skip=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def matrix(rows, std, pad):
        flat = torch.full((rows * (h + pad) + shift + 8,), float("nan"), dtype=DT[dt], device="cuda")
        m = flat[shift:shift + rows * (h + pad)].view(rows, h + pad)[:, :h]
        m.copy_(torch.randn(rows, h, generator=g, device="cuda").mul_(std))
        return m

    x, w = matrix(n, 1.0, padx), matrix(v, 1.5 * scale / math.sqrt(h), padw)
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    t[torch.rand(n, generator=g, device="cuda") < skip] = IGNORE
    return x, w, t


def reference(x, w, t, weight, v):
    keep = (t >= 0) & (t < v)
    rows = keep.nonzero()[:, 0]
    n, h = x.shape
    xd, wd = x[rows].double().cpu(), w.double().cpu()
    td, g = t[rows].cpu(), (torch.ones(n) if weight is None else weight.cpu())[rows.cpu()].double()[:, None]
    z = xd @ wd.t()
    lse = torch.logsumexp(z, 1) if rows.numel() else torch.zeros(0, dtype=torch.float64)
    at = torch.arange(rows.numel())
    out = {k: torch.zeros(n, dtype=torch.float64) for k in ("loss", "lse")}
    out["loss"][rows.cpu()], out["lse"][rows.cpu()] = lse - z[at, td], lse
    p = torch.exp(z - lse[:, None])
    hot = torch.zeros_like(p)
    hot[at, td] = 1
    d = g * (p - hot)
    dx = torch.zeros(n, h, dtype=torch.float64)
    dx[rows.cpu()] = d @ wd
    out["dx"], out["dw"] = dx, d.t() @ xd
    # what the products are made of, for the bounds
    size = g.abs() * (p + hot)
    big = torch.zeros(n, h, dtype=torch.float64)
    big[rows.cpu()] = size @ wd.abs()
    zs = torch.zeros(n, dtype=torch.float64)
    if rows.numel():
        zs[rows.cpu()] = (xd.abs() @ wd.abs().t()).amax(1)
    return out, {"dx": big, "dw": size.t() @ xd.abs(), "z": zs, "x": xd.abs().sum(0), "top": float(g.abs().max()) if g.numel() else 0.0}


def check(r, x, w, t, weight, dt, v):
    want, size = reference(x, w, t, weight, v)
    h = x.shape[1]
    # a logit: products of the inputs are exact (binary32: 22 bits on either side), h sums in binary32 whose
    # roundings add up as a random walk, four deviations
    uz = (4 * math.sqrt(h) + 8) * 2.0 ** -24 + (2.0 ** -20 if dt == "f32" else 0)
    ez = uz * size["z"]
    # exponentials and sums of positive terms: within 2^-19; the last roundings of lse and of the difference
    lim = 2 * ez + 2.0 ** -19 + 2.0 ** -22 * (want["lse"].abs() + want["loss"].abs())
    for k in ("loss", "lse"):
        got = getattr(r, k).double().cpu()
        assert torch.isfinite(got).all()
        assert bool(((got - want[k]).abs() <= lim).all()), (k, float(((got - want[k]).abs() - lim).max()))
        assert bool((got[(t < 0).cpu()] == 0).all())
    if not hasattr(r, "dx"):
        return
    # an entry is off by its roundings and, relatively, by its logit's and lse's error; the products' sums in binary32
    rel = UD[dt] + 3 * float(ez.max() if ez.numel() else 0) + 2.0 ** -18 + 64 * 2.0 ** -24
    low = 2.0 ** -38 if dt != "bf16" else 0.0                 # what binary16 operands reach down to
    g = torch.ones(x.shape[0]) if weight is None else weight.cpu()
    lim = rel * size["dx"] + U[dt] * want["dx"].abs() + (2.0 ** -24 if dt == "f16" else 1e-38) + \
        2 * low * g.double().abs()[:, None] * w.double().cpu().abs().sum(0)
    err = (r.dx.double().cpu() - want["dx"]).abs()
    assert bool((err <= lim).all()), ("dx", float((err - lim).max()), float(err.max()))
    lim = rel * size["dw"] + U[dt] * want["dw"].abs() + (2.0 ** -24 if dt == "f16" else 1e-38) + 2 * low * size["top"] * size["x"]
    err = (r.dw.double().cpu() - want["dw"]).abs()
    assert bool((err <= lim).all()), ("dw", float((err - lim).max()), float(err.max()))


SIZES = [(1, 1, 1), (1, 50, 64), (3, 2, 5), (17, 129, 33), (64, 255, 64), (65, 256, 32), (100, 257, 96), (128, 1000, 40),
         (129, 64, 300), (200, 65, 257), (333, 700, 128)]


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("n,v,h", SIZES)
def test_sizes(head, dt, n, v, h):
    x, w, t = inputs(n, v, h, dt, seed=n + v)
    weight = torch.rand(n, device="cuda") + 0.5
    check(head.linear_xent_step(x, w, t, weight), x, w, t, weight, dt, v)
    loss, lse = head.linear_xent(x, w, t)
    assert loss.shape == (n,)
    check(type("R", (), {"loss": loss, "lse": lse})(), x, w, t, weight, dt, v)


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("padx,padw,shift", [(8, 0, 0), (0, 24, 0), (3, 5, 0), (0, 0, 1), (64, 64, 8)])
def test_strides_and_addresses(head, dt, padx, padw, shift):
    n, v, h = 130, 300, 128
    x, w, t = inputs(n, v, h, dt, 1, padx=padx, padw=padw, shift=shift)
    check(head.linear_xent_step(x, w, t), x, w, t, None, dt, v)
    loss, lse = head.linear_xent(x, w, t)
    check(type("R", (), {"loss": loss, "lse": lse})(), x, w, t, None, dt, v)


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("skip", [0.5, 0.95, 1.0])
def test_tokens_that_do_not_count(head, dt, skip):
    """their rows of x may hold anything"""
    n, v, h = 300, 500, 72
    x, w, t = inputs(n, v, h, dt, 2, skip=skip)
    if skip == 1.0:
        t.fill_(IGNORE)
    x[t == IGNORE] = float("nan")
    x[(t == IGNORE).nonzero()[:1, 0]] = float("inf")
    r = head.linear_xent_step(x, w, t)
    assert torch.isfinite(r.dw).all()
    check(r, x, w, t, None, dt, v)
    assert not r.dx[t == IGNORE].any()
    if skip == 1.0:
        assert not r.dw.any() and not r.loss.any()
    loss, lse = head.linear_xent(x, w, t)
    assert torch.equal(loss, r.loss) and torch.equal(lse, r.lse)


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("chunk", [128, 192])
def test_chunks(head, dt, chunk):
    """more than one chunk, the last ones partly or wholly without tokens"""
    for n, skip in ((500, 0.0), (500, 0.4), (700, 0.9)):
        v, h = 260, 100
        x, w, t = inputs(n, v, h, dt, 3, skip=skip)
        weight = torch.rand(n, device="cuda")
        check(head.linear_xent_step(x, w, t, weight, chunk=chunk), x, w, t, weight, dt, v)
        loss, lse = head.linear_xent(x, w, t, chunk=chunk)
        check(type("R", (), {"loss": loss, "lse": lse})(), x, w, t, weight, dt, v)


@pytest.mark.parametrize("dt", list(DT))
def test_many_splits_and_pieces(head, dt):
    """few tokens and a long vocabulary: dx is summed in many parts"""
    n, v, h = 70, 20011, 48
    x, w, t = inputs(n, v, h, dt, 4)
    check(head.linear_xent_step(x, w, t), x, w, t, None, dt, v)


@pytest.mark.parametrize("dt", list(DT))
def test_far_logits(head, dt):
    """logits of some hundreds: one entry holds all of the softmax, others are far below the smallest number"""
    n, v, h = 90, 300, 64
    x, w, t = inputs(n, v, h, dt, 5, scale=60.0)
    check(head.linear_xent_step(x, w, t), x, w, t, None, dt, v)


@pytest.mark.parametrize("dt", list(DT))
def test_weights(head, dt):
    n, v, h = 100, 200, 64
    x, w, t = inputs(n, v, h, dt, 6)
    weight = torch.randn(n, device="cuda") * 1e-3
    weight[::3] = 0.0
    check(head.linear_xent_step(x, w, t, weight), x, w, t, weight, dt, v)
    zero = torch.zeros(n, device="cuda")
    r = head.linear_xent_step(x, w, t, zero)
    assert not r.dx.any() and not r.dw.any() and bool((r.loss > 0).any())


def test_binary32_far_scales(head):
    """the planes' scaling follows the largest magnitude"""
    for sx, sw in ((1e-20, 1e20), (1e15, 1e-15), (1e-3, 1e-3)):
        x, w, t = inputs(40, 100, 64, "f32", 7)
        x, w = x * sx, w * sw
        check(head.linear_xent_step(x, w, t), x, w, t, None, "f32", 100)
    x, w = torch.zeros(4, 64, device="cuda"), torch.zeros(7, 64, device="cuda")
    r = head.linear_xent_step(x, w, torch.zeros(4, dtype=torch.int64, device="cuda"))
    assert torch.allclose(r.loss, torch.full((4,), math.log(7), device="cuda"), atol=1e-6) and not r.dx.any() and not r.dw.any()


def test_target_outside_the_vocabulary(head, tc):
    x, w, t = inputs(20, 30, 16, "f32", 8)
    t[3], t[9] = 30, -5
    r = head.linear_xent_step(x, w, t)
    check(r, x, w, t, None, "f32", 30)
    assert float(r.loss[3]) == 0 and not r.dx[9].any()
    assert tc.device_errors() == tc.TC_KERR_BAD_INDEX
    head.linear_xent(x, w, t.clamp(0, 29), ignore_index=5)
    assert tc.device_errors() == 0


def test_no_tokens(head):
    x, w, t = inputs(0, 30, 16, "bf16", 9)
    r = head.linear_xent_step(x, w, t, out=None)
    assert r.loss.numel() == 0 and not r.dw.any()
    assert head.linear_xent(x, w, t)[0].numel() == 0


@pytest.mark.parametrize("dt", list(DT))
def test_gradients_against_differences(head, dt):
    """along random directions, differences of the 64-bit loss; through autograd"""
    n, v, h = 40, 150, 64
    x, w, t = inputs(n, v, h, dt, 10, skip=0.2)
    x, w = x.contiguous().requires_grad_(), w.contiguous().requires_grad_()
    weight = torch.rand(n, device="cuda")
    loss, _ = head.linear_xent(x, w, t)
    (loss * weight).sum().backward()

    def total(a, b):
        z = a @ b.t()
        keep = t != IGNORE
        one = torch.logsumexp(z, 1) - z.gather(1, t.clamp(min=0)[:, None])[:, 0]
        return float((one * weight.double())[keep].sum())

    xd, wd = x.detach().double(), w.detach().double()
    for k in range(3):
        a, b = torch.randn_like(xd), torch.randn_like(wd)
        e = 1e-4
        for u, p, g in ((a, 0, x.grad), (b, 1, w.grad)):
            plus = total(xd + e * u, wd) if p == 0 else total(xd, wd + e * u)
            minus = total(xd - e * u, wd) if p == 0 else total(xd, wd - e * u)
            # the differences themselves are good to e^2; a random direction sees the gradient's
            # relative error of 2 U + UD as a share of its length, six deviations
            lim = 6 * (2 * U[dt] + UD[dt]) * float(g.double().norm()) + 1e-5
            assert abs((plus - minus) / (2 * e) - float((g.double() * u).sum())) < lim


def test_same_bits_again_and_on_another_stream(head):
    x, w, t = inputs(300, 900, 64, "bf16", 11, skip=0.3)
    a = head.linear_xent_step(x, w, t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = head.linear_xent_step(x, w, t)
    side.synchronize()
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_replays_in_a_graph(head):
    """every replay, with eager work between, equals the eager result"""
    x, w, t = inputs(150, 600, 64, "bf16", 12, skip=0.3)
    x2, _, t2 = inputs(150, 600, 64, "bf16", 13, skip=0.6)
    out = head.linear_xent_step(x, w, t)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    xs, ts = x.clone(), t.clone()
    head.linear_xent_step(xs, w, ts, out=out, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        head.linear_xent_step(xs, w, ts, out=out, ws=ws)
    for k in range(4):
        a, b = ((x, t), (x2, t2))[k % 2]
        xs.copy_(a)
        ts.copy_(b)
        want = head.linear_xent_step(a, w, b)
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(out, want):
            assert torch.equal(p, q)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("first,count", [(0, 64), (64, 130), (190, 110), (3, 296)])
def test_logits_of_minus_infinity(head, dt, first, count):
    """entries that a row of w takes out: whole pieces of them, and all but a few"""
    n, v, h = 70, 300, 64
    x, w, t = inputs(n, v, h, dt, 14)
    x[:, 0] = 1.0
    out = torch.zeros(v, dtype=torch.bool, device="cuda")
    out[first:first + count] = True
    w[out] = 0.0
    w[out, 0] = -math.inf
    keep = (~out).nonzero()[:, 0]
    t = keep[t % len(keep)]
    r = head.linear_xent_step(x, w, t)
    place = torch.full((v,), -1, device="cuda")
    place[keep] = torch.arange(len(keep), device="cuda")
    dense = type("R", (), {"loss": r.loss, "lse": r.lse})()
    check(dense, x, w[keep], place[t], None, dt, len(keep))
    loss, lse = head.linear_xent(x, w, t)
    assert torch.equal(loss, r.loss) and torch.equal(lse, r.lse)
    # (dx holds 0 times -inf in every definition)
    want, size = reference(x, w[keep], place[t], None, len(keep))
    rel = UD[dt] + 2.0 ** -10
    assert not r.dw[out].any()
    lim = rel * size["dw"] + U[dt] * want["dw"].abs() + (2.0 ** -24 if dt == "f16" else 1e-38) + 2.0 ** -37 * size["x"]
    assert bool(((r.dw[keep].double().cpu() - want["dw"]).abs() <= lim).all())


@pytest.mark.parametrize("dt", list(DT))
def test_nan_entries_reach_every_loss(head, dt):
    n, v, h = 40, 300, 64
    x, w, t = inputs(n, v, h, dt, 15)
    w[128:192] = math.nan
    assert torch.isnan(head.linear_xent(x, w, t)[0]).all()
    assert torch.isnan(head.linear_xent_step(x, w, t).loss).all()


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_a_token_that_is_not_finite_spoils_no_other(head, dt, bad):
    n, v, h = 140, 300, 64
    x, w, t = inputs(n, v, h, dt, 16)
    weight = torch.rand(n, device="cuda") + 0.5
    others = torch.ones(n, dtype=torch.bool, device="cuda")
    others[33] = False
    for into_x in (True, False):
        x2, weight2 = x.clone(), weight.clone()
        if into_x:
            x2[33, 5] = bad
        else:
            weight2[33] = bad
        r = head.linear_xent_step(x2, w, t, weight2)
        assert torch.isnan(r.loss[33]) == into_x and not torch.isfinite(r.dx[33]).all()
        assert torch.isfinite(r.dx[others]).all() and torch.isfinite(r.loss[others]).all()
        part = type("R", (), {"loss": r.loss[others], "lse": r.lse[others]})()
        check(part, x[others], w, t[others], weight[others], dt, v)
        want, size = reference(x[others], w, t[others], weight[others], v)
        rel = UD[dt] + 2.0 ** -10
        lim = rel * size["dx"] + U[dt] * want["dx"].abs() + (2.0 ** -24 if dt == "f16" else 1e-38) + \
            2.0 ** -36 * w.double().cpu().abs().sum(0)
        assert bool(((r.dx[others].double().cpu() - want["dx"]).abs() <= lim).all())


def test_a_graph_has_a_workspace_of_its_own(head):
    """a larger call on the same stream between the replays does not reach it"""
    x, w, t = inputs(150, 600, 64, "bf16", 17)
    want = head.linear_xent_step(x, w, t)
    out = head.XentStep(*[torch.empty_like(p) for p in want])
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        head.linear_xent_step(x, w, t)
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        head.linear_xent_step(x, w, t, out=out)
    big = inputs(1000, 5000, 64, "bf16", 18)
    for _ in range(3):
        for p in out:
            p.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            head.linear_xent_step(*big)
            filler = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
        side.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        del filler
        for p, q in zip(out, want):
            assert torch.equal(p, q)


def test_the_gradients_are_not_differentiable(head):
    """a second derivative is refused, not taken for zero"""
    x, w, t = inputs(20, 30, 16, "f32", 19)
    x, w = x.contiguous().requires_grad_(), w.contiguous().requires_grad_()
    loss, _ = head.linear_xent(x, w, t)
    dx, = torch.autograd.grad(loss.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        dx.square().sum().backward()


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("n,v,h,chunk", [(2100, 300, 130, 0), (2100, 70, 33, 1600), (70, 70001, 40, 0), (70, 20011, 200, 0)])
def test_dw_in_parts(head, dt, n, v, h, chunk):
    """few tiles and many tokens, or tiles past the last whole round: dw is summed in parts"""
    x, w, t = inputs(n, v, h, dt, 20, skip=0.1)
    check(head.linear_xent_step(x, w, t, chunk=chunk), x, w, t, None, dt, v)


@pytest.mark.parametrize("dt", list(DT))
def test_small_losses(head, dt):
    """tokens that the model is sure of: a loss of 1e-3 or less next to logits of 30 is not their difference"""
    n, v, h = 60, 300, 64
    x, w, t = inputs(n, v, h, dt, 21)
    wt = w[t].float()
    x = (wt * (30 / wt.square().sum(1, keepdim=True))).to(DT[dt])
    loss, _ = head.linear_xent(x, w, t)
    want, _ = reference(x, w, t, None, v)
    want = want["loss"]
    assert float(want.median()) < 1e-3
    # the logits' errors (of sums of h terms, up to 30) move the other terms of the sum, which are the loss; the
    # sum near 1, its correction and the logarithm: four roundings
    lim = want * (2 * (4 * math.sqrt(h) + 8) * 2.0 ** -24 * 60 + 2.0 ** -16) + 4 * 2.0 ** -24
    assert bool(((loss.double().cpu() - want).abs() <= lim).all())


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("n,skip", [(1, 0.0), (7, 0.0), (1100, 0.7)])
def test_dw_of_few_tokens(head, dt, n, skip):
    """the roundings of few entries of d do not average out: dw is as exact as its own rounding"""
    v, h = 400, 96
    x, w, t = inputs(n, v, h, dt, 22, skip=skip)
    weight = torch.full((n,), 1 / 3.0, device="cuda")
    r = head.linear_xent_step(x, w, t, weight)
    want, size = reference(x, w, t, weight, v)
    # two planes of d: its entries to 2^-14 (numerators in 16 bits over more than 128 tokens: 2^-10), logits to 2^-14
    rel = 2.0 ** -12 if n <= 128 else 2.0 ** -9
    lim = U[dt] * want["dw"].abs() + rel * size["dw"] + (2.0 ** -24 if dt == "f16" else 1e-38) + 2.0 ** -36 * size["x"]
    assert bool(((r.dw.double().cpu() - want["dw"]).abs() <= lim).all())


def large_logits(n, v, dt, size, sign, on_target):
    """logits of about sign * 2^size whose differences are whole numbers of `q`, all of them exact: token i's are
    sign * X_i W - k_v q; one entry has k = 0 and stands alone on top, by 1 to 200 q"""
    g = torch.Generator(device="cuda").manual_seed(size + n)
    half = size // 2
    q = 2.0 ** max(size - 20, -4)        # 2^-20 of the logits at the least: a sum of binary32 holds them
    x, w = torch.zeros(n, 40, device="cuda"), torch.zeros(v, 40, device="cuda")
    x[:, 0] = (128 + torch.arange(n, device="cuda") % 120) * 2.0 ** (half - 8) * sign
    x[:, 1] = 1.0
    w[:, 0] = 179 * 2.0 ** (size - half - 8)
    k = torch.randint(1, 201, (v,), generator=g, device="cuda")
    top = v // 3
    k[top] = 0
    w[:, 1] = -q * k
    t = torch.randint(0, v, (n,), generator=g, device="cuda")
    t[t == top] = top + 1
    if on_target:
        t[::2] = top
    return x.to(DT[dt]), w.to(DT[dt]), t


@pytest.mark.parametrize("n", [40, 100, 200])
@pytest.mark.parametrize("on_target", [True, False])
@pytest.mark.parametrize("dt,size", [(dt, size) for dt in DT for size in (12, 20, 25, 28)] + [("f32", 60), ("bf16", 60)])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_logits(head, dt, n, on_target, size, sign):
    """the softmax depends on differences of the logits, however large they are"""
    v = 300
    x, w, t = large_logits(n, v, dt, size, sign, on_target)
    weight = (torch.rand(n, device="cuda") + 0.5) / n
    r = head.linear_xent_step(x, w, t, weight)
    want, bound = reference(x, w, t, weight, v)
    # the logits, their maximum and the difference to the target's are exact.  The sum of exponentials, 1 at the least:
    # two roundings of each difference d, of which d exp(-d) <= 0.37 reaches the sum, the exponential's and 300 of the sum
    lim = 2.0 ** -18 + 2.0 ** -22 * want["loss"].abs()
    assert bool((r.loss >= 0).all())
    assert bool(((r.loss.double().cpu() - want["loss"]).abs() <= lim).all())
    assert bool(((r.lse.double().cpu() - want["lse"]).abs() <= 2.0 ** -18 + 2.0 ** -22 * want["lse"].abs()).all())
    loss, lse = head.linear_xent(x, w, t)
    assert torch.equal(loss, r.loss) and torch.equal(lse, r.lse)
    # an entry of d: its roundings, two of a difference of up to 126 (2^-16), up to 300 of a product's sum (2^-16); below
    # 2^-126 (bfloat16: the exponential) or 2^-38 (the others' operands) of the largest weight an entry may be 0
    rel, low = UD[dt] + 2.0 ** -14, 2.0 ** -38 if dt != "bf16" else 2.0 ** -126
    for k, more in (("dx", w.double().cpu().abs().sum(0)), ("dw", bound["x"])):
        got = getattr(r, k).double().cpu()
        assert float(want[k].abs().max()) < 0.9 * torch.finfo(DT[dt]).max
        lim = rel * bound[k] + U[dt] * want[k].abs() + (2.0 ** -24 if dt == "f16" else 1e-38) + 2 * low * bound["top"] * more
        assert bool(((got - want[k]).abs() <= lim).all()), (k, float(((got - want[k]).abs() - lim).max()))


@pytest.mark.parametrize("sx,sw", [(1e-32, 1e32), (1e32, 1e-32), (2.0 ** -110, 2.0 ** 100), (2.0 ** 100, 2.0 ** -110)])
@pytest.mark.parametrize("n", [40, 200])
def test_binary32_gradients_far_from_one(head, sx, sw, n):
    """gradients that are ordinary numbers although the factors they are made of are not"""
    x, w, t = inputs(n, 100, 64, "f32", 23)
    x, w = x * sx, w * sw
    weight = torch.full((n,), 1 / 3000.0, device="cuda")
    check(head.linear_xent_step(x, w, t, weight), x, w, t, weight, "f32", 100)


def test_binary32_token_of_zeros_among_large_ones(head):
    """its logits are 0, and stay so under the scaling that the others need"""
    v = 100
    x, w, t = inputs(40, v, 64, "f32", 24)
    x, w = x * 2.0 ** 90, w * 2.0 ** 90
    x[7] = 0.0
    for r in (head.linear_xent_step(x, w, t), None):
        loss = r.loss if r else head.linear_xent(x, w, t)[0]
        assert abs(float(loss[7]) - math.log(v)) < 2.0 ** -19 * math.log(v)
        if r:
            d = torch.full((v,), 1.0 / v, dtype=torch.float64, device="cuda")
            d[t[7]] -= 1
            # d and w as pairs of binary16 (22 bits each), 100 products summed
            lim = (2.0 ** -20 + 2.0 ** -17) * (d.abs() @ w.double().abs())
            assert bool(((r.dx[7].double() - d @ w.double()).abs() <= lim).all())


def test_two_threads_on_one_stream(head):
    """forward passes of one thread beside another's steps: each gets what it gets alone"""
    import threading
    a, b = inputs(150, 700, 64, "bf16", 30), inputs(300, 500, 96, "bf16", 31)
    want_a, want_b = head.linear_xent_step(*a), head.linear_xent(*b)
    torch.cuda.synchronize()
    got_a, got_b = [], []
    threads = [threading.Thread(target=lambda: got_a.extend(head.linear_xent_step(*a) for _ in range(40))),
               threading.Thread(target=lambda: got_b.extend(head.linear_xent(*b) for _ in range(80)))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert len(got_a) == 40 and len(got_b) == 80
    for got, want in [(g, want_a) for g in got_a] + [(g, want_b) for g in got_b]:
        for p, q in zip(got, want):
            assert torch.equal(p, q)


def check_large(r, x, w, t, weight, dt):
    """check() for sizes whose reference is better made on the device, in 64 bits and a part of the tokens at a time"""
    n, (v, h) = x.shape[0], w.shape
    wd, g = w.double(), torch.ones(n, device="cuda") if weight is None else weight
    keep, top = (t >= 0) & (t < v), float(g.abs().max())
    uz = (4 * math.sqrt(h) + 8) * 2.0 ** -24 + (2.0 ** -20 if dt == "f32" else 0)
    low, floor = (2.0 ** -38 if dt != "bf16" else 2.0 ** -126), (2.0 ** -24 if dt == "f16" else 1e-38)
    dw, size, worst = torch.zeros(v, h, dtype=torch.float64, device="cuda"), torch.zeros(v, h, dtype=torch.float64, device="cuda"), 0.0
    grads = hasattr(r, "dx")
    sums = lambda terms: 4 * math.sqrt(terms) * 2.0 ** -24             # (a product's sum, as a random walk, four deviations)
    spread = wd.abs().sum(0)
    for i in range(0, n, 512):
        s = slice(i, i + 512)
        kept, xd = keep[s], x[s].double()
        td, gd = torch.where(kept, t[s], 0)[:, None], torch.where(kept, g[s], 0.0).double()[:, None]
        z = xd @ wd.t().contiguous()
        lse = torch.logsumexp(z, 1)
        loss = lse - z.gather(1, td)[:, 0]
        ez = uz * (xd.abs() @ wd.abs().t().contiguous()).amax(1)
        worst = max(worst, float(ez.max()))
        lim = 2 * ez + 2.0 ** -19 + 2.0 ** -22 * (lse.abs() + loss.abs())
        for got, want in ((r.loss[s], loss), (r.lse[s], lse)):
            assert bool(((got.double() - want).abs() <= lim)[kept].all()) and bool((got[~kept] == 0).all()), i
        if not grads:
            continue
        p = torch.exp(z - lse[:, None])
        hot = torch.zeros_like(p).scatter_(1, td, 1.0)
        d, big = gd * (p - hot), gd.abs() * (p + hot)
        rel = UD[dt] + 3 * float(ez.max()) + 2.0 ** -18 + sums(v)
        want = d @ wd
        lim = rel * (big @ wd.abs()) + U[dt] * want.abs() + floor + 2 * low * gd.abs() * spread
        assert bool(((r.dx[s].double() - want).abs() <= lim).all()), ("dx", i)
        dw += d.t().contiguous() @ xd
        size += big.t().contiguous() @ xd.abs()
    if grads:
        rel = UD[dt] + 3 * worst + 2.0 ** -18 + sums(n)
        lim = rel * size + U[dt] * dw.abs() + floor + 2 * low * top * x.double().abs().sum(0)
        assert bool(((r.dw.double() - dw).abs() <= lim).all()), "dw"


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("n", [8191, 8192, 8193, 16385, 20000])
def test_lists_of_tokens_longer_than_a_pass(head, tc, dt, n):
    """8192 tokens are listed at a time; later ones follow, and their targets are looked at"""
    v, h = 300, 32
    x, w, t = inputs(n, v, h, dt, 25, skip=0.3)
    weight = torch.rand(n, device="cuda") / n
    t[-1], t[8100], t[5] = v - 1, 0, IGNORE
    t[-3] = v + 7
    r = head.linear_xent_step(x, w, t, weight)
    assert tc.device_errors() == tc.TC_KERR_BAD_INDEX
    check_large(r, x, w, t, weight, dt)
    loss, lse = head.linear_xent(x, w, t)
    assert tc.device_errors() == tc.TC_KERR_BAD_INDEX
    assert torch.equal(loss, r.loss) and torch.equal(lse, r.lse)


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("n,v,h,skip", [(4096, 50257, 32, 0.1), (3000, 40000, 513, 0.0)])
def test_more_tiles_than_workgroups(head, dt, n, v, h, skip):
    """several tiles of 256 x 256 for each workgroup, and softmax passes over several blocks of vocabulary entries"""
    x, w, t = inputs(n, v, h, dt, 26, skip=skip)
    weight = (torch.rand(n, device="cuda") + 0.5) / n
    r = head.linear_xent_step(x, w, t, weight)
    check_large(r, x, w, t, weight, dt)
    loss, lse = head.linear_xent(x, w, t)
    check_large(type("R", (), {"loss": loss, "lse": lse})(), x, w, t, weight, dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_more_than_32_tiles_for_each_workgroup(head, dt):
    """tiles are dealt out by the die then, an eighth of them in a row for each"""
    n, v, h = 8192, 70001, 32
    x, w, t = inputs(n, v, h, dt, 27)
    weight = torch.full((n,), 1.0 / n, device="cuda")
    check_large(head.linear_xent_step(x, w, t, weight), x, w, t, weight, dt)
    loss, lse = head.linear_xent(x, w, t)
    check_large(type("R", (), {"loss": loss, "lse": lse})(), x, w, t, weight, dt)
    head.free_workspaces()
