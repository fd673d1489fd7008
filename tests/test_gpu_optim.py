"""Gradient norm and AdamW over lists of tensors against 64-bit arithmetic and,
for the codes of 8-bit moments, against the format's definition bit by bit."""
import math

import numpy as np
import pytest
import torch

import optim_ref as R

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # unit roundoff: 24, 8 and 11 significant bits
HP = dict(lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)
SIZES = [1, 0, 7, 255, 256, 257, 2048, 2049, 9001]


@pytest.fixture(scope="module")
def optim(tc):
    from paper_2401_07788_amd import optim
    return optim


def views(sizes, dtype, shift, seed, scale=1.0):
    """tensors in one buffer, each `shift` elements past a 64-element boundary, with a canary between them"""
    at, places = 0, []
    for n in sizes:
        places.append(at + shift)
        at += -(-(n + shift) // 64 + 1) // 1 * 64 + 64
    flat = torch.full((at + 64,), 7.0, dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for a, n in zip(places, sizes):
        flat[a:a + n] = torch.randn(n, generator=g, device="cuda").mul_(scale).to(dtype)
        out.append(flat[a:a + n])
    used = torch.zeros(flat.numel(), dtype=torch.bool, device="cuda")
    for a, n in zip(places, sizes):
        used[a:a + n] = True
    return out, flat, ~used


def np64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------- norm
@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("sizes", [[1], SIZES, [3] * 401, [0, 0], [70001, 5, 300000]], ids=["one", "mixed", "many", "empty", "long"])
@pytest.mark.parametrize("shift", [0, 1])
def test_grad_norm(optim, dt, sizes, shift):
    gs, _, _ = views(sizes, DT[dt], shift, 1)
    want = np.sqrt(sum((np64(g) ** 2).sum() for g in gs))
    for max_norm in (0.5, 1e6):
        got = np64(optim.grad_norm(gs, max_norm))
        # binary64 sums, one rounding of the norm; the factor: three more roundings
        assert abs(got[0] - want) <= 2.0 ** -23 * want
        assert abs(got[1] - min(1.0, max_norm / (want + 1e-6))) <= 2.0 ** -21 * got[1]
    again = optim.grad_norm(optim.TensorList(gs), 0.5)
    assert torch.equal(again, optim.grad_norm(gs, 0.5))


@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_grad_norm_far_from_one(optim, scale):
    gs, _, _ = views([1000, 3], torch.float32, 0, 2, scale)
    want = np.sqrt(sum((np64(g) ** 2).sum() for g in gs))
    assert abs(float(optim.grad_norm(gs, 1.0)[0]) - want) <= 2.0 ** -23 * want


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_norm_that_is_not_finite_leaves_everything(optim, bad):
    sizes = [257, 5]
    for bits in (8, 32):
        ps, pflat, _ = views(sizes, torch.float32, 0, 3)
        gs, _, _ = views(sizes, torch.float32, 0, 4)
        opt = optim.AdamW(ps, state_bits=bits, **HP)
        opt.step(gs, clip=optim.grad_norm(gs, 1.0))
        before = [pflat.clone()] + [s.clone() for s in opt.state.values()]
        gs[1][2] = bad
        clip = optim.grad_norm(gs, 1.0)
        assert not torch.isfinite(clip[0])
        opt.step(gs, clip=clip)
        for a, b in zip(before, [pflat] + list(opt.state.values())):
            assert torch.equal(a, b)


def test_norm_leaves_its_workspace_zero_and_replays_in_a_graph(optim, tc):
    gs, flat, _ = views([3] * 250 + [50000], torch.float32, 0, 5)
    lst = optim.TensorList(gs)
    ws = torch.zeros(lst.ws_bytes, dtype=torch.uint8, device="cuda")
    out = torch.empty(2, device="cuda")
    optim.grad_norm(lst, 1.0, out=out, ws=ws)
    assert int(ws.sum()) == 0
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        optim.grad_norm(lst, 1.0, out=out, ws=ws)
    for k in range(4):
        flat.mul_(1.5)
        eager = optim.grad_norm(lst, 1.0)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    assert int(ws.sum()) == 0


# ------------------------------------------------------------------ AdamW
def check_p(got, want, p0, upd, dt):
    # decay factor, its product, the update's chain of about ten roundings and the difference in binary32,
    # then the rounding to dt
    lim = 2.0 ** -24 * (4 * np.abs(p0) + 16 * np.abs(upd)) + U[dt] * np.abs(want) + (2.0 ** -24 if dt == "f16" else 0)
    assert (np.abs(got - want) <= lim).all(), float((np.abs(got - want) - lim).max())


@pytest.mark.parametrize("pdt,gdt", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "bf16"), ("f16", "bf16"),
                                     ("f32", "f16"), ("bf16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("shift", [0, 1])
def test_adamw_32(optim, pdt, gdt, shift):
    ps, pflat, pgap = views(SIZES, DT[pdt], shift, 6)
    opt = optim.AdamW(ps, state_bits=32, **HP)
    for t in (1, 2, 3):
        gs, _, _ = views(SIZES, DT[gdt], shift, 10 + t, 0.1)
        clip = torch.tensor([2.0, 0.25], device="cuda")
        old = [(np64(p), np64(opt.state["m"][a:a + p.numel()]), np64(opt.state["v"][a:a + p.numel()])) for p, a in zip(ps, opt.places)]
        opt.step(gs, clip=clip)
        for p, g, a, (p0, m0, v0) in zip(ps, gs, opt.places, old):
            g = np64(g)
            wp, wm, wv = R.adamw64(p0, g, m0, v0, 0.25, HP["lr"], *HP["betas"], HP["eps"], HP["weight_decay"], t)
            n = p.numel()
            # betas, products and the sum: five roundings on either term
            terms = 0.9 * np.abs(m0) + 0.1 * 0.25 * np.abs(g)
            assert (np.abs(np64(opt.state["m"][a:a + n]) - wm) <= 5 * 2.0 ** -24 * terms).all()
            assert (np.abs(np64(opt.state["v"][a:a + n]) - wv) <= 7 * 2.0 ** -24 * np.abs(wv) + 1e-44).all()
            check_p(np64(p), wp, p0, wp - p0 * (1 - HP["lr"] * HP["weight_decay"]), pdt)
    assert bool((pflat[pgap] == 7.0).all())


def test_more_tensors_than_one_launch_holds(optim):
    sizes = [300 + k % 7 for k in range(200)]
    ps, _, _ = views(sizes, torch.float32, 0, 7)
    gs, _, _ = views(sizes, torch.float32, 0, 8)
    p0 = [p.clone() for p in ps]
    a = optim.AdamW(ps, state_bits=32, **HP)
    a.step(gs)
    for k in (0, 87, 88, 175, 176, 199):
        b = optim.AdamW([p0[k]], state_bits=32, **HP)
        b.step([gs[k]])
        assert torch.equal(p0[k], ps[k])
        assert torch.equal(b.state["v"][:sizes[k]], a.state["v"][a.places[k]:a.places[k] + sizes[k]])


def test_long_chunks_and_short_ones_agree(optim):
    """a list of more elements than 4096 units goes out in longer chunks"""
    n = 4096 * 2048 + 12345
    g = torch.Generator(device="cuda").manual_seed(9)
    p = torch.randn(n, generator=g, device="cuda")
    gr = torch.randn(n, generator=g, device="cuda")
    for bits in (8, 32):
        q, parts = p.clone(), [p[k:k + (1 << 20)].clone() for k in range(0, n, 1 << 20)]
        a = optim.AdamW([q], state_bits=bits, **HP)
        a.step([gr])
        for k, part in enumerate(parts):
            b = optim.AdamW([part], state_bits=bits, **HP)
            b.step([gr[k << 20:(k << 20) + part.numel()].contiguous()])
        assert torch.equal(q, torch.cat(parts))


@pytest.mark.parametrize("pdt,gdt,shift", [("f32", "f32", 0), ("bf16", "bf16", 1), ("f16", "f32", 3), ("f32", "f16", 1)])
def test_adamw_8(optim, pdt, gdt, shift):
    ps, pflat, pgap = views(SIZES, DT[pdt], shift, 11)
    opt = optim.AdamW(ps, state_bits=8, seed=40, **HP)
    for t in (1, 2, 3):
        gs, gflat, _ = views(SIZES, DT[gdt], shift, 20 + t, 0.1)
        if t == 2:
            gs[-1][256:512] = 0.0                       # a block of zeros
            gs[-1][512:520] *= 1e-4                     # small among large
        p0 = [np64(p) for p in ps]
        st = {k: s.cpu().numpy() for k, s in opt.state.items()}
        m0, v0 = R.decode(st["m"], st["em"], 7, 112), R.decode(st["v"], st["ev"], 8, 96)
        dm, dv = opt.moments()
        assert np.array_equal(dm.cpu().numpy(), m0) and np.array_equal(dv.cpu().numpy(), v0)
        g = np.zeros(opt.size, np.float32)
        for a, x in zip(opt.places, gs):
            g[a:a + x.numel()] = x.float().cpu().numpy()
        clip = torch.tensor([2.0, 0.25], device="cuda")
        opt.step(gs, clip=clip)
        m, v = R.moments32(g, m0, v0, 0.25, *HP["betas"])
        wm, wem = R.encode_m(m, 40 + t)
        wv, wev = R.encode_v(v, 40 + t)
        st = {k: s.cpu().numpy() for k, s in opt.state.items()}
        used = np.zeros(opt.size, bool)
        for a, x in zip(opt.places, gs):
            used[a:a + x.numel()] = True
        assert np.array_equal(st["em"], wem) and np.array_equal(st["ev"], wev)
        assert np.array_equal(st["m"][used], wm[used]) and np.array_equal(st["v"], wv)
        assert not st["v"][~used].any() and not (st["m"][~used] & 127).any()
        for p, q0, a in zip(ps, p0, opt.places):
            s = slice(a, a + p.numel())
            w, _, _ = R.adamw64(q0, g[s], m0[s], v0[s], 0.25, HP["lr"], *HP["betas"], HP["eps"], HP["weight_decay"], t)
            check_p(np64(p), w, q0, w - q0 * (1 - HP["lr"] * HP["weight_decay"]), pdt)
    assert bool((pflat[pgap] == 7.0).all())


def test_eight_bit_average_moves_although_a_step_is_less_than_a_code(optim):
    """moments under a constant gradient: the average of many codes follows the exact average"""
    n, steps = 1 << 16, 300
    p = torch.zeros(n, device="cuda")
    opt = optim.AdamW([p], lr=0.0, betas=(0.9, 0.99), state_bits=8)
    g = torch.ones(n, device="cuda")
    for _ in range(steps):
        opt.step([g])
    want = 1 - 0.99 ** steps
    m, v = (float(x.double().mean()) for x in opt.moments())
    got = v
    # a step moves v by at most 0.01 where codes are at most 1/8 apart: the variance it adds is below 0.01/8, the
    # average forgets at 0.02 a step, so one position's variance is below 0.0625 and the mean's deviation below 0.001;
    # neighbours share a hash, for which the deviation is doubled, and six of them are allowed
    assert abs(got - want) < 6 * 2 * 0.25 / n ** 0.5 + 2e-3
    # m forgets at 0.1 a step and a step adds at most (1/8)^2 / 4
    assert abs(m - 1.0) < 6 * 2 * 0.15 / n ** 0.5 + 2e-3


def test_master_parameters(optim):
    ps, _, _ = views(SIZES, torch.bfloat16, 0, 12)
    qs = [p.float() for p in ps]
    a = optim.AdamW(ps, state_bits=32, master=True, **HP)
    b = optim.AdamW(qs, state_bits=32, **HP)
    for t in range(3):
        gs, _, _ = views(SIZES, torch.bfloat16, 0, 30 + t)
        a.step(gs)
        b.step(gs)
    for p, w, q in zip(ps, a.w32, qs):
        assert torch.equal(w, q) and torch.equal(p, q.bfloat16())


def test_step_takes_grad_attributes_and_other_streams(optim):
    p = torch.nn.Parameter(torch.randn(3000, device="cuda"))
    q = p.detach().clone()
    p.grad = torch.randn_like(p)
    side = torch.cuda.Stream()
    a, b = optim.AdamW([p.data], **HP), optim.AdamW([q], **HP)
    a.params = [p]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step()
    side.synchronize()
    b.step([p.grad])
    assert torch.equal(p.data, q)


def test_parameters_whose_data_was_replaced(optim):
    """the step goes to the memory that they have now"""
    ps = [torch.nn.Parameter(torch.randn(300, device="cuda")), torch.nn.Parameter(torch.randn(70, device="cuda"))]
    opt = optim.AdamW(ps, **HP)
    gs = [torch.randn_like(p) for p in ps]
    opt.step(gs)
    old = ps[1].data
    kept = old.clone()
    ps[1].data = old.clone()
    opt.step(gs)
    assert torch.equal(old, kept) and not torch.equal(ps[1].data, kept)
    ps[1].data = torch.zeros(71, device="cuda")
    with pytest.raises(ValueError, match="changed"):
        opt.step([gs[0], torch.zeros(70, device="cuda")])
    assert opt.t == 2


def test_a_step_is_not_captured(optim):
    """its number and seed would be the same at every replay"""
    ps, _, _ = views([300], torch.float32, 0, 30)
    gs, _, _ = views([300], torch.float32, 0, 31)
    opt, other = optim.AdamW(ps, state_bits=8, **HP), torch.ones(4, device="cuda")
    torch.cuda.synchronize()
    before = ps[0].clone()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        other.zero_()
        with pytest.raises(RuntimeError, match="captured"):
            opt.step(gs)
    torch.cuda.synchronize()
    assert opt.t == 0 and torch.equal(ps[0], before)
    opt.step(gs)
    assert opt.t == 1 and not torch.equal(ps[0], before)


@pytest.mark.parametrize("bits", [8, 32])
def test_replaced_states(optim, bits):
    """good ones are taken, whatever the object; others are refused before the launch"""
    ps, _, _ = views([300, 70], torch.float32, 0, 32)
    gs, _, _ = views([300, 70], torch.float32, 0, 33)
    qs = [p.clone() for p in ps]
    a, b = optim.AdamW(ps, state_bits=bits, **HP), optim.AdamW(qs, state_bits=bits, **HP)
    a.step(gs)
    b.step(gs)
    a.state = {k: s.clone() for k, s in a.state.items()}
    a.state["m"].data = a.state["m"].clone()
    a.step(gs)
    b.step(gs)
    for p, q in zip(ps, qs):
        assert torch.equal(p, q)
    good, before = a.state, [p.clone() for p in ps]
    for k in good:
        for wrong in (good[k].cpu(), good[k].to(torch.float16), good[k][1:], good[k].view(1, -1), torch.cat([good[k], good[k]])[::2], None):
            a.state = {**good, k: wrong}
            with pytest.raises(ValueError, match="state"):
                a.step(gs)
            with pytest.raises(ValueError, match="state"):
                a.moments()
    a.state = dict(good)
    a.state["m"] = good["m"].clone()
    a.state["m"].data = torch.zeros(3, device="cuda")
    with pytest.raises(ValueError, match="state"):
        a.step(gs)
    assert a.t == 2
    for p, q in zip(ps, before):
        assert torch.equal(p, q)


@pytest.mark.parametrize("pdt,gdt", [("f32", "bf16"), ("bf16", "f32"), ("bf16", "f16"), ("f16", "bf16"), ("f16", "f16")])
def test_adamw_8_other_types(optim, pdt, gdt):
    """the type pairs of 8-bit moments that the bit by bit test leaves out: moments as of the same gradients in
    binary32 (exactly), parameters by the formula"""
    ps, pflat, pgap = views(SIZES, DT[pdt], 1, 34)
    qs = [p.float().clone() for p in ps]
    a, b = optim.AdamW(ps, state_bits=8, seed=7, **HP), optim.AdamW(qs, state_bits=8, seed=7, **HP)
    clip = torch.tensor([2.0, 0.25], device="cuda")
    for t in (1, 2):
        gs, _, _ = views(SIZES, DT[gdt], 1, 40 + t, 0.1)
        m0, v0 = (np64(x) for x in a.moments())
        p0 = [np64(p) for p in ps]
        a.step(gs, clip=clip)
        b.step([g.float() for g in gs], clip=clip)
        for k in a.state:
            assert torch.equal(a.state[k], b.state[k])
        for p, g, q0, at in zip(ps, gs, p0, a.places):
            s = slice(at, at + p.numel())
            w, _, _ = R.adamw64(q0, np64(g), m0[s], v0[s], 0.25, HP["lr"], *HP["betas"], HP["eps"], HP["weight_decay"], t)
            check_p(np64(p), w, q0, w - q0 * (1 - HP["lr"] * HP["weight_decay"]), pdt)
    assert bool((pflat[pgap] == 7.0).all())


@pytest.mark.parametrize("pdt", ["bf16", "f16"])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("replace", [False, True])
def test_a_resumed_run_goes_on_as_if_it_had_not_stopped(optim, pdt, bits, replace):
    """parameters, state, t and seed are all of it, the binary32 masters too"""
    ps, _, _ = views(SIZES, DT[pdt], 0, 50)
    a = optim.AdamW(ps, state_bits=bits, master=True, seed=3, **HP)
    steps = [views(SIZES, DT[pdt], 0, 51 + t, 0.1)[0] for t in range(6)]
    for gs in steps[:3]:
        a.step(gs)
    saved = {k: s.clone() for k, s in a.state.items()}
    qs = [p.clone() for p in ps]
    if replace:
        # into an optimizer that is there already
        b = optim.AdamW(qs, state_bits=bits, master=True, **HP)
        b.step(steps[5])
        for q, p in zip(qs, ps):
            q.copy_(p)
        b.state, b.t, b.seed = saved, a.t, a.seed
    else:
        b = optim.AdamW(qs, state_bits=bits, master=True, state=saved, t=a.t, seed=a.seed, **HP)
    for gs in steps[3:]:
        a.step(gs)
        b.step(gs)
    for p, q in zip(ps, qs):
        assert torch.equal(p, q)
    for w, u in zip(a.w32, b.w32):
        assert torch.equal(w, u)
    assert any(not torch.equal(w, p.float()) for w, p in zip(a.w32, ps))


@pytest.mark.parametrize("pdt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("how", ["in place", "data", "one element", "not a number"])
def test_parameters_set_between_steps_count_although_there_are_masters(optim, pdt, bits, how):
    """the next step is taken on them, not on the masters of what was there before (an element that is set to the
    rounding of its master cannot be told from one that was not set, and keeps it)"""
    ps = [torch.nn.Parameter(p.clone()) for p in views(SIZES, DT[pdt], 0, 60)[0]]
    a = optim.AdamW(ps, state_bits=bits, master=True, seed=5, **HP)
    for t in range(2):
        a.step(views(SIZES, DT[pdt], 0, 61 + t, 0.1)[0])
    before = [w.clone() for w in a.w32 or ps]
    new = views(SIZES, DT[pdt], 0, 63)[0]
    want = []
    for p, w, n in zip(ps, before, new):
        if how == "in place":
            p.data.copy_(n)
            want.append(torch.where(w.detach().to(DT[pdt]) == n, w.detach().float(), n.float()))
        elif how == "data":
            p.data = n.clone()
            want.append(torch.where(w.detach().to(DT[pdt]) == n, w.detach().float(), n.float()))
        else:
            w = w.detach().float().clone()
            if p.numel():
                p.data[-1] = w[-1] = 2.5 if how == "one element" else math.nan
            want.append(w)
    # the same step on binary32 parameters that hold what counts
    qs = [w.clone() for w in want]
    b = optim.AdamW(qs, state_bits=bits, state={k: s.clone() for k, s in a.state.items() if k != "w32"}, t=a.t, seed=a.seed, **HP)
    gs = views(SIZES, DT[pdt], 0, 64, 0.1)[0]
    a.step(gs)
    b.step(gs)
    for p, w, q in zip(ps, a.w32 or ps, qs):
        assert torch.equal(w.nan_to_num(7.0), q.nan_to_num(7.0)) and torch.equal(p.data.nan_to_num(7.0), q.to(DT[pdt]).nan_to_num(7.0))


@pytest.mark.parametrize("given", ["parameter", "detached", "view"])
def test_autograd_notices_a_step(optim, given):
    """a backward pass through values that the step has overwritten is refused; a refused step leaves no trace"""
    p = torch.nn.Parameter(torch.randn(8, 30, device="cuda"))
    own = {"parameter": p, "detached": p.detach(), "view": p.detach().view(-1)}[given]
    opt = optim.AdamW([own], **HP)
    y = (p * p).sum()
    version = p._version
    with pytest.raises(ValueError):
        opt.step([torch.zeros(3, device="cuda")])
    assert p._version == version
    opt.step([torch.ones_like(own)])
    assert p._version > version
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    (p * p).sum().backward()
    assert torch.equal(p.grad, 2 * p.detach())


def test_a_step_on_inference_tensors(optim):
    with torch.inference_mode():
        p = torch.randn(300, device="cuda")
    q = p.clone()
    g = torch.randn(300, device="cuda")
    optim.AdamW([p], **HP).step([g])
    optim.AdamW([q], **HP).step([g])
    assert torch.equal(p, q)


def test_a_graph_of_the_boundary_keeps_its_workspace(optim, tc):
    """a norm over many tensors on the same stream, between the replays, does not take it away"""
    x = torch.randn(1, 40000, device="cuda")
    xs, out = x.clone(), tc.empty_topk_payload(1, 40000, 4000, torch.float32, "cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tc.topk_compress(xs, 4000, 1, out=out)
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        tc.topk_compress(xs, 4000, 1, out=out)
    gs = views([3] * 4000, torch.float32, 0, 70)[0]
    for k in range(3):
        xs.copy_(x * (k + 1.5) + k)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            optim.grad_norm(gs, 1.0)
            filler = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
        side.synchronize()
        want = tc.topk_compress(xs, 4000, 1)
        graph.replay()
        torch.cuda.synchronize()
        del filler
        for p, q in zip(out, want):
            assert torch.equal(p, q)
    assert tc.device_errors() == 0
