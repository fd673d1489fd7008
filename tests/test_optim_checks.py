"""What the optimizer's entry points refuse, on the host and before any device
call, and the reference codes of the 8-bit moments checked by themselves."""
import ctypes as C

import numpy as np
import pytest
import torch

import optim_ref as R
from paper_2401_07788_amd import optim, tc


def test_reference_codes_are_near_and_unbiased():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal(256 * 40) * np.exp(rng.standard_normal(256 * 40))).astype(np.float32)
    v = (x * x).astype(np.float32)
    top = np.abs(x).reshape(-1, 256).max(1).repeat(256)
    tm, tv = np.zeros(x.size), np.zeros(x.size)
    for seed in range(64):
        c, e = R.encode_m(x, seed)
        d = R.decode(c, e, 7, 112)
        # 2^E is at most 16/15 above the largest; codes are 2^-3 of their power apart down to 2^-14, then evenly
        assert (np.abs(d - x) <= np.maximum(np.abs(x) / 8, top * (16 / 15) * 2.0 ** -17)).all()
        tm += d
        c, e = R.encode_v(v, seed)
        d = R.decode(c, e, 8, 96)
        assert (np.abs(d - v) <= np.maximum(v / 8, top * top * (16 / 15) * 2.0 ** -33)).all()
        tv += d
    # 10240 elements of 64 roundings, each off by at most 1/16 on average in square: the mean ratio deviates by below 1e-4
    big = np.abs(x) > top * 1e-3
    assert abs((tm[big] / 64 / x[big]).mean() - 1) < 6e-4
    assert abs((tv[big] / 64 / v[big]).mean() - 1) < 6e-4
    z = np.zeros(256, np.float32)
    assert not R.encode_m(z, 3)[0].any() and not R.encode_v(z, 3)[0].any() and R.encode_m(z, 3)[1][0] == -127
    one = z.copy()
    one[3], one[9] = 1.0, 1e-30
    assert R.encode_v(one, 5)[0][9] == 1 and R.encode_v(one, 5)[0][4] == 0
    # a largest magnitude past 15/16 of a power of two can still be rounded up
    one[3] = np.float32(1.99)
    seen = {float(R.decode(*R.encode_v(one, seed), 8, 96)[3]) for seed in range(64)}
    assert seen == {1.875, 2.0}


def test_python_refusals():
    a, b = torch.zeros(10), torch.zeros(10, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="empty"):
        optim.TensorList([])
    with pytest.raises(TypeError):
        optim.TensorList([a, b])
    with pytest.raises(TypeError, match="unsupported"):
        optim.TensorList([a.double()])
    with pytest.raises(ValueError, match="contiguous"):
        optim.TensorList([torch.zeros(4, 4).t()])
    with pytest.raises(ValueError, match="GPU"):
        optim.grad_norm([a], 1.0)
    with pytest.raises(ValueError, match="state_bits"):
        optim.AdamW([a], lr=1.0, state_bits=4)
    o = optim.AdamW([a], lr=1.0, state_bits=8)
    assert o.size == 256 and o.state["em"].numel() == 1
    with pytest.raises(ValueError, match="gradients for"):
        o.step([a, a])
    with pytest.raises(ValueError, match="fit"):
        o.step([torch.zeros(9)])
    with pytest.raises(TypeError, match="unsupported"):
        o.step([a.double()])
    with pytest.raises(ValueError, match="clip"):
        o.step([a], clip=torch.zeros(3))
    with pytest.raises(ValueError, match="GPU"):
        o.step([a])
    assert o.t == 0
    with pytest.raises(ValueError, match="state"):
        optim.AdamW([a], lr=1.0, state_bits=8, state={"m": torch.zeros(256)})


BASE = 1 << 40          # never dereferenced: the checks fail first


def row(**kw):
    d = dict(p=BASE, g=BASE + (1 << 30), w32=None, n=10, pos=0)
    d.update(kw)
    return tc.Tensor(**d)


def settings(**kw):
    d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, t=1, bits=32, seed=0, m=BASE + (2 << 30), v=BASE + (3 << 30))
    d.update(kw)
    return tc.AdamwSettings(**d)


@pytest.mark.parametrize("s,r,p_dt,g_dt,want", [
    (dict(bits=16), {}, 0, 0, tc.TC_ERR_ARG),
    (dict(t=0), {}, 0, 0, tc.TC_ERR_ARG),
    (dict(beta1=1.0), {}, 0, 0, tc.TC_ERR_ARG),
    (dict(beta2=float("nan")), {}, 0, 0, tc.TC_ERR_ARG),
    (dict(eps=-1.0), {}, 0, 0, tc.TC_ERR_ARG),
    (dict(eps=0.0, bits=8), {}, 0, 0, tc.TC_ERR_ARG),
    (dict(lr=float("inf")), {}, 0, 0, tc.TC_ERR_ARG),
    (dict(m=None), {}, 0, 0, tc.TC_ERR_NULL),
    (dict(bits=8), {}, 0, 0, tc.TC_ERR_NULL),
    (dict(m=BASE + 2), {}, 0, 0, tc.TC_ERR_ALIGN),
    ({}, {}, 3, 0, tc.TC_ERR_DTYPE),
    ({}, {}, 0, -1, tc.TC_ERR_DTYPE),
    ({}, dict(p=None), 0, 0, tc.TC_ERR_NULL),
    ({}, dict(g=None), 0, 0, tc.TC_ERR_NULL),
    ({}, dict(p=BASE + 2), 0, 0, tc.TC_ERR_ALIGN),
    ({}, dict(g=BASE + 1), 0, 1, tc.TC_ERR_ALIGN),
    ({}, dict(w32=BASE + 1), 1, 1, tc.TC_ERR_ALIGN),
    ({}, dict(pos=8), 0, 0, tc.TC_ERR_ARG),
    ({}, dict(n=1 << 40), 0, 0, tc.TC_ERR_ARG),
])
def test_step_refusals(s, r, p_dt, g_dt, want):
    L = tc.lib()
    a, t = settings(**s), row(**r)
    assert L.tc_adamw_step(C.byref(a), C.byref(t), 1, p_dt, g_dt, None, None) == want
    assert L.tc_last_error()


def test_nothing_to_do_succeeds():
    L = tc.lib()
    a, t = settings(m=None, v=None), row(n=0, p=None, g=None)
    assert L.tc_adamw_step(C.byref(a), C.byref(t), 1, 0, 0, None, None) == 0
    assert L.tc_adamw_step(C.byref(a), None, 0, 0, 0, None, None) == 0
    assert L.tc_adamw_step(C.byref(a), None, 1, 0, 0, None, None) == tc.TC_ERR_NULL
    assert L.tc_adamw_step(None, None, 0, 0, 0, None, None) == tc.TC_ERR_NULL
    assert L.tc_adamw_moments(None, None, None, None, 0, None, None, None) == 0
    assert L.tc_adamw_moments(BASE, BASE, BASE, BASE, 100, BASE, BASE, None) == tc.TC_ERR_ARG
    assert L.tc_adamw_moments(BASE, None, BASE, BASE, 256, BASE, BASE, None) == tc.TC_ERR_NULL
    assert L.tc_adamw_moments(BASE, BASE, BASE, BASE, 256, BASE + 2, BASE, None) == tc.TC_ERR_ALIGN


def test_norm_refusals():
    L = tc.lib()
    t = row()
    need = L.tc_grad_norm_workspace_bytes(1)
    out, ws = BASE + (4 << 30), BASE + (5 << 30)
    assert L.tc_grad_norm(C.byref(t), 1, 5, 1.0, out, ws, need, None) == tc.TC_ERR_DTYPE
    assert L.tc_grad_norm(C.byref(t), 1, 0, 0.0, out, ws, need, None) == tc.TC_ERR_ARG
    assert L.tc_grad_norm(C.byref(t), 1, 0, float("nan"), out, ws, need, None) == tc.TC_ERR_ARG
    assert L.tc_grad_norm(C.byref(t), 1, 0, 1.0, None, ws, need, None) == tc.TC_ERR_NULL
    assert L.tc_grad_norm(C.byref(t), 1, 0, 1.0, out, None, 0, None) == tc.TC_ERR_WORKSPACE
    assert L.tc_grad_norm(C.byref(t), 1, 0, 1.0, out, ws, need - 1, None) == tc.TC_ERR_WORKSPACE
    assert L.tc_grad_norm(C.byref(t), 1, 0, 1.0, out, ws + 4, need, None) == tc.TC_ERR_ALIGN
    bad = row(g=BASE + 2)
    assert L.tc_grad_norm(C.byref(bad), 1, 0, 1.0, out, ws, need, None) == tc.TC_ERR_ALIGN


WRONG_STATES = {
    "other dtype": lambda s: {**s, "m": s["m"].to(torch.float16)},
    "other size": lambda s: {**s, "v": s["v"][:-1]},
    "strided": lambda s: {**s, "m": torch.zeros(2 * s["m"].numel(), dtype=s["m"].dtype, device=s["m"].device)[::2]},
    "two dimensions": lambda s: {**s, "v": s["v"].view(2, -1)},
    "other device": lambda s: {**s, "m": torch.zeros_like(s["m"], device="meta")},
    "missing": lambda s: {k: t for k, t in s.items() if k != "v"},
    "none": lambda s: {**s, "m": None},
    "short exponents": lambda s: {**s, "em": s["em"][:0]},
    "wide exponents": lambda s: {**s, "ev": s["ev"].to(torch.int32)},
}


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("what", list(WRONG_STATES))
@pytest.mark.parametrize("same_object", [True, False])
def test_a_replaced_state_is_looked_at(what, bits, same_object):
    """the state is a public attribute: what a step finds there is checked every time, before anything is launched"""
    if bits == 32 and "exponents" in what:
        pytest.skip("binary32 moments have none")
    p = torch.zeros(300)
    o = optim.AdamW([p], lr=1.0, state_bits=bits)
    wrong = WRONG_STATES[what](o.state)
    if same_object:
        o.state.clear()
        o.state.update(wrong)
    else:
        o.state = wrong
    with pytest.raises(ValueError, match="state"):
        o.step([torch.zeros(300)])
    with pytest.raises(ValueError, match="state"):
        o.moments()
    assert o.t == 0


def test_the_width_of_the_moments_is_fixed():
    o = optim.AdamW([torch.zeros(300)], lr=1.0, state_bits=8)
    assert o.bits == 8
    with pytest.raises(AttributeError):
        o.bits = 32


def test_masters_are_part_of_the_state():
    p = torch.randn(5, 60).bfloat16()
    o = optim.AdamW([p, p[:1].clone()], lr=1.0, master=True)
    assert set(o.state) == {"m", "v", "w32"} and o.state["w32"].numel() == o.size == 768
    assert o.w32[0].shape == p.shape and torch.equal(o.w32[0], p.float())
    with pytest.raises(ValueError, match="w32"):
        optim.AdamW([p], lr=1.0, state={k: torch.zeros(512) for k in ("m", "v", "w32")})
    for wrong in (torch.zeros(767), torch.zeros(768, dtype=torch.bfloat16), torch.zeros(2, 384), None):
        with pytest.raises(ValueError, match="w32"):
            optim.AdamW([p, p[:1].clone()], lr=1.0, master=True, state={**o.state, "w32": wrong})
        good, o.state = o.state, {**o.state, "w32": wrong}
        with pytest.raises(ValueError, match="w32"):
            o.step([p, p[:1]])
        o.state = good
    # (as states were held before the masters were part of them)
    given = {k: torch.zeros(768) for k in ("m", "v")}
    r = optim.AdamW([p, p[:1].clone()], lr=1.0, master=True, state=given)
    assert torch.equal(r.w32[0], p.float()) and set(given) == {"m", "v"} and r.state["m"] is given["m"]
    assert optim.AdamW([p.float()], lr=1.0, master=True).w32 is None
