"""What the loss's entry points refuse, on the host and before any device call."""
import ctypes as C

import pytest
import torch

from paper_2401_07788_amd import head, tc


def test_python_refusals():
    x, w, t = torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        head.linear_xent(x, w, t)
    with pytest.raises(ValueError, match="rows of"):
        head.linear_xent(x, torch.zeros(5, 9), t)
    with pytest.raises(TypeError, match="share a dtype"):
        head.linear_xent(x, w.half(), t)
    with pytest.raises(ValueError, match="int64"):
        head.linear_xent(x, w, t.int())
    with pytest.raises(ValueError, match="int64"):
        head.linear_xent(x, w, t[:3])
    with pytest.raises(ValueError, match="matrix"):
        head.linear_xent(x[0], w, t)
    with pytest.raises(ValueError, match="contiguous rows"):
        head.linear_xent(torch.zeros(8, 4).t(), w, t)
    with pytest.raises(ValueError, match="overlap"):
        head.linear_xent(torch.zeros(1, 8).expand(4, 8), w, t)
    with pytest.raises(ValueError, match="GPU"):
        head.linear_xent_step(x, w, t, torch.zeros(4))


BASE = 1 << 40          # never dereferenced: the checks fail first


def sizes(**kw):
    d = dict(n=4, v=5, h=8, ldx=8, ldw=8, ignore=-100, chunk=0, dt=0, reserved=0)
    d.update(kw)
    return tc.Xent(**d)


@pytest.mark.parametrize("kw,want", [
    (dict(dt=3), tc.TC_ERR_DTYPE),
    (dict(reserved=1), tc.TC_ERR_ARG),
    (dict(n=1 << 31), tc.TC_ERR_ARG),
    (dict(v=0), tc.TC_ERR_ARG),
    (dict(v=(1 << 22) + 1), tc.TC_ERR_ARG),
    (dict(h=0), tc.TC_ERR_ARG),
    (dict(h=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), tc.TC_ERR_ARG),
    (dict(ldx=7), tc.TC_ERR_ARG),
    (dict(ldw=7), tc.TC_ERR_ARG),
    (dict(chunk=1 << 23), tc.TC_ERR_ARG),
])
def test_sizes_refused(kw, want):
    L = tc.lib()
    c, n = sizes(**kw), C.c_size_t(0)
    assert L.tc_xent_workspace_bytes(C.byref(c), 1, C.byref(n)) == want
    a = [BASE + (k << 30) for k in range(9)]
    assert L.tc_xent_step(C.byref(c), *a, 1 << 30, None) == want
    assert L.tc_xent_loss(C.byref(c), *a[:5], a[5], 1 << 30, None) == want


def test_pointers_and_workspace():
    L = tc.lib()
    c, n = sizes(), C.c_size_t(0)
    assert L.tc_xent_workspace_bytes(None, 1, C.byref(n)) == tc.TC_ERR_NULL
    assert L.tc_xent_workspace_bytes(C.byref(c), 1, None) == tc.TC_ERR_NULL
    a = [BASE + (k << 30) for k in range(9)]      # x w target weight loss lse dx dw ws
    for k in (0, 1, 2, 4, 5, 6, 7):
        b = list(a)
        b[k] = None
        assert L.tc_xent_step(C.byref(c), *b, 1 << 30, None) == tc.TC_ERR_NULL
    b = list(a)
    b[0] += 2
    assert L.tc_xent_step(C.byref(c), *b, 1 << 30, None) == tc.TC_ERR_ALIGN
    b = list(a)
    b[8] = None
    assert L.tc_xent_step(C.byref(c), *b, 1 << 30, None) == tc.TC_ERR_WORKSPACE
    assert L.tc_xent_step(C.byref(c), *a, 100, None) == tc.TC_ERR_WORKSPACE
    b = list(a)
    b[8] += 16
    assert L.tc_xent_step(C.byref(c), *b, 1 << 30, None) == tc.TC_ERR_ALIGN
    e = sizes(n=0)
    assert L.tc_xent_loss(C.byref(e), None, None, None, None, None, None, 0, None) == 0


def test_workspace_sizes():
    """a smaller chunk needs less; the loss alone far less than the step"""
    L = tc.lib()

    def need(grad, **kw):
        c, n = sizes(n=100000, v=50257, h=768, ldx=768, ldw=768, dt=1, **kw), C.c_size_t(0)
        assert L.tc_xent_workspace_bytes(C.byref(c), grad, C.byref(n)) == 0
        return n.value

    assert need(1, chunk=128) < need(1, chunk=1024) < need(1) < (10 << 30)
    assert need(0) < need(1)
    assert need(1, chunk=1024) < 1024 * 50304 * 4 + (1 << 30)


def test_overlapping_buffers_in_the_debug_library():
    D = tc.load(tc.DEBUG_LIB_PATH)
    c = sizes()
    a = [BASE + (k << 30) for k in range(9)]
    a[6] = a[0]
    assert D.tc_xent_step(C.byref(c), *a, 1 << 30, None) == tc.TC_ERR_PRECONDITION


def test_forward_mode_is_refused():
    """a dual tensor's derivative would else come back as none, which counts as zero"""
    x, w, t, g = torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    with torch.autograd.forward_ad.dual_level():
        dx, dw, dg = (torch.autograd.forward_ad.make_dual(a, torch.ones_like(a)) for a in (x, w, g))
        for a, b in ((dx, w), (x, dw), (dx.requires_grad_(), w)):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                head.linear_xent(a, b, t)
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                head.linear_xent(a, b, t)
            with pytest.raises(NotImplementedError, match="forward-mode"):
                head.linear_xent_step(a, b, t)
        with pytest.raises(NotImplementedError, match="forward-mode"):
            head.linear_xent_step(x, w, t, dg)
        # (others go on: to the refusal of tensors that are not on a GPU)
        with pytest.raises(ValueError, match="GPU"):
            head.linear_xent(x, w, t)
