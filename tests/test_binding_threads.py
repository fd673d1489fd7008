"""Host threads on one stream: a call's launches, all of which use the stream's
one workspace, are not interrupted by another call's.  The foreign calls are
replaced here by ones that wait for a second one to enter (a foreign call
releases the interpreter's lock, so a second thread may); no GPU is used."""
import ctypes as C
import threading
import types

import pytest
import torch

from paper_2401_07788_amd import head, optim, tc


class Library:
    """stands for the library: a call stays until another one enters the same workspace, or for a moment"""

    def __init__(self):
        self.inside, self.met, self.calls, self.lock = [], False, [], threading.Condition()

    def launch(self, name, ws):
        with self.lock:
            if ws in self.inside:
                self.met = True
            self.inside.append(ws)
            self.calls.append(name)
            self.lock.notify_all()
            self.lock.wait_for(lambda: self.met, timeout=0.3)
            self.inside.remove(ws)
        return 0

    def tc_xent_workspace_bytes(self, c, grad, n):
        C.cast(n, C.POINTER(C.c_size_t))[0] = 5000
        return 0

    def tc_xent_loss(self, *a):
        return self.launch("loss", a[-3])

    def tc_xent_step(self, *a):
        return self.launch("step", a[-3])

    def tc_grad_norm_workspace_bytes(self, n):
        return 5000

    def tc_grad_norm(self, *a):
        return self.launch("norm", a[-3])

    def tc_workspace_bytes(self, c, n):
        C.cast(n, C.POINTER(C.c_size_t))[0] = 5000
        return 0

    def tc_quant_group_bytes(self, length, bits):
        return length

    def __getattr__(self, name):
        if name not in ("tc_topk_compress", "tc_quant_pack", "tc_ef_step", "tc_aqsgd_step"):
            raise AttributeError(name)
        return lambda *a: self.launch(name, a[-3])


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(tc, "lib", lambda: lib)
    monkeypatch.setattr(tc, "_need_gpu", lambda *ts: None)
    monkeypatch.setattr(tc, "_stream", lambda device: 0)
    monkeypatch.setattr(tc, "_ws_cache", {})
    monkeypatch.setattr(head, "_ws_cache", {})
    monkeypatch.setattr(optim, "_ws_cache", {}, raising=False)
    monkeypatch.setattr(tc, "_plans", {})
    monkeypatch.setattr(head, "_ws_bytes", {})
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=0))
    return lib


X, W, T = torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int64)
E = torch.zeros(4, 8)
G = [torch.zeros(10), torch.zeros(3)]
CALLS = {
    "loss": lambda: head.linear_xent(X, W, T),
    "step": lambda: head.linear_xent_step(X, W, T),
    "norm": lambda: optim.grad_norm(G, 1.0),
    "tc_topk_compress": lambda: tc.topk_compress(X, 2, 4),
    "tc_quant_pack": lambda: tc.quant_pack(X, 4, 4),
    "tc_ef_step": lambda: tc.ef_step_topk(X, E, 2, 4),
    "tc_ef_step ": lambda: tc.ef_step_quant(X, E, 4, 4),
    "tc_ef_step  ": lambda: tc.ef_step_topk_quant(X, E, 2, 4, 4),
    "tc_aqsgd_step": lambda: tc.aqsgd_step(X, E, T, 2),
}


@pytest.mark.parametrize("first,second", [("loss", "loss"), ("step", "step"), ("loss", "step"), ("norm", "norm"),
                                          *((c, "tc_topk_compress") for c in CALLS if c.startswith("tc_"))])
def test_calls_on_one_stream_take_turns(library, first, second):
    CALLS[first](), CALLS[second]()              # (the stream has its workspace)
    library.calls.clear()
    threads = [threading.Thread(target=CALLS[c]) for c in (first, second)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert sorted(library.calls) == sorted([first.strip(), second])
    assert not library.met


def test_the_norm_leaves_the_boundarys_workspace_alone(library):
    """a graph may hold that of a boundary call; a longer list of gradients does not replace it"""
    small = tc._ws_cache[(None, 0)] = torch.zeros(100, dtype=torch.uint8)
    optim.grad_norm(G, 1.0)
    assert tc._ws_cache == {(None, 0): small}
    large = tc._ws_cache[(None, 0)] = torch.zeros(1 << 20, dtype=torch.uint8)
    library.inside.append(large.data_ptr())
    optim.grad_norm(G, 1.0)
    assert not library.met
