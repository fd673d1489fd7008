"""What a pipeline stage does with its gradients once the backward pass is
over: their global norm (with the factor that clips them, left on the device)
and an AdamW step over all of its tensors at once, with moments in binary32 or
in 8 bits.  Argument marshalling only: the arithmetic is in the HIP kernels of
libtc.so (include/tc.h), and there is no fallback."""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import tc

_WORDS, _N, _POS = C.sizeof(tc.Tensor) // 8, tc.Tensor.n.offset // 8, tc.Tensor.pos.offset // 8     # a row of the library's table

_STATE_TYPES = {torch.float32: 0, torch.uint8: 3, torch.int8: 4}     # as csrc/py_tensors.cpp numbers them

BLOCK = 256     # positions of 8-bit moments that share an exponent

_PY_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtc_py.so")
_py = None


def _native():
    """(tc_py_step, tc_py_table, tc_py_state, tc_py_written) of libtc_py.so (csrc/py_tensors.cpp)"""
    global _py
    if _py is None:
        if not os.path.exists(_PY_PATH):
            raise RuntimeError(f"{_PY_PATH} is missing: build it with paper_2401_07788_amd.build.build()")
        lib = C.PyDLL(_PY_PATH)
        f, g, h, w = lib.tc_py_step, lib.tc_py_table, lib.tc_py_state, lib.tc_py_written
        f.restype, g.restype, h.restype, w.restype = C.c_int, C.py_object, C.c_int, None
        f.argtypes = [C.py_object, C.py_object, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, C.py_object, C.c_int64,
                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_int]
        g.argtypes = [C.py_object, C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int64, C.c_void_p]
        h.argtypes = [C.py_object, C.c_int64, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]
        w.argtypes = [C.py_object]
        _py = f, g, h, w
    return _py


def _table(ts, column: int, sizes, what: str):
    """(table of a list with the tensors' addresses in a column, their
    elements and positions, what keeps their memory); sizes: filled too, or None"""
    if ts and ts[0].dtype not in tc._DT:
        raise TypeError(f"unsupported dtype {ts[0].dtype}")
    table = (tc.Tensor * len(ts))()
    held = _native()[1](ts, C.addressof(table), _WORDS, column, _N, _POS, sizes) if ts else None
    if held is None:
        _check_tensors(ts, what)
        raise ValueError(f"{what}: dense tensors with memory of their own are needed")
    return table, held


def _check_tensors(ts, what: str):
    """one dtype, one device, contiguous"""
    if not ts:
        raise ValueError(f"{what}: an empty list")
    dtype, device = ts[0].dtype, ts[0].device
    if dtype not in tc._DT:
        raise TypeError(f"unsupported dtype {dtype}")
    for t in ts:
        if t.dtype != dtype:
            raise TypeError(f"{what}: {t.dtype} among {dtype}")
        if t.device != device:
            raise ValueError(f"{what}: tensors on {t.device} and {device}")
        if not t.is_contiguous():
            raise ValueError("libtc needs contiguous tensors")
    return dtype, device


class TensorList:
    """tensors of one dtype on one device, as the library takes them: a table
    of addresses and sizes made once.  It keeps the memory that they have now
    (a tensor whose .data is replaced later needs a new list)."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        self.table, self._held = _table(self.tensors, 1, None, "tensors")
        self.dtype, self.device = self.tensors[0].dtype, self.tensors[0].device
        self.ws_bytes = int(tc.lib().tc_grad_norm_workspace_bytes(len(self.tensors)))


# by device and stream, zero between calls: not the boundary's, which graphs may
# hold and which a longer list would replace by a larger one
_ws_cache = {}


def grad_norm(grads, max_norm: float, out: torch.Tensor = None, ws: torch.Tensor = None) -> torch.Tensor:
    """float32 [2]: the norm over all tensors of `grads` (a TensorList or
    tensors), and min(1, max_norm / (norm + 1e-6)), the factor that clips them"""
    lst = grads if isinstance(grads, TensorList) else TensorList(grads)
    tc._need_gpu(lst.tensors[0], out)
    if out is None:
        out = torch.empty(2, dtype=torch.float32, device=lst.device)
    elif out.dtype != torch.float32 or out.numel() != 2 or out.device != lst.device:
        raise ValueError(f"out must be float32 [2] on {lst.device}")
    st = tc._stream(lst.device)
    if ws is None and torch.cuda.is_current_stream_capturing():
        # a graph keeps its own: a larger call would free the stream's under it
        ws = torch.zeros(lst.ws_bytes, dtype=torch.uint8, device=lst.device)
    with tc._stream_lock(lst.device, st):
        if ws is None:
            ws = _ws_cache.get((lst.device.index, st))
            if ws is None or ws.numel() < lst.ws_bytes:
                ws = _ws_cache[(lst.device.index, st)] = torch.zeros(lst.ws_bytes, dtype=torch.uint8, device=lst.device)
        tc._check(tc.lib().tc_grad_norm(lst.table, len(lst.table), tc._DT[lst.dtype], max_norm, out.data_ptr(),
                                        ws.data_ptr(), ws.numel() * ws.element_size(), st), "tc_grad_norm")
    return out


class AdamW:
    """AdamW over a stage's parameters (tensors of one dtype on one device,
    updated in place, which autograd is told; p.data has a version counter of
    its own, so give the parameters themselves).

    state_bits  32: binary32 moments; 8: codes with an exponent per 256 positions
    master      keep the parameters in binary32 beside 16-bit ones, which
                receive their rounding: state["w32"], and w32[k] for tensor k.
                A parameter that something else has set since the last step
                (a checkpoint copied into it) counts instead of its master
    state       what to go on from (as `state` holds it), else moments of zero.
                Masters that it does not hold start from the parameters
    t, seed     steps taken so far, and the seed of 8-bit rounding (the
                step's number is added to it)

    A run goes on as if it had not stopped from its parameters, state, t and
    seed.  Positions: each tensor's moments start at a multiple of 256 in the
    flat arrays `state["m"]`, `state["v"]` and `state["w32"]`; places[k] is
    tensor k's first."""

    def __init__(self, params, lr: float, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 state_bits: int = 32, master: bool = False, state: dict = None, t: int = 0, seed: int = 0):
        self.params = list(params)
        self.sizes = (C.c_int64 * len(self.params))()
        self.table, _ = _table(self.params, 0, self.sizes, "params")
        self.dtype, self.device = self.params[0].dtype, self.params[0].device
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits {state_bits}, not 8 or 32")
        self.lr, self.betas, self.eps, self.weight_decay = lr, betas, eps, weight_decay
        self._bits, self.t, self.seed = state_bits, t, seed
        self.places, size = [], 0
        for n in self.sizes:
            self.places.append(size)
            size += -(-n // BLOCK) * BLOCK
        self.size = size
        self._master = master and self.dtype != torch.float32
        spec = self._spec()
        self._names, self._at = tuple(spec), (C.c_uint64 * len(spec))()
        self._lengths = (C.c_int64 * len(spec))(*(n for n, _ in spec.values()))
        self._types = (C.c_int8 * len(spec))(*(_STATE_TYPES[dt] for _, dt in spec.values()))
        self.state = state if state is not None else {k: torch.zeros(n, dtype=dt, device=self.device)
                                                      for k, (n, dt) in spec.items() if k != "w32"}
        if not self._master and "w32" in self.state:
            raise ValueError("state holds masters ('w32') and this optimizer keeps none")
        if self._master and "w32" not in self.state:
            self.state = {**self.state, "w32": torch.zeros(size, dtype=torch.float32, device=self.device)}
            for w, p in zip(self.w32, self.params):
                w.copy_(p.detach())
        self._check_state()
        self._w32_at = 0

    @property
    def bits(self) -> int:
        """32 or 8: what the moments are held in"""
        return self._bits

    @property
    def w32(self):
        """the masters, a view of the state for each tensor (None: there are none)"""
        if not self._master:
            return None
        return [self.state["w32"][a:a + p.numel()].view(p.shape) for a, p in zip(self.places, self.params)]

    def _refuse(self, grads):
        """what is wrong with the tensors of a step"""
        if len(grads) != len(self.params):
            raise ValueError(f"{len(grads)} gradients for {len(self.params)} parameters")
        if any(g is None for g in grads):
            raise ValueError("a parameter has no gradient")
        _, device = _check_tensors(grads, "gradients")
        if device != self.device:
            raise ValueError(f"gradients must be on {self.device}")
        if [g.numel() for g in grads] != list(self.sizes):
            raise ValueError("a gradient does not fit its parameter")
        tc._need_gpu(*grads, *self.params)
        raise ValueError("a parameter changed its dtype, device or size")

    def _spec(self):
        blocks, spec = self.size // BLOCK, {}
        if self.bits == 32:
            spec.update(m=(self.size, torch.float32), v=(self.size, torch.float32))
        else:
            spec.update(m=(self.size, torch.uint8), v=(self.size, torch.uint8),
                        em=(blocks, torch.int8), ev=(blocks, torch.int8))
        if self._master:
            spec["w32"] = (self.size, torch.float32)
        return spec

    def _check_state(self):
        for k, (n, dt) in self._spec().items():
            s = self.state.get(k)
            if s is None or s.dtype != dt or s.dim() != 1 or s.numel() != n or s.device != self.device or \
                    not s.is_contiguous():
                raise ValueError(f"state[{k!r}] must be {dt} [{n}] on {self.device}")

    def _state_addresses(self):
        """where the state's tensors lie now, in their order"""
        tensors, dev = [self.state.get(k) for k in self._names], self.device
        if dev.type != "cuda" or not _native()[2](tensors, len(tensors), self._lengths, self._types, dev.index, self._at):
            self._check_state()
            tc._need_gpu(*tensors)
            raise ValueError("state: dense tensors with memory of their own are needed")
        return self._at

    def step(self, grads=None, clip: torch.Tensor = None):
        """one step.  grads: a tensor per parameter (of one dtype), else their
        .grad; clip: what grad_norm returned, else the gradients as they are.
        Where the norm is not finite nothing is changed but the step count.
        Not for a graph: the step's number and seed are part of the call."""
        if grads is None:
            grads = [p.grad for p in self.params]
        grads, dev = list(grads), self.device
        if clip is not None and (clip.dtype != torch.float32 or clip.numel() != 2 or clip.device != dev or
                                 not clip.is_contiguous()):
            raise ValueError(f"clip must be float32 [2] on {dev}")
        if dev.type == "cuda" and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a captured step would repeat its number and seed at every replay")
        # (all of them may have been replaced, or changed their memory, since they were looked at last)
        state, at = [self.state.get(k) for k in self._names], self._at
        dts = _native()[0](self.params, grads, len(self.table), self.sizes, C.addressof(self.table), _WORDS, state,
                           len(state), self._lengths, self._types, at, dev.index) if dev.type == "cuda" else -1
        if dts & 3 != tc._DT[self.dtype]:
            self._check_state()
            self._refuse(grads)
        if self._master and at[-1] != self._w32_at:
            self._w32_at = at[-1]
            for row in self.table:
                row.w32 = at[-1] + 4 * row.pos
        t = self.t + 1
        a = tc.AdamwSettings(self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay, t, self.bits,
                             (self.seed + 1) & 0x7FFFFFFF, *at[:4 if self.bits == 8 else 2])
        tc._check(tc.lib().tc_adamw_step(C.byref(a), self.table, len(self.table), dts & 3, dts >> 2,
                                         tc._ptr(clip), tc._stream(dev)), "tc_adamw_step")
        _native()[3](self.params)
        self.t, self.seed = t, (self.seed + 1) & 0x7FFFFFFF

    def moments(self):
        """(m, v) as float32 [positions]: the state itself, or the values that
        its codes stand for"""
        if self.bits == 32:
            self._check_state()
            return self.state["m"], self.state["v"]
        am, av, aem, aev = self._state_addresses()[:4]
        m = torch.empty(self.size, dtype=torch.float32, device=self.device)
        v = torch.empty(self.size, dtype=torch.float32, device=self.device)
        tc._check(tc.lib().tc_adamw_moments(am, aem, av, aev, self.size, m.data_ptr(), v.data_ptr(),
                                            tc._stream(self.device)), "tc_adamw_moments")
        return m, v
