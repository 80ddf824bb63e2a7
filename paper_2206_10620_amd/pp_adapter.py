"""ctypes binding with the same names as include/pp_adapter.h and include/pp_act8.h (argument marshalling only).

The library cannot see a tensor's sizes, type or device: they are checked here, by statements that python -O keeps."""
from __future__ import annotations

import ctypes as C
import functools
from array import array
from typing import NamedTuple, Optional, Sequence, Union

from .pp_block_gemm import BlockPlan, lib as _block_lib
from .pp_conv import PP_OK, PP_F16, PP_F32, PP_FLAG_HOST_ONLY, PPError


class _Desc(C.Structure):
    _fields_ = [("m", C.c_int32), ("k", C.c_int32), ("slots", C.c_int32), ("max_rank", C.c_int32), ("dtype", C.c_int32), ("flags", C.c_uint32)]


_ready = False


def lib() -> C.CDLL:
    """The loaded HIP library (the same shared object as the convolution's; no fallback)."""
    global _ready
    L = _block_lib()
    if not _ready:
        vp, i32 = C.c_void_p, C.c_int32
        signatures = {
            "pp_act8_pack": [vp, i32, i32, i32, vp, vp],
            "pp_act8_unpack": [vp, i32, i32, i32, vp, vp],
            "pp_adapter_plan": [C.POINTER(_Desc), C.POINTER(vp)],
            "pp_adapter_load": [vp, i32, i32, C.c_float, vp, vp, vp],
            "pp_adapter_load_many": [vp, i32, vp, vp, vp, vp, vp, vp],
            "pp_adapter_project": [vp, vp, vp, vp, i32, vp],
            "pp_adapter_run": [vp, vp, vp, vp, vp, vp, i32, vp],
            "pp_adapter_grad_input": [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp],
            "pp_adapter_grad_weights": [vp, vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp, i32, vp],
            "pp_adapter_destroy": [vp],
        }
        for name, types in signatures.items():
            getattr(L, name).argtypes = types
            getattr(L, name).restype = C.c_int
        for name, types in {"pp_act8_bytes": [i32, i32], "pp_adapter_u_bytes": [vp, i32], "pp_adapter_v_bytes": [vp, i32],
                            "pp_adapter_work_bytes": [vp, i32, i32]}.items():
            getattr(L, name).argtypes = types
            getattr(L, name).restype = C.c_int64
        _ready = True
    return L


def pp_act8_bytes(rows: int, n: int) -> int:
    return lib().pp_act8_bytes(rows, n)


_act8_bytes = functools.lru_cache(maxsize=1024)(pp_act8_bytes)


def pp_act8_pack(x_dev: int, rows: int, n: int, dtype: int, held_dev: int, hip_stream: int = 0) -> int:
    return lib().pp_act8_pack(x_dev, rows, n, dtype, held_dev, hip_stream)


def pp_act8_unpack(held_dev: int, rows: int, n: int, dtype: int, x_dev: int, hip_stream: int = 0) -> int:
    return lib().pp_act8_unpack(held_dev, rows, n, dtype, x_dev, hip_stream)


def pp_adapter_plan(m: int, k: int, slots: int, max_rank: int, dtype: int = PP_F16, flags: int = 0):
    """Returns (status, handle)."""
    d = _Desc(m, k, slots, max_rank, dtype, flags)
    h = C.c_void_p()
    st = lib().pp_adapter_plan(C.byref(d), C.byref(h))
    return st, (h if st == PP_OK else None)


def pp_adapter_load(bank, slot: int, rank: int, scale: float, a_dev: int, b_dev: int, hip_stream: int = 0) -> int:
    return lib().pp_adapter_load(bank, slot, rank, scale, a_dev, b_dev, hip_stream)


def pp_adapter_load_many(bank, slots, ranks, scales, a_dev, b_dev, hip_stream: int = 0) -> int:
    """The five sequences have one entry a slot; 0 stands for a null pointer."""
    if not (len(slots) == len(ranks) == len(scales) == len(a_dev) == len(b_dev)):
        raise AssertionError("sequences of different lengths")
    lists = array("i", slots), array("i", ranks), array("f", scales), array("Q", a_dev), array("Q", b_dev)
    return lib().pp_adapter_load_many(bank, len(slots), *[t.buffer_info()[0] for t in lists], hip_stream)


def pp_adapter_u_bytes(bank, n: int) -> int:
    return lib().pp_adapter_u_bytes(bank, n)


def pp_adapter_v_bytes(bank, n: int) -> int:
    return lib().pp_adapter_v_bytes(bank, n)


def pp_adapter_work_bytes(bank, n: int, count: int) -> int:
    return lib().pp_adapter_work_bytes(bank, n, count)


def pp_adapter_project(bank, x_dev: int, slot_of_dev: int, u_dev: int, n: int, hip_stream: int = 0) -> int:
    return lib().pp_adapter_project(bank, x_dev, slot_of_dev, u_dev, n, hip_stream)


def pp_adapter_run(bank, plan, x_dev: int, slot_of_dev: int, u_dev: int, y_dev: int, n: int, hip_stream: int = 0) -> int:
    return lib().pp_adapter_run(bank, plan, x_dev, slot_of_dev, u_dev, y_dev, n, hip_stream)


def pp_adapter_grad_input(bank, plan_t, dy_dev: int, gate_dev: int, g_dev: int, slot_of_dev: int, v_dev: int, dx_dev: int, n: int, hip_stream: int = 0) -> int:
    return lib().pp_adapter_grad_input(bank, plan_t, dy_dev, gate_dev, g_dev, slot_of_dev, v_dev, dx_dev, n, hip_stream)


def pp_adapter_grad_weights(bank, x_dev: int, x_is_act8: int, u_dev: int, g_dev: int, v_dev: int, slot_of_dev: int, which_dev: int, count: int,
                            da_dev: int, db_dev: int, work_dev: int, n: int, hip_stream: int = 0) -> int:
    return lib().pp_adapter_grad_weights(bank, x_dev, x_is_act8, u_dev, g_dev, v_dev, slot_of_dev, which_dev, count, da_dev, db_dev, work_dev, n, hip_stream)


def pp_adapter_destroy(bank) -> int:
    return lib().pp_adapter_destroy(bank)


_TORCH = None


def _torch():
    """torch, imported when it is first needed (the plain entry points above do without)."""
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _torch_dtype(dtype: int):
    t = _TORCH or _torch()
    return t.float16 if dtype == PP_F16 else t.float32


class _Call:
    """The device and stream of a call: the tensors' device is made current, and what the call allocates belongs to the stream it
    runs on."""

    def __init__(self, device, stream: Optional[int]):
        t = _torch()
        self._device = t.cuda.device(device)
        self._stream = None
        if stream is not None:
            self._stream = t.cuda.stream(t.cuda.ExternalStream(stream, device=device) if stream else t.cuda.default_stream(device))

    def __enter__(self) -> int:
        self._device.__enter__()
        if self._stream is not None:
            self._stream.__enter__()
        return _TORCH.cuda.current_stream().cuda_stream

    def __exit__(self, *exc):
        if self._stream is not None:
            self._stream.__exit__(*exc)
        self._device.__exit__(*exc)


def _on(device, stream: Optional[int], call):
    """call(handle of the stream it is to run on).  On the current device and stream, the usual case, nothing has to be changed and put
    back: two contexts would take longer than a small kernel."""
    t = _TORCH or _torch()
    if stream is None and t.cuda.current_device() == device.index:
        return call(t._C._cuda_getCurrentRawStream(device.index))
    with _Call(device, stream) as s:
        return call(s)


def _check_status(st: int, what: str) -> None:
    if st != PP_OK:
        raise PPError(st, what)


def _matrix(t, rows: int, n: Optional[int], dtype: int, device=None):
    if not (t.is_cuda and t.is_contiguous() and t.dim() == 2 and t.dtype == _torch_dtype(dtype) and t.shape[0] == rows):
        raise AssertionError("not a contiguous [rows, n] tensor of the bank's dtype on the GPU")
    if not (n is None or t.shape[1] == n):
        raise AssertionError("another number of tokens")
    if not (device is None or t.device == device):
        raise AssertionError("on another device")


def _opaque_ok(t, device):
    """t is memory of the kind that the calls here leave their state in."""
    if not (t.is_cuda and t.device == device and t.element_size() == 1 and t.is_contiguous()):
        raise AssertionError("not memory of the bank's device that a call here left")


class Act8:
    """A matrix [rows, n] held in 8 bits (buffer: pp_act8.h's form)."""

    __slots__ = ("buffer", "rows", "n", "dtype")

    def __init__(self, buffer, rows: int, n: int, dtype: int):
        if not (0 < _act8_bytes(rows, n) == buffer.numel()):
            raise AssertionError("a buffer of another size")
        _opaque_ok(buffer, buffer.device)
        self.buffer, self.rows, self.n, self.dtype = buffer, rows, n, dtype

    def unpack(self, dtype: Optional[int] = None, stream: Optional[int] = None):
        """The values held, as a tensor of dtype (default: that of the tensor that was packed)."""
        dtype = self.dtype if dtype is None else dtype
        device = self.buffer.device

        def call(s):
            out = _TORCH.empty((self.rows, self.n), dtype=_torch_dtype(dtype), device=device)
            _check_status(lib().pp_act8_unpack(self.buffer.data_ptr(), self.rows, self.n, dtype, out.data_ptr(), s), "pp_act8_unpack")
            return out
        return _on(device, stream, call)


def act8_pack(x, stream: Optional[int] = None) -> Act8:
    """x [rows, n] (fp16 or fp32, on the GPU) in 8 bits."""
    torch = _TORCH or _torch()
    dtype = PP_F16 if x.dtype == torch.float16 else PP_F32
    if not (x.is_cuda and x.is_contiguous() and x.dim() == 2 and x.dtype == _torch_dtype(dtype)):
        raise AssertionError("not a contiguous [rows, n] tensor of fp16 or fp32 on the GPU")
    rows, n = x.shape
    device = x.device

    def call(s):
        buf = torch.empty(_act8_bytes(rows, n), dtype=torch.uint8, device=device)
        _check_status(lib().pp_act8_pack(x.data_ptr(), rows, n, dtype, buf.data_ptr(), s), "pp_act8_pack")
        return Act8(buf, rows, n, dtype)
    return _on(device, stream, call)


class InputGradient(NamedTuple):
    """What grad_input leaves: dx (None if not asked for), v (opaque, for grad_weights) and g (dy behind the ReLU's gate)."""
    dx: object
    v: object
    g: object


class AdapterBank:
    """Owns one bank of adapters; the methods take torch tensors only to read their device pointers."""

    def __init__(self, m: int, k: int, slots: int, max_rank: int, dtype: int = PP_F16, device=None):
        torch = _torch()
        self.handle = None
        self.m, self.k, self.slots, self.max_rank, self.dtype = m, k, slots, max_rank, dtype
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        with torch.cuda.device(self.device):
            st, self.handle = pp_adapter_plan(m, k, slots, max_rank, dtype)
        _check_status(st, "pp_adapter_plan")
        self._state_bytes = functools.lru_cache(maxsize=1024)(lambda n, h=self.handle: (pp_adapter_u_bytes(h, n), pp_adapter_v_bytes(h, n)))
        self._work_bytes = functools.lru_cache(maxsize=1024)(lambda n, count, h=self.handle: pp_adapter_work_bytes(h, n, count))

    def _slots_of(self, slot_of, n: int):
        torch = _torch()
        if not (slot_of.is_cuda and slot_of.is_contiguous() and slot_of.dtype == torch.int32 and tuple(slot_of.shape) == (n,) and slot_of.device == self.device):
            raise AssertionError("slot_of is a contiguous int32 tensor of a slot for every token, on the bank's device")

    def _opaque(self, nbytes: int):
        return _TORCH.empty(nbytes, dtype=_TORCH.uint8, device=self.device)

    def load(self, slot: int, a, b, scale: float, stream: Optional[int] = None) -> None:
        """a [rank, k] and b [m, rank] into a slot.  They may be freed or changed once the stream has got there."""
        rank = a.shape[0]
        _matrix(a, rank, self.k, self.dtype, self.device)
        _matrix(b, self.m, rank, self.dtype, self.device)
        _on(self.device, stream, lambda s: _check_status(
            lib().pp_adapter_load(self.handle, slot, rank, scale, a.data_ptr(), b.data_ptr(), s), "pp_adapter_load"))

    def load_many(self, slots: Sequence[int], a, b, scales: Sequence[float], stream: Optional[int] = None) -> None:
        """a[i] [rank, k] and b[i] [m, rank] into slots[i], for all i in one call (in their order, where a slot stands twice; no slots: nothing)."""
        if not (len(slots) == len(a) == len(b) == len(scales)):
            raise AssertionError("sequences of different lengths")
        if len(slots) < 2:                         # the lists alone would cost 1.5 us
            return self.load(slots[0], a[0], b[0], scales[0], stream) if len(slots) else None
        tdt, index, t = _torch_dtype(self.dtype), self.device.index, _TORCH.Tensor
        both = [*a, *b]                            # a list of 64 slots takes 60 us to look over one tensor after another, 45 check by check
        sizes = list(map(t.size, a))
        ranks = [s[0] if len(s) == 2 else -1 for s in sizes]
        if not (sizes == [(r, self.k) for r in ranks] and list(map(t.size, b)) == [(self.m, r) for r in ranks]):
            raise AssertionError("a is [rank, k] and b [m, rank]")
        if not (all([x.dtype is tdt for x in both]) and set(map(t.get_device, both)) == {index} and all(map(t.is_contiguous, both))):
            raise AssertionError("a and b are contiguous tensors of the bank's dtype on its device")
        at = list(map(t.data_ptr, both))
        _on(self.device, stream, lambda s: _check_status(
            pp_adapter_load_many(self.handle, slots, ranks, scales, at[:len(a)], at[len(a):], s), "pp_adapter_load_many"))

    def unload(self, slot: int, stream: Optional[int] = None) -> None:
        _on(self.device, stream, lambda s: _check_status(lib().pp_adapter_load(self.handle, slot, 0, 0.0, None, None, s), "pp_adapter_load"))

    def project(self, x, slot_of, stream: Optional[int] = None):
        """u = A x alone (opaque, for grad_weights): what run(keep=True) returns beside y."""
        _matrix(x, self.k, None, self.dtype, self.device)
        n = x.shape[1]
        self._slots_of(slot_of, n)

        def call(s):
            u = self._opaque(self._state_bytes(n)[0])
            _check_status(lib().pp_adapter_project(self.handle, x.data_ptr(), slot_of.data_ptr(), u.data_ptr(), n, s), "pp_adapter_project")
            return u
        return _on(self.device, stream, call)

    def run(self, plan: BlockPlan, x, slot_of, y=None, keep: bool = False, stream: Optional[int] = None):
        """y = act(W x + bias + c B (A x)); with keep also u, which grad_weights takes."""
        _matrix(x, self.k, None, self.dtype, self.device)
        n = x.shape[1]
        self._slots_of(slot_of, n)
        if y is not None:
            _matrix(y, self.m, n, self.dtype, self.device)

        def call(s):
            out = _TORCH.empty((self.m, n), dtype=x.dtype, device=self.device) if y is None else y
            u = self._opaque(self._state_bytes(n)[0])
            _check_status(lib().pp_adapter_run(self.handle, plan.handle, x.data_ptr(), slot_of.data_ptr(), u.data_ptr(), out.data_ptr(), n, s),
                          "pp_adapter_run")
            return (out, u) if keep else out
        return _on(self.device, stream, call)

    def grad_input(self, plan_t: Optional[BlockPlan], dy, slot_of, gate: Optional[Act8] = None, stream: Optional[int] = None) -> InputGradient:
        """dx = W^T g + c A^T (B^T g) through plan_t, the plan of the transposed weights (None: no dx), g = dy where the output held
        in gate is above 0 (None: everywhere)."""
        _matrix(dy, self.m, None, self.dtype, self.device)
        n = dy.shape[1]
        self._slots_of(slot_of, n)
        if not (gate is None or (gate.rows == self.m and gate.n == n and gate.buffer.device == self.device)):
            raise AssertionError("the gate is the output [m, n] in 8 bits, on the bank's device")

        def call(s):
            torch = _TORCH
            g = dy if gate is None else torch.empty_like(dy)
            dx = None if plan_t is None else torch.empty((self.k, n), dtype=dy.dtype, device=self.device)
            v = self._opaque(self._state_bytes(n)[1])
            st = lib().pp_adapter_grad_input(self.handle, None if plan_t is None else plan_t.handle, dy.data_ptr(),
                                             None if gate is None else gate.buffer.data_ptr(), None if gate is None else g.data_ptr(),
                                             slot_of.data_ptr(), v.data_ptr(), None if dx is None else dx.data_ptr(), n, s)
            _check_status(st, "pp_adapter_grad_input")
            return InputGradient(dx, v, g)
        return _on(self.device, stream, call)

    def grad_weights(self, x: Union["Act8", object], u, g, v, slot_of, which, stream: Optional[int] = None):
        """Gradients of the slots that which (int32 tensor) lists: da [count, max_rank, k], db [count, m, max_rank], fp32.  x: the
        layer's input, as it was or in 8 bits (where padding tokens have to be zeros: 128 tokens share a step); u of run or project, g and
        v of grad_input."""
        torch = _TORCH or _torch()
        _matrix(g, self.m, None, self.dtype, self.device)
        n = g.shape[1]
        self._slots_of(slot_of, n)
        held = isinstance(x, Act8)
        if held:
            if not (x.rows == self.k and x.n == n and x.buffer.device == self.device):
                raise AssertionError("x is the input [k, n], on the bank's device")
        else:
            _matrix(x, self.k, n, self.dtype, self.device)
        if not (which.is_cuda and which.is_contiguous() and which.dtype == torch.int32 and which.dim() == 1 and which.device == self.device):
            raise AssertionError("which is a contiguous int32 tensor on the bank's device")
        if not ((u.numel(), v.numel()) == self._state_bytes(n)):
            raise AssertionError("u and v are those of this many tokens")
        _opaque_ok(u, self.device)
        _opaque_ok(v, self.device)
        count = which.shape[0]

        def call(s):
            da = torch.empty((count, self.max_rank, self.k), dtype=torch.float32, device=self.device)
            db = torch.empty((count, self.m, self.max_rank), dtype=torch.float32, device=self.device)
            work = self._opaque(self._work_bytes(n, count))
            st = lib().pp_adapter_grad_weights(self.handle, (x.buffer if held else x).data_ptr(), 1 if held else 0, u.data_ptr(), g.data_ptr(),
                                               v.data_ptr(), slot_of.data_ptr(), which.data_ptr(), count, da.data_ptr(), db.data_ptr(),
                                               work.data_ptr(), n, s)
            _check_status(st, "pp_adapter_grad_weights")
            return da, db
        return _on(self.device, stream, call)

    def close(self):
        if self.handle is not None:
            pp_adapter_destroy(self.handle)
            self.handle = None
            self._state_bytes, self._work_bytes = lambda n: (0, 0), lambda n, count: 0      # calls from now on are refused

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
