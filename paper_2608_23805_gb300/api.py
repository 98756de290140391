"""Convenience wrapper over the C ABI for PyTorch callers.

PyTorch supplies device memory, pinned host memory and streams; every step of
the MoE layer forward, of the key-value cache and of the operators beside them
(4-bit products, rotation, sampling) runs in libmsi.so's CUDA kernels.  This
module only marshals tensors into pointers and checks status codes.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from . import native as N


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _flags(residual: bool, single_cta: bool, shared_gate: bool = True, split_waves: bool = False) -> int:
    return ((N.MSI_FWD_RESIDUAL if residual else 0) | (N.MSI_FWD_SINGLE_CTA if single_cta else 0)
            | (0 if shared_gate else N.MSI_FWD_SHARED_UNGATED)
            | (N.MSI_FWD_SPLIT_WAVES if split_waves else 0))


def _stream(s) -> int | None:
    s = torch.cuda.current_stream() if s is None else s
    return s.cuda_stream


class RouteEvent:
    """Device buffers of one layer call's route event."""

    def __init__(self, T: int, k: int, E: int, device="cuda"):
        self.ids = torch.empty((T, k), dtype=torch.int32, device=device)
        self.weights = torch.empty((T, k), dtype=torch.float32, device=device)
        self.counts = torch.empty((E,), dtype=torch.int32, device=device)
        self.gap = torch.empty((T,), dtype=torch.float32, device=device)
        self.c = N.msi_route_event(_ptr(self.ids) if T else None, _ptr(self.weights) if T else None,
                                   _ptr(self.counts), _ptr(self.gap) if T else None)


class Plan:
    """A Plan over one slot pool (see include/msi.h, msi_plan_desc)."""

    def __init__(self, *, n_layers, n_experts, top_k, hidden, inter, n_slots, host_windows,
                 has_shared=False, shared_w=None, shared_gate_w=None, wdtype=N.MSI_W_BF16,
                 slot_pool=None, extent_off=None, wave_capacity=0, wait_timeout_s=0.0,
                 early_staging=False):
        """early_staging: give streamed calls an early-staging buffer of one
        wave of extents (msi_plan_set_bounce)."""
        lib = N.lib()
        self.E, self.k, self.H, self.I = n_experts, top_k, hidden, inter
        self.n_layers, self.S = n_layers, n_slots
        self.extent_bytes = int(lib.msi_extent_bytes(hidden, inter, wdtype))
        if self.extent_bytes == 0:
            raise ValueError("bad shape")
        if slot_pool is None:
            slot_pool = torch.empty(n_slots * self.extent_bytes, dtype=torch.uint8, device="cuda")
        self._keep = [host_windows, slot_pool, shared_w, shared_gate_w]
        self.slot_pool = slot_pool
        self._off = None
        if extent_off is not None:
            self._off = np.ascontiguousarray(extent_off, dtype=np.uint64)
        d = N.msi_plan_desc()
        d.n_layers, d.n_experts, d.top_k = n_layers, n_experts, top_k
        d.hidden, d.inter, d.has_shared, d.wdtype, d.n_slots = hidden, inter, int(has_shared), wdtype, n_slots
        d.slot_pool = slot_pool.data_ptr()
        d.extent_bytes = self.extent_bytes
        d.host_windows = host_windows.data_ptr()
        d.extent_off = self._off.ctypes.data if self._off is not None else None
        d.shared_w = _ptr(shared_w)
        d.shared_gate_w = _ptr(shared_gate_w)
        d.wave_capacity = wave_capacity
        d.wait_timeout_s = wait_timeout_s
        h = ctypes.c_void_p()
        N.check(lib.msi_plan_create(ctypes.byref(d), ctypes.byref(h)), "msi_plan_create")
        self.h = h
        self._ws = {}
        self._ws_bytes = {}
        self.bounce = None
        if early_staging:
            C = wave_capacity if wave_capacity > 0 else n_slots // 2
            self.bounce = torch.empty(C * self.extent_bytes, dtype=torch.uint8, device="cuda")
            N.check(lib.msi_plan_set_bounce(self.h, self.bounce.data_ptr(), self.bounce.numel()),
                    "msi_plan_set_bounce")

    # -- residency ---------------------------------------------------------
    def stage(self, slot: int, layer: int, expert: int, stream=None) -> int:
        g = ctypes.c_uint64()
        N.check(N.lib().msi_slot_stage(self.h, slot, layer, expert, _stream(stream), ctypes.byref(g)),
                "msi_slot_stage")
        return g.value

    def slot_table(self, layer: int):
        st = np.empty(self.E, dtype=np.int32)
        gt = np.empty(self.E, dtype=np.uint64)
        N.check(N.lib().msi_slot_table(self.h, layer, st.ctypes.data, gt.ctypes.data), "msi_slot_table")
        return st, gt

    def slot_state(self, slot: int) -> int:
        s = ctypes.c_int()
        N.check(N.lib().msi_slot_state(self.h, slot, ctypes.byref(s)), "msi_slot_state")
        return s.value

    def reset(self) -> int:
        e = ctypes.c_uint64()
        N.check(N.lib().msi_plan_reset(self.h, ctypes.byref(e)), "msi_plan_reset")
        return e.value

    def inject(self, kind: int, layer: int, expert: int):
        N.check(N.lib().msi_fault_inject(self.h, kind, layer, expert), "msi_fault_inject")

    def set_wait_cycles(self, cycles: int):
        """Limit of every bounded device wait (clock64 cycles); <= 0: default."""
        N.check(N.lib().msi_plan_set_wait_cycles(self.h, int(cycles)), "msi_plan_set_wait_cycles")

    def set_source(self, src: "Source | None", file_off=None):
        """Stage missing extents from `src` (file offsets [L*E]); None detaches."""
        if src is None:
            N.check(N.lib().msi_plan_set_source(self.h, None, None), "msi_plan_set_source")
            self._src = None
            return
        off = np.ascontiguousarray(file_off, dtype=np.uint64)
        N.check(N.lib().msi_plan_set_source(self.h, src.h, off.ctypes.data), "msi_plan_set_source")
        self._src = src  # keep the source alive while attached

    def hold(self, slot: int):
        N.check(N.lib().msi_consumer_hold(self.h, slot), "msi_consumer_hold")

    def release(self, slot: int):
        N.check(N.lib().msi_consumer_release(self.h, slot), "msi_consumer_release")

    # -- forward -------------------------------------------------------------
    def workspace(self, T: int) -> torch.Tensor:
        need = self._ws_bytes.get(T)
        if need is None:  # a pure function of the plan's shape and T
            n = ctypes.c_size_t()
            N.check(N.lib().msi_workspace_size(self.h, T, ctypes.byref(n)), "msi_workspace_size")
            need = self._ws_bytes[T] = n.value
        ws = self._ws.get("buf")
        if ws is None or ws.numel() < need:
            ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
            self._ws["buf"] = ws
        return ws

    def forward(self, layer, x, router_w, slot_table, expected, out=None, ev=None, residual=False,
                stream=None, check=True, single_cta=False, shared_gate=True, split_waves=False):
        T = x.shape[0]
        out = torch.empty_like(x) if out is None else out
        ev = RouteEvent(T, self.k, self.E) if ev is None else ev
        ws = self.workspace(T)
        st = np.ascontiguousarray(slot_table, dtype=np.int32)
        ex = np.ascontiguousarray(expected, dtype=np.uint64)
        rc = N.lib().msi_moe_forward(self.h, layer, _ptr(x), T, _ptr(router_w), st.ctypes.data,
                                     ex.ctypes.data, _ptr(out), ctypes.byref(ev.c), _ptr(ws),
                                     ws.numel(), _flags(residual, single_cta, shared_gate, split_waves),
                                     _stream(stream))
        if check:
            N.check(rc, "msi_moe_forward")
            return out, ev
        return rc, out, ev

    def forward_streamed(self, layer, x, router_w, out=None, ev=None, residual=False, stream=None,
                         stage_stream=None, check=True, single_cta=False, next_router_w=None,
                         next_ev=None, split_waves=False):
        """Streamed layer forward.  With next_router_w (layer + 1's router), the
        rows are also routed through it and layer + 1's predicted objects are
        prefetched after the last wave; the predicted route event is written to
        next_ev (allocated when None) and returned as ev.next."""
        T = x.shape[0]
        out = torch.empty_like(x) if out is None else out
        ev = RouteEvent(T, self.k, self.E) if ev is None else ev
        ws = self.workspace(T)
        if next_router_w is None:
            rc = N.lib().msi_moe_forward_streamed(self.h, layer, _ptr(x), T, _ptr(router_w), _ptr(out),
                                                  ctypes.byref(ev.c), _ptr(ws), ws.numel(),
                                                  _flags(residual, single_cta, True, split_waves),
                                                  _stream(stream), _stream(stage_stream))
            where = "msi_moe_forward_streamed"
        else:
            next_ev = RouteEvent(T, self.k, self.E) if next_ev is None else next_ev
            ev.next = next_ev
            rc = N.lib().msi_moe_forward_streamed_next(
                self.h, layer, _ptr(x), T, _ptr(router_w), _ptr(out), ctypes.byref(ev.c),
                _ptr(next_router_w), ctypes.byref(next_ev.c), _ptr(ws), ws.numel(),
                _flags(residual, single_cta, True, split_waves), _stream(stream), _stream(stage_stream))
            where = "msi_moe_forward_streamed_next"
        if check:
            N.check(rc, where)
            return out, ev
        return rc, out, ev

    def forward_streamed_stack(self, layer0, x, routers, out_a, out_b, evs, residual=False,
                               stream=None, stage_stream=None, check=True):
        """Streamed forwards of layers layer0 .. layer0 + len(routers) - 1 in
        one call (msi_moe_forward_streamed_stack): layer i reads the previous
        output (x for i = 0) and writes out_a for even i, out_b for odd i.
        evs: one RouteEvent per layer.  Returns the tensor holding the last
        layer's output."""
        n = len(routers)
        assert len(evs) == n
        T = x.shape[0]
        ws = self.workspace(T)
        rw = (ctypes.c_void_p * max(n, 1))(*[r.data_ptr() for r in routers])
        ea = (N.msi_route_event * max(n, 1))(*[e.c for e in evs])
        done = ctypes.c_int()
        rc = N.lib().msi_moe_forward_streamed_stack(
            self.h, layer0, n, _ptr(x), T, ctypes.cast(rw, ctypes.c_void_p), _ptr(out_a), _ptr(out_b),
            ctypes.cast(ea, ctypes.c_void_p), _ptr(ws), ws.numel(), _flags(residual, False),
            _stream(stream), _stream(stage_stream), ctypes.byref(done))
        last = out_a if n % 2 == 1 else out_b
        if check:
            N.check(rc, "msi_moe_forward_streamed_stack")
            return last
        return rc, done.value, last

    def workspace_host(self, T: int) -> torch.Tensor:
        n = ctypes.c_size_t()
        N.check(N.lib().msi_workspace_size_host(self.h, T, ctypes.byref(n)), "msi_workspace_size_host")
        ws = self._ws.get("host")
        if ws is None or ws.numel() < n.value:
            ws = torch.empty(max(n.value, 256), dtype=torch.uint8, device="cuda")
            self._ws["host"] = ws
        return ws

    def forward_host(self, layer, x_host, router_w, slot_table=None, expected=None, out_host=None,
                     ids_host=None, ev=None, residual=False, stream=None, stage_stream=None,
                     check=True, single_cta=False):
        """End-to-end call from and to host memory: x_host and out_host are CPU
        bf16 tensors [T, H] (pinned for the full link rate), ids_host an
        optional CPU int32 [T, k].  With a slot table the resident forward runs,
        without one the streamed forward.  The results are in out_host once the
        compute stream has passed this call."""
        T = x_host.shape[0]
        assert x_host.device.type == "cpu" and x_host.is_contiguous()
        out_host = torch.empty_like(x_host) if out_host is None else out_host
        ev = RouteEvent(T, self.k, self.E) if ev is None else ev
        ws = self.workspace_host(T)
        fl = _flags(residual, single_cta)
        if slot_table is not None:
            st = np.ascontiguousarray(slot_table, dtype=np.int32)
            ex = np.ascontiguousarray(expected, dtype=np.uint64)
            rc = N.lib().msi_moe_forward_host(self.h, layer, x_host.data_ptr(), T, _ptr(router_w),
                                              st.ctypes.data, ex.ctypes.data, out_host.data_ptr(),
                                              _ptr(ids_host), ctypes.byref(ev.c), _ptr(ws), ws.numel(),
                                              fl, _stream(stream))
            where = "msi_moe_forward_host"
        else:
            rc = N.lib().msi_moe_forward_streamed_host(self.h, layer, x_host.data_ptr(), T,
                                                       _ptr(router_w), out_host.data_ptr(),
                                                       _ptr(ids_host), ctypes.byref(ev.c), _ptr(ws),
                                                       ws.numel(), fl, _stream(stream),
                                                       _stream(stage_stream))
            where = "msi_moe_forward_streamed_host"
        if check:
            N.check(rc, where)
            return out_host, ev
        return rc, out_host, ev

    def pin(self, layer: int, expert: int, pinned: bool = True):
        N.check(N.lib().msi_plan_pin(self.h, layer, expert, int(pinned)), "msi_plan_pin")

    def status(self) -> int:
        s = ctypes.c_int()
        N.check(N.lib().msi_forward_status(self.h, ctypes.byref(s)), "msi_forward_status")
        return s.value

    # -- telemetry -------------------------------------------------------------
    def trace(self, clear: bool = False):
        """Slot trace as (call, layer, expert, slot, generation, kind, wave) tuples."""
        cap = 1 << 20
        buf = (N.msi_trace_rec * cap)()
        n = ctypes.c_size_t()
        N.check(N.lib().msi_trace_read(self.h, buf, cap, ctypes.byref(n)), "msi_trace_read")
        kinds = {N.MSI_TRACE_HIT: "hit", N.MSI_TRACE_STAGE: "stage", N.MSI_TRACE_EVICT: "evict",
                 N.MSI_TRACE_PREFETCH: "prefetch"}
        out = [(r.call, r.layer, r.expert, r.slot, int(r.generation), kinds[r.kind], r.wave)
               for r in buf[:n.value]]
        if clear:
            N.check(N.lib().msi_trace_clear(self.h), "msi_trace_clear")
        return out

    def counters(self) -> dict:
        c = N.msi_counters()
        N.check(N.lib().msi_get_counters(self.h, ctypes.byref(c)), "msi_get_counters")
        return {f: getattr(c, f) for f, _ in c._fields_}

    def timing(self, on: bool = True):
        N.check(N.lib().msi_timing_enable(self.h, int(on)), "msi_timing_enable")

    def timing_read(self, reset: bool = True) -> dict:
        """{kind: (milliseconds summed, launches)} of the timed launches."""
        ms = np.zeros(len(N.KERNEL_KINDS), dtype=np.float64)
        n = np.zeros(len(N.KERNEL_KINDS), dtype=np.uint64)
        N.check(N.lib().msi_timing_read(self.h, ms.ctypes.data, n.ctypes.data, int(reset)),
                "msi_timing_read")
        return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(N.KERNEL_KINDS)}

    def launches(self) -> int:
        return int(N.lib().msi_kernel_launches(self.h))

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            N.check(N.lib().msi_plan_destroy(self.h), "msi_plan_destroy")
            self.h = None

    def __del__(self):
        try:
            if getattr(self, "h", None) is not None and self.h.value:
                N.lib().msi_plan_destroy(self.h)
        except Exception:
            pass


class Source:
    """Bounded source service: extents read from `path` into `n_windows`
    fixed, aligned host windows (O_DIRECT covering reads when direct=True).
    The windows are pinned (page-locked) host memory when CUDA is available,
    so that the H2D copies out of them are asynchronous; otherwise aligned
    ordinary host memory (synchronous reads only)."""

    def __init__(self, path: str, window_bytes: int, n_windows: int = 8, direct: bool = True,
                 align: int = 4096):
        wb = (int(window_bytes) + align - 1) // align * align
        nbytes = wb * n_windows + align
        if torch.cuda.is_available():
            self._buf = torch.empty(nbytes, dtype=torch.uint8, pin_memory=True)
            base = self._buf.data_ptr()
        else:
            self._buf = np.empty(nbytes, dtype=np.uint8)
            base = self._buf.ctypes.data
        self._off = (-base) % align
        self.window_bytes = wb
        self.n_windows = n_windows
        self.direct = direct
        self._path = path.encode()
        d = N.msi_source_desc(self._path, 1 if direct else 0, align, n_windows,
                              base + self._off, wb)
        self.h = ctypes.c_void_p()
        N.check(N.lib().msi_source_open(ctypes.byref(d), ctypes.byref(self.h)), "msi_source_open")

    def read(self, file_off: int, nbytes: int):
        """Synchronous read: (window, bytes of the extent as a numpy copy)."""
        data = ctypes.c_void_p()
        w = ctypes.c_int()
        N.check(N.lib().msi_source_read(self.h, file_off, nbytes, ctypes.byref(data), ctypes.byref(w)),
                "msi_source_read")
        out = np.ctypeslib.as_array((ctypes.c_uint8 * nbytes).from_address(data.value)).copy()
        return w.value, out

    def release(self, window: int):
        N.check(N.lib().msi_source_release(self.h, window), "msi_source_release")

    def stats(self) -> dict:
        st = N.msi_source_stats()
        N.check(N.lib().msi_source_stats_read(self.h, ctypes.byref(st)), "msi_source_stats_read")
        return {n: getattr(st, n) for n, _ in N.msi_source_stats._fields_}

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            N.check(N.lib().msi_source_close(self.h), "msi_source_close")
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _elsewhere(stream, call, *args, **kwargs):
    """The call on `stream`: its tensors stay allocated until that stream has
    used them, and what it makes until the caller's stream has."""
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        made = call(*args, **kwargs)
    for t in (*args, *kwargs.values()):
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(stream)
    for t in made if isinstance(made, tuple) else (made,):
        t.record_stream(here)
    return made


_current_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream  # of a device: the current one, without an object made for it


# The calls below are short beside Python: their checks read each attribute once.

def _head_rows(t, name, dim, dev, heads=None):
    """Elements between the rows of bf16 [n, heads, dim] on device dev, heads packed."""
    shape = t.shape
    if (t.dtype is torch.bfloat16 and len(shape) == 3 and shape[2] == dim and shape[1] >= 1 and t.get_device() == dev
            and (heads is None or shape[1] == heads)):
        row, head, one = t.stride()
        if (one == 1 or dim == 1) and (head == dim or shape[1] == 1):
            return row if shape[0] > 1 else shape[1] * dim
        if shape[0] == 0:
            return shape[1] * dim
    raise ValueError("%s: bf16 rows [n, %s, %d], each contiguous, on the current CUDA device are needed"
                     % (name, "heads" if heads is None else heads, dim))


def _rows_of(t, name, rows, columns, dtypes, dev):
    """Elements between the rows of [rows, columns] on device dev (rows None: any number)."""
    shape = t.shape
    if t.dtype in dtypes and len(shape) == 2 and shape[1] == columns and t.get_device() == dev and (rows is None or shape[0] == rows):
        row, one = t.stride()
        if one == 1 or columns == 1 or shape[0] == 0:
            return row if shape[0] > 1 else columns
    raise ValueError("%s: rows [%s, %d] of %s, each contiguous, on the current CUDA device are needed"
                     % (name, "n" if rows is None else rows, columns, " or ".join(str(d)[6:] for d in dtypes)))


_BF16 = (torch.bfloat16,)
_EITHER = (torch.bfloat16, torch.float32)
_TYPES = {torch.bfloat16: N.MSI_BF16, torch.float32: N.MSI_F32}
_pack_linear, _pack_rotary, _pack_sample = N.pack_q4_linear_args, N.pack_rotary_args, N.pack_sample_args


class Q4Linear:
    """A matrix in 4 bits, for products with a few rows (see include/msi.h,
    msi_q4_linear): codes uint8 [n_out, n_in / 2], even column in the low nibble,
    scales fp16 [n_out, n_in / group]; code q stands for scale * (q - 8).

    The weights are laid out once for the kernel, on the current stream; codes
    and scales are not kept.  A call waits for nothing and may be captured."""

    def __init__(self, codes, scales):
        if codes.dtype is not torch.uint8 or scales.dtype is not torch.float16 or codes.dim() != 2 or scales.dim() != 2:
            raise ValueError("codes: uint8 [n_out, n_in / 2], scales: fp16 [n_out, groups] are needed")
        self.n_out, self.n_in = codes.shape[0], 2 * codes.shape[1]
        groups = scales.shape[1]
        if scales.shape[0] != self.n_out or groups == 0 or self.n_in % groups != 0:
            raise ValueError("scales: [n_out, n_in / group] is needed")
        self.group = self.n_in // groups
        dev = _current_device()
        if codes.get_device() != dev or scales.get_device() != dev:
            raise ValueError("codes, scales: tensors on the current CUDA device are needed")
        codes, scales = codes.contiguous(), scales.contiguous()
        if codes.data_ptr() % 4:  # a part of something else
            codes = codes.clone()
        lib = N.lib()
        nbytes = lib.msi_q4_packed_bytes(self.n_out, self.n_in, self.group)
        if nbytes == 0:
            raise ValueError("n_out %d, n_in %d, group %d: not a shape that msi_q4_linear takes" % (self.n_out, self.n_in, self.group))
        self.packed = torch.empty(nbytes, dtype=torch.uint8, device=codes.device)
        on = _raw_stream(dev)
        N.check(lib.msi_q4_pack(codes.data_ptr(), scales.data_ptr(), self.n_out, self.n_in, self.group,
                                self.packed.data_ptr(), nbytes, on), "msi_q4_pack")
        self._used_on = {on}
        self._device = dev
        self._linear = lib.msi_q4_linear
        self._ptr = self.packed.data_ptr()

    def __call__(self, x, out=None, add=None, dtype=torch.bfloat16, stream=None):
        """x W^T (+ add) for bf16 rows x [n, n_in], as `dtype` (bf16 or fp32).
        add: bf16 [n, n_out], added before the rounding; may be `out`."""
        if stream is not None:
            return _elsewhere(stream, self, x, out=out, add=add, dtype=dtype)
        dev = _current_device()
        n_in, n_out = self.n_in, self.n_out
        x_stride = _rows_of(x, "x", None, n_in, _BF16, dev)
        rows = x.shape[0]
        if dev != self._device:
            raise ValueError("the weights are on another device than the current one")
        add_ptr = add_stride = 0
        if add is not None:
            add_stride = _rows_of(add, "add", rows, n_out, _BF16, dev)
            add_ptr = add.data_ptr()
        x_ptr, on = x.data_ptr(), _raw_stream(dev)
        if out is None:
            if dtype not in _EITHER:
                raise ValueError("dtype: torch.bfloat16 or torch.float32 is needed")
            out = torch.empty((rows, n_out), dtype=dtype, device="cuda")  # new_empty is the longer call
            out_stride = n_out
        else:
            out_stride = _rows_of(out, "out", rows, n_out, _EITHER, dev)
            dtype = out.dtype
        if rows == 0:
            return out
        if on not in self._used_on:
            self._used_on.add(on)
            self.packed.record_stream(torch.cuda.current_stream())
        rc = self._linear(_pack_linear(self._ptr, n_out, n_in, self.group, rows, _TYPES[dtype], x_ptr, x_stride, add_ptr,
                                       add_stride, out.data_ptr(), out_stride), on)
        if rc:
            N.check(rc, "msi_q4_linear")
        return out

    @staticmethod
    def set_wait_cycles(cycles: int):
        """Limit of the products' device waits (msi_q4_set_wait_cycles); 0: the default."""
        N.check(N.lib().msi_q4_set_wait_cycles(int(cycles)), "msi_q4_set_wait_cycles")

    @staticmethod
    def inject_stall(where: int):
        """The next product waits in vain (msi_q4_inject_stall)."""
        N.check(N.lib().msi_q4_inject_stall(int(where)), "msi_q4_inject_stall")


class Rotary:
    """Rotation of heads by position (see include/msi.h, msi_rotary_desc).  Pair j
    of the first `dims` columns (None: all) turns by freqs[j] radians (None:
    base ** (-2 j / dims)) for each position along axis axes[j] (None: one axis
    for all); pairs are (j, j + dims / 2), or neighbours where interleaved."""

    def __init__(self, head_dim, dims=None, base=10000.0, freqs=None, axes=None, interleaved=False):
        dims = head_dim if dims is None else dims
        if dims < 2 or dims % 2:
            raise ValueError("dims: an even number is needed")
        f = base ** (-2.0 * np.arange(dims // 2) / dims) if freqs is None else np.ascontiguousarray(freqs, dtype=np.float64)
        ax = np.zeros(dims // 2, np.int32) if axes is None else np.ascontiguousarray(axes, dtype=np.int32)
        if f.shape != (dims // 2,) or ax.shape != (dims // 2,):
            raise ValueError("freqs, axes: one for each of the %d pairs are needed" % (dims // 2))
        self.head_dim, self.dims, self.interleaved = head_dim, dims, bool(interleaved)
        self.n_axes = int(ax.max()) + 1
        d = N.msi_rotary_desc(head_dim, dims, self.n_axes, int(self.interleaved), f.ctypes.data, ax.ctypes.data)
        h = ctypes.c_void_p()
        lib = N.lib()
        N.check(lib.msi_rotary_create(ctypes.byref(d), ctypes.byref(h)), "msi_rotary_create")
        self._apply = lib.msi_rotary_apply
        self.h = h.value

    def _positions(self, positions, rows, dev):
        """(pointer, elements between axes)."""
        shape = positions.shape
        if positions.dtype is torch.int32 and positions.get_device() == dev:
            if len(shape) == 1 and self.n_axes == 1 and shape[0] == rows and (rows < 2 or positions.stride(0) == 1):
                return positions.data_ptr(), rows
            if len(shape) == 2 and shape[0] == self.n_axes and shape[1] == rows and (rows < 2 or positions.stride(1) == 1):
                return positions.data_ptr(), positions.stride(0)
        raise ValueError("positions: int32 [%d, %d], each axis contiguous, on the current CUDA device is needed" % (self.n_axes, rows))

    def __call__(self, x, positions, out=None, stream=None):
        """Rows x [n, heads, head_dim] (bf16) rotated by positions [n] or
        [n_axes, n] (int32).  out: may be x; None: a new packed tensor."""
        if stream is not None:
            return _elsewhere(stream, self, x, positions, out=out)
        dev, dim = _current_device(), self.head_dim
        stride = _head_rows(x, "x", dim, dev)
        rows, heads = x.shape[0], x.shape[1]
        pos, pos_stride = self._positions(positions, rows, dev)
        x_ptr, on = x.data_ptr(), _raw_stream(dev)
        if out is None:
            out = torch.empty((rows, heads, dim), dtype=torch.bfloat16, device="cuda")
            out_stride = heads * dim
        else:
            out_stride = _head_rows(out, "out", dim, dev, heads)
            if out.shape[0] != rows:
                raise ValueError("out: the shape of x is needed")
        if rows == 0:
            return out
        rc = self._apply(self.h, _pack_rotary(rows, heads, x_ptr, stride, pos, pos_stride, out.data_ptr(), out_stride), on)
        if rc:
            N.check(rc, "msi_rotary_apply")
        return out

    def close(self):
        if getattr(self, "h", 0):
            N.check(N.lib().msi_rotary_destroy(self.h), "msi_rotary_destroy")
            self.h = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, stream=None):
    """A token for each row of logits [n, vocab] (fp32 or bf16) by the random
    numbers u [n] (fp32 in [0, 1)); see include/msi.h, msi_sample_args.
    temperature (0: the greatest logit), top_k (0: all), top_p (1: all) and min_p
    (0: all) are numbers, or CUDA vectors [n] (fp32; top_k int32) with a value for
    each row.  Returns (ids int32 [n], log-probabilities fp32 [n] among the tokens
    kept); a row that holds no number or has a parameter out of range gets -1."""
    if stream is not None:
        return _elsewhere(stream, sample, logits, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    dev = _current_device()
    shape = logits.shape
    if len(shape) != 2 or shape[1] < 1:
        raise ValueError("logits: rows [n, vocab] are needed")
    rows, vocab = shape
    stride = _rows_of(logits, "logits", None, vocab, _EITHER, dev)
    temperatures = top_ks = top_ps = min_ps = 0
    if type(temperature) is not float and isinstance(temperature, torch.Tensor):
        temperatures, temperature = _vector(temperature, "temperature", torch.float32, rows, dev), 0.0
    if type(top_k) is not int and isinstance(top_k, torch.Tensor):
        top_ks, top_k = _vector(top_k, "top_k", torch.int32, rows, dev), 0
    elif top_k >= vocab:
        top_k = 0
    if type(top_p) is not float and isinstance(top_p, torch.Tensor):
        top_ps, top_p = _vector(top_p, "top_p", torch.float32, rows, dev), 0.0
    if type(min_p) is not float and isinstance(min_p, torch.Tensor):
        min_ps, min_p = _vector(min_p, "min_p", torch.float32, rows, dev), 0.0
    us = _vector(u, "u", torch.float32, rows, dev)
    ids = torch.empty((rows,), dtype=torch.int32, device="cuda")
    logprobs = torch.empty_like(u)
    if rows == 0:
        return ids, logprobs
    rc = N.lib().msi_sample(_pack_sample(rows, vocab, _TYPES[logits.dtype], logits.data_ptr(), stride, us, temperature, top_k, top_p,
                                         min_p, temperatures, top_ks, top_ps, min_ps, ids.data_ptr(), logprobs.data_ptr()),
                            _raw_stream(dev))
    if rc:
        N.check(rc, "msi_sample")
    return ids, logprobs


def _vector(t, name, dtype, n, dev):
    if t.dtype is dtype and t.get_device() == dev and t.dim() == 1 and t.shape[0] == n and (n < 2 or t.stride(0) == 1):
        return t.data_ptr()
    raise ValueError("%s: a contiguous %s vector of %d on the current CUDA device is needed" % (name, str(dtype)[6:], n))


class KvCache:
    """One layer's key-value cache in 8 bits (see include/msi.h, msi_kv_desc):
    paged blocks with a scale for each block and head, append, attention over
    them, eviction by the attention weight received.

    ``buffers`` gives tensors to use in place of new ones (by the names of
    ``BUFFERS``, shapes as in msi_kv_desc; a cache that a program restores or
    shares): if it is given, it has to name all of them, and the cache is not
    emptied.  Every index argument is an int32 CUDA tensor; ``seqs`` None means
    sequences 0, 1, ...  Nothing here waits for the GPU but ``status``.

    A step captured in a graph may be replayed between other calls, larger ones
    too, as long as the cache lives: a workspace that a graph knows is kept.

    A call with `stream` runs there (None: the current stream); calls on one
    cache have to follow one another on the GPU, which is the caller's to see to."""

    BUFFERS = ("k_codes", "v_codes", "k_scale", "v_scale", "recent", "table", "seq_state", "free_ids", "control",
               "weight")

    def __init__(self, *, n_seqs, max_blocks, n_blocks, n_kv_heads, head_dim, block_tokens=32, fmt=N.MSI_KV_Q8,
                 buffers=None, stream=None):
        lib = N.lib()
        dev = _current_device()  # the handle's
        K, P, D = n_kv_heads, block_tokens, head_dim
        self.n_seqs, self.K, self.P, self.D, self.fmt = n_seqs, K, P, D, fmt
        shapes = {"k_codes": ((n_blocks, K, P, D), torch.uint8), "v_codes": ((n_blocks, K, P, D), torch.uint8),
                  "k_scale": ((n_blocks, K), torch.float32), "v_scale": ((n_blocks, K), torch.float32),
                  "recent": ((n_seqs, 2, K, 2 * P, D), torch.bfloat16), "table": ((n_seqs, max_blocks), torch.int32),
                  "seq_state": ((n_seqs, 4), torch.int32), "free_ids": ((n_blocks,), torch.int32),
                  "control": ((8,), torch.int32), "weight": ((n_blocks,), torch.float32)}
        with torch.cuda.stream(stream):  # None: the current one
            for name, (shape, dtype) in shapes.items():
                if buffers is None:
                    t = torch.empty(shape, dtype=dtype, device="cuda")
                else:
                    t = buffers[name]
                    if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous() or t.get_device() != dev:
                        raise ValueError("%s: a contiguous tensor %s of %s on the current CUDA device is needed" % (name, shape, dtype))
                setattr(self, name, t)
        d = N.msi_kv_desc(n_seqs, max_blocks, n_blocks, K, D, P, fmt, *[getattr(self, n).data_ptr() for n in self.BUFFERS])
        h = ctypes.c_void_p()
        N.check(lib.msi_kv_create(ctypes.byref(d), ctypes.byref(h)), "msi_kv_create")
        self.h = h
        self._lib = lib
        self._device = self.table.device
        self._device_index = self._device.index
        self._ws, self._ws_on = None, set()  # workspace, and the streams that it was used on
        self._ws_captured = False            # whether a graph holds its address
        self._ws_kept = []                   # workspaces that were replaced after that: the graphs write to them
        self._need = {}
        self._used_on = set()                # the streams that the buffers were used on
        if buffers is None:
            self.init(stream)

    # A decode step's calls are short: the checks read each attribute once.

    def _index(self, t, name, n=None):
        if t is None:
            return None
        shape = t.shape
        if (t.dtype is not torch.int32 or t.get_device() != self._device_index or len(shape) != 1 or (n is not None and shape[0] != n)
                or not t.is_contiguous()):
            raise ValueError("%s: a contiguous int32 vector%s on the cache's device is needed" % (name, "" if n is None else " of %d" % n))
        return t.data_ptr()

    def _rows(self, t, name, heads):
        """(pointer, elements between rows, rows) of bf16 rows [n, heads, D]."""
        shape, D = t.shape, self.D
        ok = t.dtype is torch.bfloat16 and t.get_device() == self._device_index and len(shape) == 3 and shape[1] == heads and shape[2] == D
        if ok:
            n = shape[0]
            if n == 0:
                return None, heads * D, 0
            row, head, one = t.stride()
            if one == 1 and (head == D or heads == 1):
                return t.data_ptr(), row if n > 1 else heads * D, n
        raise ValueError("%s: bf16 rows [n, %d, %d], each contiguous, on the cache's device are needed" % (name, heads, D))

    # Every call runs on the current stream: one with another stream makes that
    # the current one (_elsewhere).  What the allocator gives a call then belongs
    # to the stream that the call's kernels run on.

    def _here(self):
        """The current stream, on which the cache's buffers are about to be used."""
        on = torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())  # no object is made for it
        if on not in self._used_on:
            self._used_on.add(on)
            stream = torch.cuda.current_stream()
            for name in self.BUFFERS:
                getattr(self, name).record_stream(stream)
        return on

    @staticmethod
    def _elsewhere(stream, call, *args):
        """The call on `stream`: its arguments stay allocated until that stream
        has used them, and what it makes until the caller's stream has."""
        here = torch.cuda.current_stream()
        with torch.cuda.stream(stream):
            made = call(*args)
        for t in args:
            if isinstance(t, torch.Tensor):
                t.record_stream(stream)
        for t in (made,) if isinstance(made, torch.Tensor) else made or ():
            t.record_stream(here)
        return made

    def init(self, stream=None):
        """Empty the cache: every block free, no tokens, status 0."""
        if stream is not None:
            return self._elsewhere(stream, self.init)
        N.check(N.lib().msi_kv_init(self.h, self._here()), "msi_kv_init")

    def append(self, k, v, cu, seqs=None, start=None, stream=None, rotary=None, positions=None, q=None, q_out=None):
        """Rows cu[b] .. cu[b+1] of k and v [n, kv_heads, head_dim] (rows may be
        strided alike) become the tokens of sequence seqs[b] from start[b] on
        (None: at its end); tokens held from there on are dropped first.

        rotary (a Rotary of the cache's head_dim): the keys are rotated on the
        way, by positions ([n], or [axes, n], int32; None: each token's own in its
        sequence), and with them the queries q [n, heads, head_dim] of the same
        rows, which are returned rotated (q_out: may be q; None: a new tensor); rows of
        q behind the last sequence's are not written."""
        if stream is not None:
            return self._elsewhere(stream, self.append, k, v, cu, seqs, start, None, rotary, positions, q, q_out)
        n = cu.numel() - 1
        kp, stride, rows = self._rows(k, "k", self.K)
        vp, v_stride, v_rows = self._rows(v, "v", self.K)
        if v_rows != rows or v_stride != stride:
            raise ValueError("k and v: as many rows, with the same stride, are needed")
        ids, cup, startp, on = self._index(seqs, "seqs", n), self._index(cu, "cu"), self._index(start, "start", n), self._here()
        if rotary is None:
            if positions is not None or q is not None or q_out is not None:
                raise ValueError("positions, q and q_out go with rotary")
            rc = self._lib.msi_kv_append(self.h, n, ids, cup, startp, kp, vp, stride, rows, on)
            if rc:
                N.check(rc, "msi_kv_append")
            return None
        pp, pos_stride = (0, 0) if positions is None else rotary._positions(positions, rows, self._device_index)
        qp = op = 0
        heads = q_stride = out_stride = 0
        if q is not None:
            heads = q.shape[1] if q.dim() == 3 else 0
            qp, q_stride, q_rows = self._rows(q, "q", heads)
            if q_out is None:
                q_out = torch.empty((rows, heads, self.D), dtype=torch.bfloat16, device=self._device)
                op, out_stride, out_rows = q_out.data_ptr(), heads * self.D, rows
            else:
                op, out_stride, out_rows = self._rows(q_out, "q_out", heads)
            if q_rows != rows or out_rows != rows:
                raise ValueError("q and q_out: as many rows as k are needed")
        elif q_out is not None:
            raise ValueError("q_out goes with q")
        a = N.pack_kv_rotary_args(rotary.h, pp, pos_stride, heads, qp or 0, q_stride, op or 0, out_stride)
        rc = self._lib.msi_kv_append_rotary(self.h, n, ids, cup, startp, kp, vp, stride, rows, a, on)
        if rc:
            N.check(rc, "msi_kv_append_rotary")
        return q_out

    def attention(self, q, cu, max_rows, seqs=None, out=None, lse=None, scale=None, softcap=0.0, window=0,
                  observe=False, stream=None):
        """Attention of rows cu[b] .. cu[b+1] of q [n, heads, head_dim], the last
        tokens of sequence seqs[b], over what it holds.  max_rows: at least the
        rows of any one sequence, at most those of q.  scale None: head_dim ** -0.5.
        observe: add up each block's attention weight (decode form; no sequence
        twice).  Returns (out, lse)."""
        if stream is not None:
            return self._elsewhere(stream, self.attention, q, cu, max_rows, seqs, out, lse, scale, softcap, window, observe)
        n, heads = cu.numel() - 1, q.shape[1]
        qp, q_stride, rows = self._rows(q, "q", heads)
        if out is None:
            # packed either way: empty_like, the shorter call, keeps the order of q's strides, which rows that overlap upset
            out = torch.empty_like(q) if q_stride >= heads * self.D else q.new_empty(q.shape)
            op, out_stride = out.data_ptr() if rows else None, heads * self.D
        else:
            op, out_stride, out_rows = self._rows(out, "out", heads)
            if out_rows != rows:
                raise ValueError("out: the shape of q is needed")
        if lse is None:
            lse = torch.empty((rows, heads), dtype=torch.float32, device=self._device)
        elif tuple(lse.shape) != (rows, heads) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.get_device() != self._device_index:
            raise ValueError("lse: a contiguous fp32 tensor [n, heads] on the cache's device is needed")
        a = N.msi_kv_attention_args(n, self._index(seqs, "seqs", n), self._index(cu, "cu"), rows, max_rows, heads, qp,
                                    q_stride, op, out_stride, lse.data_ptr() if rows else None,
                                    self.D ** -0.5 if scale is None else scale, softcap, window,
                                    N.MSI_KV_OBSERVE if observe else 0)
        key = (n, rows, max_rows, heads, observe)
        need = self._need.get(key)
        if need is None:  # a pure function of the cache's and the call's shape
            b = ctypes.c_size_t()
            N.check(N.lib().msi_kv_workspace_size(self.h, ctypes.byref(a), ctypes.byref(b), None), "msi_kv_workspace_size")
            if len(self._need) >= 256:  # prompts come in any length
                self._need.clear()
            need = self._need[key] = b.value
        on = self._here()
        ws = self._ws
        if ws is None or ws.numel() < need:
            if self._ws_captured:
                self._ws_kept.append(ws)
                self._ws_captured = False
            ws = self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
            self._ws_on = {on}
        elif on not in self._ws_on:
            self._ws_on.add(on)
            ws.record_stream(torch.cuda.current_stream())
        if not self._ws_captured:
            self._ws_captured = torch._C._cuda_isCurrentStreamCapturing()
        rc = self._lib.msi_kv_attention(self.h, ctypes.byref(a), ws.data_ptr(), ws.numel(), on)
        if rc:
            N.check(rc, "msi_kv_attention")
        return out, lse

    def _which(self, seqs):
        return (seqs, None) if isinstance(seqs, int) else (seqs.numel(), self._index(seqs, "seqs"))

    def evict(self, seqs, keep, sinks=0, recent=1, stream=None):
        """Sequences that hold more than `keep` blocks keep their first `sinks`,
        their last `recent` and the heaviest others.  seqs: a tensor, or the
        number of sequences 0, 1, ..."""
        if stream is not None:
            return self._elsewhere(stream, self.evict, seqs, keep, sinks, recent)
        n, ids = self._which(seqs)
        rc = self._lib.msi_kv_evict(self.h, n, ids, keep, sinks, recent, self._here())
        if rc:
            N.check(rc, "msi_kv_evict")

    def release(self, seqs, stream=None):
        """End sequences (a tensor, or the number of sequences 0, 1, ...)."""
        if stream is not None:
            return self._elsewhere(stream, self.release, seqs)
        n, ids = self._which(seqs)
        N.check(self._lib.msi_kv_release(self.h, n, ids, self._here()), "msi_kv_release")

    def read(self, cu, rows, seqs=None, first=None, stream=None):
        """The tokens from first[b] on (None: 0) of sequence seqs[b] as bf16 rows
        cu[b] .. cu[b+1] of (k, v) [rows, kv_heads, head_dim]; rows = cu[-1]."""
        if stream is not None:
            return self._elsewhere(stream, self.read, cu, rows, seqs, first)
        n = cu.numel() - 1
        ids, firstp, cup, on = self._index(seqs, "seqs", n), self._index(first, "first", n), self._index(cu, "cu"), self._here()
        k = torch.empty((rows, self.K, self.D), dtype=torch.bfloat16, device=self._device)
        v = torch.empty_like(k)
        rc = self._lib.msi_kv_read(self.h, n, ids, firstp, cup, rows, k.data_ptr() if rows else None, v.data_ptr() if rows else None, on)
        if rc:
            N.check(rc, "msi_kv_read")
        return k, v

    def status(self, stream=None) -> int:
        """Wait for the stream; the cache's status word (MSI_OK: 0), which is cleared."""
        s = ctypes.c_int()
        N.check(N.lib().msi_kv_status(self.h, _stream(stream), ctypes.byref(s)), "msi_kv_status")
        return s.value

    def set_wait_cycles(self, cycles: int):
        """Limit of the chunk form's device waits (msi_kv_set_wait_cycles); 0: the default."""
        N.check(N.lib().msi_kv_set_wait_cycles(self.h, int(cycles)), "msi_kv_set_wait_cycles")

    def inject_stall(self, where: int):
        """A warp of the next chunk call waits in vain (msi_kv_inject_stall)."""
        N.check(N.lib().msi_kv_inject_stall(self.h, int(where)), "msi_kv_inject_stall")

    def launches(self) -> int:
        return int(N.lib().msi_kv_kernel_launches(self.h))

    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            N.check(N.lib().msi_kv_destroy(self.h), "msi_kv_destroy")
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
