"""Thin ctypes binding of libturbosparse.so (include/turbosparse.h).

Argument marshalling only: torch tensors supply device memory and the
stream; every step of the FFN runs in the library's HIP kernels.  There is no
fallback: if the library is missing this module raises on import.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libturbosparse.so")

TS_F32 = 0
TS_BF16 = 1

STATUS = {0: "TS_OK", 1: "TS_ERR_NULL", 2: "TS_ERR_SHAPE", 3: "TS_ERR_DTYPE", 4: "TS_ERR_ALIGN",
          5: "TS_ERR_WORKSPACE", 6: "TS_ERR_HIP", 7: "TS_ERR_UNSUPPORTED"}

EXPORTED = ["ts_ffn_workspace_bytes", "ts_ffn_sparse", "ts_ffn_sparse_act", "ts_ffn_sparse_topk", "ts_ffn_dense",
            "ts_ffn_given_workspace_bytes", "ts_ffn_sparse_noalloc",
            "ts_ffn_sparse_given", "ts_moe_workspace_bytes", "ts_moe_sparse",
            "ts_moe_dense", "ts_status_str", "ts_last_error", "ts_version", "ts_prof_enable", "ts_prof_reset",
            "ts_prof_read", "ts_probe_read", "ts_probe_copy", "ts_tune_set",
            "ts_moe_route_workspace_bytes", "ts_moe_route", "ts_moe_group", "ts_moe_route_grad",
            "ts_moe_balance_workspace_bytes", "ts_moe_balance", "ts_moe_balance_grad", "ts_grouped_mm",
            "ts_grouped_drelu", "ts_drelu_grad",
            "ts_grouped_drelu_pack", "ts_grouped_drelu_grad", "ts_drelu_unpack", "ts_grouped_mm_dw", "ts_fp8_quant", "ts_fp8_quant_weights",
            "ts_fp8_mm", "ts_fp8_drelu", "ts_adapter_workspace_bytes", "ts_adapter_mm", "ts_adapter_drelu", "ts_moe_combine", "ts_moe_combine_grad"]


class TSError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        super().__init__(f"{where}: {STATUS.get(code, code)}" + (f" ({detail})" if detail else ""))


class ffn_stats_t(ctypes.Structure):
    _fields_ = [("n_gate", ctypes.c_void_p), ("n_active", ctypes.c_void_p), ("gate_idx", ctypes.c_void_p),
                ("active_idx", ctypes.c_void_p), ("n_union", ctypes.c_void_p)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2406_05955_amd.build` "
                          "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    st = ctypes.c_int
    lib.ts_ffn_workspace_bytes.argtypes = [i, i, i, i]
    lib.ts_ffn_workspace_bytes.restype = sz
    lib.ts_ffn_sparse.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, vp, vp, sz, vp]
    lib.ts_ffn_sparse.restype = st
    lib.ts_ffn_sparse_noalloc.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, vp, vp]
    lib.ts_ffn_sparse_noalloc.restype = st
    lib.ts_ffn_dense.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, vp, sz, vp]
    lib.ts_ffn_dense.restype = st
    lib.ts_ffn_sparse_act.argtypes = [vp, vp, vp, vp, i, i, i, i, i, ctypes.c_float, vp, vp, vp, sz, vp]
    lib.ts_ffn_sparse_act.restype = st
    lib.ts_ffn_sparse_topk.argtypes = [vp, vp, vp, vp, i, i, i, i, i, vp, vp, vp, sz, vp]
    lib.ts_ffn_sparse_topk.restype = st
    lib.ts_ffn_given_workspace_bytes.argtypes = [i, i, i, i, i]
    lib.ts_ffn_given_workspace_bytes.restype = sz
    lib.ts_ffn_sparse_given.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, vp, i, vp, vp, vp, sz, vp]
    lib.ts_ffn_sparse_given.restype = st
    lib.ts_moe_workspace_bytes.argtypes = [i, i, i, i, i, i]
    lib.ts_moe_workspace_bytes.restype = sz
    lib.ts_moe_sparse.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, sz, vp]
    lib.ts_moe_sparse.restype = st
    lib.ts_moe_dense.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, sz, vp]
    lib.ts_moe_dense.restype = st
    lib.ts_moe_route_workspace_bytes.argtypes = [i, i, i]
    lib.ts_moe_route_workspace_bytes.restype = sz
    lib.ts_moe_balance_workspace_bytes.argtypes = [i, i, i]
    lib.ts_moe_balance_workspace_bytes.restype = sz
    lib.ts_adapter_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    lib.ts_adapter_workspace_bytes.restype = sz
    for name, args in (
            ("ts_adapter_mm", [vp, vp, vp, vp, vp, i, i, vp, vp, i, i, i, i, i, i, vp, i, vp, sz, vp]),
            ("ts_adapter_drelu", [vp, vp, vp, vp, vp, vp, vp, vp, i, vp, vp, i, i, i, i, i, i, vp, i, vp, sz, vp]),
            ("ts_moe_balance", [vp, vp, vp, i, i, i, vp, vp, vp, sz, vp]),
            ("ts_moe_balance_grad", [vp, vp, vp, vp, vp, i, i, i, vp, vp]),
            ("ts_moe_route", [vp, i, i, i, vp, vp, vp, vp, vp, vp, sz, vp]),
            ("ts_moe_group", [vp, i, i, i, vp, vp, vp, vp, sz, vp]),
            ("ts_moe_route_grad", [vp, vp, vp, i, i, i, vp, vp]),
            ("ts_grouped_mm", [vp, vp, vp, vp, i, i, vp, vp, i, i, i, i, i, vp, i, vp]),
            ("ts_grouped_drelu", [vp, vp, vp, i, vp, vp, i, i, i, i, i, vp, vp, vp, i, vp]),
            ("ts_drelu_grad", [vp, vp, vp, i, i, i, vp, vp, vp]),
            ("ts_grouped_drelu_pack", [vp, vp, vp, i, vp, vp, i, i, i, i, i, vp, vp, vp, i, vp]),
            ("ts_grouped_drelu_grad", [vp, vp, i, vp, vp, i, i, i, i, i, vp, vp, vp, vp, vp, i, vp]),
            ("ts_drelu_unpack", [vp, vp, i, i, vp, vp, vp]),
            ("ts_grouped_mm_dw", [vp, vp, i, vp, vp, i, i, i, i, i, vp, i, vp]),
            ("ts_fp8_quant", [vp, i, i, i, vp, vp, vp]),
            ("ts_fp8_quant_weights", [vp, i, i, i, i, i, vp, vp, vp]),
            ("ts_fp8_mm", [vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp, i, vp]),
            ("ts_fp8_drelu", [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp, i, vp]),
            ("ts_moe_combine", [vp, i, vp, vp, i, i, i, i, vp, i, vp]),
            ("ts_moe_combine_grad", [vp, i, vp, i, vp, vp, i, i, i, i, vp, vp, vp])):
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = st
    lib.ts_status_str.argtypes = [st]
    lib.ts_status_str.restype = ctypes.c_char_p
    lib.ts_last_error.argtypes = []
    lib.ts_last_error.restype = ctypes.c_char_p
    lib.ts_version.argtypes = []
    lib.ts_version.restype = ctypes.c_char_p
    lib.ts_prof_enable.argtypes = [i]
    lib.ts_prof_enable.restype = None
    lib.ts_prof_reset.argtypes = []
    lib.ts_prof_reset.restype = None
    lib.ts_prof_read.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_long), ctypes.POINTER(ctypes.c_double)]
    lib.ts_prof_read.restype = st
    lib.ts_probe_read.argtypes = [vp, sz, vp, vp]
    lib.ts_probe_read.restype = st
    lib.ts_probe_copy.argtypes = [vp, vp, sz, vp]
    lib.ts_probe_copy.restype = st
    lib.ts_tune_set.argtypes = [ctypes.c_char_p, i]
    lib.ts_tune_set.restype = st
    return lib


lib = _load()


def _check(code: int, where: str):
    if code != 0:
        # the HIP message; the allocation-free entry point also explains a
        # shape beyond its scratch array there
        own = where == "ts_ffn_sparse_noalloc" and code in (5, 7)
        detail = lib.ts_last_error().decode() if code == 6 or own else ""
        raise TSError(code, where, detail)


# A small call's time is the host's: per call at the 512 x 1792 layer, tensor
# checks 2.2 us, the stream object 2.9, pointer objects 1.0, a workspace size
# that the caller's own workspace makes needless 0.5, of 14.0 (the library's
# call with its two launches 6.5); now 10.8 (checks 1.6, stream 0.2).  So pointers are passed as plain integers (the argument
# types convert them), the current stream is asked for as a handle where this
# torch offers it, and well-formed tensors pass one combined test.
def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _cur_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_cur_device())


def wdtype_of(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return TS_F32
    if t.dtype == torch.bfloat16:
        return TS_BF16
    raise TypeError(f"weights must be float32 or bfloat16, got {t.dtype}")


def _need_cuda(*ts):
    dev = None
    for t in ts:
        if t is None:
            continue
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous device tensors")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError(f"tensors on different devices ({dev}, {t.device})")


def _on(t, d):
    return t.is_cuda and t.get_device() == d and t.is_contiguous()


_f32, _bf16 = torch.float32, torch.bfloat16


def _check_tensors(x, w_gate, w_up, w_down_t, out, w_router=None):
    """Raises unless the tensors are what _explain_tensors describes."""
    xs, ws, dt, d = x.shape, w_gate.shape, w_gate.dtype, x.get_device()
    if (x.dtype is _f32 and len(xs) == 2 and (dt is _bf16 or dt is _f32)
            and len(ws) == (2 if w_router is None else 3) and ws[-1] == xs[1]
            and w_up.dtype is dt and w_up.shape == ws and w_down_t.dtype is dt and w_down_t.shape == ws
            and (out is None or (out.dtype is _f32 and out.shape == xs and _on(out, d)))
            and _on(x, d) and _on(w_gate, d) and _on(w_up, d) and _on(w_down_t, d)
            and (w_router is None or (w_router.dtype is dt and w_router.shape == (ws[0], xs[1]) and _on(w_router, d)))):
        return
    _explain_tensors(x, w_gate, w_up, w_down_t, out, w_router)


def _explain_tensors(x, w_gate, w_up, w_down_t, out, w_router=None):
    """What the C ABI cannot check (it sees only pointers and the sizes passed
    with them): x float32 [B][H]; W_gate, W_up, W_down_t one dtype and one
    shape, [I][H] or, for the MoE layer, [E][I][H] with the router [E][H] of
    the same dtype; out float32 [B][H]; all contiguous on one device.  A
    mismatch here would let the kernels read or write past a buffer."""
    if x.dtype != torch.float32 or x.dim() != 2:
        raise TypeError(f"x must be a float32 [batch][hidden] tensor, got {x.dtype} {tuple(x.shape)}")
    B, H = x.shape
    moe = w_router is not None
    wdtype_of(w_gate)
    if w_gate.dim() != (3 if moe else 2) or w_gate.shape[-1] != H:
        raise ValueError(f"w_gate must be [{'experts][' if moe else ''}inter][{H}], got {tuple(w_gate.shape)}")
    for name, w in (("w_up", w_up), ("w_down_t", w_down_t)):
        if w.dtype != w_gate.dtype or w.shape != w_gate.shape:
            raise ValueError(f"{name} must match w_gate ({w_gate.dtype} {tuple(w_gate.shape)}), "
                             f"got {w.dtype} {tuple(w.shape)}")
    if moe and (w_router.dtype != w_gate.dtype or tuple(w_router.shape) != (w_gate.shape[0], H)):
        raise ValueError(f"w_router must be {w_gate.dtype} [{w_gate.shape[0]}][{H}], "
                         f"got {w_router.dtype} {tuple(w_router.shape)}")
    if out is not None and (out.dtype != torch.float32 or tuple(out.shape) != (B, H)):
        raise ValueError(f"out must be float32 [{B}][{H}], got {out.dtype} {tuple(out.shape)}")
    _need_cuda(x, out, w_gate, w_up, w_down_t, w_router)


def ffn_workspace_bytes(batch: int, hidden: int, inter: int, wdtype: int) -> int:
    return int(lib.ts_ffn_workspace_bytes(batch, hidden, inter, wdtype))


def ffn_given_workspace_bytes(batch: int, hidden: int, inter: int, max_count: int, wdtype: int) -> int:
    return int(lib.ts_ffn_given_workspace_bytes(batch, hidden, inter, max_count, wdtype))


def moe_workspace_bytes(batch: int, hidden: int, inter: int, n_experts: int, top_k: int, wdtype: int) -> int:
    return int(lib.ts_moe_workspace_bytes(batch, hidden, inter, n_experts, top_k, wdtype))


def _workspace(sizer, device, ws, *sizes):
    """The caller's workspace (any dtype; its size in bytes is passed on), or
    a new one of the size the library asks for, sizer(*sizes)."""
    if ws is not None:
        _need_cuda(ws)
        if ws.device != device:
            raise ValueError(f"workspace on {ws.device}, tensors on {device}")
        return ws
    return torch.empty(max(sizer(*sizes), 256), dtype=torch.uint8, device=device)


def _nbytes(t):
    return t.numel() * t.element_size()


def _stats_struct(batch_slots: int, inter: int, device, want: bool):
    if not want:
        return None, None
    d = {
        "n_gate": torch.empty(batch_slots, dtype=torch.int32, device=device),
        "n_active": torch.empty(batch_slots, dtype=torch.int32, device=device),
        "gate_idx": torch.empty(batch_slots, inter, dtype=torch.int32, device=device),
        "active_idx": torch.empty(batch_slots, inter, dtype=torch.int32, device=device),
    }
    s = ffn_stats_t(_ptr(d["n_gate"]), _ptr(d["n_active"]), _ptr(d["gate_idx"]), _ptr(d["active_idx"]), None)
    return s, d


def ffn_sparse(x, w_gate, w_up, w_down_t, out=None, stats: bool = False, union: bool = False, ws=None,
               stream=None):
    """ts_ffn_sparse.  x [B][H] f32; weights [I][H] f32/bf16.  Returns out, or
    (out, stats dict) when stats/union is requested."""
    _check_tensors(x, w_gate, w_up, w_down_t, out)
    B, H = x.shape
    I = w_gate.shape[0]
    dt = wdtype_of(w_gate)
    if out is None:
        out = torch.empty(B, H, dtype=torch.float32, device=x.device)
    ws = _workspace(ffn_workspace_bytes, x.device, ws, B, H, I, dt)
    st, d = _stats_struct(B, I, x.device, stats or union)
    if union:
        d["n_union"] = torch.empty(2, dtype=torch.int32, device=x.device)
        st.n_union = _ptr(d["n_union"])
    code = lib.ts_ffn_sparse(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down_t), dt, B, H, I, _ptr(out),
                             ctypes.byref(st) if st is not None else None, _ptr(ws), _nbytes(ws), _stream(stream))
    if code:
        _check(code, "ts_ffn_sparse")
    return (out, d) if d is not None else out


# the fixed scratch array of ts_ffn_sparse_noalloc (TS_NOALLOC_SCRATCH_BYTES)
NOALLOC_SCRATCH_BYTES = 32 << 20


def ffn_sparse_noalloc(x, w_gate, w_up, w_down_t, out=None, stats: bool = False, union: bool = False,
                       stream=None):
    """ts_ffn_sparse_noalloc: ts_ffn_sparse with the library's fixed scratch
    array instead of a workspace.  Pass `out` to make the call allocate
    nothing on the Python side either.  Returns out, or (out, stats dict)."""
    _check_tensors(x, w_gate, w_up, w_down_t, out)
    B, H = x.shape
    I = w_gate.shape[0]
    dt = wdtype_of(w_gate)
    if out is None:
        out = torch.empty(B, H, dtype=torch.float32, device=x.device)
    st, d = _stats_struct(B, I, x.device, stats or union)
    if union:
        d["n_union"] = torch.empty(2, dtype=torch.int32, device=x.device)
        st.n_union = _ptr(d["n_union"])
    code = lib.ts_ffn_sparse_noalloc(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down_t), dt, B, H, I, _ptr(out),
                                     ctypes.byref(st) if st is not None else None, _stream(stream))
    if code:
        _check(code, "ts_ffn_sparse_noalloc")
    return (out, d) if d is not None else out


TS_ACT_DRELU = 0
TS_ACT_RELU_GATE = 1


def ffn_sparse_act(x, w_gate, w_up, w_down_t, act: int, tau: float = 0.0, out=None, stats: bool = False,
                   union: bool = False, ws=None, stream=None):
    """ts_ffn_sparse_act: act TS_ACT_DRELU (tau 0) or TS_ACT_RELU_GATE
    (Combined = max(0, gate - tau) * up).  Returns out, or (out, stats dict)."""
    _check_tensors(x, w_gate, w_up, w_down_t, out)
    B, H = x.shape
    I = w_gate.shape[0]
    dt = wdtype_of(w_gate)
    if out is None:
        out = torch.empty(B, H, dtype=torch.float32, device=x.device)
    ws = _workspace(ffn_workspace_bytes, x.device, ws, B, H, I, dt)
    st, d = _stats_struct(B, I, x.device, stats or union)
    if union:
        d["n_union"] = torch.empty(2, dtype=torch.int32, device=x.device)
        st.n_union = _ptr(d["n_union"])
    code = lib.ts_ffn_sparse_act(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down_t), dt, B, H, I, int(act),
                                 float(tau), _ptr(out), ctypes.byref(st) if st is not None else None, _ptr(ws),
                                 _nbytes(ws), _stream(stream))
    if code:
        _check(code, "ts_ffn_sparse_act")
    return (out, d) if d is not None else out


def ffn_sparse_topk(x, w_gate, w_up, w_down_t, keep: int, out=None, stats: bool = False, ws=None, stream=None):
    """ts_ffn_sparse_topk: dReLU FFN keeping each token's `keep` largest
    Combined activations.  Returns out, or (out, stats dict)."""
    _check_tensors(x, w_gate, w_up, w_down_t, out)
    B, H = x.shape
    I = w_gate.shape[0]
    dt = wdtype_of(w_gate)
    if out is None:
        out = torch.empty(B, H, dtype=torch.float32, device=x.device)
    ws = _workspace(ffn_workspace_bytes, x.device, ws, B, H, I, dt)
    st, d = _stats_struct(B, I, x.device, stats)
    code = lib.ts_ffn_sparse_topk(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down_t), dt, B, H, I, int(keep),
                                  _ptr(out), ctypes.byref(st) if st is not None else None, _ptr(ws), _nbytes(ws),
                                  _stream(stream))
    if code:
        _check(code, "ts_ffn_sparse_topk")
    return (out, d) if d is not None else out


def ffn_dense(x, w_gate, w_up, w_down_t, out=None, ws=None, stream=None):
    """ts_ffn_dense (all neurons, all three matrices read)."""
    _check_tensors(x, w_gate, w_up, w_down_t, out)
    B, H = x.shape
    I = w_gate.shape[0]
    dt = wdtype_of(w_gate)
    if out is None:
        out = torch.empty(B, H, dtype=torch.float32, device=x.device)
    ws = _workspace(ffn_workspace_bytes, x.device, ws, B, H, I, dt)
    code = lib.ts_ffn_dense(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down_t), dt, B, H, I, _ptr(out), _ptr(ws),
                            _nbytes(ws), _stream(stream))
    if code:
        _check(code, "ts_ffn_dense")
    return out


def ffn_sparse_given(x, w_gate, w_up, w_down_t, idx, count, out=None, stats: bool = False, ws=None, stream=None):
    """ts_ffn_sparse_given: the FFN over given neuron lists.  idx int32
    [B][max_count], count int32 [B] (device tensors).  Returns out, or (out,
    {"n_gate", "n_active"}) with stats=True."""
    _check_tensors(x, w_gate, w_up, w_down_t, out)
    _need_cuda(x, idx, count)
    B, H = x.shape
    I = w_gate.shape[0]
    dt = wdtype_of(w_gate)
    if idx.dim() != 2 or idx.shape[0] != B or count.numel() != B:
        raise ValueError("idx must be [batch][max_count] and count [batch]")
    if idx.dtype != torch.int32 or count.dtype != torch.int32:
        raise TypeError("idx and count must be int32")
    maxc = idx.shape[1]
    if out is None:
        out = torch.empty(B, H, dtype=torch.float32, device=x.device)
    ws = _workspace(ffn_given_workspace_bytes, x.device, ws, B, H, I, maxc, dt)
    d = st = None
    if stats:
        d = {"n_gate": torch.empty(B, dtype=torch.int32, device=x.device),
             "n_active": torch.empty(B, dtype=torch.int32, device=x.device)}
        st = ffn_stats_t(_ptr(d["n_gate"]), _ptr(d["n_active"]), None, None, None)
    code = lib.ts_ffn_sparse_given(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(w_down_t), dt, B, H, I, _ptr(idx),
                                   _ptr(count), maxc, _ptr(out), ctypes.byref(st) if st is not None else None,
                                   _ptr(ws), _nbytes(ws), _stream(stream))
    if code:
        _check(code, "ts_ffn_sparse_given")
    return (out, d) if d is not None else out


def moe_sparse(x, w_router, w_gate, w_up, w_down_t, top_k: int, out=None, stats: bool = False, ws=None,
               stream=None, dense: bool = False):
    """ts_moe_sparse (or ts_moe_dense with dense=True).  Returns
    (out, topk_idx, topk_w) or (out, topk_idx, topk_w, stats dict)."""
    _check_tensors(x, w_gate, w_up, w_down_t, out, w_router=w_router)
    B, H = x.shape
    E, I = w_gate.shape[0], w_gate.shape[1]
    dt = wdtype_of(w_gate)
    if out is None:
        out = torch.empty(B, H, dtype=torch.float32, device=x.device)
    idx = torch.empty(B, top_k, dtype=torch.int32, device=x.device)
    wts = torch.empty(B, top_k, dtype=torch.float32, device=x.device)
    ws = _workspace(moe_workspace_bytes, x.device, ws, B, H, I, E, top_k, dt)
    if dense:
        code = lib.ts_moe_dense(_ptr(x), _ptr(w_router), _ptr(w_gate), _ptr(w_up), _ptr(w_down_t), dt, B, H, I, E,
                                top_k, _ptr(out), _ptr(idx), _ptr(wts), _ptr(ws), _nbytes(ws), _stream(stream))
        if code:
            _check(code, "ts_moe_dense")
        return out, idx, wts
    st, d = _stats_struct(B * top_k, I, x.device, stats)
    code = lib.ts_moe_sparse(_ptr(x), _ptr(w_router), _ptr(w_gate), _ptr(w_up), _ptr(w_down_t), dt, B, H, I, E,
                             top_k, _ptr(out), _ptr(idx), _ptr(wts), ctypes.byref(st) if st is not None else None,
                             _ptr(ws), _nbytes(ws), _stream(stream))
    if code:
        _check(code, "ts_moe_sparse")
    return (out, idx, wts, d) if d is not None else (out, idx, wts)


def moe_dense(x, w_router, w_gate, w_up, w_down_t, top_k: int, out=None, ws=None, stream=None):
    return moe_sparse(x, w_router, w_gate, w_up, w_down_t, top_k, out=out, ws=ws, stream=stream, dense=True)


# ---------------------------------------------------------------------------
# The MoE layer on any number of tokens, its gradients, its 8-bit form.  With
# `stream`, a call runs there and what it makes is that stream's memory, as
# under torch.cuda.stream(stream): memory that other streams freed may still be
# in use there, and a workspace is freed as the call returns.

_i32, _u8, _e4m3 = torch.int32, torch.uint8, torch.float8_e4m3fn
_int_max = 0x7fffffff


def _need_int(name, ns):
    """The library's sizes are C ints, to which larger numbers would wrap."""
    if max(ns) > _int_max:
        raise ValueError(f"{name}: extents must be below 2^31, got {tuple(ns)}")


def _need(t, name, dtype, shape):
    """Raises unless t has this dtype (or one of them) and shape (None: any
    extent; a number: so many dimensions)."""
    dt = t.dtype
    if dt is dtype or (type(dtype) is tuple and dt in dtype):
        s = t.shape
        if type(shape) is int:
            ok = len(s) == shape
        else:
            ok = s == shape
            if not ok and len(s) == len(shape):
                ok = True
                for n, w in zip(s, shape):
                    if w is not None and n != w:
                        ok = False
        if ok:
            if t.numel() > _int_max:
                _need_int(name, s)
            return
    dts = dtype if isinstance(dtype, tuple) else (dtype,)
    if dt not in dts:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dts)}, got {dt}")
    if isinstance(shape, int):
        shape = (None,) * shape
    if len(t.shape) != len(shape) or any(w is not None and n != w for n, w in zip(t.shape, shape)):
        want = "".join(f"[{'*' if w is None else w}]" for w in shape)
        raise ValueError(f"{name} must be {want}, got {tuple(t.shape)}")
    _need_int(name, t.shape)


def _run_on(stream, f, *args):
    if stream.device.index != torch.cuda.current_device():
        raise ValueError(f"stream on {stream.device}, current device cuda:{torch.cuda.current_device()}")
    with torch.cuda.stream(stream):
        return f(*args)


def _here(*ts):
    """All tensors contiguous on the current device; the current stream."""
    d = _cur_device() if _cur_device is not None and torch.cuda.is_initialized() else None
    for t in ts:
        if t is None:
            continue
        if t.get_device() == d and t.is_contiguous():  # (d is None or >= 0, -1 is the host)
            continue
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous device tensors")
        if d is None:
            d = torch.cuda.current_device()
        if t.get_device() != d:
            raise ValueError(f"tensor on {t.device}, current device cuda:{d}")
    return _stream(None)


def _new(out, name, shape, dtype, device):
    """The caller's output, checked, or a new one."""
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _need(out, name, dtype, shape)
    return out


def moe_route_workspace_bytes(tokens: int, n_experts: int, top_k: int) -> int:
    return int(lib.ts_moe_route_workspace_bytes(tokens, n_experts, top_k))


def _route_ws(dev, ws, T, E, K):
    """A workspace where the call needs one (small calls do not)."""
    n = 0 if ws is not None else moe_route_workspace_bytes(T, E, K)
    return torch.empty(n, dtype=torch.uint8, device=dev) if n else ws


def _maps(T, E, K, dev):
    return (torch.empty(E + 1, dtype=_i32, device=dev), torch.empty(T * K, dtype=_i32, device=dev),
            torch.empty(T, K, dtype=_i32, device=dev))


def moe_route(logits, top_k: int, maps: bool = True, ws=None, stream=None):
    """ts_moe_route.  logits [T][E] f32.  Returns topk_idx, topk_w [T][K] and,
    with maps, offsets [E + 1], row_token [T K], pair_row [T][K]."""
    if stream is not None:
        return _run_on(stream, moe_route, logits, top_k, maps, ws)
    _need(logits, "logits", _f32, 2)
    st = _here(logits, ws)
    T, E = logits.shape
    K = int(top_k)
    if not 1 <= K <= E:
        raise ValueError(f"top_k must be in 1..{E}, got {K}")
    dev = logits.device
    idx, w = torch.empty(T, K, dtype=_i32, device=dev), torch.empty(T, K, dtype=_f32, device=dev)
    m = _maps(T, E, K, dev) if maps else (None, None, None)
    if maps:
        ws = _route_ws(dev, ws, T, E, K)
    code = lib.ts_moe_route(_ptr(logits), T, E, K, _ptr(idx), _ptr(w), _ptr(m[0]), _ptr(m[1]), _ptr(m[2]), _ptr(ws),
                            _nbytes(ws) if ws is not None else 0, st)
    if code:
        _check(code, "ts_moe_route")
    return (idx, w, *m) if maps else (idx, w)


def moe_group(topk_idx, n_experts: int, ws=None, stream=None):
    """ts_moe_group.  topk_idx [T][K] int32.  Returns offsets [E + 1],
    row_token [T K] (entries from offsets[E] on unspecified), pair_row [T][K]."""
    if stream is not None:
        return _run_on(stream, moe_group, topk_idx, n_experts, ws)
    _need(topk_idx, "topk_idx", _i32, 2)
    T, K = topk_idx.shape
    E = int(n_experts)
    if not 1 <= E <= _int_max:
        raise ValueError(f"n_experts must be in 1..2^31 - 1, got {E}")
    st = _here(topk_idx, ws)
    m = _maps(T, E, K, topk_idx.device)
    ws = _route_ws(topk_idx.device, ws, T, E, K)
    code = lib.ts_moe_group(_ptr(topk_idx), T, E, K, _ptr(m[0]), _ptr(m[1]), _ptr(m[2]), _ptr(ws),
                            _nbytes(ws) if ws is not None else 0, st)
    if code:
        _check(code, "ts_moe_group")
    return m


def moe_route_grad(topk_idx, topk_w, d_w, n_experts: int, out=None, stream=None):
    """ts_moe_route_grad: d_logits [T][E] from d_w [T][K] (the gradient of topk_w)."""
    if stream is not None:
        return _run_on(stream, moe_route_grad, topk_idx, topk_w, d_w, n_experts, out)
    _need(topk_idx, "topk_idx", _i32, 2)
    T, K = topk_idx.shape
    E = int(n_experts)
    if not 1 <= E <= _int_max:
        raise ValueError(f"n_experts must be in 1..2^31 - 1, got {E}")
    _need(topk_w, "topk_w", _f32, (T, K))
    _need(d_w, "d_w", _f32, (T, K))
    st = _here(topk_idx, topk_w, d_w, out)
    out = _new(out, "out", (T, E), _f32, topk_idx.device)
    code = lib.ts_moe_route_grad(_ptr(topk_idx), _ptr(topk_w), _ptr(d_w), T, E, K, _ptr(out), st)
    if code:
        _check(code, "ts_moe_route_grad")
    return out


def _need_mask(mask, T):
    if mask is not None:
        _need(mask, "mask", (torch.bool, _u8), (T,))


def moe_balance(logits, topk_idx, mask=None, ws=None, stream=None):
    """ts_moe_balance.  logits [T][E] f32, topk_idx [T][K] int32, mask [T] bool or
    uint8 (tokens that count).  Returns loss f32 [2] (balance, squared log-sum)
    and counts int32 [E + 1] (pairs of each expert, tokens)."""
    if stream is not None:
        return _run_on(stream, moe_balance, logits, topk_idx, mask, ws)
    _need(logits, "logits", _f32, 2)
    T, E = logits.shape
    _need(topk_idx, "topk_idx", _i32, (T, None))
    _need_mask(mask, T)
    st = _here(logits, topk_idx, mask, ws)
    K, dev = topk_idx.shape[1], logits.device
    loss, counts = torch.empty(2, dtype=_f32, device=dev), torch.empty(E + 1, dtype=_i32, device=dev)
    n = 0 if ws is not None else int(lib.ts_moe_balance_workspace_bytes(T, E, K))
    if n:
        ws = torch.empty(n, dtype=_u8, device=dev)
    code = lib.ts_moe_balance(_ptr(logits), _ptr(topk_idx), _ptr(mask), T, E, K, _ptr(loss), _ptr(counts), _ptr(ws),
                              _nbytes(ws) if ws is not None else 0, st)
    if code:
        _check(code, "ts_moe_balance")
    return loss, counts


def moe_balance_grad(logits, counts, d_loss, top_k: int, mask=None, add=None, out=None, stream=None):
    """ts_moe_balance_grad.  d_loss f32 [2] on the device.  Returns d_logits
    [T][E], added to `add` if given (out may be add: in place)."""
    if stream is not None:
        return _run_on(stream, moe_balance_grad, logits, counts, d_loss, top_k, mask, add, out)
    _need(logits, "logits", _f32, 2)
    T, E = logits.shape
    K = int(top_k)
    if not 1 <= K <= E:
        raise ValueError(f"top_k must be in 1..{E}, got {K}")
    _need(counts, "counts", _i32, (E + 1,))
    _need(d_loss, "d_loss", _f32, (2,))
    _need_mask(mask, T)
    if add is not None:
        _need(add, "add", _f32, (T, E))
    st = _here(logits, counts, d_loss, mask, add, out)
    out = torch.empty_like(logits) if out is None else _new(out, "out", (T, E), _f32, logits.device)
    code = lib.ts_moe_balance_grad(_ptr(logits), _ptr(counts), _ptr(d_loss), _ptr(mask), _ptr(add), T, E, K, _ptr(out),
                                   st)
    if code:
        _check(code, "ts_moe_balance_grad")
    return out


def _rows_of(x, offsets, row_src, G):
    """Rows of a grouped product; checks offsets [G + 1] and row_src."""
    if offsets is not None:
        _need(offsets, "offsets", _i32, (G + 1,))
    elif G != 1:
        raise ValueError(f"{G} groups need offsets")
    if row_src is not None:
        _need(row_src, "row_src", _i32, 1)
        if x.shape[0] == 0 and row_src.shape[0] > 0:
            raise ValueError("row_src names rows of an empty x")
        return row_src.shape[0]
    return x.shape[0]


def _odtype(out, out_dtype, default):
    dt = out_dtype if out_dtype is not None else (out.dtype if out is not None else default)
    return dt, wdtype_of_rows(dt)


def wdtype_of_rows(dt) -> int:
    if dt is _f32:
        return TS_F32
    if dt is _bf16:
        return TS_BF16
    raise TypeError(f"rows must be float32 or bfloat16, got {dt}")


def grouped_mm(x, w, offsets=None, row_src=None, x2=None, w2=None, w_kn: bool = False, out=None, out_dtype=None,
               stream=None):
    """ts_grouped_mm.  x [S][k]; w [G][n][k], or [G][k][n] with w_kn; bf16 or
    f32, one dtype; x2, w2: a second product added to the first.  Returns out
    [rows][n] (out_dtype: x's unless given), rows = len(row_src) or S; rows
    outside the groups are not written."""
    if stream is not None:
        return _run_on(stream, grouped_mm, x, w, offsets, row_src, x2, w2, w_kn, out, out_dtype)
    _need(x, "x", (_f32, _bf16), 2)
    S, k = x.shape
    _need(w, "w", x.dtype, 3)
    G, n = w.shape[0], w.shape[2] if w_kn else w.shape[1]
    _need(w, "w", x.dtype, (None, k, n) if w_kn else (None, n, k))
    if (x2 is None) != (w2 is None):
        raise ValueError("x2 and w2 go together")
    if x2 is not None:
        _need(x2, "x2", x.dtype, (S, k))
        _need(w2, "w2", x.dtype, tuple(w.shape))
    R = _rows_of(x, offsets, row_src, G)
    odt, od = _odtype(out, out_dtype, x.dtype)
    st = _here(x, w, x2, w2, offsets, row_src, out)
    out = _new(out, "out", (R, n), odt, x.device)
    code = lib.ts_grouped_mm(_ptr(x), _ptr(w), _ptr(x2), _ptr(w2), wdtype_of_rows(x.dtype), int(bool(w_kn)),
                             _ptr(row_src), _ptr(offsets), R, S, G, n, k, _ptr(out), od, st)
    if code:
        _check(code, "ts_grouped_mm")
    return out


def grouped_drelu(x, w_gate, w_up, offsets=None, row_src=None, keep: bool = False, out=None, out_dtype=None,
                  stream=None):
    """ts_grouped_drelu.  x [S][k]; w_gate, w_up [G][n][k].  Returns c
    [rows][n], or (c, gate, up) with keep."""
    if stream is not None:
        return _run_on(stream, grouped_drelu, x, w_gate, w_up, offsets, row_src, keep, out, out_dtype)
    _need(x, "x", (_f32, _bf16), 2)
    S, k = x.shape
    _need(w_gate, "w_gate", x.dtype, (None, None, k))
    _need(w_up, "w_up", x.dtype, tuple(w_gate.shape))
    G, n = w_gate.shape[:2]
    R = _rows_of(x, offsets, row_src, G)
    odt, od = _odtype(out, out_dtype, x.dtype)
    st = _here(x, w_gate, w_up, offsets, row_src, out)
    out = _new(out, "out", (R, n), odt, x.device)
    gate, up = (torch.empty_like(out), torch.empty_like(out)) if keep else (None, None)
    code = lib.ts_grouped_drelu(_ptr(x), _ptr(w_gate), _ptr(w_up), wdtype_of_rows(x.dtype), _ptr(row_src),
                                _ptr(offsets), R, S, G, n, k, _ptr(out), _ptr(gate), _ptr(up), od, st)
    if code:
        _check(code, "ts_grouped_drelu")
    return (out, gate, up) if keep else out


def drelu_grad(gate, up, d_c, stream=None):
    """ts_drelu_grad: (d_gate, d_up) of c = max(0, gate) * max(0, up)."""
    if stream is not None:
        return _run_on(stream, drelu_grad, gate, up, d_c)
    _need(gate, "gate", (_f32, _bf16), 2)
    _need(up, "up", gate.dtype, tuple(gate.shape))
    _need(d_c, "d_c", gate.dtype, tuple(gate.shape))
    st = _here(gate, up, d_c)
    dg, du = torch.empty_like(gate), torch.empty_like(gate)
    code = lib.ts_drelu_grad(_ptr(gate), _ptr(up), _ptr(d_c), wdtype_of_rows(gate.dtype), gate.shape[0],
                             gate.shape[1], _ptr(dg), _ptr(du), st)
    if code:
        _check(code, "ts_drelu_grad")
    return dg, du


def _need_kept(codes, exps, rows, n):
    _need(codes, "codes", _u8, (rows, n, 2))
    _need(exps, "exps", _u8, (rows, (n + 15) // 16, 2))


def grouped_drelu_pack(x, w_gate, w_up, offsets=None, row_src=None, out=None, out_dtype=None, codes=None, exps=None,
                       stream=None):
    """ts_grouped_drelu_pack: grouped_drelu that keeps max(0, gate) and
    max(0, up) in 8 bits.  Returns c [rows][n], codes uint8 [rows][n][2], exps
    uint8 [rows][ceil(n / 16)][2]."""
    if stream is not None:
        return _run_on(stream, grouped_drelu_pack, x, w_gate, w_up, offsets, row_src, out, out_dtype, codes, exps)
    _need(x, "x", (_f32, _bf16), 2)
    S, k = x.shape
    _need(w_gate, "w_gate", x.dtype, (None, None, k))
    _need(w_up, "w_up", x.dtype, tuple(w_gate.shape))
    G, n = w_gate.shape[:2]
    R = _rows_of(x, offsets, row_src, G)
    odt, od = _odtype(out, out_dtype, x.dtype)
    st = _here(x, w_gate, w_up, offsets, row_src, out, codes, exps)
    out = _new(out, "out", (R, n), odt, x.device)
    codes = _new(codes, "codes", (R, n, 2), _u8, x.device)
    exps = _new(exps, "exps", (R, (n + 15) // 16, 2), _u8, x.device)
    code = lib.ts_grouped_drelu_pack(_ptr(x), _ptr(w_gate), _ptr(w_up), wdtype_of_rows(x.dtype), _ptr(row_src),
                                     _ptr(offsets), R, S, G, n, k, _ptr(out), _ptr(codes), _ptr(exps), od, st)
    if code:
        _check(code, "ts_grouped_drelu_pack")
    return out, codes, exps


def grouped_drelu_grad(d_y, w, codes, exps, offsets=None, row_src=None, want_c: bool = True, out_dtype=None,
                       stream=None):
    """ts_grouped_drelu_grad.  d_y [S][k], w [G][n][k] (w_down_t), codes and
    exps of grouped_drelu_pack.  Returns d_gate, d_up [rows][n] and, with want_c,
    c (d_y's dtype unless given)."""
    if stream is not None:
        return _run_on(stream, grouped_drelu_grad, d_y, w, codes, exps, offsets, row_src, want_c, out_dtype)
    _need(d_y, "d_y", (_f32, _bf16), 2)
    S, k = d_y.shape
    _need(w, "w", d_y.dtype, (None, None, k))
    G, n = w.shape[:2]
    R = _rows_of(d_y, offsets, row_src, G)
    _need_kept(codes, exps, R, n)
    odt, od = _odtype(None, out_dtype, d_y.dtype)
    st = _here(d_y, w, codes, exps, offsets, row_src)
    dg, du = (torch.empty(R, n, dtype=odt, device=d_y.device) for _ in range(2))
    c = torch.empty(R, n, dtype=odt, device=d_y.device) if want_c else None
    code = lib.ts_grouped_drelu_grad(_ptr(d_y), _ptr(w), wdtype_of_rows(d_y.dtype), _ptr(row_src), _ptr(offsets), R, S,
                                     G, n, k, _ptr(codes), _ptr(exps), _ptr(dg), _ptr(du), _ptr(c), od, st)
    if code:
        _check(code, "ts_grouped_drelu_grad")
    return (dg, du, c) if want_c else (dg, du)


def drelu_unpack(codes, exps, stream=None):
    """ts_drelu_unpack: max(0, gate) and max(0, up) as kept, bf16 [rows][n]."""
    if stream is not None:
        return _run_on(stream, drelu_unpack, codes, exps)
    _need(codes, "codes", _u8, (None, None, 2))
    R, n = codes.shape[:2]
    _need_kept(codes, exps, R, n)
    st = _here(codes, exps)
    g, u = (torch.empty(R, n, dtype=_bf16, device=codes.device) for _ in range(2))
    code = lib.ts_drelu_unpack(_ptr(codes), _ptr(exps), R, n, _ptr(g), _ptr(u), st)
    if code:
        _check(code, "ts_drelu_unpack")
    return g, u


def grouped_mm_dw(d_y, x, offsets=None, row_src=None, out=None, out_dtype=None, stream=None):
    """ts_grouped_mm_dw.  d_y [rows][n], x [S][k] -> d_w [G][n][k] (f32 unless
    out_dtype or out says otherwise), G = len(offsets) - 1."""
    if stream is not None:
        return _run_on(stream, grouped_mm_dw, d_y, x, offsets, row_src, out, out_dtype)
    _need(x, "x", (_f32, _bf16), 2)
    _need(d_y, "d_y", x.dtype, 2)
    if offsets is not None:
        _need(offsets, "offsets", _i32, 1)
    G = 1 if offsets is None else offsets.shape[0] - 1
    if G < 1:
        raise ValueError("offsets must hold n_groups + 1 entries, at least two")
    R = _rows_of(x, offsets, row_src, G)
    if d_y.shape[0] != R:
        raise ValueError(f"d_y has {d_y.shape[0]} rows, the product {R}")
    (S, k), n = x.shape, d_y.shape[1]
    odt, od = _odtype(out, out_dtype, _f32)
    st = _here(d_y, x, offsets, row_src, out)
    out = _new(out, "out", (G, n, k), odt, x.device)
    code = lib.ts_grouped_mm_dw(_ptr(d_y), _ptr(x), wdtype_of_rows(x.dtype), _ptr(row_src), _ptr(offsets), R, S, G,
                                n, k, _ptr(out), od, st)
    if code:
        _check(code, "ts_grouped_mm_dw")
    return out


def _nblk(n):
    return (n + 127) // 128


def fp8_quant(x, stream=None):
    """ts_fp8_quant.  x [rows][cols] bf16 / f32 -> (codes float8_e4m3fn
    [rows][cols], scale f32 [rows][ceil(cols / 128)])."""
    if stream is not None:
        return _run_on(stream, fp8_quant, x)
    _need(x, "x", (_f32, _bf16), 2)
    st = _here(x)
    R, C = x.shape
    q = torch.empty(R, C, dtype=_e4m3, device=x.device)
    s = torch.empty(R, _nblk(C), dtype=_f32, device=x.device)
    code = lib.ts_fp8_quant(_ptr(x), wdtype_of_rows(x.dtype), R, C, _ptr(q), _ptr(s), st)
    if code:
        _check(code, "ts_fp8_quant")
    return q, s


def fp8_quant_weights(w, w_kn: bool = False, stream=None):
    """ts_fp8_quant_weights.  w [G][n][k], or [G][k][n] with w_kn -> (codes
    [G][n][k], scale [G][ceil(n / 128)][ceil(k / 128)])."""
    if stream is not None:
        return _run_on(stream, fp8_quant_weights, w, w_kn)
    _need(w, "w", (_f32, _bf16), 3)
    st = _here(w)
    G, n, k = (w.shape[0], w.shape[2], w.shape[1]) if w_kn else w.shape
    q = torch.empty(G, n, k, dtype=_e4m3, device=w.device)
    s = torch.empty(G, _nblk(n), _nblk(k), dtype=_f32, device=w.device)
    code = lib.ts_fp8_quant_weights(_ptr(w), wdtype_of_rows(w.dtype), int(bool(w_kn)), G, n, k, _ptr(q), _ptr(s), st)
    if code:
        _check(code, "ts_fp8_quant_weights")
    return q, s


def _fp8_shapes(x, x_scale, ws):
    _need(x, "x", _e4m3, 2)
    S, k = x.shape
    _need(x_scale, "x_scale", _f32, (S, _nblk(k)))
    G, n = None, None
    for name, w, scale in ws:
        _need(w, name, _e4m3, (G, n, k))
        G, n = w.shape[:2]
        _need(scale, f"scale of {name}", _f32, (G, _nblk(n), _nblk(k)))
    return S, k, G, n


def fp8_mm(x, x_scale, w, w_scale, offsets=None, row_src=None, out=None, out_dtype=None, stream=None):
    """ts_fp8_mm on the codes and scales of fp8_quant and fp8_quant_weights.
    Returns out [rows][n] (bf16 unless out_dtype or out says otherwise).  A
    block's sums come from the matrix instructions, which keep fewer bits than
    fp32 (5e-5 of the result's 2-norm; more of one whose products cancel)."""
    if stream is not None:
        return _run_on(stream, fp8_mm, x, x_scale, w, w_scale, offsets, row_src, out, out_dtype)
    S, k, G, n = _fp8_shapes(x, x_scale, (("w", w, w_scale),))
    R = _rows_of(x, offsets, row_src, G)
    odt, od = _odtype(out, out_dtype, _bf16)
    st = _here(x, x_scale, w, w_scale, offsets, row_src, out)
    out = _new(out, "out", (R, n), odt, x.device)
    code = lib.ts_fp8_mm(_ptr(x), _ptr(x_scale), _ptr(w), _ptr(w_scale), _ptr(row_src), _ptr(offsets), R, S, G, n, k,
                         _ptr(out), od, st)
    if code:
        _check(code, "ts_fp8_mm")
    return out


def fp8_drelu(x, x_scale, w_gate, gate_scale, w_up, up_scale, offsets=None, row_src=None, out=None, out_dtype=None,
              stream=None):
    """ts_fp8_drelu: grouped_drelu on quantised rows and weights (sums as in
    fp8_mm)."""
    if stream is not None:
        return _run_on(stream, fp8_drelu, x, x_scale, w_gate, gate_scale, w_up, up_scale, offsets, row_src, out,
                       out_dtype)
    S, k, G, n = _fp8_shapes(x, x_scale, (("w_gate", w_gate, gate_scale), ("w_up", w_up, up_scale)))
    R = _rows_of(x, offsets, row_src, G)
    odt, od = _odtype(out, out_dtype, _bf16)
    st = _here(x, x_scale, w_gate, gate_scale, w_up, up_scale, offsets, row_src, out)
    out = _new(out, "out", (R, n), odt, x.device)
    code = lib.ts_fp8_drelu(_ptr(x), _ptr(x_scale), _ptr(w_gate), _ptr(gate_scale), _ptr(w_up), _ptr(up_scale),
                            _ptr(row_src), _ptr(offsets), R, S, G, n, k, _ptr(out), od, st)
    if code:
        _check(code, "ts_fp8_drelu")
    return out


def _adapter_shapes(x, offsets, adapter, scale, a, name):
    """(rows, k, segments, adapters, rank)."""
    _need(x, "x", (_f32, _bf16), 2)
    R, k = x.shape
    _need(a, name, x.dtype, (None, None, k))
    N, rank = a.shape[:2]
    _need(adapter, "adapter", _i32, 1)
    S = adapter.shape[0]
    _need(offsets, "offsets", _i32, (S + 1,))
    if scale is not None:
        _need(scale, "scale", _f32, (N,))
    return R, k, S, N, rank


def adapter_workspace_bytes(rows: int, rank: int, products: int, w_kn: bool, n: int, k: int, dtype, out_dtype) -> int:
    return int(lib.ts_adapter_workspace_bytes(rows, rank, products, int(bool(w_kn)), n, k, wdtype_of_rows(dtype),
                                              wdtype_of_rows(out_dtype)))


def _adapter_ws(dev, ws, *sizes):
    return ws if ws is not None else torch.empty(adapter_workspace_bytes(*sizes), dtype=_u8, device=dev)


def adapter_mm(x, w, a, b, offsets, adapter, scale=None, w_kn: bool = False, out=None, out_dtype=None, ws=None,
               stream=None):
    """ts_adapter_mm.  x [rows][k], w [n][k], a [N][rank][k], b [N][n][rank]; with
    w_kn w [k][n], b [N][rank][n]; bf16 or f32, one dtype; offsets [S + 1], adapter
    [S] int32, scale [N] f32 or None.  Returns out [rows][n] (x's dtype unless
    given); rows outside the segments are not written."""
    if stream is not None:
        return _run_on(stream, adapter_mm, x, w, a, b, offsets, adapter, scale, w_kn, out, out_dtype, ws)
    R, k, S, N, rank = _adapter_shapes(x, offsets, adapter, scale, a, "a")
    _need(w, "w", x.dtype, (k, None) if w_kn else (None, k))
    n = w.shape[1] if w_kn else w.shape[0]
    _need(b, "b", x.dtype, (N, rank, n) if w_kn else (N, n, rank))
    odt, od = _odtype(out, out_dtype, x.dtype)
    st = _here(x, w, a, b, offsets, adapter, scale, out, ws)
    out = _new(out, "out", (R, n), odt, x.device)
    ws = _adapter_ws(x.device, ws, R, rank, 1, w_kn, n, k, x.dtype, odt)
    code = lib.ts_adapter_mm(_ptr(x), _ptr(w), _ptr(a), _ptr(b), _ptr(scale), wdtype_of_rows(x.dtype), int(bool(w_kn)),
                             _ptr(offsets), _ptr(adapter), R, S, N, rank, n, k, _ptr(out), od, _ptr(ws), _nbytes(ws), st)
    if code:
        _check(code, "ts_adapter_mm")
    return out


def adapter_drelu(x, w_gate, w_up, a_gate, b_gate, a_up, b_up, offsets, adapter, scale=None, out=None, out_dtype=None,
                  ws=None, stream=None):
    """ts_adapter_drelu.  w_gate, w_up [n][k], a_gate, a_up [N][rank][k], b_gate,
    b_up [N][n][rank], the rest as adapter_mm.  Returns c [rows][n]."""
    if stream is not None:
        return _run_on(stream, adapter_drelu, x, w_gate, w_up, a_gate, b_gate, a_up, b_up, offsets, adapter, scale, out,
                       out_dtype, ws)
    R, k, S, N, rank = _adapter_shapes(x, offsets, adapter, scale, a_gate, "a_gate")
    _need(w_gate, "w_gate", x.dtype, (None, k))
    n = w_gate.shape[0]
    _need(w_up, "w_up", x.dtype, (n, k))
    _need(a_up, "a_up", x.dtype, (N, rank, k))
    _need(b_gate, "b_gate", x.dtype, (N, n, rank))
    _need(b_up, "b_up", x.dtype, (N, n, rank))
    odt, od = _odtype(out, out_dtype, x.dtype)
    st = _here(x, w_gate, w_up, a_gate, b_gate, a_up, b_up, offsets, adapter, scale, out, ws)
    out = _new(out, "out", (R, n), odt, x.device)
    ws = _adapter_ws(x.device, ws, R, rank, 2, False, n, k, x.dtype, odt)
    code = lib.ts_adapter_drelu(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(a_gate), _ptr(b_gate), _ptr(a_up), _ptr(b_up),
                                _ptr(scale), wdtype_of_rows(x.dtype), _ptr(offsets), _ptr(adapter), R, S, N, rank, n,
                                k, _ptr(out), od, _ptr(ws), _nbytes(ws), st)
    if code:
        _check(code, "ts_adapter_drelu")
    return out


def moe_combine(y, pair_row, w=None, out=None, out_dtype=None, stream=None):
    """ts_moe_combine.  y [rows][H] bf16 / f32, pair_row [T][K] int32, w [T][K]
    f32 or None (weights of one).  Returns out [T][H] (y's dtype unless given)."""
    if stream is not None:
        return _run_on(stream, moe_combine, y, pair_row, w, out, out_dtype)
    _need(y, "y", (_f32, _bf16), 2)
    _need(pair_row, "pair_row", _i32, 2)
    T, K = pair_row.shape
    if w is not None:
        _need(w, "w", _f32, (T, K))
    odt, od = _odtype(out, out_dtype, y.dtype)
    st = _here(y, pair_row, w, out)
    R, H = y.shape
    out = _new(out, "out", (T, H), odt, y.device)
    code = lib.ts_moe_combine(_ptr(y), wdtype_of_rows(y.dtype), _ptr(pair_row), _ptr(w), T, K, H, R, _ptr(out), od, st)
    if code:
        _check(code, "ts_moe_combine")
    return out


def moe_combine_grad(d_out, y, pair_row, w, d_y=None, stream=None):
    """ts_moe_combine_grad.  Returns d_y [rows][H] (y's dtype; rows that no
    pair names are not written) and d_w [T][K]."""
    if stream is not None:
        return _run_on(stream, moe_combine_grad, d_out, y, pair_row, w, d_y)
    _need(y, "y", (_f32, _bf16), 2)
    _need(pair_row, "pair_row", _i32, 2)
    (R, H), (T, K) = y.shape, pair_row.shape
    _need(d_out, "d_out", (_f32, _bf16), (T, H))
    _need(w, "w", _f32, (T, K))
    st = _here(d_out, y, pair_row, w, d_y)
    d_y = _new(d_y, "d_y", (R, H), y.dtype, y.device)
    d_w = torch.empty(T, K, dtype=_f32, device=y.device)
    code = lib.ts_moe_combine_grad(_ptr(d_out), wdtype_of_rows(d_out.dtype), _ptr(y), wdtype_of_rows(y.dtype),
                                   _ptr(pair_row), _ptr(w), T, K, H, R, _ptr(d_y), _ptr(d_w), st)
    if code:
        _check(code, "ts_moe_combine_grad")
    return d_y, d_w


def probe_read(src: torch.Tensor, sink: torch.Tensor, stream=None):
    """ts_probe_read: sink holds one float32 per workgroup (4096)."""
    if sink.dtype != torch.float32 or sink.numel() < 4096:
        raise ValueError("sink must be float32 with at least 4096 elements")
    _need_cuda(src, sink)
    _check(lib.ts_probe_read(_ptr(src), _nbytes(src), _ptr(sink), _stream(stream)), "ts_probe_read")


def probe_copy(src: torch.Tensor, dst: torch.Tensor, stream=None):
    """ts_probe_copy: copies all of src into the start of dst."""
    if _nbytes(dst) < _nbytes(src):
        raise ValueError("dst is smaller than src")
    _need_cuda(src, dst)
    _check(lib.ts_probe_copy(_ptr(src), _ptr(dst), _nbytes(src), _stream(stream)), "ts_probe_copy")


def prof_enable(on: bool):
    lib.ts_prof_enable(1 if on else 0)


def prof_reset():
    lib.ts_prof_reset()


def prof_read(kernel: str):
    n = ctypes.c_long()
    ms = ctypes.c_double()
    _check(lib.ts_prof_read(kernel.encode(), ctypes.byref(n), ctypes.byref(ms)), "ts_prof_read")
    return int(n.value), float(ms.value)


def tune_set(key: str, value: int):
    _check(lib.ts_tune_set(key.encode(), int(value)), "ts_tune_set")


def version() -> str:
    return lib.ts_version().decode()
