"""Thin ctypes binding over the C-ABI library (include/vig_bigla.h).

Argument marshalling only: shapes, dtypes, device pointers and the current HIP stream are
taken from torch tensors and handed to the library; every step of the path runs in the
library's kernels.  There is no CPU or PyTorch fallback: if the HIP library is missing, or a
tensor is not on the GPU, the call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvig_bigla.so")

VIG_OK = 0
VIG_ERR_NULL, VIG_ERR_SHAPE, VIG_ERR_DTYPE, VIG_ERR_UNSUPPORTED = -1, -2, -3, -4
VIG_ERR_ALIGN, VIG_ERR_WORKSPACE, VIG_ERR_HIP, VIG_ERR_LAYOUT = -5, -6, -7, -8
VIG_ERR_SCRATCH_LIMIT = -9
VIG_STATIC_SCRATCH_BYTES = 48 << 20
VIG_F32, VIG_BF16 = 0, 1
VIG_LAYOUT_BHLD, VIG_LAYOUT_BLHD = 0, 1
LAYOUTS = {"bhld": VIG_LAYOUT_BHLD, "blhd": VIG_LAYOUT_BLHD}
PLANS = {"auto": 0, "two_launches": 1, "fused_epilogue": 2}
FWD_PLANS = {"auto": 0, "four_wave": 1, "wave_specialised": 2, "slab_sweep": 3}
GATES_PLANS = {"auto": 0, "separate": 1, "in_state_pass": 2}
SCANS = {"forward": 0, "backward": 1}
ACTS = {"none": 0, "silu": 1}

# every symbol include/vig_bigla.h declares
EXPORTS = ("bigla_workspace_bytes", "bigla_fwd", "bigla_fwd_layout", "bigla_fwd_plan", "bigla_fwd_static_scratch", "locality_gate_fwd",
           "locality_gate_fwd_layout", "bigla_locality_workspace_bytes", "bigla_locality_fwd", "gate_producer_fwd",
           "gated_bigla_workspace_bytes", "gated_bigla_fwd",
           "bigla_bwd_workspace_bytes", "bigla_bwd", "bigla_bwd_plan",
           "gated_delta_workspace_bytes", "gated_delta_fwd", "gated_delta_bwd_workspace_bytes", "gated_delta_bwd",
           "gated_delta_step", "group_norm_workspace_bytes", "group_norm_act_fwd", "group_norm_bwd_workspace_bytes",
           "group_norm_act_bwd",
           "vig_status_str", "vig_last_hip_error", "vig_timing_enable",
           "vig_timing_collect", "vig_measure_alias_slabs")
KERNELS = {"segment_state": 0, "gate_lowrank": 1, "segment_out": 2, "recurrent": 3, "locality_gate": 4,
           "segment_out_general": 5, "gate_producer": 6, "slab": 7, "backward": 8,
           "gated_delta": 9, "gated_delta_backward": 10, "gated_delta_step": 11, "group_norm": 12,
           "group_norm_backward": 13}

_lib = None


class VigError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(message)
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libvig_bigla.so (built in-tree by `__graft_entry__.build()`); raise if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                              "at the repository root (there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.bigla_workspace_bytes.argtypes = [ci] * 6
        L.bigla_workspace_bytes.restype = sz
        L.bigla_fwd.argtypes = [vp] * 6 + [ci] * 6 + [vp, sz, vp]
        L.bigla_fwd.restype = ci
        L.bigla_fwd_layout.argtypes = [vp] * 6 + [ci] * 7 + [vp, sz, vp]
        L.bigla_fwd_layout.restype = ci
        L.bigla_fwd_plan.argtypes = [vp] * 6 + [ci] * 8 + [vp, sz, vp]
        L.bigla_fwd_plan.restype = ci
        L.bigla_fwd_static_scratch.argtypes = [vp] * 6 + [ci] * 7 + [vp]
        L.bigla_fwd_static_scratch.restype = ci
        L.locality_gate_fwd.argtypes = [vp] * 6 + [ci] * 6 + [vp]
        L.locality_gate_fwd.restype = ci
        L.locality_gate_fwd_layout.argtypes = [vp] * 6 + [ci] * 7 + [vp]
        L.locality_gate_fwd_layout.restype = ci
        L.bigla_locality_workspace_bytes.argtypes = [ci] * 7
        L.bigla_locality_workspace_bytes.restype = sz
        L.bigla_locality_fwd.argtypes = [vp] * 10 + [ci] * 9 + [vp, sz, vp]
        L.bigla_locality_fwd.restype = ci
        L.bigla_bwd_workspace_bytes.argtypes = [ci] * 6
        L.bigla_bwd_workspace_bytes.restype = sz
        L.bigla_bwd.argtypes = [vp] * 11 + [ci] * 7 + [vp, sz, vp]
        L.bigla_bwd.restype = ci
        L.bigla_bwd_plan.argtypes = [vp] * 11 + [ci] * 8 + [vp, sz, vp]
        L.bigla_bwd_plan.restype = ci
        L.gate_producer_fwd.argtypes = [vp] * 6 + [ci] * 5 + [ctypes.c_float, ci, ci, vp]
        L.gate_producer_fwd.restype = ci
        L.gated_bigla_workspace_bytes.argtypes = [ci] * 6
        L.gated_bigla_workspace_bytes.restype = sz
        L.gated_bigla_fwd.argtypes = [vp] * 10 + [ci] * 6 + [ctypes.c_float, ci, ci, ci, vp, sz, vp]
        L.gated_bigla_fwd.restype = ci
        L.gated_delta_workspace_bytes.argtypes = [ci] * 7
        L.gated_delta_workspace_bytes.restype = sz
        L.gated_delta_fwd.argtypes = [vp] * 8 + [ci] * 9 + [vp, sz, vp]
        L.gated_delta_fwd.restype = ci
        L.gated_delta_bwd_workspace_bytes.argtypes = [ci] * 7
        L.gated_delta_bwd_workspace_bytes.restype = sz
        L.gated_delta_bwd.argtypes = [vp] * 14 + [ci] * 9 + [vp, sz, vp]
        L.gated_delta_bwd.restype = ci
        L.gated_delta_step.argtypes = [vp] * 8 + [ci] * 7 + [vp]
        L.gated_delta_step.restype = ci
        L.group_norm_workspace_bytes.argtypes = [ci] * 5
        L.group_norm_workspace_bytes.restype = sz
        L.group_norm_act_fwd.argtypes = [vp] * 5 + [ci] * 4 + [ctypes.c_float, ci, ci, vp, sz, vp]
        L.group_norm_act_fwd.restype = ci
        L.group_norm_bwd_workspace_bytes.argtypes = [ci] * 5
        L.group_norm_bwd_workspace_bytes.restype = sz
        L.group_norm_act_bwd.argtypes = [vp] * 8 + [ci] * 6 + [vp, sz, vp]
        L.group_norm_act_bwd.restype = ci
        L.vig_status_str.argtypes = [ci]
        L.vig_status_str.restype = ctypes.c_char_p
        L.vig_last_hip_error.argtypes = []
        L.vig_last_hip_error.restype = ci
        L.vig_timing_enable.argtypes = [ci]
        L.vig_timing_enable.restype = ci
        L.vig_measure_alias_slabs.argtypes = [ci]
        L.vig_measure_alias_slabs.restype = ci
        L.vig_timing_collect.argtypes = [ci, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_long)]
        L.vig_timing_collect.restype = ci
        _lib = L
    return _lib


def status_str(status: int) -> str:
    return lib().vig_status_str(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != VIG_OK:
        msg = f"{what}: {status_str(status)}"
        if status == VIG_ERR_HIP:
            msg += f" (hipError_t {lib().vig_last_hip_error()})"
        raise VigError(status, msg)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return VIG_F32
    if t.dtype == torch.bfloat16:
        return VIG_BF16
    raise VigError(VIG_ERR_DTYPE, f"unsupported tensor dtype {t.dtype}")


def _dev(t: torch.Tensor, name: str, shape=None, like: torch.Tensor | None = None) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise VigError(VIG_ERR_NULL, f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise VigError(VIG_ERR_SHAPE, f"{name} must be contiguous")
    if shape is not None and t.shape != shape:  # torch.Size compares with tuples
        raise VigError(VIG_ERR_SHAPE, f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise VigError(VIG_ERR_DTYPE, f"{name} must match dtype/device of the other tensors")
    return t


class _SameDevice:
    """Stands in for torch.cuda.device where the tensors' device is the current one already."""

    def __enter__(self):
        return None

    def __exit__(self, *exc):
        return False


_SAME_DEVICE = _SameDevice()


def _on_device(device):
    """The tensors' device as the current one.  A small call is bound by what the host does for it: two calls on a
    64-token sequence took 21.3 us, 11.5 us of it kernels, and take 15.5 us without switching to the device that is
    the current one already and without a Stream object per call."""
    return _SAME_DEVICE if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _stream_ptr(device) -> int:
    # the raw handle: building a Stream object around it takes longer than the launch it is for
    return torch._C._cuda_getCurrentRawStream(device.index)


def bigla_workspace_bytes(B: int, H: int, L: int, dk: int, dv: int, dtype: int) -> int:
    return int(lib().bigla_workspace_bytes(B, H, L, dk, dv, dtype))


def _layout_code(layout) -> int:
    if layout not in LAYOUTS:
        raise VigError(VIG_ERR_LAYOUT, f"layout must be one of {sorted(LAYOUTS)}")
    return LAYOUTS[layout]


def bigla_fwd(q, k, v, g_fwd, g_bwd, out=None, workspace=None, layout="bhld", static_scratch=False, plan="auto"):
    """BiGLA forward (Section 4.2.1).  q,k,g_fwd,g_bwd: [B,H,L,dk]; v: [B,H,L,dv] -> out [B,H,L,dv]
    (layout "bhld"), or all of them token-major, [B,L,H,d] (layout "blhd").

    g_* are LOG forget gates (<= 0).  `workspace` is an optional uint8 GPU tensor of at least
    bigla_workspace_bytes(...) bytes; one is allocated with torch when absent.
    static_scratch=True calls bigla_fwd_static_scratch instead: the library's own per-GPU scratch
    array serves as workspace and, given `out`, nothing is allocated.  `plan` other than "auto" goes
    through bigla_fwd_plan ("four_wave", "wave_specialised" or "slab_sweep" kernels of the chunkwise path).
    """
    lay = _layout_code(layout)
    q = _dev(q, "q")
    if q.dim() != 4:
        raise VigError(VIG_ERR_SHAPE, "q must be 4-dimensional")
    if lay == VIG_LAYOUT_BHLD:
        B, H, L, dk = q.shape
    else:
        B, L, H, dk = q.shape
    k = _dev(k, "k", q.shape, q)
    g_fwd = _dev(g_fwd, "g_fwd", q.shape, q)
    g_bwd = _dev(g_bwd, "g_bwd", q.shape, q)
    v = _dev(v, "v", like=q)
    if v.dim() != 4 or tuple(v.shape[:3]) != tuple(q.shape[:3]):
        raise VigError(VIG_ERR_SHAPE, "v must have the leading dimensions of q")
    dv = v.shape[3]
    if out is None:
        out = torch.empty(tuple(v.shape), dtype=q.dtype, device=q.device)
    out = _dev(out, "out", tuple(v.shape), q)
    code = _dtype_code(q)
    if static_scratch:
        with _on_device(q.device):
            st = lib().bigla_fwd_static_scratch(q.data_ptr(), k.data_ptr(), v.data_ptr(), g_fwd.data_ptr(),
                                                g_bwd.data_ptr(), out.data_ptr(), B, H, L, dk, dv, code, lay,
                                                _stream_ptr(q.device))
        _check(st, "bigla_fwd_static_scratch")
        return out
    need = bigla_workspace_bytes(B, H, L, dk, dv, code)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    if plan not in FWD_PLANS:
        raise VigError(VIG_ERR_UNSUPPORTED, f"plan must be one of {sorted(FWD_PLANS)}")
    with _on_device(q.device):
        if plan != "auto":
            st = lib().bigla_fwd_plan(q.data_ptr(), k.data_ptr(), v.data_ptr(), g_fwd.data_ptr(), g_bwd.data_ptr(),
                                      out.data_ptr(), B, H, L, dk, dv, code, lay, FWD_PLANS[plan], ws_ptr, ws_bytes,
                                      _stream_ptr(q.device))
        elif lay == VIG_LAYOUT_BHLD:
            st = lib().bigla_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g_fwd.data_ptr(), g_bwd.data_ptr(),
                                 out.data_ptr(), B, H, L, dk, dv, code, ws_ptr, ws_bytes, _stream_ptr(q.device))
        else:
            st = lib().bigla_fwd_layout(q.data_ptr(), k.data_ptr(), v.data_ptr(), g_fwd.data_ptr(),
                                        g_bwd.data_ptr(), out.data_ptr(), B, H, L, dk, dv, code, lay, ws_ptr,
                                        ws_bytes, _stream_ptr(q.device))
    _check(st, "bigla_fwd")
    return out


def locality_gate_fwd(x, w, gate_logits, o_global, Hg: int, Wg: int, bias=None, out=None, layout="bhld"):
    """2D gating locality injection (Section 4.2.2).

    x, gate_logits, o_global: [B,H,Hg*Wg,dv] (layout "bhld") or [B,Hg*Wg,H,dv] (layout "blhd");
    w: [H*dv,3,3]; bias: [H*dv] or None -> out like x.
    """
    lay = _layout_code(layout)
    x = _dev(x, "x")
    if x.dim() != 4:
        raise VigError(VIG_ERR_SHAPE, "x must be 4-dimensional")
    if lay == VIG_LAYOUT_BHLD:
        B, H, L, dv = x.shape
    else:
        B, L, H, dv = x.shape
    if L != Hg * Wg:
        raise VigError(VIG_ERR_SHAPE, "x.shape[2] must equal Hg*Wg")
    w = _dev(w, "w", (H * dv, 3, 3), x)
    gate_logits = _dev(gate_logits, "gate_logits", x.shape, x)
    o_global = _dev(o_global, "o_global", x.shape, x)
    if bias is not None:
        bias = _dev(bias, "bias", (H * dv,), x)
    if out is None:
        out = torch.empty_like(x)
    out = _dev(out, "out", x.shape, x)
    with _on_device(x.device):
        bias_ptr = bias.data_ptr() if bias is not None else None
        if lay == VIG_LAYOUT_BHLD:
            st = lib().locality_gate_fwd(x.data_ptr(), w.data_ptr(), bias_ptr, gate_logits.data_ptr(),
                                         o_global.data_ptr(), out.data_ptr(), B, H, Hg, Wg, dv, _dtype_code(x),
                                         _stream_ptr(x.device))
        else:
            st = lib().locality_gate_fwd_layout(x.data_ptr(), w.data_ptr(), bias_ptr, gate_logits.data_ptr(),
                                                o_global.data_ptr(), out.data_ptr(), B, H, Hg, Wg, dv,
                                                _dtype_code(x), lay, _stream_ptr(x.device))
    _check(st, "locality_gate_fwd")
    return out


def bigla_locality_fwd(q, k, v, g_fwd, g_bwd, x, w, gate_logits, Hg: int, Wg: int, bias=None, out=None,
                       workspace=None, layout="bhld", plan="auto"):
    """Token mixer and locality blend in one call (Sections 4.2.1 and 4.2.2):
    out = G * DWConv3x3(x) + (1 - G) * BiGLA(q, k, v, g_fwd, g_bwd), G = sigmoid(gate_logits).
    Tensors as for bigla_fwd and locality_gate_fwd, L = Hg*Wg.  plan: "auto", "two_launches" or
    "fused_epilogue" (the blend inside the chunkwise output pass; bf16, dv = 64, dk = 64 or 32).
    """
    lay = _layout_code(layout)
    if plan not in PLANS:
        raise VigError(VIG_ERR_UNSUPPORTED, f"plan must be one of {sorted(PLANS)}")
    q = _dev(q, "q")
    if q.dim() != 4:
        raise VigError(VIG_ERR_SHAPE, "q must be 4-dimensional")
    if lay == VIG_LAYOUT_BHLD:
        B, H, L, dk = q.shape
    else:
        B, L, H, dk = q.shape
    if L != Hg * Wg:
        raise VigError(VIG_ERR_SHAPE, "the sequence length must equal Hg*Wg")
    k = _dev(k, "k", q.shape, q)
    g_fwd = _dev(g_fwd, "g_fwd", q.shape, q)
    g_bwd = _dev(g_bwd, "g_bwd", q.shape, q)
    v = _dev(v, "v", like=q)
    if v.dim() != 4 or tuple(v.shape[:3]) != tuple(q.shape[:3]):
        raise VigError(VIG_ERR_SHAPE, "v must have the leading dimensions of q")
    dv = v.shape[3]
    x = _dev(x, "x", v.shape, q)
    gate_logits = _dev(gate_logits, "gate_logits", v.shape, q)
    w = _dev(w, "w", (H * dv, 3, 3), q)
    if bias is not None:
        bias = _dev(bias, "bias", (H * dv,), q)
    if out is None:
        out = torch.empty(tuple(v.shape), dtype=q.dtype, device=q.device)
    out = _dev(out, "out", tuple(v.shape), q)
    code = _dtype_code(q)
    need = int(lib().bigla_locality_workspace_bytes(B, H, L, dk, dv, code, PLANS[plan]))
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    with _on_device(q.device):
        st = lib().bigla_locality_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g_fwd.data_ptr(), g_bwd.data_ptr(),
                                      x.data_ptr(), w.data_ptr(), bias.data_ptr() if bias is not None else None,
                                      gate_logits.data_ptr(), out.data_ptr(), B, H, Hg, Wg, dk, dv, code, lay,
                                      PLANS[plan], ws_ptr, ws_bytes, _stream_ptr(q.device))
    _check(st, "bigla_locality_fwd")
    return out


BWD_PLANS = {"auto": 0, "recurrent": 1}


def bigla_bwd(q, k, v, g_fwd, g_bwd, d_out, workspace=None, layout="bhld", plan="auto"):
    """Gradient of bigla_fwd (Section 4.2.1): returns (dq, dk, dv, dg_fwd, dg_bwd) for the output
    gradient d_out (shaped like v); tensors as for bigla_fwd.  plan: "auto" (bigla_bwd) or
    "recurrent" (bigla_bwd_plan with VIG_BWD_RECURRENT: the exact token-by-token kernels only)."""
    if plan not in BWD_PLANS:
        raise VigError(VIG_ERR_UNSUPPORTED, f"unknown plan {plan!r}")
    lay = _layout_code(layout)
    q = _dev(q, "q")
    if q.dim() != 4:
        raise VigError(VIG_ERR_SHAPE, "q must be 4-dimensional")
    if lay == VIG_LAYOUT_BHLD:
        B, H, L, dk = q.shape
    else:
        B, L, H, dk = q.shape
    k = _dev(k, "k", q.shape, q)
    g_fwd = _dev(g_fwd, "g_fwd", q.shape, q)
    g_bwd = _dev(g_bwd, "g_bwd", q.shape, q)
    v = _dev(v, "v", like=q)
    if v.dim() != 4 or tuple(v.shape[:3]) != tuple(q.shape[:3]):
        raise VigError(VIG_ERR_SHAPE, "v must have the leading dimensions of q")
    dv = v.shape[3]
    d_out = _dev(d_out, "d_out", v.shape, q)
    dq, dk_, dgf, dgb = (torch.empty_like(q) for _ in range(4))
    dv_ = torch.empty_like(v)
    code = _dtype_code(q)
    need = int(lib().bigla_bwd_workspace_bytes(B, H, L, dk, dv, code))
    if need == 0:
        raise VigError(VIG_ERR_UNSUPPORTED, "unsupported shape for bigla_bwd")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    with _on_device(q.device):
        args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), g_fwd.data_ptr(), g_bwd.data_ptr(), d_out.data_ptr(),
                dq.data_ptr(), dk_.data_ptr(), dv_.data_ptr(), dgf.data_ptr(), dgb.data_ptr(), B, H, L, dk, dv, code, lay)
        tail = (workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(q.device))
        if plan == "auto":
            st = lib().bigla_bwd(*args, *tail)
        else:
            st = lib().bigla_bwd_plan(*args, BWD_PLANS[plan], *tail)
    _check(st, "bigla_bwd")
    return dq, dk_, dv_, dgf, dgb


def gate_producer_fwd(x, w1, w2, H: int, dk: int, bias=None, tau: float = 16.0, layout="bhld", g_fwd=None,
                      g_bwd=None):
    """Direction-wise log forget gates (Section 3 gate; Eq. (BiGLA) lines 1-2).

    x: [B,L,D]; w1: [16,D] and w2: [2*H*dk,16] (linear-layer weight layout); bias: [2*H*dk] or None
    -> (g_fwd, g_bwd), each [B,H,L,dk] (layout "bhld") or [B,L,H,dk] ("blhd").
    """
    lay = _layout_code(layout)
    x = _dev(x, "x")
    if x.dim() != 3:
        raise VigError(VIG_ERR_SHAPE, "x must be [B,L,D]")
    B, L, D = x.shape
    w1 = _dev(w1, "w1", (16, D), x)
    w2 = _dev(w2, "w2", (2 * H * dk, 16), x)
    if bias is not None:
        bias = _dev(bias, "bias", (2 * H * dk,), x)
    shape = (B, H, L, dk) if lay == VIG_LAYOUT_BHLD else (B, L, H, dk)
    if g_fwd is None:
        g_fwd = torch.empty(shape, dtype=x.dtype, device=x.device)
    if g_bwd is None:
        g_bwd = torch.empty(shape, dtype=x.dtype, device=x.device)
    g_fwd = _dev(g_fwd, "g_fwd", shape, x)
    g_bwd = _dev(g_bwd, "g_bwd", shape, x)
    with _on_device(x.device):
        st = lib().gate_producer_fwd(x.data_ptr(), w1.data_ptr(), w2.data_ptr(),
                                     bias.data_ptr() if bias is not None else None, g_fwd.data_ptr(),
                                     g_bwd.data_ptr(), B, H, L, D, dk, float(tau), _dtype_code(x), lay,
                                     _stream_ptr(x.device))
    _check(st, "gate_producer_fwd")
    return g_fwd, g_bwd


def gated_bigla_fwd(x, w1, w2, q, k, v, bias=None, tau: float = 16.0, layout="bhld", plan="auto", out=None,
                    g_fwd=None, g_bwd=None, workspace=None):
    """gate_producer_fwd then bigla_fwd as one call (Section 3 gate; Eq. (BiGLA)): returns (out, g_fwd, g_bwd).

    plan "in_state_pass": the chunkwise state pass makes the gates itself from x W1; "separate": two launches.
    """
    lay = _layout_code(layout)
    if plan not in GATES_PLANS:
        raise VigError(VIG_ERR_UNSUPPORTED, f"plan must be one of {sorted(GATES_PLANS)}")
    q = _dev(q, "q")
    if q.dim() != 4:
        raise VigError(VIG_ERR_SHAPE, "q must be 4-dimensional")
    if lay == VIG_LAYOUT_BHLD:
        B, H, L, dk = q.shape
    else:
        B, L, H, dk = q.shape
    dv = v.shape[-1]
    x = _dev(x, "x", None, q)
    if x.dim() != 3 or x.shape[0] != B or x.shape[1] != L:
        raise VigError(VIG_ERR_SHAPE, "x must be [B,L,D]")
    D = x.shape[2]
    w1 = _dev(w1, "w1", (16, D), q)
    w2 = _dev(w2, "w2", (2 * H * dk, 16), q)
    if bias is not None:
        bias = _dev(bias, "bias", (2 * H * dk,), q)
    kshape = tuple(q.shape)
    vshape = kshape[:-1] + (dv,)
    k = _dev(k, "k", kshape, q)
    v = _dev(v, "v", vshape, q)
    g_fwd = torch.empty(kshape, dtype=q.dtype, device=q.device) if g_fwd is None else _dev(g_fwd, "g_fwd", kshape, q)
    g_bwd = torch.empty(kshape, dtype=q.dtype, device=q.device) if g_bwd is None else _dev(g_bwd, "g_bwd", kshape, q)
    out = torch.empty(vshape, dtype=q.dtype, device=q.device) if out is None else _dev(out, "out", vshape, q)
    code = _dtype_code(q)
    need = lib().gated_bigla_workspace_bytes(B, H, L, dk, dv, code)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    with _on_device(q.device):
        st = lib().gated_bigla_fwd(x.data_ptr(), w1.data_ptr(), w2.data_ptr(),
                                   bias.data_ptr() if bias is not None else None, q.data_ptr(), k.data_ptr(),
                                   v.data_ptr(), g_fwd.data_ptr(), g_bwd.data_ptr(), out.data_ptr(), B, H, L, D, dk,
                                   dv, float(tau), code, lay, GATES_PLANS[plan], workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(), _stream_ptr(q.device))
    _check(st, "gated_bigla_fwd")
    return out, g_fwd, g_bwd


def _as(t, name, shape, like, dtype, device: int):
    """_dev(t, name, shape, like) where like has that dtype and device index: a small call is bound by what the host does for it,
    and four comparisons take a third of what _dev takes."""
    try:
        if t.shape == shape and t.dtype is dtype and t.get_device() == device and t.is_contiguous():
            return t
    except AttributeError:
        pass
    return _dev(t, name, shape, like)


def _fp32(t, name, shape, like):
    """An fp32 tensor (a state, statistics) beside tensors of either dtype."""
    try:
        if t.shape == shape and t.dtype is torch.float32 and t.get_device() == like.get_device() and t.is_contiguous():
            return t  # (as in _as; like is a GPU tensor)
    except AttributeError:
        pass
    t = _dev(t, name, shape)
    if t.dtype != torch.float32 or t.device != like.device:
        raise VigError(VIG_ERR_DTYPE, f"{name} must be float32, on the device of the other tensors")
    return t


@functools.lru_cache(maxsize=256)
def _bytes(query: str, *sizes) -> int:
    """Workspace of a problem: a function of its sizes alone."""
    return int(getattr(lib(), query)(*sizes))


def _here(device):
    """_on_device for a tensor's device index."""
    return _SAME_DEVICE if torch._C._cuda_getDevice() == device else torch.cuda.device(device)


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _workspace(workspace, need: int, device):
    """(workspace, bytes): the caller's, or one allocated with torch where some is needed."""
    if workspace is None:
        return (torch.empty(need, dtype=torch.uint8, device=device), need) if need > 0 else (None, 0)
    workspace = _dev(workspace, "workspace")
    if workspace.device != device:
        raise VigError(VIG_ERR_DTYPE, "workspace must be on the device of the other tensors")
    return workspace, workspace.numel() * workspace.element_size()


def _delta_args(q, k, v, g, beta, layout, direction):
    lay = _layout_code(layout)
    if direction not in SCANS:
        raise VigError(VIG_ERR_UNSUPPORTED, f"direction must be one of {sorted(SCANS)}")
    q = _dev(q, "q")
    v = _dev(v, "v", like=q)
    if q.dim() != 4 or v.dim() != 4:
        raise VigError(VIG_ERR_SHAPE, "q and v must be 4-dimensional")
    if lay == VIG_LAYOUT_BHLD:
        (B, Hk, L, dk), H = q.shape, v.shape[1]
    else:
        (B, L, Hk, dk), H = q.shape, v.shape[2]
    dv = v.shape[3]
    heads = (B, H, L) if lay == VIG_LAYOUT_BHLD else (B, L, H)
    dtype, device = q.dtype, q.get_device()
    if v.shape != heads + (dv,):
        raise VigError(VIG_ERR_SHAPE, "v must have the batch and length of q")
    _as(k, "k", q.shape, q, dtype, device)
    _as(g, "g", heads, q, dtype, device)
    _as(beta, "beta", heads, q, dtype, device)
    return (B, H, Hk, L, dk, dv, _dtype_code(q)), lay, SCANS[direction]


def gated_delta_workspace_bytes(B: int, H: int, Hk: int, L: int, dk: int, dv: int, dtype: int) -> int:
    return int(lib().gated_delta_workspace_bytes(B, H, Hk, L, dk, dv, dtype))


def gated_delta_fwd(q, k, v, g, beta, initial_state=None, return_final_state=False, out=None, final_state=None,
                    workspace=None, layout="bhld", direction="forward"):
    """Gated delta rule: S_t = exp(g_t) (I - beta_t k_t^T k_t) S_{t-1} + beta_t k_t^T v_t, out_t = q_t S_t.

    q, k: [B,Hk,L,dk] with Hk dividing H; v: [B,H,L,dv]; g (log gates), beta: [B,H,L] (layout "bhld"), or [B,L,H,...]
    (layout "blhd"); initial_state: float32 [B,H,dk,dv] or None (zero).  direction "backward" scans from the last token.
    Returns out, or (out, final_state) where the final state is asked for (return_final_state, or a tensor for it, which
    may be initial_state); bf16 calls that ask for it work with more bits, and single values of out may differ in the last one.
    """
    sizes, lay, scan = _delta_args(q, k, v, g, beta, layout, direction)
    B, H, Hk, L, dk, dv, code = sizes
    if initial_state is not None:
        _fp32(initial_state, "initial_state", (B, H, dk, dv), q)
    if final_state is None and return_final_state:
        final_state = torch.empty((B, H, dk, dv), dtype=torch.float32, device=q.device)
    elif final_state is not None:
        _fp32(final_state, "final_state", (B, H, dk, dv), q)
    out = torch.empty_like(v) if out is None else _dev(out, "out", v.shape, q)
    workspace, ws_bytes = _workspace(workspace, _bytes("gated_delta_workspace_bytes", *sizes), q.device)
    with _here(q.get_device()):
        st = lib().gated_delta_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(),
                                   _ptr(initial_state), out.data_ptr(), _ptr(final_state), *sizes, lay, scan,
                                   _ptr(workspace), ws_bytes, torch._C._cuda_getCurrentRawStream(q.get_device()))
    _check(st, "gated_delta_fwd")
    return out if final_state is None else (out, final_state)


def gated_delta_bwd(q, k, v, g, beta, d_out, initial_state=None, d_final_state=None, workspace=None, layout="bhld",
                    direction="forward"):
    """Gradient of gated_delta_fwd: (dq, dk, dv, dg, dbeta) for the output gradient d_out (shaped like v) and, where given,
    the gradient d_final_state of the final state; with an initial_state its gradient follows as a sixth tensor (float32)."""
    sizes, lay, scan = _delta_args(q, k, v, g, beta, layout, direction)
    B, H, Hk, L, dk, dv, code = sizes
    _dev(d_out, "d_out", v.shape, q)
    d_initial = None
    if initial_state is not None:
        _fp32(initial_state, "initial_state", (B, H, dk, dv), q)
        d_initial = torch.empty_like(initial_state)
    if d_final_state is not None:
        _fp32(d_final_state, "d_final_state", (B, H, dk, dv), q)
    grads = tuple(torch.empty_like(t) for t in (q, k, v, g, beta))
    workspace, ws_bytes = _workspace(workspace, _bytes("gated_delta_bwd_workspace_bytes", *sizes), q.device)
    with _here(q.get_device()):
        st = lib().gated_delta_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(),
                                   _ptr(initial_state), d_out.data_ptr(), _ptr(d_final_state),
                                   *(t.data_ptr() for t in grads), _ptr(d_initial), *sizes, lay, scan, _ptr(workspace),
                                   ws_bytes, torch._C._cuda_getCurrentRawStream(q.get_device()))
    _check(st, "gated_delta_bwd")
    return grads if d_initial is None else grads + (d_initial,)


def gated_delta_step(q, k, v, g, beta, state, slots=None, out=None):
    """The gated delta rule for one token of each of B sequences; `state` (float32 [n_slots,H,dk,dv]) is updated in place.

    q, k: [B,Hk,dk]; v: [B,H,dv]; g, beta: [B,H]; slots: int32 [B], the state of each sequence (distinct; one outside
    [0, n_slots) marks a padded row, whose output is zero), or None (sequence b has state b) -> out [B,H,dv].
    """
    # (a small call is bound by what the host does for it: one expression first, and what is wrong only where it is false)
    try:
        (B, Hk, dk), (_, H, dv), n_slots = q.shape, v.shape, state.shape[0]
        dtype, device, heads = q.dtype, q.get_device(), (B, H)
        fits = (device >= 0 and k.shape == q.shape and v.shape[0] == B and g.shape == heads and beta.shape == heads
                and state.shape == (n_slots, H, dk, dv) and k.dtype is dtype and v.dtype is dtype and g.dtype is dtype
                and beta.dtype is dtype and state.dtype is torch.float32 and k.get_device() == device
                and v.get_device() == device and g.get_device() == device and beta.get_device() == device
                and state.get_device() == device and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
                and g.is_contiguous() and beta.is_contiguous() and state.is_contiguous())
    except (AttributeError, ValueError, IndexError):
        fits = False
    if not fits:
        q, state = _dev(q, "q"), _dev(state, "state")
        v = _dev(v, "v", like=q)
        if q.dim() != 3 or v.dim() != 3 or state.dim() != 4:
            raise VigError(VIG_ERR_SHAPE, "q and v must be 3-dimensional, state 4-dimensional")
        (B, Hk, dk), (_, H, dv), n_slots = q.shape, v.shape, state.shape[0]
        if v.shape[0] != B:
            raise VigError(VIG_ERR_SHAPE, "v must have the leading dimension of q")
        _dev(k, "k", q.shape, q)
        _dev(g, "g", (B, H), q)
        _dev(beta, "beta", (B, H), q)
        _fp32(state, "state", (n_slots, H, dk, dv), q)
        device = q.get_device()
    if slots is not None:
        _dev(slots, "slots", (B,))
        if slots.dtype != torch.int32 or slots.get_device() != device:
            raise VigError(VIG_ERR_DTYPE, "slots must be int32, on the device of the other tensors")
    out = torch.empty_like(v) if out is None else _dev(out, "out", v.shape, q)
    with _here(device):
        st = lib().gated_delta_step(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(),
                                    state.data_ptr(), _ptr(slots), out.data_ptr(), B, H, Hk, dk, dv, n_slots,
                                    _dtype_code(q), torch._C._cuda_getCurrentRawStream(device))
    _check(st, "gated_delta_step")
    return out


def _norm_args(x, groups, weight, bias, act):
    try:  # (as in gated_delta_step)
        channels, dtype, device, n = x.shape[-1:], x.dtype, x.get_device(), x.numel()
        fits = device >= 0 and n > 0 and x.dim() >= 2 and x.is_contiguous()
        if weight is not None:
            fits = (fits and weight.shape == channels and bias.shape == channels and weight.dtype is dtype and bias.dtype is dtype
                    and weight.get_device() == device and bias.get_device() == device and weight.is_contiguous()
                    and bias.is_contiguous())
    except (AttributeError, IndexError):
        fits = False
    if act not in ACTS:
        raise VigError(VIG_ERR_UNSUPPORTED, f"act must be one of {sorted(ACTS)}")
    if (weight is None) != (bias is None):
        raise VigError(VIG_ERR_NULL, "weight and bias come together")
    if not fits:
        _dev(x, "x")
        if x.dim() < 2:
            raise VigError(VIG_ERR_SHAPE, "x must be [B, ..., C]")
        if x.numel() == 0:
            raise VigError(VIG_ERR_SHAPE, "x has no elements")
        if weight is not None:
            _dev(weight, "weight", x.shape[-1:], x)
            _dev(bias, "bias", x.shape[-1:], x)
        n = x.numel()
    B, C = x.shape[0], x.shape[-1]
    return (B, n // (B * C), C, groups), _dtype_code(x), ACTS[act]


def group_norm_act_fwd(x, groups: int, weight=None, bias=None, eps: float = 1e-5, act="silu", out=None, stats=None,
                       workspace=None):
    """Channels-last group norm and activation: act((x - mean) / sqrt(var + eps) * weight + bias), the statistics over all
    positions (later ones too: for a norm of each token by itself x is [B L, 1, C]) and the C / groups channels of a group.
    x: [B, ..., C]; weight, bias: [C] or both None; act: "silu" or "none".
    Returns (out, stats), stats: float32 [B, groups, 2], mean and 1 / sqrt(var + eps), for group_norm_act_bwd."""
    sizes, code, act_code = _norm_args(x, groups, weight, bias, act)
    out = torch.empty_like(x) if out is None else _dev(out, "out", x.shape, x)
    if stats is None:
        stats = torch.empty(sizes[0], max(groups, 0), 2, dtype=torch.float32, device=x.device)
    else:
        _fp32(stats, "stats", (sizes[0], groups, 2), x)
    workspace, ws_bytes = _workspace(workspace, _bytes("group_norm_workspace_bytes", *sizes, code), x.device)
    with _here(x.get_device()):
        st = lib().group_norm_act_fwd(x.data_ptr(), _ptr(weight), _ptr(bias), out.data_ptr(), stats.data_ptr(), *sizes,
                                      float(eps), act_code, code, _ptr(workspace), ws_bytes, torch._C._cuda_getCurrentRawStream(x.get_device()))
    _check(st, "group_norm_act_fwd")
    return out, stats


def group_norm_act_bwd(x, d_out, stats, groups: int, weight=None, bias=None, act="silu", workspace=None):
    """Gradient of group_norm_act_fwd: (dx, d_weight, d_bias) for the output gradient d_out and the forward's stats
    (d_weight and d_bias are None without a weight)."""
    sizes, code, act_code = _norm_args(x, groups, weight, bias, act)
    _as(d_out, "d_out", x.shape, x, x.dtype, x.get_device())
    _fp32(stats, "stats", (sizes[0], groups, 2), x)
    dx = torch.empty_like(x)
    dw, db = (torch.empty_like(weight), torch.empty_like(bias)) if weight is not None else (None, None)
    workspace, ws_bytes = _workspace(workspace, _bytes("group_norm_bwd_workspace_bytes", *sizes, code), x.device)
    with _here(x.get_device()):
        st = lib().group_norm_act_bwd(x.data_ptr(), _ptr(weight), _ptr(bias), stats.data_ptr(), d_out.data_ptr(),
                                      dx.data_ptr(), _ptr(dw), _ptr(db), *sizes, act_code, code, _ptr(workspace), ws_bytes,
                                      torch._C._cuda_getCurrentRawStream(x.get_device()))
    _check(st, "group_norm_act_bwd")
    return dx, dw, db


def timing_enable(on: bool) -> None:
    """Start (and clear) or stop per-kernel HIP-event timing of this thread's launches."""
    _check(lib().vig_timing_enable(1 if on else 0), "vig_timing_enable")


def timing_collect(kernel: str):
    """(total milliseconds, launches) of one kernel since timing was enabled."""
    ms, n = ctypes.c_double(0.0), ctypes.c_long(0)
    _check(lib().vig_timing_collect(KERNELS[kernel], ctypes.byref(ms), ctypes.byref(n)), "vig_timing_collect")
    return ms.value, n.value


def measure_alias_slabs(on: bool) -> None:
    """Measurement aid: make every slab of the chunkwise forward kernels read slab 0's inputs."""
    _check(lib().vig_measure_alias_slabs(1 if on else 0), "vig_measure_alias_slabs")
