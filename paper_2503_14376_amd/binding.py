"""ctypes binding with the same names and argument order as include/tfla_mlstm.h."""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

EXP, SIG = 0, 1
F32, BF16 = 0, 1
FWD, BWD = 0, 1
NORM_RMS, NORM_LAYER = 0, 1
ACT_NONE, ACT_SILU, ACT_GELU, ACT_RELU = 0, 1, 2, 3

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "lib", "libtfla_mlstm.so")
_lib = None

EXPORTS = ("tfla_mlstm_fwd", "tfla_mlstm_bwd", "tfla_mlstm_step", "tfla_mlstm_workspace_bytes", "tfla_mlstm_check",
           "tfla_status_string", "tfla_version", "tfla_profile_enable", "tfla_profile_read",
           "tfla_profile_kernels", "tfla_mlstm_layer_fwd", "tfla_mlstm_layer_bwd", "tfla_mlstm_layer_workspace_bytes",
           "tfla_transfer_gain", "tfla_mlstm_layer_step", "tfla_tile_width", "tfla_mlstm_fwd_static",
           "tfla_static_scratch_bytes", "tfla_norm_workspace_bytes", "tfla_norm_fwd", "tfla_norm_bwd",
           "tfla_linear_workspace_bytes", "tfla_linear_fwd", "tfla_linear_bwd", "tfla_gated_workspace_bytes",
           "tfla_gated_fwd", "tfla_gated_bwd", "tfla_q8_quant", "tfla_norm_q8_fwd", "tfla_linear_q8_workspace_bytes",
           "tfla_linear_q8_fwd", "tfla_linear_q8_bwd", "tfla_gated_q8_workspace_bytes", "tfla_gated_q8_fwd", "tfla_gated_q8_bwd")


class TflaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed with status %d: %s" % (where, status, status_string(status)))


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libtfla_mlstm.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError("libtfla_mlstm.so is missing at %s: build it with "
                          "`python -m paper_2503_14376_amd.build` (there is no fallback path)" % _LIB_PATH)
    lib = ctypes.CDLL(_LIB_PATH)
    vp, fp, ci, cf, sz = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.tfla_mlstm_fwd.restype = ci
    lib.tfla_mlstm_fwd.argtypes = [vp, vp, vp, fp, fp, fp, fp, fp, ci, ci, ci, ci, ci, ci, ci, ci, cf,
                                   vp, fp, fp, fp, fp, fp, vp, sz, vp]
    lib.tfla_mlstm_fwd_static.restype = ci
    lib.tfla_mlstm_fwd_static.argtypes = [vp, vp, vp, fp, fp, fp, fp, fp, ci, ci, ci, ci, ci, ci, ci, ci, cf,
                                          vp, fp, fp, fp, fp, fp, vp]
    lib.tfla_static_scratch_bytes.restype = sz
    lib.tfla_static_scratch_bytes.argtypes = []
    lib.tfla_mlstm_bwd.restype = ci
    lib.tfla_mlstm_bwd.argtypes = [vp, vp, vp, fp, fp, fp, fp, fp, fp, fp, vp, fp, ci, ci, ci, ci, ci, ci, ci, ci, cf,
                                   vp, vp, vp, fp, fp, fp, vp, sz, vp, sz, vp]
    lib.tfla_mlstm_step.restype = ci
    lib.tfla_mlstm_step.argtypes = [vp, vp, vp, fp, fp, fp, fp, fp, ci, ci, ci, ci, ci, ci, cf, vp, fp, fp, fp, vp]
    lib.tfla_mlstm_layer_fwd.restype = ci
    lib.tfla_mlstm_layer_fwd.argtypes = [vp, vp, vp, fp, fp, vp, fp, fp, fp, fp, fp, ci, ci, ci, ci, ci, ci, ci, ci, cf,
                                         cf, ci, cf, vp, vp, fp, fp, fp, fp, fp, vp, sz, vp]
    lib.tfla_mlstm_layer_bwd.restype = ci
    lib.tfla_mlstm_layer_bwd.argtypes = [vp, vp, vp, fp, fp, vp, fp, fp, fp, fp, fp, vp, fp, fp, vp, fp,
                                         ci, ci, ci, ci, ci, ci, ci, ci, cf, cf, ci, cf,
                                         vp, vp, vp, fp, fp, vp, fp, fp, fp, vp, sz, vp, sz, vp]
    lib.tfla_mlstm_layer_workspace_bytes.restype = sz
    lib.tfla_mlstm_layer_workspace_bytes.argtypes = [ci] * 9
    lib.tfla_mlstm_layer_step.restype = ci
    lib.tfla_mlstm_layer_step.argtypes = [vp, vp, vp, fp, fp, vp, fp, fp, fp, fp, fp, ci, ci, ci, ci, ci, ci, cf, cf, ci, cf,
                                          vp, vp, fp, fp, fp, vp]
    lib.tfla_transfer_gain.restype = ci
    lib.tfla_transfer_gain.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, cf, fp, fp, vp]
    lib.tfla_mlstm_workspace_bytes.restype = sz
    lib.tfla_mlstm_workspace_bytes.argtypes = [ci] * 9
    lib.tfla_mlstm_check.restype = ci
    lib.tfla_mlstm_check.argtypes = [ci] * 9
    lib.tfla_status_string.restype = ctypes.c_char_p
    lib.tfla_status_string.argtypes = [ci]
    lib.tfla_version.restype = ci
    lib.tfla_profile_enable.restype = ci
    lib.tfla_profile_enable.argtypes = [ci]
    lib.tfla_profile_read.restype = ci
    lib.tfla_profile_read.argtypes = [ci, ctypes.c_char_p, ci, ctypes.POINTER(ctypes.c_double),
                                      ctypes.POINTER(ctypes.c_long)]
    lib.tfla_profile_kernels.restype = ci
    lib.tfla_tile_width.restype = ci
    lib.tfla_tile_width.argtypes = [ci]
    lib.tfla_norm_workspace_bytes.restype = sz
    lib.tfla_norm_workspace_bytes.argtypes = [ci] * 5
    lib.tfla_norm_fwd.restype = ci
    lib.tfla_norm_fwd.argtypes = [vp, fp, fp, ci, ci, ci, ci, cf, vp, fp, fp, vp]
    lib.tfla_norm_bwd.restype = ci
    lib.tfla_norm_bwd.argtypes = [vp, vp, fp, fp, fp, vp, ci, ci, ci, ci, vp, fp, fp, vp, sz, vp]
    lib.tfla_linear_workspace_bytes.restype = sz
    lib.tfla_linear_workspace_bytes.argtypes = [ci] * 7
    lib.tfla_linear_fwd.restype = ci
    lib.tfla_linear_fwd.argtypes = [vp, vp, fp, vp, ci, ci, ci, ci, ci, vp, vp, vp, sz, vp]
    lib.tfla_linear_bwd.restype = ci
    lib.tfla_linear_bwd.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, vp, vp, fp, vp, sz, vp]
    lib.tfla_gated_workspace_bytes.restype = sz
    lib.tfla_gated_workspace_bytes.argtypes = [ci] * 7
    lib.tfla_gated_fwd.restype = ci
    lib.tfla_gated_fwd.argtypes = [vp, vp, vp, fp, fp, ci, ci, ci, ci, ci, vp, vp, vp, vp, sz, vp]
    lib.tfla_gated_bwd.restype = ci
    lib.tfla_gated_bwd.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, vp, vp, vp, fp, fp, vp, sz, vp]
    lib.tfla_q8_quant.restype = ci
    lib.tfla_q8_quant.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp, vp]
    lib.tfla_norm_q8_fwd.restype = ci
    lib.tfla_norm_q8_fwd.argtypes = [vp, fp, fp, vp, ci, ci, ci, ci, cf, vp, vp, vp, vp, fp, fp, vp]
    lib.tfla_linear_q8_workspace_bytes.restype = sz
    lib.tfla_linear_q8_workspace_bytes.argtypes = [ci] * 6
    lib.tfla_linear_q8_fwd.restype = ci
    lib.tfla_linear_q8_fwd.argtypes = [vp, vp, vp, vp, fp, vp, ci, ci, ci, ci, vp, vp, vp, sz, vp]
    lib.tfla_linear_q8_bwd.restype = ci
    lib.tfla_linear_q8_bwd.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, fp, vp, sz, vp]
    lib.tfla_gated_q8_workspace_bytes.restype = sz
    lib.tfla_gated_q8_workspace_bytes.argtypes = [ci] * 6
    lib.tfla_gated_q8_fwd.restype = ci
    lib.tfla_gated_q8_fwd.argtypes = [vp, vp, vp, vp, vp, vp, fp, fp, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.tfla_gated_q8_bwd.restype = ci
    lib.tfla_gated_q8_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp, fp, fp, vp, sz, vp]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().tfla_status_string(int(status)).decode()


def workspace_bytes(direction, B, NH, T, dqk, dhv, chunk, variant, dtype) -> int:
    return int(load_library().tfla_mlstm_workspace_bytes(direction, B, NH, T, dqk, dhv, chunk, variant, dtype))


def layer_workspace_bytes(direction, B, NH, T, dqk, dhv, chunk, variant, dtype) -> int:
    return int(load_library().tfla_mlstm_layer_workspace_bytes(direction, B, NH, T, dqk, dhv, chunk, variant, dtype))


def check(direction, B, NH, T, dqk, dhv, chunk, variant, dtype) -> int:
    return int(load_library().tfla_mlstm_check(direction, B, NH, T, dqk, dhv, chunk, variant, dtype))


def tile_width(width: int) -> None:
    """Output-column block of the bf16 tiled kernels for tile-size sweeps: 0 = automatic, 64, 128 (256 = automatic)."""
    rc = load_library().tfla_tile_width(int(width))
    if rc != 0:
        raise TflaError(rc, "tfla_tile_width")


def profile_enable(max_launches: int) -> None:
    rc = load_library().tfla_profile_enable(int(max_launches))
    if rc != 0:
        raise TflaError(rc, "tfla_profile_enable")


def profile_read() -> Dict[str, Dict[str, float]]:
    """Per-kernel-family totals since tfla_profile_enable: {name: {ms, launches}}."""
    lib = load_library()
    out = {}
    for kidx in range(lib.tfla_profile_kernels()):
        name = ctypes.create_string_buffer(64)
        ms, n = ctypes.c_double(0.0), ctypes.c_long(0)
        lib.tfla_profile_read(kidx, name, 64, ctypes.byref(ms), ctypes.byref(n))
        out[name.value.decode()] = {"ms": ms.value, "launches": n.value}
    return out


# A generation step is a call of some ten microseconds on the GPU, so what the binding does per argument counts: pointers
# and the stream go to ctypes as plain integers (the argument types turn them into pointers), shapes are compared as they
# are (one sequence of 8 heads 256 / 512, mlstm_layer_step in a loop: 17 us per step with a ctypes object per pointer and
# a stream object and two tuples per check, 13 us without).
def _ptr(t):
    return None if t is None else t.data_ptr()


def _torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == BF16 else torch.float32


def _stream_handle(stream=None):
    if stream is not None:
        return stream.cuda_stream
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # the current stream without a stream object around it
    return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())


# Memory and streams.  A call on an explicit stream is the call on the current stream with that one made current, so that new memory comes
# from its pool, where a block that was dropped before has had its last use in the stream's order.  (From the pool of the stream that the
# caller works on, the block of a tensor dropped a moment ago could come back while work queued there still reads it.)  The caller drops
# results on its own stream, which is recorded on them.  The call's other tensors may belong to any stream: the call's own is recorded on
# them, so that none is handed out again before the call has run.
def _within(call, stream, args):
    """call(**args), args with stream among them, on `stream`"""
    import torch
    if not hasattr(stream, "device"):       # (anything with a handle will do)
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    device = stream.device.index
    given = [t for t in (*args.values(), *(args.get("out") or {}).values()) if hasattr(t, "record_stream")]
    for t in given:
        if t.get_device() not in (device, -1):
            raise ValueError("the stream is one of cuda:%d, a tensor is on %s" % (device, t.device))
    args["stream"] = None
    before = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        result = call(**args)
    for t in given:
        if t.is_cuda:
            t.record_stream(stream)
    for t in result.values() if isinstance(result, dict) else result:
        if getattr(t, "is_cuda", False):
            t.record_stream(before)
    return result


def _want(t, dtype, shape, name):
    """shape: a tuple"""
    if t is None:
        return
    if not t.is_cuda or not t.is_contiguous() or t.dtype != dtype or t.shape != shape:
        raise ValueError("%s must be a contiguous device tensor of dtype %s and shape %s (got %s %s)"
                         % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))


def mlstm_fwd(q, k, v, i_pre, f_pre, C0=None, n0=None, m0=None, chunk=256, variant=EXP, eps=1e-6,
              return_state=True, workspace=None, stream=None, out: Optional[Dict] = None) -> Dict:
    """tfla_mlstm_fwd on torch device tensors.  q,k: (B,NH,T,dqk); v: (B,NH,T,dhv) in bf16 or
    fp32; gates fp32 (B,NH,T).  Returns a dict with H, Cn, nn, mn, n_out, m_out."""
    if stream is not None:
        return _within(mlstm_fwd, stream, locals())
    import torch
    lib = load_library()
    B, NH, T, dqk = q.shape
    dhv = v.shape[-1]
    dtype = BF16 if q.dtype == torch.bfloat16 else F32
    td, f32 = _torch_dtype(dtype), torch.float32
    _want(q, td, (B, NH, T, dqk), "q"); _want(k, td, (B, NH, T, dqk), "k"); _want(v, td, (B, NH, T, dhv), "v")
    _want(i_pre, f32, (B, NH, T), "i_pre"); _want(f_pre, f32, (B, NH, T), "f_pre")
    _want(C0, f32, (B, NH, dqk, dhv), "C0"); _want(n0, f32, (B, NH, dqk), "n0"); _want(m0, f32, (B, NH), "m0")
    dev = q.device
    o = out if out is not None else {}
    if "H" not in o:
        o["H"] = torch.empty((B, NH, T, dhv), dtype=td, device=dev)
    if return_state and "Cn" not in o:
        o["Cn"] = torch.empty((B, NH, dqk, dhv), dtype=f32, device=dev)
        o["nn"] = torch.empty((B, NH, dqk), dtype=f32, device=dev)
        o["mn"] = torch.empty((B, NH), dtype=f32, device=dev)
    if "n_out" not in o:
        o["n_out"] = torch.empty((B, NH, T), dtype=f32, device=dev)
        o["m_out"] = torch.empty((B, NH, T), dtype=f32, device=dev)
    need = workspace_bytes(FWD, B, NH, T, dqk, dhv, chunk, variant, dtype)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    rc = lib.tfla_mlstm_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(i_pre), _ptr(f_pre), _ptr(C0), _ptr(n0), _ptr(m0),
                            B, NH, T, dqk, dhv, int(chunk), int(variant), dtype, float(eps),
                            _ptr(o["H"]), _ptr(o.get("Cn")), _ptr(o.get("nn")), _ptr(o.get("mn")),
                            _ptr(o["n_out"]), _ptr(o["m_out"]),
                            _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle())
    if rc != 0:
        raise TflaError(rc, "tfla_mlstm_fwd")
    o["workspace"] = workspace
    return o


def static_scratch_bytes() -> int:
    return int(load_library().tfla_static_scratch_bytes())


def mlstm_fwd_static(q, k, v, i_pre, f_pre, C0=None, n0=None, m0=None, chunk=256, variant=EXP, eps=1e-6, stream=None,
                     out: Optional[Dict] = None) -> Dict:
    """tfla_mlstm_fwd_static on torch device tensors: the forward pass on the library's own static scratch memory.
    `out` must hold every output tensor (H, Cn, nn, mn, n_out, m_out; the state and per-step entries may be
    missing = not wanted): this wrapper allocates nothing either."""
    if stream is not None:
        return _within(mlstm_fwd_static, stream, locals())
    import torch
    lib = load_library()
    B, NH, T, dqk = q.shape
    dhv = v.shape[-1]
    dtype = BF16 if q.dtype == torch.bfloat16 else F32
    td, f32 = _torch_dtype(dtype), torch.float32
    _want(q, td, (B, NH, T, dqk), "q"); _want(k, td, (B, NH, T, dqk), "k"); _want(v, td, (B, NH, T, dhv), "v")
    _want(i_pre, f32, (B, NH, T), "i_pre"); _want(f_pre, f32, (B, NH, T), "f_pre")
    _want(C0, f32, (B, NH, dqk, dhv), "C0"); _want(n0, f32, (B, NH, dqk), "n0"); _want(m0, f32, (B, NH), "m0")
    if out is None or "H" not in out:
        raise ValueError("mlstm_fwd_static writes into caller-provided tensors: pass out={'H': ..., ...}")
    o = out
    _want(o["H"], td, (B, NH, T, dhv), "H"); _want(o.get("Cn"), f32, (B, NH, dqk, dhv), "Cn")
    _want(o.get("nn"), f32, (B, NH, dqk), "nn"); _want(o.get("mn"), f32, (B, NH), "mn")
    _want(o.get("n_out"), f32, (B, NH, T), "n_out"); _want(o.get("m_out"), f32, (B, NH, T), "m_out")
    rc = lib.tfla_mlstm_fwd_static(_ptr(q), _ptr(k), _ptr(v), _ptr(i_pre), _ptr(f_pre), _ptr(C0), _ptr(n0), _ptr(m0),
                                   B, NH, T, dqk, dhv, int(chunk), int(variant), dtype, float(eps),
                                   _ptr(o["H"]), _ptr(o.get("Cn")), _ptr(o.get("nn")), _ptr(o.get("mn")),
                                   _ptr(o.get("n_out")), _ptr(o.get("m_out")), _stream_handle())
    if rc != 0:
        raise TflaError(rc, "tfla_mlstm_fwd_static")
    return o


def mlstm_bwd(q, k, v, i_pre, f_pre, dH, n_out=None, m_out=None, C0=None, n0=None, m0=None, dCn=None,
              chunk=256, variant=EXP, eps=1e-6, want_dC0=True, workspace=None, stream=None,
              out: Optional[Dict] = None, fwd_workspace=None) -> Dict:
    """tfla_mlstm_bwd on torch device tensors.  Returns dq, dk, dv, d_i_pre, d_f_pre, dC0.
    fwd_workspace: the (untouched) workspace tensor of the matching mlstm_fwd call, or None to
    recompute gates and chunk states."""
    if stream is not None:
        return _within(mlstm_bwd, stream, locals())
    import torch
    lib = load_library()
    B, NH, T, dqk = q.shape
    dhv = v.shape[-1]
    dtype = BF16 if q.dtype == torch.bfloat16 else F32
    td, f32 = _torch_dtype(dtype), torch.float32
    _want(q, td, (B, NH, T, dqk), "q"); _want(k, td, (B, NH, T, dqk), "k"); _want(v, td, (B, NH, T, dhv), "v")
    _want(dH, td, (B, NH, T, dhv), "dH")
    _want(i_pre, f32, (B, NH, T), "i_pre"); _want(f_pre, f32, (B, NH, T), "f_pre")
    _want(n_out, f32, (B, NH, T), "n_out"); _want(m_out, f32, (B, NH, T), "m_out")
    _want(C0, f32, (B, NH, dqk, dhv), "C0"); _want(n0, f32, (B, NH, dqk), "n0"); _want(m0, f32, (B, NH), "m0")
    _want(dCn, f32, (B, NH, dqk, dhv), "dCn")
    dev = q.device
    o = out if out is not None else {}
    if "dq" not in o:
        o["dq"] = torch.empty_like(q); o["dk"] = torch.empty_like(k); o["dv"] = torch.empty_like(v)
        o["d_i_pre"] = torch.empty((B, NH, T), dtype=f32, device=dev)
        o["d_f_pre"] = torch.empty((B, NH, T), dtype=f32, device=dev)
    if want_dC0 and "dC0" not in o:
        o["dC0"] = torch.empty((B, NH, dqk, dhv), dtype=f32, device=dev)
    need = workspace_bytes(BWD, B, NH, T, dqk, dhv, chunk, variant, dtype)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    rc = lib.tfla_mlstm_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(i_pre), _ptr(f_pre), _ptr(C0), _ptr(n0), _ptr(m0),
                            _ptr(n_out), _ptr(m_out), _ptr(dH), _ptr(dCn),
                            B, NH, T, dqk, dhv, int(chunk), int(variant), dtype, float(eps),
                            _ptr(o["dq"]), _ptr(o["dk"]), _ptr(o["dv"]), _ptr(o["d_i_pre"]), _ptr(o["d_f_pre"]),
                            _ptr(o.get("dC0")),
                            _ptr(fwd_workspace), 0 if fwd_workspace is None else fwd_workspace.numel(),
                            _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle())
    if rc != 0:
        raise TflaError(rc, "tfla_mlstm_bwd")
    o["workspace"] = workspace
    return o


def mlstm_step(q, k, v, i_pre, f_pre, C, n=None, m=None, variant=EXP, eps=1e-6, stream=None,
               out: Optional[Dict] = None, inplace_C: bool = False) -> Dict:
    """tfla_mlstm_step on torch device tensors.  q, k: (B,NH,dqk); v: (B,NH,dhv); i_pre, f_pre: (B,NH);
    C: (B,NH,dqk,dhv) fp32, n: (B,NH,dqk), m: (B,NH).  Returns h and the new state C, n, m."""
    if stream is not None:
        return _within(mlstm_step, stream, locals())
    import torch
    lib = load_library()
    B, NH, dqk = q.shape
    dhv = v.shape[-1]
    dtype = BF16 if q.dtype == torch.bfloat16 else F32
    td, f32 = _torch_dtype(dtype), torch.float32
    _want(q, td, (B, NH, dqk), "q"); _want(k, td, (B, NH, dqk), "k"); _want(v, td, (B, NH, dhv), "v")
    _want(i_pre, f32, (B, NH), "i_pre"); _want(f_pre, f32, (B, NH), "f_pre")
    _want(C, f32, (B, NH, dqk, dhv), "C"); _want(n, f32, (B, NH, dqk), "n"); _want(m, f32, (B, NH), "m")
    dev = q.device
    o = out if out is not None else {}
    if "h" not in o:
        o["h"] = torch.empty((B, NH, dhv), dtype=td, device=dev)
    if "C" not in o:
        o["C"] = C if inplace_C else torch.empty_like(C)
    if "n" not in o:
        o["n"] = torch.empty((B, NH, dqk), dtype=f32, device=dev)
        o["m"] = torch.empty((B, NH), dtype=f32, device=dev)
    rc = lib.tfla_mlstm_step(_ptr(q), _ptr(k), _ptr(v), _ptr(i_pre), _ptr(f_pre), _ptr(C), _ptr(n), _ptr(m),
                             B, NH, dqk, dhv, int(variant), dtype, float(eps),
                             _ptr(o["h"]), _ptr(o["C"]), _ptr(o["n"]), _ptr(o["m"]), _stream_handle())
    if rc != 0:
        raise TflaError(rc, "tfla_mlstm_step")
    return o


def mlstm_layer_fwd(q, k, v, i_pre, f_pre, o_pre=None, gamma=None, beta=None, C0=None, n0=None, m0=None, chunk=256,
                    variant=EXP, eps=1e-6, gate_softcap=0.0, norm_kind=NORM_RMS, norm_eps=1e-6, return_state=True,
                    workspace=None, stream=None, out: Optional[Dict] = None) -> Dict:
    """tfla_mlstm_layer_fwd on torch device tensors: soft-capped gates, cell, multi-head norm, output gate.
    o_pre: (B,NH,T,dhv) like v or None; gamma, beta: (NH,dhv) fp32 or None.  Returns Y, H (cell output), the
    final state, n_out, m_out and the workspace."""
    if stream is not None:
        return _within(mlstm_layer_fwd, stream, locals())
    import torch
    lib = load_library()
    B, NH, T, dqk = q.shape
    dhv = v.shape[-1]
    dtype = BF16 if q.dtype == torch.bfloat16 else F32
    td, f32 = _torch_dtype(dtype), torch.float32
    _want(q, td, (B, NH, T, dqk), "q"); _want(k, td, (B, NH, T, dqk), "k"); _want(v, td, (B, NH, T, dhv), "v")
    _want(i_pre, f32, (B, NH, T), "i_pre"); _want(f_pre, f32, (B, NH, T), "f_pre")
    _want(o_pre, td, (B, NH, T, dhv), "o_pre"); _want(gamma, f32, (NH, dhv), "gamma"); _want(beta, f32, (NH, dhv), "beta")
    _want(C0, f32, (B, NH, dqk, dhv), "C0"); _want(n0, f32, (B, NH, dqk), "n0"); _want(m0, f32, (B, NH), "m0")
    dev = q.device
    o = out if out is not None else {}
    if "Y" not in o:
        o["Y"] = torch.empty((B, NH, T, dhv), dtype=td, device=dev)
        o["H"] = torch.empty((B, NH, T, dhv), dtype=td, device=dev)
    if return_state and "Cn" not in o:
        o["Cn"] = torch.empty((B, NH, dqk, dhv), dtype=f32, device=dev)
        o["nn"] = torch.empty((B, NH, dqk), dtype=f32, device=dev)
        o["mn"] = torch.empty((B, NH), dtype=f32, device=dev)
    if "n_out" not in o:
        o["n_out"] = torch.empty((B, NH, T), dtype=f32, device=dev)
        o["m_out"] = torch.empty((B, NH, T), dtype=f32, device=dev)
    need = layer_workspace_bytes(FWD, B, NH, T, dqk, dhv, chunk, variant, dtype)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    rc = lib.tfla_mlstm_layer_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(i_pre), _ptr(f_pre), _ptr(o_pre), _ptr(gamma), _ptr(beta),
                                  _ptr(C0), _ptr(n0), _ptr(m0), B, NH, T, dqk, dhv, int(chunk), int(variant), dtype,
                                  float(eps), float(gate_softcap), int(norm_kind), float(norm_eps),
                                  _ptr(o["Y"]), _ptr(o["H"]), _ptr(o.get("Cn")), _ptr(o.get("nn")), _ptr(o.get("mn")),
                                  _ptr(o["n_out"]), _ptr(o["m_out"]),
                                  _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle())
    if rc != 0:
        raise TflaError(rc, "tfla_mlstm_layer_fwd")
    o["workspace"] = workspace
    return o


def mlstm_layer_bwd(q, k, v, i_pre, f_pre, H, dY, o_pre=None, gamma=None, beta=None, n_out=None, m_out=None, C0=None,
                    n0=None, m0=None, dCn=None, chunk=256, variant=EXP, eps=1e-6, gate_softcap=0.0, norm_kind=NORM_RMS,
                    norm_eps=1e-6, want_dC0=True, workspace=None, stream=None, out: Optional[Dict] = None,
                    fwd_workspace=None) -> Dict:
    """tfla_mlstm_layer_bwd on torch device tensors.  Returns dq, dk, dv, d_i_pre, d_f_pre, do_pre (if o_pre is
    given), dgamma, dbeta, dC0."""
    if stream is not None:
        return _within(mlstm_layer_bwd, stream, locals())
    import torch
    lib = load_library()
    B, NH, T, dqk = q.shape
    dhv = v.shape[-1]
    dtype = BF16 if q.dtype == torch.bfloat16 else F32
    td, f32 = _torch_dtype(dtype), torch.float32
    _want(q, td, (B, NH, T, dqk), "q"); _want(k, td, (B, NH, T, dqk), "k"); _want(v, td, (B, NH, T, dhv), "v")
    _want(H, td, (B, NH, T, dhv), "H"); _want(dY, td, (B, NH, T, dhv), "dY"); _want(o_pre, td, (B, NH, T, dhv), "o_pre")
    _want(gamma, f32, (NH, dhv), "gamma"); _want(beta, f32, (NH, dhv), "beta")
    _want(i_pre, f32, (B, NH, T), "i_pre"); _want(f_pre, f32, (B, NH, T), "f_pre")
    _want(n_out, f32, (B, NH, T), "n_out"); _want(m_out, f32, (B, NH, T), "m_out")
    _want(C0, f32, (B, NH, dqk, dhv), "C0"); _want(n0, f32, (B, NH, dqk), "n0"); _want(m0, f32, (B, NH), "m0")
    _want(dCn, f32, (B, NH, dqk, dhv), "dCn")
    dev = q.device
    o = out if out is not None else {}
    if "dq" not in o:
        o["dq"] = torch.empty_like(q); o["dk"] = torch.empty_like(k); o["dv"] = torch.empty_like(v)
        o["d_i_pre"] = torch.empty((B, NH, T), dtype=f32, device=dev)
        o["d_f_pre"] = torch.empty((B, NH, T), dtype=f32, device=dev)
        o["dgamma"] = torch.empty((NH, dhv), dtype=f32, device=dev)
        o["dbeta"] = torch.empty((NH, dhv), dtype=f32, device=dev)
        if o_pre is not None:
            o["do_pre"] = torch.empty_like(o_pre)
    if want_dC0 and "dC0" not in o:
        o["dC0"] = torch.empty((B, NH, dqk, dhv), dtype=f32, device=dev)
    need = layer_workspace_bytes(BWD, B, NH, T, dqk, dhv, chunk, variant, dtype)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    rc = lib.tfla_mlstm_layer_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(i_pre), _ptr(f_pre), _ptr(o_pre), _ptr(gamma), _ptr(beta),
                                  _ptr(C0), _ptr(n0), _ptr(m0), _ptr(H), _ptr(n_out), _ptr(m_out), _ptr(dY), _ptr(dCn),
                                  B, NH, T, dqk, dhv, int(chunk), int(variant), dtype, float(eps), float(gate_softcap),
                                  int(norm_kind), float(norm_eps),
                                  _ptr(o["dq"]), _ptr(o["dk"]), _ptr(o["dv"]), _ptr(o["d_i_pre"]), _ptr(o["d_f_pre"]),
                                  _ptr(o.get("do_pre")), _ptr(o.get("dgamma")), _ptr(o.get("dbeta")), _ptr(o.get("dC0")),
                                  _ptr(fwd_workspace), 0 if fwd_workspace is None else fwd_workspace.numel(),
                                  _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream_handle())
    if rc != 0:
        raise TflaError(rc, "tfla_mlstm_layer_bwd")
    o["workspace"] = workspace
    return o


def mlstm_layer_step(q, k, v, i_pre, f_pre, C, n=None, m=None, o_pre=None, gamma=None, beta=None, variant=EXP, eps=1e-6,
                     gate_softcap=0.0, norm_kind=NORM_RMS, norm_eps=1e-6, stream=None, out: Optional[Dict] = None,
                     inplace_C: bool = False) -> Dict:
    """tfla_mlstm_layer_step on torch device tensors: mlstm_step with soft-capped gates, then norm and output gate.
    o_pre: (B,NH,dhv) like v or None.  Returns y, h (cell output) and the new state C, n, m."""
    if stream is not None:
        return _within(mlstm_layer_step, stream, locals())
    import torch
    lib = load_library()
    B, NH, dqk = q.shape
    dhv = v.shape[-1]
    dtype = BF16 if q.dtype == torch.bfloat16 else F32
    td, f32 = _torch_dtype(dtype), torch.float32
    _want(q, td, (B, NH, dqk), "q"); _want(k, td, (B, NH, dqk), "k"); _want(v, td, (B, NH, dhv), "v")
    _want(o_pre, td, (B, NH, dhv), "o_pre"); _want(gamma, f32, (NH, dhv), "gamma"); _want(beta, f32, (NH, dhv), "beta")
    _want(i_pre, f32, (B, NH), "i_pre"); _want(f_pre, f32, (B, NH), "f_pre")
    _want(C, f32, (B, NH, dqk, dhv), "C"); _want(n, f32, (B, NH, dqk), "n"); _want(m, f32, (B, NH), "m")
    dev = q.device
    o = out if out is not None else {}
    if "y" not in o:
        o["y"] = torch.empty((B, NH, dhv), dtype=td, device=dev)
        o["h"] = torch.empty((B, NH, dhv), dtype=td, device=dev)
    if "C" not in o:
        o["C"] = C if inplace_C else torch.empty_like(C)
    if "n" not in o:
        o["n"] = torch.empty((B, NH, dqk), dtype=f32, device=dev)
        o["m"] = torch.empty((B, NH), dtype=f32, device=dev)
    rc = lib.tfla_mlstm_layer_step(_ptr(q), _ptr(k), _ptr(v), _ptr(i_pre), _ptr(f_pre), _ptr(o_pre), _ptr(gamma), _ptr(beta),
                                   _ptr(C), _ptr(n), _ptr(m), B, NH, dqk, dhv, int(variant), dtype, float(eps),
                                   float(gate_softcap), int(norm_kind), float(norm_eps), _ptr(o["y"]), _ptr(o["h"]),
                                   _ptr(o["C"]), _ptr(o["n"]), _ptr(o["m"]), _stream_handle())
    if rc != 0:
        raise TflaError(rc, "tfla_mlstm_layer_step")
    return o


def transfer_gain(h, v, norm_kind=NORM_RMS, norm_eps=1e-6, stream=None):
    """tfla_transfer_gain on torch device tensors h, v (B,NH,T,dhv).  Returns (g_before, g_after), each (B,NH) fp32."""
    if stream is not None:
        return _within(transfer_gain, stream, locals())
    import torch
    lib = load_library()
    B, NH, T, dhv = h.shape
    dtype = BF16 if h.dtype == torch.bfloat16 else F32
    td = _torch_dtype(dtype)
    _want(h, td, (B, NH, T, dhv), "h"); _want(v, td, (B, NH, T, dhv), "v")
    gb = torch.empty((B, NH), dtype=torch.float32, device=h.device)
    ga = torch.empty((B, NH), dtype=torch.float32, device=h.device)
    rc = lib.tfla_transfer_gain(_ptr(h), _ptr(v), B, NH, T, dhv, dtype, int(norm_kind), float(norm_eps), _ptr(gb), _ptr(ga),
                                _stream_handle())
    if rc != 0:
        raise TflaError(rc, "tfla_transfer_gain")
    return gb, ga


# ---- the rest of a residual block: norm over the model's columns, linear projection, gated projection pair --------------
# `out` belongs to one sequence of calls: it holds the outputs and the workspace of the last, which the next writes again.  Calls that share
# it have to be ordered when they run on different streams, and a graph that was captured with it needs it kept.
# These calls are the shortest of all while generating, so they do little per argument: outputs and the workspace that `out`
# holds from the call before are taken after a check of type and shape, torch's names are looked up once, and the current
# stream is asked for without an object around it (one token, norm_fwd in a loop: 7.0 us per call without these, 6.2 with).
# Every tensor of a call is on the device of its first, whose current stream takes the launch, and that device is made current for it: the
# handle of a default stream is 0 on every device and means the current one's.
_torch_names = None


def _torch_types():
    global _torch_names
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        def raw(device):
            return torch.cuda.current_stream(device).cuda_stream
    # (of a single device there is no other to be current)
    device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device) if torch.cuda.device_count() > 1 else None
    _torch_names = (torch.bfloat16, torch.float32, raw, device)
    return _torch_names


def norm_workspace_bytes(direction, M, D, dtype, norm_kind) -> int:
    return int((_lib or load_library()).tfla_norm_workspace_bytes(direction, M, D, dtype, norm_kind))


def linear_workspace_bytes(direction, M, K, N, act, dtype, unaligned=False) -> int:
    return int((_lib or load_library()).tfla_linear_workspace_bytes(direction, M, K, N, act, dtype, int(unaligned)))


def gated_workspace_bytes(direction, M, K, N, act, dtype, unaligned=False) -> int:
    return int((_lib or load_library()).tfla_gated_workspace_bytes(direction, M, K, N, act, dtype, int(unaligned)))


def _rows(x, name, b16, f32):
    """dtype code, (M, columns) and device of a dense matrix of rows"""
    t = x.dtype
    shape = x.shape
    dev = x.get_device()
    if t != b16 and t != f32:       # (f32 is b16 where a call takes that type alone)
        raise ValueError("%s must be bfloat16%s (got %s)" % (name, "" if f32 is b16 else " or float32", t))
    if len(shape) != 2 or dev < 0 or not x.is_contiguous():
        raise ValueError("%s must be a contiguous device tensor of two dimensions" % name)
    return BF16 if t == b16 else F32, shape[0], shape[1], dev


def _like(t, dtype, shape, name, dev):
    """shape: a tuple; None passes"""
    if t is None or (t.dtype == dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous()):
        return
    raise ValueError("%s must be a contiguous tensor of dtype %s and shape %s on cuda:%d (got %s %s on %s)"
                     % (name, dtype, tuple(shape), dev, t.dtype, tuple(t.shape), t.device))


def _too_large(*sizes):
    """sizes go to the library as 32-bit integers, which ctypes would cut off without a word"""
    raise ValueError("sizes of 2^31 and more are not supported (got %s)" % (sizes,))


def _columns(x, w, want_dx, want_dw):
    """input columns of a backward call by the tensors that it reads (for bias gradients alone neither, and any number will do)"""
    if (want_dw and x is None) or (want_dx and w is None):
        raise ValueError("%s is needed for the gradients that are wanted" % ("x" if want_dw and x is None else "the weight"))
    t = w if x is None else x
    return 1 if t is None else t.shape[-1]


def _elsewhere(call, dev, names):
    """call with its arguments (among the local names of its first lines) and the tensors' device current, which another one is"""
    import torch
    code = call.__code__
    with torch.cuda.device(dev):
        return call(**{k: names[k] for k in code.co_varnames[:code.co_argcount]})


def _out(o, name, shape, dtype, dev):
    """address of o[name], checked, or of a new tensor there"""
    t = o.get(name)
    if t is None:
        import torch
        t = o[name] = torch.empty(shape, dtype=dtype, device=dev)
    elif t.dtype != dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _like(t, dtype, shape, name, dev)
    return t.data_ptr()


def _bytes(workspace):
    return workspace.numel() * workspace.element_size()


def _memory(workspace, dev):
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on cuda:%d (got one on %s)" % (dev, workspace.device))


def _scratch(o, workspace, need, dev, handle):
    """address and size of the workspace: the caller's, which `out` does not keep, or the one in `out` that earlier calls left, or a new one
    there.  The kept one remembers the stream it was last used on and is recorded on another that uses it.  One that has become too small
    stays alive beside its successor: a captured graph may hold its address (a change of sizes with the same `out` is rare)."""
    if workspace is not None:
        _memory(workspace, dev)
        o.setdefault("workspace", None)
        return workspace.data_ptr(), _bytes(workspace)
    kept = o.get("workspace")
    if kept is not None:
        _memory(kept, dev)
    if need and (kept is None or _bytes(kept) < need):
        import torch
        new = o["workspace"] = torch.empty(need, dtype=torch.uint8, device=dev)
        new.tfla_before, new.tfla_stream = kept, handle
        return new.data_ptr(), need
    if kept is None:
        o["workspace"] = None
        return None, 0
    if getattr(kept, "tfla_stream", None) != handle:
        import torch
        kept.record_stream(torch.cuda.current_stream(dev))
        kept.tfla_stream = handle
    return kept.data_ptr(), _bytes(kept)


def norm_fwd(x, gamma=None, beta=None, norm_kind=NORM_RMS, norm_eps=1e-6, stream=None, out: Optional[Dict] = None) -> Dict:
    """tfla_norm_fwd on torch device tensors.  x: (M, D) in bf16 or fp32; gamma, beta: (D,) fp32 or None.  Returns y and the row
    statistics rstd and (LayerNorm) mean, which norm_bwd needs."""
    if stream is not None:
        return _within(norm_fwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    dtype, M, D, dev = _rows(x, "x", b16, f32)
    if device is not None and dev != device():
        return _elsewhere(norm_fwd, dev, locals())
    if (M | D) >> 31:
        _too_large(M, D)
    gammap = betap = None
    if gamma is not None:
        _like(gamma, f32, (D,), "gamma", dev)
        gammap = gamma.data_ptr()
    if beta is not None:
        _like(beta, f32, (D,), "beta", dev)
        betap = beta.data_ptr()
    o = out if out is not None else {}
    y, rstd = _out(o, "y", (M, D), x.dtype, dev), _out(o, "rstd", (M,), f32, dev)
    mean = _out(o, "mean", (M,), f32, dev) if norm_kind == NORM_LAYER else None
    rc = (_lib or load_library()).tfla_norm_fwd(x.data_ptr(), gammap, betap, M, D, dtype, int(norm_kind), float(norm_eps), y,
                                                rstd, mean, raw_stream(dev))
    if rc != 0:
        raise TflaError(rc, "tfla_norm_fwd")
    return o


def norm_bwd(x, dy, rstd, mean=None, gamma=None, d_residual=None, norm_kind=NORM_RMS, want_dgamma=True, want_dbeta=False,
             workspace=None, stream=None, out: Optional[Dict] = None) -> Dict:
    """tfla_norm_bwd on torch device tensors.  rstd, mean: as norm_fwd returned them; d_residual: (M, D), added to dx, or None.
    Returns dx, dgamma, dbeta (the last two where wanted)."""
    if stream is not None:
        return _within(norm_bwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    dtype, M, D, dev = _rows(x, "x", b16, f32)
    if device is not None and dev != device():
        return _elsewhere(norm_bwd, dev, locals())
    if (M | D) >> 31:
        _too_large(M, D)
    _like(dy, x.dtype, (M, D), "dy", dev); _like(d_residual, x.dtype, (M, D), "d_residual", dev); _like(gamma, f32, (D,), "gamma", dev)
    _like(rstd, f32, (M,), "rstd", dev); _like(mean, f32, (M,), "mean", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    dx = _out(o, "dx", (M, D), x.dtype, dev)
    dgamma = _out(o, "dgamma", (D,), f32, dev) if want_dgamma else None
    dbeta = _out(o, "dbeta", (D,), f32, dev) if want_dbeta else None
    need = norm_workspace_bytes(BWD, M, D, dtype, int(norm_kind)) if want_dgamma or want_dbeta else 0
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_norm_bwd(x.data_ptr(), _ptr(dy), _ptr(rstd), _ptr(mean), _ptr(gamma), _ptr(d_residual), M, D,
                                                dtype, int(norm_kind), dx, dgamma, dbeta, ws, wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_norm_bwd")
    return o


def linear_fwd(x, w, bias=None, residual=None, act=ACT_NONE, keep_pre=False, workspace=None, stream=None,
               out: Optional[Dict] = None) -> Dict:
    """tfla_linear_fwd on torch device tensors.  x: (M, K), w: (N, K), residual: (M, N) in bf16 or fp32; bias: (N,) fp32.  Returns
    y and, with keep_pre, the pre-activation z, which linear_bwd needs where act is not ACT_NONE."""
    if stream is not None:
        return _within(linear_fwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    dtype, M, K, dev = _rows(x, "x", b16, f32)
    if device is not None and dev != device():
        return _elsewhere(linear_fwd, dev, locals())
    N = w.shape[0]
    if (M | K | N) >> 31:
        _too_large(M, K, N)
    _like(w, x.dtype, (N, K), "w", dev)
    if bias is not None:
        _like(bias, f32, (N,), "bias", dev)
    if residual is not None:
        _like(residual, x.dtype, (M, N), "residual", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    y = _out(o, "y", (M, N), x.dtype, dev)
    z = _out(o, "z", (M, N), x.dtype, dev) if keep_pre else None
    need = linear_workspace_bytes(FWD, M, K, N, int(act), dtype, (x.data_ptr() | w.data_ptr()) & 15)
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_linear_fwd(x.data_ptr(), w.data_ptr(), _ptr(bias), _ptr(residual), M, K, N, int(act), dtype, y, z,
                                                  ws, wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_linear_fwd")
    return o


def linear_bwd(x, w, dy, z=None, act=ACT_NONE, want_dx=True, want_dw=True, want_db=False, workspace=None, stream=None,
               out: Optional[Dict] = None) -> Dict:
    """tfla_linear_bwd on torch device tensors.  dy: (M, N); z: the pre-activation of the forward call where act is not ACT_NONE.
    Returns dx, dw, db (those that are wanted); the gradient of the residual is dy itself.  x may be None without dw, w without dx."""
    if stream is not None:
        return _within(linear_bwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    dtype, M, N, dev = _rows(dy, "dy", b16, f32)
    if device is not None and dev != device():
        return _elsewhere(linear_bwd, dev, locals())
    K = _columns(x, w, want_dx, want_dw)
    if (M | K | N) >> 31:
        _too_large(M, K, N)
    t = dy.dtype
    _like(x, t, (M, K), "x", dev); _like(w, t, (N, K), "w", dev); _like(z, t, (M, N), "z", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    dx = _out(o, "dx", (M, K), t, dev) if want_dx else None
    dw = _out(o, "dw", (N, K), t, dev) if want_dw else None
    db = _out(o, "db", (N,), f32, dev) if want_db else None
    need = linear_workspace_bytes(BWD, M, K, N, int(act), dtype, ((_ptr(x) or 0) | (_ptr(w) or 0) | dy.data_ptr()) & 15)
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_linear_bwd(_ptr(x), _ptr(w), dy.data_ptr(), _ptr(z), M, K, N, int(act), dtype, dx, dw, db, ws,
                                                  wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_linear_bwd")
    return o


def gated_fwd(x, w_gate, w_up, b_gate=None, b_up=None, act=ACT_SILU, keep_pre=False, workspace=None, stream=None,
              out: Optional[Dict] = None) -> Dict:
    """tfla_gated_fwd on torch device tensors: h = act(x w_gate^T + b_gate) * (x w_up^T + b_up).  x: (M, K), w_gate, w_up: (N, K) in
    bf16 or fp32; b_gate, b_up: (N,) fp32.  Returns h and, with keep_pre, a and u, which gated_bwd needs."""
    if stream is not None:
        return _within(gated_fwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    dtype, M, K, dev = _rows(x, "x", b16, f32)
    if device is not None and dev != device():
        return _elsewhere(gated_fwd, dev, locals())
    N = w_gate.shape[0]
    if (M | K | N) >> 31:
        _too_large(M, K, N)
    _like(w_gate, x.dtype, (N, K), "w_gate", dev); _like(w_up, x.dtype, (N, K), "w_up", dev)
    _like(b_gate, f32, (N,), "b_gate", dev); _like(b_up, f32, (N,), "b_up", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    h = _out(o, "h", (M, N), x.dtype, dev)
    a = _out(o, "a", (M, N), x.dtype, dev) if keep_pre else None
    u = _out(o, "u", (M, N), x.dtype, dev) if keep_pre else None
    need = gated_workspace_bytes(FWD, M, K, N, int(act), dtype, (x.data_ptr() | w_gate.data_ptr() | w_up.data_ptr()) & 15)
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_gated_fwd(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), _ptr(b_gate), _ptr(b_up), M, K, N,
                                                 int(act), dtype, h, a, u, ws, wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_gated_fwd")
    return o


def gated_bwd(x, w_gate, w_up, a, u, dh, act=ACT_SILU, want_dx=True, want_dw=True, want_db=False, workspace=None, stream=None,
              out: Optional[Dict] = None) -> Dict:
    """tfla_gated_bwd on torch device tensors.  a, u: as gated_fwd with keep_pre returned them; dh: (M, N).  Returns dx, dw_gate,
    dw_up, db_gate, db_up (those that are wanted).  x may be None without the weights' gradients, the weights without dx."""
    if stream is not None:
        return _within(gated_bwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    dtype, M, N, dev = _rows(dh, "dh", b16, f32)
    if device is not None and dev != device():
        return _elsewhere(gated_bwd, dev, locals())
    K = _columns(x, w_gate, want_dx, want_dw)
    if (M | K | N) >> 31:
        _too_large(M, K, N)
    t = dh.dtype
    _like(x, t, (M, K), "x", dev); _like(w_gate, t, (N, K), "w_gate", dev); _like(w_up, t, (N, K), "w_up", dev)
    _like(a, t, (M, N), "a", dev); _like(u, t, (M, N), "u", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    dx = _out(o, "dx", (M, K), t, dev) if want_dx else None
    dwg = _out(o, "dw_gate", (N, K), t, dev) if want_dw else None
    dwu = _out(o, "dw_up", (N, K), t, dev) if want_dw else None
    dbg = _out(o, "db_gate", (N,), f32, dev) if want_db else None
    dbu = _out(o, "db_up", (N,), f32, dev) if want_db else None
    need = gated_workspace_bytes(BWD, M, K, N, int(act), dtype, ((_ptr(x) or 0) | (_ptr(w_gate) or 0) | (_ptr(w_up) or 0) | dh.data_ptr()) & 15)
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_gated_bwd(_ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(a), _ptr(u), dh.data_ptr(), M, K, N, int(act),
                                                 dtype, dx, dwg, dwu, dbg, dbu, ws, wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_gated_bwd")
    return o


# ---- the residual block in 8 bits ------------------------------------------------------------------------------------------
# Codes are tensors of type float8_e4m3fn, scales of type float8_e8m0fnu: one for 128 columns of a row, (blocks of columns, rows), or for
# a block of 128 x 128, (blocks of columns, blocks of rows).  Everything else as for the block above.
_q8_names = None


def _q8_types():
    global _q8_names
    import torch
    _q8_names = (torch.float8_e4m3fn, torch.float8_e8m0fnu)
    return _q8_names


def linear_q8_workspace_bytes(direction, M, K, N, act, unaligned=False) -> int:
    return int((_lib or load_library()).tfla_linear_q8_workspace_bytes(direction, M, K, N, act, int(unaligned)))


def gated_q8_workspace_bytes(direction, M, K, N, act, unaligned=False) -> int:
    return int((_lib or load_library()).tfla_gated_q8_workspace_bytes(direction, M, K, N, act, int(unaligned)))


def _codes(q, name, e4m3):
    """(rows, columns) and device of a dense matrix of codes"""
    shape = q.shape
    dev = q.get_device()
    if q.dtype != e4m3 or len(shape) != 2 or dev < 0 or not q.is_contiguous():
        raise ValueError("%s must be a contiguous device tensor of two dimensions and dtype float8_e4m3fn (got %s %s)" % (name, q.dtype, tuple(shape)))
    return shape[0], shape[1], dev


def q8_quant(x, rows=1, want_q=True, want_t=False, stream=None, out: Optional[Dict] = None) -> Dict:
    """tfla_q8_quant on torch device tensors.  x: (M, K) in bf16 or fp32; rows: 1 (activations: a scale for 128 columns of a row) or 128
    (weights: one for a block of 128 x 128).  Returns q, scale and, with want_t, those of the transpose, qt, scale_t."""
    if stream is not None:
        return _within(q8_quant, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    e4m3, e8m0 = _q8_names or _q8_types()
    dtype, M, K, dev = _rows(x, "x", b16, f32)
    if device is not None and dev != device():
        return _elsewhere(q8_quant, dev, locals())
    if (M | K) >> 31:
        _too_large(M, K)
    if rows != 1 and rows != 128:
        raise ValueError("rows must be 1 or 128 (got %s)" % (rows,))
    o = out if out is not None else {}
    q = scale = qt = scale_t = None
    if want_q:
        q, scale = _out(o, "q", (M, K), e4m3, dev), _out(o, "scale", (-(-K // 128), -(-M // rows)), e8m0, dev)
    if want_t:
        qt, scale_t = _out(o, "qt", (K, M), e4m3, dev), _out(o, "scale_t", (-(-M // 128), -(-K // rows)), e8m0, dev)
    rc = (_lib or load_library()).tfla_q8_quant(x.data_ptr(), M, K, dtype, rows, q, scale, qt, scale_t, raw_stream(dev))
    if rc != 0:
        raise TflaError(rc, "tfla_q8_quant")
    return o


def norm_q8_fwd(x, gamma=None, beta=None, residual=None, norm_kind=NORM_RMS, norm_eps=1e-6, keep_y=False, stream=None,
                out: Optional[Dict] = None) -> Dict:
    """tfla_norm_q8_fwd on torch device tensors: norm of x + residual, quantised.  x, residual: (M, D) in bf16 or fp32; gamma, beta: (D,)
    fp32 or None.  Returns q, scale, rstd, (LayerNorm) mean, with a residual sum, and with keep_y y, the values before quantisation.
    The gradient of x and residual is norm_bwd's dx for x = sum."""
    if stream is not None:
        return _within(norm_q8_fwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    e4m3, e8m0 = _q8_names or _q8_types()
    dtype, M, D, dev = _rows(x, "x", b16, f32)
    if device is not None and dev != device():
        return _elsewhere(norm_q8_fwd, dev, locals())
    if (M | D) >> 31:
        _too_large(M, D)
    t = x.dtype
    gammap = betap = res = total = y = mean = None
    if gamma is not None:
        _like(gamma, f32, (D,), "gamma", dev)
        gammap = gamma.data_ptr()
    if beta is not None:
        _like(beta, f32, (D,), "beta", dev)
        betap = beta.data_ptr()
    o = out if out is not None else {}
    q, scale = _out(o, "q", (M, D), e4m3, dev), _out(o, "scale", (-(-D // 128), M), e8m0, dev)
    rstd = _out(o, "rstd", (M,), f32, dev)
    if residual is not None:
        _like(residual, t, (M, D), "residual", dev)
        res, total = residual.data_ptr(), _out(o, "sum", (M, D), t, dev)
    if keep_y:
        y = _out(o, "y", (M, D), t, dev)
    if norm_kind == NORM_LAYER:
        mean = _out(o, "mean", (M,), f32, dev)
    rc = (_lib or load_library()).tfla_norm_q8_fwd(x.data_ptr(), gammap, betap, res, M, D, dtype, int(norm_kind), float(norm_eps), q, scale,
                                                   total, y, rstd, mean, raw_stream(dev))
    if rc != 0:
        raise TflaError(rc, "tfla_norm_q8_fwd")
    return o


def linear_q8_fwd(xq, x_scale, wq, w_scale, bias=None, residual=None, act=ACT_NONE, keep_pre=False, workspace=None, stream=None,
                  out: Optional[Dict] = None) -> Dict:
    """tfla_linear_q8_fwd on torch device tensors.  xq, x_scale: (M, K) as norm_q8_fwd or q8_quant with rows = 1 returns them; wq, w_scale:
    (N, K) as q8_quant with rows = 128; bias: (N,) fp32; residual: (M, N) bf16.  Returns y and, with keep_pre, z, in bf16."""
    if stream is not None:
        return _within(linear_q8_fwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    e4m3, e8m0 = _q8_names or _q8_types()
    M, K, dev = _codes(xq, "xq", e4m3)
    if device is not None and dev != device():
        return _elsewhere(linear_q8_fwd, dev, locals())
    N = wq.shape[0]
    if (M | K | N) >> 31:
        _too_large(M, K, N)
    kb = -(-K // 128)
    _like(x_scale, e8m0, (kb, M), "x_scale", dev); _like(wq, e4m3, (N, K), "wq", dev); _like(w_scale, e8m0, (kb, -(-N // 128)), "w_scale", dev)
    if bias is not None:
        _like(bias, f32, (N,), "bias", dev)
    if residual is not None:
        _like(residual, b16, (M, N), "residual", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    y = _out(o, "y", (M, N), b16, dev)
    z = _out(o, "z", (M, N), b16, dev) if keep_pre else None
    need = linear_q8_workspace_bytes(FWD, M, K, N, int(act), (xq.data_ptr() | wq.data_ptr()) & 15)
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_linear_q8_fwd(xq.data_ptr(), x_scale.data_ptr(), wq.data_ptr(), w_scale.data_ptr(), _ptr(bias),
                                                     _ptr(residual), M, K, N, int(act), y, z, ws, wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_linear_q8_fwd")
    return o


def linear_q8_bwd(x, wqt, wt_scale, dy, z=None, act=ACT_NONE, want_dx=True, want_dw=True, want_db=False, workspace=None, stream=None,
                  out: Optional[Dict] = None) -> Dict:
    """tfla_linear_q8_bwd on torch device tensors.  x: (M, K) bf16, what the forward call's codes were made of; wqt, wt_scale: the
    transposed weights (K, N) as q8_quant with rows = 128 returns them; dy: (M, N) bf16; z: as linear_q8_fwd with keep_pre returned it, where
    act is not ACT_NONE.  Returns dx, dw, db (those that are wanted).  x may be None without dw, wqt and wt_scale without dx."""
    if stream is not None:
        return _within(linear_q8_bwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    e4m3, e8m0 = _q8_names or _q8_types()
    dtype, M, N, dev = _rows(dy, "dy", b16, b16)
    if device is not None and dev != device():
        return _elsewhere(linear_q8_bwd, dev, locals())
    K = _q8_columns(x, wqt, wt_scale, want_dx, want_dw)
    if (M | K | N) >> 31:
        _too_large(M, K, N)
    _like(x, b16, (M, K), "x", dev); _like(wqt, e4m3, (K, N), "wqt", dev); _like(z, b16, (M, N), "z", dev)
    _like(wt_scale, e8m0, (-(-N // 128), -(-K // 128)), "wt_scale", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    dx = _out(o, "dx", (M, K), b16, dev) if want_dx else None
    dw = _out(o, "dw", (N, K), b16, dev) if want_dw else None
    db = _out(o, "db", (N,), f32, dev) if want_db else None
    need = linear_q8_workspace_bytes(BWD, M, K, N, int(act), (_ptr(wqt) or 0) & 15)
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_linear_q8_bwd(_ptr(x), _ptr(wqt), _ptr(wt_scale), dy.data_ptr(), _ptr(z), M, K, N, int(act), dx, dw,
                                                     db, ws, wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_linear_q8_bwd")
    return o


def gated_q8_fwd(xq, x_scale, wq_gate, w_scale_gate, wq_up, w_scale_up, b_gate=None, b_up=None, act=ACT_SILU, keep_pre=False, workspace=None,
                 stream=None, out: Optional[Dict] = None) -> Dict:
    """tfla_gated_q8_fwd on torch device tensors: h = act(x w_gate^T + b_gate) * (x w_up^T + b_up) in 8 bits.  Codes and scales as for
    linear_q8_fwd; b_gate, b_up: (N,) fp32.  Returns hq, h_scale, which linear_q8_fwd takes, and, with keep_pre, h, a and u in bf16."""
    if stream is not None:
        return _within(gated_q8_fwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    e4m3, e8m0 = _q8_names or _q8_types()
    M, K, dev = _codes(xq, "xq", e4m3)
    if device is not None and dev != device():
        return _elsewhere(gated_q8_fwd, dev, locals())
    N = wq_gate.shape[0]
    if (M | K | N) >> 31:
        _too_large(M, K, N)
    kb, nb = -(-K // 128), -(-N // 128)
    _like(x_scale, e8m0, (kb, M), "x_scale", dev)
    _like(wq_gate, e4m3, (N, K), "wq_gate", dev); _like(w_scale_gate, e8m0, (kb, nb), "w_scale_gate", dev)
    _like(wq_up, e4m3, (N, K), "wq_up", dev); _like(w_scale_up, e8m0, (kb, nb), "w_scale_up", dev)
    _like(b_gate, f32, (N,), "b_gate", dev); _like(b_up, f32, (N,), "b_up", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    hq, h_scale = _out(o, "hq", (M, N), e4m3, dev), _out(o, "h_scale", (nb, M), e8m0, dev)
    h = a = u = None
    if keep_pre:
        h, a, u = _out(o, "h", (M, N), b16, dev), _out(o, "a", (M, N), b16, dev), _out(o, "u", (M, N), b16, dev)
    need = gated_q8_workspace_bytes(FWD, M, K, N, int(act), (xq.data_ptr() | wq_gate.data_ptr() | wq_up.data_ptr()) & 15)
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_gated_q8_fwd(xq.data_ptr(), x_scale.data_ptr(), wq_gate.data_ptr(), w_scale_gate.data_ptr(),
                                                    wq_up.data_ptr(), w_scale_up.data_ptr(), _ptr(b_gate), _ptr(b_up), M, K, N, int(act),
                                                    hq, h_scale, h, a, u, ws, wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_gated_q8_fwd")
    return o


def gated_q8_bwd(x, wqt_gate, wt_scale_gate, wqt_up, wt_scale_up, a, u, dh, act=ACT_SILU, want_dx=True, want_dw=True, want_db=False,
                 workspace=None, stream=None, out: Optional[Dict] = None) -> Dict:
    """tfla_gated_q8_bwd on torch device tensors.  x: (M, K) bf16, what the forward call's codes were made of; the transposed weights (K, N)
    as q8_quant with rows = 128 returns them; a, u: as gated_q8_fwd with keep_pre returned them; dh: (M, N) bf16.  Returns dx, dw_gate,
    dw_up, db_gate, db_up (those that are wanted).  x may be None without the weights' gradients, the weights without dx."""
    if stream is not None:
        return _within(gated_q8_bwd, stream, locals())
    b16, f32, raw_stream, device = _torch_names or _torch_types()
    e4m3, e8m0 = _q8_names or _q8_types()
    dtype, M, N, dev = _rows(dh, "dh", b16, b16)
    if device is not None and dev != device():
        return _elsewhere(gated_q8_bwd, dev, locals())
    K = _q8_columns(x, wqt_gate, wt_scale_gate, want_dx, want_dw)
    if want_dx and (wqt_up is None or wt_scale_up is None):
        raise ValueError("the weights are needed for dx")
    if (M | K | N) >> 31:
        _too_large(M, K, N)
    blocks = (-(-N // 128), -(-K // 128))
    _like(x, b16, (M, K), "x", dev); _like(a, b16, (M, N), "a", dev); _like(u, b16, (M, N), "u", dev)
    _like(wqt_gate, e4m3, (K, N), "wqt_gate", dev); _like(wt_scale_gate, e8m0, blocks, "wt_scale_gate", dev)
    _like(wqt_up, e4m3, (K, N), "wqt_up", dev); _like(wt_scale_up, e8m0, blocks, "wt_scale_up", dev)
    handle = raw_stream(dev)
    o = out if out is not None else {}
    dx = _out(o, "dx", (M, K), b16, dev) if want_dx else None
    dwg = _out(o, "dw_gate", (N, K), b16, dev) if want_dw else None
    dwu = _out(o, "dw_up", (N, K), b16, dev) if want_dw else None
    dbg = _out(o, "db_gate", (N,), f32, dev) if want_db else None
    dbu = _out(o, "db_up", (N,), f32, dev) if want_db else None
    need = gated_q8_workspace_bytes(BWD, M, K, N, int(act), ((_ptr(wqt_gate) or 0) | (_ptr(wqt_up) or 0)) & 15)
    ws, wsb = _scratch(o, workspace, need, dev, handle)
    rc = (_lib or load_library()).tfla_gated_q8_bwd(_ptr(x), _ptr(wqt_gate), _ptr(wt_scale_gate), _ptr(wqt_up), _ptr(wt_scale_up), _ptr(a),
                                                    _ptr(u), dh.data_ptr(), M, K, N, int(act), dx, dwg, dwu, dbg, dbu, ws, wsb, handle)
    if rc != 0:
        raise TflaError(rc, "tfla_gated_q8_bwd")
    return o


def _q8_columns(x, wqt, wt_scale, want_dx, want_dw):
    """input columns of a backward call by the tensors that it reads"""
    if (want_dw and x is None) or (want_dx and (wqt is None or wt_scale is None)):
        raise ValueError("%s needed for the gradients that are wanted" % ("x is" if want_dw and x is None else "the weights and their scales are"))
    return x.shape[-1] if x is not None else (1 if wqt is None else wqt.shape[0])
