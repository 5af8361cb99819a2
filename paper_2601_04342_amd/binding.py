"""Thin ctypes binding of the C-ABI library ``librehyat.so``.

Argument marshalling only: every step of the operator runs in the library's HIP
kernels.  torch is used for device memory and streams.  There is no fallback:
if the library is missing or cannot be loaded, importing a symbol from it
raises.
"""
import ctypes
import functools
import math
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librehyat.so")

OK = 0
E_NULL, E_SHAPE, E_UNSUPPORTED, E_WORKSPACE, E_HIP = -1, -2, -3, -4, -5
STAB_ROWMAX, STAB_NONE = 0, 1

# every symbol include/rehyat.h declares
EXPORTS = ("rehyat_chunk_plan", "rehyat_workspace_bytes", "rehyat_set_workspace",
           "rehyat_forward", "rehyat_forward_ex", "rehyat_forward_ws", "rehyat_forward_noalloc",
           "rehyat_step", "rehyat_state", "rehyat_shutdown",
           "rehyat_phi_backward", "rehyat_phi_backward_workspace_bytes",
           "rehyat_rope", "rehyat_rope_turns",
           "rehyat_distill_loss", "rehyat_distill_loss_workspace_bytes",
           "rehyat_adamw_table_bytes", "rehyat_adamw_prepare", "rehyat_adamw_step", "rehyat_adamw_moments",
           "rehyat_status_string", "rehyat_version", "rehyat_last_hip_error",
           "rehyat_attn_kernel_name",
           "rehyat_profile_enable", "rehyat_profile_read", "rehyat_debug_set_xcd_mask")


class PhiParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("w1_q", "b1_q", "w2_q", "b2_q", "w1_k", "b1_k", "w2_k", "b2_k")] + [
        ("hidden", ctypes.c_int32), ("dprime", ctypes.c_int32),
        ("degree", ctypes.c_int32), ("act", ctypes.c_int32)]


class DebugOut(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("m", "nS", "aS", "nL", "aL")]


class PhiGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("w1_q", "b1_q", "w2_q", "b2_q", "w1_k", "b1_k", "w2_k", "b2_k")]


class ForwardSaved(ctypes.Structure):
    _fields_ = [("nS", ctypes.c_void_p), ("nL", ctypes.c_void_p)]


BACKWARD_MAX_CHUNKS = 1024
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
ROPE_LAYOUTS = {"interleaved": 0, "half": 1}


class RopePlan(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_void_p), ("d", ctypes.c_int32), ("rot", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("axes", ctypes.c_int32), ("section", ctypes.c_int32 * 3),
                ("scale", ctypes.c_float)]


class RopePositions(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_n", ctypes.c_int64),
                ("start", ctypes.c_int64), ("bits", ctypes.c_int32), ("rows", ctypes.c_int32),
                ("cols", ctypes.c_int32)]


class RopeOperand(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("out", ctypes.c_void_p)] + [
        (f"{t}_stride_{n}", ctypes.c_int64) for t in ("x", "out") for n in "bhn"] + [("heads", ctypes.c_int32)]


class AdamWTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "master", "grad", "m", "v", "m_exp", "v_exp")] + [
        ("n", ctypes.c_int64), ("param_type", ctypes.c_int32), ("grad_type", ctypes.c_int32)]


class AdamWPlan(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("items", ctypes.c_int64), ("n_tensors", ctypes.c_int32),
                ("state_bits", ctypes.c_int32)]


class AdamWHyper(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [
        ("lr_device", ctypes.c_void_p), ("nearest_steps", ctypes.c_int64)]


class RehyatError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        lib = _load()
        msg = lib.rehyat_status_string(code).decode()
        hip = lib.rehyat_last_hip_error().decode()
        super().__init__(f"{where} failed: {code} ({msg}){' [' + hip + ']' if hip else ''}")


_lib = None


def _load():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2601_04342_amd.build` "
            "(there is no CPU or PyTorch fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci = ctypes.c_void_p, ctypes.c_int
    lib.rehyat_chunk_plan.restype = ci
    lib.rehyat_chunk_plan.argtypes = [ci, ci, ci, ci, ctypes.POINTER(ctypes.c_int64),
                                      ctypes.POINTER(ci)]
    lib.rehyat_workspace_bytes.restype = ctypes.c_size_t
    lib.rehyat_workspace_bytes.argtypes = [ci, ci, ci, ci]
    lib.rehyat_set_workspace.restype = ci
    lib.rehyat_set_workspace.argtypes = [vp, ctypes.c_size_t]
    lib.rehyat_forward.restype = ci
    lib.rehyat_forward.argtypes = [vp, vp, vp, ctypes.POINTER(PhiParams), vp,
                                   ci, ci, ci, ci, ci, ci, vp]
    lib.rehyat_forward_ex.restype = ci
    lib.rehyat_forward_ex.argtypes = [vp, vp, vp, ctypes.POINTER(PhiParams), vp,
                                      ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                      ctypes.POINTER(DebugOut), vp]
    lib.rehyat_forward_ws.restype = ci
    lib.rehyat_forward_ws.argtypes = [vp, vp, vp, ctypes.POINTER(PhiParams), vp,
                                      ci, ci, ci, ci, ci, ci, ci, ci, ci,
                                      vp, ctypes.c_size_t, vp]
    lib.rehyat_forward_noalloc.restype = ci
    lib.rehyat_forward_noalloc.argtypes = [vp, vp, vp, ctypes.POINTER(PhiParams), vp,
                                           ci, ci, ci, ci, ci, ci, vp]
    lib.rehyat_step.restype = ci
    lib.rehyat_step.argtypes = [vp, vp, vp, ctypes.POINTER(PhiParams), vp, vp, vp,
                                ci, ci, ci, ci, ci, ci, ci, vp]
    lib.rehyat_state.restype = ci
    lib.rehyat_state.argtypes = [vp, vp, ctypes.POINTER(PhiParams), vp, vp,
                                 ci, ci, ci, ci, ci, ci, vp]
    lib.rehyat_phi_backward_workspace_bytes.restype = ctypes.c_size_t
    lib.rehyat_phi_backward_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci]
    lib.rehyat_phi_backward.restype = ci
    lib.rehyat_phi_backward.argtypes = [vp, vp, vp, ctypes.POINTER(PhiParams), vp, vp,
                                        ctypes.POINTER(ForwardSaved), ctypes.POINTER(PhiGrads),
                                        ci, ci, ci, ci, ci, ci, ci, vp, ctypes.c_size_t, vp]
    lib.rehyat_rope_turns.restype = ci
    lib.rehyat_rope_turns.argtypes = [ctypes.POINTER(ctypes.c_double), ci, ctypes.POINTER(ctypes.c_uint64)]
    lib.rehyat_rope.restype = ci
    lib.rehyat_rope.argtypes = [vp, ci, ctypes.POINTER(RopePlan), vp, ci, ci, ci, ci, vp]   # packed structs
    lib.rehyat_distill_loss_workspace_bytes.restype = ctypes.c_size_t
    lib.rehyat_distill_loss_workspace_bytes.argtypes = [ci, ci, ci, ci]
    lib.rehyat_distill_loss.restype = ci
    lib.rehyat_distill_loss.argtypes = [vp, vp, ci, vp, ctypes.c_float, vp, vp, ci, ci, ci, ci, vp,
                                        ctypes.c_size_t, vp]
    lib.rehyat_adamw_table_bytes.restype = ctypes.c_size_t
    lib.rehyat_adamw_table_bytes.argtypes = [ctypes.POINTER(ctypes.c_int64), ci]
    lib.rehyat_adamw_prepare.restype = ci
    lib.rehyat_adamw_prepare.argtypes = [ctypes.POINTER(AdamWTensor), ci, ci, ctypes.c_int64, vp, ctypes.c_size_t,
                                         ctypes.POINTER(AdamWPlan), vp]
    lib.rehyat_adamw_step.restype = ci
    lib.rehyat_adamw_step.argtypes = [ctypes.POINTER(AdamWPlan), ctypes.POINTER(AdamWHyper), vp]
    lib.rehyat_adamw_moments.restype = ci
    lib.rehyat_adamw_moments.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_int64, vp]
    lib.rehyat_shutdown.restype = ci
    lib.rehyat_shutdown.argtypes = []
    lib.rehyat_status_string.restype = ctypes.c_char_p
    lib.rehyat_status_string.argtypes = [ci]
    lib.rehyat_version.restype = ci
    lib.rehyat_version.argtypes = []
    lib.rehyat_last_hip_error.restype = ctypes.c_char_p
    lib.rehyat_last_hip_error.argtypes = []
    lib.rehyat_attn_kernel_name.restype = ctypes.c_char_p
    lib.rehyat_attn_kernel_name.argtypes = [ci]
    lib.rehyat_profile_enable.restype = ci
    lib.rehyat_profile_enable.argtypes = [ci]
    lib.rehyat_debug_set_xcd_mask.restype = ci
    lib.rehyat_debug_set_xcd_mask.argtypes = [ctypes.c_uint]
    lib.rehyat_profile_read.restype = ci
    lib.rehyat_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ci)]
    _lib = lib
    return lib


def library():
    """The loaded ctypes library (raises if it is not built)."""
    return _load()


def version():
    return _load().rehyat_version()


def attn_kernel_name(d):
    return _load().rehyat_attn_kernel_name(d).decode()


def status_string(code):
    return _load().rehyat_status_string(code).decode()


def chunk_plan(T, HW, chunk, overlap=0):
    """[n_chunks, 5] int64 tensor of (q_lo, q_hi, s_lo, s_hi, l_hi) rows."""
    lib = _load()
    n = ctypes.c_int(0)
    rc = lib.rehyat_chunk_plan(T, HW, chunk, overlap, None, ctypes.byref(n))
    if rc != OK:
        raise RehyatError(rc, "rehyat_chunk_plan")
    table = torch.zeros(n.value, 5, dtype=torch.int64)
    rc = lib.rehyat_chunk_plan(T, HW, chunk, overlap,
                               ctypes.cast(table.data_ptr(), ctypes.POINTER(ctypes.c_int64)),
                               ctypes.byref(n))
    if rc != OK:
        raise RehyatError(rc, "rehyat_chunk_plan")
    return table


def workspace_bytes(B, H, d, dprime=None):
    return _load().rehyat_workspace_bytes(B, H, d, 2 * d if dprime is None else dprime)


def set_workspace(tensor):
    """Hand a caller-owned CUDA byte tensor to the library (None to undo)."""
    lib = _load()
    if tensor is None:
        rc = lib.rehyat_set_workspace(None, 0)
    else:
        rc = lib.rehyat_set_workspace(tensor.data_ptr(), tensor.numel() * tensor.element_size())
    if rc != OK:
        raise RehyatError(rc, "rehyat_set_workspace")


def shutdown():
    rc = _load().rehyat_shutdown()
    if rc != OK:
        raise RehyatError(rc, "rehyat_shutdown")


KERNEL_KINDS = ("state", "prefix", "attn")


def profile_enable(on=True):
    rc = _load().rehyat_profile_enable(1 if on else 0)
    if rc != OK:
        raise RehyatError(rc, "rehyat_profile_enable")


def debug_set_xcd_mask(mask):
    """Measurement hook (timing only): attention workgroups on XCDs whose bit is clear exit at once."""
    rc = _load().rehyat_debug_set_xcd_mask(int(mask))
    if rc != OK:
        raise RehyatError(rc, "rehyat_debug_set_xcd_mask")


def profile_read():
    """{kind: (total_ms, launches)} since the last read; waits for the events."""
    ms = (ctypes.c_double * 3)()
    n = (ctypes.c_int * 3)()
    rc = _load().rehyat_profile_read(ms, n)
    if rc != OK:
        raise RehyatError(rc, "rehyat_profile_read")
    return {k: (ms[i], n[i]) for i, k in enumerate(KERNEL_KINDS)}


def phi_to_device(phi, device="cuda"):
    """dict of fp32 CPU tensors -> dict of device tensors in the library's dtypes
    (weights bf16, biases fp32)."""
    out = {}
    for name, t in phi.items():
        dt = torch.bfloat16 if name.startswith("w") else torch.float32
        out[name] = t.to(device=device, dtype=dt).contiguous()
    return out


# Every call goes through the next two: 6.4 us of the 20 us that enqueueing a small call took, now 3.2.
def _phi_struct(phi, d):
    bf16, f32 = torch.bfloat16, torch.float32
    for name, t in phi.items():
        want = bf16 if name.startswith("w") else f32
        if t.dtype is not want or not t.is_cuda or not t.is_contiguous():
            raise TypeError(f"phi[{name}] must be a contiguous CUDA {want} tensor")
    w1, w2 = phi["w1_q"], phi["w2_q"]
    b1, b2 = phi["b1_q"], phi["b2_q"]
    w1k, b1k, w2k, b2k = phi["w1_k"], phi["b1_k"], phi["w2_k"], phi["b2_k"]
    s1, s2 = w1.shape, w2.shape
    H, hidden, dd = s1
    dprime = s2[1]
    if dd != d:
        raise ValueError("phi weights do not match the head dimension")
    n1, n2 = (H, hidden), (H, dprime)
    if (w1k.shape != s1 or b1.shape != n1 or b1k.shape != n1 or s2 != (H, dprime, hidden) or w2k.shape != s2
            or b2.shape != n2 or b2k.shape != n2):
        raise ValueError("inconsistent phi parameter shapes")
    return PhiParams(w1.data_ptr(), b1.data_ptr(), w2.data_ptr(), b2.data_ptr(), w1k.data_ptr(), b1k.data_ptr(),
                     w2k.data_ptr(), b2k.data_ptr(), hidden, dprime, 2, 0), H


# torch's own shortcuts past the stream object; where a torch does not have them, that object serves
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_handle(stream):
    """The caller's stream, or the current one of the current device, as the library takes it."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _current_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_current_device())


def _check_qkv(q, k, v):
    for t in (q, k, v):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("q, k, v must be contiguous CUDA bf16 tensors [B, H, N, d]")
    if k.shape != q.shape or v.shape != q.shape:
        raise ValueError("q, k, v shapes differ")


def forward(q, k, v, phi, T, HW, chunk, out=None, overlap=0, causal=True,
            stab_mode=STAB_ROWMAX, debug=False, stream=None, plain=False, workspace=None,
            noalloc=False):
    """Hybrid attention forward.  q, k, v: CUDA bf16 [B, H, T*HW, d].

    Returns ``out`` (bf16, same shape), or ``(out, components)`` with
    ``debug=True`` where components is a dict of fp32 tensors m, nS, aS, nL, aL.
    ``plain=True`` calls ``rehyat_forward`` (no extra knobs) instead of
    ``rehyat_forward_ex``; ``workspace`` (a CUDA byte tensor) calls
    ``rehyat_forward_ws``; ``noalloc=True`` calls ``rehyat_forward_noalloc``.
    """
    lib = _load()
    _check_qkv(q, k, v)
    B, H, N, d = q.shape
    if N != T * HW:
        raise ValueError("N != T*HW")
    p, Hp = _phi_struct(phi, d)
    if Hp != H:
        raise ValueError("phi head count differs from q")
    if out is None:
        out = torch.empty_like(q)
    sp = _stream_handle(stream)
    if plain or noalloc:
        fn, name = ((lib.rehyat_forward_noalloc, "rehyat_forward_noalloc") if noalloc
                    else (lib.rehyat_forward, "rehyat_forward"))
        rc = fn(q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(p),
                out.data_ptr(), B, H, T, HW, d, chunk, sp)
        if rc != OK:
            raise RehyatError(rc, name)
        return out
    if workspace is not None:
        rc = lib.rehyat_forward_ws(q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(p),
                                   out.data_ptr(), B, H, T, HW, d, chunk, overlap,
                                   int(bool(causal)), stab_mode, workspace.data_ptr(),
                                   workspace.numel() * workspace.element_size(), sp)
        if rc != OK:
            raise RehyatError(rc, "rehyat_forward_ws")
        return out
    comps, dbg = None, None
    if debug:
        f32 = dict(device=q.device, dtype=torch.float32)
        comps = dict(m=torch.zeros(B, H, N, **f32), nS=torch.zeros(B, H, N, **f32),
                     aS=torch.zeros(B, H, N, d, **f32), nL=torch.zeros(B, H, N, **f32),
                     aL=torch.zeros(B, H, N, d, **f32))
        dbg = DebugOut(*(comps[n].data_ptr() for n in ("m", "nS", "aS", "nL", "aL")))
    rc = lib.rehyat_forward_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(p),
                               out.data_ptr(), B, H, T, HW, d, chunk, overlap,
                               int(bool(causal)), stab_mode,
                               ctypes.byref(dbg) if dbg is not None else None, sp)
    if rc != OK:
        raise RehyatError(rc, "rehyat_forward_ex")
    return (out, comps) if debug else out


def step(q_t, k_win, v_win, phi, S, z, n_absorb, out=None, stab_mode=STAB_ROWMAX, stream=None):
    """One chunk of the chunk-wise RNN (Eq. 14-18).  q_t: CUDA bf16 [B, H, n_q, d];
    k_win, v_win: [B, H, n_win, d], the softmax window oldest token first; S
    [B, H, D', d] and z [B, H, D'] fp32 are read for the read-out and then
    advanced in place by the first ``n_absorb`` window tokens.  Returns y_t."""
    lib = _load()
    for t in (q_t, k_win, v_win):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise TypeError("q_t, k_win, v_win must be contiguous CUDA bf16 tensors [B, H, n, d]")
    if k_win.shape != v_win.shape or k_win.shape[:2] != q_t.shape[:2] or k_win.shape[3] != q_t.shape[3]:
        raise ValueError("q_t / k_win / v_win shapes are inconsistent")
    B, H, n_q, d = q_t.shape
    n_win = k_win.shape[2]
    p, _ = _phi_struct(phi, d)
    for t, shape in ((S, (B, H, p.dprime, d)), (z, (B, H, p.dprime))):
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != shape:
            raise TypeError(f"state tensors must be contiguous CUDA fp32 of shape {shape}")
    if out is None:
        out = torch.empty_like(q_t)
    elif out.shape != q_t.shape or out.dtype != torch.bfloat16 or not out.is_contiguous():
        raise TypeError("out must match q_t")
    rc = lib.rehyat_step(q_t.data_ptr(), k_win.data_ptr(), v_win.data_ptr(), ctypes.byref(p),
                         S.data_ptr(), z.data_ptr(), out.data_ptr(), B, H, d, n_q, n_win,
                         int(n_absorb), stab_mode, _stream_handle(stream))
    if rc != OK:
        raise RehyatError(rc, "rehyat_step")
    return out


def state(k, v, phi, T, HW, upto_frames, stream=None):
    """(S [B,H,D',d] fp32, z [B,H,D'] fp32) after absorbing the first
    ``upto_frames`` latent frames (Eq. 14-15, 17-18)."""
    lib = _load()
    _check_qkv(k, k, v)
    B, H, N, d = k.shape
    p, _ = _phi_struct(phi, d)
    S = torch.empty(B, H, p.dprime, d, device=k.device, dtype=torch.float32)
    z = torch.empty(B, H, p.dprime, device=k.device, dtype=torch.float32)
    rc = lib.rehyat_state(k.data_ptr(), v.data_ptr(), ctypes.byref(p), S.data_ptr(),
                          z.data_ptr(), B, H, T, HW, d, upto_frames,
                          _stream_handle(stream))
    if rc != OK:
        raise RehyatError(rc, "rehyat_state")
    return S, z


def phi_backward_workspace_bytes(B, H, T, HW, d, chunk):
    return _load().rehyat_phi_backward_workspace_bytes(B, H, T, HW, d, chunk)


def phi_backward(q, k, v, phi, grad_out, T, HW, chunk, overlap=0, workspace=None, out=None,
                 grads=None, stream=None, saved=None):
    """Gradients of a loss w.r.t. the parameters of phi_q and phi_k for a given
    ``grad_out`` = dL/dy_hat (CUDA bf16 [B, H, T*HW, d]): one step of the distillation of
    Eq. 19.  Returns ``(grads, y_hat)``: a dict of eight fp32 CUDA tensors shaped like the
    parameters, and the output of the recomputed forward pass.  ``workspace`` is a CUDA
    byte tensor of at least ``phi_backward_workspace_bytes`` bytes (allocated here if
    None).  ``saved`` = (out, nS, nL) from ``forward(..., debug=True)`` on the same arguments
    skips the attention kernel of the recomputation."""
    lib = _load()
    _check_qkv(q, k, v)
    if grad_out.shape != q.shape or grad_out.dtype != torch.bfloat16 or not grad_out.is_cuda \
            or not grad_out.is_contiguous():
        raise TypeError("grad_out must be a contiguous CUDA bf16 tensor shaped like q")
    B, H, N, d = q.shape
    if N != T * HW:
        raise ValueError("N != T*HW")
    p, Hp = _phi_struct(phi, d)
    if Hp != H:
        raise ValueError("phi head count differs from q")
    if workspace is None:
        need = lib.rehyat_phi_backward_workspace_bytes(B, H, T, HW, d, chunk)
        if need == 0:
            raise RehyatError(E_UNSUPPORTED, "rehyat_phi_backward_workspace_bytes")
        workspace = torch.empty(need, device=q.device, dtype=torch.uint8)
    sv = None
    if saved is not None:
        out, nS, nL = saved
        for t in (nS, nL):
            if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.shape != q.shape[:3]:
                raise TypeError("saved nS, nL must be contiguous CUDA fp32 tensors [B, H, N]")
        if out.shape != q.shape or out.dtype != torch.bfloat16 or not out.is_contiguous():
            raise TypeError("saved out must match q")
        sv = ForwardSaved(nS.data_ptr(), nL.data_ptr())
    if out is None:
        out = torch.empty_like(q)
    if grads is None:
        grads = {n: torch.empty(t.shape, device=q.device, dtype=torch.float32) for n, t in phi.items()}
    g = PhiGrads()
    for name in ("w1_q", "b1_q", "w2_q", "b2_q", "w1_k", "b1_k", "w2_k", "b2_k"):
        t = grads[name]
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.shape != phi[name].shape:
            raise TypeError(f"grads[{name}] must be a contiguous CUDA fp32 tensor shaped like phi[{name}]")
        setattr(g, name, t.data_ptr())
    rc = lib.rehyat_phi_backward(q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(p),
                                 grad_out.data_ptr(), out.data_ptr(),
                                 ctypes.byref(sv) if sv is not None else None, ctypes.byref(g),
                                 B, H, T, HW, d, chunk, overlap, workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(),
                                 _stream_handle(stream))
    if rc != OK:
        raise RehyatError(rc, "rehyat_phi_backward")
    return grads, out


def _elsewhere(t, stream):
    """What to enter so that work on ``t`` and what is allocated for it belong to ``stream`` (None: the current
    stream of the tensor's device); None where that is so already."""
    if stream is not None:
        if stream.device != t.device:
            raise ValueError("the stream belongs to another device than the tensors")
        return torch.cuda.stream(stream)
    here = _current_device() if _current_device is not None else torch.cuda.current_device()
    return torch.cuda.device(t.device) if here != t.get_device() else None


class Rope:
    """Rotary positions of heads of width ``d``, of which the first ``rot`` elements turn.

    ``layout``: "interleaved" (pairs 2i, 2i+1) or "half" (pairs i, i + rot/2).  ``sections``: pairs of each axis
    (default: one axis); pair i of an axis with n pairs turns by base^(-i/n) radians a position.  ``scaling`` for
    contexts longer than the ones trained on, of the first axis: dict(kind=..., factor=s) with kind "linear" (positions
    divided by s), "base" (base times s^(n/(n-1)): the slowest pair is divided by s, the fastest kept) or "parts" (with
    original=L: pairs that make fewer than ``low`` = 1 turns in L positions are divided by s, those of more than
    ``high`` = 32 are kept, a ramp between them; rotated values times 0.1 ln s + 1).  ``freqs`` (radians a position,
    one for each pair) and ``scale`` replace all that."""

    def __init__(self, d, rot=None, layout="interleaved", base=10000.0, sections=None, scaling=None, freqs=None,
                 scale=None, device="cuda"):
        rot = d if rot is None else rot
        if not 2 <= rot <= d <= 512 or rot % 2 or d % 2:
            raise ValueError("rot and d must be even, 2 <= rot <= d <= 512")
        sections = (rot // 2,) if sections is None else tuple(int(n) for n in sections)
        if not 1 <= len(sections) <= 3 or min(sections) < 1 or sum(sections) != rot // 2:
            raise ValueError("sections must be one to three positive counts of pairs that add up to rot / 2")
        if layout not in ROPE_LAYOUTS:
            raise ValueError(f"layout must be one of {tuple(ROPE_LAYOUTS)}")
        mu = 1.0
        if freqs is None:
            freqs = []
            for axis, n in enumerate(sections):
                f, m = self._frequencies(n, float(base), scaling if axis == 0 else None)
                freqs.append(f)
                mu *= m
            freqs = torch.cat(freqs)
        elif scaling is not None:
            raise ValueError("give either freqs or scaling")
        freqs = torch.as_tensor(freqs, dtype=torch.float64).detach().cpu().contiguous()
        if freqs.shape != (rot // 2,):
            raise ValueError("freqs must hold rot / 2 values")
        self.d, self.rot, self.layout, self.sections = d, rot, layout, sections
        self.freqs, self.scale = freqs, mu if scale is None else float(scale)
        turns = torch.empty(rot // 2, dtype=torch.int64)
        rc = _load().rehyat_rope_turns(ctypes.cast(freqs.data_ptr(), ctypes.POINTER(ctypes.c_double)), rot // 2,
                                       ctypes.cast(turns.data_ptr(), ctypes.POINTER(ctypes.c_uint64)))
        if rc != OK:
            raise RehyatError(rc, "rehyat_rope_turns")
        self.turns = turns.to(device)
        self._plan = RopePlan(self.turns.data_ptr(), d, rot, ROPE_LAYOUTS[layout], len(sections),
                              (ctypes.c_int32 * 3)(*sections), self.scale)
        self._ref = ctypes.byref(self._plan)

    @staticmethod
    def _frequencies(n, base, scaling):
        """n frequencies of one axis in 64 bits, and the factor on rotated values."""
        if scaling is None:
            return base ** (-torch.arange(n, dtype=torch.float64) / n), 1.0
        kind, s = scaling.get("kind"), float(scaling.get("factor", 0.0))
        if kind not in ("linear", "base", "parts") or not 0 < s < math.inf:
            raise ValueError('scaling needs kind "linear", "base" or "parts" and a positive factor')
        if kind == "base" and n > 1:
            base *= s ** (n / (n - 1))
        f = base ** (-torch.arange(n, dtype=torch.float64) / n)
        if kind == "linear":
            return f / s, 1.0
        if kind == "base":
            return f, 1.0
        low, high = float(scaling.get("low", 1.0)), float(scaling.get("high", 32.0))
        original = float(scaling.get("original", 0.0))
        if not low < high or not original > 0:
            raise ValueError("scaling by parts needs low < high and the original length")
        made = original * f / (2 * math.pi)
        keep = ((made - low) / (high - low)).clamp(0.0, 1.0)
        return f * keep + f / s * (1.0 - keep), 0.1 * math.log(s) + 1.0 if s > 1 else 1.0

    @classmethod
    def video(cls, d, layout="interleaved", base=10000.0, scaling=None, device="cuda"):
        """Heads that turn by frame, row and column: a third of the pairs each, the frame takes what is left over."""
        third = d // 2 // 3
        return cls(d, layout=layout, base=base, sections=(d // 2 - 2 * third, third, third), scaling=scaling,
                   device=device)


# rehyat_rope_operand (two of them) and rehyat_rope_positions as they lie in memory, packed in one go: a call for one token
# is 12 us of host work, 3 of them the launch, and was 13.5 with a ctypes struct for each
_rope_operands = struct.Struct("QQ6qi4x" * 2)
_rope_positions = struct.Struct("Q3q3i4x")
_NO_OPERAND = (0,) * 9
_ROPE_OPERAND = "q and k must be CUDA tensors [B, H, N, d] in bf16, fp16 or fp32 with contiguous rows"


def _rope_operand(x, shape, stride, out):
    """The fields of a rehyat_rope_operand, and its output."""
    _, H, N, d = shape
    if out is None:
        out, n = x.new_empty(shape), N * d
        return (x.data_ptr(), out.data_ptr(), *stride[:3], n * H, n, d, H), out
    to = out.stride()
    if out.shape != shape or out.dtype != x.dtype or out.device != x.device or to[3] != 1:
        raise TypeError("out must match its operand, with contiguous rows")
    return (x.data_ptr(), out.data_ptr(), *stride[:3], *to[:3], H), out


def rope(q, k, plan, grid=None, start=0, positions=None, inverse=False, out=None, stream=None):
    """Queries and keys turned by their positions in one launch.  q, k: CUDA bf16 / fp16 / fp32 [B, H, N, d] with any
    strides but contiguous rows (token-major projections as x.view(B, N, H, d).transpose(1, 2)); k may be None or have
    another number of heads.  ``plan``: a ``Rope``.

    Positions: ``positions``, CUDA int32 or int64 [N] or [B, N] ([N, axes], [B, N, axes] for more than one axis), or the
    place in a grid: with axes = 3 and grid=(rows, cols) token n stands at frame start + n // (rows cols), row
    n // cols % rows, column n % cols; with two axes and grid=(cols,) at (start + n // cols, n % cols); with one at
    start + n.  ``inverse=True`` turns back, which is also the gradient.  ``out``: tensors to write, of any strides (a
    part of a K window), or the operands themselves; new contiguous ones by default.  Returns (q', k'), or q' without k."""
    kind = _TYPES.get(q.dtype)
    if kind is None or not q.is_cuda or q.dim() != 4:
        raise TypeError(_ROPE_OPERAND)
    ctx = _elsewhere(q, stream)
    if ctx is not None:
        with ctx:
            return rope(q, k, plan, grid, start, positions, inverse, out)
    shape, stride = q.shape, q.stride()
    B, _, N, d = shape
    if stride[3] != 1:
        raise TypeError(_ROPE_OPERAND)
    if d != plan.d:
        raise ValueError("q and k must have the plan's head width")
    if plan.turns.device != q.device:
        raise ValueError("the plan is on another device than the tensors")
    q_out, k_out = (None, None) if out is None else (out if isinstance(out, (tuple, list)) else (out, None))
    q_op, q_out = _rope_operand(q, shape, stride, q_out)
    if k is None:
        k_op = _NO_OPERAND
    else:
        k_shape, k_stride = k.shape, k.stride()
        if k.dtype != q.dtype or k.device != q.device or len(k_shape) != 4 or k_stride[3] != 1:
            raise TypeError(_ROPE_OPERAND + ", of one type and on one device")
        if k_shape[0] != B or k_shape[2] != N or k_shape[3] != d:
            raise ValueError("q and k must have one head width, number of sequences and number of tokens")
        k_op, k_out = _rope_operand(k, k_shape, k_stride, k_out)
    if not -2**63 <= start < 2**63:
        raise ValueError("start must fit 64 bits")
    axes = len(plan.sections)
    at = bits = rows = cols = stride_b = stride_n = 0
    if positions is not None:
        if grid is not None or start != 0:
            raise ValueError("give either positions or a grid and a start")
        tail = () if axes == 1 else (axes,)
        if positions.dtype not in (torch.int32, torch.int64) or positions.device != q.device:
            raise TypeError("positions must be int32 or int64 on the tensors' device")
        strides = positions.stride()
        if positions.shape not in ((N,) + tail, (B, N) + tail) or (tail and strides[-1] != 1):
            raise ValueError(f"positions must have shape {(N,) + tail} or {(B, N) + tail}")
        at, bits = positions.data_ptr(), 32 if positions.dtype == torch.int32 else 64
        stride_b, stride_n = strides[:2] if len(strides) == 2 + len(tail) else (0, strides[0])
    elif axes > 1:
        if grid is None or len(grid) != axes - 1:
            raise ValueError(f"a plan of {axes} axes needs a grid of {axes - 1} sizes, or positions")
        rows, cols = (0, int(grid[0])) if axes == 2 else (int(grid[0]), int(grid[1]))
        if not (1 <= cols < 2**31 and (axes == 2 or 1 <= rows < 2**31)):
            raise ValueError("the sizes of a grid must be positive and fit 32 bits")
    elif grid is not None:
        raise ValueError("a plan of one axis takes no grid")
    rc = _load().rehyat_rope(_rope_operands.pack(*q_op, *k_op), 1 if k is None else 2, plan._ref,
                             _rope_positions.pack(at, stride_b, stride_n, int(start), bits, rows, cols), B, N,
                             kind, 1 if inverse else 0, _stream_handle(None))
    if rc != OK:
        raise RehyatError(rc, "rehyat_rope")
    return q_out if k is None else (q_out, k_out)


@functools.lru_cache(maxsize=1024)
def distill_loss_workspace_bytes(B, H, N, d):
    return _load().rehyat_distill_loss_workspace_bytes(B, H, N, d)


def distill_loss(y_hat, y, scale=None, weight=None, grad=None, loss=None, workspace=None, stream=None):
    """The loss of Eq. 19, scale * sum weight |y_hat - y|, and its gradient with respect to y_hat (bf16, what
    ``phi_backward`` takes as ``grad_out``).  y_hat: CUDA bf16 [B, H, N, d]; y: the same shape in bf16, fp16 or fp32;
    ``weight``: fp32 [B, N], 0 for tokens that do not count, whatever they hold.  ``scale`` is 1 / (number of elements)
    by default.  ``workspace``: a CUDA byte tensor of ``distill_loss_workspace_bytes`` (allocated here if None).
    Returns ``(loss, grad)``: one fp32 on the device, and a bf16 tensor like y_hat."""
    ctx = _elsewhere(y_hat, stream) if y_hat.is_cuda else None
    if ctx is not None:
        with ctx:
            return distill_loss(y_hat, y, scale, weight, grad, loss, workspace)
    lib = _load()
    if y_hat.dtype != torch.bfloat16 or not y_hat.is_cuda or not y_hat.is_contiguous() or y_hat.dim() != 4:
        raise TypeError("y_hat must be a contiguous CUDA bf16 tensor [B, H, N, d]")
    dev = y_hat.device
    if y.dtype not in _TYPES or y.device != dev or not y.is_contiguous():
        raise TypeError("y must be a contiguous CUDA tensor in bf16, fp16 or fp32 on y_hat's device")
    if y.shape != y_hat.shape:
        raise ValueError("y_hat and y shapes differ")
    B, H, N, d = y_hat.shape
    if weight is not None and (weight.dtype != torch.float32 or weight.device != dev or not weight.is_contiguous()
                               or weight.shape != (B, N)):
        raise TypeError("weight must be a contiguous CUDA fp32 tensor [B, N]")
    if grad is None:
        grad = torch.empty_like(y_hat)
    elif grad.shape != y_hat.shape or grad.dtype != torch.bfloat16 or grad.device != dev or not grad.is_contiguous():
        raise TypeError("grad must be a contiguous CUDA bf16 tensor like y_hat")
    if loss is None:
        loss = torch.empty((), device=dev, dtype=torch.float32)
    elif loss.numel() != 1 or loss.dtype != torch.float32 or loss.device != dev:
        raise TypeError("loss must be one CUDA fp32")
    if workspace is None:
        workspace = torch.empty(distill_loss_workspace_bytes(B, H, N, d), device=dev, dtype=torch.uint8)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous tensor on y_hat's device")
    if scale is None:
        scale = 1.0 / max(1, y_hat.numel())
    rc = lib.rehyat_distill_loss(y_hat.data_ptr(), y.data_ptr(), _TYPES[y.dtype],
                                 None if weight is None else weight.data_ptr(), scale, grad.data_ptr(), loss.data_ptr(),
                                 B, H, N, d, workspace.data_ptr(), workspace.nbytes, _stream_handle(None))
    if rc != OK:
        raise RehyatError(rc, "rehyat_distill_loss")
    return loss, grad


def _leaves(x):
    """The tensors of nested dicts, lists and tuples, in order."""
    if isinstance(x, torch.Tensor):
        return [x]
    return [t for v in (x.values() if isinstance(x, dict) else x) for t in _leaves(v)]


def _leaves_like(x, y):
    """The tensors of ``y`` in the order of those of ``x``, which has its structure: dicts go by their keys."""
    if isinstance(x, torch.Tensor) != isinstance(y, torch.Tensor) or isinstance(x, dict) != isinstance(y, dict) or \
            not isinstance(x, torch.Tensor) and (x.keys() != y.keys() if isinstance(x, dict) else len(x) != len(y)):
        raise ValueError("grads must have a tensor for each parameter, in the same structure")
    if isinstance(x, torch.Tensor):
        return [y]
    pairs = ((v, y[n]) for n, v in x.items()) if isinstance(x, dict) else zip(x, y)
    return [t for a, b in pairs for t in _leaves_like(a, b)]


def _like(x, tensors):
    """The structure of ``x`` with the tensors of an iterator in it."""
    if isinstance(x, torch.Tensor):
        return next(tensors)
    return {n: _like(v, tensors) for n, v in x.items()} if isinstance(x, dict) else [_like(v, tensors) for v in x]


def _offsets(sizes, step=256):
    """Where each of these many elements begins in one buffer, at multiples of ``step``; and the buffer's size."""
    out, at = [], 0
    for n in sizes:
        out.append(at)
        at += -(-n // step) * step
    return out, at


class AdamW:
    """AdamW over all of ``params`` (tensors in nested dicts and lists: the phi of one block, or a list of the phi of
    all; CUDA, contiguous, bf16 / fp16 / fp32), one launch a step.

    ``grads``, of the same structure (dicts by their keys) and shapes, in bf16, fp16 or fp32, are what a step reads; without them fp32 ones
    are made, to be written by ``phi_backward(grads=opt.grads)``.  A step goes by the addresses that parameters and
    gradients have here: assign into them (what replaces one in its dict, or its storage, is not seen).  ``master=True`` keeps an fp32 copy of parameters that
    are not fp32, which is what is updated (``reset_master`` after a change of the parameters from elsewhere).
    ``state_bits``: 32, or 8 for moments in 8 bits under an exponent for each 32 elements.  Those are rounded at random,
    by bits that depend on the step and the element alone, so that they follow the means of g and g^2; steps up to number
    ``nearest_steps``, which change them by more than their rounding does, to nearest (with many of those, and the usual
    betas, v stays far behind: see the header).

    ``lr``, ``betas``, ``eps``, ``weight_decay`` and ``nearest_steps`` may be set between steps.  State: ``m``, ``v`` (fp32, or e4m3 and
    uint8 with ``m_exp``, ``v_exp``), each one buffer in which tensor i begins at ``offsets[i]``; ``master``, likewise at
    ``master_offsets[i]`` (None: no copy); ``step_count``, on the device."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, master=True,
                 grads=None, nearest_steps=8):
        self.params = _leaves(params)
        self._names = list(params) if isinstance(params, dict) else None
        self.lr, self.betas, self.eps, self.weight_decay, self.state_bits = lr, betas, eps, weight_decay, state_bits
        self.nearest_steps = nearest_steps
        if not self.params:
            raise ValueError("no parameters")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        dev = self.params[0].device
        for p in self.params:
            if p.dtype not in _TYPES or not p.is_cuda or p.device != dev or not p.is_contiguous():
                raise TypeError("parameters must be contiguous CUDA tensors in bf16, fp16 or fp32 on one device")
        with torch.cuda.device(dev):
            self._allocate(params, grads, bool(master), dev)
            self._prepare(0)

    def _allocate(self, params, grads, master, dev):
        sizes = [p.numel() for p in self.params]
        self.offsets, total = _offsets(sizes)
        zeros = lambda n, dtype: torch.zeros(n, device=dev, dtype=dtype)
        if grads is None:
            flat = zeros(total, torch.float32)
            self._grads = [flat[o:o + n].view(p.shape) for o, n, p in zip(self.offsets, sizes, self.params)]
            self.grads = _like(params, iter(self._grads))
        else:
            self._grads, self.grads = _leaves_like(params, grads), grads
            for p, g in zip(self.params, self._grads):
                if g.dtype not in _TYPES or g.device != dev or not g.is_contiguous() or g.shape != p.shape:
                    raise TypeError("grads must be contiguous CUDA tensors shaped like the parameters")
        if self.state_bits == 32:
            self.m, self.v = zeros(total, torch.float32), zeros(total, torch.float32)
            self.m_exp = self.v_exp = None
        else:
            self.m, self.v = zeros(total, torch.float8_e4m3fn), zeros(total, torch.uint8)
            self.m_exp, self.v_exp = zeros(total // 32, torch.uint8), zeros(total // 32, torch.uint8)
        held = [n if master and p.dtype != torch.float32 else None for p, n in zip(self.params, sizes)]
        at, total = _offsets([n or 0 for n in held])
        self.master_offsets = [o if n is not None else None for o, n in zip(at, held)]
        self.master = zeros(total, torch.float32) if total else None
        self.reset_master()

    @torch.no_grad()   # parameters may be leaves of an autograd graph, of which the copies are no part
    def reset_master(self):
        """The fp32 copies <- the parameters as they are now."""
        held = [(self.master[o:o + p.numel()].view(p.shape), p) for p, o in zip(self.params, self.master_offsets) if o is not None]
        if held:
            torch._foreach_copy_(*zip(*held))   # 100 tensors: 100 us, with a call for each 590

    def _prepare(self, step):
        n = len(self.params)
        tensors, sizes = (AdamWTensor * n)(), (ctypes.c_int64 * n)()
        at = lambda buffer, element: None if buffer is None else buffer.data_ptr() + element * buffer.element_size()
        for i, (p, g, o, mo) in enumerate(zip(self.params, self._grads, self.offsets, self.master_offsets)):
            sizes[i] = p.numel()
            tensors[i] = AdamWTensor(p.data_ptr(), None if mo is None else at(self.master, mo), g.data_ptr(),
                                     at(self.m, o), at(self.v, o), at(self.m_exp, o // 32), at(self.v_exp, o // 32),
                                     p.numel(), _TYPES[p.dtype], _TYPES[g.dtype])
        lib = _load()
        need = lib.rehyat_adamw_table_bytes(sizes, n)
        if need == 0:
            raise RehyatError(E_SHAPE, "rehyat_adamw_table_bytes")
        self._table = torch.empty(need, device=self.m.device, dtype=torch.uint8)
        self.step_count = self._table[:8].view(torch.int64).view(())
        self._plan, self._hyper, self._method, self._step = AdamWPlan(), None, None, lib.rehyat_adamw_step
        rc = lib.rehyat_adamw_prepare(tensors, n, self.state_bits, step, self._table.data_ptr(), need,
                                      ctypes.byref(self._plan), _stream_handle(None))
        if rc != OK:
            raise RehyatError(rc, "rehyat_adamw_prepare")

    def step(self, lr=None, stream=None):
        """One update of every parameter from ``grads``.  ``lr``: a number for this step, or one fp32 on the device,
        which a captured step reads at every replay."""
        ctx = _elsewhere(self.m, stream)
        if ctx is not None:
            with ctx:
                return self.step(lr)
        lr, at = self.lr if lr is None else lr, None
        if isinstance(lr, torch.Tensor):
            if lr.dtype != torch.float32 or lr.numel() != 1 or lr.device != self.m.device:
                raise TypeError("lr must be a number or one fp32 on the parameters' device")
            lr, at = 0.0, lr.data_ptr()
        method = (lr, *self.betas, self.eps, self.weight_decay, at, self.nearest_steps)
        if method != self._method:   # the struct as it is otherwise: 1.2 of 6 us
            self._hyper, self._method = AdamWHyper(*method), method
        rc = self._step(ctypes.byref(self._plan), ctypes.byref(self._hyper), _stream_handle(None))
        if rc != OK:
            raise RehyatError(rc, "rehyat_adamw_step")

    def moments(self, out=None, stream=None):
        """(m, v) in fp32, laid out like the buffers of the state: those themselves with 32 bits, with 8 their values in
        new buffers or in ``out``."""
        if self.state_bits == 32:
            return self.m, self.v
        ctx = _elsewhere(self.m, stream)
        if ctx is not None:
            with ctx:
                return self.moments(out)
        n = self.m.numel()
        if out is None:
            out = [torch.empty(n, device=self.m.device, dtype=torch.float32) for _ in range(2)]
        for t in out:
            if t.dtype != torch.float32 or t.device != self.m.device or not t.is_contiguous() or t.numel() != n:
                raise TypeError("out must be two contiguous CUDA fp32 tensors as long as the state")
        m, v = out
        rc = _load().rehyat_adamw_moments(self.m.data_ptr(), self.m_exp.data_ptr(), self.v.data_ptr(),
                                          self.v_exp.data_ptr(), m.data_ptr(), v.data_ptr(), n, _stream_handle(None))
        if rc != OK:
            raise RehyatError(rc, "rehyat_adamw_moments")
        return m, v

    @torch.no_grad()
    def load_state(self, m, v, step, m_exp=None, v_exp=None, master=None):
        """Copies a state in (buffers as in ``m``, ``v``, ``m_exp``, ``v_exp``, ``master``; ``step`` updates made).  Without
        a ``master`` the fp32 copies are made of the parameters as they are now."""
        step = int(step)
        if not 0 <= step < 2**63:
            raise ValueError("step must not be negative, and fit 64 bits")
        given = [(self.m, m), (self.v, v), (self.m_exp, m_exp), (self.v_exp, v_exp)]
        if master is not None:
            given.append((self.master, master))
        for mine, other in given:
            if (mine is None) != (other is None):
                raise ValueError("the state is one of other bits")
            if mine is not None and (mine.shape != other.shape or mine.dtype != other.dtype):
                raise ValueError("the state has another shape or type")
        for mine, other in given:
            if mine is not None:
                mine.copy_(other)
        if master is None:
            self.reset_master()
        self.step_count.fill_(step)


def distill_gradients(q, k, v, y, phi, grads, T, HW, chunk, overlap=0, rope_plan=None, grid=None, start=0,
                      positions=None, weight=None, scale=None, workspace=None, stream=None):
    """Loss of one block's distillation (Eq. 19) on one batch, and the gradients of its feature maps, written to
    ``grads`` (a dict like ``phi``, fp32: an ``AdamW``'s): rotary positions (with a ``rope_plan``; q and k may then have
    any strides, see ``rope``), the forward pass, ``distill_loss`` against the teacher's output y, ``phi_backward`` on
    that same forward pass.  Tokens of ``weight`` 0 do not count, but their q, k and v must be finite: they go through
    the forward pass, and its gradient multiplies what comes of them by 0.  (Their y may hold anything.)  The forward pass
    uses the library-held workspace: order such calls on one stream.  Returns the loss, one fp32 on the device."""
    ctx = _elsewhere(q, stream) if q.is_cuda else None
    if ctx is not None:
        with ctx:
            return distill_gradients(q, k, v, y, phi, grads, T, HW, chunk, overlap, rope_plan, grid, start, positions,
                                     weight, scale, workspace)
    if rope_plan is None and (grid is not None or start != 0 or positions is not None):
        raise ValueError("positions need a rope_plan")
    if rope_plan is not None:
        if grid is not None and len(grid) == 2 and grid[0] * grid[1] != HW:
            raise ValueError("the grid's rows and columns do not make a frame of HW tokens")
        q, k = rope(q, k, rope_plan, grid=grid, start=start, positions=positions)
    _check_qkv(q, k, v)
    B, H, N, d = q.shape
    if N != T * HW:
        raise ValueError("N != T*HW")
    p, Hp = _phi_struct(phi, d)
    if Hp != H:
        raise ValueError("phi head count differs from q")
    out = torch.empty_like(q)
    nS, nL = (torch.empty(B, H, N, device=q.device, dtype=torch.float32) for _ in range(2))
    kept = DebugOut(nS=nS.data_ptr(), nL=nL.data_ptr())
    rc = _load().rehyat_forward_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), ctypes.byref(p), out.data_ptr(), B, H, T,
                                   HW, d, chunk, overlap, 1, STAB_ROWMAX, ctypes.byref(kept), _stream_handle(None))
    if rc != OK:
        raise RehyatError(rc, "rehyat_forward_ex")
    loss, g = distill_loss(out, y, scale=scale, weight=weight)
    phi_backward(q, k, v, phi, g, T, HW, chunk, overlap=overlap, workspace=workspace, grads=grads, saved=(out, nS, nL))
    return loss


def distill_step(q, k, v, y, phi, opt, T, HW, chunk, lr=None, stream=None, **kw):
    """One step of the distillation of one block: ``distill_gradients`` (which see for the other arguments), then
    phi <- AdamW(phi).  ``opt`` is an ``AdamW`` over ``phi``, a dict.  (Several blocks share one optimiser, and one
    launch, with AdamW([phi_0, phi_1, ...]), a ``distill_gradients`` into ``opt.grads[i]`` each, and ``opt.step()``.)
    Returns the loss before the update."""
    names = opt._names
    if names is None or set(names) != phi.keys() or opt.grads.keys() != phi.keys() or \
            any(a is not phi[n] for n, a in zip(names, opt.params)) or \
            any(a is not opt.grads[n] for n, a in zip(names, opt._grads)):
        raise ValueError("opt must be an AdamW over this phi, and its grads those it was made with")
    ctx = _elsewhere(q, stream) if q.is_cuda else None
    if ctx is not None:
        with ctx:
            return distill_step(q, k, v, y, phi, opt, T, HW, chunk, lr, **kw)
    loss = distill_gradients(q, k, v, y, phi, opt.grads, T, HW, chunk, **kw)
    opt.step(lr=lr)
    return loss
