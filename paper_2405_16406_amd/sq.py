"""ctypes binding of libsq.so (include/sq.h).

Argument marshalling only: tensors become device pointers, sizes become int64, the
current torch HIP stream becomes the `stream` argument.  Every step of the path runs in
the library's HIP kernels; there is no fallback.  A missing library raises.
Outputs are allocated with torch (device memory is torch's job here) unless passed in.
"""

import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsq.so")

SQ_OK, SQ_ERR_NULL, SQ_ERR_SHAPE, SQ_ERR_UNSUPPORTED, SQ_ERR_ALIGN, SQ_ERR_ALIAS, SQ_ERR_HIP = range(7)
STATUS_NAMES = {0: "SQ_OK", 1: "SQ_ERR_NULL", 2: "SQ_ERR_SHAPE", 3: "SQ_ERR_UNSUPPORTED",
                4: "SQ_ERR_ALIGN", 5: "SQ_ERR_ALIAS", 6: "SQ_ERR_HIP"}

EXPORTS = ("sq_abi_version", "sq_last_error", "sq_time_next_call", "sq_hadamard_factor", "sq_had_quant_act",
           "sq_had_quant_act_ex", "sq_pack_w4", "sq_pack_w4_ex", "sq_w4a4_linear", "sq_w4a8_linear",
           "sq_w4a4_linear_swiglu", "sq_qk_had_kvquant", "sq_qk_had_kvquant_ex", "sq_attn_decode_kv4",
           "sq_attn_decode_kv4_ex", "sq_attn_decode_workspace", "sq_attn_decode_kv4_split",
           "sq_attn_decode_kv4_split_noalloc", "sq_rope_frequencies", "sq_rope_kv_write", "sq_kv_read",
           "sq_attn_paged", "sq_attn_paged_workspace", "sq_attn_prompt", "sq_attn_prompt_workspace")


class SqError(RuntimeError):
    def __init__(self, status: int, where: str, msg: str):
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


_lib = None
_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I32 = ctypes.c_int32
_U64 = ctypes.c_uint64
_F32 = ctypes.c_float
_F64 = ctypes.c_double


def lib() -> ctypes.CDLL:
    """Load libsq.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2405_16406_amd.build`")
    _lib = load(LIB_PATH)
    return _lib


def load(path: str) -> ctypes.CDLL:
    """Open a build of the library at `path` and declare the signatures of include/sq.h."""
    L = ctypes.CDLL(path)
    L.sq_abi_version.restype = _I32
    L.sq_abi_version.argtypes = []
    L.sq_last_error.restype = ctypes.c_char_p
    L.sq_last_error.argtypes = []
    L.sq_time_next_call.restype = _I32
    L.sq_time_next_call.argtypes = [_P, _P]
    L.sq_hadamard_factor.restype = _I32
    L.sq_hadamard_factor.argtypes = [_I32, _P]
    L.sq_had_quant_act.restype = _I32
    L.sq_had_quant_act.argtypes = [_P, _I64, _I64, _I64, _I32, _P, _I32, _I32, _I32, _P, _P, _P, _P, _P]
    L.sq_had_quant_act_ex.restype = _I32
    L.sq_had_quant_act_ex.argtypes = [_P, _I64, _I64, _I64, _I32, _P, _I32, _P, _I32, _I32, _F32,
                                      _P, _P, _P, _P, _P]
    L.sq_pack_w4.restype = _I32
    L.sq_pack_w4.argtypes = [_P, _I64, _I64, _I64, _I32, _P, _I32, _P, _P, _P, _P]
    L.sq_pack_w4_ex.restype = _I32
    L.sq_pack_w4_ex.argtypes = [_P, _I64, _I64, _I64, _I32, _P, _I32, _P, _P, _P, _P, _P]
    L.sq_w4a4_linear.restype = _I32
    L.sq_w4a4_linear.argtypes = [_P, _P, _P, _I64, _P, _P, _P, _I64, _I64, _P, _P, _I64, _P, _P]
    L.sq_w4a8_linear.restype = _I32
    L.sq_w4a8_linear.argtypes = [_P, _P, _P, _I64, _P, _P, _P, _I64, _I64, _P, _P, _I64, _P, _P]
    L.sq_w4a4_linear_swiglu.restype = _I32
    L.sq_w4a4_linear_swiglu.argtypes = [_P, _P, _P, _I64, _P, _P, _P, _I64, _I64, _P, _P, _I64, _P]
    L.sq_qk_had_kvquant.restype = _I32
    L.sq_qk_had_kvquant.argtypes = [_P, _P, _P, _I64, _I64, _I64, _I64, _I32, _I32,
                                    _P, _P, _P, _P, _P, _P, _P, _P, _P]
    L.sq_qk_had_kvquant_ex.restype = _I32
    L.sq_qk_had_kvquant_ex.argtypes = [_P, _P, _P, _I64, _I64, _I64, _I64, _I32, _I32, _F32, _F32, _I32,
                                       _P, _P, _P, _P, _P, _P, _P, _P, _P]
    L.sq_attn_decode_kv4.restype = _I32
    L.sq_attn_decode_kv4.argtypes = [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I64, _F32, _P, _P]
    L.sq_attn_decode_kv4_ex.restype = _I32
    L.sq_attn_decode_kv4_ex.argtypes = [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I64, _F32, _I32, _P, _P]
    L.sq_attn_decode_workspace.restype = _I32
    L.sq_attn_decode_workspace.argtypes = [_I64, _I64, _I64, _I64, _P]
    L.sq_attn_decode_kv4_split.restype = _I32
    L.sq_attn_decode_kv4_split.argtypes = [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I64, _F32, _I32, _P, _P,
                                           ctypes.c_uint64, _P]
    L.sq_attn_decode_kv4_split_noalloc.restype = _I32
    L.sq_attn_decode_kv4_split_noalloc.argtypes = [_P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I64, _F32, _I32,
                                                   _P, _P]
    L.sq_rope_frequencies.restype = _I32
    L.sq_rope_frequencies.argtypes = [_I32, _F64, _I32, _F64, _F64, _F64, _F64, _P]
    L.sq_rope_kv_write.restype = _I32
    L.sq_rope_kv_write.argtypes = [_P, _I64, _P, _I64, _P, _I64, _I64, _I64, _I64, _P, _P, _I64, _P, _I64, _I64,
                                   _P, _P, _P, _I64, _I64, _I64, _I32, _I32, _P, _I32, _I32, _F32, _F32, _F32,
                                   _P, _P, _P]
    L.sq_kv_read.restype = _I32
    L.sq_kv_read.argtypes = [_P, _P, _I64, _I64, _P, _I64, _I64, _P, _P, _P, _I64, _I64, _I64, _I64, _I32, _I32,
                             _I32, _P, _I64, _P, _I64, _P]
    L.sq_attn_paged.restype = _I32
    L.sq_attn_paged.argtypes = [_P, _I64, _P, _I64, _P, _I64, _I64, _P, _P, _P, _I64, _I64, _I64, _I64, _I64, _I32,
                                _I32, _I64, _F32, _P, _I64, _P, _U64, _P]
    L.sq_attn_paged_workspace.restype = _I32
    L.sq_attn_paged_workspace.argtypes = [_I64, _I64, _I64, _I64, _I64, _P]
    L.sq_attn_prompt.restype = _I32
    L.sq_attn_prompt.argtypes = [_P, _I64, _P, _I64, _P, _I64, _P, _P, _I64, _I64, _I64, _I64, _I64, _I64, _F32,
                                 _I32, _P, _I64, _P, _U64, _P]
    L.sq_attn_prompt_workspace.restype = _I32
    L.sq_attn_prompt_workspace.argtypes = [_I64, _I64, _I64, _I64, _I64, _I64, _P]
    return L


def _check(status: int, where: str) -> None:
    if status != SQ_OK:
        raise SqError(status, where, lib().sq_last_error().decode())


# A call's host time is what a decode step of small kernels waits for, so the marshalling is
# kept short: plain integers (the argument types make them pointers), the raw stream without a
# torch.cuda.Stream object, no view of a tensor that is contiguous already.  Measured per call
# (us, launch included, against marshalling with pointer and stream objects): had_quant_act 8.2
# vs 10.9, w4a4_linear 7.0 vs 10.0, qk_had_kvquant 13.2 vs 18.3, attn_decode_kv4_split 9.6 vs
# 11.9; the launch alone is 2.9, each new output 1 - 1.3.

def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(t: torch.Tensor) -> int:
    """The current stream of t's device as an integer (a hipStream_t)."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _flat(t: torch.Tensor) -> torch.Tensor:
    """t's values in order: t itself where they are contiguous."""
    return t if t.is_contiguous() else t.reshape(-1)


def _need(t: torch.Tensor, dtype, name: str):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_cuda:
        raise TypeError(f"{name} must be a {dtype} tensor on the GPU")


def _workspace_bytes(t: torch.Tensor) -> int:
    """The bytes of a caller's workspace: its elements must lie side by side, since the call writes as
    many bytes from its first on (those of a strided or expanded one would be other memory)."""
    if isinstance(t, torch.Tensor) and not t.is_contiguous():
        raise ValueError("workspace must be contiguous")
    _need(t, torch.uint8, "workspace")
    return t.numel()


def abi_version() -> int:
    return int(lib().sq_abi_version())


def time_next_call(start: "torch.cuda.Event", stop: "torch.cuda.Event") -> None:
    """Arm two timing events (torch.cuda.Event(enable_timing=True)) for this thread's next
    library call: start.elapsed_time(stop) is then that call's kernel time on the device."""
    for e in (start, stop):
        if e.cuda_event == 0:  # torch creates the HIP event on its first record
            e.record()
    _check(lib().sq_time_next_call(ctypes.c_void_p(start.cuda_event), ctypes.c_void_p(stop.cuda_event)),
           "sq_time_next_call")


def hadamard_factor(n: int) -> np.ndarray:
    """The library's +-1 Hadamard matrix of order n (1, 28, 172) as int8 [n, n] (host)."""
    out = np.empty((n, n), dtype=np.int8)
    _check(lib().sq_hadamard_factor(n, out.ctypes.data_as(ctypes.c_void_p)), "sq_hadamard_factor")
    return out


def had_quant_act(x: torch.Tensor, had: torch.Tensor | None = None, pow2: int = 1,
                  group: int | None = None, bits: int = 4, dbg: bool = False, out=None,
                  clip: float = 1.0, signs: torch.Tensor | None = None):
    """Rotate rows of x (fp16 [M, K], row stride x.stride(0)) and quantize (asym, 4 or 8 bits).

    had: int8 +-1 [a, a] on the device or None.  clip (range clipping ratio in (0, 1]) and
    signs (int8 +-1 [a * pow2] on the device: the random Hadamard S H) select sq_had_quant_act_ex.
    Returns (q uint8 [M, K/2] (4-bit) or [M, K] (8-bit), alpha fp32 [M, K/group],
    beta fp32 [M, K/group], dbg_rot fp32 [M, K] or None).
    """
    _need(x, torch.float16, "x")
    if x.dim() != 2 or x.stride(1) != 1:
        raise ValueError("x must be 2-D with unit column stride")
    M, K = x.shape
    group = K if group is None else group
    a = 1 if had is None else had.shape[0]
    if had is not None:
        _need(had, torch.int8, "had")
    if out is None:
        q = x.new_empty((M, K * bits // 8), dtype=torch.uint8)
        al = x.new_empty((M, K // group), dtype=torch.float32)
        be = torch.empty_like(al)
    else:
        q, al, be = out
    rot = x.new_empty((M, K), dtype=torch.float32) if dbg else None
    if clip == 1.0 and signs is None:
        _check(lib().sq_had_quant_act(_ptr(x), M, K, x.stride(0), a, _ptr(had), pow2, bits, group,
                                      _ptr(q), _ptr(al), _ptr(be), _ptr(rot), _stream(x)), "sq_had_quant_act")
    else:
        if signs is not None:
            _need(signs, torch.int8, "signs")
        _check(lib().sq_had_quant_act_ex(_ptr(x), M, K, x.stride(0), a, _ptr(had), pow2, _ptr(signs), bits, group,
                                         float(clip), _ptr(q), _ptr(al), _ptr(be), _ptr(rot), _stream(x)),
               "sq_had_quant_act_ex")
    return q, al, be, rot


def pack_w4(w: torch.Tensor, had: torch.Tensor | None = None, pow2: int = 1, signs: torch.Tensor | None = None):
    """Offline: W' = W R (optional), symmetric per-row 4-bit quant, pack.

    signs (int8 +-1 [a * pow2] on the device) fold the random Hadamard S H instead
    (sq_pack_w4_ex).  Returns (wq uint8 [N, K/2], w_alpha fp32 [N], w_rowsum int32 [N]).
    """
    _need(w, torch.float16, "w")
    if w.dim() != 2 or w.stride(1) != 1:
        raise ValueError("w must be 2-D with unit column stride")
    N, K = w.shape
    a = 1 if had is None else had.shape[0]
    dev = w.device
    wq = torch.empty((N, K // 2), dtype=torch.uint8, device=dev)
    wa = torch.empty((N,), dtype=torch.float32, device=dev)
    rs = torch.empty((N,), dtype=torch.int32, device=dev)
    if signs is None:
        _check(lib().sq_pack_w4(_ptr(w), N, K, w.stride(0), a, _ptr(had), pow2, _ptr(wq), _ptr(wa), _ptr(rs),
                                _stream(w)), "sq_pack_w4")
    else:
        _need(signs, torch.int8, "signs")
        _check(lib().sq_pack_w4_ex(_ptr(w), N, K, w.stride(0), a, _ptr(had), pow2, _ptr(signs), _ptr(wq), _ptr(wa),
                                   _ptr(rs), _stream(w)), "sq_pack_w4_ex")
    return wq, wa, rs


def w4a4_linear(xq, x_alpha, x_beta, wq, w_alpha, w_rowsum, bias=None, out=None, dbg=False):
    """y = fp16(s_n (alpha_m acc + beta_m rowsum_n) + bias_n) with acc the exact int GEMM.

    Returns (y fp16 [M, N], acc int32 [M, N] or None).
    """
    _need(xq, torch.uint8, "xq")
    _need(wq, torch.uint8, "wq")
    M, KB = xq.shape
    N = wq.shape[0]
    if wq.shape[1] != KB:
        raise ValueError("xq and wq disagree on K")
    K = 2 * KB
    y = xq.new_empty((M, N), dtype=torch.float16) if out is None else out
    acc = xq.new_empty((M, N), dtype=torch.int32) if dbg else None
    x_alpha, x_beta = _flat(x_alpha), _flat(x_beta)
    _check(lib().sq_w4a4_linear(_ptr(xq), _ptr(x_alpha), _ptr(x_beta), M, _ptr(wq), _ptr(w_alpha), _ptr(w_rowsum),
                                N, K, _ptr(bias), _ptr(y), y.stride(0), _ptr(acc), _stream(xq)), "sq_w4a4_linear")
    return y, acc


def w4a8_linear(xq, x_alpha, x_beta, wq, w_alpha, w_rowsum, bias=None, out=None, dbg=False):
    """y = fp16(s_n (alpha_m acc + beta_m rowsum_n) + bias_n) with 8-bit activation codes
    xq uint8 [M, K] (had_quant_act bits=8) and packed 4-bit weights wq uint8 [N, K/2].
    Returns (y fp16 [M, N], acc int32 [M, N] or None).
    """
    _need(xq, torch.uint8, "xq")
    _need(wq, torch.uint8, "wq")
    M, K = xq.shape
    N = wq.shape[0]
    if 2 * wq.shape[1] != K:
        raise ValueError("xq and wq disagree on K")
    y = xq.new_empty((M, N), dtype=torch.float16) if out is None else out
    acc = xq.new_empty((M, N), dtype=torch.int32) if dbg else None
    x_alpha, x_beta = _flat(x_alpha), _flat(x_beta)
    _check(lib().sq_w4a8_linear(_ptr(xq), _ptr(x_alpha), _ptr(x_beta), M, _ptr(wq), _ptr(w_alpha), _ptr(w_rowsum),
                                N, K, _ptr(bias), _ptr(y), y.stride(0), _ptr(acc), _stream(xq)), "sq_w4a8_linear")
    return y, acc


def w4a4_linear_swiglu(xq, x_alpha, x_beta, wq, w_alpha, w_rowsum, bias=None, out=None):
    """h = fp16(SiLU(gate) * up) from gate/up weights packed as one matrix whose rows
    interleave them in blocks of 32 (see interleave_gate_up).  Returns h fp16 [M, N/2].
    """
    _need(xq, torch.uint8, "xq")
    _need(wq, torch.uint8, "wq")
    M, KB = xq.shape
    N = wq.shape[0]
    if wq.shape[1] != KB:
        raise ValueError("xq and wq disagree on K")
    h = xq.new_empty((M, N // 2), dtype=torch.float16) if out is None else out
    x_alpha, x_beta = _flat(x_alpha), _flat(x_beta)
    _check(lib().sq_w4a4_linear_swiglu(_ptr(xq), _ptr(x_alpha), _ptr(x_beta), M, _ptr(wq), _ptr(w_alpha),
                                       _ptr(w_rowsum), N, 2 * KB, _ptr(bias), _ptr(h), h.stride(0), _stream(xq)),
           "sq_w4a4_linear_swiglu")
    return h


def interleave_gate_up(gate: torch.Tensor, up: torch.Tensor) -> torch.Tensor:
    """Rows of gate [I, ...] and up [I, ...] interleaved in blocks of 32 (I % 32 == 0): the
    row order sq_w4a4_linear_swiglu expects of its weights, scales, row sums and bias."""
    I = gate.shape[0]
    if up.shape != gate.shape or I % 32:
        raise ValueError("gate and up need the same shape with a multiple of 32 rows")
    return torch.stack([gate.reshape(I // 32, 32, *gate.shape[1:]), up.reshape(I // 32, 32, *up.shape[1:])],
                       dim=1).reshape(2 * I, *gate.shape[1:])


def qk_had_kvquant(q, k, v, dbg: bool = False, out=None, bits: int = 4, k_clip: float = 1.0,
                   v_clip: float = 1.0, param_dtype=torch.float32):
    """R3 on Q and K per head (D = 128) + 4-bit (or 8-bit) asymmetric K/V quantization, group 128.

    k_clip, v_clip: range clipping ratios in (0, 1]; param_dtype torch.float32 or
    torch.float16 for the group parameters (either away from the default:
    sq_qk_had_kvquant_ex).  Returns dict(q_rot, k_q, k_alpha, k_beta, v_q, v_alpha, v_beta,
    k_rot (or None)).
    """
    for t, nme in ((q, "q"), (k, "k"), (v, "v")):
        _need(t, torch.float16, nme)
        if not t.is_contiguous():
            raise ValueError(f"{nme} must be contiguous")
    B, S, H, D = q.shape
    if out is None:
        k_q = q.new_empty((B, S, H, D * bits // 8), dtype=torch.uint8)
        k_alpha = q.new_empty((B, S, H, 1), dtype=param_dtype)
        out = dict(q_rot=torch.empty_like(q), k_q=k_q, k_alpha=k_alpha, k_beta=torch.empty_like(k_alpha),
                   v_q=torch.empty_like(k_q), v_alpha=torch.empty_like(k_alpha), v_beta=torch.empty_like(k_alpha))
    pbits = {torch.float32: 32, torch.float16: 16}[param_dtype]
    for nme in ("k_alpha", "k_beta", "v_alpha", "v_beta"):
        _need(out[nme], param_dtype, nme)
    kr = q.new_empty((B, S, H, D), dtype=torch.float32) if dbg else None
    outs = (_ptr(out["q_rot"]), _ptr(out["k_q"]), _ptr(out["k_alpha"]), _ptr(out["k_beta"]), _ptr(out["v_q"]),
            _ptr(out["v_alpha"]), _ptr(out["v_beta"]), _ptr(kr), _stream(q))
    if k_clip == 1.0 and v_clip == 1.0 and pbits == 32:
        _check(lib().sq_qk_had_kvquant(_ptr(q), _ptr(k), _ptr(v), B, S, H, D, bits, 128, *outs), "sq_qk_had_kvquant")
    else:
        _check(lib().sq_qk_had_kvquant_ex(_ptr(q), _ptr(k), _ptr(v), B, S, H, D, bits, 128, float(k_clip),
                                          float(v_clip), pbits, *outs), "sq_qk_had_kvquant_ex")
    out = dict(out)
    out["k_rot"] = kr
    return out


def attn_decode_workspace_bytes(B, S, H, D=128):
    """Device bytes of the workspace attn_decode_kv4_split needs on the current device."""
    n = ctypes.c_uint64(0)
    _check(lib().sq_attn_decode_workspace(B, S, H, D, ctypes.byref(n)), "sq_attn_decode_workspace")
    return n.value


def attn_decode_kv4_split(q_rot, k_q, k_alpha, k_beta, v_q, v_alpha, v_beta, scale=None, out=None, workspace=None):
    """attn_decode_kv4 split over the sequence (sq_attn_decode_kv4_split).  workspace: a
    uint8 device tensor of at least attn_decode_workspace_bytes() bytes, allocated here
    when None.  Returns out fp16 [B, H, 128]."""
    _need(q_rot, torch.float16, "q_rot")
    for t, nme in ((q_rot, "q_rot"), (k_q, "k_q"), (v_q, "v_q"), (k_alpha, "k_alpha"), (k_beta, "k_beta"),
                   (v_alpha, "v_alpha"), (v_beta, "v_beta")):
        if not t.is_contiguous():
            raise ValueError(f"{nme} must be contiguous")
    B, H, D = q_rot.shape
    S = k_q.shape[1]
    scale = 1.0 / D ** 0.5 if scale is None else scale
    out = torch.empty_like(q_rot) if out is None else out
    pdt = k_alpha.dtype
    for t, nme in ((k_alpha, "k_alpha"), (k_beta, "k_beta"), (v_alpha, "v_alpha"), (v_beta, "v_beta")):
        _need(t, pdt, nme)
    if workspace is None:
        workspace = torch.empty(max(attn_decode_workspace_bytes(B, S, H, D), 1), dtype=torch.uint8,
                                device=q_rot.device)
    size = _workspace_bytes(workspace)
    _check(lib().sq_attn_decode_kv4_split(_ptr(q_rot), _ptr(k_q), _ptr(k_alpha), _ptr(k_beta), _ptr(v_q),
                                          _ptr(v_alpha), _ptr(v_beta), B, S, H, D, float(scale),
                                          {torch.float32: 32, torch.float16: 16}[pdt], _ptr(out), _ptr(workspace),
                                          size, _stream(q_rot)), "sq_attn_decode_kv4_split")
    return out


def attn_decode_kv4_split_noalloc(q_rot, k_q, k_alpha, k_beta, v_q, v_alpha, v_beta, scale=None, out=None):
    """attn_decode_kv4_split with the library's own scratch (sq_attn_decode_kv4_split_noalloc):
    the call allocates no device memory (out must then be given).  Returns out."""
    _need(q_rot, torch.float16, "q_rot")
    for t, nme in ((q_rot, "q_rot"), (k_q, "k_q"), (v_q, "v_q"), (k_alpha, "k_alpha"), (k_beta, "k_beta"),
                   (v_alpha, "v_alpha"), (v_beta, "v_beta")):
        if not t.is_contiguous():
            raise ValueError(f"{nme} must be contiguous")
    B, H, D = q_rot.shape
    S = k_q.shape[1]
    scale = 1.0 / D ** 0.5 if scale is None else scale
    out = torch.empty_like(q_rot) if out is None else out
    pdt = k_alpha.dtype
    for t, nme in ((k_alpha, "k_alpha"), (k_beta, "k_beta"), (v_alpha, "v_alpha"), (v_beta, "v_beta")):
        _need(t, pdt, nme)
    _check(lib().sq_attn_decode_kv4_split_noalloc(_ptr(q_rot), _ptr(k_q), _ptr(k_alpha), _ptr(k_beta), _ptr(v_q),
                                                  _ptr(v_alpha), _ptr(v_beta), B, S, H, D, float(scale),
                                                  {torch.float32: 32, torch.float16: 16}[pdt], _ptr(out),
                                                  _stream(q_rot)), "sq_attn_decode_kv4_split_noalloc")
    return out


def attn_decode_kv4(q_rot, k_q, k_alpha, k_beta, v_q, v_alpha, v_beta, scale=None, out=None):
    """Attention of one rotated query per (batch, head), q_rot fp16 [B, H, 128], over the
    4-bit cache of qk_had_kvquant (k_q, v_q uint8 [B, S, H, 64], group parameters fp32, or
    fp16 through sq_attn_decode_kv4_ex, [B, S, H(, 1)]).  Returns out fp16 [B, H, 128]."""
    _need(q_rot, torch.float16, "q_rot")
    for t, nme in ((q_rot, "q_rot"), (k_q, "k_q"), (v_q, "v_q"), (k_alpha, "k_alpha"), (k_beta, "k_beta"),
                   (v_alpha, "v_alpha"), (v_beta, "v_beta")):
        if not t.is_contiguous():
            raise ValueError(f"{nme} must be contiguous")
    B, H, D = q_rot.shape
    S = k_q.shape[1]
    scale = 1.0 / D ** 0.5 if scale is None else scale
    out = torch.empty_like(q_rot) if out is None else out
    pdt = k_alpha.dtype
    for t, nme in ((k_alpha, "k_alpha"), (k_beta, "k_beta"), (v_alpha, "v_alpha"), (v_beta, "v_beta")):
        _need(t, pdt, nme)
    if pdt == torch.float32:
        _check(lib().sq_attn_decode_kv4(_ptr(q_rot), _ptr(k_q), _ptr(k_alpha), _ptr(k_beta), _ptr(v_q),
                                        _ptr(v_alpha), _ptr(v_beta), B, S, H, D, float(scale), _ptr(out),
                                        _stream(q_rot)), "sq_attn_decode_kv4")
    else:
        _check(lib().sq_attn_decode_kv4_ex(_ptr(q_rot), _ptr(k_q), _ptr(k_alpha), _ptr(k_beta), _ptr(v_q),
                                           _ptr(v_alpha), _ptr(v_beta), B, S, H, D, float(scale),
                                           {torch.float16: 16}[pdt], _ptr(out), _stream(q_rot)),
               "sq_attn_decode_kv4_ex")
    return out


# ------------------------------------------------------------------ the paged cache

_ROPE_SCALING = {"none": 0, "linear": 1, "by parts": 2}
_PARAM_BITS = {torch.float32: 32, torch.float16: 16}


def rope_frequencies(rotary_dim: int = 128, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     low: float = 1.0, high: float = 4.0, original_len: float = 8192.0, device=None) -> torch.Tensor:
    """Angle per position of each pair of dims, fp64 [rotary_dim / 2] (sq_rope_frequencies) on
    `device`.  scaling "none", "linear" (divided by factor) or "by parts" (kept above `high` turns
    within original_len positions, divided by factor below `low`, mixed between)."""
    out = np.empty(max(rotary_dim, 0) // 2, dtype=np.float64)
    if scaling not in _ROPE_SCALING:
        raise ValueError(f"scaling must be one of {sorted(_ROPE_SCALING)}")
    _check(lib().sq_rope_frequencies(rotary_dim, theta, _ROPE_SCALING[scaling], factor, low, high, original_len,
                                     out.ctypes.data), "sq_rope_frequencies")
    return torch.from_numpy(out).to(device) if device is not None else torch.from_numpy(out)


def kv_cache(pages: int, page: int, heads: int, bits: int = 4, param_dtype=torch.float32, device="cuda"):
    """An empty paged cache (k_q, v_q, params): codes uint8 [pages, heads, page, 64 (4 bits) or 128],
    group parameters [pages, heads, page, 4] (k_alpha, k_beta, v_alpha, v_beta).  Zeroed."""
    k_q = torch.zeros((pages, heads, page, 16 * bits), dtype=torch.uint8, device=device)
    return k_q, torch.zeros_like(k_q), torch.zeros((pages, heads, page, 4), dtype=param_dtype, device=device)


# A decode step is two of the calls below on small tensors, and their host time is most of it: checks
# use each property once, and the device is switched only where another one is current.
_F16, _U8, _I32T, _F64T = torch.float16, torch.uint8, torch.int32, torch.float64
_current_device = torch._C._cuda_getDevice


def _heads(t, name):
    """(rows, heads, ld) of fp16 [rows, heads, 128] whose heads are contiguous."""
    if not isinstance(t, torch.Tensor) or t.dtype is not _F16 or not t.is_cuda:
        raise TypeError(f"{name} must be a torch.float16 tensor on the GPU")
    shape = t.shape
    if len(shape) != 3 or shape[2] != 128:
        raise ValueError(f"{name} must be [rows, heads, 128]")
    rows, heads, _ = shape
    ld, sh, sd = t.stride()
    if sd != 1 or (sh != 128 and heads > 1):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    return rows, heads, ld if rows > 1 else heads * 128


def _index(t, name, n=None):
    """A contiguous int32 vector (of n entries) on the GPU."""
    if not isinstance(t, torch.Tensor) or t.dtype is not _I32T or not t.is_cuda:
        raise TypeError(f"{name} must be a torch.int32 tensor on the GPU")
    if t.dim() != 1 or not t.is_contiguous() or (n is not None and t.shape[0] != n):
        raise ValueError(f"{name} must be a contiguous vector" + ("" if n is None else f" of {n} entries"))
    return t.shape[0]


def _cache_args(cache, table, B):
    """The cache's arguments: table, its stride and columns, the three tensors, pages, page, heads; and
    (bits, param_bits)."""
    k_q, v_q, params = cache
    if not (isinstance(k_q, torch.Tensor) and isinstance(v_q, torch.Tensor) and k_q.dtype is v_q.dtype is _U8):
        raise TypeError("k_q and v_q must be torch.uint8 tensors on the GPU")
    if not isinstance(params, torch.Tensor) or params.dtype not in _PARAM_BITS:
        raise TypeError("params must be a torch.float32 or torch.float16 tensor on the GPU")
    if not isinstance(table, torch.Tensor) or table.dtype is not _I32T:
        raise TypeError("block_table must be a torch.int32 tensor on the GPU")
    shape = k_q.shape
    if len(shape) != 4 or v_q.shape != shape or params.shape != (shape[0], shape[1], shape[2], 4):
        raise ValueError("the cache is codes [pages, heads, page, bytes] twice and parameters [pages, heads, page, 4]")
    if not (k_q.is_contiguous() and v_q.is_contiguous() and params.is_contiguous()):
        raise ValueError("the cache's tensors must be contiguous")
    pages, heads, page, row = shape
    if row != 64 and row != 128:
        raise ValueError("a token's codes are 64 (4 bits) or 128 (8 bits) bytes")
    if table.dim() != 2 or table.shape[0] != B or (table.stride(1) != 1 and table.shape[1] > 1):
        raise ValueError(f"block_table must be [{B}, blocks] with unit column stride")
    cols = table.shape[1]
    return ((table.data_ptr(), table.stride(0) if B > 1 else cols, cols, k_q.data_ptr(), v_q.data_ptr(), params.data_ptr(),
             pages, page, heads), (row // 16, _PARAM_BITS[params.dtype]))


def _same_device(t, *others):
    """The device of t, which all other tensors must be on."""
    d = t.get_device()
    for o in others:
        if o is not None and o.get_device() != d:
            raise ValueError("all tensors of a call must be on one GPU")
    return d


def rope_kv_write(q, k, v, cache, block_table, lens, freq=None, cu=None, interleaved: bool = False, magnitude: float = 1.0,
                  k_clip: float = 1.0, v_clip: float = 1.0, out=None, k_out=None):
    """Rotary positions and R3 on q, k and the quantized write of k, v into the pages
    (sq_rope_kv_write).  q fp16 [T, Hq, 128], k, v fp16 [T, Hkv, 128] before positions (slices of a
    fused projection are fine); lens int32 [B] with the new tokens; cu int32 [B + 1], or None for one
    token a sequence; freq fp64 [rotary_dim / 2] (rope_frequencies), None for no positions.
    k_out: optional fp16 [T, Hkv, 128] that takes the rotated keys.  Returns q rotated, fp16 [T, Hq, 128]."""
    T, Hq, ldq = _heads(q, "q")
    tk, Hkv, ldk = _heads(k, "k")
    tv, hv, ldv = _heads(v, "v")
    if tk != T or tv != T or hv != Hkv:
        raise ValueError("q, k and v disagree on their rows or heads")
    B = _index(lens, "lens")
    if cu is not None:
        _index(cu, "cu", B + 1)
    args, bits = _cache_args(cache, block_table, B)
    if args[-1] != Hkv:
        raise ValueError("k and the cache disagree on their heads")
    rotary = 0
    if freq is not None:
        _need(freq, torch.float64, "freq")
        if freq.dim() != 1 or not freq.is_contiguous():
            raise ValueError("freq must be a contiguous vector")
        rotary = 2 * freq.shape[0]
    for t, h, n in ((out, Hq, "out"), (k_out, Hkv, "k_out")):
        if t is not None:
            _need(t, torch.float16, n)
            if tuple(t.shape) != (T, h, 128) or not t.is_contiguous():
                raise ValueError(f"{n} must be contiguous [{T}, {h}, 128]")
    if out is None:
        out = q.new_empty((T, Hq, 128))
    d = _same_device(q, k, v, *cache, block_table, lens, cu, freq, out, k_out)
    if T == 0 or B == 0:  # an empty tensor has no address
        return out
    if d != _current_device():
        with torch.cuda.device(d):
            return rope_kv_write(q, k, v, cache, block_table, lens, freq, cu, interleaved, magnitude, k_clip, v_clip, out, k_out)
    status = lib().sq_rope_kv_write(q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, T, Hq, 128, _ptr(cu),
                                    lens.data_ptr(), B, *args, *bits, _ptr(freq), rotary, int(interleaved), magnitude,
                                    k_clip, v_clip, out.data_ptr(), _ptr(k_out), _stream(q))
    if status:
        _check(status, "sq_rope_kv_write")
    return out


def kv_read(cache, block_table, lens, cu, rows: int, plain_basis: bool = False, out=None):
    """Keys and values of the sequences' last tokens out of the pages (sq_kv_read): (k, v) fp16
    [rows, Hkv, 128] packed by cu int32 [B + 1], keys in R3's basis, or turned back with plain_basis.
    Rows of no sequence are left as they are in `out` (a pair of tensors; allocated unset when None)."""
    B = _index(lens, "lens")
    _index(cu, "cu", B + 1)
    args, bits = _cache_args(cache, block_table, B)
    Hkv = args[-1]
    if out is None:
        k = cache[2].new_empty((rows, Hkv, 128), dtype=torch.float16)
        v = torch.empty_like(k)
    else:
        k, v = out
    tk, hk, ldk = _heads(k, "k")
    tv, hv, ldv = _heads(v, "v")
    if (tk, hk, tv, hv) != (rows, Hkv, rows, Hkv):
        raise ValueError(f"out must be two [{rows}, {Hkv}, 128] tensors")
    d = _same_device(k, v, *cache, block_table, lens, cu)
    if rows == 0 or B == 0:
        return k, v
    if d != _current_device():
        with torch.cuda.device(d):
            return kv_read(cache, block_table, lens, cu, rows, plain_basis, (k, v))
    status = lib().sq_kv_read(cu.data_ptr(), lens.data_ptr(), B, rows, *args, 128, *bits, int(plain_basis), k.data_ptr(), ldk,
                              v.data_ptr(), ldv, _stream(k))
    if status:
        _check(status, "sq_kv_read")
    return k, v


def attn_paged_workspace_bytes(B, max_len, Hq, Hkv):
    """Device bytes of attn_paged's workspace on the current device."""
    n = _U64(0)
    _check(lib().sq_attn_paged_workspace(B, max_len, Hq, Hkv, 128, ctypes.byref(n)), "sq_attn_paged_workspace")
    return n.value


def attn_paged(q, cache, block_table, lens, max_len: int, scale=None, out=None, workspace=None):
    """Attention of one rotated query per sequence over its pages (sq_attn_paged): q fp16
    [B, Hq, 128]; max_len at least the longest of lens.  workspace: a uint8 device tensor of at least
    attn_paged_workspace_bytes() bytes, allocated here when None.  Returns out fp16 [B, Hq, 128]."""
    B, Hq, ldq = _heads(q, "q")
    _index(lens, "lens", B)
    args, bits = _cache_args(cache, block_table, B)
    if out is None:
        out, ldo = q.new_empty((B, Hq, 128)), Hq * 128
    else:
        to, ho, ldo = _heads(out, "out")
        if (to, ho) != (B, Hq):
            raise ValueError(f"out must be [{B}, {Hq}, 128]")
    d = _same_device(q, *cache, block_table, lens, out, workspace)
    if B == 0:
        return out
    if d != _current_device():
        with torch.cuda.device(d):
            return attn_paged(q, cache, block_table, lens, max_len, scale, out, workspace)
    if workspace is None:
        size = attn_paged_workspace_bytes(B, max_len, Hq, args[-1])
        workspace = q.new_empty(size, dtype=_U8) if size else None
    else:
        size = _workspace_bytes(workspace)
    status = lib().sq_attn_paged(q.data_ptr(), ldq, lens.data_ptr(), B, *args, Hq, 128, *bits, max_len,
                                 0.08838834764831845 if scale is None else scale, out.data_ptr(), ldo, _ptr(workspace), size,
                                 _stream(q))
    if status:
        _check(status, "sq_attn_paged")
    return out


def attn_prompt_workspace_bytes(B, Tq, Tk, Hq, Hkv):
    """Device bytes of attn_prompt's workspace on the current device."""
    n = _U64(0)
    _check(lib().sq_attn_prompt_workspace(B, Tq, Tk, Hq, Hkv, 128, ctypes.byref(n)), "sq_attn_prompt_workspace")
    return n.value


def attn_prompt(q, k, v, cu_q, cu_k, scale=None, causal: bool = True, out=None, workspace=None):
    """Attention of packed sequences (sq_attn_prompt): q fp16 [Tq, Hq, 128], k, v fp16 [Tk, Hkv, 128],
    sequence b the rows cu_q[b] .. of q and cu_k[b] .. of k and v (int32 [B + 1] each); causal: its
    queries are its last tokens.  workspace: a uint8 device tensor of at least
    attn_prompt_workspace_bytes() bytes, allocated here when None.  Returns out fp16 [Tq, Hq, 128]; rows
    of no sequence are left as they are in `out` (allocated unset when None)."""
    Tq, Hq, ldq = _heads(q, "q")
    Tk, Hkv, ldk = _heads(k, "k")
    tv, hv, ldv = _heads(v, "v")
    if tv != Tk or hv != Hkv:
        raise ValueError("k and v disagree on their rows or heads")
    B = _index(cu_q, "cu_q") - 1
    _index(cu_k, "cu_k", B + 1)
    if out is None:
        out, ldo = q.new_empty((Tq, Hq, 128)), Hq * 128
    else:
        to, ho, ldo = _heads(out, "out")
        if (to, ho) != (Tq, Hq):
            raise ValueError(f"out must be [{Tq}, {Hq}, 128]")
    d = _same_device(q, k, v, cu_q, cu_k, out, workspace)
    if Tq == 0 or B == 0:
        return out
    if d != _current_device():
        with torch.cuda.device(d):
            return attn_prompt(q, k, v, cu_q, cu_k, scale, causal, out, workspace)
    if workspace is None:
        size = attn_prompt_workspace_bytes(B, Tq, Tk, Hq, Hkv)
        workspace = q.new_empty(size, dtype=_U8) if size else None
    else:
        size = _workspace_bytes(workspace)
    status = lib().sq_attn_prompt(q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, cu_q.data_ptr(), cu_k.data_ptr(), B,
                                  Tq, Tk, Hq, Hkv, 128, 0.08838834764831845 if scale is None else scale, int(causal),
                                  out.data_ptr(), ldo, _ptr(workspace), size, _stream(q))
    if status:
        _check(status, "sq_attn_prompt")
    return out
