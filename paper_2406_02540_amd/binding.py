"""Thin Python binding of the C-ABI library libvidiq.so (declared in include/vq.h).

Argument marshalling only: torch supplies device memory and the current HIP
stream, every step of the quantized linear layer runs in the library's kernels.
Tensors are checked and turned into pointers in csrc/vq_torch.cpp (in Python it
took longer than a small layer runs on the device).  There is no fallback: if
the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import operator
import os
import re

import torch

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
# the in-tree build; VQ_LIBVIDIQ_PATH names another build of the same sources (e.g. one with host sanitizers)
LIB_PATH = os.environ.get("VQ_LIBVIDIQ_PATH") or os.path.join(PKG_DIR, "libvidiq.so")
EXT_PATH = os.path.join(PKG_DIR, "_vq_torch.so")  # csrc/vq_torch.cpp

VQ_OK = 0
STATUS_NAMES = {0: "VQ_OK", 1: "VQ_ERR_NULL", 2: "VQ_ERR_SHAPE", 3: "VQ_ERR_ALIGN",
                4: "VQ_ERR_WORKSPACE", 5: "VQ_ERR_LAUNCH", 6: "VQ_ERR_ARCH", 7: "VQ_ERR_BITS", 8: "VQ_ERR_TYPE"}

# name -> (restype, argtypes); mirrors include/vq.h
_P, _I, _SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
_F, _D = ctypes.c_float, ctypes.c_double
SIGNATURES = {
    "vq_quantize_per_token": (_I, [_P, _P, _P, _P, _I, _I, _P]),
    "vq_gelu_quantize": (_I, [_P, _I, _P, _P, _P, _I, _I, _P]),
    "vq_layernorm_quantize": (_I, [_P, _P, _P, _I, ctypes.c_float, _P, _P, _P, _I, _I, _P]),
    "vq_residual_quantize": (_I, [_P, _P, _P, _I, _P, _P, _P, _P, _I, _I, _P]),
    "vq_channel_absmax": (_I, [_P, _I, _P, _I, _I, _I, _P]),
    "vq_balance_mask": (_I, [_P, _P, ctypes.c_float, _P, _P, _I, _P]),
    "vq_hadamard_quantize": (_I, [_P, _P, _P, _P, _I, _I, _P]),
    "vq_rotate_weight": (_I, [_P, _P, _P, _I, _I, _P]),
    "vq_gemm_f16": (_I, [_P, _P, _P, _P, _I, _I, _I, _P]),
    "vq_quantize_static": (_I, [_P, _P, ctypes.c_float, _P, _I, _I, _P]),
    "vq_gemm_w8a8": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _P]),
    "vq_gemm_w4a8": (_I, [_P, _P, _P, _P, _P, _P, _P, _I, _I, _I, _P]),
    "vq_linear": (_I, [_P, _P, _P, _I, _P, _P, _P, _P, _SZ, _I, _I, _I, _P]),
    "vq_linear_workspace_bytes": (_SZ, [_I, _I, _I, _I]),
    "vq_layernorm_linear": (_I, [_P, _P, _P, _I, ctypes.c_float, _P, _P, _I, _P, _P, _P, _P, _SZ, _I, _I, _I, _P]),
    "vq_gelu_linear": (_I, [_P, _I, _P, _P, _I, _P, _P, _P, _P, _SZ, _I, _I, _I, _P]),
    "vq_residual_linear": (_I, [_P, _P, _P, _I, _P, _P, _P, _I, _P, _P, _P, _P, _SZ, _I, _I, _I, _P]),
    "vq_hadamard_linear": (_I, [_P, _P, _P, _I, _P, _P, _P, _P, _SZ, _I, _I, _I, _P]),
    "vq_linear_static": (_I, [_P, _P, _P, _I, _P, _P, _P, _I, _I, _I, _P]),
    "vq_quantize_weight": (_I, [_P, _P, _I, _P, _P, _I, _I, _P]),
    "vq_mx4_quantize": (_I, [_P, _I, _P, _P, _P, _I, _I, _P]),
    "vq_mx4_dequantize": (_I, [_P, _P, _P, _I, _I, _I, _P]),
    "vq_gemm_mx4": (_I, [_P, _P, _P, _P, _P, _P, _I, _I, _I, _I, _P]),
    "vq_linear_mx4": (_I, [_P, _P, _P, _P, _P, _P, _I, _P, _SZ, _I, _I, _I, _P]),
    "vq_linear_mx4_workspace_bytes": (_SZ, [_I, _I, _I]),
    "vq_rotary": (_I, [_P, _P, _P, _P, _I, _P, _P, _F, _I, _I, _I, _I, _I, _I, _P, _P]),
    "vq_rotary_frequencies": (_I, [_P, _P, _I, _D, _I, _D, _I]),
    "vq_attention": (_I, [_P, _P, _P, _P, _I, _P, _P, _I, _I, _I, _I, _I, _I, _P, _F, _I, _P, _SZ, _P]),
    "vq_attention_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _I]),
    "vq_rotary_axes": (_I, [_P, _P, _P, _P, _I, _P, _P, _F, _I, _I, _P, _I, _I, _I, _I, _P, _P]),
    "vq_norm_rotary": (_I, [_P, _P, _P, _P, _I, _I, _F, _P, _P, _P, _P, _P, _P, _F, _I, _I, _P, _I, _I, _I, _I, _P, _P]),
    "vq_attention_window": (_I, [_P, _P, _P, _P, _I, _P, _P, _I, _I, _I, _I, _I, _I, _P, _F, _I, _I, _I, _I, _P, _SZ, _P]),
    "vq_attention_prefix": (_I, [_P, _P, _P, _P, _P, _P, _I, _P, _P, _I, _I, _I, _I, _I, _I, _I, _P, _F, _I, _P, _SZ, _P]),
    "vq_attention_window_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _I, _I, _I, _I, _I]),
    "vq_attention_prefix_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _I, _I]),
    "vq_status_string": (ctypes.c_char_p, [_I]),
}


class VqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)} ({status_string(status)})")


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libvidiq.so; raises if it has not been built (python -m paper_2406_02540_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} not found: build it with `python -m paper_2406_02540_amd.build`")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def status_string(status: int) -> str:
    return lib().vq_status_string(int(status)).decode()


# order of the entry points' addresses in csrc/vq_torch.cpp
_BOUND = ("vq_quantize_per_token", "vq_gelu_quantize", "vq_layernorm_quantize", "vq_residual_quantize",
          "vq_hadamard_quantize", "vq_quantize_static", "vq_channel_absmax", "vq_balance_mask", "vq_rotate_weight",
          "vq_quantize_weight", "vq_gemm_f16", "vq_gemm_w8a8", "vq_gemm_w4a8", "vq_linear_workspace_bytes", "vq_linear",
          "vq_linear_static", "vq_layernorm_linear", "vq_gelu_linear", "vq_residual_linear", "vq_hadamard_linear",
          "vq_mx4_quantize", "vq_mx4_dequantize", "vq_gemm_mx4", "vq_linear_mx4", "vq_linear_mx4_workspace_bytes",
          "vq_rotary", "vq_attention", "vq_attention_workspace_bytes", "vq_rotary_axes", "vq_norm_rotary", "vq_attention_window",
          "vq_attention_prefix", "vq_attention_window_workspace_bytes", "vq_attention_prefix_workspace_bytes")

_ext = None


def _load():
    """Loads the extension and hands it the entry points of libvidiq.so."""
    global _ext
    handle = lib()
    if not os.path.exists(EXT_PATH):
        raise RuntimeError(f"{EXT_PATH} not found: build it with `python -m paper_2406_02540_amd.build`")
    loader = importlib.machinery.ExtensionFileLoader("_vq_torch", EXT_PATH)
    spec = importlib.util.spec_from_file_location("_vq_torch", EXT_PATH, loader=loader)
    rebuild = "build it again with `python -m paper_2406_02540_amd.build`"
    try:
        ext = importlib.util.module_from_spec(spec)
        loader.exec_module(ext)
    except ImportError as e:  # (symbols of another torch)
        raise RuntimeError(f"{EXT_PATH} does not load: {rebuild}") from e
    # the extension holds the layout of the torch that it was compiled against
    if ext.TORCH_VERSION != re.match(r"[\d.]*\d", torch.__version__).group():
        raise RuntimeError(f"{EXT_PATH} was built for torch {ext.TORCH_VERSION}, this is {torch.__version__}: {rebuild}")
    ext.bind(VqError, tuple(ctypes.cast(getattr(handle, n), ctypes.c_void_p).value for n in _BOUND))
    _ext = ext
    return ext


def vq_quantize_per_token(x, chan_mul=None, xq=None, x_scale=None, stream=None):
    """x fp16 [M,K] (+ chan_mul fp32 [K]) -> (xq int8 [M,K], x_scale fp32 [M])."""
    return (_ext or _load()).quantize_per_token(x, chan_mul, xq, x_scale, stream)


def vq_gelu_quantize(h, approximate=False, chan_mul=None, xq=None, x_scale=None, stream=None):
    """GELU (exact or tanh form) fused with the quantizer: h fp16 [M,K] -> (xq, x_scale)."""
    return (_ext or _load()).gelu_quantize(h, approximate, chan_mul, xq, x_scale, stream)


def vq_layernorm_quantize(x, mod_scale=None, mod_shift=None, tokens_per_sample=None, eps=1e-6,
                          chan_mul=None, xq=None, x_scale=None, stream=None):
    """LayerNorm + (1 + scale) y + shift fused with the quantizer: x fp16 [M,K] -> (xq, x_scale)."""
    return (_ext or _load()).layernorm_quantize(x, mod_scale, mod_shift, tokens_per_sample, eps, chan_mul, xq, x_scale,
                                                stream)


def vq_residual_quantize(x, y, gate=None, tokens_per_sample=None, r=None, chan_mul=None, xq=None,
                         x_scale=None, stream=None):
    """r = x + gate * y fused with the quantizer: fp16 [M,K] twice -> (r fp16, xq, x_scale)."""
    return (_ext or _load()).residual_quantize(x, y, gate, tokens_per_sample, r, chan_mul, xq, x_scale, stream)


def vq_channel_absmax(a, amax=None, accumulate=False, stream=None):
    """Per-column absmax of fp16 activations [M,K] or fp32 weights [N,K] -> amax fp32 [K]."""
    return (_ext or _load()).channel_absmax(a, amax, accumulate, stream)


def vq_balance_mask(amax_x, amax_w, alpha, stream=None):
    """Eq. 3: (s, chan_mul = 1/s), fp32 [K] each, from the two absmax statistics."""
    return (_ext or _load()).balance_mask(amax_x, amax_w, alpha, stream)


def vq_hadamard_quantize(x, chan_mul=None, xq=None, x_scale=None, stream=None):
    """Scaling, block Hadamard rotation, per-token quantizer: x fp16 [M,K] -> (xq, x_scale)."""
    return (_ext or _load()).hadamard_quantize(x, chan_mul, xq, x_scale, stream)


def vq_rotate_weight(w, chan_s=None, out=None, stream=None):
    """Weight side of the rotation: w fp32 [N,K] (* chan_s) -> fp32 [N,K]."""
    return (_ext or _load()).rotate_weight(w, chan_s, out, stream)


def vq_gemm_f16(x, w, bias=None, y=None, stream=None):
    """FP16 comparison layer: x fp16 [M,K], w fp16 [N,K] (+ bias fp16 [N]) -> y fp16 [M,N]."""
    return (_ext or _load()).gemm_f16(x, w, bias, y, stream)


def vq_quantize_static(x, scale, chan_mul=None, xq=None, stream=None):
    """One fixed scale for the whole tensor: x fp16 [M,K] -> xq int8 [M,K] (clipped at +-127)."""
    return (_ext or _load()).quantize_static(x, scale, chan_mul, xq, stream)


def vq_gemm_w8a8(xq, x_scale, wq, w_scale, bias=None, y=None, return_acc=False, stream=None):
    """int8 [M,K] x int8 [N,K] -> fp16 [M,N] (and the int32 sums if return_acc)."""
    return (_ext or _load()).gemm_w8a8(xq, x_scale, wq, w_scale, bias, y, return_acc, stream)


def vq_gemm_w4a8(xq, x_scale, wq4, w_scale, bias=None, y=None, return_acc=False, stream=None):
    """int8 [M,K] x packed 4-bit [N,K/2] -> fp16 [M,N] (and the int32 sums if return_acc)."""
    return (_ext or _load()).gemm_w4a8(xq, x_scale, wq4, w_scale, bias, y, return_acc, stream)


def vq_linear_workspace_bytes(M, N, K, w_bits) -> int:
    return int(lib().vq_linear_workspace_bytes(int(M), int(N), int(K), int(w_bits)))


LINEAR_STATIC_SCRATCH_BYTES = 40 << 20  # VQ_LINEAR_STATIC_SCRATCH_BYTES of include/vq.h


def vq_linear_static(x, chan_mul, w, w_bits, w_scale, bias=None, y=None, stream=None):
    """The whole layer with the library's built-in scratch instead of a workspace (the call allocates nothing
    when y is given); layers whose int8 activations exceed LINEAR_STATIC_SCRATCH_BYTES raise VQ_ERR_WORKSPACE."""
    return (_ext or _load()).linear_static(x, chan_mul, w, w_bits, w_scale, bias, y, stream)


def vq_linear(x, chan_mul, w, w_bits, w_scale, bias=None, y=None, workspace=None, stream=None):
    """The whole layer on fp16 activations; workspace is a uint8 device tensor (allocated if None)."""
    return (_ext or _load()).linear(x, chan_mul, w, w_bits, w_scale, bias, y, workspace, stream)


def vq_layernorm_linear(x, w, w_bits, w_scale, mod_scale=None, mod_shift=None, tokens_per_sample=None, eps=1e-6,
                        chan_mul=None, bias=None, y=None, workspace=None, stream=None):
    """LayerNorm + modulation, quantizer and GEMM in one call: x fp16 [M,K] -> y fp16 [M,N]."""
    return (_ext or _load()).layernorm_linear(x, w, w_bits, w_scale, mod_scale, mod_shift, tokens_per_sample, eps,
                                              chan_mul, bias, y, workspace, stream)


def vq_gelu_linear(h, w, w_bits, w_scale, approximate=False, chan_mul=None, bias=None, y=None, workspace=None,
                   stream=None):
    """GELU, quantizer and GEMM in one call: h fp16 [M,K] -> y fp16 [M,N]."""
    return (_ext or _load()).gelu_linear(h, w, w_bits, w_scale, approximate, chan_mul, bias, y, workspace, stream)


def vq_residual_linear(x, y_in, w, w_bits, w_scale, gate=None, tokens_per_sample=None, r=None, chan_mul=None,
                       bias=None, y=None, workspace=None, stream=None):
    """r = x + gate * y_in, quantizer and GEMM in one call: fp16 [M,K] twice -> (r fp16 [M,K], y fp16 [M,N])."""
    return (_ext or _load()).residual_linear(x, y_in, w, w_bits, w_scale, gate, tokens_per_sample, r, chan_mul, bias, y,
                                             workspace, stream)


def vq_hadamard_linear(x, chan_mul, w, w_bits, w_scale, bias=None, y=None, workspace=None, stream=None):
    """Scaling, block Hadamard rotation, quantizer and GEMM in one call (w quantized from rotated weights)."""
    return (_ext or _load()).hadamard_linear(x, chan_mul, w, w_bits, w_scale, bias, y, workspace, stream)


def vq_quantize_weight(w_f32, chan_s=None, w_bits=8, stream=None):
    """W fp32 [N,K] (+ s fp32 [K]) -> (wq int8 [N,K] or packed uint8 [N,K/2], w_scale fp32 [N])."""
    return (_ext or _load()).quantize_weight(w_f32, chan_s, w_bits, stream)


def vq_mx4_quantize(x, chan_mul=None, xq=None, x_scale=None, stream=None):
    """x fp16, bf16 or fp32 [M,K] (* chan_mul fp32 [K]) -> microscaled 4-bit codes: (xq uint8 [M,K/2], x_scale uint8
    [M, MX4_SCALE_STRIDE(K)])."""
    return (_ext or _load()).mx4_quantize(x, chan_mul, xq, x_scale, stream)


def vq_mx4_dequantize(xq, x_scale, dtype=torch.float16, x=None, stream=None):
    """The values that the codes stand for, in fp16, bf16 or fp32 (the type of x where it is given): [M,K]."""
    return (_ext or _load()).mx4_dequantize(xq, x_scale, dtype, x, stream)


def vq_gemm_mx4(xq, x_scale, wq, w_scale, bias=None, y=None, dtype=torch.float16, stream=None):
    """Codes [M,K/2] x codes [N,K/2] (+ bias [N]) -> y [M,N] in fp16 or bf16 (the type of y or bias where one is given)."""
    return (_ext or _load()).gemm_mx4(xq, x_scale, wq, w_scale, bias, y, dtype, stream)


def vq_linear_mx4_workspace_bytes(M, N, K) -> int:
    return int(lib().vq_linear_mx4_workspace_bytes(int(M), int(N), int(K)))


def MX4_SCALE_STRIDE(K) -> int:
    """Bytes of a row of scales: K/32 of them, rounded up to four (VQ_MX4_SCALE_STRIDE of include/vq.h)."""
    return (K // 32 + 3) // 4 * 4


def vq_linear_mx4(x, chan_mul, w, w_scale, bias=None, y=None, workspace=None, stream=None):
    """The microscaled 4-bit layer on fp16 or bf16 activations: x [M,K] -> y [M,N] of the same type."""
    return (_ext or _load()).linear_mx4(x, chan_mul, w, w_scale, bias, y, workspace, stream)


def vq_rotary(q, k, positions, inv_freq, interleaved=False, amplitude=1.0, q_out=None, k_out=None, stream=None):
    """Rotary positions on views q [T,Hq,D] and k [T,Hk,D] (or None), fp16 or bf16; positions int32 [T], inv_freq fp32
    [rot_dim/2] -> (q_out, k_out); q_out=q, k_out=k works in place."""
    return (_ext or _load()).rotary(q, k, positions, inv_freq, interleaved, amplitude, q_out, k_out, stream)


ROPE_SCALING = {"plain": 0, "linear": 1, "base": 2, "parts": 3}


def vq_rotary_frequencies(rot_dim, base=10000.0, scaling="plain", factor=1.0, original_length=0):
    """(inv_freq fp32 [rot_dim/2] in host memory, amplitude) for vq_rotary; scaling "plain", "linear", "base" or "parts"."""
    if scaling not in ROPE_SCALING:
        raise ValueError(f"scaling must be one of {tuple(ROPE_SCALING)}")
    table, amplitude = (ctypes.c_float * max(int(rot_dim) // 2, 1))(), ctypes.c_float()
    status = lib().vq_rotary_frequencies(table, ctypes.byref(amplitude), int(rot_dim), float(base), ROPE_SCALING[scaling],
                                         float(factor), int(original_length))
    if status != VQ_OK:
        raise VqError(status, "vq_rotary_frequencies")
    return torch.tensor(list(table), dtype=torch.float32), float(amplitude.value)


def vq_attention_workspace_bytes(sequences, Tq, Tk, heads, kv_heads, head_dim) -> int:
    return int(lib().vq_attention_workspace_bytes(int(sequences), int(Tq), int(Tk), int(heads), int(kv_heads), int(head_dim)))


def vq_attention(q, k, v, cu_q, cu_k, softmax_scale=None, causal=False, out=None, workspace=None, stream=None):
    """Softmax attention over packed sequences: views q [Tq,H,D], k and v [Tk,G,D], fp16 or bf16, sequence b between rows
    cu[b] and cu[b+1] (int32 [sequences + 1]) -> out [Tq,H,D].  softmax_scale: 1/sqrt(D) if not given; workspace is a
    uint8 device tensor (allocated if None).  Rows outside all sequences are not written (a new out is not cleared)."""
    return (_ext or _load()).attention(q, k, v, cu_q, cu_k, softmax_scale, causal, out, workspace, stream)


ROPE_PAIRS = {"halves": 0, "neighbours": 1, "axis_halves": 2}
NORMS = {"rms": 0, "layer": 1}


def _named(table, name, what):
    if name not in table:
        raise ValueError(f"{what} must be one of {tuple(table)}")
    return table[name]


def vq_rotary_axes(q, k, positions, inv_freq, sections, pairing="halves", amplitude=1.0, q_out=None, k_out=None, stream=None):
    """Rotary positions of several axes on views q [T,Hq,D] and k [T,Hk,D] (or None), fp16 or bf16: axis a turns sections[a]
    pairs by positions[a] (int32 [axes,T]) times their part of inv_freq fp32 [sum(sections)]; pairing "halves" (over all axes),
    "neighbours" or "axis_halves" (every axis in channels of its own) -> (q_out, k_out); q_out=q, k_out=k works in place."""
    return (_ext or _load()).rotary_axes(q, k, positions, inv_freq, sections, _named(ROPE_PAIRS, pairing, "pairing"), amplitude, q_out,
                                         k_out, stream)


def vq_norm_rotary(q, k, q_weight=None, k_weight=None, q_bias=None, k_bias=None, norm="rms", eps=1e-6, positions=None, inv_freq=None,
                   sections=None, pairing="halves", amplitude=1.0, q_out=None, k_out=None, stream=None):
    """The norm of every head of q and k ("rms", or "layer": mean and variance), weights and biases fp32 [D] or None, and the
    rotary positions of vq_rotary_axes behind it in the same pass (sections=None: the norm alone) -> (q_out, k_out)."""
    return (_ext or _load()).norm_rotary(q, k, q_weight, k_weight, q_bias, k_bias, _named(NORMS, norm, "norm"), eps, positions, inv_freq,
                                         sections, _named(ROPE_PAIRS, pairing, "pairing"), amplitude, q_out, k_out, stream)


def _int(n) -> int:
    """n as the library's int; what does not fit is a number that it takes for nothing (ctypes would cut it to another)."""
    n = int(n)
    return n if -2**31 <= n < 2**31 else -2**31


def _limit(n) -> int:
    return -1 if n is None else _int(operator.index(n))


def vq_attention_window_workspace_bytes(sequences, Tq, Tk, heads, kv_heads, head_dim, causal, left, right, sinks) -> int:
    return int(lib().vq_attention_window_workspace_bytes(_int(sequences), _int(Tq), _int(Tk), _int(heads), _int(kv_heads), _int(head_dim),
                                                         int(bool(causal)), _limit(left), _limit(right), _int(operator.index(sinks))))


def vq_attention_window(q, k, v, cu_q, cu_k, left, right=None, sinks=0, softmax_scale=None, causal=False, out=None, workspace=None,
                        stream=None):
    """vq_attention in a sliding window: of n queries and m keys query i, at p = i + m - n, sees the keys p - left .. p + right
    (None: no limit) and the first `sinks`; causal: none behind p.  Other arguments as vq_attention's."""
    return (_ext or _load()).attention_window(q, k, v, cu_q, cu_k, left, right, sinks, softmax_scale, causal, out, workspace, stream)


def vq_attention_prefix_workspace_bytes(sequences, Tq, prefix, Tk, heads, kv_heads, head_dim) -> int:
    return int(lib().vq_attention_prefix_workspace_bytes(_int(sequences), _int(Tq), _int(prefix), _int(Tk), _int(heads), _int(kv_heads),
                                                         _int(head_dim)))


def vq_attention_prefix(q, prefix_k, prefix_v, k, v, cu_q, cu_k, softmax_scale=None, causal=False, out=None, workspace=None, stream=None):
    """vq_attention of sequences that share their first keys prefix_k, prefix_v [P,G,D]: a query sees all of them, then its own
    sequence's keys (causal: up to its place).  Other arguments as vq_attention's."""
    return (_ext or _load()).attention_prefix(q, prefix_k, prefix_v, k, v, cu_q, cu_k, softmax_scale, causal, out, workspace, stream)
