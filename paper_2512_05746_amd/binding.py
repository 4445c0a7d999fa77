"""Python face of libhq.so: one function per C entry point declared in ``include/hq.h``.

Tensors are PyTorch tensors used purely as device buffers, and the work is enqueued on PyTorch's
current HIP stream.  The library is loaded with ctypes; the checks of the arguments, the allocation of
results and the calls themselves are native (``csrc/marshal.cpp``).  There is no fallback: if a library
cannot be loaded or a call is refused, an exception is raised.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import build as _build

SYMBOLS = ("hq_status_string", "hq_quantize_weights", "hq_act_hadamard_quant",
           "hq_int_linear", "hq_int_conv2d", "hq_act_hadamard_quant_static",
           "hq_int_linear_static", "hq_int_conv2d_static",
           "hq_quantize_weights_single", "hq_int_linear_single",
           "hq_act_hadamard_quant_width", "hq_int_conv2d_width",
           "hq_int_linear_i8", "hq_int_conv2d_i8", "hq_act_hadamard_quant_i8",
           "hq_act_quant_int_conv2d", "hq_act_quant_int_linear",
           "hq_fp8_quantize_rows", "hq_fp8_quantize_blocks", "hq_fp8_linear", "hq_act_quant_fp8_linear",
           "hq_fp8_linear_backward", "hq_qk_norm_rope", "hq_qk_norm_rope_backward")
# entry points that return the bytes of a workspace
WORKSPACE_SYMBOLS = ("hq_act_quant_fp8_linear_workspace", "hq_fp8_linear_backward_workspace",
                     "hq_qk_norm_rope_backward_workspace")
# entry points that do not return a status
INFO_SYMBOLS = ("hq_int_conv2d_kernel_name", "hq_fp8_linear_kernel_name", "hq_fp8_linear_backward_kernel_name") + WORKSPACE_SYMBOLS


class HqError(RuntimeError):
    def __init__(self, fn: str, code: int, text: str):
        super().__init__("%s failed: %s (status %d)" % (fn, text, code))
        self.code = code


_lib = None
_marshal = None      # the native module, bound to the loaded library


def _native():
    """The native module; loads the library on first use."""
    if _marshal is None:
        load_library()
    return _marshal


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads libhq.so.  The in-tree library is built first if it is missing or older than one of
    its sources (a child-process compile; nothing here touches the GPU before that)."""
    global _lib, _marshal
    if _lib is not None and path is None:
        return _lib
    if path is None:
        path = _build.LIB
        if _build.is_stale():
            _build.build_lib()
    lib = ctypes.CDLL(path)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    lib.hq_status_string.argtypes = [i32]
    lib.hq_status_string.restype = ctypes.c_char_p
    lib.hq_quantize_weights.argtypes = [vp, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.hq_act_hadamard_quant.argtypes = [vp, i32, i64, i32, i32, i32, vp, vp, vp]
    lib.hq_int_linear.argtypes = [vp, vp, vp, vp, vp, i64, i32, i32, vp, i32, vp]
    lib.hq_int_conv2d.argtypes = [vp] * 5 + [i32] * 9 + [vp, i32, vp]
    lib.hq_act_hadamard_quant_static.argtypes = [vp, i32, i64, i32, i32, i32, vp, vp, vp]
    lib.hq_int_linear_static.argtypes = lib.hq_int_linear.argtypes
    lib.hq_int_conv2d_static.argtypes = lib.hq_int_conv2d.argtypes
    lib.hq_quantize_weights_single.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.hq_int_linear_single.argtypes = [vp, vp, vp, vp, vp, i64, i32, i32, i32, vp, i32, vp]
    lib.hq_act_hadamard_quant_width.argtypes = [vp, i32, i32, i32, i32, i32, i32, i32, vp, vp, vp]
    lib.hq_int_conv2d_width.argtypes = [vp] * 5 + [i32] * 10 + [vp, i32, vp]
    lib.hq_int_linear_i8.argtypes = lib.hq_int_linear.argtypes
    lib.hq_act_hadamard_quant_i8.argtypes = lib.hq_act_hadamard_quant.argtypes
    lib.hq_int_conv2d_i8.argtypes = lib.hq_int_conv2d.argtypes
    lib.hq_act_quant_int_conv2d.argtypes = [vp, i32, vp, vp, vp] + [i32] * 11 + [vp, i32, vp, vp, vp]
    lib.hq_act_quant_int_linear.argtypes = [vp, i32, vp, vp, vp, i64, i32, i32, i32, i32, vp, i32, vp, vp, vp]
    lib.hq_fp8_quantize_rows.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp]
    lib.hq_fp8_quantize_blocks.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, vp]
    lib.hq_fp8_linear.argtypes = [vp] * 4 + [i32, vp, i64, i32, i32, vp, i32, vp]
    lib.hq_act_quant_fp8_linear.argtypes = [vp, i32, i64, vp, vp, vp, i64, i32, i32, vp, vp, i32, vp]
    lib.hq_fp8_linear_backward.argtypes = [vp, i64, vp, i64, i32, vp, vp, i64, i32, i32] + [vp] * 5
    f32 = ctypes.c_float
    lib.hq_qk_norm_rope.argtypes = [vp, vp, i32, i64, i32, i32, i32, vp, vp, vp, i32, vp, vp, i64, i32, i32, vp, i32,
                                    f32, vp, vp, vp]
    lib.hq_qk_norm_rope_backward.argtypes = [vp] * 4 + [i32, i64, i32, i32, i32, vp, vp, vp, i32, vp, vp, i64, i32, i32,
                                                        vp, i32, f32] + [vp] * 6
    lib.hq_act_quant_fp8_linear_workspace.argtypes = [i32, i64, i32, i32, i32]
    lib.hq_fp8_linear_backward_workspace.argtypes = [i64, i32, i32]
    lib.hq_qk_norm_rope_backward_workspace.argtypes = [i32, i64, i32, i32, i32, i32]
    for name in SYMBOLS[1:]:
        getattr(lib, name).restype = i32
    for name in WORKSPACE_SYMBOLS:
        getattr(lib, name).restype = i64
    lib.hq_fp8_linear_kernel_name.argtypes = [i32, i64, i32, i32, i32]
    lib.hq_fp8_linear_backward_kernel_name.argtypes = [i32, i64, i32, i32, i32]
    lib.hq_fp8_linear_kernel_name.restype = lib.hq_fp8_linear_backward_kernel_name.restype = ctypes.c_char_p
    lib.hq_int_conv2d_kernel_name.argtypes = [i32] * 11
    lib.hq_int_conv2d_kernel_name.restype = ctypes.c_char_p
    from . import _marshal as marshal
    marshal.bind({name: ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in SYMBOLS + WORKSPACE_SYMBOLS}, HqError)
    _lib, _marshal = lib, marshal
    return lib


def hq_int_conv2d_kernel_name(nb: int, h: int, w: int, c_in: int, c_out: int, ksize: int = 3, stride: int = 1,
                              pad: Optional[int] = None, static_scale: bool = False, bits: int = 4) -> str:
    """Name of the kernel the convolution calls run for this geometry, and its tile (host logic only)."""
    pad = (ksize - 1) // 2 if pad is None else pad
    return load_library().hq_int_conv2d_kernel_name(nb, h, w, c_in, c_out, ksize, ksize, stride, pad,
                                                    1 if static_scale else 0, bits).decode()


def status_string(code: int) -> str:
    return load_library().hq_status_string(code).decode()


def hq_quantize_weights(w: torch.Tensor, had_block: int = 64, w_bits: int = 4
                        ) -> Tuple[torch.Tensor, torch.Tensor]:
    """w [n_out, taps, k_in] fp16/fp32 -> (wq uint8 [n_out, taps, k_in/2], w_scale fp32 [n_out]);
    w_bits = 8: wq int8 [n_out, taps, k_in], one code per byte."""
    return _native().quantize_weights(w, had_block, w_bits)


def hq_act_hadamard_quant(x: torch.Tensor, had_block: int = 64, a_bits: int = 4,
                          out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                          ) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [..., k] fp16/fp32 -> (xq uint8 [..., k/2], x_scale fp32 [...]); a_bits = 8: xq int8 [..., k]."""
    return _native().act_hadamard_quant(x, had_block, a_bits, out)


def hq_int_linear(xq: torch.Tensor, x_scale: Optional[torch.Tensor], wq: torch.Tensor,
                  w_scale: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                  y_dtype: torch.dtype = torch.float16, out: Optional[torch.Tensor] = None
                  ) -> torch.Tensor:
    """xq [m, k/2], wq [n, k/2] (or [n, 1, k/2]) -> y [m, n]; y_dtype int32 returns the raw sums."""
    return _native().linear(xq, x_scale, wq, w_scale, bias, y_dtype, out)


def hq_int_conv2d(xq: torch.Tensor, x_scale: Optional[torch.Tensor], wq: torch.Tensor,
                  w_scale: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                  ksize: int = 3, stride: int = 1, pad: Optional[int] = None,
                  y_dtype: torch.dtype = torch.float16, out: Optional[torch.Tensor] = None
                  ) -> torch.Tensor:
    """xq [nb, h, w, cin/2], wq [cout, ksize*ksize, cin/2] -> y [nb, ho, wo, cout] (same size for
    stride 1; ksize 3, stride 2, pad 1 halves it, rounding up); y_dtype int32 returns the per-tap
    sums [nb, ho, wo, ksize*ksize, cout]."""
    return _native().conv2d(xq, x_scale, wq, w_scale, bias, ksize, stride, pad, y_dtype, out)


def hq_act_quant_int_conv2d(x: torch.Tensor, wq: torch.Tensor, w_scale: Optional[torch.Tensor],
                            bias: Optional[torch.Tensor] = None, had_block: int = 64, a_bits: int = 4,
                            ksize: int = 3, stride: int = 1, pad: Optional[int] = None,
                            y_dtype: torch.dtype = torch.float16, out: Optional[torch.Tensor] = None,
                            codes_out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> torch.Tensor:
    """The whole 3x3 layer in one launch: x [nb, h, w, cin] fp16, wq [cout, 9, cin/2] -> y [nb, h, w, cout]
    (y_dtype int32: per-tap sums [nb, h, w, 9, cout]).  codes_out = (xq uint8 [nb, h, w, cin/2],
    x_scale fp32 [nb, h, w]) receives the codes and scales the kernel used."""
    return _native().act_quant_conv2d(x, wq, w_scale, bias, had_block, a_bits, ksize, stride, pad, y_dtype, out,
                                      codes_out)


def hq_act_quant_int_linear(x: torch.Tensor, wq: torch.Tensor, w_scale: Optional[torch.Tensor],
                            bias: Optional[torch.Tensor] = None, had_block: int = 64, a_bits: int = 4,
                            y_dtype: torch.dtype = torch.float16, out: Optional[torch.Tensor] = None,
                            codes_out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> torch.Tensor:
    """A linear layer / 1x1 convolution in one launch: x [..., k] fp16, wq [n, k/2] (or [n, 1, k/2]) ->
    y [..., n] (y_dtype int32: the integer sums).  codes_out = (xq uint8 [..., k/2], x_scale fp32 [...])
    receives the codes and scales the kernel used."""
    return _native().act_quant_linear(x, wq, w_scale, bias, had_block, a_bits, y_dtype, out, codes_out)


def hq_act_hadamard_quant_static(x: torch.Tensor, x_scale: torch.Tensor, had_block: int = 64,
                                 a_bits: int = 4, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [..., k] fp16/fp32, x_scale one fp32 on the device -> xq uint8 [..., k/2]."""
    return _native().act_hadamard_quant_static(x, x_scale, had_block, a_bits, out)


def hq_int_linear_static(xq: torch.Tensor, x_scale: Optional[torch.Tensor], wq: torch.Tensor,
                         w_scale: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                         y_dtype: torch.dtype = torch.float16, out: Optional[torch.Tensor] = None
                         ) -> torch.Tensor:
    """As hq_int_linear with one activation scale (a device tensor holding one float32)."""
    return _native().linear_static(xq, x_scale, wq, w_scale, bias, y_dtype, out)


def hq_int_conv2d_static(xq: torch.Tensor, x_scale: Optional[torch.Tensor], wq: torch.Tensor,
                         w_scale: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                         ksize: int = 3, stride: int = 1, pad: Optional[int] = None,
                         y_dtype: torch.dtype = torch.float16, out: Optional[torch.Tensor] = None
                         ) -> torch.Tensor:
    """As hq_int_conv2d with one activation scale; y_dtype int32 returns the sums over all
    taps and input channels, [nb, h, w, cout]."""
    return _native().conv2d_static(xq, x_scale, wq, w_scale, bias, ksize, stride, pad, y_dtype, out)


# ---- Single scheme: un-transformed quantised weights, integer H folded into digit planes -------

def hq_quantize_weights_single(w: torch.Tensor, had_block: int = 64, w_bits: int = 4
                               ) -> Tuple[torch.Tensor, torch.Tensor]:
    """w [n_out, k_in] fp16/fp32 -> (wq3 uint8 [n_out, 3, k_in/2] digit planes, w_scale fp32 [n_out])."""
    return _native().quantize_weights_single(w, had_block, w_bits)


def hq_int_linear_single(xq: torch.Tensor, x_scale: Optional[torch.Tensor], wq3: torch.Tensor,
                         w_scale: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                         had_block: int = 64, y_dtype: torch.dtype = torch.float16,
                         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """xq [m, k/2], wq3 [n, 3, k/2] -> y [m, n]; y_dtype int32 returns the three sums [m, 3, n]."""
    return _native().linear_single(xq, x_scale, wq3, w_scale, bias, had_block, y_dtype, out)


# ---- width-axis convolution: the paper's own convolution ---------------------------------------

def hq_act_hadamard_quant_width(x: torch.Tensor, x_scale: torch.Tensor, had_block: int, a_bits: int = 4,
                                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [N, H, W, C] fp16/fp32, x_scale one fp32 on the device -> xu3 uint8 [3, N, H, W, C/2]
    (digit planes of the codes taken back along the width axis with the +-1 matrix)."""
    return _native().act_hadamard_quant_width(x, x_scale, had_block, a_bits, out)


def hq_int_conv2d_width(xu3: torch.Tensor, x_scale: Optional[torch.Tensor], wq: torch.Tensor,
                        w_scale: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                        had_block: int = 64, y_dtype: torch.dtype = torch.float16,
                        out: Optional[torch.Tensor] = None, stride: int = 1) -> torch.Tensor:
    """xu3 [3, N, H, W, Cin/2], wq [Cout, 9, Cin/2] (or [Cout, 3, 3, Cin/2]) -> y [N, Ho, Wo, Cout]
    (same size for stride 1; stride 2 halves it, rounding up); y_dtype int32 returns the exact integer sums.  The
    integers in the planes must lie within 8 * had_block, as those of hq_act_hadamard_quant_width do."""
    return _native().conv2d_width(xu3, x_scale, wq, w_scale, bias, had_block, y_dtype, out, stride)


# ---- 8-bit codes (W8A8): int8 operands, one code per byte ---------------------------------------

def hq_act_hadamard_quant_i8(x: torch.Tensor, had_block: int = 64, a_bits: int = 4
                             ) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [..., k] fp16/fp32 -> (xq int8 [..., k] with codes of a_bits bits, x_scale fp32 [...])."""
    return _native().act_hadamard_quant_i8(x, had_block, a_bits)


def hq_int_linear_i8(xq: torch.Tensor, x_scale: Optional[torch.Tensor], wq: torch.Tensor,
                     w_scale: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                     y_dtype: torch.dtype = torch.float16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """xq int8 [m, k], wq int8 [n, k] (or [n, 1, k]) -> y [m, n]; y_dtype int32 returns the raw sums."""
    return _native().linear_i8(xq, x_scale, wq, w_scale, bias, y_dtype, out)


def hq_int_conv2d_i8(xq: torch.Tensor, x_scale: Optional[torch.Tensor], wq: torch.Tensor,
                     w_scale: Optional[torch.Tensor], bias: Optional[torch.Tensor] = None,
                     ksize: int = 3, y_dtype: torch.dtype = torch.float16,
                     out: Optional[torch.Tensor] = None, stride: int = 1) -> torch.Tensor:
    """xq int8 [N, H, W, Cin], wq int8 [Cout, ksize*ksize, Cin] -> y [N, Ho, Wo, Cout] (same size for
    stride 1; ksize 3 at stride 2 halves it, rounding up); y_dtype int32 returns the per-tap sums
    [N, Ho, Wo, ksize*ksize, Cout]."""
    return _native().conv2d_i8(xq, x_scale, wq, w_scale, bias, ksize, stride, None, y_dtype, out)


# ---- 8-bit floats with block scales ---------------------------------------------------------------
# The calls from here on record nothing for autograd.  Those that take activations refuse tensors that require a gradient while gradients
# are recorded; under torch.no_grad(), or in an autograd function, with the _backward calls, they take them.

def hq_fp8_quantize_rows(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """x [..., k] fp16/bf16/fp32 -> (xq float8_e4m3fn [..., k up to a multiple of 16], x_scale fp32 [ceil(k / 128), rows]):
    one scale for each row and 128 columns.  x is contiguous, or a matrix of contiguous rows."""
    return _native().fp8_quantize_rows(x)


def hq_fp8_quantize_blocks(w: torch.Tensor, transposed: bool = False) -> Tuple[torch.Tensor, ...]:
    """w [n, k] fp16/bf16/fp32 -> (wq float8_e4m3fn [n, k up to a multiple of 16], w_scale fp32 [ceil(n / 128), ceil(k / 128)]):
    one scale for each block of 128 x 128.  transposed: (wq, wq_t, w_scale), wq_t [k, n up to a multiple of 16] the same
    codes transposed, for hq_fp8_linear_backward."""
    return _native().fp8_quantize_blocks(w, transposed)


def hq_fp8_linear(xq: torch.Tensor, x_scale: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor,
                  bias: Optional[torch.Tensor] = None, y_dtype: torch.dtype = torch.float16,
                  out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """xq [..., kp], wq [n, kp] float8_e4m3fn codes as the quantisers write them, with their scales -> y [..., n].  w_scale may be
    the transposed view of the scales of a matrix whose transposed codes wq holds.  out shares no memory with the inputs.

    Sums are fp32, but for fp16 and bf16 results eight neighbouring products are first cut 13 bits below the largest: at most 2^-10 of
    the sum of magnitudes (2^-7 among products of subnormal codes), 1.5e-5 of the norm over normal values.  Where products cancel, take
    float32."""
    return _native().fp8_linear(xq, x_scale, wq, w_scale, bias, y_dtype, out)


def hq_act_quant_fp8_linear(x: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                            y_dtype: torch.dtype = torch.float16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The whole layer: x [..., k] fp16/bf16/fp32 -> y [..., n], with the codes of hq_fp8_quantize_rows and the sums of hq_fp8_linear
    (in the order of another kernel where it is one launch: the last bits may differ).  out shares no memory with the inputs."""
    return _native().act_quant_fp8_linear(x, wq, w_scale, bias, y_dtype, out)


_FLOATS = {torch.float16: 0, torch.float32: 1, torch.bfloat16: 3}


def hq_fp8_linear_kernel_name(m: int, n: int, k: int, y_dtype: torch.dtype = torch.float16,
                              x_dtype: Optional[torch.dtype] = None) -> str:
    """Name of the kernel that hq_fp8_linear takes for these sizes, or hq_act_quant_fp8_linear for x_dtype (host logic only)."""
    return load_library().hq_fp8_linear_kernel_name(2 if x_dtype is None else _FLOATS[x_dtype], m, n, k, _FLOATS[y_dtype]).decode()


def hq_fp8_linear_backward_kernel_name(m: int, n: int, k: int, dtype: torch.dtype = torch.float16, bias_grad: bool = False) -> str:
    """Name of the kernel that multiplies in hq_fp8_linear_backward (host logic only)."""
    return load_library().hq_fp8_linear_backward_kernel_name(_FLOATS[dtype], m, n, k, 1 if bias_grad else 0).decode()


def hq_fp8_linear_backward(dy: torch.Tensor, x: torch.Tensor, wq_t: torch.Tensor, w_scale: torch.Tensor,
                           bias_grad: bool = False) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Gradients of hq_act_quant_fp8_linear: dy [..., n], x [..., k] of one type, wq_t and w_scale of
    hq_fp8_quantize_blocks(w, transposed=True) -> (dx [..., k] of that type, dw fp32 [n, k], db fp32 [n] or None)."""
    return _native().fp8_linear_backward(dy, x, wq_t, w_scale, bias_grad)


# ---- query and key heads: norm and rotation ---------------------------------------------------------

def hq_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                    cos: torch.Tensor, sin: torch.Tensor, positions: Optional[torch.Tensor] = None, eps: float = 1e-6,
                    interleaved: bool = False, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                    ) -> Tuple[torch.Tensor, torch.Tensor]:
    """q [t, heads, d], k [t, kv_heads, d] fp16/bf16/fp32 with contiguous channels (views of a projection's result, say), weights
    [d], cos and sin fp32 [positions, rotary / 2], positions int32/int64 [t] (None: 0 .. t - 1; negative: padding) ->
    both normalised head by head and rotated, contiguous or in `out`, which may be (q, k); otherwise its two tensors share memory neither
    with each other nor with an input."""
    return _native().qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, out)


def hq_qk_norm_rope_backward(dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                             q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor], cos: torch.Tensor,
                             sin: torch.Tensor, positions: Optional[torch.Tensor] = None, eps: float = 1e-6,
                             interleaved: bool = False, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None
                             ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Gradients of hq_qk_norm_rope: dq, dk of its results, its inputs -> (gradients of q and k, contiguous or in `out`; of the
    weights, fp32 [d], None for a weight that is None).  out[0] may be dq or q, out[1] dk or k; otherwise they share memory with nothing
    that is passed."""
    return _native().qk_norm_rope_backward(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved, out)
