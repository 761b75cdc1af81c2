"""Thin ctypes binding of the grouped products (see include/moe_products.h for the contract).

Argument marshalling only, like `moe`: torch tensors on the GPU are checked and their addresses and the current HIP stream
passed to the C entry point of the same name.  8-bit matrices may be torch.float8_e4m3fn or torch.uint8 tensors.
"""
from __future__ import annotations

import ctypes

import torch

from . import moe
from .moe import _check, _dtype_code

EXPORTS = ("moe_product_workspace_bytes", "moe_grouped_product", "moe_grouped_product_dgrad", "moe_grouped_product_wgrad",
           "moe_quantize_rows_fp8", "moe_quantize_weights_fp8", "moe_grouped_product_fp8")
BLOCK = 128  # values that share a scale, along each dimension that is blocked


class MoeProduct(ctypes.Structure):
    _fields_ = [("n_experts", ctypes.c_int32), ("out_features", ctypes.c_int32), ("in_features", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


_bound = None


def lib() -> ctypes.CDLL:
    """The loaded C library with this header's functions declared (raises if it has not been built)."""
    global _bound
    L = moe.lib()
    if _bound is not L:
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        pp = ctypes.POINTER(MoeProduct)
        L.moe_product_workspace_bytes.argtypes = [pp, i32, ctypes.POINTER(sz)]
        L.moe_grouped_product.argtypes = [pp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.moe_grouped_product_dgrad.argtypes = [pp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.moe_grouped_product_wgrad.argtypes = [pp, i32, vp, vp, vp, vp, i32, i32, vp, sz, vp]
        L.moe_quantize_rows_fp8.argtypes = [i32, i32, i32, vp, vp, vp, vp]
        L.moe_quantize_weights_fp8.argtypes = [pp, vp, vp, vp, vp, vp, vp]
        L.moe_grouped_product_fp8.argtypes = [pp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        _bound = L
    return L


def make_product(n_experts: int, out_features: int, in_features: int, dtype: torch.dtype) -> MoeProduct:
    code = moe.MOE_F32 if dtype == torch.float32 else moe.MOE_BF16 if dtype == torch.bfloat16 else -1
    return MoeProduct(n_experts, out_features, in_features, code)


def moe_product_workspace_bytes(product: MoeProduct, max_rows: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().moe_product_workspace_bytes(ctypes.byref(product), max_rows, ctypes.byref(out)), "moe_product_workspace_bytes")
    return out.value


def alloc_workspace(product: MoeProduct, max_rows: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(moe_product_workspace_bytes(product, max_rows), 256), dtype=torch.uint8, device=device)


def _p(t, dtype, shape, name, device):
    """Device address of a contiguous tensor on GPU `device` (None -> NULL), with dtype/shape checks."""
    if t is None:
        return None
    if device < 0 or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous GPU tensor, on the same GPU as the others")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _e4m3(t, shape, name, device):
    """Device address of a matrix of e4m3 numbers (float8_e4m3fn, or their bytes)."""
    if t is not None and t.dtype not in (torch.float8_e4m3fn, torch.uint8):
        raise TypeError(f"{name} must be torch.float8_e4m3fn or torch.uint8, got {t.dtype}")
    return _p(t, None, shape, name, device)


def _stream(device):
    """The current HIP stream of GPU `device`, which has to be the current one: kernels are launched there.  (As an integer straight from
    torch: making a stream object of it takes 2.4 of the 8 microseconds of a small call.)"""
    if torch.cuda.current_device() != device:
        raise ValueError(f"the tensors are on GPU {device}, the current one is {torch.cuda.current_device()}")
    return torch._C._cuda_getCurrentRawStream(device)


def _blocks(n: int) -> int:
    return (n + BLOCK - 1) // BLOCK


def moe_grouped_product(x, offsets, w, y, workspace):
    """y[r] = w[e] @ x[r] for the rows r of each expert e; offsets None: one expert, all rows."""
    (R, K), (E, N, _), dt, g = x.shape, w.shape, x.dtype, x.get_device()
    product = MoeProduct(E, N, K, _dtype_code(x))
    _check(lib().moe_grouped_product(ctypes.byref(product), R, _p(x, None, None, "x", g),
                                     _p(offsets, torch.int32, (E + 1,), "offsets", g), _p(w, dt, (E, N, K), "w", g),
                                     _p(y, dt, (R, N), "y", g), _p(workspace, torch.uint8, None, "workspace", g),
                                     workspace.numel(), _stream(g)), "moe_grouped_product")


def moe_grouped_product_dgrad(dy, offsets, w, dx, workspace):
    """dx[r] = w[e]^T @ dy[r]: the gradient of moe_grouped_product with respect to its rows."""
    (R, N), (E, _, K), dt, g = dy.shape, w.shape, dy.dtype, dy.get_device()
    product = MoeProduct(E, N, K, _dtype_code(dy))
    _check(lib().moe_grouped_product_dgrad(ctypes.byref(product), R, _p(dy, None, None, "dy", g),
                                           _p(offsets, torch.int32, (E + 1,), "offsets", g), _p(w, dt, (E, N, K), "w", g),
                                           _p(dx, dt, (R, K), "dx", g), _p(workspace, torch.uint8, None, "workspace", g),
                                           workspace.numel(), _stream(g)), "moe_grouped_product_dgrad")


def moe_grouped_product_wgrad(dy, x, offsets, dw, accumulate: bool, workspace):
    """dw[e] (+)= sum over the rows r of expert e of dy[r] x[r]^T: the gradient with respect to the matrices."""
    (R, N), (_, K), E, dt, g = dy.shape, x.shape, dw.shape[0], dy.dtype, dy.get_device()
    product = MoeProduct(E, N, K, _dtype_code(dy))
    _check(lib().moe_grouped_product_wgrad(ctypes.byref(product), R, _p(dy, None, None, "dy", g), _p(x, dt, (R, K), "x", g),
                                           _p(offsets, torch.int32, (E + 1,), "offsets", g), _p(dw, None, (E, N, K), "dw", g),
                                           _dtype_code(dw), int(bool(accumulate)),
                                           _p(workspace, torch.uint8, None, "workspace", g), workspace.numel(), _stream(g)),
           "moe_grouped_product_wgrad")


def moe_quantize_rows_fp8(x, q, scales):
    """x [R, K] -> e4m3 numbers q [R, K] and a scale for each 128 values of a row, scales [R, ceil(K / 128)]."""
    (R, K), g = x.shape, x.get_device()
    _check(lib().moe_quantize_rows_fp8(R, K, _dtype_code(x), _p(x, None, None, "x", g), _e4m3(q, (R, K), "q", g),
                                       _p(scales, torch.float32, (R, _blocks(K)), "scales", g), _stream(g)),
           "moe_quantize_rows_fp8")


def moe_quantize_weights_fp8(w, q, scales, q_t=None, scales_t=None):
    """w [E, N, K] -> e4m3 numbers q and a scale for each tile of 128 x 128, and both transposed where q_t and scales_t are given."""
    (E, N, K), g = w.shape, w.get_device()
    product = MoeProduct(E, N, K, _dtype_code(w))
    _check(lib().moe_quantize_weights_fp8(ctypes.byref(product), _p(w, None, None, "w", g), _e4m3(q, (E, N, K), "q", g),
                                          _p(scales, torch.float32, (E, _blocks(N), _blocks(K)), "scales", g),
                                          _e4m3(q_t, (E, K, N), "q_t", g),
                                          _p(scales_t, torch.float32, (E, _blocks(K), _blocks(N)), "scales_t", g), _stream(g)),
           "moe_quantize_weights_fp8")


def moe_grouped_product_fp8(xq, x_scales, offsets, wq, w_scales, y, workspace):
    """moe_grouped_product on quantised rows and weights; y is bf16."""
    (R, K), (E, N, _), g = xq.shape, wq.shape, xq.get_device()
    product = MoeProduct(E, N, K, moe.MOE_BF16)
    f32 = torch.float32
    _check(lib().moe_grouped_product_fp8(ctypes.byref(product), R, _e4m3(xq, None, "xq", g),
                                         _p(x_scales, f32, (R, _blocks(K)), "x_scales", g),
                                         _p(offsets, torch.int32, (E + 1,), "offsets", g), _e4m3(wq, (E, N, K), "wq", g),
                                         _p(w_scales, f32, (E, _blocks(N), _blocks(K)), "w_scales", g),
                                         _p(y, torch.bfloat16, (R, N), "y", g),
                                         _p(workspace, torch.uint8, None, "workspace", g), workspace.numel(), _stream(g)),
           "moe_grouped_product_fp8")
