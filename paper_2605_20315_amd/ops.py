"""Thin Python binding of the C ABI in include/mixquant.h: same names, argument marshalling only.

The calls of the hot path first go to their native form (csrc/binding.cpp: a call with one launch and its outputs given takes 2.6 to
2.8 us of host time instead of 5.3 to 6.5, 2.2 of them the launch), which returns None, with nothing enqueued, for anything but
plain GPU tensors of the expected types and strides; the general path below it then accepts the call or says what is wrong
with it.  A status that the library returns is raised from either, with the same message.

Every function takes torch tensors that live on the GPU, passes their device pointers and
the current HIP stream to the library, and returns the output tensors.  PyTorch provides
device memory and streams; all arithmetic runs in the HIP kernels.
"""
from __future__ import annotations

import math

import torch

from . import _lib
from ._lib import (MQ_LAYOUT_KTILE, MQ_LAYOUT_LINEAR, MQ_OUT_BF16, MQ_OUT_FP32, MQ_ROPE_LINEAR,  # noqa: F401
                   MQ_ROPE_PLAIN, MQ_ROPE_YARN, MixQuantError)

BLOCK = 16


# The current stream's handle without the torch.cuda.Stream object around it, which costs 2.8 us to build
# against 0.4: two of them were a third of the host time of a small nvfp4_linear call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


class _Unbound:
    """Stands for the native module until the first call on GPU tensors loads it.  Anything else is refused by the
    general path, with neither library loaded."""

    def __getattr__(self, name):
        def first(*args):
            global _fast
            tensors = [a for a in args if isinstance(a, torch.Tensor)]
            if not tensors or not all(t.is_cuda for t in tensors):
                return None
            _fast = _lib.load_binding()
            return getattr(_fast, name)(*args)
        return first


_fast = _Unbound()


def _need_gpu(*tensors) -> None:
    for t in tensors:
        if not t.is_cuda:
            raise MixQuantError("tensors must live on the GPU (the library has no CPU path)")


def _rows_k_ld(x: torch.Tensor):
    if x.dim() != 2 or x.stride(1) != 1:
        raise MixQuantError("expected a 2-D tensor whose last dimension is contiguous")
    ld = x.stride(0) if x.shape[0] > 1 else max(x.stride(0), x.shape[1])
    return x.shape[0], x.shape[1], ld


def nvfp4_global_scale(x_bf16: torch.Tensor, alpha_out: torch.Tensor | None = None) -> torch.Tensor:
    """alpha = max|x| / (6*448) as a one-element float32 device tensor."""
    done = _fast.global_scale(x_bf16, alpha_out)
    if done is not None:
        return done
    _need_gpu(x_bf16)
    assert x_bf16.dtype == torch.bfloat16
    rows, K, ld = _rows_k_ld(x_bf16)
    alpha = alpha_out if alpha_out is not None else torch.empty(1, dtype=torch.float32, device=x_bf16.device)
    rc = _lib.load().nvfp4_global_scale(x_bf16.data_ptr(), rows, K, ld, alpha.data_ptr(), _stream())
    _lib.check(rc, "nvfp4_global_scale")
    return alpha


def nvfp4_quantize(x_bf16: torch.Tensor, alpha: torch.Tensor, codes: torch.Tensor | None = None,
                   scales: torch.Tensor | None = None, layout: int = MQ_LAYOUT_LINEAR):
    """Eq. 2 then Eq. 1 of Section 3.3.  Returns (codes uint8 [rows, K/2], scales uint8 [rows, K/16]);
    with MQ_LAYOUT_KTILE the same two buffers hold the bytes in K-step-major order."""
    done = _fast.quantize(x_bf16, alpha, codes, scales, layout)
    if done is not None:
        return done
    _need_gpu(x_bf16, alpha)
    assert x_bf16.dtype == torch.bfloat16 and alpha.dtype == torch.float32
    rows, K, ld = _rows_k_ld(x_bf16)
    if K % BLOCK:
        _lib.check(2, "nvfp4_quantize")
    if codes is None:
        codes = torch.empty((rows, K // 2), dtype=torch.uint8, device=x_bf16.device)
    if scales is None:
        scales = torch.empty((rows, K // BLOCK), dtype=torch.uint8, device=x_bf16.device)
    assert codes.is_contiguous() and scales.is_contiguous()
    rc = _lib.load().nvfp4_quantize(x_bf16.data_ptr(), rows, K, ld, alpha.data_ptr(),
                                    codes.data_ptr(), scales.data_ptr(), layout, _stream())
    _lib.check(rc, "nvfp4_quantize")
    return codes, scales


def _quant_outputs(rows: int, K: int, device, codes, scales, want_bf16: bool):
    if codes is None:
        codes = torch.empty((rows, K // 2), dtype=torch.uint8, device=device)
    if scales is None:
        scales = torch.empty((rows, K // BLOCK), dtype=torch.uint8, device=device)
    assert codes.is_contiguous() and scales.is_contiguous()
    dbg = torch.empty((rows, K), dtype=torch.bfloat16, device=device) if want_bf16 else None
    return codes, scales, dbg


def nvfp4_quantize_silu_mul(gate_up_bf16: torch.Tensor, alpha: torch.Tensor, codes: torch.Tensor | None = None,
                            scales: torch.Tensor | None = None, layout: int = MQ_LAYOUT_LINEAR,
                            return_bf16: bool = False):
    """NVFP4 of silu(gate) * up for gate_up = [gate | up] of shape [rows, 2K] (fused producer).
    Returns (codes, scales), plus the BF16 tensor that was quantized when return_bf16 is set."""
    if not return_bf16:
        done = _fast.quantize_silu_mul(gate_up_bf16, alpha, codes, scales, layout)
        if done is not None:
            return done
    _need_gpu(gate_up_bf16, alpha)
    assert gate_up_bf16.dtype == torch.bfloat16 and alpha.dtype == torch.float32
    rows, k2, ld = _rows_k_ld(gate_up_bf16)
    if k2 % (2 * BLOCK):
        _lib.check(2, "nvfp4_quantize_silu_mul")
    K = k2 // 2
    codes, scales, p = _quant_outputs(rows, K, gate_up_bf16.device, codes, scales, return_bf16)
    rc = _lib.load().nvfp4_quantize_silu_mul(gate_up_bf16.data_ptr(), rows, K, ld, alpha.data_ptr(),
                                             codes.data_ptr(), scales.data_ptr(), layout,
                                             p.data_ptr() if p is not None else None, K, _stream())
    _lib.check(rc, "nvfp4_quantize_silu_mul")
    return (codes, scales, p) if return_bf16 else (codes, scales)


def nvfp4_quantize_rmsnorm(x_bf16: torch.Tensor, w_bf16: torch.Tensor, eps: float, alpha: torch.Tensor,
                           codes: torch.Tensor | None = None, scales: torch.Tensor | None = None,
                           layout: int = MQ_LAYOUT_LINEAR, return_bf16: bool = False):
    """NVFP4 of x / sqrt(mean(x^2) + eps) * w per row (fused producer).
    Returns (codes, scales), plus the BF16 tensor that was quantized when return_bf16 is set."""
    if not return_bf16:
        done = _fast.quantize_rmsnorm(x_bf16, w_bf16, eps, alpha, codes, scales, layout)
        if done is not None:
            return done
    _need_gpu(x_bf16, w_bf16, alpha)
    assert x_bf16.dtype == torch.bfloat16 and w_bf16.dtype == torch.bfloat16 and alpha.dtype == torch.float32
    rows, K, ld = _rows_k_ld(x_bf16)
    assert w_bf16.shape == (K,) and w_bf16.is_contiguous()
    if K % 64:
        _lib.check(2, "nvfp4_quantize_rmsnorm")
    codes, scales, y = _quant_outputs(rows, K, x_bf16.device, codes, scales, return_bf16)
    rc = _lib.load().nvfp4_quantize_rmsnorm(x_bf16.data_ptr(), rows, K, ld, w_bf16.data_ptr(), float(eps),
                                            alpha.data_ptr(), codes.data_ptr(), scales.data_ptr(), layout,
                                            y.data_ptr() if y is not None else None, K, _stream())
    _lib.check(rc, "nvfp4_quantize_rmsnorm")
    return (codes, scales, y) if return_bf16 else (codes, scales)


def nvfp4_relayout(codes: torch.Tensor, scales: torch.Tensor, from_layout: int, to_layout: int):
    """Copy an NVFP4 tensor into the other byte order (offline weight pre-pack).  Returns (codes, scales)."""
    done = _fast.relayout(codes, scales, from_layout, to_layout)
    if done is not None:
        return done
    _need_gpu(codes, scales)
    rows, K = codes.shape[0], codes.shape[1] * 2
    assert codes.dtype == torch.uint8 and scales.dtype == torch.uint8
    assert codes.is_contiguous() and scales.is_contiguous() and scales.shape == (rows, K // BLOCK)
    oc, os_ = torch.empty_like(codes), torch.empty_like(scales)
    rc = _lib.load().nvfp4_relayout(codes.data_ptr(), scales.data_ptr(), oc.data_ptr(), os_.data_ptr(),
                                    rows, K, from_layout, to_layout, _stream())
    _lib.check(rc, "nvfp4_relayout")
    return oc, os_


def nvfp4_gemm(a_codes, a_scales, a_alpha, b_codes, b_scales, b_alpha, out: int = MQ_OUT_BF16,
               y: torch.Tensor | None = None, layout: int = MQ_LAYOUT_LINEAR) -> torch.Tensor:
    """Y[M, N] = dequant(A)[M, K] . dequant(B)[N, K]^T, FP32 accumulate, BF16 or FP32 out."""
    _need_gpu(a_codes, a_scales, a_alpha, b_codes, b_scales, b_alpha)
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    N = b_codes.shape[0]
    assert b_codes.shape[1] * 2 == K and a_scales.shape == (M, K // BLOCK) and b_scales.shape == (N, K // BLOCK)
    for t in (a_codes, a_scales, b_codes, b_scales):
        assert t.dtype == torch.uint8 and t.is_contiguous()
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16 if out == MQ_OUT_BF16 else torch.float32,
                        device=a_codes.device)
    ldy = y.stride(0) if M > 1 else max(y.stride(0), N)
    rc = _lib.load().nvfp4_gemm(a_codes.data_ptr(), a_scales.data_ptr(), a_alpha.data_ptr(),
                                b_codes.data_ptr(), b_scales.data_ptr(), b_alpha.data_ptr(),
                                M, N, K, y.data_ptr(), ldy, out, layout, _stream())
    _lib.check(rc, "nvfp4_gemm")
    return y


def mq_init() -> None:
    """One-time set-up of the current device (kernel attributes, static scratch address); optional
    except before capturing the calls into a HIP graph."""
    _lib.check(_lib.load().mq_init(), "mq_init")


NOALLOC_SCRATCH_BYTES = 4 << 20


def nvfp4_gemm_noalloc(a_codes, a_scales, a_alpha, b_codes, b_scales, b_alpha, out: int = MQ_OUT_BF16,
                       y: torch.Tensor | None = None, layout: int = MQ_LAYOUT_LINEAR) -> torch.Tensor:
    """nvfp4_gemm_ws with the library's static scratch array as the workspace (allocates nothing;
    pass `y` to keep the binding from allocating the output)."""
    _need_gpu(a_codes, a_scales, a_alpha, b_codes, b_scales, b_alpha)
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    N = b_codes.shape[0]
    assert b_codes.shape[1] * 2 == K and a_scales.shape == (M, K // BLOCK) and b_scales.shape == (N, K // BLOCK)
    for t in (a_codes, a_scales, b_codes, b_scales):
        assert t.dtype == torch.uint8 and t.is_contiguous()
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16 if out == MQ_OUT_BF16 else torch.float32,
                        device=a_codes.device)
    ldy = y.stride(0) if M > 1 else max(y.stride(0), N)
    rc = _lib.load().nvfp4_gemm_noalloc(a_codes.data_ptr(), a_scales.data_ptr(), a_alpha.data_ptr(),
                                        b_codes.data_ptr(), b_scales.data_ptr(), b_alpha.data_ptr(),
                                        M, N, K, y.data_ptr(), ldy, out, layout, _stream())
    _lib.check(rc, "nvfp4_gemm_noalloc")
    return y


def mq_gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    """Workspace size that lets nvfp4_gemm_ws choose its K slabs freely (0: it would use none)."""
    return int(_lib.load().mq_gemm_workspace_bytes(M, N, K))


def nvfp4_gemm_ws(a_codes, a_scales, a_alpha, b_codes, b_scales, b_alpha, workspace: torch.Tensor | None,
                  out: int = MQ_OUT_BF16, y: torch.Tensor | None = None,
                  layout: int = MQ_LAYOUT_LINEAR) -> torch.Tensor:
    """nvfp4_gemm with a caller-owned workspace (any contiguous GPU tensor, or None) for the partial
    sums of small-M problems."""
    done = _fast.gemm_ws(a_codes, a_scales, a_alpha, b_codes, b_scales, b_alpha, workspace, out, y, layout)
    if done is not None:
        return done
    _need_gpu(a_codes, a_scales, a_alpha, b_codes, b_scales, b_alpha)
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    N = b_codes.shape[0]
    assert b_codes.shape[1] * 2 == K and a_scales.shape == (M, K // BLOCK) and b_scales.shape == (N, K // BLOCK)
    for t in (a_codes, a_scales, b_codes, b_scales):
        assert t.dtype == torch.uint8 and t.is_contiguous()
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16 if out == MQ_OUT_BF16 else torch.float32,
                        device=a_codes.device)
    ldy = y.stride(0) if M > 1 else max(y.stride(0), N)
    ws_ptr, ws_bytes = 0, 0
    if workspace is not None:
        assert workspace.is_cuda and workspace.is_contiguous()
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = _lib.load().nvfp4_gemm_ws(a_codes.data_ptr(), a_scales.data_ptr(), a_alpha.data_ptr(),
                                   b_codes.data_ptr(), b_scales.data_ptr(), b_alpha.data_ptr(),
                                   M, N, K, y.data_ptr(), ldy, out, layout, ws_ptr, ws_bytes, _stream())
    _lib.check(rc, "nvfp4_gemm_ws")
    return y


def bf16_gemm(x_bf16: torch.Tensor, w_bf16: torch.Tensor, out: int = MQ_OUT_BF16,
              y: torch.Tensor | None = None) -> torch.Tensor:
    """Y = X . W^T with BF16 inputs and FP32 accumulation (the high-precision baseline)."""
    _need_gpu(x_bf16, w_bf16)
    assert x_bf16.dtype == torch.bfloat16 and w_bf16.dtype == torch.bfloat16
    M, K, ldx = _rows_k_ld(x_bf16)
    N, K2, ldw = _rows_k_ld(w_bf16)
    assert K == K2
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16 if out == MQ_OUT_BF16 else torch.float32,
                        device=x_bf16.device)
    ldy = y.stride(0) if M > 1 else max(y.stride(0), N)
    rc = _lib.load().bf16_gemm(x_bf16.data_ptr(), ldx, w_bf16.data_ptr(), ldw, M, N, K,
                               y.data_ptr(), ldy, out, _stream())
    _lib.check(rc, "bf16_gemm")
    return y


def mq_bf16_gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    """Workspace size that lets bf16_gemm_ws choose its K slabs freely (0: it would use none)."""
    return int(_lib.load().mq_bf16_gemm_workspace_bytes(M, N, K))


def bf16_gemm_ws(x_bf16: torch.Tensor, w_bf16: torch.Tensor, workspace: torch.Tensor | None,
                 out: int = MQ_OUT_BF16, y: torch.Tensor | None = None) -> torch.Tensor:
    """bf16_gemm with a caller-owned workspace (any contiguous GPU tensor, or None) for the partial
    sums of decode batches."""
    done = _fast.bf16_gemm_ws(x_bf16, w_bf16, workspace, out, y)
    if done is not None:
        return done
    _need_gpu(x_bf16, w_bf16)
    assert x_bf16.dtype == torch.bfloat16 and w_bf16.dtype == torch.bfloat16
    M, K, ldx = _rows_k_ld(x_bf16)
    N, K2, ldw = _rows_k_ld(w_bf16)
    assert K == K2
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16 if out == MQ_OUT_BF16 else torch.float32,
                        device=x_bf16.device)
    ldy = y.stride(0) if M > 1 else max(y.stride(0), N)
    ws_ptr, ws_bytes = 0, 0
    if workspace is not None:
        assert workspace.is_cuda and workspace.is_contiguous()
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = _lib.load().bf16_gemm_ws(x_bf16.data_ptr(), ldx, w_bf16.data_ptr(), ldw, M, N, K,
                                  y.data_ptr(), ldy, out, ws_ptr, ws_bytes, _stream())
    _lib.check(rc, "bf16_gemm_ws")
    return y


def nvfp4_linear(x_bf16: torch.Tensor, alpha_x: torch.Tensor, w_codes, w_scales, alpha_w,
                 out: int = MQ_OUT_BF16, y: torch.Tensor | None = None, codes=None, scales=None,
                 layout: int = MQ_LAYOUT_LINEAR, workspace: torch.Tensor | None = None):
    """One prefill linear layer: quantize the activations, then the block-scaled GEMM (two library
    calls).  `layout` is the byte order of the weight arrays and of the activation arrays produced here."""
    done = _fast.linear(x_bf16, alpha_x, w_codes, w_scales, alpha_w, out, y, codes, scales, layout, workspace)
    if done is not None:
        return done
    xc, xs = nvfp4_quantize(x_bf16, alpha_x, codes, scales, layout)
    return nvfp4_gemm_ws(xc, xs, alpha_x, w_codes, w_scales, alpha_w, workspace, out, y, layout)


def mq_nvfp4_matvec_workspace_bytes(M: int, N: int, K: int) -> int:
    """Workspace size that nvfp4_matvec needs (0: none)."""
    return int(_lib.load().mq_nvfp4_matvec_workspace_bytes(M, N, K))


def nvfp4_matvec(x_bf16: torch.Tensor, w_codes: torch.Tensor, w_scales: torch.Tensor, w_alpha: torch.Tensor,
                 out: int = MQ_OUT_BF16, y: torch.Tensor | None = None, layout: int = MQ_LAYOUT_LINEAR,
                 workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Y = X . dequant(W)^T for the few tokens of a decode step: BF16 activations, NVFP4 weights, FP32 accumulation.
    workspace: any contiguous GPU tensor of mq_nvfp4_matvec_workspace_bytes; where that is not 0 and none is given, one is
    taken from torch's allocator for the call."""
    done = _fast.matvec(x_bf16, w_codes, w_scales, w_alpha, out, y, layout, workspace)
    if done is not None:
        return done
    _need_gpu(x_bf16, w_codes, w_scales, w_alpha)
    assert x_bf16.dtype == torch.bfloat16 and w_alpha.dtype == torch.float32
    M, K, ldx = _rows_k_ld(x_bf16)
    N = w_codes.shape[0]
    for t in (w_codes, w_scales):
        assert t.dtype == torch.uint8 and t.is_contiguous()
    if K % BLOCK:
        _lib.check(2, "nvfp4_matvec")
    assert w_codes.shape == (N, K // 2) and w_scales.shape == (N, K // BLOCK)
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16 if out == MQ_OUT_BF16 else torch.float32, device=x_bf16.device)
    assert y.is_cuda and y.shape == (M, N) and (N <= 1 or y.stride(1) == 1)
    assert y.dtype == (torch.bfloat16 if out == MQ_OUT_BF16 else torch.float32)
    ldy = y.stride(0) if M > 1 else max(y.stride(0), N)
    ws_bytes = mq_nvfp4_matvec_workspace_bytes(M, N, K)
    if workspace is None and ws_bytes:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=x_bf16.device)
    ws_ptr = 0
    if workspace is not None:
        assert workspace.is_cuda and workspace.is_contiguous()
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = _lib.load().nvfp4_matvec(x_bf16.data_ptr(), ldx, w_codes.data_ptr(), w_scales.data_ptr(), w_alpha.data_ptr(), M, N, K,
                                  y.data_ptr(), ldy, out, layout, ws_ptr, ws_bytes, _stream())
    _lib.check(rc, "nvfp4_matvec")
    return y


def mq_rope_table(max_pos: int, rot_dim: int, base: float = 10000.0, scaling: int = MQ_ROPE_PLAIN, factor: float = 1.0,
                  original_max_pos: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0, gain: float | None = None,
                  table: torch.Tensor | None = None, device="cuda") -> torch.Tensor:
    """Cosines and sines of the position rotation for kv8_append, float32 [max_pos, rot_dim]; gain: 0.1 ln(factor) + 1 for
    MQ_ROPE_YARN where it is not given, else 1."""
    if gain is None:
        gain = 0.1 * math.log(factor) + 1.0 if scaling == MQ_ROPE_YARN and factor > 0 else 1.0
    if table is None:
        table = torch.empty((max(max_pos, 0), max(rot_dim, 0)), dtype=torch.float32, device=device)
    _need_gpu(table)
    assert table.dtype == torch.float32 and table.shape == (max(max_pos, 0), max(rot_dim, 0)) and table.is_contiguous()
    rc = _lib.load().mq_rope_table(table.data_ptr(), max_pos, rot_dim, base, scaling, factor, original_max_pos, beta_fast, beta_slow,
                                   gain, _stream())
    _lib.check(rc, "mq_rope_table")
    return table


def _heads_ld(x: torch.Tensor):
    """(tokens, heads, D, token stride) of a [T, H, D] tensor whose heads are adjacent."""
    if x.dim() != 3 or x.dtype != torch.bfloat16 or x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != x.shape[2]):
        raise MixQuantError("expected a BF16 [tokens, heads, D] tensor whose heads are adjacent")
    T, H, D = x.shape
    return T, H, D, x.stride(0) if T > 1 else max(x.stride(0), H * D)


def _cache(k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, T, D):
    """Checks of the cache and of the sequences, and their sizes: (pages, P, Hkv, row stride of the table, W, B)."""
    _need_gpu(k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens)
    if k_codes.dim() != 4 or k_codes.shape[3] != D:
        raise MixQuantError("expected a cache of codes [pages, heads, tokens, D]")
    pages, Hkv, P, _ = k_codes.shape
    assert v_codes.shape == k_codes.shape and k_scales.shape == (pages, Hkv) and v_scales.shape == (pages, Hkv)
    for t in (k_codes, k_scales, v_codes, v_scales):
        assert t.dtype == torch.uint8 and t.is_contiguous()
    B = kv_lens.shape[0]
    for t in (page_table, cu_q, kv_lens):
        assert t.dtype == torch.int32
    assert kv_lens.shape == (B,) and cu_q.shape == (B + 1,) and kv_lens.is_contiguous() and cu_q.is_contiguous()
    assert page_table.dim() == 2 and page_table.shape[0] == B and (page_table.shape[1] <= 1 or page_table.stride(1) == 1)
    W = page_table.shape[1]
    return pages, P, Hkv, page_table.stride(0) if B > 1 else max(page_table.stride(0), W), W, B


def kv8_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_codes: torch.Tensor, k_scales: torch.Tensor,
               v_codes: torch.Tensor, v_scales: torch.Tensor, page_table: torch.Tensor, cu_q: torch.Tensor, kv_lens: torch.Tensor,
               table: torch.Tensor | None = None, positions: torch.Tensor | None = None, interleaved: bool = False,
               q_out: torch.Tensor | None = None) -> torch.Tensor:
    """Rotates q [T, Hq, D] and k [T, Hkv, D] and appends k and v to the paged FP8 cache; returns the rotated queries.
    table: what mq_rope_table gives, [max_pos, rot_dim], or None for no rotation.  kv_lens count the new tokens."""
    done = _fast.append(q, k, v, k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, table, positions, interleaved, q_out)
    if done is not None:
        return done
    _need_gpu(q, k, v)
    T, Hq, D, ldq = _heads_ld(q)
    Tk, Hkv, Dk, ldk = _heads_ld(k)
    Tv, Hv, Dv, ldv = _heads_ld(v)
    pages, P, heads, pt_ld, W, B = _cache(k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, T, D)
    assert (Tk, Hkv, Dk) == (Tv, Hv, Dv) == (T, heads, D)
    max_pos, rot = 0, 0
    if table is not None:
        _need_gpu(table)
        assert table.dtype == torch.float32 and table.dim() == 2 and table.is_contiguous()
        max_pos, rot = table.shape
    if positions is not None:
        _need_gpu(positions)
        assert positions.dtype == torch.int32 and positions.shape == (T,) and positions.is_contiguous()
    if q_out is None:
        q_out = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=q.device)
    assert q_out.is_cuda and q_out.dtype == torch.bfloat16 and q_out.shape == (T, Hq, D) and q_out.is_contiguous()
    rc = _lib.load().kv8_append(q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, q_out.data_ptr(), k_codes.data_ptr(),
                                k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(), pages, P, Hq, Hkv, D,
                                page_table.data_ptr(), pt_ld, W, cu_q.data_ptr(), kv_lens.data_ptr(), B, T,
                                table.data_ptr() if rot else None, max_pos, rot, positions.data_ptr() if positions is not None else None,
                                int(bool(interleaved)), _stream())
    _lib.check(rc, "kv8_append")
    return q_out


def mq_kv8_attention_workspace_bytes(T: int, B: int, Hq: int, Hkv: int, D: int) -> int:
    """Workspace size that lets kv8_attention cut long histories across workgroups."""
    return int(_lib.load().mq_kv8_attention_workspace_bytes(T, B, Hq, Hkv, D))


def kv8_attention(q: torch.Tensor, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor, v_scales: torch.Tensor,
                  page_table: torch.Tensor, cu_q: torch.Tensor, kv_lens: torch.Tensor, sm_scale: float, window: int = 0,
                  y: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Causal attention of q [T, Hq, D], the last tokens of their sequences, over the paged FP8 cache; BF16 [T, Hq, D].
    window > 0: a token sees itself and the window - 1 places before it.  workspace: any contiguous GPU tensor of
    mq_kv8_attention_workspace_bytes; without one (None, or a smaller one) no history is cut across workgroups, and one long sequence
    is read by as many workgroups as it has key heads."""
    done = _fast.attention(q, k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, sm_scale, window, y, workspace)
    if done is not None:
        return done
    _need_gpu(q)
    T, Hq, D, ldq = _heads_ld(q)
    pages, P, Hkv, pt_ld, W, B = _cache(k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, T, D)
    if y is None:
        y = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=q.device)
    _need_gpu(y)
    assert y.shape == (T, Hq, D)
    ldy = _heads_ld(y)[3]
    ws_ptr, ws_bytes = 0, 0
    if workspace is not None:
        assert workspace.is_cuda and workspace.is_contiguous()
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = _lib.load().kv8_attention(q.data_ptr(), ldq, k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(),
                                   v_scales.data_ptr(), pages, P, Hq, Hkv, D, page_table.data_ptr(), pt_ld, W, cu_q.data_ptr(),
                                   kv_lens.data_ptr(), B, T, sm_scale, window, y.data_ptr(), ldy, ws_ptr, ws_bytes, _stream())
    _lib.check(rc, "kv8_attention")
    return y


def _here(*tensors) -> None:
    """The kernels run on the current device's stream."""
    _need_gpu(*tensors)
    device = torch.cuda.current_device()
    for t in tensors:
        if t.device.index != device:
            raise MixQuantError(f"a tensor lives on {t.device}, the current device is cuda:{device}")


def _vector(what: str, t: torch.Tensor, n: int, dtype=torch.int32) -> torch.Tensor:
    if t.dtype != dtype or t.shape != (n,) or not t.is_contiguous():
        raise MixQuantError(f"expected {what} as a contiguous {dtype} [{n}]")
    return t


def _ptr(t: torch.Tensor | None):
    return t.data_ptr() if t is not None else None


def _new_tokens(parents: torch.Tensor, cu_q: torch.Tensor, kv_lens: torch.Tensor):
    """Checks of the sequences' new tokens; (T, B)."""
    _here(parents, cu_q, kv_lens)
    T, B = parents.numel(), kv_lens.numel()
    _vector("parents", parents, T)
    _vector("kv_lens", kv_lens, B)
    _vector("cu_q", cu_q, B + 1)
    return T, B


def mq_draft_tree(parents: torch.Tensor, cu_q: torch.Tensor, kv_lens: torch.Tensor, words: int, window: int = 0,
                  tree: torch.Tensor | None = None, positions: torch.Tensor | None = None):
    """(tree, positions) of drafted tokens: int32 [T, words], whose bit j says that a token has the j-th new token of its sequence above it
    or is it, and int32 [T], for kv8_tree_attention and kv8_append.  parents int32 [T]: the number of each token's parent among its
    sequence's new tokens, -1 for none.  words: 32 tokens each, for the longest of the sequences.  window > 0: only the window - 1
    tokens next above."""
    done = _fast.draft_tree(parents, cu_q, kv_lens, words, window, tree, positions)
    if done is not None:
        return done
    T, B = _new_tokens(parents, cu_q, kv_lens)
    words = int(words)
    if tree is None:
        tree = torch.empty((T, max(words, 0)), dtype=torch.int32, device=parents.device)
    if positions is None:
        positions = torch.empty(T, dtype=torch.int32, device=parents.device)
    _here(tree, positions)
    if tree.dtype != torch.int32 or tree.shape != (T, words) or not tree.is_contiguous():
        raise MixQuantError(f"expected tree as a contiguous int32 [tokens, words] of [{T}, {words}]")
    _vector("positions", positions, T)
    rc = _lib.load().mq_draft_tree(parents.data_ptr(), cu_q.data_ptr(), kv_lens.data_ptr(), B, T, words, window, tree.data_ptr(),
                                   positions.data_ptr(), _stream())
    _lib.check(rc, "mq_draft_tree")
    return tree, positions


def kv8_tree_attention(q: torch.Tensor, k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor, v_scales: torch.Tensor,
                       page_table: torch.Tensor, cu_q: torch.Tensor, kv_lens: torch.Tensor, tree: torch.Tensor, sm_scale: float,
                       window: int = 0, positions: torch.Tensor | None = None, y: torch.Tensor | None = None,
                       workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of drafted tokens' queries q [T, Hq, D] over the paged FP8 cache, which holds them as the last tokens of their
    sequences: each sees the places before its sequence's new tokens, and of those its mask's; BF16 [T, Hq, D].  tree: int32 [T, words], what
    mq_draft_tree gives.  window > 0: of the places before them only those behind position - window; positions int32 [T], else
    the tokens' places.  workspace: as in kv8_attention."""
    done = _fast.tree_attention(q, k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, tree, sm_scale, window, positions, y,
                                workspace)
    if done is not None:
        return done
    _here(q, k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, tree)
    T, Hq, D, ldq = _heads_ld(q)
    pages, P, Hkv, pt_ld, W, B = _cache(k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, T, D)
    if tree.dtype != torch.int32 or tree.dim() != 2 or tree.shape[0] != T or not tree.is_contiguous():
        raise MixQuantError(f"expected tree as a contiguous int32 [{T}, words]")
    if positions is not None:
        _here(positions)
        _vector("positions", positions, T)
    if y is None:
        y = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=q.device)
    _here(y)
    if y.shape != (T, Hq, D):
        raise MixQuantError("y has another shape than q")
    ldy = _heads_ld(y)[3]
    ws_ptr, ws_bytes = 0, 0
    if workspace is not None:
        _here(workspace)
        assert workspace.is_contiguous()
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = _lib.load().kv8_tree_attention(q.data_ptr(), ldq, k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(),
                                        v_scales.data_ptr(), pages, P, Hq, Hkv, D, page_table.data_ptr(), pt_ld, W, cu_q.data_ptr(),
                                        kv_lens.data_ptr(), B, T, tree.data_ptr(), tree.shape[1], _ptr(positions), sm_scale, window,
                                        y.data_ptr(), ldy, ws_ptr, ws_bytes, _stream())
    _lib.check(rc, "kv8_tree_attention")
    return y


def mq_sample_workspace_bytes(rows: int, V: int) -> int:
    """Workspace size that mq_sample needs; 0 for rows of at most 8192 logits."""
    return int(_lib.load().mq_sample_workspace_bytes(rows, V))


def mq_sample(logits: torch.Tensor, uniform: torch.Tensor, temperature: torch.Tensor | None = None, top_k: torch.Tensor | None = None,
              top_p: torch.Tensor | None = None, min_p: torch.Tensor | None = None, tokens: torch.Tensor | None = None,
              workspace: torch.Tensor | None = None) -> torch.Tensor:
    """One token from each row of BF16 or FP32 logits [rows, V], as int32 [rows]: the first top_k of the order of falling logits, of
    those the ones with less than top_p of their mass in front of them, of those the ones with at least min_p of the largest
    weight; then the lowest index up to which the kept ones have more than `uniform` of their mass.  The settings are float32 (top_k
    int32) [rows], or None for 1, none, none and none; a temperature of 0 gives the largest logit's index.  workspace: any contiguous GPU
    tensor of mq_sample_workspace_bytes; without one it is taken from torch's allocator for the call."""
    done = _fast.sample(logits, uniform, temperature, top_k, top_p, min_p, tokens, workspace)
    if done is not None:
        return done
    _here(logits, uniform)
    if logits.dtype not in (torch.bfloat16, torch.float32):
        raise MixQuantError("expected BF16 or FP32 logits")
    rows, V, ld = _rows_k_ld(logits)
    _vector("uniform", uniform, rows, torch.float32)
    for name, t, dtype in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                           ("min_p", min_p, torch.float32)):
        if t is not None:
            _here(t)
            _vector(name, t, rows, dtype)
    if tokens is None:
        tokens = torch.empty(rows, dtype=torch.int32, device=logits.device)
    _here(tokens)
    _vector("tokens", tokens, rows)
    ws_bytes = mq_sample_workspace_bytes(rows, V)
    if workspace is None and ws_bytes:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=logits.device)
    ws_ptr = 0
    if workspace is not None:
        _here(workspace)
        assert workspace.is_contiguous()
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = _lib.load().mq_sample(logits.data_ptr(), rows, V, ld, MQ_OUT_BF16 if logits.dtype == torch.bfloat16 else MQ_OUT_FP32,
                               uniform.data_ptr(), _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), tokens.data_ptr(), ws_ptr,
                               ws_bytes, _stream())
    _lib.check(rc, "mq_sample")
    return tokens


def mq_draft_accept(parents: torch.Tensor, tokens: torch.Tensor, sampled: torch.Tensor, cu_q: torch.Tensor, kv_lens: torch.Tensor,
                    path: torch.Tensor | None = None, counts: torch.Tensor | None = None, next: torch.Tensor | None = None,
                    lens: torch.Tensor | None = None):
    """The drafted tokens that the sampled ones confirm: (path, counts, next, lens).  From token 0 of a sequence's new ones on, the lowest
    child whose token is the one sampled at its parent.  path int32 [T]: at cu_q[b] the numbers of b's path, then -1; counts int32 [B]: its
    length; next int32 [B]: the token sampled at its end; lens int32 [B]: the sequence's length with the path alone."""
    done = _fast.draft_accept(parents, tokens, sampled, cu_q, kv_lens, path, counts, next, lens)
    if done is not None:
        return done
    T, B = _new_tokens(parents, cu_q, kv_lens)
    _here(tokens, sampled)
    _vector("tokens", tokens, T)
    _vector("sampled", sampled, T)
    made = []
    for name, t, n in (("path", path, T), ("counts", counts, B), ("next", next, B), ("lens", lens, B)):
        t = torch.empty(n, dtype=torch.int32, device=parents.device) if t is None else t
        _here(t)
        made.append(_vector(name, t, n))
    path, counts, next, lens = made
    rc = _lib.load().mq_draft_accept(parents.data_ptr(), tokens.data_ptr(), sampled.data_ptr(), cu_q.data_ptr(), kv_lens.data_ptr(), B, T,
                                     path.data_ptr(), counts.data_ptr(), next.data_ptr(), lens.data_ptr(), _stream())
    _lib.check(rc, "mq_draft_accept")
    return path, counts, next, lens


def kv8_compact(k_codes: torch.Tensor, k_scales: torch.Tensor, v_codes: torch.Tensor, v_scales: torch.Tensor, page_table: torch.Tensor,
                cu_q: torch.Tensor, kv_lens: torch.Tensor, path: torch.Tensor, counts: torch.Tensor) -> None:
    """Brings the tokens of the paths together in the paged FP8 cache, in place: path and counts as mq_draft_accept gives them, cu_q and
    kv_lens those of the step that appended the drafted tokens."""
    if _fast.compact(k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, path, counts) is not None:
        return
    _here(k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, path, counts)
    if k_codes.dim() != 4:
        raise MixQuantError("expected a cache of codes [pages, heads, tokens, D]")
    T, D = path.numel(), k_codes.shape[3]
    pages, P, Hkv, pt_ld, W, B = _cache(k_codes, k_scales, v_codes, v_scales, page_table, cu_q, kv_lens, T, D)
    _vector("path", path, T)
    _vector("counts", counts, B)
    rc = _lib.load().kv8_compact(k_codes.data_ptr(), k_scales.data_ptr(), v_codes.data_ptr(), v_scales.data_ptr(), pages, P, Hkv, D,
                                 page_table.data_ptr(), pt_ld, W, cu_q.data_ptr(), kv_lens.data_ptr(), B, T, path.data_ptr(),
                                 counts.data_ptr(), _stream())
    _lib.check(rc, "kv8_compact")


def mfma_probe(iters: int = 4000) -> float:
    """Enqueue the matrix-pipe rate probe on the current stream; returns the flop count of the launch."""
    import ctypes
    scratch = torch.zeros(1, dtype=torch.float32, device="cuda")
    flop = ctypes.c_double(0.0)
    rc = _lib.load().mq_mfma_probe(scratch.data_ptr(), iters, _stream(), ctypes.byref(flop))
    _lib.check(rc, "mq_mfma_probe")
    return flop.value


KERNEL_NAMES = ("simple", "fp4_direct", "fp4_small", "bf16_ring", "bf16_stage", "bf16_d2l", "bf16_short", "matvec", "matvec_lds")


def _launches(n: int, out) -> list:
    if n < 0:
        _lib.check(-n, "mq_gemm_launches")
    return [{"kernel": KERNEL_NAMES[l.kernel], "tile": (l.bm, l.bn), "waves": l.waves, "slabs": l.slabs,
             "rows": l.rows, "cols": l.cols} for l in out[:n]]


def mq_gemm_launches(M: int, N: int, K: int, layout: int = MQ_LAYOUT_LINEAR, workspace_bytes: int = 0,
                     compute_units: int = 256) -> list:
    """What the NVFP4 product launches for this problem (host only): kernel, tile, waves, K slabs, part of Y."""
    got = (_lib.Launch * 2)()
    return _launches(_lib.load().mq_gemm_launches(M, N, K, layout, workspace_bytes, compute_units, got), got)


def mq_bf16_gemm_launches(M: int, N: int, K: int, workspace_bytes: int = 0, compute_units: int = 256) -> list:
    """What the BF16 product launches for this problem (host only)."""
    got = (_lib.Launch * 2)()
    return _launches(_lib.load().mq_bf16_gemm_launches(M, N, K, workspace_bytes, compute_units, got), got)


def mq_nvfp4_matvec_launches(M: int, N: int, K: int) -> list:
    """What nvfp4_matvec launches for this problem beside its packing and joining kernels (host only)."""
    got = (_lib.Launch * 1)()
    return _launches(_lib.load().mq_nvfp4_matvec_launches(M, N, K, got), got)


def mq_kv8_attention_launches(pages: int, P: int, Hq: int, Hkv: int, D: int, W: int, B: int, T: int, workspace_bytes: int = 0) -> list:
    """What kv8_attention launches for these sizes (host only): kernel, rows of a tile, whether histories may be cut, workgroups,
    and the places that a sequence has at most."""
    got = (_lib.Kv8Launch * 2)()
    n = _lib.load().mq_kv8_attention_launches(pages, P, Hq, Hkv, D, W, B, T, workspace_bytes, got)
    if n < 0:
        _lib.check(-n, "mq_kv8_attention_launches")
    return [{"kernel": ("few", "many")[l.kernel], "rows": l.rows, "cut": bool(l.cut), "workgroups": l.workgroups, "places": l.places}
            for l in got[:n]]
