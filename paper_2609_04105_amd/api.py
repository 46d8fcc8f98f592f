"""Torch-facing wrappers of the C-ABI (argument marshalling only).

Shapes follow include/fp4attn.h.  Inputs must be contiguous CUDA (HIP) tensors;
outputs are allocated with torch unless passed in.  Work is enqueued on the
current torch stream of the tensors' device.

The calls of the attention path go through ``_binding`` (csrc/binding.cpp), which
checks, allocates and launches natively and returns None for arguments that it does
not take as they stand; those calls, and every error, go through the checks here.
``_binding`` is built for one torch: where it is missing or does not load, every call
goes through the checks here, with the same results and about 7 us more host time.
"""
import ctypes
import math
import operator
import warnings
from typing import NamedTuple

import torch

from ._lib import FP4ATTN_BF16, FP4ATTN_F32, AttentionOptions, Cache, ForwardOptions, check, lib


class _NoBinding:
    """Takes no call."""

    @staticmethod
    def _leave(*args):
        return None

    forward = quantize_qkv = attention = forward_bf16 = _leave
    rotary = cache_write = cache_read = cache_assign = cache_attention = _leave


try:
    from . import _binding   # needs torch loaded
except ImportError as e:
    _binding = _NoBinding
    warnings.warn(f"the native call path _binding.so is missing or does not load with this torch ({e}): calls take "
                  "more host time until it is built with `python paper_2609_04105_amd/build.py`", RuntimeWarning,
                  stacklevel=2)

_DTYPES = {torch.float32: FP4ATTN_F32, torch.bfloat16: FP4ATTN_BF16}


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr())


def _stream(t):
    # the raw handle of torch's current stream on t's device (the same value as
    # torch.cuda.current_stream(device).cuda_stream, without building a Stream)
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(t.get_device()))


def _same_device(*tensors):
    """The one device every tensor of a call lives on (the library launches on the
    current HIP device, so each call runs with that device made current)."""
    dev = tensors[0].device
    for t in tensors[1:]:
        if t.device != dev:
            raise ValueError(f"tensors of one call must share a device: {dev} and {t.device}")
    return dev


def _native(r):
    """The result of a native call; raises its status."""
    return check(r) if r.__class__ is int else r


def _launch(device, fn, *args):
    if device.index == torch.cuda.current_device():
        check(fn(*args))
        return
    with torch.cuda.device(device):
        check(fn(*args))


def _need(t, name, dtype=None, ndim=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if ndim is not None and t.ndim != ndim:
        raise ValueError(f"{name} must have {ndim} dimensions, got shape {tuple(t.shape)}")


def quantize_mxfp4(x, axis=-1, n_anchor=0):
    """MXFP4 codes and E8M0 scales of ``x`` [..., rows, cols] (fp32 or bf16).

    axis=-1: blocks of 32 along cols -> codes [..., rows, cols/2], scales [..., rows, cols/32].
    axis=-2: blocks along rows, stored transposed -> codes [..., cols, rows/2], scales [..., cols, rows/32].
    n_anchor > 0: the rows are taken in anchor order (fp4attn_quantize_mxfp4_anchored).
    """
    _need(x, "x", (torch.float32, torch.bfloat16))
    if x.dim() < 2:
        raise ValueError("x needs at least two dimensions")
    lead = tuple(x.shape[:-2])
    rows, cols = x.shape[-2:]
    batch = math.prod(lead) if lead else 1
    if axis in (-1, x.dim() - 1):
        c_axis, cshape, sshape = 1, lead + (rows, cols // 2), lead + (rows, cols // 32)
    elif axis in (-2, x.dim() - 2):
        c_axis, cshape, sshape = 0, lead + (cols, rows // 2), lead + (cols, rows // 32)
    else:
        raise ValueError("axis must be -1 or -2")
    codes = torch.empty(cshape, dtype=torch.uint8, device=x.device)
    scales = torch.empty(sshape, dtype=torch.uint8, device=x.device)
    if n_anchor:
        _launch(x.device, lib.fp4attn_quantize_mxfp4_anchored, _ptr(x), _DTYPES[x.dtype], batch, rows, cols, c_axis,
                n_anchor, _ptr(codes), _ptr(scales), _stream(x))
    else:
        _launch(x.device, lib.fp4attn_quantize_mxfp4, _ptr(x), _DTYPES[x.dtype], batch, rows, cols, c_axis,
                _ptr(codes), _ptr(scales), _stream(x))
    return codes, scales


def quantize_mxfp8(x, axis=-1):
    """MXFP8 (E4M3 + E8M0 per 32) codes and scales of ``x`` [..., rows, cols], one
    code byte per value; axis as :func:`quantize_mxfp4`."""
    _need(x, "x", (torch.float32, torch.bfloat16))
    if x.dim() < 2:
        raise ValueError("x needs at least two dimensions")
    lead = tuple(x.shape[:-2])
    rows, cols = x.shape[-2:]
    batch = math.prod(lead) if lead else 1
    if axis in (-1, x.dim() - 1):
        c_axis, cshape, sshape = 1, lead + (rows, cols), lead + (rows, cols // 32)
    elif axis in (-2, x.dim() - 2):
        c_axis, cshape, sshape = 0, lead + (cols, rows), lead + (cols, rows // 32)
    else:
        raise ValueError("axis must be -1 or -2")
    codes = torch.empty(cshape, dtype=torch.uint8, device=x.device)
    scales = torch.empty(sshape, dtype=torch.uint8, device=x.device)
    _launch(x.device, lib.fp4attn_quantize_mxfp8, _ptr(x), _DTYPES[x.dtype], batch, rows, cols, c_axis, _ptr(codes),
            _ptr(scales), _stream(x))
    return codes, scales


def _one_launch(q, k, v):
    """Whether Q, K and V can be quantized together: GPU tensors of one shape, type
    and device (otherwise each is quantized, and checked, by itself)."""
    return (isinstance(q, torch.Tensor) and isinstance(k, torch.Tensor) and isinstance(v, torch.Tensor)
            and q.is_cuda and q.dtype in _DTYPES and q.dim() >= 2 and q.dtype == k.dtype == v.dtype
            and q.shape == k.shape == v.shape and q.device == k.device == v.device
            and q.is_contiguous() and k.is_contiguous() and v.is_contiguous())


def quantize_qkv(q, k, v, anchored=False, pv_fp8=False):
    """Operands of the forward: MXFP4 Q, K along d; V along the sequence
    (transposed), MXFP4 or, with ``pv_fp8``, MXFP8.  ``anchored``: K and V in the
    anchor key order of the guarded forward (128 anchors)."""
    r = _binding.quantize_qkv(q, k, v, anchored, pv_fp8)
    if r is not None:
        return _native(r)
    n_anchor = 128 if anchored else 0
    if _one_launch(q, k, v) and not (anchored and pv_fp8):
        lead, (rows, cols) = q.shape[:-2], q.shape[-2:]
        def empty(*shape):
            return torch.empty(lead + shape, dtype=torch.uint8, device=q.device)
        out = (empty(rows, cols // 2), empty(rows, cols // 32), empty(rows, cols // 2), empty(rows, cols // 32),
               empty(cols, rows if pv_fp8 else rows // 2), empty(cols, rows // 32))
        _launch(q.device, lib.fp4attn_quantize_qkv, _ptr(q), _ptr(k), _ptr(v), _DTYPES[q.dtype], math.prod(lead), rows,
                cols, n_anchor, 1 if pv_fp8 else 0, *(_ptr(t) for t in out), _stream(q))
        return out
    qc, qs = quantize_mxfp4(q, axis=-1)
    kc, ks = quantize_mxfp4(k, axis=-1, n_anchor=n_anchor)
    if pv_fp8:
        if anchored:
            raise ValueError("the FP8 P/V route has no anchored form")
        vc, vs = quantize_mxfp8(v, axis=-2)
    else:
        vc, vs = quantize_mxfp4(v, axis=-2, n_anchor=n_anchor)
    return qc, qs, kc, ks, vc, vs


def _fp4_shape(q_codes):
    _need(q_codes, "q_codes", torch.uint8, 4)
    B, H, N, half_d = q_codes.shape
    return B, H, N, 2 * half_d


def _check_operands(B, H, N, d, ops, pv_fp8=False):
    names = ("q_codes", "q_scales", "k_codes", "k_scales", "vt_codes", "vt_scales")
    shapes = ((B, H, N, d // 2), (B, H, N, d // 32), (B, H, N, d // 2), (B, H, N, d // 32),
              (B, H, d, N if pv_fp8 else N // 2), (B, H, d, N // 32))
    for t, name, shape in zip(ops, names, shapes):
        _need(t, name, torch.uint8, 4)
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")


def _out(out, B, H, N, d, out_dtype, device):
    if out is None:
        return torch.empty((B, H, N, d), dtype=out_dtype, device=device)
    _need(out, "out", (torch.float32, torch.bfloat16), 4)
    if tuple(out.shape) != (B, H, N, d):
        raise ValueError(f"out has shape {tuple(out.shape)}, expected {(B, H, N, d)}")
    return out


def forward_options(affine_a=1.5, affine_b=1.2, ex2_pairs=0, guard=None, causal=False, lse=None, pv_fp8=False):
    """An fp4attn_forward_options struct: the library's defaults, then the given
    fields; ``guard`` = (margin, shift) turns the sampled guard on; ``lse`` is a
    contiguous fp32 GPU tensor [B, H, N] or None."""
    o = ForwardOptions()
    lib.fp4attn_forward_options_init(ctypes.byref(o))
    o.affine_a, o.affine_b, o.ex2_pairs = affine_a, affine_b, ex2_pairs
    if guard is not None:
        o.guard, (o.guard_margin, o.guard_shift) = 1, guard
    o.causal = 1 if causal else 0
    o.pv_fp8 = 1 if pv_fp8 else 0
    if lse is not None:
        _need(lse, "lse", torch.float32, 3)
        o.lse = lse.data_ptr()
    return o


def forward_mxfp4(q_codes, q_scales, k_codes, k_scales, vt_codes, vt_scales, softmax_scale=None,
                  affine_a=1.5, affine_b=1.2, out=None, out_dtype=torch.float32, ex2_pairs=None, guard=None,
                  causal=False, lse=None, pv_fp8=False):
    """Direct-P full-MXFP4 attention forward; returns O [B, H, N, d].

    ``ex2_pairs`` (0, 1, 2, 4, 8 or 16 of the 16 key pairs of each 32-key
    block take the native exponential), ``guard`` = (margin, shift) (the
    sampled guard; K and V from ``quantize_qkv(..., anchored=True)``),
    ``causal``, ``lse`` (an fp32 [B, H, N] tensor that receives the row
    normaliser) or ``pv_fp8`` (FP8 P and V; V from ``quantize_qkv(..., pv_fp8=True)``)
    select the extended entry point; otherwise the plain forward runs.
    """
    r = _binding.forward(q_codes, q_scales, k_codes, k_scales, vt_codes, vt_scales, softmax_scale, affine_a, affine_b,
                         out, out_dtype, ex2_pairs, guard, causal, lse, pv_fp8)
    if r is not None:
        return _native(r)
    B, H, N, d = _fp4_shape(q_codes)
    ops = (q_codes, q_scales, k_codes, k_scales, vt_codes, vt_scales)
    _check_operands(B, H, N, d, ops, pv_fp8)
    out = _out(out, B, H, N, d, out_dtype, q_codes.device)
    dev = _same_device(*ops, out, *(() if lse is None else (lse,)))
    s = 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale
    if ex2_pairs is None and guard is None and not causal and lse is None and not pv_fp8:
        _launch(dev, lib.fp4attn_forward_mxfp4, *(_ptr(t) for t in ops), B, H, N, d, s, affine_a, affine_b, _ptr(out),
                _DTYPES[out.dtype], _stream(out))
    else:
        if lse is not None and tuple(lse.shape) != (B, H, N):
            raise ValueError(f"lse has shape {tuple(lse.shape)}, expected {(B, H, N)}")
        o = forward_options(affine_a, affine_b, ex2_pairs or 0, guard, causal, lse, pv_fp8)
        _launch(dev, lib.fp4attn_forward_mxfp4_ex, *(_ptr(t) for t in ops), B, H, N, d, s, ctypes.byref(o),
                _ptr(out), _DTYPES[out.dtype], _stream(out))
    return out


def attention_mxfp4(q, k, v, softmax_scale=None, causal=False, lse=None, ex2_pairs=None, guard=None,
                    pv_fp8=False, out=None, out_dtype=torch.float32):
    """Quantize ``q``, ``k``, ``v`` ([B, H, N, d], bf16 or fp32) and run the Direct-P
    forward in one call: MXFP4 Q and K; V in MXFP4 or, with ``pv_fp8``, MXFP8; K and
    V in anchor order when ``guard`` is given.  The quantized operands are not kept
    (use :func:`quantize_qkv` and :func:`forward_mxfp4` to reuse them)."""
    r = _binding.attention(q, k, v, softmax_scale, 1.5, 1.2, out, out_dtype, ex2_pairs, guard, causal, lse, pv_fp8)
    if r is not None:
        return _native(r)
    ops = quantize_qkv(q, k, v, anchored=guard is not None, pv_fp8=pv_fp8)
    return forward_mxfp4(*ops, softmax_scale=softmax_scale, out=out, out_dtype=out_dtype, ex2_pairs=ex2_pairs,
                         guard=guard, causal=causal, lse=lse, pv_fp8=pv_fp8)


def debug_directp_mxfp4(q_codes, q_scales, k_codes, k_scales, vt_codes, vt_scales, row_ids, softmax_scale=None,
                        affine_a=1.5, affine_b=1.2, out_dtype=torch.float32, wg_clock=False, ex2_pairs=0,
                        guard=None, causal=False, lse=False, pv_fp8=False):
    """Forward plus the Direct-P state of the (strictly ascending) flattened ``row_ids``.

    Returns a dict: out, p_codes [R, N/2] uint8 ([R, N] E4M3 bytes with
    ``pv_fp8``), block_exp [R, N/32] int16, row_m [R] int32, row_d [R] fp32,
    with ``lse`` also lse [B, H, N], and with ``wg_clock`` also wg_clock
    [B*H*N/128, 2] int64 (per workgroup: shader-clock cycles, 100 MHz ticks;
    rows past the launch's workgroup count stay zero).
    """
    B, H, N, d = _fp4_shape(q_codes)
    ops = (q_codes, q_scales, k_codes, k_scales, vt_codes, vt_scales)
    _check_operands(B, H, N, d, ops, pv_fp8)
    _need(row_ids, "row_ids", torch.int64, 1)
    R = row_ids.numel()   # 0: no dump, the launch is the plain forward kernel
    dev = _same_device(*ops, row_ids)
    out = torch.empty((B, H, N, d), dtype=out_dtype, device=dev)
    res = {
        "out": out,
        "p_codes": torch.empty((R, N if pv_fp8 else N // 2), dtype=torch.uint8, device=dev),
        "block_exp": torch.empty((R, N // 32), dtype=torch.int16, device=dev),
        "row_m": torch.empty((R,), dtype=torch.int32, device=dev),
        "row_d": torch.empty((R,), dtype=torch.float32, device=dev),
    }
    if wg_clock:
        res["wg_clock"] = torch.zeros((B * H * N // 128, 2), dtype=torch.int64, device=dev)
    if lse:
        res["lse"] = torch.empty((B, H, N), dtype=torch.float32, device=dev)
    s = 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale
    o = forward_options(affine_a, affine_b, ex2_pairs, guard, causal, res.get("lse"), pv_fp8)
    _launch(dev, lib.fp4attn_debug_directp_mxfp4, *(_ptr(t) for t in ops), B, H, N, d, s, ctypes.byref(o),
            _ptr(out), _DTYPES[out_dtype], _ptr(row_ids) if R else None, R, _ptr(res["p_codes"]),
            _ptr(res["block_exp"]), _ptr(res["row_m"]), _ptr(res["row_d"]),
            _ptr(res["wg_clock"]) if wg_clock else None, _stream(out))
    return res


def debug_mfma_stream(a_codes, b_codes, blocks, iters):
    """Sustained FP4 matrix-unit stream on given operands (fp4attn_debug_mfma_stream):
    ``blocks`` x 256 threads, each with 64 bytes of ``a_codes`` and of ``b_codes``
    (uint8, at least blocks * 256 * 64 bytes each); returns the per-thread
    accumulator sums [blocks * 256] fp32 and the flop count of the launch."""
    need = blocks * 256 * 64
    for t, name in ((a_codes, "a_codes"), (b_codes, "b_codes")):
        _need(t, name, torch.uint8)
        if t.numel() < need:
            raise ValueError(f"{name} holds {t.numel()} bytes, the launch reads {need}")
    dev = _same_device(a_codes, b_codes)
    out = torch.empty(blocks * 256, dtype=torch.float32, device=dev)
    _launch(dev, lib.fp4attn_debug_mfma_stream, _ptr(a_codes), _ptr(b_codes), blocks, iters, _ptr(out), _stream(out))
    return out, blocks * 4 * iters * 4 * 2.0 * 32 * 32 * 64


def forward_bf16(q, k, v, softmax_scale=None, out=None, out_dtype=torch.float32):
    """Same-design BF16 attention forward; q, k, v [B, H, N, d] bf16."""
    r = _binding.forward_bf16(q, k, v, softmax_scale, out, out_dtype)
    if r is not None:
        return _native(r)
    _need(q, "q", torch.bfloat16, 4)
    _need(k, "k", torch.bfloat16, 4)
    _need(v, "v", torch.bfloat16, 4)
    B, H, N, d = q.shape
    if tuple(k.shape) != (B, H, N, d) or tuple(v.shape) != (B, H, N, d):
        raise ValueError("q, k and v must all be [B, H, N, d]")
    out = _out(out, B, H, N, d, out_dtype, q.device)
    dev = _same_device(q, k, v, out)
    s = 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale
    _launch(dev, lib.fp4attn_forward_bf16, _ptr(q), _ptr(k), _ptr(v), B, H, N, d, s, _ptr(out), _DTYPES[out.dtype],
            _stream(out))
    return out


def _tokens(t, name, dtype, heads=None, d=None):
    """Checks a [tokens, heads, d] tensor whose tokens may lie apart (a slice of a fused
    projection); returns the stride of a token."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype not in dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.ndim != 3 or (heads is not None and tuple(t.shape[1:]) != (heads, d)):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected [tokens, {heads or 'heads'}, {d or 'd'}]")
    if t.numel() and not t[0].is_contiguous():
        raise ValueError(f"the heads of a token of {name} must be contiguous, got strides {t.stride()}")
    return t.stride(0)


def _overlaps_itself(t):
    """Whether two elements of ``t`` may share memory."""
    reach = 1
    for stride, size in sorted((st, n) for n, st in zip(t.shape, t.stride()) if n > 1):
        if stride < reach:
            return True
        reach = stride * size
    return False


def rotary_frequencies(rotary_dim, base=10000.0, scaling=None, factor=1.0, original_length=None, fast_turns=32.0,
                       slow_turns=1.0, device="cuda"):
    """Radians per position of each pair of :func:`rotary`, ``base ** (-2 j / rotary_dim)`` in
    fp64, and the magnitude that goes with them.  ``scaling`` stretches a model's context by
    ``factor``:

    * ``"linear"``: every angle divided by ``factor`` (position interpolation);
    * ``"ntk"``: a larger base, ``base * factor ** (r / (r - 2))``, which keeps the fastest
      pair and divides the slowest by ``factor``;
    * ``"yarn"``: pairs that turn more than ``fast_turns`` times in ``original_length``
      positions keep their angle, those under ``slow_turns`` are divided by ``factor``, those
      between are mixed linearly; magnitude ``0.1 ln(factor) + 1``.
    """
    r = rotary_dim
    if not isinstance(r, int) or r < 2 or r % 2:
        raise ValueError(f"rotary_dim={r} must be a positive even number")
    if not (base > 1.0 and math.isfinite(base) and factor >= 1.0 and math.isfinite(factor)):
        raise ValueError(f"base={base} must be above 1 and factor={factor} at least 1")
    j = torch.arange(r // 2, dtype=torch.float64)
    magnitude = 1.0
    if scaling == "ntk":
        if r == 2:
            raise ValueError("the ntk scaling needs more than one pair")
        base = base * factor ** (r / (r - 2))
    freq = base ** (-2.0 * j / r)
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "yarn":
        if original_length is None or original_length < 1 or not fast_turns > slow_turns > 0:
            raise ValueError("the yarn scaling needs original_length and fast_turns > slow_turns > 0")
        # the pair that makes `turns` turns in original_length positions
        low, high = (r * math.log(original_length / (2 * math.pi * turns)) / (2 * math.log(base))
                     for turns in (fast_turns, slow_turns))
        low, high = max(math.floor(low), 0), min(math.ceil(high), r - 1)
        mix = ((j - low) / max(high - low, 1e-3)).clamp(0.0, 1.0)
        freq = freq * (1.0 - mix) + freq / factor * mix
        magnitude = 0.1 * math.log(factor) + 1.0
    elif scaling not in (None, "ntk"):
        raise ValueError(f"scaling {scaling!r} is not None, 'linear', 'ntk' or 'yarn'")
    return freq.to(device), magnitude


class _Rotary(torch.autograd.Function):
    """:func:`rotary` with its gradient, the turn back of the result's gradient."""

    @staticmethod
    def forward(ctx, x, positions, inv_freq, interleaved, magnitude, inverse):
        y = rotary(x, positions, inv_freq, interleaved, magnitude, inverse)
        ctx.save_for_backward(positions, inv_freq)
        ctx.back = (interleaved, magnitude, not inverse)
        return y

    @staticmethod
    def backward(ctx, dy):
        return (rotary(dy.contiguous(), *ctx.saved_tensors, *ctx.back), *(None,) * 5)


def rotary(x, positions, inv_freq, interleaved=False, magnitude=1.0, inverse=False, out=None):
    """Rotary positions on ``x`` (bf16 or fp32): [n, H, d] with ``positions`` [n], or [B, H, N, d]
    with ``positions`` [N] or [B, N] (int64).  The first ``2 * len(inv_freq)`` channels of
    every head turn by ``position * inv_freq[j]`` (fp64, :func:`rotary_frequencies`); pairs are
    (j, j + r / 2), or (2 j, 2 j + 1) with ``interleaved``.  ``inverse`` turns back: applied
    to the gradient of the result it gives the gradient of ``x``, which is what autograd does for an ``x``
    that requires one (``positions`` and ``inv_freq`` have none).  ``x`` may have any strides
    with d contiguous; ``out`` may be ``x`` (in place), and autograd does not see what is written to it."""
    if out is None and getattr(x, "requires_grad", False) and torch.is_grad_enabled():
        return _Rotary.apply(x, positions, inv_freq, interleaved, magnitude, inverse)
    r = _binding.rotary(x, positions, inv_freq, interleaved, magnitude, inverse, out)
    if r is not None:
        return _native(r)
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("x must be a GPU tensor")
    if x.dtype not in _DTYPES:
        raise TypeError(f"x has dtype {x.dtype}, expected {tuple(_DTYPES)}")
    if x.ndim not in (3, 4):
        raise ValueError(f"x must be [n, H, d] or [B, H, N, d], got shape {tuple(x.shape)}")
    _need(positions, "positions", torch.int64)
    _need(inv_freq, "inv_freq", torch.float64, 1)
    if x.ndim == 3:
        (N, H, d), B = x.shape, 1
    else:
        B, H, N, d = x.shape
    if tuple(positions.shape) not in (((N,),) if x.ndim == 3 else ((N,), (B, N))):
        raise ValueError(f"positions have shape {tuple(positions.shape)} for x {tuple(x.shape)}")
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        if not isinstance(out, torch.Tensor) or not out.is_cuda:
            raise ValueError("out must be a GPU tensor")
        if out.dtype != x.dtype or out.shape != x.shape:
            raise ValueError(f"out is {out.dtype} {tuple(out.shape)}, expected {x.dtype} {tuple(x.shape)}")
        if _overlaps_itself(out):
            raise ValueError("elements of out share memory")
        if out.numel() and out.data_ptr() == x.data_ptr() and out.stride() != x.stride():
            raise ValueError("out begins where x does, with other strides")
    dev = _same_device(x, positions, inv_freq, out)
    if x.numel() == 0:
        return out
    for t, name in ((x, "x"), (out, "out")):
        if t.stride(-1) != 1 and d != 1:
            raise ValueError(f"the channels of {name} must be contiguous")

    def strides(t):
        st = (0, t.stride(1), t.stride(0)) if t.ndim == 3 else t.stride()[:3]
        sizes = (1, H, N) if t.ndim == 3 else t.shape[:3]
        return (ctypes.c_int64 * 3)(*(s if n > 1 else 0 for s, n in zip(st, sizes)))   # of one element: any

    _launch(dev, lib.fp4attn_rotary, _ptr(x), _ptr(out), _DTYPES[x.dtype], B, H, N, d, strides(x), strides(out),
            _ptr(positions), N if positions.ndim == 2 else 0, _ptr(inv_freq), 2 * inv_freq.numel(), magnitude,
            int(bool(interleaved)), int(bool(inverse)), _stream(x))
    return out


class KVCache(NamedTuple):
    """A paged cache of quantized keys and values (fp4attn_cache in include/fp4attn.h): uint8
    tensors k_codes [pages, heads, page_size, b], k_scales [pages, heads, page_size, d / 32],
    v_codes [pages, heads, page_size / 8, 16, 8, b / 16] and v_scales [pages, heads,
    page_size / 8, d / 32, 8]; b = d / 2 for MXFP4, d for MXFP8."""
    k_codes: torch.Tensor
    k_scales: torch.Tensor
    v_codes: torch.Tensor
    v_scales: torch.Tensor


def kv_cache(pages, heads, page_size, d, fp8=False, device="cuda"):
    """An empty :class:`KVCache` (all bytes zero): MXFP4, or MXFP8 with ``fp8``."""
    if d not in (64, 128) or pages < 1 or heads < 1 or page_size < 16 or page_size & (page_size - 1):
        raise ValueError(f"no cache of {pages} pages of {page_size} tokens, {heads} heads of {d}: sizes from 1, page_size "
                         "a power of two from 16, d 64 or 128")
    b = d if fp8 else d // 2
    return KVCache(*(torch.zeros((pages, heads) + s, dtype=torch.uint8, device=device)
                     for s in ((page_size, b), (page_size, d // 32), (page_size // 8, 16, 8, b // 16),
                               (page_size // 8, d // 32, 8))))


def _cache(cache):
    """The C description of a cache's tensors."""
    if len(cache) != 4:
        raise ValueError("a cache is (k_codes, k_scales, v_codes, v_scales)")
    for t, name, ndim in zip(cache, KVCache._fields, (4, 4, 6, 5)):
        _need(t, name, torch.uint8, ndim)
    k_codes, k_scales, v_codes, v_scales = cache
    pages, H, page, b = k_codes.shape
    d = 32 * k_scales.shape[3]
    shapes = ((pages, H, page, b), (pages, H, page, d // 32), (pages, H, page // 8, 16, 8, b // 16),
              (pages, H, page // 8, d // 32, 8))
    for t, name, shape in zip(cache, KVCache._fields, shapes):
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    if b not in (d, d // 2):
        raise ValueError(f"k_codes has {b} bytes a token for d = {d}")
    _same_device(*cache)
    return Cache(ctypes.sizeof(Cache), int(b == d), pages, H, page, d, *(t.data_ptr() for t in cache))


def cache_write(k, v, cache, slots):
    """Quantize ``k`` and ``v`` ([n, heads, d], bf16 or fp32; tokens may lie apart, as slices of
    a fused projection do) into ``slots`` (int64 [n], page * page_size + place) of ``cache``.
    Slots outside the cache (-1) mark padding and are skipped."""
    r = _binding.cache_write(k, v, cache, slots)
    if r is not None:
        _native(r)
        return
    c = _cache(cache)
    types = tuple(_DTYPES)
    ks, vs = _tokens(k, "k", types, c.heads, c.head_dim), _tokens(v, "v", types, c.heads, c.head_dim)
    if k.dtype != v.dtype:
        raise TypeError(f"k is {k.dtype} and v {v.dtype}")
    _need(slots, "slots", torch.int64, 1)
    n = slots.numel()
    if k.shape[0] != n or v.shape[0] != n:
        raise ValueError(f"{k.shape[0]} keys and {v.shape[0]} values for {n} slots")
    dev = _same_device(k, v, slots, cache[0])
    if n:
        _launch(dev, lib.fp4attn_cache_write, ctypes.byref(c), _ptr(k), _ptr(v), _DTYPES[k.dtype], n, ks if n > 1 else 0,
                vs if n > 1 else 0, _ptr(slots), _stream(k))


def cache_read(cache, slots, out_dtype=torch.float32):
    """(k, v), each [n, heads, d]: the values that ``slots`` (int64 [n]) of ``cache`` stand for;
    zeros for slots outside it."""
    r = _binding.cache_read(cache, slots, out_dtype)
    if r is not None:
        return _native(r)
    c = _cache(cache)
    _need(slots, "slots", torch.int64, 1)
    if out_dtype not in _DTYPES:
        raise TypeError(f"out_dtype {out_dtype} is not one of {tuple(_DTYPES)}")
    dev = _same_device(slots, cache[0])
    n = slots.numel()
    k, v = (torch.empty((n, c.heads, c.head_dim), dtype=out_dtype, device=dev) for _ in range(2))
    if n:
        _launch(dev, lib.fp4attn_cache_read, ctypes.byref(c), _ptr(slots), n, _ptr(k), _ptr(v), _DTYPES[out_dtype],
                _stream(slots))
    return k, v


class KVPool(NamedTuple):
    """Free pages of a cache (fp4attn_cache_assign in include/fp4attn.h): ``free`` int32 [size], a ring, and
    ``counts`` int64 [2], the pages taken from it and those that came to it so far."""
    free: torch.Tensor
    counts: torch.Tensor


class CacheStep(NamedTuple):
    """What :func:`cache_assign` makes for a step: ``slots`` (:func:`cache_write`) and ``positions``
    (:func:`rotary`) int64 [tokens], ``q_starts`` int32 [B + 1] and ``lengths`` int32 [B]
    (:func:`cache_attention`), and the pool after it."""
    slots: torch.Tensor
    positions: torch.Tensor
    q_starts: torch.Tensor
    lengths: torch.Tensor
    pool: KVPool


def cache_pool(pages, first=0, device="cuda"):
    """A :class:`KVPool` of pages ``first`` to ``pages - 1`` of a cache, all free, with room for the others."""
    if not 0 <= first < pages:
        raise ValueError(f"no pool of pages {first} to {pages - 1}")
    free = torch.arange(first, first + pages, dtype=torch.int32, device=device)
    free[pages - first:] = -1
    return KVPool(free, torch.tensor([0, pages - first], dtype=torch.int64, device=device))


def cache_assign(page_table, held, lengths, pool, page_size, tokens, new=None, shared=None, in_place=False):
    """Pages, slots and positions of a step's ``tokens`` tokens; returns a :class:`CacheStep`.

    ``page_table`` [B, max_pages], ``held`` and ``lengths`` [B] (keys before the step, and after it with the new
    tokens) are int32.  Rows of ``page_table`` grow by pages of ``pool``, whose ``free`` takes the pages that are
    returned (both are written in place).  ``new`` (int32 [B]): new tokens of each sequence, the last of its keys; without it
    ``tokens / B`` each; tokens past their sum are padding.  ``shared`` (int32 [B]): keys at the start of a
    sequence whose whole pages belong to others.

    Pages go out in the order of the sequences; one that the pool cannot serve, and every later one that asks
    for pages, keeps what it held: its length in the result is ``held``, and its tokens have slot -1.  ``in_place`` writes the
    lengths and counts after the step into ``held`` and ``pool.counts``, for captured steps."""
    r = _binding.cache_assign(page_table, held, lengths, pool, page_size, tokens, new, shared, in_place)
    if r is not None:
        slots, positions, starts, after, counts = _native(r)
        return CacheStep(slots, positions, starts, after, KVPool(pool[0], counts))
    _need(page_table, "page_table", torch.int32, 2)
    B, width = page_table.shape
    if len(pool) != 2:
        raise ValueError("a pool is (free, counts)")
    free, counts = pool
    page_size, tokens = operator.index(page_size), operator.index(tokens)
    named = ((held, "held", torch.int32, B), (lengths, "lengths", torch.int32, B), (new, "new", torch.int32, B),
             (shared, "shared", torch.int32, B), (free, "pool.free", torch.int32, None), (counts, "pool.counts", torch.int64, 2))
    used = [page_table]
    for t, name, dtype, size in named:
        if t is None and name in ("new", "shared"):
            continue
        _need(t, name, dtype, 1)
        if size is not None and t.numel() != size:
            raise ValueError(f"{name} has {t.numel()} entries, expected {size}")
        used.append(t)
    dev = _same_device(*used)
    n = max(tokens, 0)   # below 0: the call says so
    slots, positions = (torch.empty(n, dtype=torch.int64, device=dev) for _ in range(2))
    starts = torch.empty(B + 1, dtype=torch.int32, device=dev)
    after, counts_after = (held, counts) if in_place else (torch.empty_like(held), torch.empty_like(counts))
    size = lib.fp4attn_cache_assign_workspace(B, tokens)
    work = torch.empty(size, dtype=torch.uint8, device=dev) if size > 0 else None   # -1: the call says why
    _launch(dev, lib.fp4attn_cache_assign, _ptr(page_table), B, width, page_size, _ptr(held), _ptr(lengths),
            None if new is None else _ptr(new), None if shared is None else _ptr(shared), _ptr(free), free.numel(),
            _ptr(counts), tokens, _ptr(slots), _ptr(positions), _ptr(starts), _ptr(after), _ptr(counts_after),
            None if work is None else _ptr(work), max(size, 0), _stream(page_table))
    return CacheStep(slots, positions, starts, after, KVPool(free, counts_after))


def cache_attention(q, cache, page_table, lengths, q_starts=None, max_q=None, tree=None, softmax_scale=None, out=None,
                    lse=None, out_dtype=torch.float32, softcap=None, slopes=None, window=None, prefix=None, shared=0):
    """Attention of new tokens over ``cache``; returns O [n, Hq, d] (``out_dtype``, or ``out``).

    ``q`` [n, Hq, d] bf16 (tokens may lie apart), Hq a multiple of the cache's heads;
    ``page_table`` [B, max_pages] and ``lengths`` [B] int32, the lengths with the new tokens,
    whose keys and values are in the cache already.  Without ``q_starts`` every sequence
    has n / B tokens; with it (int32 [B + 1]) sequence b has rows ``q_starts[b]`` to
    ``q_starts[b + 1]``, at most ``max_q`` of them, and other rows of ``out`` and ``lse`` are left as they were.

    The table's width chooses the launch before the lengths are known: one no wider than the
    longest sequence needs is the fastest.

    Token t of T sees the keys up to its own, or with ``tree`` (int64 [n], or [n, words] for more
    than 64 tokens) the keys before the new tokens and the new tokens u whose bit is set.
    ``lse`` (fp32 [n, Hq]) receives the log normaliser.  A row that sees no key is 0 (-inf).

    With a token at position p: ``softcap`` c caps its scores, z becomes c tanh(z / c); ``slopes`` (fp32 [Hq]) then take
    slope |p - j| off the score of key j; ``window`` hides keys up to p - window; ``prefix``
    (int32 [B]) shows the first keys of a sequence to all of its new tokens.  A tree goes with ``softcap`` only.

    ``shared``: the first ``shared`` keys of every sequence are the same (a system prompt, in the same pages or in
    copies).  They are then read once for the batch where that is faster; the result is the same but for the order of sums.
    Sequences that end inside them are served by themselves."""
    if slopes is not None and getattr(slopes, "requires_grad", False) and torch.is_grad_enabled():
        raise ValueError("slopes get no gradient here: detach them, or call under torch.no_grad()")
    r = _binding.cache_attention(q, cache, page_table, lengths, q_starts, max_q, tree, softmax_scale, out, lse, out_dtype,
                                 softcap, slopes, window, prefix, shared)
    if r is not None:
        return _native(r)
    c = _cache(cache)
    H, d = c.heads, c.head_dim
    stride = _tokens(q, "q", (torch.bfloat16,))
    n, Hq = q.shape[:2]
    if q.shape[2] != d or Hq == 0 or Hq % H:
        raise ValueError(f"q has shape {tuple(q.shape)}, expected [tokens, a multiple of {H}, {d}]")
    _need(page_table, "page_table", torch.int32, 2)
    _need(lengths, "lengths", torch.int32, 1)
    B = lengths.numel()
    if B == 0 or page_table.shape[0] != B or page_table.shape[1] == 0:
        raise ValueError(f"page_table has shape {tuple(page_table.shape)} for {B} sequences")
    used = [q, page_table, lengths, cache[0]]
    if q_starts is not None:
        _need(q_starts, "q_starts", torch.int32, 1)
        if q_starts.numel() != B + 1:
            raise ValueError(f"q_starts has {q_starts.numel()} entries for {B} sequences")
        if max_q is None:
            raise ValueError("q_starts needs max_q, the tokens of the longest sequence")
        used.append(q_starts)
    else:
        if n % B or max_q not in (None, n // B):
            raise ValueError(f"{n} tokens are not {B} sequences of {max_q or 'one length'}: pass q_starts and max_q")
        max_q = n // B
    words = 0
    if tree is not None:
        _need(tree, "tree", torch.int64)
        if tree.ndim not in (1, 2) or tree.shape[0] != n:
            raise ValueError(f"tree has shape {tuple(tree.shape)}, expected [{n}] or [{n}, words]")
        words = tree.shape[1] if tree.ndim == 2 else 1
        used.append(tree)
    o = AttentionOptions(ctypes.sizeof(AttentionOptions))
    if softcap is not None:
        if not softcap > 0:
            raise ValueError(f"softcap={softcap} must be positive")
        o.softcap = softcap
        if o.softcap == 0:   # (0 would be no cap)
            raise ValueError(f"softcap={softcap} is not in [2^-64, 2^64]")
    if window is not None:
        if operator.index(window) < 1:
            raise ValueError(f"window={window} must be positive")
        o.window = min(operator.index(window), 1 << 40)   # (above 2^30 the call refuses it)
    o.shared = max(-1, min(operator.index(shared), 1 << 40))
    if slopes is not None:
        _need(slopes, "slopes", torch.float32, 1)
        if slopes.numel() != Hq:
            raise ValueError(f"slopes have {slopes.numel()} entries for {Hq} heads")
        o.slopes = slopes.data_ptr()
        used.append(slopes)
    if prefix is not None:
        _need(prefix, "prefix", torch.int32, 1)
        if prefix.numel() != B:
            raise ValueError(f"prefix has {prefix.numel()} entries for {B} sequences")
        o.prefix = prefix.data_ptr()
        used.append(prefix)
    if out is None:
        if out_dtype not in _DTYPES:
            raise TypeError(f"out_dtype {out_dtype} is not one of {tuple(_DTYPES)}")
        out = torch.empty((n, Hq, d), dtype=out_dtype, device=q.device)
    else:
        _need(out, "out", tuple(_DTYPES), 3)
        if tuple(out.shape) != (n, Hq, d):
            raise ValueError(f"out has shape {tuple(out.shape)}, expected {(n, Hq, d)}")
    if lse is not None:
        _need(lse, "lse", torch.float32, 2)
        if tuple(lse.shape) != (n, Hq):
            raise ValueError(f"lse has shape {tuple(lse.shape)}, expected {(n, Hq)}")
        used.append(lse)
    dev = _same_device(*used, out)
    if n == 0:
        return out
    ref, opts = ctypes.byref(c), ctypes.byref(o)
    size = lib.fp4attn_cache_attention_ex_workspace(ref, n, Hq, B, page_table.shape[1], max_q, opts)
    work = torch.empty(size, dtype=torch.uint8, device=dev) if size > 0 else None   # -1: the call says why
    _launch(dev, lib.fp4attn_cache_attention_ex, ref, _ptr(q), n, Hq, stride if n > 1 else 0, B, _ptr(page_table),
            page_table.shape[1], _ptr(lengths), None if q_starts is None else _ptr(q_starts), max_q,
            None if tree is None else _ptr(tree), words, 1.0 / math.sqrt(d) if softmax_scale is None else softmax_scale,
            opts, _ptr(out), _DTYPES[out.dtype], None if lse is None else _ptr(lse), None if work is None else _ptr(work),
            max(size, 0), _stream(q))
    return out
