"""Binding of the dense operators of a training step (the last part of include/emb.h): layer norm,
the relative position bias, AdamW.

As in the package's other calls, outputs and workspaces may be passed in; what is not is allocated, of the
stream that the call runs on.

A call first goes the short way (csrc/native.c), which reads and checks the tensors in C and makes the
call; where that declines (-1: an argument does not fit, this torch has no C functions to read a tensor
with, or native.c could not be compiled for it), the same checks in Python say what is wrong, or make the
call through ctypes.
"""
from __future__ import annotations

from array import array

import torch

from . import (EMB_ADAMW_BLOCK, EMB_ADAMW_COEFFS_WORDS, EMB_BF16, EMB_F32, EmbError, _call_workspace, _check,
               _empties, _need, _out, _ptr, _stream, lib)

try:
    from . import _native
except ModuleNotFoundError:  # not built (see build.py); one that is there and does not load is an error
    class _native:
        """Declines every call."""

        @staticmethod
        def use(*args):
            return False

        @staticmethod
        def layer_norm(*args):
            return -1

        layer_norm_backward = relative_bias = relative_bias_backward = adamw_step = layer_norm
        dropout = block_norm = block_norm_backward = vocab_loss = vocab_loss_backward = layer_norm

_native.use(getattr(torch.Tensor, "__dlpack_c_exchange_api__", None), torch.Tensor, torch.nn.Parameter)

_CODES = {torch.float32: EMB_F32, torch.bfloat16: EMB_BF16}


def _fit(n, name, top=1 << 31):
    """A whole number that a C integer of 32 bits (64: top = 1 << 63) holds; ctypes would cut others to their
    lowest bits."""
    if not -top <= n < top:
        raise EmbError(f"{name} = {n} is out of range")


def _rows2(t, what):
    """A 2-D CUDA tensor of float32 or bfloat16 whose rows are contiguous; returns (dtype code, elements
    from one row to the next)."""
    code = _CODES.get(t.dtype)
    if code is None or not t.is_cuda or t.dim() != 2:
        raise EmbError(f"{what} must be a 2-D float32 or bfloat16 CUDA tensor (got {t.dtype}, {t.device}, "
                       f"{t.dim()} dimensions)")
    n, D = t.shape
    if (n | D) >> 31:
        raise EmbError(f"{what} is {n} rows of {D} elements: out of range")
    ld, one = t.stride()
    if one != 1 and D > 1:
        raise EmbError(f"the rows of {what} must be contiguous (strides {t.stride()})")
    return code, (ld if n > 1 else D)


def _status(t):
    """Address of a device status word, or of none."""
    if t is not None:
        _out(t, torch.int32, 1, "dev_status")
    return _ptr(t)


def _scratch(t):
    """(address, bytes) of a workspace, or of none."""
    if t is None:
        return None, 0
    if not t.is_cuda or not t.is_contiguous():
        raise EmbError(f"workspace must be a contiguous CUDA tensor (got {t.device}, strides {t.stride()})")
    return _ptr(t), t.numel() * t.element_size()


def _out_rows(t, n, D, dtype, what):
    code, ld = _rows2(t, what)
    if t.shape[0] != n or t.shape[1] != D or t.dtype != dtype:
        raise EmbError(f"{what} is {tuple(t.shape)} {t.dtype}; the call writes ({n}, {D}) {dtype}")
    if ld < D:
        raise EmbError(f"the rows of {what} overlap")
    return code, ld


def _norm_source(x, ids):
    """The rows of layer_norm: (dtype code, ld, V, T, D)."""
    code, ld = _rows2(x, "x")
    if ids is None:
        return code, ld, 0, x.shape[0], x.shape[1]
    _need(ids, torch.int32, "ids")
    T = ids.numel()
    _fit(T, "T")
    return code, ld, x.shape[0], T, x.shape[1]


def layer_norm(x, weight=None, bias=None, eps=1e-5, ids=None, out=None, out_dtype=None, dev_status=None, stream=None):
    """Layer norm of the rows of x [T, D], or of the rows ids [T] of a table x [V, D] (emb_layer_norm).

    Returns (y [T, D] of out_dtype (x's type unless given), mean [T], rstd [T]); `out` may pass those
    three tensors in.  Rows of x and y may lie apart (a column slice of a wider buffer)."""
    if out is None:
        _rows2(x, "x")
        T = x.shape[0] if ids is None else ids.numel()
        _fit(T, "T")
        y, (mean, rstd) = _empties(stream, x.device, ((T, x.shape[1]), out_dtype or x.dtype), ((2, T), torch.float32))
        out = (y, mean, rstd)
    y, mean, rstd = out
    if out_dtype is None or out_dtype == y.dtype:
        st = _native.layer_norm(x, weight, bias, eps, ids, y, mean, rstd, dev_status, _stream(stream))
        if st >= 0:
            _check(st, "emb_layer_norm")
            return out
    code, ldx, V, T, D = _norm_source(x, ids)
    for t, n in ((weight, "weight"), (bias, "bias")):
        if t is not None:
            _out(t, torch.float32, D, n)
    ycode, ldy = _out_rows(y, T, D, out_dtype or y.dtype, "y")
    _out(mean, torch.float32, T, "mean")
    _out(rstd, torch.float32, T, "rstd")
    _check(lib.emb_layer_norm(_ptr(x), code, ldx, _ptr(ids), V, T, D, _ptr(weight), _ptr(bias), float(eps), _ptr(y),
                              ycode, ldy, _ptr(mean), _ptr(rstd), _status(dev_status), _stream(stream)),
           "emb_layer_norm")
    return out


def layer_norm_backward_workspace_bytes(T, D) -> int:
    _fit(T, "T")
    _fit(D, "D")
    return int(lib.emb_layer_norm_backward_workspace_bytes(T, D))


def layer_norm_backward(dy, x, mean, rstd, weight=None, ids=None, out=None, workspace=None, dev_status=None,
                        stream=None):
    """The gradient of layer_norm (emb_layer_norm_backward).

    dy [T, D]; x, weight and ids as in the forward call, mean and rstd as it returned them.  Returns
    (dx [T, D] of dy's type, dweight [D], dbias [D]); `out` may pass those three in, None in the place of
    one that is not wanted."""
    if out is None:
        _rows2(x, "x")
        _rows2(dy, "dy")
        D = x.shape[1]
        dx, (dw, db) = _empties(stream, x.device, ((dy.shape[0], D), dy.dtype), ((2, D), torch.float32))
        out = (dx, dw, db)
    dx, dw, db = out
    if workspace is not None:
        st = _native.layer_norm_backward(dy, x, mean, rstd, weight, ids, dx, dw, db, workspace, dev_status,
                                         _stream(stream))
        if st >= 0:
            _check(st, "emb_layer_norm_backward")
            return out
    xcode, ldx, V, T, D = _norm_source(x, ids)
    gcode, lddy = _rows2(dy, "dy")
    if dy.shape[0] != T or dy.shape[1] != D:
        raise EmbError(f"dy is {tuple(dy.shape)}; the rows are ({T}, {D})")
    _out(mean, torch.float32, T, "mean")
    _out(rstd, torch.float32, T, "rstd")
    if weight is not None:
        _out(weight, torch.float32, D, "weight")
    lddx = D
    if dx is not None:
        _, lddx = _out_rows(dx, T, D, dy.dtype, "dx")
    for t, n in ((dw, "dweight"), (db, "dbias")):
        if t is not None:
            _out(t, torch.float32, D, n)
    if workspace is None and (dw is not None or db is not None):
        workspace = _call_workspace(stream, x.device, layer_norm_backward_workspace_bytes(T, D))
    ws, nbytes = _scratch(workspace)
    _check(lib.emb_layer_norm_backward(_ptr(dy), gcode, lddy, _ptr(x), xcode, ldx, _ptr(ids), V, T, D, _ptr(weight),
                                       _ptr(mean), _ptr(rstd), _ptr(dx), lddx, _ptr(dw), _ptr(db), ws, nbytes,
                                       _status(dev_status), _stream(stream)), "emb_layer_norm_backward")
    return out


def relative_buckets(num_buckets, max_distance, causal=False, device=None):
    """The usual bucket map of the relative position bias (emb_relative_buckets), [2 * max_distance + 1]
    int32 on the device; causal: keys after the query are masked (-1)."""
    _fit(num_buckets, "num_buckets")
    _fit(max_distance, "max_distance")
    host = torch.empty(2 * max(int(max_distance), 0) + 1, dtype=torch.int32)
    _check(lib.emb_relative_buckets(num_buckets, max_distance, 1 if causal else 0, host.data_ptr()),
           "emb_relative_buckets")
    return host.to(device or "cuda")


def _radius(bucket_of):
    _need(bucket_of, torch.int32, "bucket_of")
    n = bucket_of.numel()
    if n % 2 != 1:
        raise EmbError(f"bucket_of holds {n} entries; a map of the differences -R .. R has 2 R + 1")
    _fit(n // 2, "R")
    return n // 2


def _fit_bias(N, H, Q, K, num_buckets, q0):
    if (N | H | Q | K | num_buckets) >> 31 not in (0, -1):  # negative ones are for the call to refuse
        raise EmbError(f"N = {N}, H = {H}, Q = {Q}, K = {K}, num_buckets = {num_buckets}: out of range")
    _fit(q0, "q0", 1 << 63)


def relative_bias(table, bucket_of, Q, K, q0=0, out=None, out_dtype=torch.float32, dev_status=None, stream=None):
    """out[h, i, j] = table[bucket_of[clamp(j - (q0 + i), -R, R) + R], h] (emb_relative_bias).

    table [num_buckets, H] fp32, bucket_of [2 R + 1] int32 (relative_buckets, or any map; negative entries
    mask: -infinity).  Returns out [H, Q, K], which may be passed in; its rows may lie apart."""
    if out is not None:
        st = _native.relative_bias(table, bucket_of, Q, K, q0, out, dev_status, _stream(stream))
        if st >= 0:
            _check(st, "emb_relative_bias")
            return out
    _need(table, torch.float32, "table")
    if table.dim() != 2:
        raise EmbError("table must be 2-D [num_buckets, H]")
    B, H = table.shape
    R = _radius(bucket_of)
    _fit_bias(1, H, Q, K, B, q0)
    if out is None:
        if Q < 0 or K < 0:
            raise EmbError(f"Q = {Q} and K = {K} must not be negative")
        out, = _empties(stream, table.device, ((H, Q, K), out_dtype))
    code = _CODES.get(out.dtype)
    if code is None or not out.is_cuda or tuple(out.shape) != (H, Q, K):
        raise EmbError(f"out must be a float32 or bfloat16 CUDA tensor ({H}, {Q}, {K}) (got {out.dtype}, "
                       f"{out.device}, {tuple(out.shape)})")
    ldh, ldq, one = out.stride()
    if one != 1 and K > 1:
        raise EmbError(f"the rows of out must be contiguous (strides {out.stride()})")
    if Q <= 1:
        ldq = K
    _check(lib.emb_relative_bias(_ptr(table), B, H, _ptr(bucket_of), R, Q, K, q0, _ptr(out), code, ldq, ldh,
                                 _status(dev_status), _stream(stream)), "emb_relative_bias")
    return out


def relative_bias_backward_workspace_bytes(N, H, Q, K) -> int:
    _fit_bias(N, H, Q, K, 1, 0)
    return int(lib.emb_relative_bias_backward_workspace_bytes(N, H, Q, K))


def relative_bias_backward(grad, bucket_of, num_buckets, q0=0, out=None, workspace=None, dev_status=None,
                           stream=None):
    """The gradient of relative_bias's table (emb_relative_bias_backward).

    grad [N, H, Q, K] (or [H, Q, K]), the gradient of the scores that the bias was added to, for every
    batch entry; its rows may lie apart.  Returns dtable [num_buckets, H] fp32, which may be passed in."""
    if out is not None and workspace is not None:
        st = _native.relative_bias_backward(grad, bucket_of, num_buckets, q0, out, workspace, dev_status,
                                            _stream(stream))
        if st >= 0:
            _check(st, "emb_relative_bias_backward")
            return out
    code = _CODES.get(grad.dtype)
    if code is None or not grad.is_cuda or grad.dim() not in (3, 4):
        raise EmbError(f"grad must be a float32 or bfloat16 CUDA tensor [N, H, Q, K] or [H, Q, K] (got {grad.dtype}, "
                       f"{grad.device}, {grad.dim()} dimensions)")
    strides = grad.stride() if grad.dim() == 4 else (0, *grad.stride())
    N, H, Q, K = grad.shape if grad.dim() == 4 else (1, *grad.shape)
    ldn, ldh, ldq, one = strides
    if one != 1 and K > 1:
        raise EmbError(f"the rows of grad must be contiguous (strides {grad.stride()})")
    R = _radius(bucket_of)
    _fit_bias(N, H, Q, K, num_buckets, q0)
    if out is None:
        out, = _empties(stream, grad.device, ((num_buckets, H), torch.float32))
    _out(out, torch.float32, num_buckets * H, "out")
    if workspace is None:
        workspace = _call_workspace(stream, grad.device, relative_bias_backward_workspace_bytes(N, H, Q, K))
    ws, nbytes = _scratch(workspace)
    _check(lib.emb_relative_bias_backward(_ptr(grad), code, N, H, Q, K, ldn, ldh, ldq, _ptr(bucket_of), R, num_buckets,
                                          q0, _ptr(out), ws, nbytes, _status(dev_status), _stream(stream)),
           "emb_relative_bias_backward")
    return out


def adamw_state8(param):
    """Zero moments in 8 bits for a parameter: (exp_avg float8_e4m3fn, exp_avg_sq float8_e5m2, scales); a
    moment is its value times its block's scale (emb_adamw_tensor in include/emb.h)."""
    n = param.numel()
    blocks = -(-n // EMB_ADAMW_BLOCK)
    return (torch.zeros(n, dtype=torch.uint8, device=param.device).view(torch.float8_e4m3fn).view(param.shape),
            torch.zeros(n, dtype=torch.uint8, device=param.device).view(torch.float8_e5m2).view(param.shape),
            torch.zeros(2 * blocks, dtype=torch.float32, device=param.device))


def adamw_coeffs(lr, beta1, beta2, eps, weight_decay, step, out, seed=0):
    """Write one adamw_step's coefficients (emb_adamw_coeffs) into `out`, a float32 CPU tensor of
    EMB_ADAMW_COEFFS_WORDS elements (for instance a row of a pinned buffer)."""
    if out.dtype != torch.float32 or out.device.type != "cpu" or not out.is_contiguous() or \
            out.numel() < EMB_ADAMW_COEFFS_WORDS:
        raise EmbError(f"out must be a contiguous float32 CPU tensor of {EMB_ADAMW_COEFFS_WORDS} elements")
    _fit(step, "step", 1 << 63)
    _check(lib.emb_adamw_coeffs(lr, beta1, beta2, eps, weight_decay, step, seed & _MASK64, out.data_ptr()),
           "emb_adamw_coeffs")
    return out


_MASK64 = (1 << 64) - 1


def _same(ts, dtype, sizes, what):
    """Addresses of a list of contiguous CUDA tensors of these sizes."""
    if len(ts) != len(sizes):
        raise EmbError(f"{len(ts)} {what} for {len(sizes)} parameters")
    for t, n in zip(ts, sizes):
        if t.dtype != dtype or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
            _need(t, dtype, what)
            raise EmbError(f"one of {what} has {t.numel()} elements; its parameter's call uses {n}")
    return [t.data_ptr() for t in ts]


def _adamw_table(params, grads, exp_avgs, exp_avg_sqs, scales, copies):
    """(emb_adamw_tensor structs, gradient dtype code) of the lists; raises where one does not fit."""
    sizes = [p.numel() for p in params]
    n = len(sizes)
    p = _same(params, torch.float32, sizes, "params")
    gt = grads[0].dtype if n and len(grads) else torch.float32
    code = _CODES.get(gt)
    if code is None:
        raise EmbError(f"gradient dtype {gt} is not float32 or bfloat16")
    g = _same(grads, gt, sizes, "grads")
    none = [0] * n
    if scales is None:
        s = none
        m = _same(exp_avgs, torch.float32, sizes, "exp_avgs")
        v = _same(exp_avg_sqs, torch.float32, sizes, "exp_avg_sqs")
    else:
        m = _same(exp_avgs, torch.float8_e4m3fn, sizes, "exp_avgs")
        v = _same(exp_avg_sqs, torch.float8_e5m2, sizes, "exp_avg_sqs")
        s = _same(scales, torch.float32, [2 * -(-k // EMB_ADAMW_BLOCK) for k in sizes], "scales")
    c = none if copies is None else _same(copies, torch.bfloat16, sizes, "copies")
    words = [0] * (7 * n)  # seven words each, written column by column
    for k, column in enumerate((p, g, m, v, s, c, sizes)):
        words[k::7] = column
    return array("q", words), code


def adamw_step(params, grads, exp_avgs, exp_avg_sqs, lr, beta1, beta2, eps, weight_decay, step, scales=None,
               copies=None, grad_scale=None, seed=0, coeffs=None, dev_status=None, stream=None):
    """One AdamW step of a list of parameters, in place (emb_adamw_step).

    params float32; grads all float32 or all bfloat16; exp_avgs and exp_avg_sqs float32, or with `scales`
    (see adamw_state8) float8_e4m3fn and float8_e5m2.  copies: bfloat16 tensors that receive the updated
    parameters.  grad_scale: one float32 on the device that the gradients are multiplied by.  seed: of
    the random rounding of 8-bit moments (the step number enters beside it).  coeffs: adamw_coeffs in
    device memory, read in place of lr .. seed when the step runs."""
    st = _native.adamw_step(params, grads, exp_avgs, exp_avg_sqs, scales, copies, lr, beta1, beta2, eps, weight_decay,
                            step, seed, coeffs, grad_scale, dev_status, _stream(stream))
    if st >= 0:
        _check(st, "emb_adamw_step")
        return
    _fit(step, "step", 1 << 63)
    table, code = _adamw_table(params, grads, exp_avgs, exp_avg_sqs, scales, copies)
    bits = 32 if scales is None else 8
    if grad_scale is not None:
        _out(grad_scale, torch.float32, 1, "grad_scale")
    if coeffs is not None:
        _out(coeffs, torch.float32, EMB_ADAMW_COEFFS_WORDS, "coeffs")
    _check(lib.emb_adamw_step(table.buffer_info()[0], len(params), code, bits, lr, beta1, beta2, eps, weight_decay, step,
                              seed & _MASK64, _ptr(coeffs), _ptr(grad_scale), _status(dev_status), _stream(stream)),
           "emb_adamw_step")
