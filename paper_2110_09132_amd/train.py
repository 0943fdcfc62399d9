"""Binding of the operators around and after a model's blocks (the end of include/emb.h): dropout, the norms before
and after a block with its gate and residual scale, the cross entropy over a table's vocabulary.

As in the package's other calls, outputs and workspaces may be passed in; what is not is allocated, of the
stream that the call runs on.  All tensors of a call are on the current device.  A call goes the short way of
dense.py first, where its outputs and workspace are given.
"""
from __future__ import annotations

import ctypes

import torch

from . import (BlockNormArgs, BlockNormGradArgs, EmbError, _call_workspace, _check, _empties, _need, _ptr, _stream,
               lib)
from .dense import _CODES, _MASK64, _fit, _native, _out_rows, _rows2, _scratch, _status

try:
    from torch._C import _cuda_getDevice as _device
except ImportError:
    _device = torch.cuda.current_device


def _here(first, *others):
    """All of these tensors (None: not given) are on the current device."""
    at = first.device
    for t in others:
        if t is not None and t.device != at:
            raise EmbError(f"the tensors of a call are on one device (got {at} and {t.device})")
    if at.index is not None and at.index != _device():
        raise EmbError(f"the tensors are on {at}, the current device is {_device()}")


def _row(t, D, what):
    """A contiguous fp32 row of D elements, or None."""
    if t is not None:
        _need(t, torch.float32, what)
        if t.numel() != D:
            raise EmbError(f"{what} holds {t.numel()} elements; the rows have {D}")
    return _ptr(t)


def _seed(seed):
    """(seed, device seed): a number, or an int64 CUDA tensor of one element that the kernel reads."""
    if isinstance(seed, torch.Tensor):
        _need(seed, torch.int64, "seed")
        if seed.numel() != 1:
            raise EmbError(f"seed holds {seed.numel()} elements, not one")
        return 0, seed
    return int(seed) & _MASK64, None


def dropout(x, p, seed, residual=None, out=None, stream=None):
    """residual + keep x / (1 - p) of the rows x [T, D], the mask from the seed (emb_dropout).

    seed: a whole number, or an int64 CUDA tensor of one element that is read when the kernel runs (for replayed
    graphs).  Returns y [T, D] of x's type; `out` may pass it in, and may be x or residual.  The gradient of x is
    dropout(dy, p, seed)."""
    if out is not None:
        st = _native.dropout(x, p, seed, residual, out, _device(), _stream(stream))
        if st >= 0:
            _check(st, "emb_dropout")
            return out
    code, ldx = _rows2(x, "x")
    T, D = x.shape
    ldr = 0
    if residual is not None:
        _, ldr = _rows2(residual, "residual")
        if residual.shape != x.shape or residual.dtype != x.dtype:
            raise EmbError(f"residual is {tuple(residual.shape)} {residual.dtype}; x is {tuple(x.shape)} {x.dtype}")
    if out is None:
        out, = _empties(stream, x.device, ((T, D), x.dtype))
    _, ldy = _out_rows(out, T, D, x.dtype, "out")
    number, seed_dev = _seed(seed)
    _here(x, residual, out, seed_dev)
    _check(lib.emb_dropout(_ptr(x), code, ldx, T, D, float(p), number, _ptr(seed_dev), _ptr(residual), ldr, _ptr(out),
                           ldy, _stream(stream)), "emb_dropout")
    return out


def _gate(gate, gate_rows, T, D):
    """(address, rows that share one) of a gate [D], or [ceil(T / gate_rows), D]."""
    _fit(gate_rows, "gate_rows", 1 << 63)
    if gate is not None:
        _need(gate, torch.float32, "gate")
    n = -(-T // gate_rows) if gate_rows > 0 else 1
    if gate_rows >= 0 and gate is not None and gate.numel() != n * D:
        raise EmbError(f"gate holds {gate.numel()} elements; {n} rows of {D} are needed")
    return _ptr(gate), gate_rows


def _pair(norm, D, what):
    """Addresses of a norm's weight and bias, each of which may be None."""
    if norm is None:
        return None, None
    weight, bias = norm
    return _row(weight, D, what + " weight"), _row(bias, D, what + " bias")


def _stats(t, T, what):
    if t is not None:
        _need(t, torch.float32, what)
        if t.numel() != 2 * T:
            raise EmbError(f"{what} holds {t.numel()} elements, not 2 x {T}")
    return _ptr(t)


def _flat(norm):
    return (None, None) if norm is None else norm


def _block_rows(x, branch, what):
    """Checks the two kinds of rows; returns (stream code, ld, branch code, ld, T, D)."""
    sc, ldx = _rows2(x, what)
    bc, ldb = _rows2(branch, "branch")
    if x.shape != branch.shape:
        raise EmbError(f"{what} is {tuple(x.shape)}, branch {tuple(branch.shape)}")
    if x.dtype == torch.bfloat16 and branch.dtype != torch.bfloat16:
        raise EmbError(f"{what} of bfloat16 takes a branch of bfloat16 (got {branch.dtype})")
    return sc, ldx, bc, ldb, x.shape[0], x.shape[1]


def block_norm(x, branch, gate=None, gate_rows=0, alpha=1.0, post=(None, None), pre=(None, None), eps=1e-5, p=0.0,
               seed=0, out=None, stream=None):
    """h = alpha x + gate dropout(N_post(branch)) and y = N_pre(h) in one pass (emb_block_norm).

    x [T, D], the residual stream, and branch [T, D], what the block added to it: both of one type, or x float32
    and branch bfloat16.  post and pre: (weight, bias) of the two norms, either of which may be None (1 and 0), or
    None: no norm.  gate: float32 [D], or [ceil(T / gate_rows), D] where gate_rows rows share one.  p, seed: as in
    dropout.  Returns (h of x's type, y of branch's type, post_stats [2, T], pre_stats [2, T]), None in the places
    that no norm fills; `out` may pass those four in, h may be x and y may be branch."""
    if out is not None:
        st = _native.block_norm(x, branch, gate, gate_rows, alpha, post, pre, p, seed, eps, *out, _device(),
                                _stream(stream))
        if st >= 0:
            _check(st, "emb_block_norm")
            return out
    sc, ldx, bc, ldb, T, D = _block_rows(x, branch, "x")
    if out is None:
        made = _empties(stream, x.device, ((T, D), x.dtype), *([((2, T), torch.float32)] * (post is not None)),
                        *([((T, D), branch.dtype), ((2, T), torch.float32)] if pre is not None else []))
        h, rest = made[0], list(made[1:])
        post_stats = rest.pop(0) if post is not None else None
        y, pre_stats = rest if pre is not None else (None, None)
        out = (h, y, post_stats, pre_stats)
    h, y, post_stats, pre_stats = out
    if (post is None) != (post_stats is None) or (pre is None) != (pre_stats is None) or (pre is None) != (y is None):
        raise EmbError("out holds post_stats where there is a norm after the block, y and pre_stats where there is one "
                       "before the next, and None in the other places")
    _, ldh = _out_rows(h, T, D, x.dtype, "h")
    ldy = D if y is None else _out_rows(y, T, D, branch.dtype, "y")[1]
    gate_p, gate_rows = _gate(gate, gate_rows, T, D)
    number, seed_dev = _seed(seed)
    _here(x, branch, gate, h, y, post_stats, pre_stats, seed_dev, *_flat(post), *_flat(pre))
    args = BlockNormArgs(T, D, sc, bc, _ptr(x), ldx, _ptr(branch), ldb, gate_p, gate_rows, *_pair(post, D, "post"),
                         *_pair(pre, D, "pre"), float(alpha), float(eps), float(p), number, _ptr(seed_dev), _ptr(h), ldh,
                         _ptr(y), ldy, _stats(post_stats, T, "post_stats"), _stats(pre_stats, T, "pre_stats"))
    _check(lib.emb_block_norm(ctypes.addressof(args), _stream(stream)), "emb_block_norm")
    return out


def block_norm_backward_workspace_bytes(T, D, gate_rows=0) -> int:
    _fit(T, "T")
    _fit(D, "D")
    _fit(gate_rows, "gate_rows", 1 << 63)
    return int(lib.emb_block_norm_backward_workspace_bytes(T, D, gate_rows))


def block_norm_backward(dh, dy, h, branch, post_stats, pre_stats, gate=None, gate_rows=0, alpha=1.0, post=(None, None),
                        pre=(None, None), p=0.0, seed=0, out=None, workspace=None, stream=None):
    """The gradient of block_norm (emb_block_norm_backward).

    dh [T, D] of h's type (None: 0) and dy [T, D] of branch's type (None where pre_stats is None); h and the
    statistics as the forward call returned them, the rest as it was given.  Returns (dx of h's type, dbranch of
    branch's type, dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias), the last five float32; None in the
    places of a norm or gate that there is not.  `out` may pass those seven in, None in the place of one that is not
    wanted; dx may be dh and dbranch may be dy."""
    if out is not None and workspace is not None:
        st = _native.block_norm_backward(dh, dy, h, branch, gate, gate_rows, alpha, post, pre, p, seed, post_stats,
                                         pre_stats, *out, workspace, _device(), _stream(stream))
        if st >= 0:
            _check(st, "emb_block_norm_backward")
            return out
    sc, ldh, bc, ldb, T, D = _block_rows(h, branch, "h")
    if (post is None) != (post_stats is None) or (pre is None) != (pre_stats is None):
        raise EmbError("post_stats and pre_stats are given where their norms are, and only there")
    lddh = lddy = 0
    for t, like, what in ((dh, h, "dh"), (dy, branch, "dy")):
        if t is not None:
            _rows2(t, what)
            if t.shape != like.shape or t.dtype != like.dtype:
                raise EmbError(f"{what} is {tuple(t.shape)} {t.dtype}; {tuple(like.shape)} {like.dtype} is needed")
    if dh is not None:
        lddh = _rows2(dh, "dh")[1]
    if pre_stats is not None:
        if dy is None:
            raise EmbError("dy is needed where there is a norm before the next block")
        lddy = _rows2(dy, "dy")[1]
    gate_p, gate_rows = _gate(gate, gate_rows, T, D)
    if out is None:
        n = 2 * (post is not None) + 2 * (pre is not None)
        made = _empties(stream, h.device, ((T, D), h.dtype), ((T, D), branch.dtype),
                        *([(gate.shape, torch.float32)] if gate is not None else []),
                        *([((n, D), torch.float32)] if n else []))
        rest = list(made[2:])
        dgate = rest.pop(0) if gate is not None else None
        rows = list(rest[0]) if n else []
        out = (made[0], made[1], dgate, *(rows[:2] if post is not None else (None, None)),
               *(rows[-2:] if pre is not None else (None, None)))
    dx, dbranch, dgate, dw0, db0, dw1, db1 = out
    lddx = D if dx is None else _out_rows(dx, T, D, h.dtype, "dx")[1]
    lddb = D if dbranch is None else _out_rows(dbranch, T, D, branch.dtype, "dbranch")[1]
    if dgate is not None:
        _gate(dgate, gate_rows, T, D)
    number, seed_dev = _seed(seed)
    if workspace is None:
        workspace = _call_workspace(stream, h.device, block_norm_backward_workspace_bytes(T, D, gate_rows))
    _here(h, branch, dh, dy, post_stats, pre_stats, gate, seed_dev, workspace, *out, *_flat(post), *_flat(pre))
    ws, nbytes = _scratch(workspace)
    args = BlockNormGradArgs(T, D, sc, bc, _ptr(dh), lddh, _ptr(dy), lddy, _ptr(h), ldh, _ptr(branch), ldb, gate_p,
                             gate_rows, *_pair(post, D, "post"), _pair(pre, D, "pre")[0],
                             _stats(post_stats, T, "post_stats"), _stats(pre_stats, T, "pre_stats"), float(alpha), float(p),
                             number, _ptr(seed_dev), _ptr(dx), lddx, _ptr(dbranch), lddb, _ptr(dgate),
                             _row(dw0, D, "dpost_weight"), _row(db0, D, "dpost_bias"), _row(dw1, D, "dpre_weight"),
                             _row(db1, D, "dpre_bias"), ws, nbytes)
    _check(lib.emb_block_norm_backward(ctypes.addressof(args), _stream(stream)), "emb_block_norm_backward")
    return out


def _loss_size(size, T, V, D, dtype):
    _fit(T, "T")
    _fit(V, "V", 1 << 63)
    _fit(D, "D")
    if dtype not in _CODES:
        raise EmbError(f"dtype {dtype} is not float32 or bfloat16")
    return int(size(T, V, D, _CODES[dtype]))


def vocab_loss_workspace_bytes(T, V, D, dtype=torch.float32) -> int:
    return _loss_size(lib.emb_vocab_loss_workspace_bytes, T, V, D, dtype)


def vocab_loss_backward_workspace_bytes(T, V, D, dtype=torch.float32) -> int:
    return _loss_size(lib.emb_vocab_loss_backward_workspace_bytes, T, V, D, dtype)


def _loss_rows(x, table, targets):
    """(dtype code, ldx, ldw, T, V, D) of the rows, the table and the targets."""
    code, ldx = _rows2(x, "x")
    _, ldw = _rows2(table, "table")
    if table.dtype != x.dtype or table.shape[1] != x.shape[1]:
        raise EmbError(f"x is {tuple(x.shape)} {x.dtype}, the table {tuple(table.shape)} {table.dtype}")
    _vector(targets, x.shape[0], torch.int32, "targets")
    return code, ldx, ldw, x.shape[0], table.shape[0], x.shape[1]


def _vector(t, n, dtype, what):
    _need(t, dtype, what)
    if t.numel() != n:
        raise EmbError(f"{what} holds {t.numel()} elements for {n} tokens")


def vocab_loss(x, table, targets, smoothing=0.0, out=None, workspace=None, dev_status=None, stream=None):
    """Softmax cross entropy of the rows x [T, D] over the vocabulary of table [V, D], the logits never in memory as a
    whole (emb_vocab_loss).

    x and table of one type, float32 or bfloat16; targets [T] int32, negative: the token has none (loss 0).  Returns
    (loss [T], lse [T]) float32; `out` may pass those in."""
    if out is not None and workspace is not None:
        st = _native.vocab_loss(x, table, targets, smoothing, *out, workspace, dev_status, _device(), _stream(stream))
        if st >= 0:
            _check(st, "emb_vocab_loss")
            return out
    code, ldx, ldw, T, V, D = _loss_rows(x, table, targets)
    if out is None:
        both, = _empties(stream, x.device, ((2, T), torch.float32))
        out = tuple(both)
    loss, lse = out
    _vector(loss, T, torch.float32, "loss")
    _vector(lse, T, torch.float32, "lse")
    if workspace is None:
        workspace = _call_workspace(stream, x.device, vocab_loss_workspace_bytes(T, V, D, x.dtype))
    _here(x, table, targets, loss, lse, workspace, dev_status)
    ws, nbytes = _scratch(workspace)
    _check(lib.emb_vocab_loss(_ptr(x), code, ldx, _ptr(table), ldw, T, V, D, _ptr(targets), float(smoothing), _ptr(loss),
                              _ptr(lse), ws, nbytes, _status(dev_status), _stream(stream)), "emb_vocab_loss")
    return out


def vocab_loss_backward(dloss, x, table, targets, lse, smoothing=0.0, out=None, workspace=None, dev_status=None,
                        stream=None):
    """The gradient of vocab_loss (emb_vocab_loss_backward).

    dloss [T] float32, the gradient of each token's loss, or one element for all of them (a mean's 1 / tokens); lse as
    the forward call returned it.  Returns (dx [T, D], dtable [V, D]) of x's type; `out` may pass those in, None in the
    place of one that is not wanted."""
    if out is not None and workspace is not None:
        st = _native.vocab_loss_backward(dloss, x, table, targets, lse, smoothing, *out, workspace, dev_status, _device(),
                                         _stream(stream))
        if st >= 0:
            _check(st, "emb_vocab_loss_backward")
            return out
    code, ldx, ldw, T, V, D = _loss_rows(x, table, targets)
    _need(dloss, torch.float32, "dloss")
    step = 0 if dloss.numel() == 1 else 1
    if step:
        _vector(dloss, T, torch.float32, "dloss")
    _vector(lse, T, torch.float32, "lse")
    if out is None:
        out = _empties(stream, x.device, ((T, D), x.dtype), ((V, D), x.dtype))
    dx, dtable = out
    lddx = D if dx is None else _out_rows(dx, T, D, x.dtype, "dx")[1]
    lddt = D if dtable is None else _out_rows(dtable, V, D, x.dtype, "dtable")[1]
    if workspace is None:
        workspace = _call_workspace(stream, x.device, vocab_loss_backward_workspace_bytes(T, V, D, x.dtype))
    _here(x, table, targets, dloss, lse, dx, dtable, workspace, dev_status)
    ws, nbytes = _scratch(workspace)
    _check(lib.emb_vocab_loss_backward(_ptr(dloss), step, _ptr(x), code, ldx, _ptr(table), ldw, T, V, D, _ptr(targets),
                                       float(smoothing), _ptr(lse), _ptr(dx), lddx, _ptr(dtable), lddt, ws, nbytes,
                                       _status(dev_status), _stream(stream)), "emb_vocab_loss_backward")
    return out
