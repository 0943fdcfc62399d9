"""Plain 64-bit forms of dropout, the norms around a block and the cross entropy over a vocabulary, on the CPU, with
the bounds that an fp32 evaluation keeps (U, R16 and the bounds of layer norm: dense_ref.py).

Bounds are first order in the roundings with a margin of a tenth for the rest.  A product of N x D by D x V on the
matrix instructions adds up D products in fp32, in an order of its own; where it cuts instead of rounding a step is
2 U instead of U, which is what is taken."""
import numpy as np
import torch

import dense_ref as ref
from dense_ref import R16, TINY, U, f64

M64 = (1 << 64) - 1
GAMMA = 0x9E3779B97F4A7C15


def mix64(z):
    """SplitMix64's output function on numpy uint64."""
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def cut_of(p):
    return min(65535, int(round(65536 * p)))


def kept(T, D, p, seed):
    """[T, D] truth values: the elements that stay."""
    per = -(-D // 4)
    key = mix64(np.array([seed & M64], dtype=np.uint64))
    with np.errstate(over="ignore"):
        draws = mix64(key + (np.arange(T * per, dtype=np.uint64) + np.uint64(1)) * np.uint64(GAMMA))
    bits = draws.astype("<u8").view("<u2").reshape(T, 4 * per)[:, :D]
    return torch.from_numpy(bits.astype(np.int64) >= cut_of(p))


def scale_of(p):
    return 65536.0 / (65536 - cut_of(p))


def dropout(x, p, seed, residual=None):
    """(y, bound): the scale, the product and the sum are rounded once each."""
    xs = torch.where(kept(*x.shape, p, seed), f64(x) * scale_of(p), 0.0)
    y = xs if residual is None else f64(residual) + xs
    return y, 2 * U * xs.abs() + U * y.abs() + ref.rounding(x.dtype, y)


def gate_of(gate, gate_rows, T, D):
    if gate is None:
        return torch.ones(1, D, dtype=torch.float64)
    g = f64(gate).reshape(-1, D)
    return g[torch.arange(T) // gate_rows] if gate_rows else g


def _norm(x, wb, eps, dx):
    """Layer norm of x that is known to dx; bounds with what dx adds."""
    r = ref.layer_norm(x, *wb, eps)
    w = torch.ones(x.shape[1], dtype=torch.float64) if wb[0] is None else f64(wb[0])
    rstd, xh = r["rstd"][:, None], (x - r["mean"][:, None]) * r["rstd"][:, None]
    rms, mean = (dx ** 2).mean(1, keepdim=True).sqrt(), dx.mean(1, keepdim=True)
    r["tol"] = r["tol"] + 1.1 * w.abs() * rstd * (dx + mean + xh.abs() * rms)
    r["mean_tol"] = r["mean_tol"] + mean[:, 0]
    r["rstd_tol"] = r["rstd_tol"] + 1.1 * r["rstd"] ** 2 * rms[:, 0]
    return r


def block_norm(x, branch, gate, gate_rows, alpha, post, pre, eps, p, seed):
    x, n = f64(x), f64(branch)
    T, D = x.shape
    out, n_tol = {}, torch.zeros_like(n)
    if post is not None:
        out["post"] = _norm(n, post, eps, n_tol)
        n, n_tol = out["post"]["y"], out["post"]["tol"]
    s, keep, g = scale_of(p), kept(T, D, p, seed), gate_of(gate, gate_rows, T, D)
    add = torch.where(keep, g * n * s, 0.0)
    h = alpha * x + add
    # scale, its product, the gate's; alpha, its product, the sum (or one fused rounding of both)
    h_tol = torch.where(keep, g.abs() * s * n_tol, 0.0) + 3 * U * add.abs() + 2 * U * (alpha * x).abs() + U * h.abs()
    out["h"], out["h_tol"] = h, 1.1 * h_tol
    if pre is not None:
        out["pre"] = _norm(h, pre, eps, out["h_tol"])
    return out


def _norm_backward(dy, dy_tol, x, stats, w):
    """layer_norm_backward of a dy that is known to dy_tol."""
    r = ref.layer_norm_backward(dy, x, stats[0], stats[1], w)
    mean, rstd = f64(stats[0])[:, None], f64(stats[1])[:, None]
    xh = (f64(x) - mean) * rstd
    wd = dy_tol * (1.0 if w is None else f64(w).abs())
    r["dx_tol"] = r["dx_tol"] + 1.1 * rstd * (wd + wd.mean(1, keepdim=True) + xh.abs() * (wd * xh.abs()).mean(1, keepdim=True))
    r["dw_tol"] = r["dw_tol"] + 1.1 * (dy_tol * xh.abs()).sum(0) + 2 * U * (f64(dy) * xh).abs().sum(0)
    r["db_tol"] = r["db_tol"] + 1.1 * dy_tol.sum(0)
    return r


def block_norm_backward(dh, dy, h, branch, post_stats, pre_stats, gate, gate_rows, alpha, post, pre, p, seed):
    T, D = h.shape
    d = torch.zeros(T, D, dtype=torch.float64) if dh is None else f64(dh)
    d_tol, out = torch.zeros_like(d), {}
    if pre is not None:
        r = _norm_backward(f64(dy), torch.zeros_like(d), h, pre_stats, pre[0])
        d_tol = r["dx_tol"] + U * (d + r["dx"]).abs()
        d = d + r["dx"]
        out["dpre_weight"], out["dpre_bias"] = (r["dw"], r["dw_tol"]), (r["db"], r["db_tol"])
    s, keep, g = scale_of(p), kept(T, D, p, seed), gate_of(gate, gate_rows, T, D)
    out["dx"] = (alpha * d, 1.1 * (abs(alpha) * d_tol + 2 * U * (alpha * d).abs()))
    dn = torch.where(keep, d * g * s, 0.0)
    dn_tol = torch.where(keep, 1.1 * (g.abs() * s * d_tol + 4 * U * dn.abs()), 0.0)
    n = f64(branch)
    n_tol = torch.zeros_like(n)
    if post is not None:
        r = _norm_backward(dn, dn_tol, branch, post_stats, post[0])
        out["dbranch"] = r["dx"], r["dx_tol"]
        out["dpost_weight"], out["dpost_bias"] = (r["dw"], r["dw_tol"]), (r["db"], r["db_tol"])
        w = torch.ones(D, dtype=torch.float64) if post[0] is None else f64(post[0])
        b = torch.zeros(D, dtype=torch.float64) if post[1] is None else f64(post[1])
        n = (n - f64(post_stats[0])[:, None]) * f64(post_stats[1])[:, None] * w
        n_tol = 4 * U * (n.abs() + b.abs())
        n = n + b
    else:
        out["dbranch"] = dn, dn_tol
    each = torch.where(keep, d * n * s, 0.0)
    each_tol = torch.where(keep, 1.1 * s * (d_tol * n.abs() + d.abs() * n_tol) + 4 * U * each.abs(), 0.0)
    rows = gate_rows or max(T, 1)
    G = -(-T // rows) if gate_rows else 1
    at = torch.arange(T) // rows
    sums = [torch.zeros(G, D, dtype=torch.float64).index_add_(0, at, v) for v in (each, each_tol, each.abs())]
    out["dgate"] = sums[0], sums[1] + (min(rows, T) + 4) * U * sums[2] + TINY
    return out


def logits(x, table):
    """z and its bound: D products added up, and for fp32 the products of the planes that are left out."""
    x, w = f64(x), f64(table)
    return x @ w.t(), (2.2 * (x.shape[1] + 8) * U + 4 * U) * (x.abs() @ w.abs().t()) + TINY


def vocab_loss(x, table, targets, smoothing):
    targets = targets.cpu().long()
    V = table.shape[0]
    z, z_tol = logits(x, table)
    live = (targets >= 0) & (targets < V)
    lse = torch.logsumexp(z, 1)
    at = targets.clamp(0, V - 1)[:, None]
    loss = lse - (1 - smoothing) * z.gather(1, at)[:, 0] - smoothing * z.mean(1)
    p = torch.exp(z - lse[:, None])
    # a term's exponent is rounded twice and exp2 is good to two units; a lane adds up 64 terms of every tile of 256 that
    # its run has (8 tiles here at most), then come the joins of lanes, waves and runs, 16 at most
    chain = 64 * min(8, -(-V // 256)) + 16
    rel = (p * (z_tol + 4 * U * (z - z.amax(1, keepdim=True)).abs())).sum(1) + (chain + 8) * U
    lse_tol = 1.1 * rel + 2 * U * lse.abs() + 2 * U * z.amax(1).abs() + TINY
    mean_tol = smoothing * (z_tol.mean(1) + (chain + 4) * U * z.abs().mean(1))
    loss_tol = lse_tol + z_tol.gather(1, at)[:, 0] + 1.1 * mean_tol + 3 * U * (
        lse.abs() + z.gather(1, at)[:, 0].abs() + z.mean(1).abs())
    zero = torch.zeros_like(loss)
    return dict(loss=torch.where(live, loss, zero), loss_tol=loss_tol, lse=torch.where(live, lse, zero), lse_tol=lse_tol)


def vocab_loss_backward(dloss, x, table, targets, lse, smoothing):
    targets = targets.cpu().long()
    T, V = x.shape[0], table.shape[0]
    live = (targets >= 0) & (targets < V)
    z, z_tol = logits(x, table)
    lse, d = f64(lse)[:, None], f64(dloss).expand(T)[:, None]
    p = torch.exp(z - lse)
    hot = torch.zeros_like(z)
    hot[torch.nonzero(live)[:, 0], targets[live]] = 1.0
    g = d * (p - (1 - smoothing) * hot - smoothing / V)
    g_tol = 1.1 * d.abs() * (p * (z_tol + 4 * U * (z - lse).abs() + 4 * U) + 3 * U * (p + hot + smoothing / V))
    # g is rounded once to an operand of bf16, or of three planes of it
    g_tol = g_tol + (R16 if x.dtype == torch.bfloat16 else 2 * U) * g.abs()
    g, g_tol = (torch.where(live[:, None], v, 0.0) for v in (g, g_tol))
    a, b = f64(x), f64(table)
    a = torch.where(live[:, None], a, 0.0)
    dx, dx_tol = g @ b, 1.1 * (g_tol @ b.abs()) + 2.2 * (V + 8) * U * (g.abs() @ b.abs()) + TINY
    dw, dw_tol = g.t() @ a, 1.1 * (g_tol.t() @ a.abs()) + 2.2 * (T + 8) * U * (g.abs().t() @ a.abs()) + TINY
    return dict(dx=dx, dx_tol=dx_tol + ref.rounding(x.dtype, dx), dtable=dw, dtable_tol=dw_tol + ref.rounding(x.dtype, dw))
