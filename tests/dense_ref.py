"""Plain 64-bit forms of the dense operators on the CPU, with the bounds that an fp32 evaluation keeps.

U is the largest relative error of rounding to nearest in fp32 (24 significant bits: 2**-24), R16 that of
bf16 (8 significant bits: 2**-8).  A sum of n terms in any order is within (n - 1) U sum|x| of the exact sum
(Higham, Accuracy and Stability of Numerical Algorithms, section 4.2).  The row sums of layer norm are
short chains: at most 32 terms per lane for a row held in registers, then 6 levels of lanes and 8 waves;
the widest rows add D / 1024 terms per lane and 16 waves.
"""
import numpy as np
import torch

U = 2.0 ** -24
R16 = 2.0 ** -8
TINY = 2.0 ** -126  # results below the normal range are left out of the relative bounds


def f64(t):
    return t.detach().cpu().double()


def rounding(dtype, value):
    """Bound of the one rounding of a result to its type."""
    return value.abs() * (R16 if dtype == torch.bfloat16 else U) + TINY


def chain(D):
    return max(32, -(-D // 1024)) + 24


def layer_norm(x, w, b, eps):
    x = f64(x)
    D = x.shape[1]
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(var + eps)
    xh = (x - mean) * rstd
    w = torch.ones(D, dtype=torch.float64) if w is None else f64(w)
    b = torch.zeros(D, dtype=torch.float64) if b is None else f64(b)
    n = chain(D)
    dmean = n * U * x.abs().mean(1, keepdim=True) + U * mean.abs()
    # the variance is relative to its own size, but for the shift of the mean, which enters squared
    rel = (n + 8) * U + 0.5 * (dmean * rstd) ** 2
    dxh = rstd * dmean + xh.abs() * (rel + 3 * U)
    y = xh * w + b
    tol = dxh * w.abs() + 2 * U * ((xh * w).abs() + b.abs())
    return dict(y=y, mean=mean[:, 0], rstd=rstd[:, 0], tol=tol, mean_tol=dmean[:, 0] + TINY,
                rstd_tol=rstd[:, 0] * rel[:, 0] + TINY)


def layer_norm_backward(dy, x, mean, rstd, w):
    """mean and rstd as the fp32 values the kernel is given."""
    dy, x = f64(dy), f64(x)
    T, D = x.shape
    mean, rstd = f64(mean)[:, None], f64(rstd)[:, None]
    w = torch.ones(D, dtype=torch.float64) if w is None else f64(w)
    xh = (x - mean) * rstd
    g = dy * w
    c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    n = chain(D)
    dx = rstd * (g - c1 - xh * c2)
    tol = rstd * ((n + 2) * U * g.abs().mean(1, keepdim=True)
                  + xh.abs() * (n + 6) * U * (g * xh).abs().mean(1, keepdim=True)
                  + 4 * U * (g.abs() + c1.abs() + 3 * (xh * c2).abs()))
    dw, db = (dy * xh).sum(0), dy.sum(0)
    return dict(dx=dx, dx_tol=tol, dw=dw, dw_tol=(T + 4) * U * (dy * xh).abs().sum(0) + TINY, db=db,
                db_tol=T * U * dy.abs().sum(0) + TINY)


def assert_within(got, want, tol, what):
    got = f64(got)
    err = (got - want).abs()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    worst = (err / torch.as_tensor(tol)).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times its bound"


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(shape, seed, sigma=1.0):
    return torch.randn(shape, generator=gen(seed)) * sigma


def np_bits(t):
    t = t.detach().cpu().contiguous()
    return t.view(torch.uint8).numpy() if t.numel() else np.zeros(0, np.uint8)


def bias_buckets(bucket_of, Q, K, q0):
    """Bucket of every (query, key) pair, [Q, K] int64, negative where masked."""
    m = bucket_of.detach().cpu().long()
    R = m.numel() // 2
    rel = torch.arange(K)[None, :] - (torch.arange(Q)[:, None] + q0)
    return m[rel.clamp(-R, R) + R]


def relative_bias(table, bucket_of, Q, K, q0, dtype):
    """The bias is a copy, rounded once: equal bit for bit."""
    t = table.detach().cpu()
    b = bias_buckets(bucket_of, Q, K, q0)
    t = torch.cat((t, torch.zeros((1, t.shape[1])), torch.full((1, t.shape[1]), -float("inf"))))
    B = table.shape[0]
    rows = torch.where(b < 0, B + 1, torch.where(b >= B, B, b))
    return t[rows].permute(2, 0, 1).to(dtype)


def relative_bias_backward(grad, bucket_of, num_buckets, q0):
    """(dtable, bound): a bucket's sum has as many terms as pairs."""
    g = f64(grad)
    N, H, Q, K = g.shape
    b = bias_buckets(bucket_of, Q, K, q0).reshape(-1)
    out, tol = torch.zeros((num_buckets, H), dtype=torch.float64), torch.zeros((num_buckets, H), dtype=torch.float64)
    flat = g.permute(2, 3, 0, 1).reshape(Q * K, N, H)
    for k in range(num_buckets):
        here = flat[b == k].reshape(-1, H)
        out[k] = here.sum(0)
        tol[k] = here.shape[0] * U * here.abs().sum(0) + TINY
    return out, tol


# ------------------------------------------------------------------ AdamW
GAMMA = 0x9E3779B97F4A7C15
MASK64 = (1 << 64) - 1
BLOCK = 256


def adamw64(w, g, m, v, h):
    """The definition in 64 bits: (w, m, v) and the bounds of an fp32 evaluation (h: lr, b1, b2, eps, wd, t)."""
    lr, b1, b2, eps, wd, t = h
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    dm = 3 * U * ((b1 * m).abs() + ((1 - b1) * g).abs())      # coefficient, product, sum
    dv = 5 * U * v1.abs()                                      # terms of one sign
    den = torch.sqrt(v1 / (1 - b2 ** t)) + eps
    step = lr / (1 - b1 ** t)
    up = step * m1 / den
    w1 = w * (1 - lr * wd) - up
    # root: half of dv's 5 U, of the coefficient's and the product's roundings, and its own; sum, quotient,
    # product and coefficient of the step one each
    dw = step * dm / den + 12 * U * up.abs() + 4 * U * (w.abs() + up.abs())
    return w1, m1, v1, dw + TINY, dm + TINY, dv + TINY


def moments32(g, m, v, h):
    """m and v operation by operation in fp32, as the header writes them."""
    b1, b2 = h[1], h[2]
    f = np.float32
    with np.errstate(over="ignore", invalid="ignore", under="ignore"):
        return m * f(b1) + g * f(1.0 - b1), v * f(b2) + g * g * f(1.0 - b2)


def mix64(z):
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def random16(k, n, seed, t, start=0):
    """The 16 random bits for m and for v of elements start .. start + n - 1 of tensor k (start even)."""
    def one(z):
        return int(mix64(np.array([z & MASK64], np.uint64))[0])
    key = one(one(seed + t * GAMMA) + (k + 1) * GAMMA)
    j = np.arange(start // 2, start // 2 + (n + 1) // 2, dtype=np.uint64)
    with np.errstate(over="ignore"):
        z = mix64(np.uint64(key) + (j + np.uint64(1)) * np.uint64(GAMMA))
    h = np.stack((z & np.uint64(0xFFFFFFFF), z >> np.uint64(32)), 1).reshape(-1)[:n].astype(np.int64)
    return h & 0xFFFF, h >> 16


def grid8(mant, bias):
    """The values of the codes 0 .. 0x78 of an 8-bit float, ascending, in 64 bits."""
    out = []
    for c in range(0x79):
        e, f = c >> mant, c & ((1 << mant) - 1)
        out.append(f * 2.0 ** (1 - bias - mant) if e == 0 else (1 + f * 2.0 ** -mant) * 2.0 ** (e - bias))
    return np.array(out)


def round8(x, rnd, mant, bias, top, never_zero):
    """(codes of |x|, scales) of one tensor: each value between two neighbours of the grid, the upper one where
    the fraction of the step plus (rnd + 1/2) / 2^16 reaches 1."""
    n = x.size
    a = np.abs(x.astype(np.float64))
    pad = np.zeros(-(-n // BLOCK) * BLOCK)
    pad[:n] = a
    most = pad.reshape(-1, BLOCK).max(1)
    e = np.where(most > 0, np.floor(np.log2(np.where(most > 0, most, 1.0))), -200.0)
    e = np.where(most >= 2.0 ** np.clip(e + 1, -1000, 1000), e + 1, np.where(most < 2.0 ** np.clip(e, -1000, 1000), e - 1, e))
    scale = 2.0 ** np.maximum(e - top, -126.0)
    grid = grid8(mant, bias)
    t = a / np.repeat(scale, BLOCK)[:n]
    lo = np.searchsorted(grid, t, side="right") - 1
    hi = np.minimum(lo + 1, grid.size - 1)
    frac = np.where(hi > lo, (t - grid[lo]) / np.where(hi > lo, grid[hi] - grid[lo], 1.0), 0.0)
    code = np.where(frac + (rnd + 0.5) / 65536.0 >= 1.0, hi, lo)
    if never_zero:
        code = np.where((code == 0) & (a > 0), 1, code)
    return code, scale.astype(np.float32)
