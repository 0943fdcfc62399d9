"""The measured cases of the dense operators that stand around the embedding tables in a training step:
layer norm (on rows looked up by id, or on rows at hand) and its gradient, the relative position bias by
buckets and its gradient, and AdamW over many tensors with states of 32 or 8 bits.

Sizes are those of the workloads (workloads/configs.py) and the benchmark, smaller, ragged and wider ones
beside them.  prepare() makes what a training program has in hand before the call, and the buffers that
it keeps between calls; run() makes one call and returns everything that it wrote.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LN_EPS = 1e-5
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
STEP, SEED = 20, 1234      # AdamW's step number and the seed of its rounding to 8 bits
QBLOCK = 256               # elements that share a scale in 8-bit states
GAMMA, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB  # SplitMix64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BUCKETS, FAR = 32, 128     # buckets of the position bias; differences of FAR and more share the last one


def listed():
    def norm(name, kind, T, D, V=0, law=0.0, x="f32", y="f32"):
        return {"name": name, "kind": kind, "T": T, "D": D, "V": V, "law": law, "x": x, "y": y}

    def bias(name, kind, N, H, Q, K, causal, dtype):
        return {"name": name, "kind": kind, "N": N, "H": H, "Q": Q, "K": K, "causal": causal, "dtype": dtype}

    def adamw(name, bits, D, layers, H, grad, copy, clip, align):
        return {"name": name, "kind": "adamw", "bits": bits, "D": D, "layers": layers, "H": H, "grad": grad,
                "copy": copy, "clip": clip, "align": align}
    # V: rows of the table that the ids look up (0: the rows are at hand); law: exponent of the ids' Zipf law
    return [
        # the smallest workload's batch, looked up and normalised: launch and latency only
        norm("norm_lookup_tiny", "norm", 512, 64, 1000, 1.1),
        # a language model's batch: looked up in the large fp32 table, handed on in bf16
        norm("norm_lookup_lm", "norm", 16384, 1024, 262144, 1.0, "f32", "bf16"),
        # activations of a wide layer inside a model
        norm("norm_wide_bf16", "norm", 8192, 8192, 0, 0.0, "bf16", "bf16"),
        # ragged sizes: rows of 300 floats and a token count that divides by nothing; dx goes to the coalesce
        norm("norm_grad_ragged", "norm_grad", 9999, 300, 30011, 1.0),
        # the backward pass of a large batch
        norm("norm_grad_large", "norm_grad", 65536, 1024, 0, 0.0, "bf16", "bf16"),
        # one new token after 4095 others: one row of the bias per head
        bias("bias_one_token", "bias", 1, 16, 1, 4096, False, "bf16"),
        # a whole sequence of a shared-vocabulary translation model
        bias("bias_large", "bias", 1, 16, 2048, 2048, False, "f32"),
        # a short odd sequence, masked above the diagonal, three in the batch
        bias("bias_grad_ragged", "bias_grad", 3, 6, 257, 257, True, "f32"),
        # the gradient of a bias that a batch of sequences shares
        bias("bias_grad_large", "bias_grad", 8, 16, 1024, 1024, False, "bf16"),
        # the dense parameters of a small model: many tensors, little in them
        adamw("adamw_tiny", 32, 64, 2, 4, "f32", False, True, 256),
        # the dense parameters beside the 1024-wide tables, bf16 gradients and a bf16 copy of the weights
        adamw("adamw_large", 32, 1024, 6, 16, "bf16", True, True, 256),
        # the same with states in 8 bits
        adamw("adamw8_large", 8, 1024, 6, 16, "bf16", True, True, 256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm_grad", "bias", "bias_grad", "adamw", "adamw8"))
    if kind in ("norm", "norm_grad"):
        T, D = _log(rng, 1, 65536), _log(rng, 16, 8192)
        if rng.random() < 0.75:  # most rows are a multiple of 4 or of 64 wide; the rest anything
            m = 64 if D >= 96 and rng.random() < 0.6 else 4
            D = max(m, D // m * m)
        T = min(T, (1 << 26) // D)
        V = min(_log(rng, 1000, 1 << 20), (1 << 28) // D) if rng.random() < 0.4 else 0
        return {"kind": kind, "T": T, "D": D, "V": V, "law": round(rng.choice((0.0, rng.uniform(0.8, 1.3))), 3),
                "x": "f32" if V else rng.choice(("f32", "bf16")), "y": rng.choice(("f32", "bf16"))}
    if kind in ("bias", "bias_grad"):
        H, K = rng.choice((1, 2, 3, 4, 6, 8, 12, 16, 20, 32)), _log(rng, 16, 4096)
        if rng.random() < 0.5:
            K = max(16, K // 16 * 16)
        Q = rng.choice((1, K, K, _log(rng, 1, K)))
        N = _log(rng, 1, 8) if kind == "bias_grad" else 1
        while N * H * Q * K > 1 << 27:
            N, H, Q = (N, H, (Q + 1) // 2) if N == 1 and H == 1 else ((N + 1) // 2, (H + 1) // 2, Q)
        return {"kind": kind, "N": N, "H": H, "Q": Q, "K": K, "causal": rng.random() < 0.5,
                "dtype": rng.choice(("f32", "bf16"))}
    D, layers = _log(rng, 16, 1024), rng.randint(1, 6)
    if rng.random() < 0.6:
        D = D // 16 * 16
    return {"kind": "adamw", "bits": 8 if kind == "adamw8" else 32, "D": D, "layers": layers,
            "H": rng.choice((1, 3, 4, 8, 12, 16)), "grad": rng.choice(("f32", "bf16")), "copy": rng.random() < 0.5,
            "clip": rng.random() < 0.5, "align": rng.choice((256, 256, 1))}


# ------------------------------------------------------------------ inputs
def _gen(seed, k=0):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + k) & ((1 << 62) - 1))
    return g


def _normal(shape, seed, k, sigma=1.0):
    return torch.randn(shape, generator=_gen(seed, k), device="cuda").mul_(sigma)


def _ids(c, seed, k):
    T, V = c["T"], c["V"]
    u = torch.rand(T, generator=_gen(seed, k), device="cuda", dtype=torch.float64)
    if c["law"] == 0.0:
        ids = (u * V).long()
    else:  # bounded Zipf: P(id) proportional to (id + 1) ** -law
        cdf = torch.arange(1, V + 1, device="cuda", dtype=torch.float64).pow_(-c["law"]).cumsum_(0)
        ids = torch.searchsorted(cdf, u * cdf[-1], right=True)
    return ids.clamp_(max=V - 1).to(torch.int32)


def _bucket_map(causal):
    """Bucket of every position difference key - query in [-FAR, FAR]: half of a direction's buckets hold one
    distance each, the others widen by a constant factor up to FAR; causal: -1 (masked) for keys after the query."""
    per = BUCKETS if causal else BUCKETS // 2
    one = per // 2

    def of(n):  # distance n >= 0
        if n < one:
            return n
        return min(per - 1, one + int(math.log(n / one) / math.log(FAR / one) * (per - one) + 1e-9))
    got = [(-1 if causal and r > 0 else of(abs(r)) + (0 if causal or r <= 0 else per)) for r in range(-FAR, FAR + 1)]
    return torch.tensor(got, dtype=torch.int32, device="cuda")


def _shapes(c):
    """Parameters of `layers` transformer blocks of width D and one position bias table."""
    D, F = c["D"], 4 * c["D"]
    block = [(D, D)] * 4 + [(F, D), (F,), (D, F), (D,)] + [(D,)] * 4
    return block * c["layers"] + [(BUCKETS, c["H"])]


def _flat_layout(c):
    """Start of every parameter in the flat buffers, and their length; `align`: elements that a start is a multiple of."""
    sizes = [math.prod(s) for s in _shapes(c)]
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // c["align"]) * c["align"]
    return sizes, starts, at


def _views(flat, sizes, starts):
    return [flat[a:a + n] for a, n in zip(starts, sizes)]


def _q0(c):
    """Position of the first query: the queries are the last Q of the K positions."""
    return max(c["K"] - c["Q"], 0)


def prepare(case, seed):
    c, dev = dict(case), "cuda"
    s = {"c": c}
    if c["kind"] in ("norm", "norm_grad"):
        T, D, xt, yt = c["T"], c["D"], DTYPES[c["x"]], DTYPES[c["y"]]
        # activations have a few columns that are much larger than the rest
        col = 1.0 + 10.0 * (torch.rand(D, generator=_gen(seed, 1), device=dev) < 0.01)
        s["x"] = (_normal((c["V"] or T, D), seed, 2) * col + 0.1).to(xt)
        s["ids"] = _ids(c, seed, 3) if c["V"] else None
        s["w"] = 1.0 + _normal((D,), seed, 4, 0.1)
        s["b"] = _normal((D,), seed, 5, 0.1)
        s["mean"], s["rstd"] = (torch.empty(T, device=dev) for _ in range(2))
        if c["kind"] == "norm":
            s["y"] = torch.empty((T, D), dtype=yt, device=dev)
        else:
            s["dy"] = _normal((T, D), seed, 6, 0.01).to(yt)
            _, s["mean"], s["rstd"] = _norm(s["x"], s["ids"], s["w"], s["b"], yt)
            s["dx"] = torch.empty((T, D), dtype=yt, device=dev)
            s["dw"], s["db"] = (torch.empty(D, device=dev) for _ in range(2))
        return s
    if c["kind"] in ("bias", "bias_grad"):
        s["map"] = _bucket_map(c["causal"])
        dt = DTYPES[c["dtype"]]
        if c["kind"] == "bias":
            s["table"] = _normal((BUCKETS, c["H"]), seed, 1)
            s["out"] = torch.empty((c["H"], c["Q"], c["K"]), dtype=dt, device=dev)
        else:  # the gradient of attention scores: zero where the mask took the key out
            N, H, Q, K = c["N"], c["H"], c["Q"], c["K"]
            d = _normal((N, H, Q, K), seed, 1, 0.01)
            if c["causal"]:
                d.mul_(_rel(c) <= 0)
            s["d"] = d.to(dt)
            s["dtable"] = torch.empty((BUCKETS, H), device=dev)
        return s
    sizes, starts, n = _flat_layout(c)
    live = torch.zeros(n, device=dev)  # the elements that belong to a parameter
    for v in _views(live, sizes, starts):
        v.fill_(1.0)
    s["sizes"], s["starts"] = sizes, starts
    s["p"] = _normal((n,), seed, 1, 0.02) * live
    s["g"] = (_normal((n,), seed, 2, 0.003) * live).to(DTYPES[c["grad"]])
    s["copy"] = (s["p"].to(torch.bfloat16) if c["copy"] else None)
    s["clip"] = torch.rand(1, generator=_gen(seed, 3), device=dev) if c["clip"] else None
    s["m"] = _normal((n,), seed, 4, 0.001) * live
    s["v"] = (_normal((n,), seed, 5, 0.003) * live).square_()
    s["scales"] = None
    if c["bits"] == 8:  # states as earlier steps leave them: values of 8 bits, a power of two for every QBLOCK of them
        s["m"] = (s["m"] * 2.0 ** 15).to(torch.float8_e4m3fn)
        s["v"] = (s["v"] * 2.0 ** 28).to(torch.float8_e5m2)
        blocks = [-(-k // QBLOCK) for k in sizes]
        s["sstarts"] = [2 * (sum(blocks[:i])) for i in range(len(blocks))]
        s["blocks"] = blocks
        s["scales"] = torch.empty(2 * sum(blocks), device=dev)
        for a, b in zip(s["sstarts"], blocks):
            s["scales"][a:a + b], s["scales"][a + b:a + 2 * b] = 2.0 ** -15, 2.0 ** -28
    return s


# ------------------------------------------------------------------ the plain forms
def _norm(x, ids, w, b, dtype):
    x = (x if ids is None else x[ids.long()]).float()
    mean = x.sum(1) / x.shape[1]
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / x.shape[1] + LN_EPS)
    return (d * rstd[:, None] * w + b).to(dtype), mean, rstd


def _norm_grad(dy, x, ids, w, mean, rstd):
    x = (x if ids is None else x[ids.long()]).float()
    xh = (x - mean[:, None]) * rstd[:, None]
    dyf = dy.float()
    g = dyf * w
    c1, c2 = g.sum(1, keepdim=True) / x.shape[1], (g * xh).sum(1, keepdim=True) / x.shape[1]
    return (rstd[:, None] * (g - c1 - xh * c2)).to(dy.dtype), (dyf * xh).sum(0), dyf.sum(0)


def _rel(c):
    """Position difference key - query of every (query, key), [Q, K]."""
    return torch.arange(c["K"], device="cuda")[None, :] - (torch.arange(c["Q"], device="cuda")[:, None] + _q0(c))


def _bucket_of(c, bmap, rel):
    return bmap[rel.clamp(-FAR, FAR) + FAR].long()


def _bias(c, table, bmap):
    b = _bucket_of(c, bmap, _rel(c))
    rows = torch.where((b < 0)[..., None], -math.inf, table[b.clamp(min=0)])
    return rows.permute(2, 0, 1).contiguous().to(DTYPES[c["dtype"]])


def _bias_grad(c, d, bmap):
    """Sum over the batch, then along every diagonal of the (query, key) plane, then over a bucket's diagonals."""
    H, Q, K = c["H"], c["Q"], c["K"]
    d = d.float().sum(0).flip(1)  # query Q - 1 first: (i, j) of the flipped plane is on the diagonal i + j
    d = torch.nn.functional.pad(d, (0, Q)).reshape(H, -1)[:, :Q * (K + Q) - Q].reshape(H, Q, K + Q - 1)
    diag = d.sum(1)               # [H, K + Q - 1], difference key - query = column - (Q - 1) - q0
    b = _bucket_of(c, bmap, torch.arange(K + Q - 1, device="cuda") - (Q - 1) - _q0(c))
    diag = torch.where(b < 0, 0.0, diag)
    here = b == torch.arange(BUCKETS, device="cuda")[:, None]
    return torch.where(here[:, None, :], diag, 0.0).sum(2)


def _mix(z):
    """SplitMix64's output function on int64 (Steele, Lea and Flood 2014)."""
    m1, m2 = MIX1 - (1 << 64), MIX2 - (1 << 64)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * m1
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * m2
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _mix_int(z):
    z &= (1 << 64) - 1
    z = ((z ^ (z >> 30)) * MIX1) & ((1 << 64) - 1)
    z = ((z ^ (z >> 27)) * MIX2) & ((1 << 64) - 1)
    return z ^ (z >> 31)


def _signed(z):
    z &= (1 << 64) - 1
    return z - (1 << 64) if z >> 63 else z


def _random16(k, n):
    """Two 16-bit numbers for each of the n elements of tensor k: elements 2i and 2i + 1 share draw i of the
    tensor's stream, the even one its lower half."""
    key = _mix_int(_mix_int(SEED + STEP * GAMMA) + (k + 1) * GAMMA)
    i = torch.arange((n + 1) // 2, device="cuda", dtype=torch.int64)
    z = _mix((i + 1) * _signed(GAMMA) + _signed(key))
    h = torch.stack((z & 0xFFFFFFFF, (z >> 32) & 0xFFFFFFFF), 1).reshape(-1)[:n]
    return h & 0xFFFF, h >> 16


def _to8(x, rnd, mant, bias, top, never_zero):
    """|x| / scale in an 8-bit float of `mant` mantissa bits, rounded up with the probability of the part cut off;
    the scale of a block is the power of two that puts its largest magnitude in [2 ** top, 2 ** (top + 1))."""
    n = x.numel()
    a = torch.nn.functional.pad(x.abs(), (0, -n % QBLOCK)).view(-1, QBLOCK)
    e = a.view(torch.int32).amax(1) >> 23
    field = (e - top).clamp(min=1)
    scale = torch.where(e == 255, math.nan, (field << 23).view(torch.float32))
    inv = ((254 - field) << 23).view(torch.float32)
    t = (a * inv[:, None]).reshape(-1)[:n]
    low = 2.0 ** (1 - bias)   # below the smallest normal value the codes are evenly spaced
    cut = 23 - mant
    r = (rnd << (cut - 16)) + (1 << (cut - 17))
    t2 = torch.where(t < low, t + low, t)
    code = ((t2.view(torch.int32).long() + r) >> cut) - torch.where(t < low, (128 - bias) << mant, (127 - bias) << mant)
    if never_zero:
        code = torch.where((code == 0) & (t > 0), 1, code)
    finite = (e != 255).repeat_interleave(QBLOCK)[:n]
    return torch.where(finite, code, 0), scale


def _adamw_one(c, k, p, g, m, v, scales, copy, clip):
    n = p.numel()
    if scales is not None:
        nb = scales.numel() // 2
        per = scales.view(2, nb).repeat_interleave(QBLOCK, 1)[:, :n]
        m8, v8, m, v = m, v, m.float() * per[0], v.float() * per[1]
    gf = g.float() if clip is None else g.float() * clip
    m1 = m * BETA1 + gf * (1.0 - BETA1)
    v1 = v * BETA2 + gf * gf * (1.0 - BETA2)
    w = p - p * (LR * DECAY)
    w = w - (m1 / (torch.sqrt(v1 * (1.0 / (1.0 - BETA2 ** STEP))) + EPS)) * (LR / (1.0 - BETA1 ** STEP))
    p.copy_(w)
    if copy is not None:
        copy.copy_(w.to(torch.bfloat16))
    if scales is None:
        m.copy_(m1)
        v.copy_(v1)
        return
    rm, rv = _random16(k, n)
    cm, sm = _to8(m1, rm, 3, 7, 7, False)
    cv, sv = _to8(v1, rv, 2, 15, 14, True)
    m8.view(torch.uint8).copy_(cm + torch.where(torch.signbit(m1), 128, 0))
    v8.view(torch.uint8).copy_(cv)
    scales.copy_(torch.cat((sm, sv)))


def _adamw_lists(s):
    cut = lambda t: [None] * len(s["sizes"]) if t is None else _views(t, s["sizes"], s["starts"])  # noqa: E731
    scales = ([None] * len(s["sizes"]) if s["scales"] is None
              else [s["scales"][a:a + 2 * b] for a, b in zip(s["sstarts"], s["blocks"])])
    return [cut(s[k]) for k in ("p", "g", "m", "v")] + [scales, cut(s["copy"])]


# ------------------------------------------------------------------ one pass
def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        return _run_own(s, c, kind)
    if kind == "norm":
        y, mean, rstd = _norm(s["x"], s["ids"], s["w"], s["b"], DTYPES[c["y"]])
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        dx, dw, db = _norm_grad(s["dy"], s["x"], s["ids"], s["w"], s["mean"], s["rstd"])
        return {"dx": dx, "dw": dw, "db": db}
    if kind == "bias":
        return {"bias": _bias(c, s["table"], s["map"])}
    if kind == "bias_grad":
        return {"dtable": _bias_grad(c, s["d"], s["map"])}
    [_adamw_one(c, k, *t, s["clip"]) for k, t in enumerate(zip(*_adamw_lists(s)))]
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {k: s[k] for k in ("p", "m", "v", "scales", "copy") if s[k] is not None}


def _run_own(s, c, kind):
    import paper_2110_09132_amd as emb
    if kind == "norm":
        y, mean, rstd = emb.layer_norm(s["x"], s["w"], s["b"], LN_EPS, ids=s["ids"], out=(s["y"], s["mean"], s["rstd"]))
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        if "ws" not in s:  # a workspace, kept as a training program keeps it
            s["ws"] = emb.new_workspace(emb.layer_norm_backward_workspace_bytes(c["T"], c["D"]))
        dx, dw, db = emb.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["w"], ids=s["ids"],
                                             out=(s["dx"], s["dw"], s["db"]), workspace=s["ws"])
        return {"dx": dx, "dw": dw, "db": db}
    if kind == "bias":
        return {"bias": emb.relative_bias(s["table"], s["map"], c["Q"], c["K"], _q0(c), out=s["out"])}
    if kind == "bias_grad":
        if "ws" not in s:
            s["ws"] = emb.new_workspace(emb.relative_bias_backward_workspace_bytes(c["N"], c["H"], c["Q"], c["K"]))
        return {"dtable": emb.relative_bias_backward(s["d"], s["map"], BUCKETS, _q0(c), out=s["dtable"],
                                                     workspace=s["ws"])}
    if "lists" not in s:  # the program's parameters, gradients and states are lists of tensors
        s["lists"] = _adamw_lists(s)
    p, g, m, v, scales, copy = s["lists"]
    emb.adamw_step(p, g, m, v, LR, BETA1, BETA2, EPS, DECAY, STEP, scales=scales if c["bits"] == 8 else None,
                   copies=copy if c["copy"] else None, grad_scale=s["clip"], seed=SEED)
    return _adamw_outputs(s)


# ------------------------------------------------------------------ what a pass cannot do without
def _distinct(c):
    """Expected number of distinct ids of a batch."""
    if c["law"] == 0.0:
        return c["V"] * -math.expm1(c["T"] * math.log1p(-1.0 / c["V"]))
    p = np.arange(1, c["V"] + 1, dtype=np.float64) ** -c["law"]
    p /= p.sum()
    return float(-np.expm1(c["T"] * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())


def work(case):
    c = case
    size = {"f32": 4, "bf16": 2}
    if c["kind"] in ("norm", "norm_grad"):
        T, D = c["T"], c["D"]
        x = (_distinct(c) if c["V"] else T) * D * size[c["x"]] + (4 * T if c["V"] else 0)
        if c["kind"] == "norm":
            return {"bytes": x + T * D * size[c["y"]] + 8 * T + 8 * D, "flops": 8.0 * T * D}
        return {"bytes": x + 2 * T * D * size[c["y"]] + 8 * T + 12 * D, "flops": 14.0 * T * D}
    if c["kind"] in ("bias", "bias_grad"):
        n = c["N"] * c["H"] * c["Q"] * c["K"]
        if c["kind"] == "bias_grad" and c["causal"]:  # keys after the query need not be read
            n = c["N"] * c["H"] * sum(min(c["K"], i + _q0(c) + 1) for i in range(c["Q"]))
        return {"bytes": n * size[c["dtype"]] + 4 * BUCKETS * c["H"], "flops": float(n)}
    n = sum(_flat_layout(c)[0])
    state = 16 if c["bits"] == 32 else 4 + 16 / QBLOCK
    return {"bytes": n * (8 + size[c["grad"]] + state + (2 if c["copy"] else 0)), "flops": 15.0 * n}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] in ("norm", "norm_grad"):
        x = s["x"].double() if s["ids"] is None else s["x"].index_select(0, s["ids"].long()).double()
        if c["kind"] == "norm":
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = (var + LN_EPS).rsqrt()
            y = torch.addcmul(s["b"].double(), (x - mean.unsqueeze(1)) * rstd.unsqueeze(1), s["w"].double())
            return {"y": y, "mean": mean, "rstd": rstd}
        mean, rstd = s["mean"].double().unsqueeze(1), s["rstd"].double().unsqueeze(1)
        xh, dy = (x - mean) * rstd, s["dy"].double()
        g = dy * s["w"].double()
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return {"dx": dx, "dw": (dy * xh).sum(0), "db": dy.sum(0)}
    if c["kind"] in ("bias", "bias_grad"):
        rel = torch.arange(c["K"], device="cuda") - torch.arange(_q0(c), _q0(c) + c["Q"], device="cuda").unsqueeze(1)
        b = s["map"][(rel + FAR).clamp(0, 2 * FAR)]
        if c["kind"] == "bias":
            t = torch.cat((s["table"].double(), torch.full((1, c["H"]), -math.inf, device="cuda", dtype=torch.float64)))
            return {"bias": t.t()[:, torch.where(b < 0, BUCKETS, b).long()]}
        d = s["d"].to(torch.float64).sum(0)
        rows = [torch.where(b == k, d, 0.0).sum((1, 2)) for k in range(BUCKETS)]
        return {"dtable": torch.stack(rows)}
    out = {k: torch.zeros(s[k].numel(), device="cuda", dtype=torch.float64) if k in ("p", "m", "v", "copy") else None
           for k in ("p", "m", "v", "scales", "copy") if s[k] is not None}
    clip = 1.0 if s["clip"] is None else float(s["clip"].double())
    for k, (a, n) in enumerate(zip(s["starts"], s["sizes"])):
        cut = slice(a, a + n)
        w, g, m, v = (s[q][cut].to(torch.float64) for q in ("p", "g", "m", "v"))
        if c["bits"] == 8:
            sc = s["scales"][s["sstarts"][k]:s["sstarts"][k] + 2 * s["blocks"][k]].double()
            at = torch.arange(n, device="cuda") // QBLOCK
            m, v = m * sc[at], v * sc[at + s["blocks"][k]]
        g = g * clip
        m = torch.lerp(g, m, BETA1)
        v = torch.lerp(g * g, v, BETA2)
        mh, vh = m / (1 - BETA1 ** STEP), v / (1 - BETA2 ** STEP)
        w = w * (1 - LR * DECAY) - LR * mh / (vh.sqrt() + EPS)
        out["p"][cut] = w
        if "copy" in out:
            out["copy"][cut] = w
        if c["bits"] == 32:
            out["m"][cut], out["v"][cut] = m, v
    if c["bits"] == 8:  # rounded by random numbers: no value of its own in 64 bits
        out["m"] = out["v"] = None
    return out
