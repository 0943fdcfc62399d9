"""The measured cases of the operators around and after a model's blocks in a training step: dropout
from a counter-based generator, the norms before and after a block with its gate and residual scale, and
the softmax cross entropy over a table's whole vocabulary, each with its gradient.

Sizes are those of the workloads (workloads/configs.py) and of perf/operators.py, smaller, ragged and wider
ones beside them.  prepare() makes what a training program has in hand before the call, and the buffers that
it keeps between calls; run() makes one call and returns everything that it wrote.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
SEED = 4321                # of the dropout masks
GAMMA, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB  # SplitMix64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
PIECE = 1 << 27            # logits that the plain forms hold at a time


def listed():
    def drop(name, T, D, p, residual, dtype):
        return {"name": name, "kind": "drop", "T": T, "D": D, "p": p, "residual": residual, "dtype": dtype}

    # stream, dtype: types of the residual stream and of the block's rows; rows: rows that share a row of the gate (0: all)
    def block(name, kind, T, D, stream, dtype, p, post, rows, alpha):
        return {"name": name, "kind": kind, "T": T, "D": D, "stream": stream, "dtype": dtype, "p": p, "post": post,
                "rows": rows, "alpha": alpha}

    # live: share of the tokens that have a target; each: whether every token has a weight of its own
    def loss(name, kind, T, V, D, dtype, smoothing, live, each):
        return {"name": name, "kind": kind, "T": T, "V": V, "D": D, "dtype": dtype, "smoothing": smoothing, "live": live,
                "each": each}
    return [
        # the smallest workload's batch: launch and latency only
        drop("drop_tiny", 512, 64, 0.1, True, "f32"),
        # a large batch's block output, dropped and added to the residual stream
        drop("drop_large", 65536, 1024, 0.1, True, "bf16"),
        # one new token per sequence of a small serving batch, nothing dropped
        block("block_tokens", "block", 16, 1024, "bf16", "bf16", 0.0, True, 0, 1.0),
        # a language model's batch, the residual stream kept in fp32
        block("block_lm", "block", 16384, 1024, "f32", "bf16", 0.1, True, 0, 1.0),
        # ragged sizes: rows of 300 floats, 33 tokens share a gate, a scaled residual
        block("block_grad_ragged", "block_grad", 9999, 300, "f32", "f32", 0.1, True, 33, 1.5),
        # the backward pass of a large batch
        block("block_grad_large", "block_grad", 65536, 1024, "bf16", "bf16", 0.1, True, 0, 1.0),
        # the smallest workload's table as an output layer
        loss("loss_tiny", "loss", 512, 1000, 64, "f32", 0.0, 1.0, False),
        # one token scored against a large vocabulary
        loss("loss_one_token", "loss", 1, 262144, 1024, "bf16", 0.0, 1.0, False),
        # a language model's batch over its large vocabulary
        loss("loss_lm", "loss", 16384, 262144, 1024, "bf16", 0.0, 1.0, False),
        # a vocabulary and a width that divide by nothing, most of the tokens without a target (masked-word training)
        loss("loss_grad_ragged", "loss_grad", 6001, 30011, 300, "bf16", 0.0, 0.15, True),
        # a translation model's shared vocabulary in fp32, smoothed targets, padded sequences
        loss("loss_grad_shared", "loss_grad", 25000, 32768, 512, "f32", 0.1, 0.9, True),
        # the backward pass of a language model's batch
        loss("loss_grad_lm", "loss_grad", 16384, 262144, 1024, "bf16", 0.0, 1.0, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("drop", "block", "block_grad", "loss", "loss", "loss_grad", "loss_grad"))
    if kind in ("loss", "loss_grad"):
        T, V, D = rng.choice((1, _log(rng, 1, 64), _log(rng, 64, 32768))), _log(rng, 500, 262144), _log(rng, 32, 1024)
        if rng.random() < 0.7:
            D = max(32, D // 32 * 32)
        if rng.random() < 0.5:
            V = max(512, V // 128 * 128)
        dtype = rng.choice(("f32", "bf16", "bf16"))
        T = max(1, min(T, (1 << (42 if dtype == "bf16" else 39)) // (V * D)))
        return {"kind": kind, "T": T, "V": V, "D": D, "dtype": dtype, "smoothing": rng.choice((0.0, 0.0, 0.1)),
                "live": 1.0 if T < 64 else rng.choice((1.0, 0.9, 0.15)), "each": rng.random() < 0.5}
    T, D = _log(rng, 1, 65536), _log(rng, 16, 8192)
    if rng.random() < 0.75:  # most rows are a multiple of 4 or of 64 wide; the rest anything
        m = 64 if D >= 96 and rng.random() < 0.6 else 4
        D = max(m, D // m * m)
    T = min(T, (1 << 26) // D)
    p = rng.choice((0.0, 0.1, round(rng.uniform(0.01, 0.6), 3)))
    dtype = rng.choice(("f32", "bf16"))
    if kind == "drop":
        return {"kind": kind, "T": T, "D": D, "p": p, "residual": rng.random() < 0.5, "dtype": dtype}
    return {"kind": kind, "T": T, "D": D, "stream": "f32" if dtype == "f32" else rng.choice(("f32", "bf16")), "dtype": dtype,
            "p": p, "post": rng.random() < 0.7, "rows": rng.choice((0, 0, 1, _log(rng, 1, 4096))),
            "alpha": rng.choice((1.0, 1.5))}


# ------------------------------------------------------------------ inputs
def _gen(seed, k=0):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + k) & ((1 << 62) - 1))
    return g


def _normal(shape, seed, k, sigma=1.0):
    return torch.randn(shape, generator=_gen(seed, k), device="cuda").mul_(sigma)


def _uniform(n, seed, k):
    return torch.rand(n, generator=_gen(seed, k), device="cuda", dtype=torch.float64)


def _gates(c):
    """Rows of the gate."""
    return -(-c["T"] // c["rows"]) if c["rows"] else 1


def prepare(case, seed):
    c, dev = dict(case), "cuda"
    s = {"c": c}
    T, D, dt = c["T"], c["D"], DTYPES[c["dtype"]]
    if c["kind"] == "drop":
        s["x"] = _normal((T, D), seed, 1).to(dt)
        s["r"] = _normal((T, D), seed, 2, 3.0).to(dt) if c["residual"] else None
        s["y"] = torch.empty((T, D), dtype=dt, device=dev)
        return s
    if c["kind"] in ("block", "block_grad"):
        st = DTYPES[c["stream"]]
        # the residual stream has a few columns that are much larger than the rest
        col = 1.0 + 10.0 * (torch.rand(D, generator=_gen(seed, 1), device=dev) < 0.01)
        s["x"] = (_normal((T, D), seed, 2, 2.0) * col + 0.1).to(st)
        s["b"] = (_normal((T, D), seed, 3) * col).to(dt)
        s["gate"] = _normal((_gates(c), D), seed, 4, 0.3)
        s["post"] = (1.0 + _normal((D,), seed, 5, 0.1), _normal((D,), seed, 6, 0.1)) if c["post"] else None
        s["pre"] = (1.0 + _normal((D,), seed, 7, 0.1), _normal((D,), seed, 8, 0.1))
        s["seed"] = SEED + int(seed)
        new = lambda t: torch.empty((T, D), dtype=t, device=dev)  # noqa: E731
        if c["kind"] == "block":
            stats = [torch.empty((2, T), device=dev) for _ in range(2)]
            s["out"] = (new(st), new(dt), stats[0] if c["post"] else None, stats[1])
            return s
        s["h"], _, s["post_stats"], s["pre_stats"] = _block(s, c)
        s["dh"], s["dy"] = _normal((T, D), seed, 9, 0.01).to(st), _normal((T, D), seed, 10, 0.01).to(dt)
        row = lambda on=True: torch.empty(D, device=dev) if on else None  # noqa: E731
        s["out"] = (new(st), new(dt), torch.empty_like(s["gate"]), row(c["post"]), row(c["post"]), row(), row())
        return s
    V = c["V"]
    s["x"] = _normal((T, D), seed, 1).to(dt)                         # the last norm's output
    s["W"] = _normal((V, D), seed, 2, 2.0 / math.sqrt(D)).to(dt)     # logits of deviation 2
    # targets by a Zipf law of exponent 1 (the id's logarithm is uniform); -1: none
    ids = torch.exp(_uniform(T, seed, 3) * math.log(V)).long().clamp_(max=V) - 1
    s["ids"] = torch.where(_uniform(T, seed, 4) < c["live"], ids, -1).to(torch.int32)
    s["loss"], s["lse"] = torch.empty(T, device=dev), torch.empty(T, device=dev)
    if c["kind"] == "loss_grad":
        s["loss"], s["lse"] = _loss(s, c)
        n = max(1.0, c["live"] * T)
        s["dloss"] = ((0.5 + _uniform(T, seed, 5)) / n).float() if c["each"] else torch.full((1,), 1.0 / n, device=dev)
        s["dx"], s["dW"] = torch.empty((T, D), dtype=dt, device=dev), torch.empty((V, D), dtype=dt, device=dev)
    return s


# ------------------------------------------------------------------ the plain forms
def _mix(z):
    """SplitMix64's output function on int64 (Steele, Lea and Flood 2014)."""
    m1, m2 = MIX1 - (1 << 64), MIX2 - (1 << 64)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * m1
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * m2
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _signed(z):
    z &= (1 << 64) - 1
    return z - (1 << 64) if z >> 63 else z


def _kept(T, D, p, seed):
    """(which elements of T rows of D stay, the factor of those): draw t ceil(D / 4) + d / 4 of the seed's stream holds
    16 bits for each of four elements of row t; an element goes where its bits are below 65536 p."""
    cut = min(round(65536 * p), 65535)
    per = -(-D // 4)
    key = _mix(torch.tensor(_signed(seed), dtype=torch.int64, device="cuda"))
    z = _mix((torch.arange(T * per, device="cuda") + 1) * _signed(GAMMA) + key)
    bits = torch.stack([(z >> k) & 0xFFFF for k in (0, 16, 32, 48)], 1).view(T, 4 * per)[:, :D]
    return bits >= cut, 65536.0 / (65536 - cut)


def _drop(s, c):
    keep, scale = _kept(c["T"], c["D"], c["p"], SEED)
    y = torch.where(keep, s["x"].float() * scale, 0.0)
    return (y if s["r"] is None else s["r"].float() + y).to(s["x"].dtype)


def _norm(x, wb):
    mean = x.sum(1) / x.shape[1]
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / x.shape[1] + EPS)
    return d * rstd[:, None] * wb[0] + wb[1], torch.stack((mean, rstd))


def _rows_of(c, gate):
    """The gate of every row."""
    return gate.repeat_interleave(c["rows"], 0)[:c["T"]] if c["rows"] else gate


def _block(s, c):
    b, post_stats = s["b"].float(), None
    if s["post"] is not None:
        b, post_stats = _norm(b, s["post"])
    if c["p"] > 0:
        keep, scale = _kept(c["T"], c["D"], c["p"], s["seed"])
        b = torch.where(keep, b * scale, 0.0)
    h = c["alpha"] * s["x"].float() + _rows_of(c, s["gate"]) * b
    y, pre_stats = _norm(h, s["pre"])
    return h.to(s["x"].dtype), y.to(s["b"].dtype), post_stats, pre_stats


def _norm_grad(dy, x, w, stats):
    xh = (x - stats[0][:, None]) * stats[1][:, None]
    g = dy * w
    c1, c2 = g.sum(1, keepdim=True) / x.shape[1], (g * xh).sum(1, keepdim=True) / x.shape[1]
    return stats[1][:, None] * (g - c1 - xh * c2), xh, (dy * xh).sum(0), dy.sum(0)


def _block_grad(s, c):
    dx, _, dw1, db1 = _norm_grad(s["dy"].float(), s["h"].float(), s["pre"][0], s["pre_stats"])
    d = s["dh"].float() + dx
    b, dw0, db0 = s["b"].float(), None, None
    n = b
    if s["post"] is not None:
        st = s["post_stats"]
        n = (b - st[0][:, None]) * st[1][:, None] * s["post"][0] + s["post"][1]
    keep, scale = _kept(c["T"], c["D"], c["p"], s["seed"]) if c["p"] > 0 else (torch.ones_like(b, dtype=torch.bool), 1.0)
    dgate = torch.where(keep, d * n * scale, 0.0)
    if c["rows"]:
        G = _gates(c)
        dgate = torch.nn.functional.pad(dgate, (0, 0, 0, G * c["rows"] - c["T"])).view(G, c["rows"], -1).sum(1)
    else:
        dgate = dgate.sum(0, keepdim=True)
    dn = torch.where(keep, d * _rows_of(c, s["gate"]) * scale, 0.0)
    if s["post"] is not None:
        dn, _, dw0, db0 = _norm_grad(dn, b, s["post"][0], s["post_stats"])
    return (c["alpha"] * d).to(s["x"].dtype), dn.to(s["b"].dtype), dgate, dw0, db0, dw1, db1


def _pieces(c):
    n = max(256, min(c["V"], PIECE // c["T"]))
    return [(a, min(a + n, c["V"])) for a in range(0, c["V"], n)]


def _loss(s, c):
    x, W, ids = s["x"].float(), s["W"], s["ids"].long()
    T, V = c["T"], c["V"]
    top, total = torch.full((T,), -math.inf, device="cuda"), torch.zeros(T, device="cuda")
    at, every = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    for a, b in _pieces(c):
        z = x @ W[a:b].float().t()
        m = torch.maximum(top, z.amax(1))
        total = total * torch.exp(top - m) + torch.exp(z - m[:, None]).sum(1)
        top = m
        here = (ids >= a) & (ids < b)
        at = torch.where(here, z.gather(1, (ids - a).clamp(0, b - a - 1)[:, None])[:, 0], at)
        every += z.sum(1)
    lse = top + torch.log(total)
    e = c["smoothing"]
    loss = lse - (1.0 - e) * at - e * every / V
    live = ids >= 0
    return torch.where(live, loss, 0.0), torch.where(live, lse, 0.0)


def _loss_grad(s, c):
    x, W, ids = s["x"].float(), s["W"], s["ids"].long()
    live, e = ids >= 0, c["smoothing"]
    d = torch.where(live, s["dloss"].expand(c["T"]), 0.0)[:, None]
    dx = torch.zeros_like(x)
    dW = torch.empty(W.shape, device="cuda", dtype=W.dtype)
    for a, b in _pieces(c):
        w = W[a:b].float()
        g = torch.exp(x @ w.t() - s["lse"][:, None]) - e / c["V"]
        here = (ids >= a) & (ids < b)
        t = torch.nonzero(here)[:, 0]
        g[t, ids[t] - a] -= 1.0 - e
        g = torch.where(live[:, None], g * d, 0.0)
        dx += g @ w
        dW[a:b] = (g.t() @ x).to(W.dtype)
    return dx.to(s["x"].dtype), dW


# ------------------------------------------------------------------ one pass
def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        return _run_own(s, c, kind)
    if kind == "drop":
        return {"y": _drop(s, c)}
    if kind == "block":
        return _named(("h", "y", "post_stats", "pre_stats"), _block(s, c))
    if kind == "block_grad":
        return _named(_BLOCK_GRADS, _block_grad(s, c))
    if kind == "loss":
        return _named(("loss", "lse"), _loss(s, c))
    return _named(("dx", "dW"), _loss_grad(s, c))


_BLOCK_GRADS = ("dx", "dbranch", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")


def _named(names, values):
    return {n: v for n, v in zip(names, values) if v is not None}


def _run_own(s, c, kind):
    import paper_2110_09132_amd as emb
    if kind == "drop":
        return {"y": emb.dropout(s["x"], c["p"], SEED, residual=s["r"], out=s["y"])}
    if kind == "block":
        return _named(("h", "y", "post_stats", "pre_stats"),
                      emb.block_norm(s["x"], s["b"], gate=s["gate"], gate_rows=c["rows"], alpha=c["alpha"], post=s["post"],
                                     pre=s["pre"], eps=EPS, p=c["p"], seed=s["seed"], out=s["out"]))
    if kind == "block_grad":
        if "ws" not in s:  # a workspace, kept as a training program keeps it
            s["ws"] = emb.new_workspace(emb.block_norm_backward_workspace_bytes(c["T"], c["D"], c["rows"]))
        return _named(_BLOCK_GRADS,
                      emb.block_norm_backward(s["dh"], s["dy"], s["h"], s["b"], s["post_stats"], s["pre_stats"],
                                              gate=s["gate"], gate_rows=c["rows"], alpha=c["alpha"], post=s["post"],
                                              pre=s["pre"], p=c["p"], seed=s["seed"], out=s["out"], workspace=s["ws"]))
    if kind == "loss":
        if "ws" not in s:
            s["ws"] = emb.new_workspace(emb.vocab_loss_workspace_bytes(c["T"], c["V"], c["D"], s["x"].dtype))
        return _named(("loss", "lse"), emb.vocab_loss(s["x"], s["W"], s["ids"], smoothing=c["smoothing"],
                                                      out=(s["loss"], s["lse"]), workspace=s["ws"]))
    if "ws" not in s:
        s["ws"] = emb.new_workspace(emb.vocab_loss_backward_workspace_bytes(c["T"], c["V"], c["D"], s["x"].dtype))
    return _named(("dx", "dW"), emb.vocab_loss_backward(s["dloss"], s["x"], s["W"], s["ids"], s["lse"],
                                                        smoothing=c["smoothing"], out=(s["dx"], s["dW"]),
                                                        workspace=s["ws"]))


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    size = {"f32": 4, "bf16": 2}
    T, D, n = c["T"], c["D"], size[c["dtype"]]
    if c["kind"] == "drop":
        return {"bytes": T * D * n * (3 if c["residual"] else 2), "flops": 3.0 * T * D}
    if c["kind"] in ("block", "block_grad"):
        m, gate = size[c["stream"]], 4 * _gates(c) * D
        stats, params = 8 * T * (2 if c["post"] else 1), 4 * D * (4 if c["post"] else 2)
        if c["kind"] == "block":
            return {"bytes": T * D * 2 * (n + m) + gate + stats + params, "flops": 20.0 * T * D}
        # read: dh, dy, h, branch; written: dx, dbranch
        return {"bytes": T * D * 3 * (n + m) + 2 * gate + stats + 2 * params, "flops": 45.0 * T * D}
    V, live = c["V"], max(1.0, c["live"] * T)
    if c["kind"] == "loss":
        return {"bytes": (live + V) * D * n + 12 * T, "flops": 2.0 * live * V * D}
    # the logits again, and a product for each of the two gradients
    return {"bytes": (live + T + 2 * V) * D * n + 8 * T + 4 * (T if c["each"] else 1), "flops": 6.0 * live * V * D}


# ------------------------------------------------------------------ the definitions in 64 bits
def _mask(c, seed):
    """1 / (1 - p) for the elements that stay, 0 for the others, in 64 bits; the generator's numbers are 32-bit halves here."""
    D, per = c["D"], -(-c["D"] // 4)
    lo, hi = 0xFFFFFFFF, 32

    def times(ah, al, b):  # (ah, al) * b modulo 2 ** 64, as 32-bit halves in int64; partial products below 2 ** 63
        bh, bl = b >> 32, b & lo
        al0, al1 = al & 0xFFFF, al >> 16
        p0, p1 = al0 * bl, al1 * bl                       # below 2 ** 48
        mid = (p0 >> 16) + p1
        low = ((mid & 0xFFFF) << 16) | (p0 & 0xFFFF)
        wide = lambda u, v: (u & 0xFFFF) * v + (((u >> 16) * (v & 0xFFFF) & 0xFFFF) << 16)  # noqa: E731  (mod 2 ** 32)
        return ((mid >> 16) + wide(ah, bl) + wide(al, bh)) & lo, low

    def shifted(h, l, k):  # (h, l) ^ (h, l) >> k, k < 32
        return h ^ (h >> k), l ^ (((h << (hi - k)) & lo) | (l >> k))

    def mix(h, l):
        h, l = times(*shifted(h, l, 30), MIX1)
        h, l = times(*shifted(h, l, 27), MIX2)
        return shifted(h, l, 31)
    kh, kl = mix(*(torch.tensor(v, device="cuda") for v in ((seed >> 32) & lo, seed & lo)))
    n = torch.arange(1, c["T"] * per + 1, device="cuda")
    h, l = times(n >> 32, n & lo, GAMMA)
    l = l + kl
    h, l = mix((h + kh + (l >> 32)) & lo, l & lo)
    bits = torch.stack((l & 0xFFFF, l >> 16, h & 0xFFFF, h >> 16), 1).reshape(c["T"], -1)[:, :D]
    cut = min(round(65536 * c["p"]), 65535)
    return torch.where(bits < cut, 0.0, 1.0 / (1.0 - cut / 65536.0)).double()


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "drop":
        y = s["x"].double() * _mask(c, SEED)
        return {"y": y if s["r"] is None else y.add_(s["r"])}
    if c["kind"] in ("block", "block_grad"):
        T, D = c["T"], c["D"]
        gate = s["gate"].double()[torch.arange(T, device="cuda") // (c["rows"] or T)]
        mask = _mask(c, s["seed"]) if c["p"] > 0 else 1.0

        def norm(x, wb):
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = (var + EPS).rsqrt()
            return torch.addcmul(wb[1].double(), (x - mean[:, None]) * rstd[:, None], wb[0].double()), \
                torch.stack((mean, rstd))
        if c["kind"] == "block":
            n, post_stats = norm(s["b"].double(), s["post"]) if c["post"] else (s["b"].double(), None)
            h = s["x"].double() * c["alpha"] + gate * mask * n
            y, pre_stats = norm(h, s["pre"])
            return _named(("h", "y", "post_stats", "pre_stats"), (h, y, post_stats, pre_stats))

        def back(d, x, w, stats):  # the gradient of a norm whose statistics are given
            mean, rstd = stats.double().unsqueeze(2)
            xh = (x.double() - mean) * rstd
            g = d * w.double()
            return rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)), (d * xh).sum(0), xh
        dy = s["dy"].double()
        dx, dw1, _ = back(dy, s["h"], s["pre"][0], s["pre_stats"])
        d = dx + s["dh"].double()
        dn, n, dw0, db0 = d * gate * mask, s["b"].double(), None, None
        if c["post"]:
            db0 = dn.sum(0)
            dn, dw0, n = back(dn, s["b"], s["post"][0], s["post_stats"])
            n = torch.addcmul(s["post"][1].double(), n, s["post"][0].double())
        dgate = torch.zeros(s["gate"].shape, device="cuda", dtype=torch.float64)
        dgate.index_add_(0, torch.arange(T, device="cuda") // (c["rows"] or T), d * mask * n)
        return _named(_BLOCK_GRADS, (d * c["alpha"], dn, dgate, dw0, db0, dw1, dy.sum(0)))
    T, V, e = c["T"], c["V"], c["smoothing"]
    live = torch.nonzero(s["ids"] >= 0)[:, 0]
    x, ids = s["x"].double()[live], s["ids"].long()[live]
    step = max(256, (1 << 27) // max(1, len(live)))
    if c["kind"] == "loss":
        parts, mean = [], torch.zeros(len(live), device="cuda", dtype=torch.float64)
        for w in s["W"].split(step):
            z = torch.mm(x, w.double().t())
            parts.append(torch.logsumexp(z, 1))
            mean += z.sum(1) / V
        lse = torch.logsumexp(torch.stack(parts), 0)
        loss = lse - (1 - e) * (x * s["W"][ids].double()).sum(1) - e * mean
        whole = torch.zeros((2, T), device="cuda", dtype=torch.float64)
        whole[0, live], whole[1, live] = loss, lse
        return {"loss": whole[0], "lse": whole[1]}
    lse, d = s["lse"].double()[live], s["dloss"].double().expand(T)[live]
    dx, dW = torch.zeros_like(x), []
    for k, w in enumerate(s["W"].split(step)):
        w = w.double()
        g = torch.mm(x, w.t()).sub_(lse[:, None]).exp_().sub_(e / V)
        t = torch.nonzero((ids >= k * step) & (ids < k * step + w.shape[0]))[:, 0]
        g[t, ids[t] - k * step] += e - 1
        g.mul_(d[:, None])
        dx.addmm_(g, w)
        dW.append(torch.mm(g.t(), x))
    whole = torch.zeros((T, c["D"]), device="cuda", dtype=torch.float64)
    whole[live] = dx
    return {"dx": whole, "dW": torch.cat(dW)}
