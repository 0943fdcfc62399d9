"""emb_block_norm and emb_block_norm_backward against the 64-bit forms of train_ref.py, within the bounds derived there:
row widths on both sides of every change of plan, ragged widths, the three pairs of types, every norm, gate and output
left out in turn, gates shared by groups of rows, masks, strides, in-place calls, rows with infinities and NaN beside
others, empty batches, other streams, replayed graphs, repeated runs bit for bit, gradients against differences."""
import ctypes
import math

import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb
import train_ref as tr
from dense_way import way  # noqa: F401

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5
TYPES = [(F32, F32), (F32, BF16), (BF16, BF16)]
SIZES = [(1, 1), (1, 2), (1, 7), (3, 8), (300, 3), (200, 4), (150, 5), (90, 9), (70, 31), (5, 33), (64, 64), (17, 255), (9, 256),
         (7, 257), (33, 300), (4, 511), (5, 513), (3, 770), (6, 1000), (5, 1024), (3, 1025), (5, 1500), (3, 2047), (4, 2048),
         (3, 2049), (3, 4095), (2, 4096), (2, 4100), (3, 5000), (3, 8191), (2, 8192), (2, 8193), (2, 16400), (1, 20001)]
GRADS = ("dx", "dbranch", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")


def rows(T, D, seed, dtype, sigma=1.0):
    return (sigma * (ref.randn((T, D), seed) * (1 + 3 * (torch.arange(D) % 13 == 5)) + 0.3)).to(dtype).cuda()


def case(T, D, st, bt, p=0.2, gate_rows=0, alpha=1.25, post=True, pre=True, gate=True, seed=17):
    G = -(-T // gate_rows) if gate_rows else 1
    wb = lambda k: ((1 + ref.randn((D,), k, 0.2)).cuda(), ref.randn((D,), k + 1, 0.2).cuda())  # noqa: E731
    common = dict(gate=ref.randn((G, D), 3, 0.5).cuda() if gate else None, gate_rows=gate_rows, alpha=alpha,
                  post=wb(4) if post else None, pre=wb(6) if pre else None, p=p, seed=seed)
    return rows(T, D, 1, st, 2.0), rows(T, D, 2, bt), common


def check_forward(x, branch, c, out, eps=EPS):
    h, y, post_stats, pre_stats = out
    r = tr.block_norm(x, branch, c["gate"], c["gate_rows"], c["alpha"], c["post"], c["pre"], eps, c["p"], c["seed"])
    ref.assert_within(h, r["h"], r["h_tol"] + ref.rounding(h.dtype, r["h"]), "h")
    for name, stats in (("post", post_stats), ("pre", pre_stats)):
        assert (stats is None) == (c[name] is None)
        if stats is not None:
            ref.assert_within(stats[0], r[name]["mean"], r[name]["mean_tol"], name + " mean")
            ref.assert_within(stats[1], r[name]["rstd"], r[name]["rstd_tol"], name + " rstd")
    assert (y is None) == (c["pre"] is None)
    if y is not None:
        ref.assert_within(y, r["pre"]["y"], r["pre"]["tol"] + ref.rounding(y.dtype, r["pre"]["y"]), "y")


def check_backward(dh, dy, h, branch, post_stats, pre_stats, c, got):
    r = tr.block_norm_backward(dh, dy, h, branch, post_stats, pre_stats, c["gate"], c["gate_rows"], c["alpha"], c["post"],
                               c["pre"], c["p"], c["seed"])
    for name, t in zip(GRADS, got):
        if t is not None:
            want, tol = r[name]
            ref.assert_within(t, want.reshape(t.shape), tol.reshape(t.shape) + ref.rounding(t.dtype, want).reshape(t.shape), name)


def both(T, D, st, bt, **kw):
    x, branch, c = case(T, D, st, bt, **kw)
    out = emb.block_norm(x, branch, eps=EPS, **c)
    check_forward(x, branch, c, out)
    h, y, post_stats, pre_stats = out
    dh, dy = rows(T, D, 11, st, 0.1), rows(T, D, 12, bt, 0.1) if c["pre"] is not None else None
    got = emb.block_norm_backward(dh, dy, h, branch, post_stats, pre_stats, **c)
    assert (got[2] is None) == (c["gate"] is None) and (got[3] is None) == (c["post"] is None)
    check_backward(dh, dy, h, branch, post_stats, pre_stats, c, got)
    again = emb.block_norm_backward(dh, dy, h, branch, post_stats, pre_stats, **c)
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b)  # the order of the sums depends on the sizes only
    return x, branch, c, out, dh, dy, got


@pytest.mark.parametrize("st,bt", TYPES)
@pytest.mark.parametrize("T,D", SIZES)
def test_forward_and_backward(T, D, st, bt):
    both(T, D, st, bt)


@pytest.mark.parametrize("T,D,st,bt", [(5000, 40, F32, F32), (2600, 260, BF16, BF16), (2049, 1030, F32, BF16),
                                       (1100, 4096, BF16, BF16), (600, 5000, F32, F32), (300, 17000, BF16, BF16)])
def test_more_rows_than_workgroups(T, D, st, bt):
    both(T, D, st, bt)


@pytest.mark.parametrize("T,D,gate_rows", [(1, 64, 1), (7, 20, 1), (100, 64, 7), (3000, 40, 1), (3000, 40, 3), (3000, 260, 700),
                                           (900, 1024, 899), (900, 1024, 900), (500, 1024, 10 ** 12), (257, 2048, 16),
                                           (5000, 8, 33), (64, 20000, 9), (2000, 512, 2)])
@pytest.mark.parametrize("st,bt", [(F32, F32), (BF16, BF16)])
def test_gates_of_groups(T, D, gate_rows, st, bt):
    both(T, D, st, bt, gate_rows=gate_rows)


@pytest.mark.parametrize("D", [24, 1023, 20000])
@pytest.mark.parametrize("post,pre,gate,p", [(False, True, True, 0.3), (True, False, True, 0.3), (False, False, True, 0.0),
                                             (True, True, False, 0.0), (False, False, False, 0.5), (True, True, True, 0.999)])
def test_parts_left_out(post, pre, gate, p, D):
    both(40, D, F32, BF16, post=post, pre=pre, gate=gate, p=p)


def test_norms_without_weight_or_bias():
    x, branch, c = case(50, 200, F32, F32)
    for post, pre in (((None, None), (None, None)), ((c["post"][0], None), (None, c["pre"][1])),
                      ((None, c["post"][1]), (c["pre"][0], None))):
        c["post"], c["pre"] = post, pre
        out = emb.block_norm(x, branch, eps=EPS, **c)
        check_forward(x, branch, c, out)
        dh, dy = rows(50, 200, 11, F32, 0.1), rows(50, 200, 12, F32, 0.1)
        check_backward(dh, dy, out[0], branch, out[2], out[3], c,
                       emb.block_norm_backward(dh, dy, out[0], branch, out[2], out[3], **c))


@pytest.mark.parametrize("D", [100, 1024, 5000, 20000])
def test_outputs_left_out(D, way):
    x, branch, c, (h, _, s0, s1), dh, dy, want = both(60, D, F32, BF16, gate_rows=25)
    for k in range(7):
        out = [torch.full_like(t, 9.0) if i == k else None for i, t in enumerate(want)]
        emb.block_norm_backward(dh, dy, h, branch, s0, s1, out=tuple(out), **c)
        assert torch.equal(out[k], want[k]), GRADS[k]
    got = emb.block_norm_backward(None, dy, h, branch, s0, s1, **c)
    check_backward(None, dy, h, branch, s0, s1, c, got)


@pytest.mark.parametrize("st,bt", TYPES)
@pytest.mark.parametrize("D", [48, 61, 1024, 4097])
def test_strides_and_in_place(D, st, bt, way):
    x, branch, c, out, dh, dy, want = both(20, D, st, bt)
    lay = lambda t: torch.full((20, D + 7), 5.0, dtype=t.dtype, device="cuda")[:, 3:3 + D].copy_(t)  # noqa: E731
    xs, bs = lay(x), lay(branch)
    stats = [torch.empty_like(s) for s in out[2:]]
    got = emb.block_norm(xs, bs, eps=EPS, out=(xs, bs, *stats), **c)  # h over x, y over branch
    for a, b in zip(got, out):
        assert torch.equal(a, b)
    assert all((t._base[:, :3] == 5.0).all() and (t._base[:, 3 + D:] == 5.0).all() for t in (xs, bs))
    dhs, dys = lay(dh), lay(dy)
    rest = [torch.empty_like(t) for t in want[2:]]
    got = emb.block_norm_backward(dhs, dys, lay(out[0]), lay(branch), *stats, out=(dhs, dys, *rest), **c)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert all((t._base[:, :3] == 5.0).all() and (t._base[:, 3 + D:] == 5.0).all() for t in (dhs, dys))


@pytest.mark.parametrize("D", [64, 1000, 9000])
def test_rows_that_are_not_finite_leave_the_others_alone(D):
    x, branch, c, out, dh, dy, want = both(30, D, F32, F32, gate_rows=1)
    for bad in (math.nan, math.inf):
        x2, b2 = x.clone(), branch.clone()
        x2[3, D // 2], b2[17, 0] = bad, bad
        got = emb.block_norm(x2, b2, eps=EPS, **c)
        keep = [t for t in range(30) if t not in (3, 17)]
        assert torch.equal(got[0][keep], out[0][keep]) and torch.equal(got[1][keep], out[1][keep])
        assert got[1][3].isnan().all() and got[1][17].isnan().all()
        h2 = out[0].clone()
        h2[3, D // 2] = bad
        g2 = emb.block_norm_backward(dh, dy, h2, branch, out[2], out[3], **c)
        assert all(torch.equal(a[keep], b[keep]) for a, b in zip(g2[:3], want[:3]))


@pytest.mark.parametrize("D", [64, 1000, 9000])
def test_what_is_dropped_is_not_used(D):
    """Without a norm after the block, a dropped element of it reaches nothing."""
    x, branch, c, out, dh, dy, want = both(30, D, F32, F32, post=False, p=0.5)
    gone = ~tr.kept(30, D, 0.5, c["seed"]).cuda()
    for bad in (math.nan, math.inf):
        b2 = torch.where(gone, bad, branch)
        for a, b in zip(emb.block_norm(x, b2, eps=EPS, **c), out):
            assert b is None or torch.equal(a, b)
        for a, b in zip(emb.block_norm_backward(dh, dy, out[0], b2, None, out[3], **c), want):
            assert b is None or torch.equal(a, b)


def test_no_rows(way):
    x = torch.empty(0, 40, device="cuda")
    c = dict(gate=torch.ones(40, device="cuda"), post=(None, None), pre=(None, None))
    h, y, s0, s1 = emb.block_norm(x, x, **c)
    assert h.shape == y.shape == (0, 40) and s0.shape == s1.shape == (2, 0)
    out = (h, y, *(torch.full((40,), 9.0, device="cuda") for _ in range(5)))
    emb.block_norm_backward(x, x, h, x, s0, s1, out=out, **c)
    assert all((t == 0).all() for t in out[2:])
    # gates of groups: none, so what stands at dgate's address stays
    behind = torch.full((40,), 9.0, device="cuda")
    args = emb.BlockNormGradArgs(T=0, D=40, stream_dtype=0, dtype=0, ldh=40, ldb=40, gate_rows=5, alpha=1.0,
                                 dgate=behind.data_ptr(), dpre_bias=out[6].data_ptr())
    assert emb.lib.emb_block_norm_backward(ctypes.addressof(args), torch.cuda.current_stream().cuda_stream) == emb.EMB_OK
    assert (behind == 9.0).all() and (out[6] == 0).all()


def test_one_gate_for_more_rows_than_there_are(way):
    x, branch, c, out, dh, dy, want = both(30, 40, F32, F32, gate_rows=30)
    c["gate_rows"] = (1 << 63) - 1
    for a, b in zip(emb.block_norm(x, branch, eps=EPS, **c), out):
        assert torch.equal(a, b)
    for a, b in zip(emb.block_norm_backward(dh, dy, out[0], branch, out[2], out[3], **c), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,D", [(50, 96), (300, 1024), (4, 9000)])
def test_graph_and_another_stream(T, D):
    x, branch, c, out, dh, dy, want = both(T, D, BF16, BF16)
    seed = torch.full((1,), c["seed"], dtype=torch.int64, device="cuda")
    c["seed"] = seed
    fresh = tuple(torch.empty_like(t) for t in out)
    grads = tuple(torch.empty_like(t) for t in want)
    ws = emb.new_workspace(emb.block_norm_backward_workspace_bytes(T, D))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    emb.block_norm(x, branch, eps=EPS, out=fresh, stream=s, **c)
    emb.block_norm_backward(dh, dy, fresh[0], branch, fresh[2], fresh[3], out=grads, workspace=ws, stream=s, **c)
    s.synchronize()
    for a, b in zip((*fresh, *grads), (*out, *want)):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        emb.block_norm(x, branch, eps=EPS, out=fresh, **c)
        emb.block_norm_backward(dh, dy, fresh[0], branch, fresh[2], fresh[3], out=grads, workspace=ws, **c)
    for k in (17, 18, 17, 99):
        seed.fill_(k)
        for t in (*fresh, *grads):
            t.fill_(3.0)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        eager = emb.block_norm(x, branch, eps=EPS, **{**c, "seed": k})
        back = emb.block_norm_backward(dh, dy, eager[0], branch, eager[2], eager[3], **{**c, "seed": k})
        for a, b in zip((*fresh, *grads), (*eager, *back)):
            assert torch.equal(a, b)


def test_gradients_against_differences():
    """The gradient of sum(h u + y v) in a direction, against the 64-bit form's difference: its own error is of the order
    of the step squared (1e-4 ** 2 times third derivatives of order 1e2 here), the fp32 gradients' of order 1e-5."""
    T, D = 12, 50
    x, branch, c = case(T, D, F32, F32, gate_rows=5)
    u, v = ref.randn((T, D), 21, 0.3).cuda(), ref.randn((T, D), 22, 0.3).cuda()
    h, _, s0, s1 = emb.block_norm(x, branch, eps=EPS, **c)
    got = emb.block_norm_backward(u, v, h, branch, s0, s1, **c)
    names = ("x", "branch", "gate", "post_w", "post_b", "pre_w", "pre_b")
    base = dict(zip(names, (x, branch, c["gate"], *c["post"], *c["pre"])))
    base = {k: ref.f64(t) for k, t in base.items()}

    def value(a):
        r = tr.block_norm(a["x"], a["branch"], a["gate"], 5, c["alpha"], (a["post_w"], a["post_b"]), (a["pre_w"], a["pre_b"]),
                          EPS, c["p"], c["seed"])
        return (r["h"] * ref.f64(u)).sum() + (r["pre"]["y"] * ref.f64(v)).sum()
    for k, (name, g) in enumerate(zip(names, got)):
        way = ref.randn(base[name].shape, 30 + k).double()
        step = [value({**base, name: base[name] + e * way}) for e in (1e-4, -1e-4)]
        diff, want = (step[0] - step[1]) / 2e-4, (ref.f64(g).reshape(way.shape) * way).sum()
        assert abs(diff - want) <= 1e-4 * max(1.0, ref.f64(g).norm() * way.norm()), name
