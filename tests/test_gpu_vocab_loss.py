"""emb_vocab_loss and emb_vocab_loss_backward against the 64-bit forms of train_ref.py, within the bounds derived there:
one token to more than a tile, vocabularies and widths that divide by nothing, both types, tables read where they stand
and laid out first, tokens without a target (some, all, bad ones, with NaN in their rows), smoothing, pieces, strides,
extreme logits, outputs left out, streams, graphs, repeated runs bit for bit, gradients against differences."""
import math

import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb
import train_ref as tr
from dense_way import way  # noqa: F401

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SIZES = [(1, 1, 1), (1, 5, 3), (2, 256, 64), (3, 257, 65), (1, 1000, 64), (31, 500, 40), (32, 1024, 128), (33, 700, 72),
         (64, 513, 100), (65, 2000, 256), (130, 999, 37), (255, 300, 192), (256, 512, 64), (257, 1025, 320), (700, 1500, 130),
         (1030, 260, 520), (5, 4100, 1024)]


def case(T, V, D, dtype, live=0.8, seed=1, sigma=2.0):
    x, w = ref.randn((T, D), seed).to(dtype).cuda(), ref.randn((V, D), seed + 1, sigma / math.sqrt(D)).to(dtype).cuda()
    g = ref.gen(seed + 2)
    ids = torch.randint(0, V, (T,), generator=g)
    ids[torch.rand(T, generator=g) >= live] = -100
    if T > 2:
        ids[0], ids[-1] = 0, V - 1
    return x, w, ids.int().cuda()


def check_forward(x, w, ids, smoothing, out):
    r = tr.vocab_loss(x, w, ids, smoothing)
    ref.assert_within(out[1], r["lse"], r["lse_tol"], "lse")
    ref.assert_within(out[0], r["loss"], r["loss_tol"], "loss")


def check_backward(d, x, w, ids, lse, smoothing, out):
    r = tr.vocab_loss_backward(d, x, w, ids, lse, smoothing)
    for name, t in zip(("dx", "dtable"), out):
        if t is not None:
            ref.assert_within(t, r[name], r[name + "_tol"], name)


def both(x, w, ids, smoothing=0.0, d=None):
    out = emb.vocab_loss(x, w, ids, smoothing)
    check_forward(x, w, ids, smoothing, out)
    d = ref.randn((x.shape[0],), 9, 0.1).cuda() if d is None else d
    got = emb.vocab_loss_backward(d, x, w, ids, out[1], smoothing)
    check_backward(d, x, w, ids, out[1], smoothing, got)
    for a, b in zip((*out, *got), (*emb.vocab_loss(x, w, ids, smoothing),
                                   *emb.vocab_loss_backward(d, x, w, ids, out[1], smoothing))):
        assert torch.equal(a, b)
    return out, d, got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_forward_and_backward(T, V, D, dtype):
    both(*case(T, V, D, dtype))
    both(*case(T, V, D, dtype, live=1.0, seed=5), smoothing=0.1, d=torch.full((1,), 1.0 / T, device="cuda"))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,D", [(1, 70, 2000), (16, 300, 1024), (17, 45, 1000), (33, 310, 1001), (48, 200, 700), (64, 130, 1024),
                                   (64, 1, 5), (7, 16, 31), (2, 17, 129), (9, 33, 4097)])
def test_few_tokens_of_wide_rows(T, V, D, dtype):
    both(*case(T, V, D, dtype), smoothing=0.1)


@pytest.mark.parametrize("dtype,T,V,D", [(BF16, 64, 17001, 1000), (F32, 1, 40003, 130), (BF16, 40, 30011, 64), (F32, 300, 9000, 300), (BF16, 2000, 6000, 64)])
def test_larger(dtype, T, V, D):
    both(*case(T, V, D, dtype, live=0.5), smoothing=0.05)


def test_several_pieces_of_the_table():
    """More than one piece: of a table that is laid out (fp32, 2^26 elements of three planes), and of g (2^27)."""
    T, V, D = 4096, 33000, 1024
    x, w, ids = case(T, V, D, F32, live=0.9)
    loss, lse = emb.vocab_loss(x, w, ids, 0.1)
    d = torch.full((1,), 1.0 / T, device="cuda")
    dx, dw = emb.vocab_loss_backward(d, x, w, ids, lse, 0.1)
    # a sample of tokens, and of entries of both ends and the pieces' seams, in 64 bits
    pick = torch.tensor([0, 1, 777, 4095])
    r = tr.vocab_loss(x[pick], w, ids[pick], 0.1)
    ref.assert_within(loss[pick.cuda()], r["loss"], r["loss_tol"], "loss")
    ref.assert_within(lse[pick.cuda()], r["lse"], r["lse_tol"], "lse")
    r = tr.vocab_loss_backward(d, x[pick], w, ids[pick], lse[pick.cuda()], 0.1)
    ref.assert_within(dx[pick.cuda()], r["dx"], r["dx_tol"], "dx")
    some = torch.cat([torch.arange(0, 40), torch.arange(10750, 11010), torch.arange(21500, 22020), torch.arange(32700, 33000)])
    z = x.double() @ w[some.cuda()].double().t()
    hot = (ids[:, None] == some.cuda()[None, :]).double()
    g = torch.where(ids[:, None] >= 0, torch.exp(z - lse.double()[:, None]) - 0.9 * hot - 0.1 / V, 0.0) / T
    want = (g.t() @ x.double()).cpu()
    scale = (g.abs().t() @ x.double().abs()).cpu()
    ref.assert_within(dw[some.cuda()], want, 2.2 * (T + D + 64) * ref.U * scale + ref.TINY, "dtable")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [1, 40, 300])
def test_tokens_without_a_target(dtype, T):
    x, w, ids = case(T, 600, 96, dtype)
    status = emb.new_status()
    none = torch.full_like(ids, -1)
    loss, lse = emb.vocab_loss(x, w, none, dev_status=status)
    assert (loss == 0).all() and (lse == 0).all()
    dx, dw = emb.vocab_loss_backward(torch.ones(T, device="cuda"), x, w, none, lse, dev_status=status)
    assert (dx == 0).all() and (dw == 0).all() and status.item() == 0
    one = torch.full((1,), math.inf, device="cuda")  # a mean over no tokens
    dx, dw = emb.vocab_loss_backward(one, x, w, none, lse, dev_status=status)
    assert (dx == 0).all() and (dw == 0).all() and status.item() == 0
    ids[T // 2] = -7
    want = emb.vocab_loss(x, w, ids)
    d = torch.ones(T, device="cuda")
    grads = emb.vocab_loss_backward(d, x, w, ids, want[1])
    x2, ids2 = x.clone(), ids.clone()
    x2[T // 2] = math.nan         # what stands in its row is not used
    d[T // 2] = math.inf
    lse2 = want[1].clone()
    lse2[T // 2] = math.nan
    ids2[T // 2] = 600            # nor is a target that is no row, which is flagged
    for a, b in zip((*emb.vocab_loss(x2, w, ids2, dev_status=status),
                     *emb.vocab_loss_backward(d, x2, w, ids2, lse2, dev_status=status)), (*want, *grads)):
        assert torch.equal(a, b)
    assert status.item() == emb.EMB_DEV_ID_OUT_OF_RANGE


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,first,ld", [(64, 0, 64), (64, 8, 96), (64, 3, 75), (50, 1, 131), (256, 0, 264)])
def test_strides(dtype, D, first, ld, way):
    T, V = 70, 530
    x, w, ids = case(T, V, D, dtype)
    (loss, lse), d, (dx, dw) = both(x, w, ids)

    def lay(t):
        wide = torch.full((t.shape[0], ld), 7.0, dtype=dtype, device="cuda")
        return wide, wide[:, first:first + D].copy_(t)
    (_, xs), (_, ws) = lay(x), lay(w)
    (wx, ox), (ww, ow) = lay(torch.zeros_like(x)), lay(torch.zeros_like(w))
    kept = torch.empty_like(loss), torch.empty_like(lse)
    got = emb.vocab_loss(xs, ws, ids, out=kept, workspace=emb.new_workspace(emb.vocab_loss_workspace_bytes(T, V, D, dtype)))
    assert got is kept and torch.equal(got[0], loss) and torch.equal(got[1], lse)
    emb.vocab_loss_backward(d, xs, ws, ids, lse, out=(ox, ow),
                            workspace=emb.new_workspace(emb.vocab_loss_backward_workspace_bytes(T, V, D, dtype)))
    assert torch.equal(ox, dx) and torch.equal(ow, dw)
    for wide in (wx, ww):
        assert (wide[:, :first] == 7.0).all() and (wide[:, first + D:] == 7.0).all()


def test_outputs_left_out_and_behind_the_last(way):
    x, w, ids = case(90, 300, 64, BF16)
    (loss, lse), d, (dx, dw) = both(x, w, ids)
    a, b = torch.full((92, 64), 3.0, dtype=BF16, device="cuda"), torch.full((303, 64), 3.0, dtype=BF16, device="cuda")
    emb.vocab_loss_backward(d, x, w, ids, lse, out=(a[:90], None))
    emb.vocab_loss_backward(d, x, w, ids, lse, out=(None, b[:300]))
    assert torch.equal(a[:90], dx) and torch.equal(b[:300], dw) and (a[90:] == 3.0).all() and (b[300:] == 3.0).all()


def test_no_tokens(way):
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(30, 64, device="cuda")
    ids, d = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    loss, lse = emb.vocab_loss(x, w, ids)
    assert loss.shape == lse.shape == (0,)
    dx, dw = emb.vocab_loss_backward(d, x, w, ids, lse)
    assert dx.shape == (0, 64) and (dw == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_far_apart(dtype):
    """Hundreds apart and far from zero: only the differences to the largest count."""
    x, w, ids = case(50, 700, 64, dtype, sigma=60.0)
    both(x, w, ids)
    w2 = torch.zeros_like(w)
    w2[:, 0], x[:, 0] = 512.0, 16.0   # all logits 8192: a uniform distribution
    out, _, _ = both(x, w2, ids)
    live = ids >= 0
    assert (out[0][live] - math.log(700)).abs().max() <= 2 * 8192 * ref.U + 1e-5  # lse and z are rounded at 8192


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_that_are_not_finite(dtype, bad):
    x, w, ids = case(300, 520, 64, dtype, live=1.0)
    loss, lse = emb.vocab_loss(x, w, ids)
    x2 = x.clone()
    x2[5, 7] = bad
    got = emb.vocab_loss(x2, w, ids)
    rest = [t for t in range(300) if t != 5]
    assert got[0][5].isnan() and torch.equal(got[0][rest], loss[rest]) and torch.equal(got[1][rest], lse[rest])


def test_graphs_streams_and_a_shared_workspace():
    T, V, D = 200, 1100, 128
    x, w, ids = case(T, V, D, BF16)
    x2, _, ids2 = case(T, V, D, BF16, seed=40)
    (loss, lse), d, (dx, dw) = both(x, w, ids)
    outs = [torch.empty_like(t) for t in (loss, lse, dx, dw)]
    ws = emb.new_workspace(emb.vocab_loss_workspace_bytes(T, V, D, BF16))
    wb = emb.new_workspace(emb.vocab_loss_backward_workspace_bytes(T, V, D, BF16))

    def step(stream=None):
        emb.vocab_loss(xin, w, idin, out=tuple(outs[:2]), workspace=ws, stream=stream)
        emb.vocab_loss_backward(d, xin, w, idin, outs[1], out=tuple(outs[2:]), workspace=wb, stream=stream)
    xin, idin, s = x.clone(), ids.clone(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(s)
    s.synchronize()
    for a, b in zip(outs, (loss, lse, dx, dw)):
        assert torch.equal(a, b)
    graphs = []
    for _ in range(2):  # two graphs with one workspace, replayed one after the other
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for k in range(4):
        a, b = (x, ids) if k % 2 == 0 else (x2, ids2)
        xin.copy_(a)
        idin.copy_(b)
        for t in (*outs, ws, wb):
            t.fill_(77)
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        l2 = emb.vocab_loss(a, w, b)
        g2 = emb.vocab_loss_backward(d, a, w, b, l2[1])
        for u, v in zip(outs, (*l2, *g2)):
            assert torch.equal(u, v)


def test_gradients_against_differences():
    """The sum of weighted losses in a direction, against the 64-bit form's difference (error of the order of the step
    squared); the fp32 gradients are good to about 1e-6 of their size."""
    x, w, ids = case(20, 90, 32, F32)
    d = ref.randn((20,), 4).cuda()
    _, lse = emb.vocab_loss(x, w, ids, 0.1)
    got = emb.vocab_loss_backward(d, x, w, ids, lse, 0.1)
    for k, g in enumerate(got):
        way = ref.randn(g.shape, 50 + k).double()

        def value(e):
            a = [ref.f64(x), ref.f64(w)]
            a[k] = a[k] + e * way
            return (tr.vocab_loss(*a, ids, 0.1)["loss"] * ref.f64(d)).sum()
        diff = (value(1e-4) - value(-1e-4)) / 2e-4
        assert abs(diff - (ref.f64(g) * way).sum()) <= 1e-5 * ref.f64(g).norm() * way.norm()
