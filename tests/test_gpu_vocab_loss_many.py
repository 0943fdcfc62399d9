"""emb_vocab_loss and emb_vocab_loss_backward above the work that the few tokens' way takes, so in tiles of 256 tokens and
entries: bf16 and fp32, plain and smoothed, tables read where they stand and laid out first, tokens without a target, rows
that are not finite, strides, logits far apart, streams and graphs, several pieces of the table and of g.  WAYS names the
kernel that every size is here for; tests/test_loss_ways_host.py holds the library to it."""
import math

import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb
import train_ref as tr
from test_gpu_vocab_loss import BF16, F32, both, case

pytestmark = pytest.mark.gpu

# (tokens, entries, columns, type, whether the table is read where it stands, pieces of it forward, of g backward)
WAYS = {
    "stands": (1030, 5003, 512, BF16, True, 1, 1),
    "columns": (1030, 5003, 500, BF16, False, 1, 1),
    "narrow": (9000, 5003, 64, BF16, True, 1, 1),
    "odd": (300, 9001, 801, BF16, False, 1, 1),
    "planes": (1030, 5003, 512, F32, False, 1, 1),
    "planes_odd": (300, 9001, 801, F32, False, 1, 1),
    "table_pieces": (70, 600001, 65, BF16, False, 2, 1),
    "table_pieces_planes": (90, 340001, 72, F32, False, 2, 1),
    "g_pieces": (8000, 66003, 128, BF16, True, 1, 3),
    "g_pieces_columns": (8000, 66003, 72, BF16, False, 1, 3),
    "g_pieces_planes": (8000, 33003, 72, F32, False, 1, 3),
}


def size(name):
    T, V, D, dtype, *_ = WAYS[name]
    return T, V, D, dtype


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("name", ["stands", "columns", "narrow", "odd", "planes", "planes_odd"])
def test_forward_and_backward(name, smoothing):
    x, w, ids = case(*size(name), live=0.7)
    d = torch.full((1,), 1.0 / len(ids), device="cuda") if smoothing else None
    both(x, w, ids, smoothing=smoothing, d=d)


@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("name", ["table_pieces", "table_pieces_planes", "g_pieces", "g_pieces_columns", "g_pieces_planes"])
def test_pieces(name, each):
    """A sample of the tokens and of the entries, those at the pieces' seams among them, in 64 bits."""
    T, V, D, dtype = size(name)
    x, w, ids = case(T, V, D, dtype, live=0.9)
    smoothing = 0.1 if each else 0.0
    loss, lse = emb.vocab_loss(x, w, ids, smoothing)
    d = ref.randn((T,), 9, 0.1).cuda() if each else torch.full((1,), 1.0 / T, device="cuda")
    dx, dw = emb.vocab_loss_backward(d, x, w, ids, lse, smoothing)
    pick = torch.tensor([0, 1, T // 2, T - 2, T - 1])
    at = pick.cuda()
    r = tr.vocab_loss(x[at], w, ids[at], smoothing)
    ref.assert_within(loss[at], r["loss"], r["loss_tol"], "loss")
    ref.assert_within(lse[at], r["lse"], r["lse_tol"], "lse")
    r = tr.vocab_loss_backward(d[at] if each else d, x[at], w, ids[at], lse[at], smoothing)
    ref.assert_within(dx[at], r["dx"], r["dx_tol"], "dx")
    seams = [v for n in (1 << 28, 1 << 27, 1 << 26) for p in range(1, 8) for v in [p * n // (-(-T // 256) * 256)]]
    some = sorted({v + e for v in [0, V - 1, 524288, 174592, *seams] for e in (-1, 0, 1, 2) if 0 <= v + e < V})
    some = torch.tensor(some, device="cuda")
    # dtable of those entries: the form of train_ref.py with lse given, V only in the smoothing's share
    z = x.double() @ w[some].double().t()
    z_tol = (2.2 * (D + 8) * ref.U + 4 * ref.U) * (x.double().abs() @ w[some].double().abs().t()) + ref.TINY
    live, hot = (ids >= 0)[:, None], (ids[:, None] == some[None, :]).double()
    p, dd = torch.exp(z - lse.double()[:, None]), d.double().expand(T)[:, None]
    g = torch.where(live, dd * (p - (1 - smoothing) * hot - smoothing / V), 0.0)
    tol = 1.1 * dd.abs() * (p * (z_tol + 4 * ref.U * (z - lse.double()[:, None]).abs() + 4 * ref.U)
                            + 3 * ref.U * (p + hot + smoothing / V))
    tol = torch.where(live, tol + (ref.R16 if dtype == BF16 else 2 * ref.U) * g.abs(), 0.0)
    want = (g.t() @ x.double()).cpu()
    bound = (1.1 * (tol.t() @ x.double().abs()) + 2.2 * (T + 8) * ref.U * (g.abs().t() @ x.double().abs())).cpu()
    ref.assert_within(dw[some], want, bound + ref.TINY + ref.rounding(dtype, want), "dtable")


@pytest.mark.parametrize("name", ["stands", "planes"])
def test_tokens_without_a_target_and_rows_that_are_not_finite(name):
    T, V, D, dtype = size(name)
    x, w, ids = case(T, V, D, dtype)
    ids[500] = -7
    loss, lse = emb.vocab_loss(x, w, ids)
    d = ref.randn((T,), 9, 0.1).cuda()
    grads = emb.vocab_loss_backward(d, x, w, ids, lse)
    x2, ids2, d2, lse2, status = x.clone(), ids.clone(), d.clone(), lse.clone(), emb.new_status()
    x2[500], d2[500], lse2[500], ids2[500] = math.nan, math.inf, math.nan, V  # what stands there is not used
    for a, b in zip((*emb.vocab_loss(x2, w, ids2, dev_status=status),
                     *emb.vocab_loss_backward(d2, x2, w, ids2, lse2, dev_status=status)), (loss, lse, *grads)):
        assert torch.equal(a, b)
    assert status.item() == emb.EMB_DEV_ID_OUT_OF_RANGE
    none = torch.full_like(ids, -1)
    assert all((t == 0).all() for t in emb.vocab_loss(x, w, none))
    assert all((t == 0).all() for t in emb.vocab_loss_backward(d, x, w, none, lse))
    t = int(torch.nonzero(ids >= 0)[300])
    rest = torch.arange(T, device="cuda") != t
    for bad in (math.nan, math.inf):
        x2 = x.clone()
        x2[t, 7] = bad
        got = emb.vocab_loss(x2, w, ids)
        assert got[0][t].isnan() and torch.equal(got[0][rest], loss[rest]) and torch.equal(got[1][rest], lse[rest])
        dx, _ = emb.vocab_loss_backward(d, x2, w, ids, got[1])
        assert torch.equal(dx[rest], grads[0][rest]) and dx[t].isnan().all()


@pytest.mark.parametrize("dtype,first,ld", [(BF16, 8, 528), (BF16, 3, 523), (BF16, 0, 519), (F32, 1, 515)])
def test_strides(dtype, first, ld):
    """On 16-byte boundaries the table is read where it stands, else it is laid out: the sums are the same."""
    T, V, D = 1030, 5003, 512
    x, w, ids = case(T, V, D, dtype)
    loss, lse = emb.vocab_loss(x, w, ids)
    d = ref.randn((T,), 9, 0.1).cuda()
    want = emb.vocab_loss_backward(d, x, w, ids, lse)

    def lay(t):
        wide = torch.full((t.shape[0], ld), 7.0, dtype=dtype, device="cuda")
        return wide, wide[:, first:first + D].copy_(t)
    (_, xs), (_, ws) = lay(x), lay(w)
    (wx, ox), (ww, ow) = lay(torch.zeros_like(x)), lay(torch.zeros_like(w))
    got = emb.vocab_loss(xs, ws, ids)
    assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
    emb.vocab_loss_backward(d, xs, ws, ids, lse, out=(ox, ow))
    assert torch.equal(ox, want[0]) and torch.equal(ow, want[1])
    for wide in (wx, ww):
        assert (wide[:, :first] == 7.0).all() and (wide[:, first + D:] == 7.0).all()


@pytest.mark.parametrize("name", ["stands", "columns", "planes"])
def test_logits_far_apart(name):
    x, w, ids = case(*size(name), sigma=60.0)
    both(x, w, ids)


@pytest.mark.parametrize("name", ["stands", "columns", "planes"])
def test_graphs_streams_and_a_shared_workspace(name):
    T, V, D, dtype = size(name)
    x, w, ids = case(T, V, D, dtype)
    x2, _, ids2 = case(T, V, D, dtype, seed=40)
    d = ref.randn((T,), 9, 0.1).cuda()

    def eager(a, b):
        out = emb.vocab_loss(a, w, b)
        return (*out, *emb.vocab_loss_backward(d, a, w, b, out[1]))
    want = eager(x, ids), eager(x2, ids2)
    outs = [torch.empty_like(t) for t in want[0]]
    ws = emb.new_workspace(emb.vocab_loss_workspace_bytes(T, V, D, dtype))
    wb = emb.new_workspace(emb.vocab_loss_backward_workspace_bytes(T, V, D, dtype))
    xin, idin, s = x.clone(), ids.clone(), torch.cuda.Stream()

    def step(stream=None):
        emb.vocab_loss(xin, w, idin, out=tuple(outs[:2]), workspace=ws, stream=stream)
        emb.vocab_loss_backward(d, xin, w, idin, outs[1], out=tuple(outs[2:]), workspace=wb, stream=stream)
    s.wait_stream(torch.cuda.current_stream())
    step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want[0]))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for k in range(4):
        xin.copy_((x, x2)[k % 2])
        idin.copy_((ids, ids2)[k % 2])
        for t in (*outs, ws, wb):
            t.fill_(77)
        graphs[k // 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want[k % 2]))
