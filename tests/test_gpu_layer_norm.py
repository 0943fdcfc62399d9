"""emb_layer_norm and emb_layer_norm_backward against the 64-bit forms of tests/dense_ref.py, within the
bounds derived there: row widths on both sides of every change of plan (several rows per wave, one wave,
4 and 8 waves per row, rows read again from memory), ragged widths, both types in every combination,
looked-up rows with ids that are no rows, strided and broadcast rows, offsets past 2^31 elements, rows
with infinities and NaN beside others, constant rows, rows far from zero, empty batches, in-place calls,
another stream, graph replays, repeated runs bit for bit, and the gradient against differences."""
import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb
from dense_way import way  # noqa: F401

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-5
SIZES = [(1, 1), (1, 7), (3, 8), (700, 2), (300, 3), (200, 4), (150, 5), (90, 9), (70, 31), (5, 33), (64, 64), (17, 255), (9, 256), (3, 770), (5, 1500), (7, 257), (33, 300), (4, 511),
         (5, 513), (6, 1000), (5, 1024), (3, 1025), (4, 1536), (3, 2047), (4, 2048), (3, 2049), (2, 4100), (3, 5000), (3, 6150),
         (3, 8192), (2, 8193), (2, 12290), (2, 16384), (1, 16385), (3, 20001)]
TYPES = [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)]


def rows(T, D, seed, dtype):
    return (ref.randn((T, D), seed) * (1 + 3 * (torch.arange(D) % 13 == 5)) + 0.3).to(dtype).cuda()


def params(D, seed):
    return (1 + ref.randn((D,), seed, 0.2)).cuda(), ref.randn((D,), seed + 1, 0.2).cuda()


def check_forward(x_rows, w, b, out, eps=EPS):
    y, mean, rstd = out
    r = ref.layer_norm(x_rows, w, b, eps)
    ref.assert_within(mean, r["mean"], r["mean_tol"], "mean")
    ref.assert_within(rstd, r["rstd"], r["rstd_tol"], "rstd")
    ref.assert_within(y, r["y"], r["tol"] + ref.rounding(y.dtype, r["y"]), "y")


def check_backward(dy, x_rows, mean, rstd, w, out):
    dx, dw, db = out
    r = ref.layer_norm_backward(dy, x_rows, mean, rstd, w)
    if dx is not None:
        ref.assert_within(dx, r["dx"], r["dx_tol"] + ref.rounding(dx.dtype, r["dx"]), "dx")
    if dw is not None:
        ref.assert_within(dw, r["dw"], r["dw_tol"], "dweight")
    if db is not None:
        ref.assert_within(db, r["db"], r["db_tol"], "dbias")


@pytest.mark.parametrize("xt,yt", TYPES)
@pytest.mark.parametrize("T,D", SIZES)
def test_forward_and_backward(T, D, xt, yt):
    x, (w, b) = rows(T, D, 1, xt), params(D, 2)
    out = emb.layer_norm(x, w, b, EPS, out_dtype=yt)
    assert out[0].dtype == yt
    check_forward(x, w, b, out)
    dy = ref.randn((T, D), 5, 0.1).to(yt).cuda()
    _, mean, rstd = out
    check_backward(dy, x, mean, rstd, w, emb.layer_norm_backward(dy, x, mean, rstd, w))


@pytest.mark.parametrize("T,D,xt,yt", [(5000, 40, F32, F32), (2600, 260, BF16, BF16), (2049, 1030, F32, BF16),
                                       (700, 4096, BF16, BF16), (300, 17000, F32, F32)])
def test_more_rows_than_workgroups(T, D, xt, yt):
    x, (w, b) = rows(T, D, 11, xt), params(D, 12)
    out = emb.layer_norm(x, w, b, EPS, out_dtype=yt)
    check_forward(x, w, b, out)
    dy = ref.randn((T, D), 15, 0.1).to(yt).cuda()
    got = emb.layer_norm_backward(dy, x, out[1], out[2], w)
    check_backward(dy, x, out[1], out[2], w, got)
    again = emb.layer_norm_backward(dy, x, out[1], out[2], w)
    for a, c in zip(got, again):
        assert torch.equal(a, c)  # the order of the sums depends on the sizes only


@pytest.mark.parametrize("D", [64, 300, 1024, 5000, 16400])
def test_looked_up_rows(D, way):
    V, T = 500, 77
    table, (w, b) = rows(V, D, 21, F32), params(D, 22)
    ids = torch.randint(0, V, (T,), generator=ref.gen(3), dtype=torch.int32)
    ids[5], ids[40], ids[76] = -1, V, 2 ** 31 - 1
    st = emb.new_status()
    d_ids = ids.cuda()
    out = emb.layer_norm(table, w, b, EPS, ids=d_ids, out_dtype=BF16, dev_status=st)
    x = torch.where(((ids >= 0) & (ids < V))[:, None], table.cpu()[ids.clamp(0, V - 1).long()], 0.0)
    check_forward(x, w, b, out)
    assert st.item() == emb.EMB_DEV_ID_OUT_OF_RANGE
    # the lookup and the norm in two calls give the same bits
    two = emb.layer_norm(emb.gather(table, d_ids), w, b, EPS, out_dtype=BF16)
    for a, c in zip(out, two):
        assert torch.equal(a, c)
    dy = ref.randn((T, D), 25, 0.1).to(BF16).cuda()
    st.zero_()
    got = emb.layer_norm_backward(dy, table, out[1], out[2], w, ids=d_ids, dev_status=st)
    check_backward(dy, x, out[1], out[2], w, got)
    assert st.item() == emb.EMB_DEV_ID_OUT_OF_RANGE
    st.zero_()
    ok = d_ids.clamp(0, V - 1)
    emb.layer_norm(table, w, b, EPS, ids=ok, dev_status=st)
    emb.layer_norm_backward(dy, table, out[1], out[2], w, ids=ok, dev_status=st)
    assert st.item() == 0


@pytest.mark.parametrize("T,D,xt", [(13, 100, F32), (13, 101, BF16), (9, 1500, BF16), (3, 16390, F32)])
def test_strided_rows_and_optional_arguments(T, D, xt, way):
    wide = rows(T, 3 * D + 5, 31, xt)
    x = wide[:, 3:3 + D]  # rows at odd places of a wider buffer
    dy_wide = ref.randn((T, 2 * D + 1), 32, 0.1).to(xt).cuda()
    dy = dy_wide[:, 1:1 + D]
    keep = torch.full((T, D + 9), 7.0, dtype=xt, device="cuda")
    y = keep[:, 4:4 + D]
    stats = torch.empty((2, T), device="cuda")
    out = emb.layer_norm(x, None, None, EPS, out=(y, stats[0], stats[1]))
    check_forward(x, None, None, out)
    assert (keep[:, :4] == 7).all() and (keep[:, 4 + D:] == 7).all()
    w, _ = params(D, 33)
    mean, rstd = out[1], out[2]
    check_forward(x, w, None, emb.layer_norm(x, w, None, EPS))
    check_forward(x, None, w, emb.layer_norm(x, None, w, EPS))
    ws = emb.new_workspace(emb.layer_norm_backward_workspace_bytes(T, D))
    full = emb.layer_norm_backward(dy, x, mean, rstd, w)
    check_backward(dy, x, mean, rstd, w, full)
    keep.fill_(7.0)
    dw, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    for want in ((y, None, None), (None, dw, None), (None, None, db), (y, dw, None)):
        got = emb.layer_norm_backward(dy, x, mean, rstd, w, out=want, workspace=ws)
        for a, c in zip(got, full):
            assert a is None or torch.equal(a, c)
    assert (keep[:, :4] == 7).all() and (keep[:, 4 + D:] == 7).all()
    check_backward(dy, x, mean, rstd, None, emb.layer_norm_backward(dy, x, mean, rstd))
    # one row for every token
    one = rows(1, D, 35, xt).expand(T, D)
    out = emb.layer_norm(one, w, None, EPS)
    check_forward(one, w, None, out)
    got = emb.layer_norm_backward(dy[:1].expand(T, D), one, out[1], out[2], w)
    check_backward(dy[:1].expand(T, D), one, out[1], out[2], w, got)


@pytest.mark.parametrize("D", [60, 1024, 4096, 16400])
def test_in_place(D, way):
    x, (w, b) = rows(6, D, 41, F32), params(D, 42)
    y, mean, rstd = emb.layer_norm(x, w, b, EPS)
    x2 = x.clone()
    emb.layer_norm(x2, w, b, EPS, out=(x2, mean, rstd))
    assert torch.equal(x2, y)
    dy = ref.randn((6, D), 43, 0.1).cuda()
    want = emb.layer_norm_backward(dy, x, mean, rstd, w)
    got = emb.layer_norm_backward(dy, x, mean, rstd, w, out=(dy, torch.empty_like(w), torch.empty_like(w)))
    for a, c in zip(got, want):
        assert torch.equal(a, c)


@pytest.mark.parametrize("D", [24, 700, 3000])
def test_rows_that_are_not_ordinary(D):
    x, (w, b) = rows(40, D, 51, F32), params(D, 52)
    x[3] = 0.0
    x[4] = 5.0                                     # constant: the variance is zero, eps decides
    x[5] = 1000.0 + x[5]                           # far from zero
    x[6] *= 1e-20                                  # far below eps
    x[7] *= 1e15                                   # squares near the top of the range
    check_forward(x, w, b, emb.layer_norm(x, w, b, EPS))
    want, mean, rstd = emb.layer_norm(x, w, b, EPS)
    dy = ref.randn((40, D), 53, 0.1).cuda()
    check_backward(dy, x, mean, rstd, w, emb.layer_norm_backward(dy, x, mean, rstd, w))
    bad = x.clone()
    bad[10, D // 2], bad[20, 0], bad[30, D - 1] = float("nan"), float("inf"), -float("inf")
    y, m2, r2 = emb.layer_norm(bad, w, b, EPS)
    sick = torch.zeros(40, dtype=torch.bool, device="cuda")
    sick[[10, 20, 30]] = True
    assert torch.isnan(y[sick]).all()
    assert torch.equal(y[~sick], want[~sick])
    dx, _, _ = emb.layer_norm_backward(dy, bad, m2, r2, w)
    assert torch.isnan(dx[sick]).all() and torch.isfinite(dx[~sick]).all()


def test_empty_batch(way):
    x, (w, b) = torch.empty((0, 40), device="cuda"), params(40, 61)
    y, mean, rstd = emb.layer_norm(x, w, b)
    assert y.shape == (0, 40) and mean.numel() == 0 and rstd.numel() == 0
    dw, db = torch.full((40,), 3.0, device="cuda"), torch.full((40,), 3.0, device="cuda")
    emb.layer_norm_backward(x, x, mean, rstd, w, out=(None, dw, db))
    assert (dw == 0).all() and (db == 0).all()


def test_more_rows_than_one_launch_takes():
    # a launch holds 2^20 workgroups of 32 rows of 24 elements, two at a time: 2^26 rows
    T, D = (1 << 26) + 1001, 24
    one = rows(1, D, 64, BF16)
    w, b = params(D, 65)
    y, mean, rstd = emb.layer_norm(one.expand(T, D), w, b, EPS)
    want = emb.layer_norm(one, w, b, EPS)
    for a, c in zip((y, mean[:, None], rstd[:, None]), want):
        assert (a == c.view(1, -1)).all()


def test_offsets_past_32_bits():
    D, ld = 1000, (1 << 30) + 12345  # row 2 starts past 2^31 elements
    flat = torch.empty(2 * ld + D, dtype=BF16, device="cuda")
    x = flat.as_strided((3, D), (ld, 1))
    x.copy_(rows(3, D, 71, BF16))
    w, b = params(D, 72)
    out = emb.layer_norm(x, w, b, EPS)
    check_forward(x, w, b, out)
    check_forward(x[[0, 2]], w, b, emb.layer_norm(x, w, b, EPS, ids=torch.tensor([0, 2], dtype=torch.int32,
                                                                                  device="cuda"), out_dtype=BF16))
    dy = ref.randn((3, D), 73, 0.1).to(BF16).cuda()
    want = emb.layer_norm_backward(dy, x, out[1], out[2], w)
    check_backward(dy, x, out[1], out[2], w, want)
    keep = x.clone()
    got = emb.layer_norm_backward(dy, keep, out[1], out[2], w,
                                  out=(x, torch.empty(D, device="cuda"), torch.empty(D, device="cuda")))
    for a, c in zip(got, want):
        assert torch.equal(a, c)


@pytest.mark.parametrize("D", [12, 300])
def test_gradient_against_differences(D):
    T, h = 4, 1e-4
    x, (w, b) = rows(T, D, 81, F32), params(D, 82)
    dy = ref.randn((T, D), 83).cuda()
    _, mean, rstd = emb.layer_norm(x, w, b, EPS)
    grads = [ref.f64(t) for t in emb.layer_norm_backward(dy, x, mean, rstd, w)]
    at = [ref.f64(t) for t in (x, w, b)]

    def loss(x, w, b):
        return (ref.layer_norm(x, w, b, EPS)["y"] * ref.f64(dy)).sum().item()
    for i, g in enumerate(grads):
        for seed in range(3):
            u = ref.randn(g.shape, 84 + seed).double()
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * u, at[i] - h * u
            slope = (loss(*up) - loss(*down)) / (2 * h)
            # central differences are off by h^2 / 6 times the third derivative (below 1e3 of the scale
            # here), the kernel by fp32 roundings
            scale = (g.abs() * u.abs()).sum().item()
            assert abs(slope - (g * u).sum().item()) <= 1e-5 * scale


def test_another_stream_and_graph_replays(way):
    T, D = 200, 320
    x, (w, b) = rows(T, D, 91, F32), params(D, 92)
    dy = ref.randn((T, D), 93, 0.1).cuda()
    want = emb.layer_norm(x, w, b, EPS)
    gwant = emb.layer_norm_backward(dy, x, want[1], want[2], w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = emb.layer_norm(x, w, b, EPS, stream=side)
    ggot = emb.layer_norm_backward(dy, x, got[1], got[2], w, stream=side)
    side.synchronize()
    for a, c in zip(got + ggot, want + gwant):
        assert torch.equal(a, c)
    outs = [torch.zeros_like(t) for t in want + gwant]
    ws = emb.new_workspace(emb.layer_norm_backward_workspace_bytes(T, D))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        emb.layer_norm(x, w, b, EPS, out=tuple(outs[:3]))
        emb.layer_norm_backward(dy, x, outs[1], outs[2], w, out=tuple(outs[3:]), workspace=ws)
    for k in range(4):
        x.copy_(rows(T, D, 100 + k, F32))
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        want = emb.layer_norm(x, w, b, EPS)
        gwant = emb.layer_norm_backward(dy, x, want[1], want[2], w)
        for a, c in zip(outs, want + gwant):
            assert torch.equal(a, c)


def test_refusals(way):
    x, w = rows(4, 32, 1, F32), torch.ones(32, device="cuda")
    y, mean, rstd = emb.layer_norm(x, w, w)
    ws = emb.new_workspace(1 << 20)
    for call in (lambda: emb.layer_norm(x.double()), lambda: emb.layer_norm(x.cpu()), lambda: emb.layer_norm(x[0]),
                 lambda: emb.layer_norm(x.t()), lambda: emb.layer_norm(x, w[:31]), lambda: emb.layer_norm(x, w.bfloat16()),
                 lambda: emb.layer_norm(x, w, w[:5]), lambda: emb.layer_norm(x, eps=-1.0),
                 lambda: emb.layer_norm(x, eps=float("nan")), lambda: emb.layer_norm(x, ids=torch.zeros(3, device="cuda")),
                 lambda: emb.layer_norm(x, out=(y[:3], mean, rstd)), lambda: emb.layer_norm(x, out=(y, mean[:3], rstd)),
                 lambda: emb.layer_norm(x, out=(y[:1].expand(4, 32), mean, rstd)),
                 lambda: emb.layer_norm(x, out=(y, mean, rstd), out_dtype=BF16),
                 lambda: emb.layer_norm_backward(y[:3], x, mean, rstd, w),
                 lambda: emb.layer_norm_backward(y, x, mean[:2], rstd, w),
                 lambda: emb.layer_norm_backward(y, x, mean, rstd, w, out=(y.bfloat16(), None, None)),
                 lambda: emb.layer_norm_backward(y, x, mean, rstd, w, out=(None, w[:31], None)),
                 lambda: emb.layer_norm_backward(y, x, mean, rstd, w, out=(None, None, None)),
                 lambda: emb.layer_norm_backward(y, x, mean, rstd, w, workspace=emb.new_workspace(16)),
                 lambda: emb.layer_norm_backward(y, x, mean, rstd, w, out=(y, w, w[:3]), workspace=ws),
                 lambda: emb.layer_norm_backward(y, x, mean, rstd, w, out=(y[:, :31], w, w), workspace=ws),
                 lambda: emb.layer_norm_backward(y, x, mean.double(), rstd, w, workspace=ws),
                 lambda: emb.layer_norm_backward(y.t(), x, mean, rstd, w, workspace=ws)):
        with pytest.raises(emb.EmbError):
            call()
