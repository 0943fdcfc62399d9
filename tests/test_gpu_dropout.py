"""emb_dropout against its 64-bit form with the same mask (train_ref.py): both types, with and without a residual, widths
on every side of the vectors and draws, strided and offset rows, in-place calls, infinities and NaN in what is dropped,
seeds on the device and in graphs, another stream, rows behind the last."""
import math

import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb
import train_ref as tr
from dense_way import way  # noqa: F401

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SIZES = [(1, 1), (1, 4), (3, 7), (5, 8), (70, 31), (64, 64), (33, 255), (9, 300), (5, 1023), (4, 1024), (3, 2049),
         (2, 8192), (1, 100003), (3000, 12), (700, 513)]


def rows(T, D, seed, dtype):
    return ref.randn((T, D), seed).to(dtype).cuda()


def check(x, p, seed, residual, y):
    want, tol = tr.dropout(x, p, seed, residual)
    ref.assert_within(y, want, tol, "y")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,D", SIZES)
def test_forward(T, D, dtype):
    x, r = rows(T, D, 1, dtype), rows(T, D, 2, dtype)
    check(x, 0.3, 77, r, emb.dropout(x, 0.3, 77, residual=r))
    y = emb.dropout(x, 0.3, 77)
    check(x, 0.3, 77, None, y)
    assert torch.equal((y != 0).cpu(), tr.kept(T, D, 0.3, 77) & (x != 0).cpu())


@pytest.mark.parametrize("p", [0.0, 1e-9, 1 / 65536, 0.1, 0.5, 0.99, 0.99999, math.nextafter(1.0, 0.0)])
def test_shares(p):
    x = torch.ones(64, 1000, device="cuda")
    y = emb.dropout(x, p, 5)
    check(x, p, 5, None, y)
    n, q = x.numel(), tr.cut_of(p) / 65536
    gone = int((y == 0).sum())
    assert abs(gone - n * q) <= 6 * math.sqrt(n * q * (1 - q)) + 1e-9  # six deviations of a binomial count


@pytest.mark.parametrize("seed", [0, 1, -1, (1 << 63) + 5, 1 << 64])
def test_seeds(seed):
    x = rows(7, 130, 3, F32)
    y = emb.dropout(x, 0.4, seed)
    check(x, 0.4, seed, None, y)
    assert torch.equal(y, emb.dropout(x, 0.4, seed))
    assert not torch.equal(y, emb.dropout(x, 0.4, seed + 1))


def test_neighbouring_seeds_and_places_are_independent():
    x = torch.ones(400, 1000, device="cuda")
    a, b = (emb.dropout(x, 0.5, s) != 0 for s in (10, 11))
    n = x.numel()
    for u, v in ((a, b), (a[:, 1:], a[:, :-1]), (a[1:], a[:-1]), (a[:, 4:], a[:, :-4])):
        same = (u == v).float().mean().item()
        assert abs(same - 0.5) <= 6 * 0.5 / math.sqrt(n - 4000)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first,D", [(0, 40), (1, 40), (3, 41), (2, 300)])
def test_strides(first, D, dtype, way):
    wide, out = rows(9, 400, 4, dtype), torch.full((9, 400), 7.0, dtype=dtype, device="cuda")
    x, r, y = wide[:, first:first + D], wide[:, 100:100 + D], out[:, 50 + first:50 + first + D]
    assert emb.dropout(x, 0.25, 9, residual=r, out=y) is y
    check(x, 0.25, 9, r, y)
    rest = torch.ones_like(out, dtype=torch.bool)
    rest[:, 50 + first:50 + first + D] = False
    assert (out[rest] == 7.0).all()
    check(x[:1].expand(9, D), 0.25, 9, None, emb.dropout(x[:1].expand(9, D), 0.25, 9))  # one row, read again


@pytest.mark.parametrize("D", [64, 301])
def test_in_place(D, way):
    x, r = rows(50, D, 5, BF16), rows(50, D, 6, BF16)
    want = emb.dropout(x, 0.2, 3, residual=r)
    a, b = x.clone(), r.clone()
    assert torch.equal(emb.dropout(a, 0.2, 3, residual=r, out=a), want)
    assert torch.equal(emb.dropout(x, 0.2, 3, residual=b, out=b), want)


def test_what_is_dropped_is_not_used():
    x, r = rows(20, 100, 7, F32), rows(20, 100, 8, F32)
    gone = ~tr.kept(20, 100, 0.5, 1).cuda()
    want = emb.dropout(x, 0.5, 1, residual=r)
    for bad in (math.nan, math.inf, -math.inf):
        assert torch.equal(emb.dropout(torch.where(gone, bad, x), 0.5, 1, residual=r), want)


def test_gradient_is_the_same_call():
    x, dy, u = (ref.randn((12, 90), s).cuda() for s in (1, 2, 3))
    dx = emb.dropout(dy, 0.3, 4)
    # linear in x: a difference in direction u is the gradient times u, but for the roundings of the two sums
    diff = ((emb.dropout(x + u, 0.3, 4) - emb.dropout(x, 0.3, 4)).double() * dy.double()).sum()
    assert abs(diff - (dx.double() * u.double()).sum()) <= 90 * 12 * 64 * ref.U


def test_rows_behind_the_last_and_none():
    y = torch.full((6, 33), 3.0, device="cuda")
    emb.dropout(rows(4, 33, 1, F32), 0.5, 1, out=y[:4])
    assert (y[4:] == 3.0).all()
    assert emb.dropout(torch.empty(0, 8, device="cuda"), 0.5, 1).shape == (0, 8)


def test_past_31_bits():
    x = torch.ones((1 << 16) + 3, 1 << 15, dtype=BF16, device="cuda")  # 2^31 elements and three rows
    y = emb.dropout(x, 0.5, 2, out=x)
    per = (1 << 15) // 4
    for t in (0, (1 << 16) - 1, (1 << 16) + 2):
        import numpy as np
        with np.errstate(over="ignore"):
            key = tr.mix64(np.array([2], dtype=np.uint64))
            n = np.arange(t * per + 1, (t + 1) * per + 1, dtype=np.uint64)
            bits = tr.mix64(key + n * np.uint64(tr.GAMMA)).astype("<u8").view("<u2")
        assert torch.equal((y[t] != 0).cpu(), torch.from_numpy(bits.astype(np.int64) >= tr.cut_of(0.5)))


def test_seed_on_the_device_in_a_graph_and_on_another_stream():
    x, r = rows(300, 70, 1, BF16), rows(300, 70, 2, BF16)
    seed, y, s = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty_like(x), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    emb.dropout(x, 0.3, seed, residual=r, out=y, stream=s)
    s.synchronize()
    assert torch.equal(y, emb.dropout(x, 0.3, 0, residual=r))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        emb.dropout(x, 0.3, seed, residual=r, out=y)
    for k in (1, -5, 1 << 40):
        seed.fill_(k)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, emb.dropout(x, 0.3, k, residual=r))
