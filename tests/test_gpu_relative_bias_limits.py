"""The relative position bias at the ends of its sizes: the largest map, with differences near and past
both of its ends; more rows, places and buckets than one launch takes."""
import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def largest_map():
    """R = 2^30 - 1: bucket 0 in the middle; five places at each end have buckets of their own."""
    m = torch.zeros((1 << 31) - 1, dtype=torch.int32, device="cuda")
    m[:5] = torch.arange(1, 6, device="cuda")
    m[-5:] = torch.arange(6, 11, device="cuda")
    yield m
    del m
    torch.cuda.empty_cache()


@pytest.mark.parametrize("side", [-1, 1])
@pytest.mark.parametrize("past", [-6000, -70, -20, 0, 20, 1 << 30, 1 << 40])
def test_the_largest_map(largest_map, side, past):
    R, H, Q, K, B = (1 << 30) - 1, 2, 30, 50, 11
    q0 = -side * (R + past)  # the differences lie around side * (R + past)
    rel = torch.arange(K)[None, :] - (torch.arange(Q)[:, None] + q0)
    at = rel.clamp(-R, R) + R
    bucket = torch.where(at < 5, at + 1, torch.where(at > 2 * R - 5, at - (2 * R - 5) + 5, 0))
    t, g = ref.randn((B, H), 1), ref.randn((1, H, Q, K), 2)
    got = emb.relative_bias(t.cuda(), largest_map, Q, K, q0)
    assert torch.equal(got.cpu(), t[bucket].permute(2, 0, 1))
    d = emb.relative_bias_backward(g.cuda(), largest_map, B, q0)
    flat = g.double()[0].reshape(H, -1)
    for b in range(B):
        here = flat[:, bucket.reshape(-1) == b]
        ref.assert_within(d[b], here.sum(1), here.shape[1] * ref.U * here.abs().sum(1) + ref.TINY, f"bucket {b}")


def test_more_rows_than_one_launch_takes():
    # tiles of 64 rows of 64 columns, 2^20 tiles to a launch: 2^26 rows, where the differences are small
    at, K, B = 1 << 26, 64, 32
    Q, q0 = at + 70, -at
    t, m = ref.randn((B, 1), 1), emb.relative_buckets(B, 128)
    got = emb.relative_bias(t.cuda(), m, Q, K, q0)
    assert torch.equal(got[:, -400:].cpu(), ref.relative_bias(t, m, 400, K, q0 + Q - 400, torch.float32))
    for part in got[0, :-400].split(1 << 24):  # keys far to the right: one bucket
        assert (part == t[B - 1, 0]).all()


def test_more_places_than_one_launch_takes():
    # 2^26 places to a launch; whole numbers, so that every sum is exact
    K, B, R = (1 << 26) + 1000, 6, (1 << 26) + 2000
    m = torch.zeros(2 * R + 1, dtype=torch.int32, device="cuda")
    g = torch.zeros((1, 1, 1, K), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 63, 64, 12345, (1 << 26) - 1, 1 << 26, (1 << 26) + 999], device="cuda")  # keys
    bucket = torch.tensor([1, 2, 3, 4, 5, 1, 2], dtype=torch.int32, device="cuda")
    m[R + at] = bucket
    g[..., at] = torch.arange(1, 8, device="cuda").to(torch.bfloat16)
    g[..., 1000:1100] = 1.0  # bucket 0
    st = emb.new_status()
    got = emb.relative_bias_backward(g, m, B, dev_status=st)
    assert got[:, 0].tolist() == [100, 1 + 6, 2 + 7, 3, 4, 5]
    assert st.item() == 0
    m[R + K - 1] = B  # the last place that occurs, in the last launch
    emb.relative_bias_backward(g, m, B, dev_status=st)
    assert st.item() == emb.EMB_DEV_BUCKET_OUT_OF_RANGE


@pytest.mark.parametrize("R", [40, 1000])  # the sums in one launch, or the buckets in several of 2^22
def test_more_buckets_than_one_launch_takes(R):
    K, B = 2 * R + 1, (1 << 22) + 5
    m = torch.zeros(2 * R + 1, dtype=torch.int32, device="cuda")
    bucket = torch.tensor([1, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, (1 << 22) + 4, 2], dtype=torch.int32, device="cuda")
    at = torch.tensor([0, 5, 7, 11, 2 * R - 1, 2 * R], device="cuda")
    m[at] = bucket
    g = torch.ones((1, 1, 1, K), device="cuda")
    g[..., at] = torch.arange(2.0, 8.0, device="cuda")
    got = emb.relative_bias_backward(g, m, B, q0=R)
    want = torch.zeros((B, 1), device="cuda")
    want[bucket.long(), 0] = torch.arange(2.0, 8.0, device="cuda")
    want[0] = K - 6
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_entries_without_a_pair_set_no_flag(dtype):
    R, B = 300, 4
    for Q, K, q0 in ((5, 8, 0), (1, 40, 39), (100, 3, -20), (70, 700, 100)):
        low, high = -(Q - 1) - q0 + R, K - 1 - q0 + R  # places of the first and the last difference
        m = torch.zeros(2 * R + 1, dtype=torch.int32)
        m[:max(low, 0)] = B
        m[high + 1:] = B
        t, g = ref.randn((B, 2), 1).cuda(), ref.randn((1, 2, Q, K), 2).to(dtype).cuda()
        for end in (None, max(low, 0), min(high, 2 * R)):
            n = m.clone()
            if end is not None:
                n[end] = B
            for call in (lambda st: emb.relative_bias(t, n.cuda(), Q, K, q0, out_dtype=dtype, dev_status=st),
                         lambda st: emb.relative_bias_backward(g, n.cuda(), B, q0, dev_status=st)):
                st = emb.new_status()
                call(st)
                assert st.item() == (0 if end is None else emb.EMB_DEV_BUCKET_OUT_OF_RANGE)
