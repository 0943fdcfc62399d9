"""The relative position bias at the ends of its sizes: the largest map, with differences near and past
both of its ends."""
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
