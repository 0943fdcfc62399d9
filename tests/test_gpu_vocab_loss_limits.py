"""emb_vocab_loss and emb_vocab_loss_backward where only one of their ways, or only the end of a range, goes wrong: tables
with entries that are not finite beside tokens without a target, at the sizes of every way."""
import math

import pytest
import torch

import paper_2110_09132_amd as emb
from test_gpu_vocab_loss import BF16, F32, case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T", [1, 16, 40, 64, 65, 300])
def test_no_gradient_without_a_target_whatever_the_table_holds(T, bad, dtype):
    x, w, ids = case(T, 600, 96, dtype)
    ids[T // 2] = -1
    if T > 1:
        ids[T // 3] = 600  # no row: counts as none
    w[77, 5] = bad
    gone = (ids < 0) | (ids >= 600)
    loss, lse = emb.vocab_loss(x, w, ids)
    assert (loss[gone] == 0).all() and (lse[gone] == 0).all()
    for d in (torch.ones(T, device="cuda"), torch.ones(1, device="cuda")):
        dx, _ = emb.vocab_loss_backward(d, x, w, ids, lse)
        assert (dx[gone] == 0).all()
        none = torch.full_like(ids, -1)
        dx, dw = emb.vocab_loss_backward(d, x, w, none, lse)
        assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("each", [False, True])
def test_gradient_of_logits_far_from_zero(each):
    """All logits 2^20, exactly, and lse what the caller gives, 2^20 + 6: the gradient's exponent is the difference of the
    two, -6 for every entry, so that g = dloss (exp(-6) - [v == target]), rounded to bf16 once (2^-8), and dx and dtable a
    second time; the exponential is good to 4 units of 2^-24, and so are the sums of up to 2.2 (V + 8) of them."""
    T, V, D = 90, 520, 64
    x, w = torch.zeros(T, D, dtype=BF16, device="cuda"), torch.zeros(V, D, dtype=BF16, device="cuda")
    x[:, 0], w[:, 0] = 1024.0, 1024.0
    ids = (torch.arange(T, device="cuda") * 5 % 400).int()  # no token's target from 446 on
    lse = torch.full((T,), 2.0 ** 20 + 6.0, device="cuda")
    d = torch.full((T,) if each else (1,), 0.75, device="cuda")
    dx, dw = emb.vocab_loss_backward(d, x, w, ids, lse)
    p, rel = math.exp(-6.0), 2 * 2.0 ** -8 + 2.2 * (V + 16) * 2.0 ** -24
    want = 0.75 * p * T * 1024.0
    got = dw[450:, 0].double()
    assert ((got - want).abs() <= 1.01 * rel * want).all(), (got / want - 1).abs().max().item()
    want = 0.75 * 1024.0 * (p * V - 1.0)   # each of the V - 1 and the target's within 2^-8 of its size
    got = dx[:, 0].double()
    tol = 1.01 * rel * 0.75 * 1024.0 * (p * V + 1.0)
    assert ((got - want).abs() <= tol).all(), (got - want).abs().max().item() / tol
    assert (dx[:, 1:] == 0).all() and (dw[:, 1:] == 0).all()


@pytest.mark.parametrize("T", [3, 70])
def test_the_largest_vocabulary(T):
    """2^31 - 1 entries, all the same row: every logit is 8, exactly.  The sums of ones are exact in a lane and rounded in
    the joins (16 at most), then come the logarithm and the sum with 8."""
    V, D = (1 << 31) - 1, 64
    x = torch.full((T, D), 0.25, dtype=BF16, device="cuda")
    w = torch.full((1, D), 0.5, dtype=BF16, device="cuda").expand(V, D)
    ids = torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    ids[0], ids[1] = 0, -1
    loss, lse = emb.vocab_loss(x, w, ids)
    live = ids >= 0
    for t, want in ((lse, 8.0 + math.log(V)), (loss, math.log(V))):
        assert ((t[live].double() - want).abs() <= (16 + 8 + 4 * 30) * 2.0 ** -24).all()
        assert (t[~live] == 0).all()
