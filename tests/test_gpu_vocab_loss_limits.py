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
