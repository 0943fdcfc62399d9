"""The gradient of layer norm for rows so wide that the columns' sums take more than one launch."""
import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb

pytestmark = pytest.mark.gpu


def test_rows_of_more_columns_than_one_launch_sums():
    T, D = 2, (1 << 26) + 5  # a launch sums 2^25 of the 2 D columns
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn((T, D), generator=g, device="cuda") for _ in range(2))
    mean, rstd = torch.tensor([[0.25, -0.5], [0.75, 1.5]], device="cuda")
    out = (None, torch.full((D,), 7.0, device="cuda"), torch.full((D,), 7.0, device="cuda"))
    _, dw, db = emb.layer_norm_backward(dy, x, mean, rstd, out=out)
    terms = dy.double() * ((x.double() - mean.double()[:, None]) * rstd.double()[:, None])
    assert ((dw.double() - terms.sum(0)).abs() <= (T + 4) * ref.U * terms.abs().sum(0) + ref.TINY).all()
    assert ((db.double() - dy.double().sum(0)).abs() <= T * ref.U * dy.double().abs().sum(0) + ref.TINY).all()
