"""The gradient of layer norm for rows so wide that the columns' sums take more than one launch; rows looked up
in a table of bfloat16 by a batch of ids."""
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


@pytest.mark.parametrize("D", [96, 512, 1024])
def test_looked_up_rows_of_bf16_tables(D):
    V, T = 3000, 5000
    table = ref.randn((V, D), 1).to(torch.bfloat16).cuda()
    w, b = (1 + ref.randn((D,), 2, 0.2)).cuda(), ref.randn((D,), 3, 0.2).cuda()
    ids = torch.randint(0, V, (T,), generator=ref.gen(4), dtype=torch.int32)
    x, st = table.cpu()[ids.long()], emb.new_status()
    dy = ref.randn((T, D), 5, 0.1).to(torch.bfloat16).cuda()
    for out_dtype in (torch.float32, torch.bfloat16):
        y, mean, rstd = emb.layer_norm(table, w, b, ids=ids.cuda(), out_dtype=out_dtype, dev_status=st)
        r = ref.layer_norm(x, w, b, 1e-5)
        ref.assert_within(y, r["y"], r["tol"] + ref.rounding(out_dtype, r["y"]), "y")
        g = dy.to(out_dtype)
        dx, dw, db = emb.layer_norm_backward(g, table, mean, rstd, w, ids=ids.cuda(), dev_status=st)
        r = ref.layer_norm_backward(g, x, mean, rstd, w)
        ref.assert_within(dx, r["dx"], r["dx_tol"] + ref.rounding(out_dtype, r["dx"]), "dx")
        ref.assert_within(dw, r["dw"], r["dw_tol"], "dweight")
        ref.assert_within(db, r["db"], r["db_tol"], "dbias")
    assert st.item() == 0
