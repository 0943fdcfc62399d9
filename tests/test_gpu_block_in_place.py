"""emb_block_norm and its gradient in place (h over x, y over branch; dx over dh, dbranch over dy) against the same call
with buffers of its own, bit for bit: every combination of the two norms, whose sums' barriers are there or not, at widths
whose cut vector begins another wave than the one before it, one to eight waves per row.  (tests/test_block_order_host.py
has the orders in which the waves may get there.)"""
import pytest
import torch

import paper_2110_09132_amd as emb
from test_gpu_block_norm import BF16, EPS, F32, case, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("post,pre", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("st,bt,D", [(F32, F32, 1025), (F32, F32, 1281), (F32, BF16, 2049), (F32, BF16, 3333), (F32, F32, 8193),
                                     (BF16, BF16, 1025), (BF16, BF16, 1537), (BF16, BF16, 2049), (BF16, BF16, 4097),
                                     (BF16, BF16, 8199), (F32, F32, 513), (F32, F32, 20001)])
def test_in_place(st, bt, D, post, pre):
    T = 700
    x, branch, c = case(T, D, st, bt, post=post, pre=pre)
    out = emb.block_norm(x, branch, eps=EPS, **c)
    x2, b2 = x.clone(), branch.clone()
    stats = [None if s is None else torch.empty_like(s) for s in out[2:]]
    got = emb.block_norm(x2, b2, eps=EPS, out=(x2, b2 if pre else None, *stats), **c)
    for a, b in zip(got, out):
        assert b is None or torch.equal(a, b)
    dh, dy = rows(T, D, 11, st, 0.1), rows(T, D, 12, bt, 0.1) if pre else None
    want = emb.block_norm_backward(dh, dy, out[0], branch, *out[2:], **c)
    rest = [None if t is None else torch.empty_like(t) for t in want[2:]]
    db = torch.empty_like(branch) if dy is None else dy
    got = emb.block_norm_backward(dh, dy, out[0], branch, *out[2:], out=(dh, db, *rest), **c)
    for a, b in zip(got, want):
        assert b is None or torch.equal(a, b)
