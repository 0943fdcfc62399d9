"""The example that runs the table's sparse path and the dense operators together: its gradients against
the same model written with plain torch operations in 64 bits, and that training lowers the loss with
moments of 32 and of 8 bits."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def plain_loss(block, table, p, ids, targets, eps):
    N, L, H, D = block.N, block.L, block.H, block.D

    def norm(x, w, b):
        return torch.nn.functional.layer_norm(x, (D,), w, b, eps)
    x = norm(table[ids.long()], p["n1w"], p["n1b"])
    q, k, v = (t.view(N, L, H, D // H).transpose(1, 2) for t in (x @ p["qkv"]).split(D, 1))
    m = block.buckets.cpu().long()
    R = m.numel() // 2
    rel = torch.arange(L)[None, :] - torch.arange(L)[:, None]
    b = m[rel.clamp(-R, R) + R]
    bias = torch.where(b[..., None] < 0, -torch.inf, p["bias"][b.clamp(min=0)]).permute(2, 0, 1)
    a = torch.softmax(q @ k.transpose(2, 3) * (D // H) ** -0.5 + bias, 3) @ v
    x = x + a.transpose(1, 2).reshape(N * L, D) @ p["out"]
    x = x + torch.relu(norm(x, p["n2w"], p["n2b"]) @ p["up"]) @ p["down"]
    return torch.nn.functional.cross_entropy(x @ p["head"], targets.long())


def test_gradients_of_the_whole_model():
    ex = example()
    block = ex.Block(V=60, D=32, H=2, batch=3, length=20)
    ids, targets = ex.batch(block, 3)
    p64 = {k: v.detach().cpu().double().requires_grad_(True) for k, v in block.params.items()}
    table = block.table.cpu().double().requires_grad_(True)
    want = plain_loss(block, table, p64, ids.cpu(), targets.cpu(), ex.EPS)
    want.backward()
    got = block.loss(ids, targets)
    grads = dict(zip(block.params, torch.autograd.grad(got, list(block.params.values()))))
    # a chain of about a dozen fp32 operators, each some tens of roundings long: 1e-4 of a tensor's
    # largest gradient is a thousand roundings
    assert abs(got.item() - want.item()) <= 1e-5 * abs(want.item())
    for k, g in grads.items():
        ref = p64[k].grad
        assert (g.cpu().double() - ref).abs().max() <= 1e-4 * ref.abs().max(), k
    rows = torch.zeros_like(table).index_add_(0, ids.cpu().long(), block.rows.cpu().double())
    assert (rows - table.grad).abs().max() <= 1e-4 * table.grad.abs().max()


@pytest.mark.parametrize("bits", [32, 8])
def test_training_lowers_the_loss(bits):
    ex = example()
    block = ex.Block(V=200, D=64, H=4, batch=8, length=40, bits=bits)
    before = block.table.clone()
    losses = [block.step(*ex.batch(block, k % 4)).item() for k in range(40)]
    assert losses[0] > 4.5 and losses[-1] < 0.5 * losses[0]
    assert block.status.item() == 0
    used = torch.zeros(200, dtype=torch.bool)
    for k in range(4):
        used[ex.batch(block, k)[0].cpu().long()] = True
    moved = (block.table != before).any(1).cpu()
    assert torch.equal(moved, used)  # rows that no batch holds are as they were
