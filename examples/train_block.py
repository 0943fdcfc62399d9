"""Training steps of a small causal language model around one embedding table: the sparse path of the
table and the dense operators beside it, together as a program uses them.

  lookup and layer norm in one pass (layer_norm with ids) -> attention, its scores with a learned relative
  position bias (relative_bias) -> layer norm -> two-layer perceptron -> cross entropy of the next token

Backward, the lookup's gradient rows go to the coalesce and the row-wise Adam of the table; everything else
(projections, norm parameters, the bias table) takes one AdamW step, with moments in 32 or in 8 bits.

With --fused, the attention's output, dropped and gated, joins the residual stream in one pass with the norm that
follows (block_norm), the perceptron's is dropped and added in one (dropout), and the loss is taken over the
vocabulary without its logits (vocab_loss).

  python examples/train_block.py [--steps 60] [--bits 8] [--fused [--dropout 0.1]]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2110_09132_amd as emb  # noqa: E402

EPS = 1e-5
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8)


class LookupNorm(torch.autograd.Function):
    """Layer norm of table rows by id; the rows' gradient is left in `rows`, for the coalesce."""

    @staticmethod
    def forward(ctx, weight, bias, table, ids, rows, status):
        y, mean, rstd = emb.layer_norm(table, weight, bias, EPS, ids=ids, dev_status=status)
        ctx.save_for_backward(weight, table, ids, mean, rstd)
        ctx.rows = rows
        return y

    @staticmethod
    def backward(ctx, dy):
        weight, table, ids, mean, rstd = ctx.saved_tensors
        dw, db = torch.empty_like(weight), torch.empty_like(weight)
        emb.layer_norm_backward(dy.contiguous(), table, mean, rstd, weight, ids=ids, out=(ctx.rows, dw, db))
        return dw, db, None, None, None, None


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        y, mean, rstd = emb.layer_norm(x, weight, bias, EPS)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        return emb.layer_norm_backward(dy.contiguous(), x, mean, rstd, weight)


class PositionBias(torch.autograd.Function):
    """The scores [N, H, L, L] with the bias of every head added; masked pairs become -infinity."""

    @staticmethod
    def forward(ctx, scores, table, buckets):
        ctx.save_for_backward(buckets)
        ctx.num_buckets = table.shape[0]
        return scores + emb.relative_bias(table, buckets, *scores.shape[2:])

    @staticmethod
    def backward(ctx, d):
        buckets, = ctx.saved_tensors
        return d, emb.relative_bias_backward(d.contiguous(), buckets, ctx.num_buckets), None


class Join(torch.autograd.Function):
    """(x + gate dropout(branch), its layer norm)."""

    @staticmethod
    def forward(ctx, x, branch, gate, weight, bias, p, seed):
        h, y, _, stats = emb.block_norm(x, branch, gate=gate, post=None, pre=(weight, bias), eps=EPS, p=p, seed=seed)
        ctx.save_for_backward(h, branch, stats, gate, weight, bias)
        ctx.drop = dict(p=p, seed=seed)
        return h, y

    @staticmethod
    def backward(ctx, dh, dy):
        h, branch, stats, gate, weight, bias = ctx.saved_tensors
        dx, dbranch, dgate, _, _, dw, db = emb.block_norm_backward(
            dh.contiguous(), dy.contiguous(), h, branch, None, stats, gate=gate, post=None, pre=(weight, bias), **ctx.drop)
        return dx, dbranch, dgate, dw, db, None, None


class DropAdd(torch.autograd.Function):
    """x + dropout(branch)."""

    @staticmethod
    def forward(ctx, x, branch, p, seed):
        ctx.drop = p, seed
        return emb.dropout(branch, p, seed, residual=x)

    @staticmethod
    def backward(ctx, d):
        return d, emb.dropout(d.contiguous(), *ctx.drop), None, None


class VocabLoss(torch.autograd.Function):
    """Mean cross entropy over the rows of `head` [V, D]."""

    @staticmethod
    def forward(ctx, x, head, targets, status):
        loss, lse = emb.vocab_loss(x, head, targets, dev_status=status)
        ctx.save_for_backward(x, head, targets, lse)
        return loss.mean()

    @staticmethod
    def backward(ctx, d):
        x, head, targets, lse = ctx.saved_tensors
        dx, dhead = emb.vocab_loss_backward((d / x.shape[0]).view(1), x, head, targets, lse)
        return dx, dhead, None, None


class Block:
    def __init__(self, V, D, H, batch, length, bits=32, owners=2, seed=0, fused=False, dropout=0.0):
        g = torch.Generator().manual_seed(seed)
        normal = lambda *shape, s=0.05: (torch.randn(shape, generator=g) * s).cuda()  # noqa: E731
        self.V, self.D, self.H, self.N, self.L, self.P, self.t = V, D, H, batch, length, owners, 0
        self.fused, self.dropout = fused, dropout
        self.table = normal(V, D, s=1.0)
        self.m, self.v = torch.zeros_like(self.table), torch.zeros_like(self.table)
        self.row_owner = (torch.arange(V, dtype=torch.int32) % owners).cuda()
        self.buckets = emb.relative_buckets(8, 16, causal=True)
        one, zero = torch.ones(D).cuda(), torch.zeros(D).cuda()
        self.params = {"n1w": one.clone(), "n1b": zero.clone(), "qkv": normal(D, 3 * D), "out": normal(D, D),
                       "bias": normal(8, H), "n2w": one.clone(), "n2b": zero.clone(), "up": normal(D, 4 * D),
                       "down": normal(4 * D, D), "head": normal(D, V)}
        if fused:
            self.params["head"], self.params["gate"] = normal(V, D), one.clone()
        for p in self.params.values():
            p.requires_grad_(True)
        ps = [p.detach() for p in self.params.values()]
        if bits == 8:
            self.exp_avgs, self.exp_avg_sqs, self.scales = map(list, zip(*(emb.adamw_state8(p) for p in ps)))
        else:
            self.exp_avgs, self.exp_avg_sqs = ([torch.zeros_like(p) for p in ps] for _ in range(2))
            self.scales = None
        # kept between the steps: the rows' gradient, the coalesce's workspace, the device status
        T = batch * length
        self.rows = torch.empty((T, D), device="cuda")
        self.workspace = emb.new_workspace(emb.grad_coalesce_workspace_bytes(T, V, D))
        self.status = emb.new_status()

    def loss(self, ids, targets):
        """Mean cross entropy of targets [N * L] after ids [N * L]."""
        p, N, L, H, D = self.params, self.N, self.L, self.H, self.D
        x = LookupNorm.apply(p["n1w"], p["n1b"], self.table, ids, self.rows, self.status)
        q, k, v = (t.view(N, L, H, D // H).transpose(1, 2).contiguous() for t in (x @ p["qkv"]).split(D, 1))
        scores = q @ k.transpose(2, 3).contiguous() * (D // H) ** -0.5
        a = torch.softmax(PositionBias.apply(scores, p["bias"], self.buckets), 3) @ v
        if self.fused:
            x, h = Join.apply(x, a.transpose(1, 2).reshape(N * L, D) @ p["out"], p["gate"], p["n2w"], p["n2b"],
                              self.dropout, 2 * self.t)
            x = DropAdd.apply(x, torch.relu(h @ p["up"]) @ p["down"], self.dropout, 2 * self.t + 1)
            return VocabLoss.apply(x, p["head"], targets, self.status)
        x = x + a.transpose(1, 2).reshape(N * L, D) @ p["out"]
        h = Norm.apply(x, p["n2w"], p["n2b"])
        x = x + torch.relu(h @ p["up"]) @ p["down"]
        return torch.nn.functional.cross_entropy(x @ p["head"], targets.long())

    def step(self, ids, targets):
        """One training step; returns the loss (on the device)."""
        self.t += 1
        ps = list(self.params.values())
        loss = self.loss(ids, targets)
        grads = torch.autograd.grad(loss, ps)
        send_ids, _, rows, _, offsets, _ = emb.grad_coalesce_by_owner(
            ids, self.rows, self.V, self.row_owner, self.P, workspace=self.workspace, dev_status=self.status)
        emb.sparse_adam_apply(self.table, self.m, self.v, send_ids, rows, offsets, self.P, 0, self.P, **HYPER,
                              step=self.t, dev_status=self.status)
        # the gradients' norm is clipped at 1 without waiting for it
        norm = torch.stack([g.square().sum() for g in grads]).sum().sqrt()
        emb.adamw_step([p.detach() for p in ps], [g.contiguous() for g in grads], self.exp_avgs, self.exp_avg_sqs,
                       weight_decay=0.01, step=self.t, scales=self.scales, grad_scale=(1.0 / norm).clamp(max=1.0).view(1),
                       dev_status=self.status, **HYPER)
        return loss.detach()


def batch(block, seed):
    """Sequences that repeat themselves after eight tokens: the model has to look back."""
    g = torch.Generator().manual_seed(seed)
    head = torch.randint(0, block.V, (block.N, 8), generator=g, dtype=torch.int32)
    ids = head.repeat(1, block.L // 8 + 1)[:, :block.L + 1]
    return ids[:, :-1].reshape(-1).cuda(), ids[:, 1:].reshape(-1).cuda()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--bits", type=int, choices=(8, 32), default=32)
    ap.add_argument("--fused", action="store_true")
    ap.add_argument("--dropout", type=float, default=0.0)
    a = ap.parse_args()
    block = Block(V=500, D=128, H=4, batch=16, length=48, bits=a.bits, fused=a.fused, dropout=a.dropout)
    for k in range(a.steps):
        loss = block.step(*batch(block, k % 8))
        if k % 10 == 0 or k == a.steps - 1:
            print(f"step {k + 1}: loss {loss.item():.4f}", flush=True)
    if block.status.item():
        raise SystemExit(f"device status {block.status.item()}")


if __name__ == "__main__":
    main()
