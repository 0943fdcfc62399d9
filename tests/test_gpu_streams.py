"""What a call allocates when `stream` is another stream than the current one: outputs and workspaces come
from that stream's part of torch's allocator, so that no allocation of the current stream is given memory
that the call's kernels still use."""
import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb

pytestmark = pytest.mark.gpu


def owner(t):
    """The stream that the memory of a tensor belongs to."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no segment holds the tensor")


def reserved(stream):
    return sum(seg["total_size"] for seg in torch.cuda.memory_snapshot() if seg["stream"] == stream.cuda_stream)


def check(call, workspace_bytes, eager):
    """call(side) returns the outputs; workspace_bytes: of the workspace that it allocates."""
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    had = reserved(side)
    outs = call(side)
    # as much memory of the current stream as the call took, written at once
    for n in {workspace_bytes, *(t.numel() * t.element_size() for t in outs)} - {0}:
        torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
    assert all(owner(t) == side.cuda_stream for t in outs)
    assert reserved(side) - had >= workspace_bytes + sum(t.numel() * t.element_size() for t in outs)
    torch.cuda.synchronize()
    for a, b in zip(outs, eager):
        assert torch.equal(a, b)


def test_layer_norm():
    T, D = 5000, 1024
    x, w = ref.randn((T, D), 1).cuda(), ref.randn((D,), 2).cuda()
    dy = ref.randn((T, D), 3).cuda()
    eager = emb.layer_norm(x, w)
    check(lambda s: emb.layer_norm(x, w, stream=s), 0, eager)
    check(lambda s: emb.layer_norm_backward(dy, x, *eager[1:], w, stream=s),
          emb.layer_norm_backward_workspace_bytes(T, D), emb.layer_norm_backward(dy, x, *eager[1:], w))


def test_relative_bias():
    H, Q, K = 8, 700, 900
    t, m = ref.randn((32, H), 1).cuda(), emb.relative_buckets(32, 128)
    g = ref.randn((1, H, Q, K), 2).cuda()
    check(lambda s: [emb.relative_bias(t, m, Q, K, stream=s)], 0, [emb.relative_bias(t, m, Q, K)])
    check(lambda s: [emb.relative_bias_backward(g, m, 32, stream=s)],
          emb.relative_bias_backward_workspace_bytes(1, H, Q, K), [emb.relative_bias_backward(g, m, 32)])


def test_the_tables_path():
    T, D, V, P = 3000, 256, 700, 4
    table, g = ref.randn((V, D), 1).cuda(), ref.randn((T, D), 2).cuda()
    ids = torch.randint(0, V, (T,), generator=ref.gen(3), dtype=torch.int32).cuda()
    row_owner = (torch.arange(V, dtype=torch.int32) % P).cuda()
    U = emb.grad_coalesce(ids, g, V)[3].item()

    def used(out):  # the entries that are meaningful
        uniq, seg, rows, *rest = out
        return [uniq[:U], seg[:U + 1], rows[:U], *rest]
    check(lambda s: [emb.gather(table, ids, stream=s)], 0, [emb.gather(table, ids)])
    check(lambda s: used(emb.grad_coalesce(ids, g, V, stream=s)), emb.grad_coalesce_workspace_bytes(T, V, D),
          used(emb.grad_coalesce(ids, g, V)))
    check(lambda s: used(emb.grad_coalesce_by_owner(ids, g, V, row_owner, P, stream=s)),
          emb.grad_coalesce_workspace_bytes(T, V, D), used(emb.grad_coalesce_by_owner(ids, g, V, row_owner, P)))


def test_a_stream_known_by_its_handle():
    class Handle:  # what the binding asks of a stream
        def __init__(self, stream):
            self.cuda_stream = stream.cuda_stream
    x = ref.randn((400, 300), 1).cuda()
    check(lambda s: emb.layer_norm(x, stream=Handle(s)), 0, emb.layer_norm(x))
