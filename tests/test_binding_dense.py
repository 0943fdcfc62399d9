"""The dense operators' binding without a GPU: the long way through stand-ins for tensors and the library
(tests/fake_device.py; the short way takes torch's own tensors only)."""
import pytest
import torch

import paper_2110_09132_amd as emb
from fake_device import Machine, Stream, Tensor
from paper_2110_09132_amd import dense


@pytest.fixture
def machine(monkeypatch):
    return Machine(monkeypatch, emb, dense)


X, STATS, IDS = Tensor((6, 8)), Tensor(6), Tensor(6, torch.int32)
TABLE, MAP, SCORES = Tensor((4, 2)), Tensor(7, torch.int32), Tensor((3, 2, 5, 6))
# every call that allocates, and how many tensors it makes where neither outputs nor a workspace are given
ALLOCATING = {
    "layer_norm": (lambda **kw: emb.layer_norm(X, **kw), 2),
    "layer_norm_by_ids": (lambda **kw: emb.layer_norm(X, ids=IDS, **kw), 2),
    "layer_norm_backward": (lambda **kw: emb.layer_norm_backward(X, X, STATS, STATS, **kw), 3),
    "relative_bias": (lambda **kw: emb.relative_bias(TABLE, MAP, 5, 6, **kw), 1),
    "relative_bias_backward": (lambda **kw: emb.relative_bias_backward(SCORES, MAP, 4, **kw), 2),
}


@pytest.mark.parametrize("name", ALLOCATING)
def test_what_a_call_allocates_belongs_to_its_stream(name, machine):
    """torch gives a freed tensor's memory to the next allocation of the same stream: a workspace of another
    stream would be handed out while the call's kernels still use it."""
    call, count = ALLOCATING[name]
    call(stream=Stream())
    assert len(machine.made) == count
    assert [t.under for t in machine.made] == [Stream.cuda_stream] * count
    assert machine.lib.calls[-1][1][-1] == Stream.cuda_stream
    # the outputs, not the workspace, are used on the caller's stream as well
    workspaces = [t for t in machine.made if t.dtype == torch.uint8]
    assert len(workspaces) == name.endswith("backward")
    assert all(t.used_on == ([] if t in workspaces else ["current"]) for t in machine.made)


def test_a_workspace_beside_outputs_that_are_given(machine):
    dw = Tensor(8)
    emb.layer_norm_backward(X, X, STATS, STATS, out=(X, dw, dw), stream=Stream())
    emb.relative_bias_backward(SCORES, MAP, 4, out=Tensor((4, 2)), stream=Stream())
    assert [t.under for t in machine.made] == [Stream.cuda_stream] * 2


STATUS_CALLS = {
    "layer_norm": lambda st: emb.layer_norm(X, dev_status=st),
    "layer_norm_backward": lambda st: emb.layer_norm_backward(X, X, STATS, STATS, dev_status=st),
    "relative_bias": lambda st: emb.relative_bias(TABLE, MAP, 5, 6, dev_status=st),
    "relative_bias_backward": lambda st: emb.relative_bias_backward(SCORES, MAP, 4, dev_status=st),
    "adamw_step": lambda st: emb.adamw_step([X], [X], [X], [X], 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, dev_status=st),
}


@pytest.mark.parametrize("name", STATUS_CALLS)
def test_a_status_word_that_is_none_is_refused(name, machine, monkeypatch):
    monkeypatch.setattr(emb, "_stream", lambda stream: 0)
    monkeypatch.setattr(dense, "_stream", lambda stream: 0)
    for bad in (Tensor(1, torch.int32, "cpu"), Tensor(1, torch.int64), Tensor(1), Tensor(0, torch.int32)):
        with pytest.raises(emb.EmbError, match="dev_status"):
            STATUS_CALLS[name](bad)
    assert all(n.endswith("_workspace_bytes") for n, _ in machine.lib.calls)
    STATUS_CALLS[name](Tensor(1, torch.int32))
    assert not machine.lib.calls[-1][0].endswith("_workspace_bytes")


@pytest.mark.parametrize("call", [
    lambda ws: emb.layer_norm_backward(X, X, STATS, STATS, workspace=ws, stream=Stream()),
    lambda ws: emb.relative_bias_backward(SCORES, MAP, 4, workspace=ws, stream=Stream())])
def test_a_workspace_that_is_none_is_refused(call, machine):
    # host memory, and a tensor that holds less than its elements are (one element, expanded)
    for bad in (Tensor(4096, torch.uint8, "cpu"), Tensor(4096, torch.uint8, stride=(0,))):
        with pytest.raises(emb.EmbError, match="workspace"):
            call(bad)
    assert not machine.lib.calls
    for good in (Tensor(4096, torch.uint8), Tensor((4, 256))):
        call(good)
        assert 4096 in machine.lib.calls[-1][1]  # its size in bytes


BIG, HUGE = (1 << 32) + 5, (1 << 64) + 3  # what C's 32 and 64 bits would cut to 5 and 3


@pytest.mark.parametrize("call", [
    lambda **kw: emb.layer_norm(Tensor((BIG, 8)), **kw),
    lambda **kw: emb.layer_norm(Tensor((2, BIG)), **kw),
    lambda **kw: emb.layer_norm(X, ids=Tensor(BIG, torch.int32), **kw),
    lambda **kw: emb.layer_norm_backward(Tensor((BIG, 8)), Tensor((BIG, 8)), Tensor(BIG), Tensor(BIG), **kw),
    lambda **kw: emb.layer_norm_backward(Tensor((2, BIG)), Tensor((2, BIG)), STATS, STATS, **kw),
    lambda **kw: emb.relative_bias(Tensor((BIG, 2)), MAP, 5, 6, **kw),
    lambda **kw: emb.relative_bias(Tensor((4, BIG)), MAP, 5, 6, **kw),
    lambda **kw: emb.relative_bias(TABLE, Tensor(2 * BIG + 1, torch.int32), 5, 6, **kw),
    lambda **kw: emb.relative_bias(TABLE, MAP, BIG, 6, **kw),
    lambda **kw: emb.relative_bias(TABLE, MAP, 5, BIG, **kw),
    lambda **kw: emb.relative_bias(TABLE, MAP, 5, 6, HUGE, **kw),
    lambda **kw: emb.relative_bias(TABLE, MAP, 5, 6, -HUGE, **kw),
    lambda **kw: emb.relative_bias_backward(Tensor((BIG, 2, 5, 6)), MAP, 4, **kw),
    lambda **kw: emb.relative_bias_backward(Tensor((BIG, 5, 6)), MAP, 4, **kw),
    lambda **kw: emb.relative_bias_backward(Tensor((2, BIG, 6)), MAP, 4, **kw),
    lambda **kw: emb.relative_bias_backward(Tensor((2, 5, BIG)), MAP, 4, **kw),
    lambda **kw: emb.relative_bias_backward(SCORES, Tensor(2 * BIG + 1, torch.int32), 4, **kw),
    lambda **kw: emb.relative_bias_backward(SCORES, MAP, BIG, **kw),
    lambda **kw: emb.relative_bias_backward(SCORES, MAP, 4, HUGE, **kw),
    lambda **kw: emb.adamw_step([X], [X], [X], [X], 1e-3, 0.9, 0.999, 1e-8, 0.0, HUGE, **kw),
    lambda stream: emb.adamw_coeffs(1e-3, 0.9, 0.999, 1e-8, 0.0, HUGE, torch.zeros(emb.EMB_ADAMW_COEFFS_WORDS)),
    lambda stream: emb.relative_buckets(BIG, 128),
    lambda stream: emb.relative_buckets(32, BIG),
    lambda stream: emb.layer_norm_backward_workspace_bytes(BIG, 8),
    lambda stream: emb.layer_norm_backward_workspace_bytes(8, BIG),
    lambda stream: emb.relative_bias_backward_workspace_bytes(1, 2, 3, BIG)])
def test_sizes_that_the_c_types_would_cut_are_refused(call, machine):
    with pytest.raises(emb.EmbError, match="out of range"):
        call(stream=Stream())
    assert not machine.lib.calls and not machine.made


def test_sizes_that_fit(machine):
    emb.relative_bias(TABLE, MAP, 5, 6, -(1 << 60), stream=Stream())
    emb.adamw_step([X], [X], [X], [X], 1e-3, 0.9, 0.999, 1e-8, 0.0, (1 << 63) - 1, stream=Stream())
    assert len(machine.lib.calls) == 2


def test_the_size_of_a_workspace_for_negative_sizes_is_0():
    assert emb.layer_norm_backward_workspace_bytes(-1, 8) == 0
    assert emb.relative_bias_backward_workspace_bytes(1, -2, 3, 4) == 0
