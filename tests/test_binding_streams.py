"""The binding of the tables' path without a GPU: what a call on another stream allocates belongs to that
stream, so that torch gives no allocation of the current stream memory that the call's kernels still use."""
import pytest
import torch

import paper_2110_09132_amd as emb
from fake_device import Machine, Stream, Tensor

I32 = torch.int32
T, D, V, P = 6, 8, 50, 2
IDS, NUM, OWNER, COUNT = Tensor(T, I32), Tensor(1, I32), Tensor(V, I32), Tensor((P, P + 1), I32)
ROWS, TABLE = Tensor((T, D)), Tensor((V, D))
# every call that allocates: the tensors of its outputs, and whether it makes a workspace
ALLOCATING = {
    "gather": (lambda **kw: emb.gather(TABLE, IDS, **kw), 1, 0),
    "grad_coalesce": (lambda **kw: emb.grad_coalesce(IDS, ROWS, V, **kw), 4, 1),
    "grad_coalesce_by_owner": (lambda **kw: emb.grad_coalesce_by_owner(IDS, ROWS, V, OWNER, P, **kw), 6, 1),
    "grad_coalesce_split": (lambda **kw: emb.grad_coalesce_split(IDS, IDS, ROWS, V, OWNER, P, **kw), 6, 1),
    "lookup_request": (lambda **kw: emb.lookup_request(IDS, V, OWNER, P, **kw), 5, 1),
    "exchange_simulated": (lambda **kw: emb.exchange_simulated(Tensor((P, T), I32), Tensor((P, T, D)), COUNT, **kw), 4, 0),
    "exchange_simulated_ids": (lambda **kw: emb.exchange_simulated(Tensor((P, T), I32), None, COUNT, **kw), 3, 0),
    "receive_merge": (lambda **kw: emb.receive_merge(IDS, ROWS, NUM, V, OWNER, P, **kw), 6, 1),
    "pack_by_owner": (lambda **kw: emb.pack_by_owner(IDS, ROWS, NUM, OWNER, P, **kw), 4, 1),
    "pack_by_column": (lambda **kw: emb.pack_by_column(ROWS, P, **kw), 2, 0),
    "gather_by_column": (lambda **kw: emb.gather_by_column(TABLE, V, D, P, IDS, **kw), 1, 0),
    "assemble_by_column": (lambda **kw: emb.assemble_by_column(ROWS, T, D, P, **kw), 1, 0),
}


@pytest.mark.parametrize("name", ALLOCATING)
def test_what_a_call_allocates_belongs_to_its_stream(name, monkeypatch):
    call, outputs, workspaces = ALLOCATING[name]
    machine = Machine(monkeypatch, emb)
    out = call(stream=Stream())
    made = machine.made
    assert len(made) == outputs + workspaces
    assert [t.under for t in made] == [Stream.cuda_stream] * len(made)
    returned = [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]
    assert len(returned) == outputs
    assert all(t.used_on == (["current"] if any(t is r for r in returned) else []) for t in made)
    assert machine.lib.calls[-1][1][-1] == Stream.cuda_stream
