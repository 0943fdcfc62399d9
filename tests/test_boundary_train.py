"""The C calls of dropout, the norms around a block and the cross entropy without a GPU: every bad argument is refused
on the host, before anything is enqueued (the addresses passed here are never read); the structs' layout; and the
binding's own checks through stand-ins."""
import ctypes

import pytest
import torch

import paper_2110_09132_amd as emb
from fake_device import Machine, Stream, Tensor
from paper_2110_09132_amd import train
from test_abi_layout import c_layout

FAKE, ODD, NULL = 4096, 4097, None
NAN, INF = float("nan"), float("inf")
BAD = emb.EMB_ERR_INVALID_ARG
BF16 = torch.bfloat16


def test_dropout_validation():
    def call(x=FAKE, dt=0, ldx=8, T=4, D=8, p=0.1, seed=1, sd=NULL, r=NULL, ldr=0, y=FAKE, ldy=8):
        return emb.lib.emb_dropout(x, dt, ldx, T, D, p, seed, sd, r, ldr, y, ldy, NULL)
    assert call(T=0, x=NULL, y=NULL) == emb.EMB_OK
    for bad in (dict(T=-1), dict(T=1 << 30), dict(D=0), dict(D=1 << 28), dict(dt=2), dict(ldx=-1), dict(ldy=7),
                dict(p=-0.1), dict(p=1.0), dict(p=NAN), dict(x=NULL), dict(y=NULL), dict(x=ODD), dict(y=ODD),
                dict(x=ODD, dt=1), dict(r=ODD), dict(r=FAKE, ldr=-1), dict(sd=FAKE + 4)):
        assert call(**bad) == BAD, bad


def block_args(**kw):
    a = dict(T=4, D=8, x=FAKE, ldx=8, branch=FAKE, ldb=8, h=FAKE, ldh=8, y=FAKE, ldy=8, post_stats=FAKE, pre_stats=FAKE,
             alpha=1.0, eps=1e-5)
    return emb.BlockNormArgs(**{**a, **kw})


def test_block_norm_validation():
    def call(**kw):
        args = block_args(**kw)
        return emb.lib.emb_block_norm(ctypes.addressof(args), NULL)
    assert emb.lib.emb_block_norm(NULL, NULL) == BAD
    assert call(T=0, x=NULL, branch=NULL, h=NULL, y=NULL) == emb.EMB_OK
    for bad in (dict(T=-1), dict(D=0), dict(stream_dtype=2), dict(dtype=2), dict(stream_dtype=1, dtype=0), dict(ldx=-1),
                dict(ldb=-1), dict(ldh=7), dict(ldy=7), dict(gate_rows=-1), dict(eps=-1.0), dict(eps=NAN),
                dict(alpha=INF), dict(alpha=NAN), dict(p=1.0), dict(p=-1.0), dict(seed_dev=FAKE + 4), dict(x=NULL),
                dict(branch=NULL), dict(h=NULL), dict(y=NULL), dict(x=ODD), dict(branch=ODD, dtype=1), dict(h=ODD),
                dict(y=ODD), dict(gate=ODD), dict(post_weight=ODD), dict(post_bias=ODD), dict(pre_weight=ODD),
                dict(pre_bias=ODD), dict(post_stats=ODD), dict(pre_stats=ODD)):
        assert call(**bad) == BAD, bad


def test_block_norm_backward_validation():
    size = emb.lib.emb_block_norm_backward_workspace_bytes
    need = size(4, 8, 0)
    assert need > 0 and need % 256 == 0
    assert size(-1, 8, 0) == 0 and size(4, 0, 0) == 0 and size(4, 8, -1) == 0

    def call(**kw):
        a = dict(T=4, D=8, dh=FAKE, lddh=8, dy=FAKE, lddy=8, h=FAKE, ldh=8, branch=FAKE, ldb=8, post_stats=FAKE,
                 pre_stats=FAKE, alpha=1.0, dx=FAKE, lddx=8, dbranch=FAKE, lddb=8, dgate=FAKE, dpost_weight=FAKE,
                 dpost_bias=FAKE, dpre_weight=FAKE, dpre_bias=FAKE, workspace=FAKE, workspace_bytes=need)
        args = emb.BlockNormGradArgs(**{**a, **kw})
        return emb.lib.emb_block_norm_backward(ctypes.addressof(args), NULL)
    outs = ("dx", "dbranch", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias")
    assert emb.lib.emb_block_norm_backward(NULL, NULL) == BAD
    for bad in (dict(T=-1), dict(D=0), dict(stream_dtype=1, dtype=0), dict(dtype=3), dict(lddh=-1), dict(lddy=-1),
                dict(ldh=-1), dict(ldb=-1), dict(lddx=7), dict(lddb=7), dict(gate_rows=-1), dict(alpha=NAN), dict(p=1.0),
                dict(post_stats=NULL), dict(pre_stats=NULL), dict.fromkeys(outs), dict(branch=NULL), dict(dy=NULL),
                dict(h=NULL), dict(dy=ODD), dict(h=ODD), dict(dh=ODD), dict(branch=ODD), dict(dx=ODD), dict(dbranch=ODD),
                dict(dgate=ODD), dict(dpost_weight=ODD), dict(dpre_bias=ODD), dict(gate=ODD), dict(post_weight=ODD),
                dict(pre_weight=ODD), dict(workspace=NULL), dict(workspace=FAKE + 64)):
        assert call(**bad) == BAD, bad
    assert call(workspace_bytes=need - 1) == emb.EMB_ERR_WORKSPACE


def test_vocab_loss_validation():
    size = emb.lib.emb_vocab_loss_workspace_bytes
    need = size(4, 100, 8, 0)
    assert need > 0 and need % 256 == 0
    for a in ((-1, 100, 8, 0), ((1 << 22) + 1, 100, 8, 0), (4, 0, 8, 0), (4, 1 << 31, 8, 0), (4, 100, 0, 0),
              (4, 100, (1 << 16) + 1, 0), (4, 100, 8, 2)):
        assert size(*a) == 0, a

    def call(x=FAKE, dt=0, ldx=8, w=FAKE, ldw=8, T=4, V=100, D=8, t=FAKE, e=0.0, loss=FAKE, lse=FAKE, ws=FAKE, wsb=need):
        return emb.lib.emb_vocab_loss(x, dt, ldx, w, ldw, T, V, D, t, e, loss, lse, ws, wsb, NULL, NULL)
    assert call(T=0, x=NULL, w=NULL, t=NULL, loss=NULL, lse=NULL, ws=NULL) == emb.EMB_OK
    for bad in (dict(T=-1), dict(T=(1 << 22) + 1), dict(V=0), dict(V=1 << 31), dict(D=0), dict(D=(1 << 16) + 1),
                dict(dt=2), dict(ldx=-1), dict(ldw=-1), dict(e=-0.1), dict(e=1.0), dict(e=NAN), dict(x=NULL), dict(w=NULL),
                dict(t=NULL), dict(loss=NULL), dict(lse=NULL), dict(ws=NULL), dict(ws=FAKE + 64), dict(x=ODD), dict(w=ODD),
                dict(t=ODD), dict(loss=ODD), dict(lse=ODD), dict(x=ODD, dt=1)):
        assert call(**bad) == BAD, bad
    assert call(wsb=need - 1) == emb.EMB_ERR_WORKSPACE


def test_vocab_loss_backward_validation():
    size = emb.lib.emb_vocab_loss_backward_workspace_bytes
    need = size(4, 100, 8, 1)
    assert need > 0 and need % 256 == 0 and size(4, 100, 8, 7) == 0
    assert all(call(0, 100, 8, dt) >= 0 for call in (size, emb.lib.emb_vocab_loss_workspace_bytes) for dt in (0, 1))
    # gradients of the logits never take more than some GiB, whatever the vocabulary
    assert all(size(T, (1 << 31) - 1, 1, dt) < 24 << 30 for T in (1, 64, 65, 1 << 22) for dt in (0, 1))

    def call(d=FAKE, step=1, x=FAKE, dt=1, ldx=8, w=FAKE, ldw=8, T=4, V=100, D=8, t=FAKE, e=0.0, lse=FAKE, dx=FAKE, lddx=8,
             dw=FAKE, lddw=8, ws=FAKE, wsb=need):
        return emb.lib.emb_vocab_loss_backward(d, step, x, dt, ldx, w, ldw, T, V, D, t, e, lse, dx, lddx, dw, lddw, ws, wsb,
                                               NULL, NULL)
    for bad in (dict(T=-1), dict(V=0), dict(D=0), dict(dt=2), dict(ldx=-1), dict(ldw=-1), dict(e=1.0), dict(step=2),
                dict(step=-1), dict(dx=NULL, dw=NULL), dict(lddx=7), dict(lddw=7), dict(d=NULL), dict(x=NULL), dict(w=NULL),
                dict(t=NULL), dict(lse=NULL), dict(ws=NULL), dict(ws=FAKE + 64), dict(x=ODD), dict(w=ODD), dict(dx=ODD),
                dict(dw=ODD), dict(d=ODD), dict(t=ODD), dict(lse=ODD)):
        assert call(**bad) == BAD, bad
    assert call(wsb=need - 1) == emb.EMB_ERR_WORKSPACE


@pytest.mark.parametrize("mirror,struct", [(emb.BlockNormArgs, "emb_block_norm_args"),
                                           (emb.BlockNormGradArgs, "emb_block_norm_grad_args")])
def test_struct_layouts(tmp_path, mirror, struct):
    names = [f[0] for f in mirror._fields_]
    size, offs = c_layout(tmp_path, struct, names)
    assert size == ctypes.sizeof(mirror)
    assert offs == [getattr(mirror, n).offset for n in names]


# ------------------------------------------------------------------ the binding
@pytest.fixture
def machine(monkeypatch):
    monkeypatch.setattr(train, "_device", lambda: 0)
    monkeypatch.setattr(train, "_stream", lambda s: 0 if s is None else s.cuda_stream)
    return Machine(monkeypatch, emb, train)


X, ROW, STATS, TABLE, IDS, PER = (Tensor((6, 8)), Tensor(8), Tensor((2, 6)), Tensor((50, 8)), Tensor(6, torch.int32),
                                  Tensor(6))
CALLS = {
    "dropout": (lambda **kw: emb.dropout(X, 0.1, 3, **kw), 1),
    "block_norm": (lambda **kw: emb.block_norm(X, X, **kw), 4),
    "block_norm_backward": (lambda **kw: emb.block_norm_backward(X, X, X, X, STATS, STATS, gate=ROW, **kw), 5),
    "vocab_loss": (lambda **kw: emb.vocab_loss(X, TABLE, IDS, **kw), 2),
    "vocab_loss_backward": (lambda **kw: emb.vocab_loss_backward(PER, X, TABLE, IDS, PER, **kw), 3),
}


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_allocates_belongs_to_its_stream(name, machine):
    call, count = CALLS[name]
    call(stream=Stream())
    assert len(machine.made) == count
    assert [t.under for t in machine.made] == [Stream.cuda_stream] * count
    assert machine.lib.calls[-1][1][-1] == Stream.cuda_stream
    workspaces = [t for t in machine.made if t.dtype == torch.uint8]
    assert len(workspaces) == (name not in ("dropout", "block_norm"))
    assert all(t.used_on == ([] if t in workspaces else ["current"]) for t in machine.made)


def wide(**kw):
    return Tensor((6, 8), **kw)


REFUSED = [
    lambda: emb.dropout(Tensor(6), 0.1, 1),
    lambda: emb.dropout(wide(dtype=torch.float16), 0.1, 1),
    lambda: emb.dropout(wide(device="cpu"), 0.1, 1),
    lambda: emb.dropout(wide(stride=(16, 2)), 0.1, 1),
    lambda: emb.dropout(X, 0.1, 1, residual=wide(dtype=BF16)),
    lambda: emb.dropout(X, 0.1, 1, residual=Tensor((5, 8))),
    lambda: emb.dropout(X, 0.1, 1, out=Tensor((6, 9))),
    lambda: emb.dropout(X, 0.1, 1, out=wide(stride=(4, 1))),
    lambda: emb.dropout(X, 0.1, 1, out=wide(device="cuda:1")),
    lambda: emb.block_norm(X, Tensor((6, 9))),
    lambda: emb.block_norm(wide(dtype=BF16), X),
    lambda: emb.block_norm(X, X, gate=Tensor(7)),
    lambda: emb.block_norm(X, X, gate=Tensor((2, 8)), gate_rows=4, out=(X, X, STATS, None)),
    lambda: emb.block_norm(X, X, gate=Tensor((3, 8)), gate_rows=4),
    lambda: emb.block_norm(X, X, gate=wide(dtype=BF16), gate_rows=1),
    lambda: emb.block_norm(X, X, post=(Tensor(7), None)),
    lambda: emb.block_norm(X, X, pre=(None, Tensor(9))),
    lambda: emb.block_norm(X, X, pre=None, out=(X, X, STATS, STATS)),
    lambda: emb.block_norm(X, X, out=(X, X, Tensor((2, 5)), STATS)),
    lambda: emb.block_norm(X, X, out=(wide(dtype=BF16), X, STATS, STATS)),
    lambda: emb.block_norm(X, wide(device="cuda:1")),
    lambda: emb.block_norm_backward(X, None, X, X, STATS, STATS),
    lambda: emb.block_norm_backward(X, X, X, X, None, STATS),
    lambda: emb.block_norm_backward(X, X, X, X, STATS, STATS, pre=None),
    lambda: emb.block_norm_backward(wide(dtype=BF16), X, X, X, STATS, STATS),
    lambda: emb.block_norm_backward(X, Tensor((5, 8)), X, X, STATS, STATS),
    lambda: emb.block_norm_backward(X, X, X, X, STATS, STATS, out=(X, X, Tensor((2, 8)), None, None, None, None)),
    lambda: emb.block_norm_backward(X, X, X, X, STATS, STATS, out=(X, X, None, Tensor(4), None, None, None)),
    lambda: emb.vocab_loss(X, Tensor((50, 9)), IDS),
    lambda: emb.vocab_loss(X, Tensor((50, 8), dtype=BF16), IDS),
    lambda: emb.vocab_loss(X, TABLE, Tensor(6, torch.int64)),
    lambda: emb.vocab_loss(X, TABLE, Tensor(7, torch.int32)),
    lambda: emb.vocab_loss(X, TABLE, IDS, out=(PER, Tensor(5))),
    lambda: emb.vocab_loss(X, TABLE, IDS, workspace=Tensor(64, torch.uint8, device="cpu")),
    lambda: emb.vocab_loss(X, Tensor((50, 8), device="cuda:1"), IDS),
    lambda: emb.vocab_loss_backward(Tensor(5), X, TABLE, IDS, PER),
    lambda: emb.vocab_loss_backward(PER, X, TABLE, IDS, Tensor(5)),
    lambda: emb.vocab_loss_backward(PER, X, TABLE, IDS, PER, out=(Tensor((6, 9)), None)),
    lambda: emb.vocab_loss_backward(PER, X, TABLE, IDS, PER, out=(None, Tensor((49, 8)))),
    lambda: emb.vocab_loss_backward(PER, X, TABLE, IDS, PER, out=(None, Tensor((50, 8), dtype=BF16))),
    lambda: emb.vocab_loss_workspace_bytes(4, 100, 8, torch.float16),
    lambda: emb.vocab_loss_workspace_bytes(1 << 40, 100, 8),
    lambda: emb.block_norm_backward_workspace_bytes(4, 1 << 40),
]


@pytest.mark.parametrize("k", range(len(REFUSED)))
def test_the_binding_refuses(k, machine):
    with pytest.raises(emb.EmbError):
        REFUSED[k]()
    assert not [c for c in machine.lib.calls if not c[0].endswith("workspace_bytes")]


def test_a_seed_on_the_device_has_to_be_one_int64():
    for t in (torch.zeros(1, dtype=torch.int64), torch.zeros(2, dtype=torch.int64)):
        with pytest.raises(emb.EmbError):
            train._seed(t)
    assert train._seed(-1) == ((1 << 64) - 1, None)
