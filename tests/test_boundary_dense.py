"""The dense operators' C calls without a GPU: every bad argument is refused on the host, before anything
is enqueued (the addresses passed here are never read)."""
import ctypes

import paper_2110_09132_amd as emb

FAKE = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4097)
NULL = None
NAN, INF = float("nan"), float("inf")
BAD = emb.EMB_ERR_INVALID_ARG


def test_layer_norm_validation():
    def call(x=FAKE, xt=0, ldx=8, ids=NULL, V=0, T=4, D=8, w=NULL, b=NULL, eps=1e-5, y=FAKE, yt=0, ldy=8, mean=FAKE,
             rstd=FAKE):
        return emb.lib.emb_layer_norm(x, xt, ldx, ids, V, T, D, w, b, eps, y, yt, ldy, mean, rstd, NULL, NULL)
    assert call(T=0, x=NULL, y=NULL, mean=NULL, rstd=NULL) == emb.EMB_OK
    for bad in (dict(T=-1), dict(T=1 << 30), dict(D=0), dict(D=1 << 28), dict(xt=2), dict(yt=-1), dict(ldx=-1),
                dict(ldy=7), dict(eps=-1e-9), dict(eps=NAN), dict(eps=INF), dict(ids=FAKE, V=0),
                dict(ids=FAKE, V=1 << 31), dict(x=NULL), dict(y=NULL), dict(mean=NULL), dict(rstd=NULL), dict(x=ODD),
                dict(y=ODD), dict(x=ODD, xt=1), dict(w=ODD), dict(b=ODD)):
        assert call(**bad) == BAD, bad


def test_layer_norm_backward_validation():
    need = emb.lib.emb_layer_norm_backward_workspace_bytes(4, 8)
    assert need > 0 and need % 256 == 0
    assert emb.lib.emb_layer_norm_backward_workspace_bytes(-1, 8) == 0
    assert emb.lib.emb_layer_norm_backward_workspace_bytes(4, 0) == 0

    def call(dy=FAKE, gt=0, lddy=8, x=FAKE, xt=0, ldx=8, ids=NULL, V=0, T=4, D=8, w=NULL, mean=FAKE, rstd=FAKE,
             dx=FAKE, lddx=8, dw=FAKE, db=FAKE, ws=FAKE, wsb=need):
        return emb.lib.emb_layer_norm_backward(dy, gt, lddy, x, xt, ldx, ids, V, T, D, w, mean, rstd, dx, lddx, dw,
                                               db, ws, wsb, NULL, NULL)
    for bad in (dict(T=-1), dict(T=1 << 30), dict(D=0), dict(gt=2), dict(xt=2), dict(lddy=-1), dict(ldx=-1),
                dict(lddx=7), dict(ids=FAKE, V=0), dict(dx=NULL, dw=NULL, db=NULL), dict(dy=NULL), dict(x=NULL),
                dict(mean=NULL), dict(rstd=NULL), dict(dy=ODD), dict(x=ODD), dict(dx=ODD), dict(w=ODD), dict(dw=ODD),
                dict(db=ODD), dict(ws=NULL), dict(ws=ctypes.c_void_p(4096 + 64))):
        assert call(**bad) == BAD, bad
    assert call(wsb=need - 1) == emb.EMB_ERR_WORKSPACE
