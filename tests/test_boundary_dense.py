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


def test_relative_bias_validation():
    def call(t=FAKE, nb=4, H=2, m=FAKE, R=3, Q=5, K=6, q0=0, out=FAKE, dt=0, ldq=6, ldh=30):
        return emb.lib.emb_relative_bias(t, nb, H, m, R, Q, K, q0, out, dt, ldq, ldh, NULL, NULL)
    assert call(Q=0, t=NULL, m=NULL, out=NULL) == emb.EMB_OK
    assert call(K=0, t=NULL, m=NULL, out=NULL) == emb.EMB_OK
    for bad in (dict(nb=0), dict(H=0), dict(H=65536), dict(R=-1), dict(R=1 << 30), dict(Q=-1), dict(Q=1 << 30),
                dict(K=-1), dict(K=1 << 30), dict(q0=1 << 62), dict(q0=-(1 << 62)), dict(dt=2), dict(ldq=5),
                dict(ldh=29), dict(ldh=-30), dict(t=NULL), dict(m=NULL), dict(out=NULL), dict(t=ODD), dict(m=ODD),
                dict(out=ODD), dict(out=ODD, dt=1)):
        assert call(**bad) == BAD, bad


def test_relative_bias_heads_that_overlap():
    def call(Q, K, H, ldq, ldh):
        return emb.lib.emb_relative_bias(FAKE, 4, H, FAKE, 3, Q, K, 0, FAKE, 0, ldq, ldh, NULL, NULL)
    for Q, K, H, ldq, ldh in ((5, 6, 2, 11, 6), (5, 6, 2, 12, 5), (5, 6, 4, 23, 6), (5, 6, 4, 24, 7), (5, 6, 2, 12, 0),
                              (5, 6, 2, 12, -6), (2, 6, 3, 17, 6)):
        assert call(Q, K, H, ldq, ldh) == BAD, (Q, K, H, ldq, ldh)


def test_relative_bias_backward_validation():
    size = emb.lib.emb_relative_bias_backward_workspace_bytes
    need = size(2, 2, 5, 6)
    assert need > 0 and need % 256 == 0
    assert size(-1, 2, 5, 6) == 0 and size(1, 0, 5, 6) == 0 and size(1, 2, -5, 6) == 0

    def call(g=FAKE, dt=0, N=2, H=2, Q=5, K=6, ldn=60, ldh=30, ldq=6, m=FAKE, R=3, nb=4, q0=0, out=FAKE, ws=FAKE,
             wsb=need):
        return emb.lib.emb_relative_bias_backward(g, dt, N, H, Q, K, ldn, ldh, ldq, m, R, nb, q0, out, ws, wsb, NULL,
                                                  NULL)
    for bad in (dict(N=-1), dict(nb=0), dict(H=0), dict(R=-1), dict(Q=-1), dict(K=-1), dict(q0=1 << 62), dict(dt=2),
                dict(ldn=-1), dict(ldh=-1), dict(ldq=-1), dict(g=NULL), dict(g=ODD), dict(m=NULL), dict(m=ODD),
                dict(out=NULL), dict(out=ODD), dict(ws=NULL), dict(ws=ctypes.c_void_p(4096 + 64))):
        assert call(**bad) == BAD, bad
    assert call(wsb=need - 1) == emb.EMB_ERR_WORKSPACE


def test_relative_buckets():
    def of(buckets, far, causal):
        out = (ctypes.c_int32 * (2 * far + 1))()
        assert emb.lib.emb_relative_buckets(buckets, far, causal, out) == emb.EMB_OK
        return list(out)

    def worked(n, m, far):  # the largest bucket k whose start e (far / e)^((k - e) / (m - e)) is at most n, in whole numbers
        e = m // 2
        if n < e:
            return n
        k = e
        while k + 1 < m and n ** (m - e) >= e ** (m - e - (k + 1 - e)) * far ** (k + 1 - e):
            k += 1
        return k
    for buckets, far, causal in ((32, 128, 0), (32, 128, 1), (8, 16, 0), (4, 2, 0), (2, 2, 1), (64, 1000, 0), (7, 9, 1),
                                 (8, 64, 1), (16, 256, 1)):
        m = buckets if causal else buckets // 2
        got = of(buckets, far, causal)
        want = [worked(abs(r), m, far) + (m if r > 0 else 0) for r in range(-far, far + 1)]
        if causal:
            want = [w if r <= 0 else -1 for w, r in zip(want, range(-far, far + 1))]
        assert got == want, (buckets, far, causal)
    out = (ctypes.c_int32 * 9)()
    for bad in ((1, 4, 1), (0, 4, 1), (2, 4, 0), (6, 1, 0), (5, 4, 0), (8, 4, 1), (4, -1, 1), (4, 1 << 30, 1)):
        assert emb.lib.emb_relative_buckets(*bad, out) == BAD, bad
    assert emb.lib.emb_relative_buckets(4, 4, 1, NULL) == BAD


class AdamwTensor(ctypes.Structure):
    """emb_adamw_tensor of include/emb.h."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "exp_avg", "exp_avg_sq", "scales", "copy")] + \
        [("n", ctypes.c_int64)]


def test_adamw_tensor_layout(tmp_path):
    from test_abi_layout import c_layout
    names = [f[0] for f in AdamwTensor._fields_]
    size, offs = c_layout(tmp_path, "emb_adamw_tensor", names)
    assert size == ctypes.sizeof(AdamwTensor) == 7 * 8  # the binding writes seven words for each
    assert offs == [getattr(AdamwTensor, n).offset for n in names]


def test_adamw_validation():
    def call(n=1, gt=0, bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, step=1, coeffs=NULL, scale=NULL,
             second=None, **field):
        t = (AdamwTensor * 2)()
        for k in range(2):
            for name in ("param", "grad", "exp_avg", "exp_avg_sq"):
                setattr(t[k], name, 4096)
            t[k].n = 10
        for name, value in field.items():
            setattr(t[0], name, value)
        for name, value in (second or {}).items():
            setattr(t[1], name, value)
        return emb.lib.emb_adamw_step(t, n, gt, bits, lr, b1, b2, eps, wd, step, 0, coeffs, scale, NULL, NULL)
    assert call(n=0) == emb.EMB_OK
    assert emb.lib.emb_adamw_step(NULL, 0, 0, 32, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, NULL, NULL, NULL, NULL) == emb.EMB_OK
    for bad in (dict(n=-1), dict(gt=2), dict(bits=16), dict(bits=8), dict(lr=NAN), dict(lr=INF), dict(b1=1.0),
                dict(b1=-0.1), dict(b2=1.0), dict(eps=-1.0), dict(wd=-1.0), dict(wd=NAN), dict(step=0), dict(coeffs=ODD),
                dict(scale=ODD), dict(param=0), dict(grad=0), dict(exp_avg=0), dict(exp_avg_sq=0), dict(param=4097),
                dict(grad=4098), dict(exp_avg=4098), dict(exp_avg_sq=4099), dict(n=2, second=dict(copy=4096)),
                dict(copy=4097, n=1), dict(bits=8, scales=4098), dict(n=2, second=dict(n=-1)),
                dict(n=2, second=dict(n=(1 << 35) + 1))):
        assert call(**bad) == BAD, bad
    assert emb.lib.emb_adamw_step(NULL, 1, 0, 32, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, NULL, NULL, NULL, NULL) == BAD


def test_adamw_largest_tensor():
    """2^33 elements are 2^31 threads; a launch takes less than 2^32."""
    t = AdamwTensor(*[4096] * 4, 0, 0, (1 << 33) + 1)
    assert emb.lib.emb_adamw_step(ctypes.byref(t), 1, 0, 32, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, NULL, NULL, NULL,
                                  NULL) == BAD


def test_adamw_coeffs():
    out = (ctypes.c_float * emb.EMB_ADAMW_COEFFS_WORDS)()
    assert emb.lib.emb_adamw_coeffs(1e-3, 0.9, 0.999, 1e-8, 0.1, 3, 5, out) == emb.EMB_OK
    want = [0.9, 1 - 0.9, 0.999, 1 - 0.999, 1e-3 / (1 - 0.9 ** 3), 1 / (1 - 0.999 ** 3), 1e-8, 1e-4]
    assert [out[i] for i in range(8)] == [ctypes.c_float(w).value for w in want]
    assert emb.lib.emb_adamw_coeffs(1e-3, 0.9, 0.999, 1e-8, 0.1, 0, 5, out) == BAD
    assert emb.lib.emb_adamw_coeffs(1e-3, 0.9, 0.999, 1e-8, -0.1, 1, 5, out) == BAD
    assert emb.lib.emb_adamw_coeffs(1e-3, 0.9, 0.999, 1e-8, 0.1, 1, 5, NULL) == BAD
