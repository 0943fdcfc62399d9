"""emb_adamw_step against tests/dense_ref.py: parameters (and 32-bit moments) within the derived fp32 bounds
of the 64-bit definition, 8-bit moments code for code and scale for scale against a rounding that looks the
value up in the grid of the type, from moments that are evaluated operation by operation in fp32.  Sizes on
both sides of a vector, a block, a chunk and of the tensors of one launch; both gradient types; views that
start anywhere; empty tensors; copies; the gradient's scale; coefficients from device memory in replayed
graphs; gradients that are 0, huge, infinite and NaN; more than 2^31 elements; repeated runs bit for bit;
and that many small changes of an 8-bit moment add up."""
import numpy as np
import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb
from dense_way import way  # noqa: F401
from paper_2110_09132_amd import dense

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
H = (1e-3, 0.9, 0.999, 1e-8, 0.01, 7)  # lr, beta1, beta2, eps, weight decay, step
SIZES = [1, 2, 3, 4, 5, 63, 255, 256, 257, 1000, 1023, 4095, 4096, 4097, 0, 12290, 70001]


def call(p, g, m, v, h=H, **kw):
    emb.adamw_step(p, g, m, v, *h[:5], h[5], **kw)


class Tensors:
    """Parameters with gradients and moments, of given sizes; offset: where the views start in their buffers."""

    def __init__(self, sizes, bits, gt=F32, copies=False, offset=0, seed=1):
        self.sizes, self.bits = sizes, bits

        def views(make, dtype):
            out = []
            for i, n in enumerate(sizes):
                flat = torch.zeros(n + offset, dtype=dtype, device="cuda")
                flat[offset:].copy_(make(i, n))
                out.append(flat[offset:])
            return out
        r = lambda k, s: lambda i, n: ref.randn((n,), seed * 1000 + 10 * i + k, s)  # noqa: E731
        self.p, self.g = views(r(0, 0.5), F32), views(r(1, 0.02), gt)
        self.s = None
        if bits == 32:
            self.m = views(r(2, 0.01), F32)
            self.v = views(lambda i, n: r(3, 0.02)(i, n) ** 2, F32)
        else:
            self.m = views(lambda i, n: (r(2, 20.0)(i, n)).to(torch.float8_e4m3fn).view(torch.uint8), torch.uint8)
            self.v = views(lambda i, n: ((r(3, 40.0)(i, n)) ** 2).to(torch.float8_e5m2).view(torch.uint8), torch.uint8)
            self.m = [t.view(torch.float8_e4m3fn) for t in self.m]
            self.v = [t.view(torch.float8_e5m2) for t in self.v]
            blocks = [-(-n // ref.BLOCK) for n in sizes]
            self.s = [torch.cat((torch.full((b,), 2.0 ** -11), torch.full((b,), 2.0 ** -22))).cuda() for b in blocks]
        self.c = views(lambda i, n: torch.zeros(n), BF16) if copies else None

    def step(self, h=H, **kw):
        call(self.p, self.g, self.m, self.v, h, scales=self.s, copies=self.c, **kw)

    def host(self):
        """(p, g, m, v) per tensor, moments as the fp32 values they stand for."""
        out = []
        for i, n in enumerate(self.sizes):
            m, v = self.m[i].cpu().float(), self.v[i].cpu().float()
            if self.bits == 8:
                s = self.s[i].cpu()
                b = s.numel() // 2
                at = torch.arange(n) // ref.BLOCK
                m, v = m * s[at], v * s[b + at]
            out.append((self.p[i].cpu(), self.g[i].cpu().float(), m, v))
        return out


def codes(t):
    return t.view(torch.uint8).cpu().numpy().astype(np.int64)


def check8(ts, i, before, h, seed):
    p, g, m, v = before
    m1, v1 = ref.moments32(g.numpy(), m.numpy(), v.numpy(), h)
    n = m1.size
    rm, rv = ref.random16(i, n, seed, h[5])
    cm, sm = ref.round8(m1, rm, 3, 7, 7, False)
    cv, sv = ref.round8(v1, rv, 2, 15, 14, True)
    cm = cm + np.where(np.signbit(m1), 128, 0)
    assert np.array_equal(codes(ts.m[i]), cm)
    assert np.array_equal(codes(ts.v[i]), cv)
    assert np.array_equal(ts.s[i].cpu().numpy(), np.concatenate((sm, sv)))


def check_step(ts, h=H, scale=None, seed=0, **kw):
    before = ts.host()
    ts.step(h, seed=seed, grad_scale=scale, **kw)
    for i, (p, g, m, v) in enumerate(before):
        if scale is not None:
            g = g * scale.cpu()
        w1, m1, v1, dw, dm, dv = ref.adamw64(*(t.double() for t in (p, g, m, v)), h)
        ref.assert_within(ts.p[i], w1, dw, f"w of tensor {i}")
        if ts.bits == 32:
            ref.assert_within(ts.m[i], m1, dm, f"m of tensor {i}")
            ref.assert_within(ts.v[i], v1, dv, f"v of tensor {i}")
        else:
            check8(ts, i, (p, g, m, v), h, seed)
        if ts.c is not None:
            assert torch.equal(ts.c[i], ts.p[i].to(BF16))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gt,copies,offset", [(F32, False, 0), (BF16, True, 0), (F32, True, 1), (BF16, False, 3)])
def test_sizes_types_and_places(bits, gt, copies, offset):
    ts = Tensors(SIZES, bits, gt, copies, offset)
    check_step(ts, seed=5)
    check_step(ts, (2e-3, 0.8, 0.99, 1e-6, 0.0, 8), seed=6)  # from the state the step left


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [63, 64, 65, 150])
def test_many_tensors(bits, count, way):
    sizes = [(7 * i * i + 3) % 1500 if i % 9 else 0 for i in range(count)]
    check_step(Tensors(sizes, bits, BF16), seed=9)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_zero_moments_and_the_gradients_scale(bits):
    ts = Tensors([300, 5000], bits)
    if bits == 8:
        st = [emb.adamw_state8(p) for p in ts.p]
        ts.m, ts.v, ts.s = ([t[k] for t in st] for k in range(3))
    else:
        ts.m, ts.v = [torch.zeros_like(p) for p in ts.p], [torch.zeros_like(p) for p in ts.p]
    check_step(ts, H[:5] + (1,), scale=torch.tensor([0.37], device="cuda"))


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_that_are_not_ordinary(bits):
    ts = Tensors([2000], bits)
    g = ts.g[0]
    g[256:512] = 0.0
    ts.m[0].view(torch.uint8)[256 * (4 if bits == 32 else 1):512 * (4 if bits == 32 else 1)] = 0
    ts.v[0].view(torch.uint8)[256 * (4 if bits == 32 else 1):512 * (4 if bits == 32 else 1)] = 0
    g[600] = 1e15
    g[601] = 1e-15       # beside it: its moments end at the bottom of the block's range
    g[1100] = -0.0
    st = emb.new_status()
    p0 = ts.p[0].clone()
    check_step(ts, dev_status=st)
    assert st.item() == 0
    assert torch.equal(ts.p[0][256:512].cpu(), (p0[256:512].cpu() - p0[256:512].cpu() * np.float32(H[0] * H[4])))
    if bits == 8:  # a second moment that is not zero never becomes zero
        assert ((codes(ts.v[0]) == 0) == ((np.arange(2000) >= 256) & (np.arange(2000) < 512))).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf")])
def test_gradients_that_are_not_finite(bits, junk):
    ts, clean = Tensors([3000, 700], bits), Tensors([3000, 700], bits)
    ts.g[0][1000] = junk
    st = emb.new_status()
    clean.step(dev_status=st)
    assert st.item() == 0
    ts.step(dev_status=st)
    assert st.item() == emb.EMB_DEV_NOT_FINITE
    ok = torch.ones(3000, dtype=torch.bool)
    ok[1000] = False
    assert torch.equal(ts.p[0].cpu()[ok], clean.p[0].cpu()[ok]) and not torch.isfinite(ts.p[0][1000] - 0 * ts.p[0][1000] / 0)
    assert torch.equal(ts.p[1], clean.p[1])
    sick = ~ok
    if bits == 8:  # the moments of the element's block
        sick[768:1024] = True
    got, want = ts.host()[0], clean.host()[0]
    for a, b in zip(got[2:], want[2:]):
        assert torch.equal(a[~sick], b[~sick])
        assert not torch.isfinite(a[1000])
        if bits == 8:
            assert torch.isnan(a[sick]).all()


def test_copy_of_an_infinite_parameter_and_eps_zero():
    ts = Tensors([512], 32, copies=True)
    ts.p[0][5], ts.p[0][6], ts.p[0][7] = float("inf"), float("nan"), 3.3962e38  # the last rounds to infinity in bf16
    ts.step((1e-3, 0.9, 0.999, 0.0, 0.0, 3))
    assert torch.equal(ts.c[0].view(torch.int16)[:6], ts.p[0].to(BF16).view(torch.int16)[:6])
    assert torch.isnan(ts.c[0][6]) and torch.isinf(ts.c[0][7])


@pytest.mark.parametrize("bits", [32, 8])
def test_repeated_runs_and_another_stream(bits):
    a, b, c = (Tensors([5000, 33], bits, copies=True) for _ in range(3))
    a.step(seed=3)
    b.step(seed=3)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c.step(seed=3, stream=side)
    side.synchronize()
    for x in (b, c):
        for q in ("p", "m", "v", "c") + (("s",) if bits == 8 else ()):
            for s, t in zip(getattr(a, q), getattr(x, q)):
                assert np.array_equal(ref.np_bits(s), ref.np_bits(t))
    if bits == 8:  # another seed and another step round otherwise
        for kw in (dict(seed=4), dict(h=H[:5] + (8,), seed=3)):
            d = Tensors([5000, 33], bits)
            d.step(**kw)
            assert not np.array_equal(codes(d.m[0]), codes(a.m[0]))


@pytest.mark.parametrize("bits", [32, 8])
def test_graph_replays_with_coefficients_from_device_memory(bits):
    ts, eager = Tensors([5000, 300], bits, copies=True), Tensors([5000, 300], bits, copies=True)
    coeffs = torch.zeros(emb.EMB_ADAMW_COEFFS_WORDS, device="cuda")
    clip = torch.ones(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ts.step(coeffs=coeffs, grad_scale=clip)
    buf = torch.empty(emb.EMB_ADAMW_COEFFS_WORDS)
    for k in range(4):
        h = (1e-3 / (k + 1), 0.9, 0.99, 1e-8, 0.1, k + 1)
        coeffs.copy_(emb.adamw_coeffs(*h, buf, seed=11))
        clip.fill_(1.0 / (k + 1))
        for s, t in zip(ts.g, eager.g):
            s.mul_(-1.1)
            t.mul_(-1.1)
        graph.replay()
        torch.cuda.synchronize()
        eager.step(h, grad_scale=clip, seed=11)
        for q in ("p", "m", "v", "c"):
            for s, t in zip(getattr(ts, q), getattr(eager, q)):
                assert np.array_equal(ref.np_bits(s), ref.np_bits(t))


@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_2_to_the_31_elements(bits):
    n, tail = (1 << 31) + 777, 1000
    z = lambda dt: torch.zeros(n, dtype=dt, device="cuda")  # noqa: E731
    p, g = z(F32), z(BF16)
    m, v, s = emb.adamw_state8(p) if bits == 8 else (z(F32), z(F32), None)
    p[-tail:] = ref.randn((tail,), 1).cuda()
    g[-tail:] = ref.randn((tail,), 2).cuda().to(BF16)
    p0, g0 = p[-tail:].cpu(), g[-tail:].cpu().float()
    h = H[:5] + (1,)
    call([p], [g], [m], [v], h, scales=None if s is None else [s], seed=2)
    w1, m1, v1, dw, dm, dv = ref.adamw64(p0.double(), g0.double(), torch.zeros(tail).double(), torch.zeros(tail).double(), h)
    ref.assert_within(p[-tail:], w1, dw, "w")
    assert (p[:4096] == 0).all() and (p[-tail - 4096:-tail] == 0).all()
    if bits == 32:
        ref.assert_within(m[-tail:], m1, dm, "m")
        ref.assert_within(v[-tail:], v1, dv, "v")
    else:  # the last whole blocks and the part block behind them
        first = (n - tail) // ref.BLOCK * ref.BLOCK
        g1 = np.zeros(n - first, np.float32)
        g1[-tail:] = g0.numpy()
        zero = np.zeros_like(g1)
        m1, v1 = ref.moments32(g1, zero, zero, h)
        rm, rv = ref.random16(0, n - first, 2, 1, first)
        cm, sm = ref.round8(m1, rm, 3, 7, 7, False)
        cv, sv = ref.round8(v1, rv, 2, 15, 14, True)
        assert np.array_equal(codes(m[first:]), cm + np.where(np.signbit(m1), 128, 0))
        assert np.array_equal(codes(v[first:]), cv)
        b = s.numel() // 2
        k = sm.size
        assert np.array_equal(s[b - k:b].cpu().numpy(), sm) and np.array_equal(s[-k:].cpu().numpy(), sv)


def test_small_changes_of_8_bit_moments_add_up():
    # constant gradients: v approaches g^2 by 0.1 % of the way per step, far less than the step between two
    # codes; the mean over many elements follows the exact moment
    n, steps, b1, b2 = 1 << 16, 400, 0.9, 0.999
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 0.7, device="cuda")
    m, v, s = emb.adamw_state8(p)
    for t in range(1, steps + 1):
        call([p], [g], [m], [v], (0.0, b1, b2, 1e-8, 0.0, t), scales=[s], seed=1)
    blocks = s.numel() // 2
    at = torch.arange(n) // ref.BLOCK
    mean_m = (m.cpu().float() * s.cpu()[at]).double().mean().item()
    mean_v = (v.cpu().float() * s.cpu()[blocks + at]).double().mean().item()
    want_m, want_v = 0.7 * (1 - b1 ** steps), 0.49 * (1 - b2 ** steps)
    # the rounding errors of one element are a martingale with steps of at most 1/8 (m) and 1/4 (v) of the
    # value, so its deviation stays below sqrt(steps) / 4 of the value; over n independent elements five
    # standard deviations of the mean are below 5 sqrt(steps) / (4 sqrt(n))
    slack = 5 * steps ** 0.5 / (4 * n ** 0.5)
    assert abs(mean_m - want_m) <= slack * want_m
    assert abs(mean_v - want_v) <= slack * want_v


def test_empty_calls():
    emb.adamw_step([], [], [], [], *H)
    ts = Tensors([0, 0], 8)
    ts.step()


@pytest.mark.parametrize("bits", [32, 8])
def test_lists_are_read_alike_on_both_ways(bits, monkeypatch):
    # parameters as nn.Parameter, shapes of several dimensions, dimensions of one with odd strides, tuples
    a, b = (Tensors([4096, 600, 0, 7], bits, BF16, copies=True) for _ in range(2))
    for ts in (a, b):
        ts.p = (torch.nn.Parameter(ts.p[0].view(64, 64)), ts.p[1].view(20, 1, 30), ts.p[2].view(0, 5), ts.p[3])
        ts.g[1] = ts.g[1].as_strided((600, 1), (1, 77))
    clip, st = torch.full((1,), 0.5, device="cuda"), emb.new_status()
    with monkeypatch.context() as m:
        m.setattr(dense, "_adamw_table", None)  # the long way is not taken
        a.step(seed=3, grad_scale=clip, dev_status=st)
    dense._native.use(None, torch.Tensor, torch.nn.Parameter)
    try:
        b.step(seed=3, grad_scale=clip, dev_status=st)
    finally:
        dense._native.use(torch.Tensor.__dlpack_c_exchange_api__, torch.Tensor, torch.nn.Parameter)
    for q in ("p", "m", "v", "c") + (("s",) if bits == 8 else ()):
        for s, t in zip(getattr(a, q), getattr(b, q)):
            assert np.array_equal(ref.np_bits(s), ref.np_bits(t))


def test_refusals(way):
    def fresh(**kw):
        d = dict(p=Tensors([40, 50], 32))
        t, t8 = d["p"], Tensors([40, 50], 8)
        a = dict(params=t.p, grads=t.g, exp_avgs=t.m, exp_avg_sqs=t.v, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                 weight_decay=0.0, step=1)
        a.update(kw.pop("eight")(t8) if "eight" in kw else {})
        a.update(kw)
        return emb.adamw_step(**a)
    t, t8 = Tensors([40, 50], 32), Tensors([40, 50], 8)
    bf = [x.to(BF16) for x in t.p]
    for kw in (dict(params=t.p[:1]), dict(grads=t.g[:1]), dict(grads=[t.g[0], bf[1]]), dict(grads=[x.half() for x in t.g]),
               dict(params=bf), dict(params=[x.cpu() for x in t.p]), dict(exp_avgs=t.v[::-1]), dict(exp_avg_sqs=bf),
               dict(params=[torch.zeros(80, device="cuda")[::2], t.p[1]]), dict(exp_avgs=t8.m, exp_avg_sqs=t8.v),
               dict(scales=t8.s), dict(eight=lambda x: dict(exp_avgs=x.m, exp_avg_sqs=x.v, scales=x.s[:1])),
               dict(eight=lambda x: dict(exp_avgs=x.v, exp_avg_sqs=x.m, scales=x.s)),
               dict(eight=lambda x: dict(exp_avgs=x.m, exp_avg_sqs=x.v, scales=[x.s[0][:1], x.s[1]])),
               dict(copies=t.p), dict(copies=bf[:1]), dict(grad_scale=torch.ones(1)), dict(coeffs=torch.zeros(4, device="cuda")),
               dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(lr=float("nan")),
               dict(weight_decay=-1.0), dict(weight_decay=float("inf"))):
        with pytest.raises(emb.EmbError):
            fresh(**kw)
    fresh()
