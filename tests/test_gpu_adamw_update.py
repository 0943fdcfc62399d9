"""The parameter's update of emb_adamw_step bit for bit against numpy's float32 operations (each rounded to
nearest, subnormal numbers kept), as the header writes them, from moments in 32 and in 8 bits: ordinary
gradients, gradients whose second moment is subnormal, and eps of 0 or near it; and gradients that are not
finite."""
import numpy as np
import pytest
import torch

import dense_ref as ref
import paper_2110_09132_amd as emb

pytestmark = pytest.mark.gpu

N = 3000


def tensors(bits, g, p):
    p, g = torch.from_numpy(p.copy()).cuda(), torch.from_numpy(g).cuda()
    if bits == 8:
        m, v, s = emb.adamw_state8(p)
        return p, g, m, v, s
    return p, g, torch.zeros_like(p), torch.zeros_like(p), None


def moments(m, v, s):
    m, v = m.cpu().float().numpy(), v.cpu().float().numpy()
    if s is None:
        return m, v
    s, at = s.cpu().numpy(), np.arange(m.size) // ref.BLOCK
    return m * s[at], v * s[s.size // 2 + at]


def step32(p, g, m, v, h):
    """p after the step, operation by operation in float32."""
    c = emb.adamw_coeffs(*h, torch.empty(emb.EMB_ADAMW_COEFFS_WORDS)).numpy()
    step_size, inv_bc2, eps, lr_decay = c[4:8]
    m1, v1 = ref.moments32(g, m, v, h)
    with np.errstate(all="ignore"):
        p = p - p * lr_decay
        return p - m1 / (np.sqrt(v1 * inv_bc2) + eps) * step_size


def gradients(kind):
    r = np.random.default_rng(3)
    sign = np.where(r.random(N) < 0.5, -1.0, 1.0)
    if kind == "ordinary":
        return (r.standard_normal(N) * 0.02).astype(np.float32)
    # (1 - beta2) g^2 from a dozen steps of the smallest subnormal number up to normal numbers
    return (sign * 10.0 ** r.uniform(-20.4, -17.0, N)).astype(np.float32)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-30, 1e-20, 1e-8])
@pytest.mark.parametrize("kind", ["ordinary", "tiny"])
def test_update_bit_for_bit(kind, eps, bits):
    g = gradients(kind)
    for start in (np.zeros(N, np.float32), np.random.default_rng(4).standard_normal(N).astype(np.float32)):
        p, gd, m, v, s = tensors(bits, g, start)
        for t in (1, 2, 3):  # the second step reads the state that the first left
            h = (1e-3, 0.9, 0.999, eps, 0.01, t)
            want = step32(p.cpu().numpy(), g, *moments(m, v, s), h)
            st = emb.new_status()
            emb.adamw_step([p], [gd], [m], [v], *h, scales=None if s is None else [s], dev_status=st)
            assert np.isfinite(want).all()
            assert np.array_equal(p.cpu().numpy(), want)
            assert st.item() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_tiny_gradients_move_a_parameter_by_the_rate(bits):
    # the first step of any gradient is lr sign(g): 0.1 g / (1 - 0.9) over sqrt(0.001 g^2 / (1 - 0.999))
    g = gradients("tiny")
    g = g[np.abs(g) > 1e-18]  # where g^2 (1 - beta2) has 10 bits and more
    p, gd, m, v, s = tensors(bits, g, np.zeros_like(g))
    emb.adamw_step([p], [gd], [m], [v], 1e-3, 0.9, 0.999, 0.0, 0.0, 1, scales=None if s is None else [s])
    assert np.allclose(p.cpu().numpy(), -1e-3 * np.sign(g), rtol=2.0 ** -10, atol=0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -float("inf")])
def test_a_gradient_that_is_not_finite_makes_its_parameter_nan(bits, junk):
    g = gradients("ordinary")
    g[1000] = junk
    p, gd, m, v, s = tensors(bits, g, np.ones(N, np.float32))
    st = emb.new_status()
    emb.adamw_step([p], [gd], [m], [v], 1e-3, 0.9, 0.999, 1e-8, 0.01, 1, scales=None if s is None else [s],
                   dev_status=st)
    assert st.item() == emb.EMB_DEV_NOT_FINITE
    nan = torch.isnan(p).cpu().numpy()
    assert nan[1000] and nan.sum() == 1  # infinite moments give infinity over infinity


@pytest.mark.parametrize("bits", [32, 8])
def test_large_finite_moments_are_finite(bits):
    # each below the largest number, their sum is not
    p, g = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    if bits == 32:
        m, v, s = torch.full_like(p, 3.2e38), torch.full_like(p, 3.2e38), None
    else:
        m, v, s = emb.adamw_state8(p)
        m.fill_(192.0)
        v.fill_(24576.0)
        s[:2].fill_(2.0 ** 120)
        s[2:].fill_(2.0 ** 113)
    st = emb.new_status()
    emb.adamw_step([p], [g], [m], [v], 1e-3, 0.9, 0.999, 1e-8, 0.01, 5, scales=None if s is None else [s],
                   dev_status=st)
    assert torch.isfinite(p).all() and all(np.isfinite(x).all() for x in moments(m, v, s))
    assert st.item() == 0
    if bits == 32:
        v.fill_(-float("inf"))
        emb.adamw_step([p], [g], [m], [v], 1e-3, 0.9, 0.999, 1e-8, 0.01, 5, dev_status=st)
        assert st.item() == emb.EMB_DEV_NOT_FINITE
