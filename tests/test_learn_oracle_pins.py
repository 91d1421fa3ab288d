"""The oracle of the learner's operators against finite differences, closed forms and invariants (CPU only)."""
import numpy as np
import pytest

from oracle import learn_oracle as orc


def _difference(f, x, dirs, h=1e-6):
    """Central differences of the scalar f along the directions."""
    return np.array([(f(x + h * d) - f(x - h * d)) / (2 * h) for d in dirs])


@pytest.mark.parametrize("linear", (False, True))
@pytest.mark.parametrize("with_h0", (False, True))
def test_gated_gradient_against_differences(linear, with_h0):
    rng = np.random.default_rng(1)
    Bt, L, D = 2, 7, 3
    z, u, dh = (rng.normal(size=(Bt, L, D)) for _ in range(3))
    z = orc._sigmoid(z) if linear else z
    h0, dl = (rng.normal(size=(Bt, D)) if with_h0 else None), rng.normal(size=(Bt, D))
    first = rng.random((Bt, L)) < 0.3
    first[0, 0] = False

    def loss(z_, u_, h_):
        h = orc.gated_fwd(z_, u_, first, h_, linear)
        return (dh * h).sum() + (dl * h[:, -1]).sum()

    g = orc.gated_bwd(z, u, first, h0, dh, dl, linear)
    for name, f, x in (("dgate", lambda x: loss(x, u, h0), z), ("du", lambda x: loss(z, x, h0), u)) + \
                      ((("dh0", lambda x: loss(z, u, x), h0),) if with_h0 else ()):
        dirs = rng.normal(size=(6,) + x.shape)
        np.testing.assert_allclose((dirs * g[name]).sum(axis=tuple(range(1, dirs.ndim))), _difference(f, x, dirs),
                                   rtol=1e-6, atol=1e-7)


def test_gated_closed_forms():
    L = 9
    one = np.ones((1, L, 1))
    # a constant decay a on a constant input 1 is a geometric sum; coupled, it tends to the input
    h = orc.gated_fwd(0.5 * one, one, linear=True)[0, :, 0]
    np.testing.assert_allclose(h, (1 - 0.5 ** np.arange(1, L + 1)) / 0.5)
    h = orc.gated_fwd(np.zeros_like(one), 3.0 * one)[0, :, 0]
    np.testing.assert_allclose(h, 3.0 * (1 - 0.5 ** np.arange(1, L + 1)))
    # a sequence in two parts, and a reset that drops what came before
    rng = np.random.default_rng(2)
    z, u = rng.normal(size=(2, 10, 4)), rng.normal(size=(2, 10, 4))
    whole = orc.gated_fwd(z, u)
    np.testing.assert_allclose(orc.gated_fwd(z[:, 6:], u[:, 6:], None, whole[:, 5]), whole[:, 6:])
    first = np.zeros((2, 10)); first[:, 6] = 1
    np.testing.assert_allclose(orc.gated_fwd(z, u, first)[:, 6:], orc.gated_fwd(z[:, 6:], u[:, 6:]))


@pytest.mark.parametrize("kl,eta", ((0.0, 0.0), (0.3, 0.0), (0.0, 0.2), (0.3, 0.2)))
def test_policy_gradient_against_differences(kl, eta):
    rng = np.random.default_rng(3)
    N, K = 12, 5
    x, a = rng.normal(size=(N, K)), rng.integers(K, size=N)
    x[0, (a[0] + 1) % K] = -np.inf
    w, A = rng.random(N), rng.normal(size=N)
    w[3] = 0
    base = orc.policy_loss(x, a, np.zeros(N), A, w)["logp"]
    old = base + rng.normal(size=N) * 0.5                # ratios on both sides of both bounds
    ref = base + rng.normal(size=N)
    args = (a, old, A, w, ref if kl else None, 0.2, 0.3, kl, eta)
    g = orc.policy_loss(x, *args)["dlogits"]
    dirs = np.where(np.isfinite(x), rng.normal(size=(8, N, K)), 0.0)
    diff = _difference(lambda y: orc.policy_loss(y, *args)["loss"], x, dirs)
    np.testing.assert_allclose((dirs * g).sum(axis=(1, 2)), diff, rtol=1e-6, atol=1e-8)
    assert not g[3].any() and g[0, (a[0] + 1) % K] == 0
    np.testing.assert_allclose(g.sum(1), 0.0, atol=1e-12)            # logits count up to a constant


def test_policy_closed_forms():
    x = np.zeros((1, 8))
    r = orc.policy_loss(x, [3], [-np.log(8)], [2.0], [1.0], [-np.log(8)], kl_coef=1.0)
    assert abs(r["entropy"][0] - np.log(8)) < 1e-14 and abs(r["logp"][0] + np.log(8)) < 1e-14
    assert abs(r["loss"] + 2.0) < 1e-14                              # ratio one, no distance: minus the advantage
    r = orc.policy_loss(np.full((2, 4), -np.inf), [1, 2], [0, 0], [1, 1], [1, 1])
    assert r["loss"] == 0 and not r["dlogits"].any() and np.all(r["lse"] == -np.inf)


@pytest.mark.parametrize("bits", (orc.M_BITS, orc.R_BITS))
def test_code_values(bits):
    v = orc.code_values(bits)
    mantissa, bias, top = bits
    assert v[0] == 0 and np.all(np.diff(v) > 0)
    if bits is orc.M_BITS:
        assert v[126] == top                                         # (127 would be NaN in the 8-bit float of that layout)
        torch = pytest.importorskip("torch")
        t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
        np.testing.assert_array_equal(v[:127], t)
    else:
        assert v[255] == top
    step = v[2:] / v[1:-1]
    assert step[1 << mantissa:].max() <= 1 + 2.0 ** -mantissa


def test_adamw_closed_forms():
    # the first step from zero states is lr * sign(g) (eps = 0), the decay acts on the parameter alone
    g = np.array([3.0, -0.2, 1e-5])
    p, m, v = orc.adamw(np.ones(3), g, np.zeros(3), np.zeros(3), 0.1, 0.9, 0.999, 0.0, 0.01, 1)
    np.testing.assert_allclose(p, 1 - 0.1 * 0.01 - 0.1 * np.sign(g))
    np.testing.assert_allclose(m, 0.1 * g)
    np.testing.assert_allclose(v, 0.001 * g * g)
    # a constant gradient keeps the update at lr
    for t in range(2, 5):
        q, m, v = orc.adamw(p, g, m, v, 0.1, 0.9, 0.999, 0.0, 0.0, t)
        np.testing.assert_allclose(p - q, 0.1 * np.sign(g))
        p = q
