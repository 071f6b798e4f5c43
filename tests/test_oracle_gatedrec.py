"""Pins of the gated recurrence's oracle: the closed form of its sums, a reset, a stationary size, and its gradient against
differences."""
import numpy as np
import pytest

from oracle.gatedrec import gatedrec_bwd, gatedrec_fwd


def _inputs(seed, T, B, D, resets=True):
    g = np.random.Generator(np.random.PCG64(seed))
    n = lambda *s: g.standard_normal(s)  # noqa: E731
    return dict(x=n(T, B, D), r=n(T, B, D), i=n(T, B, D), lam=n(D) - 1.0, c=2.0, h0=n(B, D),
                reset=(g.random((T, B)) < 0.3).astype(np.uint8) if resets else None)


def test_outputs_are_the_decayed_sums():
    c = _inputs(0, 6, 2, 3, resets=False)
    sig = lambda z: 1.0 / (1.0 + np.exp(-z))  # noqa: E731
    a = np.exp(-c["c"] * np.log1p(np.exp(c["lam"])) * sig(c["r"]))
    b = np.sqrt(1.0 - a * a) * sig(c["i"]) * c["x"]
    h = gatedrec_fwd(**c)
    for t in range(6):
        ref = np.prod(a[:t + 1], axis=0) * c["h0"] + sum(np.prod(a[j + 1:t + 1], axis=0) * b[j] for j in range(t + 1))
        assert np.allclose(h[t], ref, rtol=1e-12, atol=1e-12)


def test_a_reset_starts_over():
    c = _inputs(1, 6, 3, 4, resets=False)
    cut = dict(c, reset=np.zeros((6, 3), np.uint8), h0=np.full((3, 4), np.nan))
    cut["reset"][2] = 1
    h = gatedrec_fwd(**cut)
    assert np.array_equal(h[2:], gatedrec_fwd(**{**c, "h0": None, **{k: c[k][2:] for k in "xri"}})) and np.isnan(h[:2]).all()


def test_open_inputs_of_size_one_keep_the_state_at_size_one():
    """sqrt(1 - a^2) is what makes the variance of the state that of the input, whatever the gates."""
    g = np.random.Generator(np.random.PCG64(2))
    x, r = g.standard_normal((4000, 50, 8)), g.standard_normal((1, 50, 8)) * np.ones((4000, 1, 1))
    h = gatedrec_fwd(x, r, np.full_like(x, 40.0), np.zeros(8), 1.0)
    assert abs(np.mean(h[100:] ** 2) - 1.0) < 0.02


@pytest.mark.parametrize("resets", [False, True])
def test_gradient_against_differences(resets):
    c = _inputs(3, 5, 2, 3, resets)
    g = np.random.Generator(np.random.PCG64(4))
    dh, dhT = g.standard_normal((5, 2, 3)), g.standard_normal((2, 3))

    def J(c):
        h = gatedrec_fwd(**c)
        return np.sum(h * dh) + np.sum(h[-1] * dhT)

    for name, grad in zip(("x", "r", "i", "lam", "h0"), gatedrec_bwd(dh=dh, dhT=dhT, **c)):
        num, eps = np.empty_like(grad), 1e-5
        for at in np.ndindex(grad.shape):
            hi, lo = c[name].copy(), c[name].copy()
            hi[at] += eps
            lo[at] -= eps
            num[at] = (J({**c, name: hi}) - J({**c, name: lo})) / (2 * eps)
        assert np.max(np.abs(num - grad)) < 1e-8 * max(1.0, np.max(np.abs(grad))), name


def test_closed_gates_have_no_gradient():
    """a = 1 exactly: nothing is taken in, nothing is forgotten, and the gradient of the gate is its limit."""
    c = _inputs(5, 3, 1, 4, resets=False)
    c["r"] = np.full_like(c["r"], -1000.0)
    assert np.array_equal(gatedrec_fwd(**c), np.broadcast_to(c["h0"], (3, 1, 4)))
    dx, dr, di, dlam, dh0 = gatedrec_bwd(dh=np.ones((3, 1, 4)), **c)
    assert not dx.any() and not dr.any() and not di.any() and not dlam.any() and (dh0 == 3).all()
