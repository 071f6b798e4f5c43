"""Pins of the linear-attention oracle: the closed form of its sums, a cut state, and its gradient against differences."""
import numpy as np
import pytest

from oracle.linattn import linattn_bwd, linattn_fwd


def _inputs(seed, T, B, nh, nkv, dk, dv, resets=True):
    r = np.random.Generator(np.random.PCG64(seed))
    q, k, v = r.standard_normal((T, B, nh * dk)), r.standard_normal((T, B, nkv * dk)), r.standard_normal((T, B, nkv * dv))
    return dict(q=q, k=k, v=v, decay=r.uniform(0.3, 1.0, nkv), scale=dk ** -0.5, nh=nh, nkv=nkv,
                S0=r.standard_normal((B, nkv, dk, dv)), reset=(r.random((T, B)) < 0.3).astype(np.uint8) if resets else None)


def test_outputs_are_the_decayed_sums():
    """o_t = scale (d^(t+1) S0^T q_t + sum_j d^(t-j) (q_t . k_j) v_j), summed directly."""
    c = _inputs(0, 5, 2, 4, 2, 3, 6, resets=False)
    o, states = linattn_fwd(**c)
    q, k, v = c["q"].reshape(5, 2, 4, 3), c["k"].reshape(5, 2, 2, 3), c["v"].reshape(5, 2, 2, 6)
    for t in range(5):
        for b in range(2):
            for h in range(4):
                n = h // 2
                ref = c["decay"][n] ** (t + 1) * c["S0"][b, n].T @ q[t, b, h]
                for j in range(t + 1):
                    ref = ref + c["decay"][n] ** (t - j) * (q[t, b, h] @ k[j, b, n]) * v[j, b, n]
                assert np.allclose(o[t, b, h * 6:(h + 1) * 6], c["scale"] * ref, rtol=1e-12, atol=1e-12)


def test_a_reset_starts_over():
    c = _inputs(1, 6, 3, 2, 2, 4, 4, resets=False)
    cut = dict(c, reset=np.zeros((6, 3), np.uint8))
    cut["reset"][2] = 1
    cut["S0"] = np.full_like(c["S0"], np.nan)
    o, states = linattn_fwd(**cut)
    tail = {k: c[k][2:] for k in ("q", "k", "v")}
    o2, states2 = linattn_fwd(**{**c, **tail, "S0": None})
    assert np.array_equal(o[2:], o2) and np.array_equal(states[2:], states2) and np.isnan(o[:2]).all()


@pytest.mark.parametrize("resets", [False, True])
def test_gradient_against_differences(resets):
    c = _inputs(2, 5, 2, 4, 2, 3, 4, resets)
    r = np.random.Generator(np.random.PCG64(3))
    do, dST = r.standard_normal((5, 2, 16)), r.standard_normal((2, 2, 3, 4))

    def J(c):
        o, states = linattn_fwd(**c)
        return np.sum(o * do) + np.sum(states[-1] * dST)

    grads = dict(zip(("q", "k", "v", "S0"), linattn_bwd(dout=do, dST=dST, **c)))
    eps = 1e-5
    for name, g in grads.items():
        num = np.empty_like(g)
        for i in np.ndindex(g.shape):
            hi, lo = c[name].copy(), c[name].copy()
            hi[i] += eps
            lo[i] -= eps
            num[i] = (J({**c, name: hi}) - J({**c, name: lo})) / (2 * eps)
        assert np.max(np.abs(num - g)) < 1e-8 * max(1.0, np.max(np.abs(g))), name
