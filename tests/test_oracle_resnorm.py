"""Pins of the norm oracle: unit rows, and the gradient against differences."""
import numpy as np
import pytest

from oracle.resnorm import resnorm_bwd, resnorm_fwd

EPS = 1e-3


def _inputs(form, gate, seed=0, N=4, D=6):
    r = np.random.Generator(np.random.PCG64(seed))
    z = lambda *s: r.standard_normal(s)  # noqa: E731
    post, pre = form != "pre", form != "post"
    return dict(x=z(N, D), u=z(N, D) if post else None, gate=z(N, D) if gate else None, w_post=z(D) if post else None,
                rho=z(D) if post else None, w_pre=z(D) if pre else None), z(N, D), z(N, D) if pre else None


def test_a_normed_row_has_unit_mean_square():
    c, _, _ = _inputs("pre", False)
    c["w_pre"] = np.ones(6)
    out = resnorm_fwd(eps=1e-12, **c)
    assert np.allclose(np.mean(out["n"] ** 2, axis=1), 1.0, atol=1e-9) and "xo" not in out


@pytest.mark.parametrize("form,gate", [("both", True), ("both", False), ("post", True), ("pre", False)])
def test_gradient_against_differences(form, gate):
    c, dxo, dn = _inputs(form, gate)

    def J(c):
        out = resnorm_fwd(eps=EPS, **c)
        return np.sum(out.get("xo", c["x"]) * dxo) + (0.0 if dn is None else np.sum(out["n"] * dn))

    xo = resnorm_fwd(eps=EPS, **c).get("xo", c["x"])
    grads = resnorm_bwd(xo, *(c[k] for k in ("u", "gate", "w_post", "rho", "w_pre")), EPS, dxo, dn)
    assert set(grads) == {"d" + k for k, v in c.items() if v is not None}
    eps = 1e-6
    for name in grads:
        g, k = grads[name], name[1:]
        num = np.empty_like(g)
        for i in np.ndindex(g.shape):
            hi, lo = c[k].copy(), c[k].copy()
            hi[i] += eps
            lo[i] -= eps
            num[i] = (J({**c, k: hi}) - J({**c, k: lo})) / (2 * eps)
        assert np.max(np.abs(num - g)) < 1e-7 * max(1.0, np.max(np.abs(g))), name
