"""Oracle: RMS norms around a block with its gate and residual scale, in fp64.

    x' = x + rho sigmoid(gate) (w_post u r_u),  n = w_pre x' r_x',  r_z = (mean z^2 + eps)^(-1/2)

Test infrastructure (see the package docstring).
"""
import numpy as np

from .precision import F


def _r(z, eps):
    return 1.0 / np.sqrt(np.mean(z * z, axis=-1, keepdims=True) + eps)


def _wide(*arrays):
    return [None if a is None else np.asarray(a, F()) for a in arrays]


def resnorm_fwd(x, u, gate, w_post, rho, w_pre, eps):
    """dict of xo, n, r_post, r_pre (those that there are)."""
    x, u, gate, w_post, rho, w_pre = _wide(x, u, gate, w_post, rho, w_pre)
    out = {}
    if u is not None:
        s = 1.0 if gate is None else 1.0 / (1.0 + np.exp(-gate))
        x = x + rho * s * w_post * u * _r(u, eps)
        out["xo"], out["r_post"] = x, _r(u, eps)[:, 0]
    if w_pre is not None:
        out["n"], out["r_pre"] = w_pre * x * _r(x, eps), _r(x, eps)[:, 0]
    return out


def _norm_bwd(z, r, a):
    """Gradient of <a, z r> with respect to z."""
    return r * a - z * r ** 3 * np.mean(a * z, axis=-1, keepdims=True)


def resnorm_bwd(xo, u, gate, w_post, rho, w_pre, eps, dxo, dn):
    """dict of dx, du, dgate, dw_post, drho, dw_pre (those that there are), x' as given."""
    xo, u, gate, w_post, rho, w_pre, dxo, dn = _wide(xo, u, gate, w_post, rho, w_pre, dxo, dn)
    out, d = {}, dxo
    if w_pre is not None:
        r = _r(xo, eps)
        d = d + _norm_bwd(xo, r, dn * w_pre)
        out["dw_pre"] = np.sum(dn * xo * r, axis=0)
    out["dx"] = d
    if u is not None:
        r = _r(u, eps)
        s = np.ones_like(u) if gate is None else 1.0 / (1.0 + np.exp(-gate))
        if gate is not None:
            out["dgate"] = d * rho * w_post * u * r * s * (1.0 - s)
        out["drho"] = np.sum(d * s * w_post * u * r, axis=0)
        out["dw_post"] = np.sum(d * s * rho * u * r, axis=0)
        out["du"] = _norm_bwd(u, r, d * s * rho * w_post)
    return out
