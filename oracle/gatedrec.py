"""Oracle: a linear recurrence whose decay and input are gated by the input, step by step in fp64.

    log a_t = -c softplus(lam) sigmoid(r_t),  h_t = a_t (1 - reset_t) h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t

Test infrastructure (see the package docstring).
"""
import numpy as np

from .precision import F


def _sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def _gates(x, r, i, lam, c):
    """(sigmoid(r), sigmoid(i), log a, a, sqrt(1 - a^2))"""
    x, r, i, lam = (np.asarray(v, F()) for v in (x, r, i, lam))
    g = _sigmoid(r)
    la = -c * np.logaddexp(0.0, lam) * g
    return g, _sigmoid(i), la, np.exp(la), np.sqrt(-np.expm1(2.0 * la))


def _cut(reset, t, h):
    return h if reset is None else np.where((np.asarray(reset[t]) != 0)[:, None], 0.0, h)


def gatedrec_fwd(x, r, i, lam, c, h0=None, reset=None):
    """The states h [T, B, D] of x, r, i [T, B, D]."""
    T, B, D = np.shape(x)
    h = np.zeros((B, D), F()) if h0 is None else np.array(h0, F())
    out = np.empty((T, B, D), F())
    for t in range(T):
        _, o, _, a, beta = _gates(x[t], r[t], i[t], lam, c)
        h = out[t] = a * _cut(reset, t, h) + beta * o * x[t]
    return out


def gatedrec_bwd(x, r, i, lam, c, dh, h0=None, reset=None, dhT=None):
    """dx, dr, di, dlam and dh0 of J = sum <dh, h> + <dhT, h_{T-1}>."""
    x, r, i, dh = (np.asarray(v, F()) for v in (x, r, i, dh))
    T, B, D = x.shape
    h = gatedrec_fwd(x, r, i, lam, c, h0, reset)
    first = np.zeros((B, D), F()) if h0 is None else np.asarray(h0, F())
    G = np.zeros((B, D), F()) if dhT is None else np.array(dhT, F())
    dx, dr, di, dlam = np.empty_like(x), np.empty_like(x), np.empty_like(x), np.zeros(D, F())
    for t in range(T - 1, -1, -1):
        g, o, la, a, beta = _gates(x[t], r[t], i[t], lam, c)
        G = G + dh[t]
        before = _cut(reset, t, h[t - 1] if t else first)
        with np.errstate(divide="ignore", invalid="ignore"):
            # d(log a) times log a: the second part's limit is 0 where a gate is closed
            e = G * (a * before * la - np.where(beta > 0, a * a * o * x[t] * (la / beta), 0.0))
        dr[t] = e * (1.0 - g)
        dx[t] = G * beta * o
        di[t] = G * beta * x[t] * o * (1.0 - o)
        dlam += np.sum(e, axis=0) * _sigmoid(np.asarray(lam, F())) / np.logaddexp(0.0, lam)
        G = _cut(reset, t, a * G)
    return dx, dr, di, dlam, G
