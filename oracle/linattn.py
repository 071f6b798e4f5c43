"""Oracle: linear attention with a decay for each head, step by step in fp64.

    S_t = d (1 - reset_t) S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t

Test infrastructure (see the package docstring).  The layouts are the C ABI's: a group of nh / nkv
query heads shares the state of one key/value head.
"""
import numpy as np

from .precision import F


def _split(x, n):
    T, B, w = x.shape
    return np.asarray(x, F()).reshape(T, B, n, w // n)


def linattn_fwd(q, k, v, decay, scale, nh, nkv, S0=None, reset=None):
    """(o [T, B, nh dv], the states S_t [T, B, nkv, dk, dv]) of q [T, B, nh dk], k, v."""
    q, k, v = _split(q, nh), _split(k, nkv), _split(v, nkv)
    T, B, _, dk = q.shape
    dv = v.shape[-1]
    d = np.asarray(decay, F()).reshape(1, nkv, 1, 1)
    S = np.zeros((B, nkv, dk, dv), F()) if S0 is None else np.array(S0, F())
    o = np.empty((T, B, nh, dv), F())
    states = np.empty((T, B, nkv, dk, dv), F())
    for t in range(T):
        if reset is not None:
            S = np.where((np.asarray(reset[t]) != 0).reshape(B, 1, 1, 1), 0.0, S)
        S = d * S + k[t][..., :, None] * v[t][..., None, :]
        states[t] = S
        for h in range(nh):
            o[t, :, h] = scale * np.sum(q[t, :, h, :, None] * S[:, h // (nh // nkv)], axis=-2)
    return o.reshape(T, B, nh * dv), states


def linattn_bwd(q, k, v, decay, scale, nh, nkv, dout, S0=None, reset=None, dST=None):
    """dq, dk, dv and dS0 of J = sum <dout, o> + <dST, S_{T-1}>."""
    _, states = linattn_fwd(q, k, v, decay, scale, nh, nkv, S0, reset)
    q, k, v, do = _split(q, nh), _split(k, nkv), _split(v, nkv), _split(dout, nh)
    T, B, _, dk = q.shape
    dv = v.shape[-1]
    G_ = nh // nkv
    d = np.asarray(decay, F()).reshape(1, nkv, 1, 1)
    G = np.zeros((B, nkv, dk, dv), F()) if dST is None else np.array(dST, F())
    dq, dkey, dval = np.empty_like(q), np.empty_like(k), np.empty_like(v)
    for t in range(T - 1, -1, -1):
        for h in range(nh):
            n = h // G_
            dq[t, :, h] = scale * np.sum(states[t, :, n] * do[t, :, h, None, :], axis=-1)
            G[:, n] += scale * q[t, :, h, :, None] * do[t, :, h, None, :]
        dkey[t] = np.sum(G * v[t][..., None, :], axis=-1)
        dval[t] = np.sum(G * k[t][..., :, None], axis=-2)
        G = d * G
        if reset is not None:
            G = np.where((np.asarray(reset[t]) != 0).reshape(B, 1, 1, 1), 0.0, G)
    return dq.reshape(T, B, -1), dkey.reshape(T, B, -1), dval.reshape(T, B, -1), G
