"""Oracle: the clipped policy loss with value, entropy and KL terms on logits, in fp64.

Test infrastructure (see the package docstring).
"""
import numpy as np

from .precision import F


def _log_softmax(z):
    """Over the last axis; -inf stays -inf."""
    m = np.max(z, axis=-1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore"):
        return z - m - np.log(np.sum(np.exp(z - m), axis=-1, keepdims=True))


def ppo_logits_grad(logits, act, logp_old, adv, head_sizes, ref=None, ret=None, weight=None, head_mask=None, avail=None,
                    clip_eps=0.2, vf_coef=1.0, ent_coef=0.01, kl_coef=0.0):
    """(stats [9], dlogits, logp [N], kl [N])."""
    z = np.asarray(logits, F())
    N, A = z.shape[0], sum(head_sizes)
    w = np.full(N, 1.0 / N) if weight is None else np.asarray(weight, F())
    dz = np.zeros(z.shape, F())
    logp, kls, terms = np.zeros(N), np.zeros(N), np.zeros((N, 8))
    for n in range(N):
        if w[n] == 0.0:
            continue
        heads, logpi, ent, kl, at = [], 0.0, 0.0, 0.0, 0
        for k, size in enumerate(head_sizes):
            seen = np.arange(at, at + size)
            at += size
            if head_mask is not None and not head_mask[n, k]:
                continue
            if avail is not None:
                seen = seen[avail[n, seen] != 0]
            cols = seen[z[n, seen] != -np.inf]
            if cols.size == 0:
                continue
            lp = _log_softmax(z[n, cols])
            p = np.exp(lp)
            a = at - size + int(act[n, k]) if 0 <= act[n, k] < size else -1
            taken = cols == a
            logpi += float(lp[taken][0]) if taken.any() else -np.inf
            S = -np.sum(np.where(p > 0, p * lp, 0.0))
            far, D = 0.0, 0.0
            if ref is not None:
                # (the reference's normaliser runs over every available choice)
                y = np.asarray(ref[n], F())
                lq = _log_softmax(y[seen])[np.searchsorted(seen, cols)]
                far = np.where(p > 0, lp - lq, 0.0)
                D = np.sum(np.where(p > 0, p * far, 0.0))
            ent, kl = ent + S, kl + D
            heads.append((cols, lp, p, taken, S, far, D))
        with np.errstate(over="ignore", invalid="ignore"):
            dlog = logpi - float(logp_old[n])
            r, A_n = np.exp(dlog), float(adv[n])
            surr = min(r * A_n, np.clip(r, 1.0 - clip_eps, 1.0 + clip_eps) * A_n)
            flow = (A_n >= 0 and r <= 1.0 + clip_eps) or (A_n < 0 and r >= 1.0 - clip_eps)
            g = -r * A_n * w[n] if flow else 0.0
            for cols, lp, p, taken, S, far, D in heads:
                d = g * (taken.astype(F()) - p)
                d += w[n] * np.where(p > 0, p * (ent_coef * (lp + S) + (kl_coef * (far - D) if kl_coef else 0.0)), 0.0)
                dz[n, cols] = d
            err = 0.0
            if ret is not None:
                err = z[n, A] - float(ret[n])
                dz[n, A] = 2.0 * vf_coef * w[n] * err
            loss = -surr + vf_coef * err ** 2 - ent_coef * ent + (kl_coef * kl if kl_coef else 0.0)
            terms[n] = (-surr, err ** 2, ent, abs(r - 1.0) > clip_eps, np.expm1(dlog) - dlog, r, 0.0, kl)
            terms[n] *= w[n]
            terms[n, 6] = not np.isfinite(loss)
        logp[n], kls[n] = logpi, kl
    s = terms.sum(0)
    total = s[0] + vf_coef * s[1] - ent_coef * s[2] + (kl_coef * s[7] if kl_coef else 0.0)
    return np.concatenate([[total], s]), dz, logp, kls
