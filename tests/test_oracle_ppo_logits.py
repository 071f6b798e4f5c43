"""Pins of the oracle of the policy loss on logits: PyTorch's distributions and automatic differentiation in fp64, the loss
through the heads' product that it shares with o5_ppo_loss_grad, padding, and what masks hide."""
import numpy as np
import pytest
import torch

from oracle.ppo import ppo_loss_grad
from oracle.ppo_logits import ppo_logits_grad

HEADS = (5, 3, 1)


def _inputs(seed, N=7, value=True, avail=True):
    g = np.random.Generator(np.random.PCG64(seed))
    A = sum(HEADS)
    z, y = g.standard_normal((N, A + value)), g.standard_normal((N, A))
    av = (g.random((N, A)) < 0.7).astype(np.uint8) if avail else None
    act = np.empty((N, len(HEADS)), np.int32)
    at = 0
    for k, n in enumerate(HEADS):
        act[:, k] = g.integers(0, n, N)
        if avail:
            av[np.arange(N), at + act[:, k]] = 1
        at += n
    return dict(logits=z, act=act, logp_old=-2.5 + 0.3 * g.standard_normal(N), adv=g.standard_normal(N), head_sizes=HEADS, ref=y,
                ret=g.standard_normal(N) if value else None, weight=g.random(N), avail=av,
                head_mask=(g.random((N, len(HEADS))) < 0.8).astype(np.uint8), kl_coef=0.3, ent_coef=0.05, vf_coef=0.7)


@pytest.mark.parametrize("avail", [False, True])
@pytest.mark.parametrize("value", [False, True])
def test_loss_and_gradient_against_torch(value, avail):
    c = _inputs(0, value=value, avail=avail)
    stats, dz, logp, kl = ppo_logits_grad(**c)
    T = lambda a: torch.tensor(a, dtype=torch.float64)  # noqa: E731
    z, w = T(c["logits"]).requires_grad_(), T(c["weight"])
    lp, S, D, at = 0.0, 0.0, 0.0, 0
    for k, n in enumerate(HEADS):
        hide = torch.zeros(7, n) if not avail else torch.where(T(c["avail"][:, at:at + n]) != 0, 0.0, -1e9)
        m = T(c["head_mask"][:, k])
        p, q = (torch.distributions.Categorical(logits=x[:, at:at + n] + hide) for x in (z, T(c["ref"])))
        lp = lp + m * p.log_prob(torch.tensor(c["act"][:, k]))
        S = S + m * p.entropy()
        D = D + m * torch.distributions.kl_divergence(p, q)
        at += n
    r = torch.exp(lp - T(c["logp_old"]))
    adv = T(c["adv"])
    loss = -torch.minimum(r * adv, r.clamp(0.8, 1.2) * adv) - 0.05 * S + 0.3 * D
    if value:
        loss = loss + 0.7 * (z[:, at] - T(c["ret"])) ** 2
    total = (w * loss).sum()
    total.backward()
    assert abs(stats[0] - float(total)) < 1e-12 and stats[7] == 0
    assert np.allclose(dz, z.grad.numpy(), rtol=1e-10, atol=1e-12)
    assert np.allclose(logp, lp.detach().numpy()) and np.allclose(kl, D.detach().numpy())
    assert abs(stats[3] - float((w * S).sum())) < 1e-12 and abs(stats[8] - float((w * D).sum())) < 1e-12


def test_it_is_the_loss_through_the_heads_product():
    """Without a reference and with even weights: the statistics and the bias gradient of oracle.ppo."""
    c = _inputs(1, N=6)
    N, A1 = 6, sum(HEADS) + 1
    stats, dz, _, _ = ppo_logits_grad(**{**c, "ref": None, "weight": None, "kl_coef": 0.0})
    out = ppo_loss_grad(c["logits"], np.eye(A1), np.zeros(A1), c["act"], c["logp_old"], c["adv"], c["ret"], HEADS,
                        head_mask=c["head_mask"], avail=c["avail"], clip_eps=0.2, vf_coef=0.7, ent_coef=0.05)
    assert np.allclose(out[1], dz, rtol=1e-12, atol=1e-14)
    assert np.allclose(out[0]["total"] if isinstance(out[0], dict) else out[0][0], stats[0], rtol=1e-12)


def test_padding_and_masks_hide_everything():
    c = _inputs(2)
    c["weight"][[1, 4]] = 0.0
    ref = ppo_logits_grad(**c)
    for k in ("logits", "ref", "logp_old", "adv", "ret"):
        c[k][[1, 4]] = np.nan
    hidden = c["avail"] == 0
    c["logits"][:, :-1][hidden], c["ref"][hidden] = np.inf, np.nan
    for a, b in zip(ref, ppo_logits_grad(**c)):
        assert np.array_equal(a, b)
    assert not ref[1][[1, 4]].any() and not ref[1][:, :-1][hidden].any()


def test_rows_without_a_choice_and_impossible_actions():
    c = _inputs(3)
    c["head_mask"][:] = 1
    c["avail"][2, :5] = 0                     # no choice left in head 0
    c["act"][3, 1] = -1
    stats, dz, logp, kl = ppo_logits_grad(**c)
    assert not dz[2, :5].any() and np.isfinite(logp[2]) and logp[3] == -np.inf and np.isfinite(dz).all()
    c["logits"][0, :5] = -np.inf              # as if none were available
    c["logits"][5, 0] = -np.inf
    _, dz, logp, kl = ppo_logits_grad(**c)
    assert np.isfinite(dz).all() and not dz[0, :5].any() and dz[5, 0] == 0
