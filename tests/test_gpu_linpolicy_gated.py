"""GPU: the policy whose blocks carry a gated recurrence, held near a reference policy and to a gradient norm.

The fp32 step's gradients against the same composition in fp64 (products by torch, so the LSTM step's 1e-4); single tokens
against the training pass; the clip against the definition on the gradients that the step left."""
import numpy as np
import pytest
import torch

from oracle.adamw import adamw_step
from oracle.gae import gae, segments_to_samples
from oracle.gatedrec import gatedrec_bwd, gatedrec_fwd
from oracle.ppo_logits import ppo_logits_grad
from oracle.resnorm import resnorm_bwd, resnorm_fwd
from paper_1912_06680_amd import linpolicy
from tests.gpu_util import TOL_BF16, TOL_F32, assert_close, banner, host, need_gpu
from tests.test_gpu_linpolicy import _batch

pytestmark = pytest.mark.gpu


def _policy(T, B, D, L, heads, seed=0, **kw):
    p = linpolicy.LinPolicy(T, B, D, L, 1, heads, core="gatedrec", seed=seed, **kw)
    for name, shape in p.shapes.items():  # gains, scales and rates that are not all alike
        if len(shape) == 1:
            g = torch.Generator("cuda").manual_seed(len(name) + seed)
            p.P[name].add_(0.2 * torch.randn(shape, device="cuda", generator=g))
    for i in range(L):
        p.S0[i].normal_(generator=torch.Generator("cuda").manual_seed(i))
    return p


def _step(p, seed, ref=True):
    """One training step; what it was given."""
    T, B, D = p.T, p.B, p.D
    x, rewards, dones = _batch(T, B, D, p.head_sizes, seed)
    act, logp, values = linpolicy.rollout(p, x, dones=dones)
    logp = logp + 0.05 * torch.randn(T * B, device="cuda", generator=torch.Generator("cuda").manual_seed(9))
    z = None
    if ref:
        other = _policy(T, B, D, p.layers, p.head_sizes, seed=5, dtype="bf16" if p.bf16 else "f32")
        other.forward(x[:T].contiguous(), None)
        z = other.logits()
    p.train_step(x[:T].contiguous(), rewards, dones, values, act, logp, ref=z)
    return x, rewards, dones, act, logp, values, z


@pytest.mark.parametrize("kl_coef", [0.0, 0.3])
@pytest.mark.parametrize("T,B", [(37, 3), (300, 2)])
def test_gradients_of_a_step(kl_coef, T, B):
    need_gpu()
    D, L, heads = 64, 2, (5, 3)
    banner(f"gated policy gradients kl_coef={kl_coef} T={T}")
    p = _policy(T, B, D, L, heads, dtype="f32", bits=32, lr=0.0, kl_coef=kl_coef)
    x, rewards, dones, act, logp, values, z = _step(p, 1, kl_coef > 0)

    P = {k: host(v) for k, v in p.P.items()}
    adv, ret = gae(host(rewards), host(values), host(dones), 0.998, 0.95)
    adv, ret, reset = segments_to_samples(adv, ret, host(dones), T)
    N = T * B
    xs, ns, saved = [host(x[:T]).reshape(N, D)], [], []
    ns.append(resnorm_fwd(xs[0], None, None, None, None, P["w_pre0"], linpolicy.EPS)["n"])
    for i in range(L):
        w = ns[i] @ P[f"W_in{i}"].T
        a, r, c, g = (w[:, j * D:(j + 1) * D] for j in range(4))
        args = dict(x=a.reshape(T, B, D), r=r.reshape(T, B, D), i=c.reshape(T, B, D), lam=P[f"lam{i}"], c=linpolicy.RATE,
                    h0=host(p.S0[i]), reset=reset)
        h = gatedrec_fwd(**args)
        assert_close(f"ST{i}", host(p.ST[i]), h[-1], TOL_F32)
        u = h.reshape(N, D) @ P[f"W_out{i}"].T
        out = resnorm_fwd(xs[i], u, g, P[f"w_post{i}"], P[f"rho{i}"], P[f"w_pre{i + 1}"], linpolicy.EPS)
        xs.append(out["xo"])
        ns.append(out["n"])
        saved.append((args, h.reshape(N, D), u, g))
    stats, dz, _, _ = ppo_logits_grad(ns[-1] @ P["Wp"].T + P["bp"], act.cpu().numpy(), host(logp), adv.reshape(N), heads,
                                      ref=host(z) if kl_coef else None, ret=ret.reshape(N), kl_coef=kl_coef)
    assert abs(float(p.stats[0]) - stats[0]) <= TOL_F32 * (1 + abs(stats[0]))
    if kl_coef:
        assert abs(float(p.stats[8]) - stats[8]) <= TOL_F32 * (1 + stats[8])
    grads = {"Wp": dz.T @ ns[-1], "bp": dz.sum(0)}
    d, dn = np.zeros((N, D)), dz @ P["Wp"]
    for i in reversed(range(L)):
        args, h, u, g = saved[i]
        r = resnorm_bwd(xs[i + 1], u, g, P[f"w_post{i}"], P[f"rho{i}"], P[f"w_pre{i + 1}"], linpolicy.EPS, d, dn)
        d = r["dx"]
        grads.update({f"w_post{i}": r["dw_post"], f"rho{i}": r["drho"], f"w_pre{i + 1}": r["dw_pre"], f"W_out{i}": r["du"].T @ h})
        da, dr, di, dlam, _ = gatedrec_bwd(dh=(r["du"] @ P[f"W_out{i}"]).reshape(T, B, D), **args)
        grads[f"lam{i}"] = dlam
        dw = np.concatenate([da.reshape(N, D), dr.reshape(N, D), di.reshape(N, D), r["dgate"]], 1)
        grads[f"W_in{i}"] = dw.T @ ns[i]
        dn = dw @ P[f"W_in{i}"]
    grads["w_pre0"] = resnorm_bwd(xs[0], None, None, None, None, P["w_pre0"], linpolicy.EPS, d, dn)["dw_pre"]
    assert set(grads) == set(p.shapes)
    for name, g in grads.items():
        assert_close(name, host(p.G[name]), g, TOL_F32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_tokens_follow_the_training_pass(dtype):
    need_gpu()
    banner(f"gated policy rollout {dtype}")
    T, B, D, heads = 70, 4, 128, (6, 4)
    p = linpolicy.LinPolicy(T, B, D, 2, 2, heads, dtype=dtype, core="gatedrec")
    x, _, dones = _batch(T, B, D, heads, 3)
    reset = torch.zeros((T, B), dtype=torch.uint8, device="cuda")
    reset[1:] = dones[:T - 1]
    _, _, values = linpolicy.rollout(p, x, dones=dones)
    p.forward(x[:T].contiguous(), reset)
    z = p.n[-1].double() @ p.W["Wp"].double().t() + p.P["bp"].double()
    assert_close("values", host(values[:T]).reshape(-1), host(z[:, -1]), TOL_F32 if dtype == "f32" else TOL_BF16)


@pytest.mark.parametrize("core", ["gatedrec", "linattn"])
def test_a_step_with_clipped_gradients(core):
    """The update is AdamW's on the gradients that the step left, times the factor that their norm gives."""
    need_gpu()
    banner(f"policy step with clipped gradients, {core}")
    T, B, D, heads = 40, 3, 64, (5, 3)
    p = linpolicy.LinPolicy(T, B, D, 2, 2, heads, dtype="bf16", bits=32, lr=1e-2, core=core, max_norm=0.05, weight_decay=0.0)
    x, rewards, dones = _batch(T, B, D, heads, 7)
    act, logp, values = linpolicy.rollout(p, x, dones=dones)
    before = {k: host(v) for k, v in p.P.items()}
    p.train_step(x[:T].contiguous(), rewards, dones, values, act, logp)
    norm = float(np.sqrt(sum(np.sum(host(g) ** 2) for g in p.G.values())))
    assert abs(float(p.clip[0]) - norm) <= 1e-6 * norm and norm > 0.05
    factor = float(np.float32(0.05)) / norm
    assert abs(float(p.clip[1]) - factor) <= 1e-6 * factor
    for k, old in before.items():
        zero = np.zeros_like(old)
        new, _, _ = adamw_step(old, zero, zero, host(p.G[k]) * factor, float(np.float32(1e-2)), 0.9, float(np.float32(0.999)), 1e-8, 5.0,
                               0.0, 1)
        assert np.max(np.abs(host(p.P[k]) - new)) <= 1e-4 * 1e-2 + 1e-6 * np.max(np.abs(new)), k


def test_a_gradient_that_is_not_finite_leaves_the_policy_as_it_was():
    need_gpu()
    banner("policy step with a gradient that is not finite")
    T, B, D, heads = 20, 2, 64, (5, 3)
    p = linpolicy.LinPolicy(T, B, D, 1, 1, heads, core="gatedrec", max_norm=1.0)
    x, rewards, dones = _batch(T, B, D, heads, 7)
    act, logp, values = linpolicy.rollout(p, x, dones=dones)
    before = [v.clone() for v in p.P.values()]
    rewards[3, 1] = float("inf")
    p.train_step(x[:T].contiguous(), rewards, dones, values, act, logp)
    assert float(p.clip[1]) == 0.0 and all(torch.equal(a, b) for a, b in zip(before, p.P.values()))


@pytest.mark.parametrize("core", ["gatedrec", "linattn"])
def test_the_command_runs(core, capsys):
    need_gpu()
    banner(f"linpolicy command {core}")
    linpolicy.main(core, steps=2)
    assert capsys.readouterr().out.count("loss") == 2
