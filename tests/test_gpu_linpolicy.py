"""GPU: the linear-attention policy as a whole.

The fp32 step's gradients against the same composition in fp64 (products with
the projections by torch, so the tolerance is the LSTM step's 1e-4); the
rollout's single tokens against the training pass over the same steps; training
with 8-bit moments lowers the loss."""
import numpy as np
import pytest
import torch

from oracle.gae import gae, segments_to_samples
from oracle.linattn import linattn_bwd, linattn_fwd
from oracle.ppo import ppo_loss_grad
from oracle.resnorm import resnorm_bwd, resnorm_fwd
from paper_1912_06680_amd import linpolicy
from tests.gpu_util import TOL_BF16, TOL_F32, assert_close, banner, host, need_gpu

pytestmark = pytest.mark.gpu


def _batch(T, B, D, heads, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((T + 1, B, D), generator=g, device="cuda")
    rewards = torch.randn((T, B), generator=g, device="cuda")
    dones = (torch.rand((T, B), generator=g, device="cuda") < 0.05).to(torch.uint8)
    return x, rewards, dones


def test_gradients_of_a_step():
    need_gpu()
    T, B, D, L, nh, heads = 37, 3, 64, 2, 4, (5, 3)
    banner("linpolicy gradients")
    p = linpolicy.LinPolicy(T, B, D, L, nh, heads, dtype="f32", bits=32, lr=0.0)
    for name in p.shapes:  # gains and scales that are not all alike
        if len(p.shapes[name]) == 1:
            p.P[name].add_(0.2 * torch.randn(p.shapes[name], device="cuda", generator=torch.Generator("cuda").manual_seed(len(name))))
    for i in range(L):
        p.S0[i].normal_(generator=torch.Generator("cuda").manual_seed(i))
    x, rewards, dones = _batch(T, B, D, heads, 1)
    act, logp, values = linpolicy.rollout(p, x, dones=dones)
    logp = logp + 0.05 * torch.randn(T * B, device="cuda", generator=torch.Generator("cuda").manual_seed(9))
    p.train_step(x[:T].contiguous(), rewards, dones, values, act, logp)

    P = {k: host(v) for k, v in p.P.items()}
    adv, ret = gae(host(rewards), host(values), host(dones), 0.998, 0.95)
    adv, ret, reset = segments_to_samples(adv, ret, host(dones), T)
    N = T * B
    xs, ns, saved = [host(x[:T]).reshape(N, D)], [], []
    ns.append(resnorm_fwd(xs[0], None, None, None, None, P["w_pre0"], linpolicy.EPS)["n"])
    for i in range(L):
        z = ns[i] @ P[f"W_in{i}"].T
        q, k, v, g = (z[:, j * D:(j + 1) * D] for j in range(4))
        args = dict(q=q.reshape(T, B, D), k=k.reshape(T, B, D), v=v.reshape(T, B, D), decay=host(p.decay), scale=p.scale, nh=nh,
                    nkv=nh, S0=host(p.S0[i]), reset=reset)
        o, states = linattn_fwd(**args)
        assert_close(f"ST{i}", host(p.ST[i]), states[-1], TOL_F32)
        u = o.reshape(N, D) @ P[f"W_out{i}"].T
        out = resnorm_fwd(xs[i], u, g, P[f"w_post{i}"], P[f"rho{i}"], P[f"w_pre{i + 1}"], linpolicy.EPS)
        xs.append(out["xo"])
        ns.append(out["n"])
        saved.append((args, o.reshape(N, D), u, g))
    _, dn, dWp, dbp, _ = ppo_loss_grad(ns[-1], P["Wp"], P["bp"], act.cpu().numpy(), host(logp), adv.reshape(N), ret.reshape(N), heads)
    grads, d = {"Wp": dWp, "bp": dbp}, np.zeros((N, D))
    for i in reversed(range(L)):
        args, o, u, g = saved[i]
        r = resnorm_bwd(xs[i + 1], u, g, P[f"w_post{i}"], P[f"rho{i}"], P[f"w_pre{i + 1}"], linpolicy.EPS, d, dn)
        d = r["dx"]
        grads.update({f"w_post{i}": r["dw_post"], f"rho{i}": r["drho"], f"w_pre{i + 1}": r["dw_pre"], f"W_out{i}": r["du"].T @ o})
        dq, dk, dv, _ = linattn_bwd(dout=(r["du"] @ P[f"W_out{i}"]).reshape(T, B, D), **args)
        dz = np.concatenate([dq.reshape(N, D), dk.reshape(N, D), dv.reshape(N, D), r["dgate"]], 1)
        grads[f"W_in{i}"] = dz.T @ ns[i]
        dn = dz @ P[f"W_in{i}"]
    grads["w_pre0"] = resnorm_bwd(xs[0], None, None, None, None, P["w_pre0"], linpolicy.EPS, d, dn)["dw_pre"]
    assert set(grads) == set(p.shapes)
    for name, g in grads.items():
        assert_close(name, host(p.G[name]), g, TOL_F32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_tokens_follow_the_training_pass(dtype):
    need_gpu()
    banner(f"linpolicy rollout {dtype}")
    T, B, D, heads = 70, 4, 128, (6, 4)
    p = linpolicy.LinPolicy(T, B, D, 2, 2, heads, dtype=dtype)
    x, _, dones = _batch(T, B, D, heads, 3)
    reset = torch.zeros((T, B), dtype=torch.uint8, device="cuda")
    reset[1:] = dones[:T - 1]
    _, _, values = linpolicy.rollout(p, x, dones=dones)
    p.forward(x[:T].contiguous(), reset)
    z = p.n[-1].double() @ p.W["Wp"].double().t() + p.P["bp"].double()
    assert_close("values", host(values[:T]).reshape(-1), host(z[:, -1]), TOL_F32 if dtype == "f32" else TOL_BF16)


@pytest.mark.parametrize("dtype,bits", [("bf16", 8), ("f32", 32)])
def test_training_lowers_the_loss(dtype, bits):
    need_gpu()
    banner(f"linpolicy training {dtype} {bits}")
    T, B, D, heads = 64, 8, 128, (6, 4)
    p = linpolicy.LinPolicy(T, B, D, 2, 2, heads, dtype=dtype, bits=bits, lr=3e-3)
    x, rewards, dones = _batch(T, B, D, heads, 5)
    act, logp, values = linpolicy.rollout(p, x, dones=dones)
    losses = []
    for _ in range(25):
        p.train_step(x[:T].contiguous(), rewards, dones, values, act, logp)
        losses.append(float(p.stats[0]))
    print("   ", losses[0], losses[-1], flush=True)
    assert np.isfinite(losses).all() and losses[-1] < 0.7 * losses[0]
