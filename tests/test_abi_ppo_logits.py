"""The policy loss on logits and the gradients' norm on the CPU: host-side refusals and size queries (no GPU: every call below
fails before any HIP call, or only computes sizes)."""
import ctypes

import pytest
import torch

from paper_1912_06680_amd import o5

F, BF = o5.O5_F32, o5.O5_BF16
P = 16  # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    return o5.lib()


def _heads(*sizes):
    return (ctypes.c_int * len(sizes))(*sizes)


def test_loss_refusals(lib):
    full = dict(dt=BF, N=5, K=2, heads=_heads(6, 3), logits=P, ldl=10, ref=P, ldr=9, act=P, logp_old=P, adv=P, ret=P, weight=None,
                head_mask=None, avail=None, hp=o5.PpoHp(0.2, 1.0, 0.01), kl_coef=0.1, stats=P, logp=None, kl=None, dlogits=P, ldd=10,
                ws=P, n=1 << 20, stream=None)
    call = lambda **kw: lib.o5_ppo_logits_grad(*{**full, **kw}.values())  # noqa: E731
    for bad, status in ((dict(dt=2), 3), (dict(N=0), 2), (dict(N=1 << 30), 2), (dict(K=0), 2), (dict(K=9, heads=_heads(*[1] * 9)), 2),
                        (dict(heads=None), 1), (dict(heads=_heads(0, 3)), 2), (dict(heads=_heads(-5, 30)), 2),
                        (dict(heads=_heads(2 ** 31 - 1, 2 ** 31 - 1)), 2), (dict(heads=_heads(1 << 24, 1)), 2), (dict(logits=None), 1),
                        (dict(logits=20), 4), (dict(ldl=9), 2), (dict(ldl=1 << 31), 2), (dict(ref=8), 4), (dict(ldr=8), 2),
                        (dict(act=None), 1), (dict(logp_old=None), 1), (dict(adv=None), 1), (dict(ret=4), 4), (dict(weight=4), 4),
                        (dict(head_mask=4), 4), (dict(avail=4), 4), (dict(stats=None), 1), (dict(logp=4), 4), (dict(kl=4), 4),
                        (dict(dlogits=None), 1), (dict(ldd=9), 2), (dict(hp=o5.PpoHp(1.0, 1.0, 0.0)), 7),
                        (dict(hp=o5.PpoHp(-0.1, 1.0, 0.0)), 7), (dict(hp=o5.PpoHp(float("nan"), 1.0, 0.0)), 7),
                        (dict(hp=o5.PpoHp(0.2, float("inf"), 0.0)), 7), (dict(kl_coef=float("nan")), 7), (dict(ws=None), 5),
                        (dict(n=16), 5), (dict(ws=8), 4)):
        assert call(**bad) == status, (bad, o5.o5_last_error())
    # without a value column a row needs one column less; without a reference its stride is not looked at
    assert call(ret=None, ldl=8) == 2 and call(ret=None, ldl=9, ldd=9, ws=None) == 5 and call(ref=None, ldr=0, ws=None) == 5


def test_loss_workspaces(lib):
    for heads in ((1,), (30, 8, 32, 4), (1000,), (32000,), (1 << 24,)):
        for N in (1, 60, 32768, (1 << 30) - 1):
            assert 0 < o5.o5_ppo_logits_grad_workspace_bytes(BF, N, heads) <= 1 << 18
    assert o5.o5_ppo_logits_grad_workspace_bytes(BF, 0, (3,)) == 0 and o5.o5_ppo_logits_grad_workspace_bytes(5, 1, (3,)) == 0
    assert lib.o5_ppo_logits_grad_workspace_bytes(BF, 1, 1, None) == 0


def test_norm_refusals(lib):
    t = o5.AdamwTensor(5000, P, P, P, P, None, None, None, 1.0, 0.0, F, 32)
    plan = torch.zeros(o5.o5_adamw_plan_bytes([t]), dtype=torch.uint8)
    o5.o5_adamw_plan([t], plan)
    at, need = plan.data_ptr(), o5.o5_adamw_grad_norm_workspace_bytes(plan)
    assert need > 0 and lib.o5_adamw_grad_norm_workspace_bytes(None) == 0
    assert o5.o5_adamw_grad_norm_workspace_bytes(torch.zeros_like(plan)) == 0
    call = lambda p=at, d=P, m=1.0, c=P, w=P, n=need: lib.o5_adamw_grad_norm(p, d, m, c, w, n, None)  # noqa: E731
    assert call(p=None) == 1 and call(d=None) == 1 and call(c=None) == 1 and call(c=8) == 4 and call(w=None) == 5
    assert call(n=need - 1) == 5 and call(m=0.0) == 7 and call(m=-1.0) == 7 and call(m=float("nan")) == 7 and call(w=8) == 4
    hp = o5.AdamHp(1e-3, 0.9, 0.999, 1e-8, 5.0)
    step = lambda p=at, d=P, hp=hp, c=P, k=1: lib.o5_adamw_step_clipped(p, d, hp, c, 0, k, None)  # noqa: E731
    assert step(p=None) == 1 and step(d=None) == 1 and step(c=None) == 1 and step(c=4) == 4 and step(k=0) == 7
    assert step(hp=o5.AdamHp(-1.0, 0.9, 0.999, 1e-8, 5.0)) == 7 and "o5_adamw_step_clipped" in o5.o5_last_error()
