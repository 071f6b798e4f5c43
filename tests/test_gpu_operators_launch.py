"""GPU: calls of more blocks than one launch can hold.

HIP takes no launch of 2^32 threads or more in a dimension, so that such a
call goes out in several.  Every element of the outputs is compared, those on
both sides of a launch's end among them.  Tolerances as in test_gpu_linattn
(bf16 outputs 1e-2 of the largest) and test_gpu_operators_large."""
import pytest
import torch

from paper_1912_06680_amd import o5
from tests.gpu_util import banner, need_gpu, workspace

pytestmark = pytest.mark.gpu


def _near(x, ref):
    assert float((x.float() - ref).abs().max()) <= 1e-2 * float(ref.abs().max())


def _rows(g, B, w):
    return torch.randn((B, w), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def test_linattn_forward_of_8_million_states():
    """One step of 2^23 + 5 states of 8 x 72, blocks of 512 threads: o = scale (q . k) v."""
    need_gpu()
    banner("linattn forward, 2^23 + 5 states")
    B, dk, dv = (1 << 23) + 5, 8, 72
    g = torch.Generator("cuda").manual_seed(0)
    q, k, v = _rows(g, B, dk), _rows(g, B, dk), _rows(g, B, dv)
    o = torch.full((B, dv), 7.0, dtype=torch.bfloat16, device="cuda")
    size = (o5.O5_BF16, 1, B, 1, 1, dk, dv)
    ws = workspace(o5.o5_linattn_fwd_workspace_bytes(*size))
    o5.o5_linattn_fwd(*size, q, dk, k, dk, v, dv, torch.ones(1, device="cuda"), 0.5, None, None, o, dv, None, ws)
    _near(o, 0.5 * (q.float() * k.float()).sum(1, keepdim=True) * v.float())


def test_linattn_backward_of_8_million_states():
    """One step of 2^20 samples with 8 states of 16 x 16, three passes each: with G = scale q do^T, dq = scale k (v . do),
    dk = G v, dv = G^T k."""
    need_gpu()
    banner("linattn backward, 2^20 samples of 8 states")
    B, n, d = 1 << 20, 8, 16
    g = torch.Generator("cuda").manual_seed(1)
    q, k, v, do = (_rows(g, B, n * d) for _ in range(4))
    out = [torch.full((B, n * d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    size = (o5.O5_BF16, 1, B, n, n, d, d)
    ws = workspace(o5.o5_linattn_bwd_workspace_bytes(*size))
    o5.o5_linattn_bwd(*size, q, n * d, k, n * d, v, n * d, torch.ones(n, device="cuda"), 0.5, None, None, do, n * d, None,
                      out[0], n * d, out[1], n * d, out[2], n * d, None, ws)
    q, k, v, do = (x.view(B, n, d).float() for x in (q, k, v, do))
    dot = lambda a, b: 0.5 * (a * b).sum(-1, keepdim=True)  # noqa: E731
    for x, ref in zip(out, (k * dot(v, do), q * dot(do, v), do * dot(q, k))):
        _near(x.view(B, n, d), ref)


def test_linattn_step_of_16_million_states():
    """The most states that a call takes, one short of 2^24, of 8 x 8, in place."""
    need_gpu()
    banner("linattn step, 2^24 - 1 states")
    B, d = (1 << 24) - 1, 8
    g = torch.Generator("cuda").manual_seed(2)
    q, k, v = (_rows(g, B, d) for _ in range(3))
    S = torch.ones((B, 1, d, d), device="cuda")
    o = torch.empty((B, d), dtype=torch.bfloat16, device="cuda")
    o5.o5_linattn_step(o5.O5_BF16, B, 1, 1, d, d, q, d, k, d, v, d, torch.full((1,), 0.5, device="cuda"), 1.0, None, S, o, d)
    for a in range(0, B, 1 << 22):  # (in parts: the states are 4 GB)
        qa, ka, va = (x[a:a + (1 << 22)].float() for x in (q, k, v))
        ref = 0.5 + ka[:, :, None] * va[:, None, :]
        assert torch.allclose(S[a:a + (1 << 22), 0], ref, rtol=1e-6, atol=1e-6)
        _near(o[a:a + (1 << 22)], (qa[:, :, None] * ref).sum(1))


def test_adamw_more_chunks_than_a_launch():
    """2^34 + 3079 elements, 8-bit moments: the first step from zero moments moves every parameter by the learning rate, and
    every moment is the gradient's, to the eighth that a code resolves."""
    need_gpu()
    banner("adamw, 2^34 + 3079 elements")
    n = (1 << 34) + 3 * 1024 + 7
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    me, ve = (torch.zeros((n + 255) // 256, dtype=torch.uint8, device="cuda") for _ in range(2))
    t = [o5.adamw_tensor(p, g, m, v, me, ve)]
    plan = torch.empty(o5.o5_adamw_plan_bytes(t), dtype=torch.uint8)
    o5.o5_adamw_plan(t, plan)
    plan_dev = plan.cuda()
    o5.o5_adamw_step(plan, plan_dev, 1e-2, 0.9, 0.999, 1e-8, 0.0, 0, 1)
    for a in range(0, n, 1 << 30):
        assert torch.all((p[a:a + (1 << 30)] + 1e-2).abs_() <= 1e-6), a
    # (the values of the moments need the moments and their exponents alone)
    size = (n + 255) // 256 * 256
    del p, g
    torch.cuda.empty_cache()
    mo, vo = torch.zeros(size, device="cuda"), torch.zeros(size, device="cuda")
    o5.o5_adamw_moments(plan, plan_dev, mo, vo)
    for x, value in ((mo, 0.05), (vo, 2.5e-4)):
        for a in range(0, n, 1 << 30):
            assert torch.all((x[a:min(n, a + (1 << 30))] / value - 1).abs_() <= 0.125), a
    del m, v, me, ve, mo, vo, x
    torch.cuda.empty_cache()
