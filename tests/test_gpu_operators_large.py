"""GPU: the recurrent core's calls on buffers whose offsets pass 32 bits, against the same rows in small buffers."""
import pytest
import torch

from paper_1912_06680_amd import o5
from tests.gpu_util import banner, need_gpu, workspace

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def test_linattn_rows_far_apart():
    """Row strides of 2^24 elements: 260 rows span 8.7 GB, and a 32-bit offset of elements or bytes would wrap."""
    need_gpu()
    banner("linattn rows far apart")
    T, B, n, d, ld = 130, 2, 2, 64, 1 << 24
    size = (o5.O5_BF16, T, B, n, n, d, d)
    decay = torch.tensor([0.9, 0.99], device="cuda")
    g = _gen(0)
    small = [torch.randn((T * B, n * d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(4)]
    S0 = torch.randn((B, n, d, d), generator=g, device="cuda")
    wide = torch.empty(T * B * ld, dtype=torch.bfloat16, device="cuda").view(T * B, ld)
    far = []
    for i, x in enumerate(small):
        far.append(wide[:, i * 1024:i * 1024 + n * d])
        far[-1].copy_(x)
    ws = workspace(max(o5.o5_linattn_fwd_workspace_bytes(*size), o5.o5_linattn_bwd_workspace_bytes(*size)))

    def both(q, k, v, do, ld, outs, ldo):
        ins = (q, ld, k, ld, v, ld, decay, 0.125, S0, None)
        ST, dS0 = torch.empty_like(S0), torch.empty_like(S0)
        o5.o5_linattn_fwd(*size, *ins, outs[0], ldo, ST, ws)
        o5.o5_linattn_bwd(*size, *ins, do, ld, None, outs[1], ldo, outs[2], ldo, outs[3], ldo, dS0, ws)
        return ST, dS0

    ref = [torch.empty_like(x) for x in small]
    states = both(*small, n * d, ref, n * d)
    out = [wide[:, 8192 + i * 1024:8192 + i * 1024 + n * d] for i in range(4)]
    assert all(torch.equal(x, y) for x, y in zip(states, both(*far, ld, out, ld)))
    assert all(torch.equal(x, y) for x, y in zip(ref, out))


def test_linattn_step_many_states():
    """2.4e9 elements of states: the last environment's next to the same environment alone."""
    need_gpu()
    banner("linattn step, 9.7 GB of states")
    B, n, d = 9200, 16, 128
    S = torch.zeros((B, n, d, d), device="cuda")
    g = _gen(1)
    S[-1].normal_(generator=g)
    one = S[-1:].clone()
    q, k, v = (torch.randn((B, n * d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    decay = torch.full((n,), 0.97, device="cuda")
    o, o1 = torch.empty_like(q), torch.empty_like(q[-1:])
    o5.o5_linattn_step(1, B, n, n, d, d, q, n * d, k, n * d, v, n * d, decay, 0.1, None, S, o, n * d)
    q1, k1, v1 = (x[-1:].clone() for x in (q, k, v))
    o5.o5_linattn_step(1, 1, n, n, d, d, q1, n * d, k1, n * d, v1, n * d, decay, 0.1, None, one, o1, n * d)
    assert torch.equal(S[-1:], one) and torch.equal(o[-1:], o1)


def test_resnorm_many_rows():
    """2.3e9 elements: the last rows next to themselves alone."""
    need_gpu()
    banner("resnorm, 2.3e9 elements")
    N, D = 560001, 4096
    x = torch.zeros((N, D), dtype=torch.bfloat16, device="cuda")
    x[-3:].normal_(generator=_gen(2))
    w = torch.rand(D, generator=_gen(3), device="cuda")
    n, r = torch.empty_like(x), torch.empty(N, device="cuda")
    o5.o5_resnorm_fwd(1, 1, N, D, x, None, None, 0, None, None, w, 1e-6, None, n, None, r)
    few, nf = x[-3:].clone(), torch.empty_like(x[-3:])
    o5.o5_resnorm_fwd(1, 1, 3, D, few, None, None, 0, None, None, w, 1e-6, None, nf, None, None)
    assert torch.equal(n[-3:], nf) and not n[:-3].any()
    dx, dw = torch.empty_like(x), torch.empty(D, device="cuda")
    ws = workspace(o5.o5_resnorm_bwd_workspace_bytes(1, 1, N, D))
    o5.o5_resnorm_bwd(1, 1, N, D, x, None, None, 0, None, None, w, None, r, x, n, dx, None, None, 0, None, None, dw, ws)
    dxf, dwf = torch.empty_like(few), torch.empty(D, device="cuda")
    rf = r[-3:].clone()
    o5.o5_resnorm_bwd(1, 1, 3, D, few, None, None, 0, None, None, w, None, rf, few, nf, dxf, None, None, 0, None, None, dwf, ws)
    assert torch.equal(dx[-3:], dxf)
    assert torch.allclose(dw, dwf, rtol=1e-5, atol=1e-5)  # three terms that are not zero, added in another order


def test_adamw_a_tensor_past_32_bits():
    """2^32 + 5 elements with 8-bit moments: the last ones move, and those that a 32-bit index would reach do not."""
    need_gpu()
    banner("adamw, 2^32 + 5 elements")
    n = (1 << 32) + 5
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    me, ve = (torch.zeros(n // 256 + 1, dtype=torch.uint8, device="cuda") for _ in range(2))
    p[-7:] = torch.arange(1.0, 8.0, device="cuda")
    g[-7:] = 0.5
    t = [o5.adamw_tensor(p, g, m, v, me, ve)]
    plan = torch.empty(o5.o5_adamw_plan_bytes(t), dtype=torch.uint8)
    o5.o5_adamw_plan(t, plan)
    o5.o5_adamw_step(plan, plan.cuda(), 1e-2, 0.9, 0.999, 1e-8, 0.0, 0, 1)
    # the first step from zero moments moves by the learning rate
    assert torch.allclose(p[-7:], torch.arange(1.0, 8.0, device="cuda") - 1e-2, atol=1e-6)
    assert not p[:64].any() and not m[:64].any() and not v[:64].any() and (m[-7:] > 0).all() and (v[-7:] > 0).all()
