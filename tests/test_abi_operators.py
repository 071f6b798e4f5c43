"""The recurrent core's entry points on the CPU: host-side refusals and size queries (no GPU: every call below fails before
any HIP call, or only computes sizes)."""
import ctypes

import pytest
import torch

from paper_1912_06680_amd import o5

FN, BF = o5.O5_F32, o5.O5_BF16
P = 16  # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    return o5.lib()


def test_linattn_refusals(lib):
    size = [BF, 16, 4, 8, 4, 64, 128]
    ins = [P, 512, P, 256, P, 512, P, 0.125]
    need = lib.o5_linattn_fwd_workspace_bytes(*size)
    assert need > 0

    def fwd(size=size, ins=ins, o=P, ldo=1024, ST=None, ws=P, n=need):
        return lib.o5_linattn_fwd(*size, *ins, None, None, o, ldo, ST, ws, n, None)

    put = lambda x, i, v: [*x[:i], v, *x[i + 1:]]  # noqa: E731
    for i, bad, status in ((0, 2, 3), (1, 0, 2), (2, -1, 2), (3, 6, 2), (3, 0, 2), (4, 0, 2), (5, 60, 2), (5, 136, 2), (6, 0, 2),
                           (1, 2 ** 31 - 1, 2), (2, 2 ** 22, 2)):
        assert fwd(size=put(size, i, bad)) == status, (i, bad, o5.o5_last_error())
        assert lib.o5_linattn_fwd_workspace_bytes(*put(size, i, bad)) == 0
        assert lib.o5_linattn_bwd_workspace_bytes(*put(size, i, bad)) == 0
    for i, bad, status in ((0, None, 1), (2, None, 1), (4, None, 1), (6, None, 1), (0, 24, 4), (1, 504, 2), (3, 252, 2), (5, 2 ** 31, 2),
                           (7, float("inf"), 7)):
        assert fwd(ins=put(ins, i, bad)) == status, (i, bad, o5.o5_last_error())
    assert fwd(o=None) == 1 and fwd(ldo=1016) == 2 and fwd(ST=20) == 4 and fwd(ws=None) == 5 and fwd(n=need - 1) == 5
    # backward and single token
    bneed = lib.o5_linattn_bwd_workspace_bytes(*size)
    outs = [P, 512, P, 256, P, 512]
    assert lib.o5_linattn_bwd(*size, *ins, None, None, None, 1024, None, *outs, None, P, bneed, None) == 1
    assert lib.o5_linattn_bwd(*size, *ins, None, None, P, 1000, None, *outs, None, P, bneed, None) == 2
    assert lib.o5_linattn_bwd(*size, *ins, None, None, P, 1024, None, *put(outs, 2, None), None, P, bneed, None) == 1
    assert lib.o5_linattn_bwd(*size, *ins, None, None, P, 1024, None, *put(outs, 3, 128), None, P, bneed, None) == 2
    assert lib.o5_linattn_bwd(*size, *ins, None, None, P, 1024, None, *outs, None, P, bneed - 1, None) == 5
    step = [BF, 4, 8, 4, 64, 128]
    assert lib.o5_linattn_step(*step, *ins, None, None, P, 1024, None) == 1
    assert lib.o5_linattn_step(*step, *ins, 20, P, P, 1024, None) == 4
    assert lib.o5_linattn_step(*put(step, 1, 0), *ins, None, P, P, 1024, None) == 2


def test_linattn_workspaces_cover_every_split(lib):
    """Long sequences of few heads are split over time; a launch of several passes never needs more than the query gives."""
    one = lib.o5_linattn_fwd_workspace_bytes(BF, 64, 1, 4, 4, 64, 64)
    many = lib.o5_linattn_fwd_workspace_bytes(BF, 1 << 20, 1, 4, 4, 64, 64)
    assert 0 < one < many < (1 << 26)
    assert lib.o5_linattn_bwd_workspace_bytes(BF, 1 << 20, 1, 4, 4, 64, 64) >= 3 * many
    assert lib.o5_linattn_fwd_workspace_bytes(BF, 256, 2048, 32, 32, 128, 128) <= 256
    assert lib.o5_linattn_bwd_workspace_bytes(FN, 2 ** 20, 1, 64, 8, 8, 8) >= lib.o5_linattn_bwd_workspace_bytes(FN, 2 ** 20, 1, 8, 8, 8, 8)


def test_resnorm_refusals(lib):
    full = dict(xt=BF, dt=BF, N=4, D=64, x=P, u=P, gate=P, ldg=64, w_post=P, rho=P, w_pre=P, eps=1e-6, xo=P, n=P, r_post=None,
                r_pre=None, stream=None)
    call = lambda **kw: lib.o5_resnorm_fwd(*{**full, **kw}.values())  # noqa: E731
    for bad, status in ((dict(xt=7), 3), (dict(dt=FN), 3), (dict(N=0), 2), (dict(N=2 ** 30), 2), (dict(D=4), 2), (dict(D=8200), 2),
                        (dict(eps=-1.0), 7), (dict(eps=float("nan")), 7), (dict(u=None), 7), (dict(u=None, gate=None, w_pre=None), 7),
                        (dict(ldg=32), 2), (dict(x=None), 1), (dict(w_post=None), 1), (dict(xo=None), 1), (dict(n=None), 1),
                        (dict(u=18), 4), (dict(r_pre=8), 4)):
        assert call(**bad) == status, (bad, o5.o5_last_error())
    need = lib.o5_resnorm_bwd_workspace_bytes(BF, BF, 4, 64)
    assert need > 0 and lib.o5_resnorm_bwd_workspace_bytes(BF, BF, 0, 64) == 0
    assert lib.o5_resnorm_bwd_workspace_bytes(BF, BF, 1 << 20, 4096) < (1 << 26)
    back = dict(xt=BF, dt=BF, N=4, D=64, xo=P, u=P, gate=P, ldg=64, w_post=P, rho=P, w_pre=P, r_post=P, r_pre=P, dxo=P, dn=P, dx=P,
                du=P, dgate=P, lddg=64, dw_post=P, drho=P, dw_pre=P, ws=P, n=need, stream=None)
    call = lambda **kw: lib.o5_resnorm_bwd(*{**back, **kw}.values())  # noqa: E731
    for bad, status in ((dict(dxo=None), 1), (dict(dx=None), 1), (dict(dn=None), 1), (dict(xo=None), 1), (dict(r_post=None), 1),
                        (dict(du=None), 1), (dict(dgate=None), 1), (dict(lddg=60), 2), (dict(drho=None), 1), (dict(dw_pre=None), 1),
                        (dict(ws=None), 5), (dict(n=need - 1), 5), (dict(u=None), 7)):
        assert call(**bad) == status, (bad, o5.o5_last_error())


def _tensor(**kw):
    base = dict(n=1000, p=P, g=P, m=P, v=P, m_exp=None, v_exp=None, p_bf16=None, lr_scale=1.0, weight_decay=0.0, g_dt=FN, bits=32)
    return o5.AdamwTensor(*{**base, **kw}.values())


def test_adamw_plans(lib):
    for bad, status in ((dict(n=0), 2), (dict(n=2 ** 40), 2), (dict(g_dt=9), 3), (dict(bits=4), 7), (dict(bits=8), 1), (dict(g=None), 1),
                        (dict(v=24), 4), (dict(p_bf16=2), 4), (dict(lr_scale=-1.0), 7), (dict(weight_decay=float("nan")), 7)):
        assert o5.o5_adamw_plan_bytes([_tensor(), _tensor(**bad)]) == 0
        plan = torch.zeros(1 << 16, dtype=torch.uint8)
        with pytest.raises(o5.O5Error) as e:
            o5.o5_adamw_plan([_tensor(), _tensor(**bad)], plan)
        assert e.value.status == status, bad
        assert not plan.any()
    assert lib.o5_adamw_plan_bytes(0, None) == 0 and lib.o5_adamw_plan_bytes(1, None) == 0
    assert o5.o5_adamw_plan_bytes([_tensor(n=2 ** 40 - 1)] * 3) == 0  # more chunks than a grid takes
    small, large = o5.o5_adamw_plan_bytes([_tensor(n=1)]), o5.o5_adamw_plan_bytes([_tensor(n=10 ** 6), _tensor(n=5)])
    assert 0 < small < large < 1 << 16
    plan = torch.zeros(large, dtype=torch.uint8)
    o5.o5_adamw_plan([_tensor(n=10 ** 6), _tensor(n=5)], plan)
    hp = o5.AdamHp(1e-3, 0.9, 0.999, 1e-8, 5.0)
    at = plan.data_ptr()
    assert lib.o5_adamw_step(None, P, hp, 0, 1, None) == 1 and lib.o5_adamw_step(at, None, hp, 0, 1, None) == 1
    assert lib.o5_adamw_step(at, P, hp, 0, 0, None) == 7
    assert lib.o5_adamw_step(at, P, o5.AdamHp(1e-3, 0.9, 0.999, 0.0, 5.0), 0, 1, None) == 7
    assert lib.o5_adamw_step(torch.zeros(large, dtype=torch.uint8).data_ptr(), P, hp, 0, 1, None) == 7
    assert lib.o5_adamw_moments(at, P, None, P, None) == 1 and lib.o5_adamw_moments(at, P, 8, P, None) == 4


def test_the_structure_is_the_headers():
    """Sizes and offsets of o5_adamw_tensor as a C compiler lays it out on this machine."""
    t = o5.AdamwTensor
    assert ctypes.sizeof(t) == 80 and t.p_bf16.offset == 56 and t.lr_scale.offset == 64 and t.bits.offset == 76
