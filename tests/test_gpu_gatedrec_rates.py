"""GPU: the gated recurrence's rates at their ends: a rate that is NaN, and rates that forget everything in a step.

Tolerances as in test_gpu_gatedrec."""
import numpy as np
import pytest
import torch

from oracle.gatedrec import gatedrec_bwd, gatedrec_fwd
from paper_1912_06680_amd import o5
from tests.gpu_util import banner, host, need_gpu
from tests.test_gpu_gatedrec import C, TOL_OUT, Case

pytestmark = pytest.mark.gpu

# every way through a call: blocks of few steps, of many and of 4 waves, few segments, many, lanes that walk the sequence
SHAPES = [(1, 2, 24), (100, 9, 256), (300, 33, 512), (290, 70, 1000), (257, 2, 64), (3001, 1, 264), (21, 260, 520)]
ids = lambda s: "x".join(map(str, s))  # noqa: E731


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_a_nan_rate_shows(bf16, shape):
    """A channel whose lam is NaN has NaN for states, gradients and tokens, and no other has."""
    need_gpu()
    banner(f"gatedrec NaN rate bf16={bf16} {shape}")
    c = Case(bf16, *shape, resets=0.05)
    T, B, D = shape
    bad = torch.zeros(D, dtype=torch.bool, device="cuda")
    bad[[3, D - 2]] = True
    h, hT = c.fwd()
    ref = (h, hT, *c.bwd())
    c.lam[bad] = float("nan")
    h, hT = c.fwd()
    got = (h, hT, *c.bwd())
    for name, x, y in zip(("h", "hT", "dx", "dr", "di", "dlam", "dh0"), got, ref):
        # (a reset at the first step leaves nothing of dh0)
        cut = torch.zeros(x.shape[:-1], dtype=torch.bool, device="cuda") if name != "dh0" else c.reset[0] != 0
        assert torch.isnan(x[..., bad][~cut]).all(), name
        assert torch.equal(x[..., ~bad], y[..., ~bad]), name
    S, out = c.h0.clone(), torch.empty((B, D), dtype=c.et, device="cuda")
    x, r, i = (a[0].clone(memory_format=torch.contiguous_format) for a in (c.x, c.r, c.i))
    o5.o5_gatedrec_step(c.dt, B, D, x, D, r, D, i, D, c.lam, C, None, S, out, D)
    assert torch.isnan(S[:, bad]).all() and torch.isnan(out[:, bad]).all()
    assert torch.isfinite(S[:, ~bad]).all() and torch.isfinite(out[:, ~bad]).all()


# A decay a = e^-y is off by y times what y is, 20 steps of 2^-24 (8 for a gate's exponential and reciprocal, 8 for a rate,
# 4 for their product in binary logs): for y of 30 that is 4e-5 of a, however small a is, and TOL_OUT holds in each channel by
# itself.
FAST = np.linspace(2.0, 60.0, 64)


def fast_rates(D):
    return np.log(np.expm1(np.resize(FAST, D) / C))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_gradients_of_channels_that_forget_in_a_step(bf16, shape):
    """dr, dlam and dh0 go with a, here e^-1 to e^-30 in its channel."""
    need_gpu()
    banner(f"gatedrec gradients of fast rates bf16={bf16} {shape}")
    T, B, D = shape
    c = Case(bf16, *shape, resets=0.05, lam=fast_rates(D))
    c.r.mul_(0.02)  # (gates near one half)
    c.fwd()
    got = [host(x) for x in c.bwd()]
    ref = gatedrec_bwd(dh=host(c.dh), dhT=host(c.dhT), **c.ref())
    tol = {"dx": TOL_OUT[bf16], "dr": TOL_OUT[bf16], "di": TOL_OUT[bf16], "dh0": TOL_OUT[False]}
    for name, x, y in zip(("dx", "dr", "di", "dlam", "dh0"), got, ref):
        if name != "dlam":
            size = np.max(np.abs(y.reshape(-1, D)), axis=0)
            worst = float(np.max(np.max(np.abs(x - y).reshape(-1, D), axis=0) / np.where(size > 0, size, 1.0)))
            print(f"    {name}: {worst:.2e} of its channel's largest", flush=True)
            assert worst <= tol[name], name
    lam = host(c.lam)
    terms = (np.abs(ref[1]) * (1.0 + np.exp(host(c.r)))).sum((0, 1)) / ((1.0 + np.exp(-lam)) * np.logaddexp(0.0, lam))
    worst = float(np.max(np.abs(got[3] - ref[3]) / terms))
    print(f"    dlam: {worst:.2e} of its channel's terms", flush=True)
    assert worst <= TOL_OUT[False]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_a_state_that_is_not_fed_decays_as_it_should(bf16, shape):
    """Every third step takes something in; between, a state is a h whatever a.

    Each of a state's terms, the inputs and h0 times the decays since, holds the bound by itself; where they cancel their sum
    does not.  |x| and |h0| in their places give the sum of the terms' sizes, which decays as the state does."""
    need_gpu()
    banner(f"gatedrec unfed states bf16={bf16} {shape}")
    T, B, D = shape
    c = Case(bf16, *shape, resets=0.05, lam=fast_rates(D))
    c.r.mul_(0.02)
    c.x[0::3] = 0.0
    c.x[1::3] = 0.0
    if not bf16:
        c.x.mul_(1e3)
    h, hT = c.fwd()
    args = c.ref()
    ref, size = gatedrec_fwd(**args), gatedrec_fwd(**{**args, "x": np.abs(args["x"]), "h0": np.abs(args["h0"])})
    size = np.maximum(size, 1e-30)  # (what a state below loses is no rounding: fp32 ends there)
    for name, x, y, z, tol in (("h", host(h), ref, size, TOL_OUT[bf16]), ("hT", host(hT), ref[-1], size[-1], TOL_OUT[False])):
        worst = float(np.max(np.abs(x - y) / z))
        print(f"    {name}: {worst:.2e} of its terms", flush=True)
        assert worst <= tol, name
