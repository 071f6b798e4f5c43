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
