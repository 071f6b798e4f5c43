"""GPU: how far bf16 outputs of linear attention are from the fp64 recurrence, as the header states it.

A value rounded to bf16 is off by at most 2^-9 of its binade's lower end; over a whole tensor the 2-norm of that error is
2^-7 / sqrt(12 m^2) of the tensor's, m^2 the mean square of a mantissa in 1..2, here at least 1.6 (7/3 if uniform): at most
1.8e-3.  A token alone rounds its output once.  The sequence form also rounds the scores and the carried state as operands of
an output's two products, each part of an output once more: at most sqrt(2) of it, 2.5e-3."""
import numpy as np
import pytest
import torch

from oracle.linattn import linattn_bwd, linattn_fwd
from paper_1912_06680_amd import o5
from tests.gpu_util import banner, host, need_gpu
from tests.test_gpu_linattn import Case

pytestmark = pytest.mark.gpu

ONE, TWO = 1.8e-3, 2.5e-3


def _off(x, ref):
    e = float(np.linalg.norm(host(x) - ref) / np.linalg.norm(ref))
    print(f"    {e:.3e}", flush=True)
    return e


@pytest.mark.parametrize("shape", [(300, 3, 2, 2, 64, 64), (256, 2, 4, 2, 128, 128), (1500, 1, 2, 1, 64, 128)], ids=str)
def test_a_sequence_rounds_twice(shape):
    need_gpu()
    banner(f"linattn rounding {shape}")
    c = Case(True, *shape, resets=0.01, seed=31)
    assert _off(c.fwd()[0], linattn_fwd(**c.ref())[0]) < TWO
    ref = linattn_bwd(dout=host(c.do), dST=host(c.dST), **c.ref())
    for x, y in zip(c.bwd()[:3], ref[:3]):
        assert _off(x, y) < TWO


def test_a_token_rounds_once():
    need_gpu()
    banner("linattn rounding of a token")
    B, nh, nkv, dk, dv = 200, 4, 2, 128, 128
    c = Case(True, 1, B, nh, nkv, dk, dv, resets=0, seed=32)
    ref = linattn_fwd(**c.ref())[0]
    o = torch.empty((B, nh * dv), dtype=torch.bfloat16, device="cuda")
    o5.o5_linattn_step(c.dt, B, nh, nkv, dk, dv, *c.inputs()[:8], None, c.S0.clone(), o, nh * dv)
    assert _off(o[None], ref) < ONE
