"""GPU: the fused norms where a block walks several rows of more than 2048 columns, against their definition in fp64.

From 2049 columns on a row takes a whole block, 512 blocks in the forward pass and 256 in the backward pass, so that these
shapes walk 2 to 5 rows a block, at the last of them some blocks with none: the next row's operands in flight, the sums
over a row used again for the next, the column sums carried over the rows.

Tolerances as in test_gpu_resnorm: fp32 1e-5 and bf16 4e-3 of the largest; a column sum adds at most N / 256 + 1 rows in
order, here 5, and then at most 16 blocks of a wave and 16 waves in order: 37 roundings of 2^-24 and those of the terms,
2e-5."""
import numpy as np
import pytest
import torch

from oracle.resnorm import resnorm_bwd, resnorm_fwd
from tests.gpu_util import assert_close, banner, dev_f32, host, need_gpu
from tests.test_gpu_resnorm import EPS, TOL, TYPES, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("form,gate", [("both", True), ("both", False), ("post", True), ("pre", False)])
@pytest.mark.parametrize("shape", [(1100, 2056), (1100, 4096), (1030, 4104), (700, 8192)], ids=str)
def test_several_rows_a_block(shape, form, gate, types):
    need_gpu()
    banner(f"resnorm rows {types} {shape} {form} gate={gate}")
    c = Case(types, *shape, form, gate, wide=gate, seed=21)
    got = c.fwd()
    ref = resnorm_fwd(*c.ref("x", "u", "gate", "w_post", "rho", "w_pre"), EPS)
    assert set(got) == set(ref)
    for k in ref:
        assert_close(k, host(got[k]), ref[k], TOL[got[k].dtype])
    xo = got.get("xo", c.x)
    inverse = lambda z: dev_f32(1.0 / np.sqrt(np.mean(host(z) ** 2, 1) + EPS))  # noqa: E731
    r_post, r_pre = (inverse(c.u) if "r_post" in got else None), (inverse(xo) if "r_pre" in got else None)
    grads = c.bwd(xo, r_post, r_pre)
    gref = resnorm_bwd(host(xo), *c.ref("u", "gate", "w_post", "rho", "w_pre"), EPS, *c.ref("dxo", "dn"))
    assert set(grads) == set(gref)
    for k in gref:
        assert_close(k, host(grads[k]), gref[k], 2e-5 if gref[k].ndim == 1 else TOL[grads[k].dtype])
    for k, v in c.bwd(xo, r_post, r_pre).items():
        assert torch.equal(v, grads[k]), f"{k}: not the same bits twice"
