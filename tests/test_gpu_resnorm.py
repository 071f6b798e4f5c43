"""GPU: the fused norms against their definition in fp64.

Tolerances (max|Y - ref| / max|ref| per output): fp32 outputs come from sums of
up to 8192 terms added in trees of at most 32 terms in a row, and from products
and square roots rounded to 2^-24 each, the gate from a reciprocal and an
exponential of about 1 ulp: 1e-5.  A bf16 output is rounded to 2^-9 of itself:
4e-3 with the terms above.  Column sums add the rows of a group in order, at
most N / 256 + 1 of them, and then the groups: 2e-5 at the sizes here."""
import numpy as np
import pytest
import torch

from oracle.resnorm import resnorm_bwd, resnorm_fwd
from paper_1912_06680_amd import o5
from tests.gpu_util import assert_close, banner, dev_f32, host, need_gpu, workspace

pytestmark = pytest.mark.gpu

EPS = 1e-6
TYPES = {"f32": (0, 0), "mixed": (0, 1), "bf16": (1, 1)}
TORCH = (torch.float32, torch.bfloat16)
TOL = {torch.float32: 1e-5, torch.bfloat16: 4e-3}


class Case:
    def __init__(self, types, N, D, form, gate, wide=False, seed=0, scale=1.0):
        r = np.random.Generator(np.random.PCG64(seed))
        self.xt, self.dt = TYPES[types]
        self.N, self.D = N, D
        x, e = TORCH[self.xt], TORCH[self.dt]
        post, pre = form != "pre", form != "post"
        z = lambda t, *s: torch.from_numpy(r.standard_normal(s).astype(np.float32) * np.float32(scale)).to(t).cuda()  # noqa: E731
        w = lambda c: dev_f32(c + 0.3 * r.standard_normal(D))  # noqa: E731
        self.x = z(x, N, D)
        self.u = z(e, N, D) if post else None
        self.gate = None
        if gate:  # part of a wider buffer: a row stride above D
            self.ldg = D + 16 if wide else D
            self.gate = torch.full((N, self.ldg), float("nan"), dtype=e, device="cuda")[:, 8 * wide:8 * wide + D]
            self.gate.copy_(z(e, N, D))
        else:
            self.ldg = 0
        self.w_post, self.rho = (w(1.0), w(0.5)) if post else (None, None)
        self.w_pre = w(1.0) if pre else None
        self.dxo, self.dn = z(x, N, D), z(e, N, D) if pre else None

    def blank(self, t, *s):
        return torch.full(s, 7.0, dtype=t, device="cuda")

    def fwd(self, x=None, xo=None, stats=True):
        post, pre = self.u is not None, self.w_pre is not None
        N, D = self.N, self.D
        x = self.x if x is None else x
        xo = xo if xo is not None or not post else self.blank(self.x.dtype, N, D)
        n = self.blank(TORCH[self.dt], N, D) if pre else None
        r_post = self.blank(torch.float32, N) if post and stats else None
        r_pre = self.blank(torch.float32, N) if pre and stats else None
        o5.o5_resnorm_fwd(self.xt, self.dt, N, D, x, self.u, self.gate, self.ldg, self.w_post, self.rho, self.w_pre, EPS, xo,
                          n, r_post, r_pre)
        return {k: v for k, v in dict(xo=xo, n=n, r_post=r_post, r_pre=r_pre).items() if v is not None}

    def bwd(self, xo, r_post, r_pre):
        post, pre = self.u is not None, self.w_pre is not None
        N, D = self.N, self.D
        b = self.blank
        e = TORCH[self.dt]
        out = dict(dx=b(self.x.dtype, N, D), du=b(e, N, D) if post else None,
                   dgate=torch.empty_strided((N, D), (max(self.ldg, 8), 1), dtype=e, device="cuda") if self.ldg else None,
                   dw_post=b(torch.float32, D) if post else None, drho=b(torch.float32, D) if post else None,
                   dw_pre=b(torch.float32, D) if pre else None)
        ws = workspace(o5.o5_resnorm_bwd_workspace_bytes(self.xt, self.dt, N, D))
        o5.o5_resnorm_bwd(self.xt, self.dt, N, D, xo if pre else None, self.u, self.gate, self.ldg, self.w_post, self.rho,
                          self.w_pre, r_post, r_pre, self.dxo, self.dn, out["dx"], out["du"], out["dgate"], self.ldg,
                          out["dw_post"], out["drho"], out["dw_pre"], ws)
        return {k: v for k, v in out.items() if v is not None}

    def ref(self, *names):
        return [None if getattr(self, n) is None else host(getattr(self, n)) for n in names]


SHAPES = [(1, 8), (3, 64), (7, 520), (60, 1024), (5, 1000), (130, 1032), (2, 2048), (33, 2056), (9, 4096), (4, 4104), (3, 8192),
          (1100, 72), (1030, 1032)]
FORMS = [("both", True), ("both", False), ("post", True), ("pre", False)]


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_backward(types, shape):
    need_gpu()
    for i, (form, gate) in enumerate(FORMS):
        banner(f"resnorm {types} {shape} {form} gate={gate}")
        c = Case(types, *shape, form, gate, wide=i == 0, seed=i)
        got = c.fwd()
        ref = resnorm_fwd(*c.ref("x", "u", "gate", "w_post", "rho", "w_pre"), EPS)
        assert set(got) == set(ref)
        for k in ref:
            assert_close(k, host(got[k]), ref[k], TOL[got[k].dtype])
        # the backward pass from the stream as it is stored and its own inverse norms
        xo = got.get("xo", c.x)
        f = lambda k: None if k not in got else dev_f32(1.0 / np.sqrt(np.mean(host(c.u if k == "r_post" else xo) ** 2, 1) + EPS))  # noqa: E731
        r_post, r_pre = f("r_post"), f("r_pre")
        grads = c.bwd(xo, r_post, r_pre)
        gref = resnorm_bwd(host(xo), *c.ref("u", "gate", "w_post", "rho", "w_pre"), EPS, *c.ref("dxo", "dn"))
        assert set(grads) == set(gref)
        for k in gref:
            assert_close(k, host(grads[k]), gref[k], 2e-5 if gref[k].ndim == 1 else TOL[grads[k].dtype])
        for k, v in c.bwd(xo, r_post, r_pre).items():
            assert torch.equal(v, grads[k]), f"{k}: not the same bits twice"


@pytest.mark.parametrize("types", list(TYPES))
def test_in_place_and_without_statistics(types):
    need_gpu()
    banner(f"resnorm in place {types}")
    c = Case(types, 37, 1040, "both", True)
    ref = c.fwd()
    x = c.x.clone()
    got = c.fwd(x=x, xo=x, stats=False)
    assert torch.equal(got["xo"], ref["xo"]) and torch.equal(got["n"], ref["n"]) and set(got) == {"xo", "n"}


def test_tiny_rows_and_zero_rows():
    """A row of zeros stays zero (eps keeps its inverse norm finite); tiny and huge rows norm to the same size."""
    need_gpu()
    banner("resnorm zero, tiny and huge rows")
    x = torch.randn(3, 256, device="cuda", generator=torch.Generator("cuda").manual_seed(0))
    x[0] = 0
    x[2] *= 1e12
    n, r = torch.empty_like(x), torch.empty(3, device="cuda")
    w = torch.ones(256, device="cuda")
    o5.o5_resnorm_fwd(0, 0, 3, 256, x, None, None, 0, None, None, w, EPS, None, n, None, r)
    ref = resnorm_fwd(host(x), None, None, None, None, host(w), EPS)
    assert not n[0].any() and torch.isfinite(n).all()
    assert_close("n", host(n), ref["n"], 1e-5)
    assert_close("r", host(r), ref["r_pre"], 1e-5)


def test_a_non_finite_row_stays_alone():
    need_gpu()
    banner("resnorm non-finite rows")
    c = Case("bf16", 12, 264, "both", True)
    c.u[3, 5] = float("inf")
    c.gate[7, 9] = float("nan")
    c.x[9, 0] = float("nan")
    got = c.fwd()
    bad = torch.tensor([i in (3, 7, 9) for i in range(12)], device="cuda")
    for k in ("xo", "n"):
        assert torch.equal(~torch.isfinite(got[k]).all(1), bad), k


def test_graph_replays():
    need_gpu()
    banner("resnorm in a graph")
    c = Case("bf16", 50, 512, "both", True)
    f = c.fwd()
    ref = c.bwd(f["xo"], f["r_post"], f["r_pre"])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = c.bwd(f["xo"], f["r_post"], f["r_pre"])
    for _ in range(3):
        for v in out.values():
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], ref[k]) for k in ref)


def test_refusals():
    need_gpu()
    banner("resnorm refusals leave outputs untouched")
    c = Case("bf16", 4, 64, "both", True)
    xo, n = c.blank(torch.bfloat16, 4, 64), c.blank(torch.bfloat16, 4, 64)

    def call(xt=1, dt=1, N=4, D=64, x=c.x, u=c.u, gate=c.gate, ldg=64, w_pre=c.w_pre, rho=c.rho, eps=EPS, xo=xo, n=n):
        o5.o5_resnorm_fwd(xt, dt, N, D, x, u, gate, ldg, c.w_post, rho, w_pre, eps, xo, n, None, None)

    for status, bad in ((3, dict(dt=4)), (3, dict(dt=0)), (2, dict(N=0)), (2, dict(D=60)), (2, dict(D=8200)), (2, dict(ldg=56)),
                        (2, dict(ldg=68)), (7, dict(eps=0.0)), (7, dict(u=None)), (7, dict(u=None, gate=None, w_pre=None)),
                        (1, dict(x=None)), (1, dict(rho=None)), (1, dict(xo=None)), (1, dict(n=None)),
                        (4, dict(x=c.x.data_ptr() + 2))):
        with pytest.raises(o5.O5Error) as e:
            call(**bad)
        assert e.value.status == status, (bad, str(e.value))
    torch.cuda.synchronize()
    assert (xo == 7).all() and (n == 7).all()
    f = c.fwd()
    d = c.blank(torch.bfloat16, 4, 64)
    need = o5.o5_resnorm_bwd_workspace_bytes(1, 1, 4, 64)
    v = [c.blank(torch.float32, 64) for _ in range(3)]
    for status, ws, dgate in ((5, torch.empty(need - 16, dtype=torch.uint8, device="cuda"), d), (1, workspace(need), None)):
        with pytest.raises(o5.O5Error) as e:
            o5.o5_resnorm_bwd(1, 1, 4, 64, f["xo"], c.u, c.gate, 64, c.w_post, c.rho, c.w_pre, f["r_post"], f["r_pre"], c.dxo,
                              c.dn, d, d, dgate, 64, *v, ws)
        assert e.value.status == status
    torch.cuda.synchronize()
    assert (d == 7).all() and all((x == 7).all() for x in v)
