"""GPU: linear attention with a decay for each head against the fp64 recurrence.

Tolerances (max|Y - ref| / max|ref| per output): in fp32 an output is a sum of
up to a few hundred products of both signs, each rounded to 2^-24: 2e-5 holds
300 of them.  In bf16 an output is rounded to 2^-9 and so are, as operands of
its products, the scores and the carried state: 3 x 2^-9 < 1e-2.  The states
and their gradients stay in fp32 and what enters them keeps 24 bits: 2e-5 as for
an output in fp32 (test_gpu_linattn_paths holds them to 1.2e-6)."""
import numpy as np
import pytest
import torch

from oracle.linattn import linattn_bwd, linattn_fwd
from paper_1912_06680_amd import o5
from tests.gpu_util import assert_close, banner, dev, dev_f32, host, need_gpu, workspace

pytestmark = pytest.mark.gpu

TOL_OUT = {False: 2e-5, True: 1e-2}
TOL_STATE = 2e-5


class Case:
    """Inputs on the host (fp64, rounded to the input type) and on the device."""

    def __init__(self, bf16, T, B, nh, nkv, dk, dv, resets=0.1, fused=False, seed=0, decay=None):
        r = np.random.Generator(np.random.PCG64(seed))
        self.bf16, self.size, self.fused = bf16, (T, B, nh, nkv, dk, dv), fused
        self.dt, self.et = (o5.O5_BF16, torch.bfloat16) if bf16 else (o5.O5_F32, torch.float32)
        self.widths = (nh * dk, nkv * dk, nkv * dv)
        x = [torch.from_numpy(r.standard_normal((T, B, w)).astype(np.float32)).to(self.et) for w in self.widths]
        self.do = torch.from_numpy(r.standard_normal((T, B, nh * dv)).astype(np.float32)).to(self.et).cuda()
        self.q, self.k, self.v = self.place(x)
        lam = r.uniform(0.8, 1.0, nkv) if decay is None else np.full(nkv, decay)
        self.decay = dev_f32(lam)
        self.scale = dk ** -0.5
        self.S0, self.dST = dev_f32(r.standard_normal((B, nkv, dk, dv))), dev_f32(r.standard_normal((B, nkv, dk, dv)))
        self.reset = dev((r.random((T, B)) < resets).astype(np.uint8)) if resets else None

    def place(self, x):
        """Contiguous tensors, or parts of one wider buffer with a gap of 8 columns before each."""
        if not self.fused:
            return [t.cuda() for t in x]
        T, B = self.size[:2]
        wide = torch.full((T, B, sum(self.widths) + 24), float("nan"), dtype=self.et, device="cuda")
        out, at = [], 0
        for t in x:
            at += 8
            out.append(wide[..., at:at + t.shape[-1]])
            out[-1].copy_(t)
            at += t.shape[-1]
        return out

    def blank(self, w, n=None):
        return torch.full((*self.size[:2], w), 7.0, dtype=self.et, device="cuda")

    def ref(self):
        f = lambda t: None if t is None else t.detach().double().cpu().numpy()  # noqa: E731
        T, B, nh, nkv, dk, dv = self.size
        return dict(q=f(self.q), k=f(self.k), v=f(self.v), decay=f(self.decay), scale=self.scale, nh=nh, nkv=nkv,
                    S0=f(self.S0), reset=None if self.reset is None else self.reset.cpu().numpy())

    def inputs(self):
        ld = lambda t: (t, t.stride(1))  # noqa: E731
        return (*ld(self.q), *ld(self.k), *ld(self.v), self.decay, self.scale, self.S0, self.reset)

    def fwd(self, state=True):
        T, B, nh, nkv, dk, dv = self.size
        o = self.blank(nh * dv)
        ST = torch.full((B, nkv, dk, dv), 7.0, device="cuda") if state else None
        ws = workspace(o5.o5_linattn_fwd_workspace_bytes(self.dt, *self.size))
        o5.o5_linattn_fwd(self.dt, *self.size, *self.inputs(), o, nh * dv, ST, ws)
        return o, ST

    def bwd(self, state=True):
        T, B, nh, nkv, dk, dv = self.size
        dq, dkey, dval = self.place([self.blank(w) for w in self.widths])
        dS0 = torch.full((B, nkv, dk, dv), 7.0, device="cuda") if state else None
        ws = workspace(o5.o5_linattn_bwd_workspace_bytes(self.dt, *self.size))
        o5.o5_linattn_bwd(self.dt, *self.size, *self.inputs(), self.do, nh * dv, self.dST, dq, dq.stride(1),
                          dkey, dkey.stride(1), dval, dval.stride(1), dS0, ws)
        return dq, dkey, dval, dS0


#        T    B  nh nkv dk  dv  resets fused
SHAPES = [
    (1, 3, 2, 2, 64, 64, 0.5, False),
    (2, 5, 4, 2, 8, 16, 0.3, False),
    (15, 2, 2, 2, 64, 128, 0.1, True),
    (16, 7, 4, 4, 128, 64, 0.1, False),
    (17, 2, 3, 1, 128, 128, 0.1, True),
    (33, 3, 2, 2, 24, 40, 0.0, True),
    (63, 1, 6, 2, 40, 72, 0.05, False),
    (64, 2, 2, 2, 64, 64, 0.02, True),
    (65, 2, 2, 1, 128, 128, 1.0, False),
    (129, 1, 2, 2, 72, 8, 0.01, True),
    (200, 2, 1, 1, 128, 120, 0.02, False),
    (777, 1, 2, 1, 64, 128, 0.003, True),
    (2050, 1, 1, 1, 32, 32, 0.0, False),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:6])))
def test_forward(bf16, shape):
    need_gpu()
    banner(f"linattn forward bf16={bf16} {shape}")
    c = Case(bf16, *shape)
    o, ST = c.fwd()
    ref_o, states = linattn_fwd(**c.ref())
    assert_close("o", host(o), ref_o, TOL_OUT[bf16])
    assert_close("ST", host(ST), states[-1], TOL_STATE)
    again, ST2 = c.fwd()
    assert torch.equal(o, again) and torch.equal(ST, ST2), "not the same bits twice"


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:6])))
def test_backward(bf16, shape):
    need_gpu()
    banner(f"linattn backward bf16={bf16} {shape}")
    c = Case(bf16, *shape)
    got = c.bwd()
    ref = linattn_bwd(dout=host(c.do), dST=host(c.dST), **c.ref())
    for name, x, y in zip(("dq", "dk", "dv", "dS0"), got, ref):
        assert_close(name, host(x), y, TOL_STATE if name == "dS0" else TOL_OUT[bf16])
    for x, y in zip(got, c.bwd()):
        assert torch.equal(x, y), "not the same bits twice"


@pytest.mark.parametrize("bf16", [False, True])
def test_optional_states(bf16):
    """No S0, no ST, no dST, no dS0, no resets."""
    need_gpu()
    banner(f"linattn optional states bf16={bf16}")
    c = Case(bf16, 70, 2, 2, 1, 64, 64, resets=0)
    c.S0, dST = None, c.dST
    c.dST = None
    o, _ = c.fwd(state=False)
    assert_close("o", host(o), linattn_fwd(**c.ref())[0], TOL_OUT[bf16])
    got = c.bwd(state=False)
    for name, x, y in zip(("dq", "dk", "dv"), got, linattn_bwd(dout=host(c.do), **c.ref())):
        assert_close(name, host(x), y, TOL_OUT[bf16])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("decay", [0.0, 1e-3, 1.0])
def test_extreme_decays(bf16, decay):
    """A state that is forgotten at once, nearly at once, and never."""
    need_gpu()
    banner(f"linattn decay={decay} bf16={bf16}")
    c = Case(bf16, 150, 2, 2, 2, 32, 64, decay=decay)
    o, ST = c.fwd()
    ref_o, states = linattn_fwd(**c.ref())
    assert_close("o", host(o), ref_o, TOL_OUT[bf16])
    assert_close("ST", host(ST), states[-1], TOL_STATE)
    for name, x, y in zip(("dq", "dk", "dv", "dS0"), c.bwd(), linattn_bwd(dout=host(c.do), dST=host(c.dST), **c.ref())):
        if np.max(np.abs(y)) > 0:
            assert_close(name, host(x), y, TOL_STATE if name == "dS0" else TOL_OUT[bf16])
        else:
            assert not torch.any(x), name


STEPS = [(1, 8, 8, 64, 64), (3, 4, 2, 8, 16), (5, 6, 2, 40, 72), (130, 4, 4, 128, 128), (2, 4, 1, 128, 120), (33, 3, 3, 24, 8)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", STEPS, ids=lambda s: "x".join(map(str, s)))
def test_single_tokens(bf16, shape):
    """Three tokens one after another equal three steps of the recurrence."""
    need_gpu()
    banner(f"linattn step bf16={bf16} {shape}")
    B, nh, nkv, dk, dv = shape
    c = Case(bf16, 3, *shape, resets=0.3, fused=True)
    S = c.S0.clone()
    outs = []
    for t in range(3):
        o = torch.full((B, nh * dv), 7.0, dtype=c.et, device="cuda")
        # rows of one buffer; pointers stay aligned only for whole rows of 8 elements, so each step takes a copy
        q, k, v = (x[t].clone(memory_format=torch.contiguous_format) for x in (c.q, c.k, c.v))
        o5.o5_linattn_step(c.dt, B, nh, nkv, dk, dv, q, q.stride(0), k, k.stride(0), v, v.stride(0), c.decay, c.scale,
                           c.reset[t].clone(), S, o, nh * dv)
        outs.append(o)
    ref_o, states = linattn_fwd(**c.ref())
    assert_close("o", host(torch.stack(outs)), ref_o, TOL_OUT[bf16])
    assert_close("S", host(S), states[-1], TOL_STATE)


@pytest.mark.parametrize("bf16", [False, True])
def test_what_a_reset_cuts_off_may_hold_anything(bf16):
    """Infinities and NaN in a stored state, a value and a key before a reset, and in values and gradients of later
    steps, reach exactly the outputs that the recurrence sends them to."""
    need_gpu()
    banner(f"linattn non-finite inputs bf16={bf16}")
    c = Case(bf16, 100, 3, 2, 1, 64, 64, resets=0, seed=5)
    c.reset = torch.zeros((100, 3), dtype=torch.uint8, device="cuda")
    c.reset[0, 0] = c.reset[40, 1] = c.reset[90, 1] = c.reset[33, 2] = 1
    c.S0[0] = float("nan")           # cut off at once
    c.S0[0, 0, 1] = float("inf")
    c.v[30, 1, 3] = float("inf")     # cut off at 40
    c.v[95, 1, 5] = float("nan")     # after the last reset
    c.k[20, 2, 7] = float("nan")     # cut off at 33
    o, ST = c.fwd()
    with np.errstate(invalid="ignore"):
        ref_o, states = linattn_fwd(**c.ref())
    fine = np.isfinite(ref_o)
    assert 0 < np.sum(~fine) < fine.size
    assert np.array_equal(np.isfinite(host(o)), fine)
    assert_close("o", np.where(fine, host(o), 0), np.where(fine, ref_o, 0), TOL_OUT[bf16])
    assert np.array_equal(np.isfinite(host(ST)), np.isfinite(states[-1]))

    # backward: the same resets over finite inputs, non-finite gradients
    c = Case(bf16, 100, 3, 2, 1, 64, 64, resets=0, seed=6)
    c.reset = torch.zeros((100, 3), dtype=torch.uint8, device="cuda")
    c.reset[50, 0] = c.reset[99, 1] = c.reset[70, 2] = c.reset[0, 2] = 1
    c.do[60, 0, 9] = float("inf")    # reaches steps 50..60 of sample 0
    c.do[80, 2, 0] = float("nan")    # reaches steps 70..80 of sample 2
    c.dST[1] = float("nan")          # reaches step 99 of sample 1 alone
    got = c.bwd()
    with np.errstate(invalid="ignore"):
        ref = linattn_bwd(dout=host(c.do), dST=host(c.dST), **c.ref())
    for name, x, y in zip(("dq", "dk", "dv", "dS0"), got, ref):
        fine = np.isfinite(y)
        assert np.array_equal(np.isfinite(host(x)), fine), name
        assert_close(name, np.where(fine, host(x), 0), np.where(fine, y, 0), TOL_STATE if name == "dS0" else TOL_OUT[bf16])


#        T    B   nh nkv dk  dv  resets fused: 512 states and more, with several query heads each
GROUPS = [
    (64, 256, 4, 2, 64, 64, 0.02, False),
    (65, 128, 12, 4, 64, 128, 0.05, True),
    (128, 128, 8, 4, 128, 128, 0.02, False),
    (47, 513, 3, 1, 40, 72, 0.1, True),
    (1, 300, 8, 2, 128, 64, 0.5, False),
]


def of_samples(c, at):
    """The inputs of some samples, which depend on no others."""
    r = c.ref()
    for name in ("q", "k", "v", "reset"):
        r[name] = r[name][:, at]
    r["S0"] = r["S0"][at]
    return r


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", GROUPS, ids=lambda s: "x".join(map(str, s[:6])))
def test_many_states_with_shared_heads(bf16, shape):
    need_gpu()
    banner(f"linattn many states with shared heads bf16={bf16} {shape}")
    c = Case(bf16, *shape, seed=9)
    B = shape[1]
    at = [0, 1, B // 2, B - 1]
    o, ST = c.fwd()
    ref_o, states = linattn_fwd(**of_samples(c, at))
    assert_close("o", host(o)[:, at], ref_o, TOL_OUT[bf16])
    assert_close("ST", host(ST)[at], states[-1], TOL_STATE)
    ref = linattn_bwd(dout=host(c.do)[:, at], dST=host(c.dST)[at], **of_samples(c, at))
    for name, x, y in zip(("dq", "dk", "dv", "dS0"), c.bwd(), ref):
        x = host(x)[at] if name == "dS0" else host(x)[:, at]
        assert_close(name, x, y, TOL_STATE if name == "dS0" else TOL_OUT[bf16])


@pytest.mark.parametrize("bf16", [False, True])
def test_many_states_and_inputs_that_are_not_finite(bf16):
    """What is cut off reaches nothing, and what is not, exactly the recurrence's outputs, of each query head."""
    need_gpu()
    banner(f"linattn many states, non-finite inputs bf16={bf16}")
    c = Case(bf16, 100, 256, 6, 2, 64, 64, resets=0, seed=10)
    c.reset = torch.zeros((100, 256), dtype=torch.uint8, device="cuda")
    c.reset[0, 0] = c.reset[40, 1] = c.reset[90, 1] = c.reset[33, 255] = 1
    c.S0[0] = float("nan")
    c.v[30, 1, 3] = float("inf")
    c.v[95, 1, 5] = float("nan")
    c.k[20, 255, 7] = float("nan")
    at = [0, 1, 2, 255]
    o, ST = c.fwd()
    with np.errstate(invalid="ignore"):
        ref_o, states = linattn_fwd(**of_samples(c, at))
    fine = np.isfinite(ref_o)
    o = host(o)[:, at]
    assert 0 < np.sum(~fine) < fine.size
    assert np.array_equal(np.isfinite(o), fine)
    assert_close("o", np.where(fine, o, 0), np.where(fine, ref_o, 0), TOL_OUT[bf16])
    assert np.array_equal(np.isfinite(host(ST)[at]), np.isfinite(states[-1]))


def test_another_stream_and_a_graph():
    """The calls run on the stream that is current, and replay from a graph."""
    need_gpu()
    banner("linattn on another stream and in a graph")
    c = Case(True, 300, 1, 2, 2, 64, 64)
    ref = [*c.fwd(), *c.bwd()]
    torch.cuda.synchronize()
    T, B, nh, nkv, dk, dv = c.size
    o, ST, dS0 = torch.empty_like(ref[0]), torch.empty_like(ref[1]), torch.empty_like(ref[1])
    dq, dkey, dval = (torch.empty_like(x) for x in ref[2:5])
    ws = workspace(max(o5.o5_linattn_fwd_workspace_bytes(c.dt, *c.size), o5.o5_linattn_bwd_workspace_bytes(c.dt, *c.size)))

    def both():
        o5.o5_linattn_fwd(c.dt, *c.size, *c.inputs(), o, nh * dv, ST, ws)
        o5.o5_linattn_bwd(c.dt, *c.size, *c.inputs(), c.do, nh * dv, c.dST, dq, dq.stride(1), dkey, dkey.stride(1), dval,
                          dval.stride(1), dS0, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    outs = (o, ST, dq, dkey, dval, dS0)
    assert all(torch.equal(x, y) for x, y in zip(outs, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for x in outs:
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, ref))


def test_refusals():
    need_gpu()
    banner("linattn refusals leave outputs untouched")
    c = Case(True, 4, 2, 4, 2, 16, 16)
    T, B, nh, nkv, dk, dv = c.size
    o, ST = c.blank(nh * dv), torch.full((B, nkv, dk, dv), 7.0, device="cuda")
    ws = workspace(o5.o5_linattn_fwd_workspace_bytes(c.dt, *c.size))

    def call(dt=c.dt, size=c.size, q=c.q, ldq=nh * dk, decay=c.decay, scale=1.0, ldo=nh * dv, ws=ws, o=o):
        o5.o5_linattn_fwd(dt, *size, q, ldq, c.k, nkv * dk, c.v, nkv * dv, decay, scale, c.S0, None, o, ldo, ST, ws)

    for status, bad in ((3, dict(dt=5)), (2, dict(size=(0, *c.size[1:]))), (2, dict(size=(T, B, 3, 2, dk, dv))),
                        (2, dict(size=(T, B, nh, nkv, 12, dv))), (2, dict(size=(T, B, nh, nkv, dk, 136))),
                        (2, dict(ldq=nh * dk - 8)), (2, dict(ldo=nh * dv + 4)), (1, dict(q=None)), (1, dict(decay=None)),
                        (4, dict(q=c.q.data_ptr() + 2)), (7, dict(scale=float("nan"))), (5, dict(ws=None))):
        with pytest.raises(o5.O5Error) as e:
            call(**bad)
        assert e.value.status == status, (bad, str(e.value))
    torch.cuda.synchronize()
    assert (o == 7).all() and (ST == 7).all()
    S = ST.clone()
    with pytest.raises(o5.O5Error):
        o5.o5_linattn_step(c.dt, B, nh, nkv, dk, dv, c.q, 8, c.k, nkv * dk, c.v, nkv * dv, c.decay, 1.0, None, S, o, nh * dv)
    torch.cuda.synchronize()
    assert (S == 7).all()
