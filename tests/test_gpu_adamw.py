"""GPU: AdamW over many tensors against its definition in fp64.

Tolerances: p, m, v in 32 bits are a handful of products, sums, a root and a
quotient, each rounded to 2^-24: 1e-6 of the largest.  In 8 bits p is held to
the same (it is formed before the moments are rounded), and every code has to
stand for one of the two values around the exact moment, which one by the
random number of its element; where the exact moment lies within 1e-5 of a step
of the place where the choice flips, or of a code's own value, both are right."""
import numpy as np
import pytest
import torch

from oracle.adamw import GROUP, adamw_step, chances, neighbours, rounded, value_of
from paper_1912_06680_amd import o5
from tests.gpu_util import assert_close, banner, host, need_gpu

pytestmark = pytest.mark.gpu

HP = (1e-3, float(np.float32(0.9)), float(np.float32(0.999)), 1e-8, 5.0)
SIZES = [1, 3, 4, 255, 256, 257, 1000, 2048, 2049, 5000, 75, 8192]


class Tensor:
    def __init__(self, n, bits, g16, mirror, seed, wd=0.1, lr_scale=1.0, spread=1.0):
        r = np.random.Generator(np.random.PCG64(seed))
        scale = np.exp(spread * r.standard_normal(n))
        f = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731
        self.n, self.bits, self.wd, self.lr_scale = n, bits, wd, lr_scale
        self.p, self.g = f(r.standard_normal(n)), f(r.standard_normal(n) * scale)
        if g16:
            self.g = self.g.to(torch.bfloat16)
        self.p16 = torch.zeros(n, dtype=torch.bfloat16, device="cuda") if mirror else None
        self.me = self.ve = None
        if bits == 32:
            self.m, self.v = f(0.1 * r.standard_normal(n) * scale), f(scale ** 2 * r.random(n))
        else:
            b = lambda hi, k: torch.from_numpy(r.integers(0, hi, k).astype(np.uint8)).cuda()  # noqa: E731
            sign = torch.from_numpy((128 * r.integers(0, 2, n)).astype(np.uint8)).cuda()
            self.m, self.v = b(121, n) + sign, b(249, n)
            groups = (n + GROUP - 1) // GROUP
            self.me, self.ve = b(12, groups) + 120, b(12, groups) + 120
        self.args = o5.adamw_tensor(self.p, self.g, self.m, self.v, self.me, self.ve, self.p16, lr_scale, wd)

    def moments(self):
        if self.bits == 32:
            return host(self.m), host(self.v)
        c = lambda t: t.cpu().numpy()  # noqa: E731
        return value_of(c(self.m), c(self.me), "m"), value_of(c(self.v), c(self.ve), "v")

    def expect(self, step):
        m, v = self.moments()
        lr = float(np.float32(HP[0]) * np.float32(self.lr_scale))
        return adamw_step(host(self.p), m, v, host(self.g), lr, *HP[1:], float(np.float32(self.wd)), step)


def _plan(tensors):
    args = [t.args for t in tensors]
    plan = torch.zeros(o5.o5_adamw_plan_bytes(args), dtype=torch.uint8)
    o5.o5_adamw_plan(args, plan)
    return plan, plan.cuda()


def _codes_right(got, x, up, which):
    """got: the values of the codes; x: the exact moments."""
    low, high, _ = neighbours(x, which)
    mag = np.abs(x)
    frac = (mag - low) / (high - low)
    edge = (np.abs(frac + up - 1.0) < 1e-5) | (frac < 1e-5) | (frac > 1 - 1e-5)
    want = rounded(x, up, which)
    assert np.mean(edge) < 0.1  # (moments of a few bits and bf16 gradients meet a code in a few per cent of the draws)
    assert np.array_equal(got[~edge], want[~edge])
    assert np.all((np.abs(got) >= low - 1e-4 * (high - low)) & (np.abs(got) <= high + (high - low) * 1.0001))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("g16", [False, True])
@pytest.mark.parametrize("step", [1, 20])
def test_many_tensors(bits, g16, step):
    need_gpu()
    banner(f"adamw bits={bits} g16={g16} step={step}")
    tensors = [Tensor(n, bits, g16, i % 2 == 0, i, wd=0.1 * (i % 3), lr_scale=1.0 + 0.5 * (i % 2)) for i, n in enumerate(SIZES)]
    expect = [t.expect(step) for t in tensors]
    plan = _plan(tensors)
    o5.o5_adamw_step(*plan, *HP, (3 << 32) + 9, step)
    for i, (t, (p, m, v)) in enumerate(zip(tensors, expect)):
        assert_close(f"p[{t.n}]", host(t.p), p, 1e-6)
        if t.p16 is not None:
            assert torch.equal(t.p16, t.p.to(torch.bfloat16))
        gm, gv = t.moments()
        if bits == 32:
            assert_close("m", gm, m, 1e-6)
            assert_close("v", gv, v, 1e-6)
        else:
            um, uv = chances(t.n, step, i, (3 << 32) + 9)
            _codes_right(gm, m, um, "m")
            _codes_right(gv, v, uv, "v")
            assert np.all(gv[v > 0] > 0)
    # the moments as a checkpoint takes them
    total = sum((t.n + 255) // 256 * 256 for t in tensors)
    mo, vo = torch.full((total,), 7.0, device="cuda"), torch.full((total,), 7.0, device="cuda")
    o5.o5_adamw_moments(*plan, mo, vo)
    at = 0
    for t in tensors:
        gm, gv = t.moments()
        assert np.array_equal(host(mo[at:at + t.n]), gm) and np.array_equal(host(vo[at:at + t.n]), gv)
        end = at + (t.n + 255) // 256 * 256
        assert (mo[at + t.n:end] == 7).all() and (vo[at + t.n:end] == 7).all()
        at = end


def test_mixed_plan_equals_single_plans():
    """Tensors of both widths and gradient types in one plan, against one plan each (the place in the plan picks the random
    numbers, so the 8-bit tensors are put at place 0 of theirs)."""
    need_gpu()
    banner("adamw mixed plan")
    make = lambda: [Tensor(3000, 8, False, True, 1), Tensor(77, 32, True, False, 2), Tensor(2500, 32, False, True, 3)]  # noqa: E731
    one, each = make(), make()
    o5.o5_adamw_step(*_plan(one), *HP, 5, 2)
    for t in each:
        o5.o5_adamw_step(*_plan([t]), *HP, 5, 2)
    for a, b in zip(one, each):
        for k in ("p", "m", "v", "me", "ve", "p16"):
            assert getattr(a, k) is None or torch.equal(getattr(a, k), getattr(b, k)), k


def test_8_bits_from_zeros_follow_32_bits():
    """From zero moments, 300 steps on a quadratic: the 8-bit run's loss falls with the 32-bit run's, and v, whose change per
    step is far below a code, follows the gradients' mean square without bias."""
    need_gpu()
    banner("adamw 8 bits over 300 steps")
    n = 4096
    runs = {}
    for bits in (32, 8):
        t = Tensor(n, bits, False, False, 4, wd=0.0)
        for k in ("m", "v", "me", "ve"):
            if getattr(t, k) is not None:
                getattr(t, k).zero_()
        gen = torch.Generator("cuda").manual_seed(1)
        plan = _plan([t])
        for step in range(1, 301):
            t.g.copy_(t.p + 0.1 * torch.randn(n, device="cuda", generator=gen))
            o5.o5_adamw_step(*plan, 1e-2, *HP[1:4], 0.0, 1, step)
        m, v = t.moments()
        runs[bits] = (float(t.p.square().mean()), float(np.mean(v)))
    print("   ", runs, flush=True)
    assert abs(runs[8][0] / runs[32][0] - 1) < 0.05 and abs(runs[8][1] / runs[32][1] - 1) < 0.02


def test_non_finite_gradients_show():
    """A gradient that is not finite leaves NaN in its own p, m and v and nowhere else."""
    need_gpu()
    banner("adamw non-finite gradients")
    for bits in (32, 8):
        t = Tensor(1000, bits, False, True, 6)
        t.g[17], t.g[600] = float("nan"), float("inf")
        o5.o5_adamw_step(*_plan([t]), *HP, 1, 3)
        bad = np.isin(np.arange(1000), (17, 600))
        m, v = t.moments()
        for x in (host(t.p), m, v):
            assert np.array_equal(~np.isfinite(x), bad)


def test_graph_replays_and_lr_zero():
    need_gpu()
    banner("adamw in a graph, lr = 0")
    t = Tensor(3001, 8, True, True, 8, wd=0.3)
    p = t.p.clone()
    plan = _plan([t])
    o5.o5_adamw_step(*plan, 0.0, *HP[1:], 1, 1)
    assert torch.equal(t.p, p) and torch.equal(t.p16, p.to(torch.bfloat16))
    state = [x.clone() for x in (t.p, t.m, t.v, t.me, t.ve)]
    o5.o5_adamw_step(*plan, *HP, 1, 2)
    ref = [x.clone() for x in (t.p, t.m, t.v, t.me, t.ve)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o5.o5_adamw_step(*plan, *HP, 1, 2)
    for _ in range(3):
        for x, y in zip((t.p, t.m, t.v, t.me, t.ve), state):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((t.p, t.m, t.v, t.me, t.ve), ref))


def test_refusals():
    need_gpu()
    banner("adamw refusals")
    t = Tensor(100, 8, False, False, 9)
    before = [x.clone() for x in (t.p, t.m, t.v)]
    for bad, status in ((dict(n=0), 2), (dict(p=None), 1), (dict(p=t.p.data_ptr() + 4), 4), (dict(m_exp=None), 1),
                        (dict(bits=16), 7), (dict(g_dt=3), 3), (dict(weight_decay=-1.0), 7), (dict(lr_scale=float("inf")), 7)):
        a = o5.AdamwTensor.from_buffer_copy(t.args)
        for k, v in bad.items():
            setattr(a, k, v)
        assert o5.o5_adamw_plan_bytes([a]) == 0
        with pytest.raises(o5.O5Error) as e:
            o5.o5_adamw_plan([a], torch.zeros(4096, dtype=torch.uint8))
        assert e.value.status == status, bad
    with pytest.raises(o5.O5Error) as e:
        o5.o5_adamw_plan([t.args], torch.zeros(o5.o5_adamw_plan_bytes([t.args]) - 16, dtype=torch.uint8))
    assert e.value.status == 5
    plan, dev = _plan([t])
    for args, status in (((torch.zeros_like(plan), dev, *HP, 1, 1), 7), ((plan, None, *HP, 1, 1), 1), ((plan, dev, *HP, 1, 0), 7),
                         ((plan, dev, -1.0, *HP[1:], 1, 1), 7), ((plan, dev, HP[0], 1.0, *HP[2:], 1, 1), 7)):
        with pytest.raises(o5.O5Error) as e:
            o5.o5_adamw_step(*args)
        assert e.value.status == status
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((t.p, t.m, t.v), before))
