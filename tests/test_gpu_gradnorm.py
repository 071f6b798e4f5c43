"""GPU: the global norm of a plan's gradients and AdamW on gradients clipped to it.

Tolerances: squares and their sum are taken in 64 bits, the norm and the factor are rounded to 2^-24 (2^-23 with a factor's
own quotient): 2.4e-7 of each.  p, m and v as in test_gpu_adamw, 1e-6 of the largest."""
import numpy as np
import pytest
import torch

from oracle.adamw import adamw_step
from paper_1912_06680_amd import o5
from tests.gpu_util import assert_close, banner, host, need_gpu, workspace
from tests.test_gpu_adamw import HP, SIZES, Tensor, _plan

pytestmark = pytest.mark.gpu

EXACT = 2.0 ** -22


def norm_of(plan, max_norm, ws=None):
    clip = torch.full((2,), 7.0, device="cuda")
    if ws is None:
        ws = workspace(o5.o5_adamw_grad_norm_workspace_bytes(plan[0])).fill_(255)
    o5.o5_adamw_grad_norm(*plan, max_norm, clip, ws)
    return clip


def true_norm(tensors):
    return float(np.sqrt(sum(np.sum(host(t.g) ** 2) for t in tensors)))


def near(x, y):
    return abs(x - y) <= EXACT * abs(y)


@pytest.mark.parametrize("g16", [False, True])
@pytest.mark.parametrize("sizes", [[1], [7], SIZES, [100003, 5, 1024, 1], [1] * 5000, [3000000, 1, 70001]], ids=len)
def test_norm_and_factor(sizes, g16):
    need_gpu()
    banner(f"grad norm of {len(sizes)} tensors g16={g16}")
    tensors = [Tensor(n, 32, g16, False, i) for i, n in enumerate(sizes)]
    plan = _plan(tensors)
    norm = true_norm(tensors)
    for max_norm, factor in ((0.5 * norm, 0.5), (2.0 * norm, 1.0), (float("inf"), 1.0)):
        max_norm = float(np.float32(max_norm))
        clip = norm_of(plan, max_norm)
        assert near(float(clip[0]), norm) and near(float(clip[1]), min(1.0, max_norm / norm))
        assert torch.equal(clip, norm_of(plan, max_norm))


def test_tensors_of_both_types_and_beside_other_memory():
    """Each tensor in the middle of a buffer of NaN: nothing beside it is read into the sum."""
    need_gpu()
    banner("grad norm beside other memory")
    tensors, keep = [], []
    for i, n in enumerate([1, 3, 8, 9, 1023, 1025, 4100]):
        t = Tensor(n, 32, i % 2 == 0, False, i)
        wide = torch.full((n + 64,), float("nan"), dtype=t.g.dtype, device="cuda")
        wide[16:16 + n] = t.g
        t.g = wide[16:16 + n]
        t.args = o5.adamw_tensor(t.p, t.g, t.m, t.v)
        tensors.append(t)
        keep.append(wide)
    assert near(float(norm_of(_plan(tensors), 1.0)[0]), true_norm(tensors))


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e18, 1e36])
def test_squares_beyond_32_bits(scale):
    need_gpu()
    banner(f"grad norm scale={scale}")
    t = Tensor(5000, 32, False, False, 3, spread=0.1)
    t.g.mul_(scale)
    clip = norm_of(_plan([t]), scale)
    assert near(float(clip[0]), true_norm([t]))
    assert abs(float(clip[1]) - scale / true_norm([t])) <= 2 * EXACT


def test_no_gradient_and_factors_that_vanish():
    need_gpu()
    banner("grad norm of zeros; a tiny largest norm")
    t = Tensor(1000, 32, False, False, 4)
    t.g.zero_()
    assert norm_of(_plan([t]), 1.0).tolist() == [0.0, 1.0]
    t.g.fill_(1e38)
    assert float(norm_of(_plan([t]), 1e-30)[1]) > 0.0


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("g16", [False, True])
def test_clipped_step(bits, g16):
    """Against the definition on the scaled gradients, and where they are fp32, bit for bit the step on a scaled copy."""
    need_gpu()
    banner(f"clipped step bits={bits} g16={g16}")
    make = lambda: [Tensor(n, bits, g16, i % 2 == 0, i, wd=0.1 * (i % 3)) for i, n in enumerate(SIZES)]  # noqa: E731
    tensors, other = make(), make()
    plan = _plan(tensors)
    clip = norm_of(plan, float(np.float32(0.1 * true_norm(tensors))))
    factor = float(clip[1])
    assert 0.099 < factor < 0.101
    expect = []
    for t in tensors:
        m, v = t.moments()
        expect.append(adamw_step(host(t.p), m, v, host(t.g) * factor, HP[0], *HP[1:], float(np.float32(t.wd)), 20))
    o5.o5_adamw_step_clipped(*plan, *HP, clip, 9, 20)
    for t, (p, m, v) in zip(tensors, expect):
        assert_close(f"p[{t.n}]", host(t.p), p, 1e-6)
        if bits == 32:
            assert_close("m", host(t.m), m, 1e-6)
            assert_close("v", host(t.v), v, 1e-6)
    if not g16:
        for t in other:
            t.g.mul_(clip[1])
        o5.o5_adamw_step(*_plan(other), *HP, 9, 20)
        for a, b in zip(tensors, other):
            for k in ("p", "m", "v", "me", "ve", "p16"):
                assert getattr(a, k) is None or torch.equal(getattr(a, k), getattr(b, k)), k


@pytest.mark.parametrize("bits", [32, 8])
def test_a_factor_of_one_changes_no_bit(bits):
    need_gpu()
    banner(f"clipped step, factor 1, bits={bits}")
    make = lambda: [Tensor(n, bits, i % 2 == 0, True, i) for i, n in enumerate(SIZES)]  # noqa: E731
    a, b = make(), make()
    plan = _plan(a)
    o5.o5_adamw_step_clipped(*plan, *HP, norm_of(plan, float("inf")), 3, 5)
    o5.o5_adamw_step(*_plan(b), *HP, 3, 5)
    for x, y in zip(a, b):
        for k in ("p", "m", "v", "me", "ve", "p16"):
            assert getattr(x, k) is None or torch.equal(getattr(x, k), getattr(y, k)), k


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite_leaves_the_step_out(bits, bad):
    need_gpu()
    banner(f"clipped step, {bad} bits={bits}")
    tensors = [Tensor(n, bits, i % 2 == 0, True, i) for i, n in enumerate([3000, 77])]
    tensors[0].g[2999] = bad
    plan = _plan(tensors)
    keep = [[getattr(t, k).clone() for k in ("p", "m", "v", "p16")] for t in tensors]
    clip = norm_of(plan, 1.0)
    assert not torch.isfinite(clip[0]) and float(clip[1]) == 0.0
    o5.o5_adamw_step_clipped(*plan, *HP, clip, 3, 5)
    for t, old in zip(tensors, keep):
        assert all(torch.equal(getattr(t, k), x) for k, x in zip(("p", "m", "v", "p16"), old))


def test_another_stream_and_a_graph():
    need_gpu()
    banner("grad norm and clipped step in a graph")
    t = Tensor(300001, 8, True, True, 8, wd=0.3)
    plan = _plan([t])
    state = [x.clone() for x in (t.p, t.m, t.v, t.me, t.ve)]
    ws, clip = workspace(o5.o5_adamw_grad_norm_workspace_bytes(plan[0])), torch.empty(2, device="cuda")
    max_norm = 0.3 * true_norm([t])

    def both():
        o5.o5_adamw_grad_norm(*plan, max_norm, clip, ws)
        o5.o5_adamw_step_clipped(*plan, *HP, clip, 1, 2)

    def reset():
        for x, y in zip((t.p, t.m, t.v, t.me, t.ve), state):
            x.copy_(y)

    both()
    ref = [x.clone() for x in (clip, t.p, t.m, t.v, t.me, t.ve)]
    reset()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((clip, t.p, t.m, t.v, t.me, t.ve), ref))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        reset()
        clip.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((clip, t.p, t.m, t.v, t.me, t.ve), ref))
        both()
        torch.cuda.synchronize()


def test_offsets_past_32_bits():
    """2^32 + 3079 gradients in bf16: only the last ones are not zero."""
    need_gpu()
    banner("grad norm, 2^32 + 3079 elements")
    n = (1 << 32) + 3079
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-3:] = torch.tensor([3.0, 4.0, 12.0])
    at = g.data_ptr()  # (the norm reads the gradients alone)
    t = o5.AdamwTensor(n, at, at, at, at, None, None, None, 1.0, 0.0, o5.O5_BF16, 32)
    plan = torch.empty(o5.o5_adamw_plan_bytes([t]), dtype=torch.uint8)
    o5.o5_adamw_plan([t], plan)
    assert norm_of((plan, plan.cuda()), 26.0).tolist() == [13.0, 1.0]
    del g
    torch.cuda.empty_cache()


def test_refusals():
    need_gpu()
    banner("grad norm refusals")
    t = Tensor(5000, 32, False, False, 9)
    plan, dev = _plan([t])
    clip = torch.full((2,), 7.0, device="cuda")
    need = o5.o5_adamw_grad_norm_workspace_bytes(plan)
    ws = workspace(need)
    for args, status in (((torch.zeros_like(plan), dev, 1.0, clip, ws), 7), ((plan, None, 1.0, clip, ws), 1),
                         ((plan, dev, 0.0, clip, ws), 7), ((plan, dev, float("nan"), clip, ws), 7), ((plan, dev, 1.0, None, ws), 1),
                         ((plan, dev, 1.0, clip, None), 5), ((plan, dev, 1.0, clip, ws[:need - 1]), 5)):
        with pytest.raises(o5.O5Error) as e:
            o5.o5_adamw_grad_norm(*args)
        assert e.value.status == status
    with pytest.raises(o5.O5Error) as e:
        o5.o5_adamw_step_clipped(plan, dev, *HP, None, 1, 1)
    assert e.value.status == 1
    p = t.p.clone()
    with pytest.raises(o5.O5Error) as e:
        o5.o5_adamw_step_clipped(plan, dev, *HP, clip, 1, 0)
    assert e.value.status == 7
    torch.cuda.synchronize()
    assert (clip == 7).all() and torch.equal(t.p, p)
