"""GPU: what a step that is left out, because the norm of its gradients is not finite, leaves to the steps behind it."""
import pytest
import torch

from paper_1912_06680_amd import linpolicy
from tests.gpu_util import banner, need_gpu
from tests.test_gpu_linpolicy import _batch

pytestmark = pytest.mark.gpu

T, B, D, HEADS = 20, 2, 64, (5, 3)


def _policy(core, bits, **kw):
    return linpolicy.LinPolicy(T, B, D, 1, 1, HEADS, core=core, bits=bits, lr=1e-3, **{"max_norm": 1.0, **kw})


def _step(p, batch, bad=False):
    x, rewards, dones, act, logp, values = batch
    if bad:
        rewards = rewards.clone()
        rewards[3, 1] = float("inf")
    p.train_step(x[:T].contiguous(), rewards, dones, values, act, logp)


def _data(p):
    out = []
    for seed in (7, 8, 9):
        x, rewards, dones = _batch(T, B, D, HEADS, seed)
        act, logp, values = linpolicy.rollout(p, x, dones=dones)
        out.append((x, rewards, dones, act, logp, values))
    return out


def _state(p):
    return [*p.P.values(), *(t for m in p.moments.values() for t in m if t is not None)]


@pytest.mark.parametrize("core", ["gatedrec", "linattn"])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("bad", [(0,), (1,), (0, 1, 2, 3), (2, 4)])
def test_a_step_that_is_left_out_leaves_no_trace(core, bits, bad):
    """Weights and moments after some bad steps among three good ones are, bit for bit, those of the three alone."""
    need_gpu()
    banner(f"policy steps around bad ones {core} bits={bits} {bad}")
    a, b = _policy(core, bits), _policy(core, bits)
    data = _data(a)
    good = 0
    for i in range(3 + len(bad)):
        if i in bad:
            keep = [t.clone() for t in _state(a)]
            _step(a, data[0], bad=True)
            assert float(a.clip[1]) == 0.0 and all(torch.equal(x, y) for x, y in zip(_state(a), keep))
        else:
            _step(a, data[good])
            good += 1
    for batch in data:
        _step(b, batch)
    assert good == 3 and all(torch.equal(x, y) for x, y in zip(_state(a), _state(b)))
    assert a.step_count == b.step_count == 3


def test_the_count_goes_on_from_where_it_is_set():
    """As when training goes on from a checkpoint."""
    need_gpu()
    banner("policy step count set")
    a, b = _policy("gatedrec", 32), _policy("gatedrec", 32)
    data = _data(a)
    for p in (a, b):
        _step(p, data[0])
    _step(a, data[1], bad=True)
    a.step_count = b.step_count = 5
    for p in (a, b):
        _step(p, data[2])
    assert a.step_count == b.step_count == 6 and all(torch.equal(x, y) for x, y in zip(_state(a), _state(b)))


def test_a_step_in_a_graph():
    """A captured step takes the number that it was captured with."""
    need_gpu()
    banner("policy step in a graph")
    a, b = _policy("gatedrec", 32), _policy("gatedrec", 32)
    x, rewards, dones, act, logp, values = _data(a)[0]
    x = x[:T].contiguous()
    step = lambda p: p.train_step(x, rewards, dones, values, act, logp)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for p in (a, b):
            step(p)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    assert a.step_count == 2
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        b.step_count = 1
        step(b)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(_state(a), _state(b)))
