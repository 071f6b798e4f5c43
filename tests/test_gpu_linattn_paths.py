"""GPU: the ways that the sequence form takes through a call, each against the fp64 recurrence.

A call with many states runs a block for each; one with few states is cut in time into splits (a launch for the splits'
own parts of the state, a scan, a launch for the outputs) of one or of several chunks (64 steps in bf16, 32 in fp32), the
first of them short where the length is no multiple.  The sizes below pick each of these; the number of splits is read off
the workspace, so that a size cannot leave its way unnoticed.

Tolerances (max|Y - ref| / max|ref|): outputs as in test_gpu_linattn, whose docstring derives them.  States: what enters
one keeps 24 bits and is summed in fp32; a chunk adds to it in 7 roundings at most (6 products of three terms and the
decay), so that the 64 chunks which a state of decay 1 - 2^-12 remembers are a random walk of 450 steps of at most 2^-24,
21 x 2^-24 = 1.2e-6 at the outside.  (Operands of 16 bits leave 2.4e-6.)"""
import numpy as np
import pytest
import torch

from oracle.linattn import linattn_bwd, linattn_fwd
from paper_1912_06680_amd import o5
from tests.gpu_util import assert_close, banner, dev_f32, host, need_gpu
from tests.test_gpu_linattn import TOL_OUT, TOL_STATE, Case

pytestmark = pytest.mark.gpu

TOL_24 = 1.2e-6
NAMES = ("dq", "dk", "dv", "dS0")


def _head(c, b, n):
    """The recurrence's inputs for one sample and one state head, with its query heads."""
    T, B, nh, nkv, dk, dv = c.size
    G = nh // nkv
    cut = lambda x, w, m: host(x).reshape(T, B, -1, w)[:, b:b + 1, n * m:(n + 1) * m].reshape(T, 1, m * w)  # noqa: E731
    one = lambda x: None if x is None else host(x)[b:b + 1, n:n + 1]  # noqa: E731
    ins = dict(q=cut(c.q, dk, G), k=cut(c.k, dk, 1), v=cut(c.v, dv, 1), decay=host(c.decay)[n:n + 1], scale=c.scale, nh=G, nkv=1,
               S0=one(c.S0), reset=None if c.reset is None else c.reset.cpu().numpy()[:, b:b + 1])
    return ins, cut(c.do, dv, G), one(c.dST), cut, one


def _same(name, x, y, tol):
    """Non-finite in the same places, and elsewhere within the tolerance."""
    fine = np.isfinite(y)
    assert np.array_equal(np.isfinite(x), fine), f"{name}: {np.sum(np.isfinite(x) != fine)} of {fine.size} places"
    x, y = np.where(fine, x, 0), np.where(fine, y, 0)
    if np.any(y):
        assert_close(name, x, y, tol)
    else:
        assert not np.any(x), name


def _forward(c, picks, tol_state=TOL_STATE, state=True):
    T, B, nh, nkv, dk, dv = c.size
    o, ST = c.fwd(state)
    for b, n in picks:
        ins, _, _, cut, one = _head(c, b, n)
        with np.errstate(invalid="ignore"):
            ref_o, states = linattn_fwd(**ins)
        _same(f"o[{b},{n}]", cut(o, dv, nh // nkv), ref_o, TOL_OUT[c.bf16])
        if state:
            _same(f"ST[{b},{n}]", one(ST), states[-1], tol_state)


def _backward(c, picks, tol_state=TOL_STATE, state=True):
    T, B, nh, nkv, dk, dv = c.size
    got = c.bwd(state)
    for b, n in picks:
        ins, do, dST, cut, one = _head(c, b, n)
        with np.errstate(invalid="ignore"):
            ref = linattn_bwd(dout=do, dST=dST, **ins)
        for name, x, y, w, m in zip(NAMES, got, ref, (dk, dk, dv, 0), (nh // nkv, 1, 1, 0)):
            if name != "dS0":
                _same(f"{name}[{b},{n}]", cut(x, w, m), y, TOL_OUT[c.bf16])
            elif state:
                _same(f"dS0[{b},{n}]", one(x), y, tol_state)


def _splits(c):
    """The splits of a forward call, from the workspace that it asks for."""
    T, B, nh, nkv, dk, dv = c.size
    floats = o5.o5_linattn_fwd_workspace_bytes(c.dt, *c.size) // 4
    pad = lambda d: 64 if d <= 64 else 128  # noqa: E731
    return max(1, floats // (B * nkv * (pad(dk) * pad(dv) + 1)))


#         T    B   nh nkv dk  dv   (sample, state head) compared                splits in fp32 and in bf16
UNSPLIT = [
    (256, 128, 2, 2, 128, 128, ((0, 0), (1, 1), (127, 0)), (1, 1)),   # whole chunks, one query head
    (256, 128, 2, 2, 64, 64, ((0, 1), (127, 0)), (1, 1)),
    (320, 64, 4, 4, 64, 128, ((5, 2), (63, 3)), (1, 1)),
    (384, 33, 8, 8, 128, 64, ((0, 0), (32, 7)), (1, 1)),
    (192, 128, 2, 2, 128, 128, ((3, 1),), (1, 1)),
    (321, 128, 2, 2, 128, 128, ((3, 1), (127, 0)), (1, 1)),           # a short first chunk, then whole ones
    (256, 256, 4, 2, 128, 128, ((0, 0), (255, 1)), (1, 1)),           # a state's query heads in turn
]
SPLIT = [
    (1024, 1, 2, 2, 64, 64, ((0, 0), (0, 1)), (32, 16)),              # one chunk a split, whole chunks
    (1000, 1, 4, 2, 128, 128, ((0, 1),), (32, 16)),
    (2560, 2, 32, 8, 64, 128, ((0, 0), (1, 7)), (8, 8)),              # several chunks a split, whole chunks
    (2050, 2, 32, 8, 64, 128, ((0, 3), (1, 7)), (8, 7)),              # ... a short first chunk, a last split of fewer
    (2048, 2, 16, 4, 128, 128, ((1, 2),), (16, 16)),
    (1999, 3, 6, 6, 72, 40, ((2, 5),), (21, 16)),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("shape", UNSPLIT + SPLIT, ids=lambda s: "x".join(map(str, s[:6])))
def test_every_way(shape, state, bf16):
    """With the last states wanted and without (the last chunk's update may then be left out)."""
    need_gpu()
    *size, picks, splits = shape
    banner(f"linattn ways bf16={bf16} {size} state={state}")
    c = Case(bf16, *size, resets=0.004, fused=True, seed=11)
    assert _splits(c) == splits[bf16]
    _forward(c, picks, state=state)
    _backward(c, picks, state=state)
    assert all(x is None or torch.equal(x, y) for x, y in zip(c.bwd(state), c.bwd(state))), "not the same bits twice"


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("decay", [0.0, 1e-3, 1.0])
@pytest.mark.parametrize("shape", [SPLIT[0], SPLIT[3], UNSPLIT[0]], ids=lambda s: "x".join(map(str, s[:6])))
def test_extreme_decays(shape, decay, bf16):
    """A state that is forgotten at once, nearly at once and never, across splits and across whole chunks."""
    need_gpu()
    *size, picks, splits = shape
    banner(f"linattn decay={decay} bf16={bf16} {size}")
    c = Case(bf16, *size, resets=0.002, seed=12, decay=decay)
    assert _splits(c) == splits[bf16]
    _forward(c, picks)
    _backward(c, picks)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("decay", [None, 0.5, 1.0])
@pytest.mark.parametrize("shape", [SPLIT[0], SPLIT[1], SPLIT[3], UNSPLIT[0], UNSPLIT[5]], ids=lambda s: "x".join(map(str, s[:6])))
def test_inputs_that_are_not_finite(shape, decay, bf16):
    """What a reset cuts off may hold anything; what none cuts off reaches what the recurrence carries it to, over the ends
    of chunks and splits, and nothing else: not the other heads and samples."""
    need_gpu()
    *size, picks, _ = shape
    banner(f"linattn non-finite bf16={bf16} decay={decay} {size}")
    T, B, nh, nkv, dk, dv = size
    c = Case(bf16, *size, resets=0, fused=True, seed=13, decay=decay)
    (b, n), other = picks[0], picks[-1]
    c.reset = torch.zeros((T, B), dtype=torch.uint8, device="cuda")
    c.reset[7, b] = c.reset[T // 2, b] = c.reset[T - 70, b] = 1
    c.S0[b, n, 3, 5] = float("nan")                         # cut off at step 7
    c.v[T // 4, b, n * dv + 1] = float("inf")               # cut off at T / 2, several chunks later
    c.k[T // 2 + 9, b, n * dk + 2] = float("nan")           # cut off at T - 70
    c.v[T - 33, b, n * dv + 3] = float("-inf")              # never cut off
    c.q[T // 8, b, n * (nh // nkv) * dk] = float("nan")     # one step's outputs of one head
    _forward(c, {(b, n), other})

    c = Case(bf16, *size, resets=0, fused=True, seed=14, decay=decay)
    c.reset = torch.zeros((T, B), dtype=torch.uint8, device="cuda")
    c.reset[T // 3, b] = c.reset[T - 7, b] = 1
    c.dST[b, n, 1] = float("nan")                           # reaches the steps from T - 7 on
    c.do[T - 80, b, n * (nh // nkv) * dv + 4] = float("inf")  # back to step T / 3
    c.do[5, b, n * (nh // nkv) * dv] = float("nan")         # back to the first step and dS0
    _backward(c, {(b, n), other})


@pytest.mark.parametrize("T,B,splits", [(6000, 1, 94), (2048, 256, 1), (2052, 256, 1)])
def test_states_keep_24_bits_in_bf16(T, B, splits):
    """A state that remembers thousands of steps, summed in one block and across splits, is as exact as an fp32 sum."""
    need_gpu()
    banner(f"linattn states of long sequences T={T} B={B}")
    c = Case(True, T, B, 1, 1, 64, 64, resets=0, seed=15)
    c.decay = dev_f32(np.array([1.0 - 2.0 ** -12]))
    assert _splits(c) == splits
    _forward(c, ((B - 1, 0),), TOL_24)
    _backward(c, ((B - 1, 0),), TOL_24)


@pytest.mark.parametrize("shape", UNSPLIT + SPLIT, ids=lambda s: "x".join(map(str, s[:6])))
def test_states_keep_24_bits_everywhere(shape):
    need_gpu()
    *size, picks, _ = shape
    banner(f"linattn states {size}")
    c = Case(True, *size, resets=0.004, seed=16)
    _forward(c, picks[:1], TOL_24)
    _backward(c, picks[:1], TOL_24)
