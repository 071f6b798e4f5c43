"""GPU: surgery on parameter vectors of more elements than one launch's threads, 2^32 for folding and 2^34 (four elements a
thread) for widening."""
import pytest
import torch

from paper_1912_06680_amd import o5
from tests.gpu_util import banner, need_gpu

pytestmark = pytest.mark.gpu

PART = 1 << 29


def _parts(n):
    return [(a, min(n, a + PART)) for a in range(0, n, PART)]


def test_fold_past_2_32():
    """Inputs 8 of 9 kept at 32768 units: every element copied from its place, zero moments, the cut column in the bias."""
    need_gpu()
    D, Dk, H, A1 = 9, 8, 1 << 15, 3
    n_old, n = o5.o5_param_count(D, H, A1), o5.o5_param_count(Dk, H, A1)
    banner(f"surgery fold to {n} elements")
    assert n > 1 << 32
    old = torch.randn(n_old, device="cuda", generator=torch.Generator("cuda").manual_seed(0))
    new, m, v = (torch.full((n,), 7.0, device="cuda") for _ in range(3))
    E = torch.tensor([0.5], device="cuda")
    o5.o5_surgery_fold_input(D, H, A1, Dk, E, old, None, None, new, m, v)
    w_old, w = 4 * H * D, 4 * H * Dk
    b_old, b = w_old + 4 * H * H, w + 4 * H * H
    rows = old[:w_old].view(4 * H, D)
    assert torch.equal(new[:w].view(4 * H, Dk), rows[:, :Dk])
    for i, j in _parts(4 * H * H):
        assert torch.equal(new[w + i:w + j], old[w_old + i:w_old + j]), i
    assert torch.equal(new[b:b + 4 * H], old[b_old:b_old + 4 * H] + rows[:, Dk] * 0.5)
    assert torch.equal(new[b + 4 * H:], old[b_old + 4 * H:])
    for i, j in _parts(n):
        assert not m[i:j].any() and not v[i:j].any(), i
    del old, new, m, v, rows
    torch.cuda.empty_cache()


def test_widen_past_2_34():
    """64 units to 65536: every element is written, the old network's where it belongs."""
    need_gpu()
    D, H, A1, H2 = 8, 64, 3, 1 << 16
    n_old, n = o5.o5_param_count(D, H, A1), o5.o5_param_count(D, H2, A1)
    banner(f"surgery widen to {n} elements")
    assert n > 1 << 34
    old = torch.randn(n_old, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    new, m, v = (torch.full((n,), 7.0, device="cuda") for _ in range(3))
    o5.o5_surgery_widen(D, H, A1, D, H2, old, None, None, new, m, v, 0.0, 3)
    new_wh = new[4 * H2 * D:4 * H2 * (D + H2)].view(4, H2, H2)
    new_b, new_wp = new[n - A1 - A1 * H2 - 4 * H2:n - A1 - A1 * H2].view(4, H2), new[n - A1 - A1 * H2:n - A1].view(A1, H2)
    blocks = [4 * H * D, 4 * H * H, 4 * H, A1 * H, A1]
    wx, wh, b, wp, bp = old.split(blocks)
    assert torch.equal(new[:4 * H2 * D].view(4, H2, D)[:, :H], wx.view(4, H, D))
    assert torch.equal(new_wh[:, :H, :H], wh.view(4, H, H)) and torch.equal(new_b[:, :H], b.view(4, H))
    assert torch.equal(new_wp[:, :H], wp.view(A1, H)) and torch.equal(new[n - A1:], bp)
    # with a scale of 0 everything else is zero: clear the old network's places and look at the rest
    new[:4 * H2 * D].view(4, H2, D)[:, :H] = 0
    new_wh[:, :H, :H] = 0
    new_b[:, :H] = 0
    new_wp[:, :H] = 0
    new[n - A1:] = 0
    for x in (new, m, v):
        for i, j in _parts(n):
            assert not x[i:j].any(), i
    del old, new, m, v, new_wh, new_b, new_wp, x
    torch.cuda.empty_cache()
