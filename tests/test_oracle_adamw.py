"""Pins of the AdamW oracle: PyTorch's AdamW in fp64, the generator's statistics, the 8-bit codes' spacing and bias."""
import numpy as np
import torch

from oracle.adamw import chances, neighbours, philox4x32_7, rounded, value_of, adamw_step


def test_against_pytorch():
    r = np.random.Generator(np.random.PCG64(0))
    p0 = r.standard_normal(50)
    w = torch.nn.Parameter(torch.from_numpy(p0.copy()))
    opt = torch.optim.AdamW([w], lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    p, m, v = p0.copy(), np.zeros(50), np.zeros(50)
    for step in range(1, 6):
        g = r.standard_normal(50)
        w.grad = torch.from_numpy(g.copy())
        opt.step()
        p, m, v = adamw_step(p, m, v, g, 1e-2, 0.9, 0.99, 1e-8, 0.0, 0.1, step)
        assert np.allclose(p, w.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_generator_is_uniform_and_counters_matter():
    um, uv = chances(20000, 3, 1, 11)
    for u in (um, uv):
        counts = np.histogram(u, 16, (0, 1))[0]
        assert np.sum((counts - 1250.0) ** 2) / 1250.0 < 45.0  # chi^2 of 15 degrees, p < 1e-4
    assert abs(np.corrcoef(um, uv)[0, 1]) < 0.03
    words = {tuple(philox4x32_7(c, k)) for c, k in (((0, 0, 1, 0), (7, 0)), ((1, 0, 1, 0), (7, 0)), ((0, 1, 1, 0), (7, 0)),
                                                    ((0, 0, 2, 0), (7, 0)), ((0, 0, 1, 1), (7, 0)), ((0, 0, 1, 0), (8, 0)),
                                                    ((0, 0, 1, 0), (7, 1)))}
    assert len(words) == 7


def test_codes_are_the_neighbours():
    """Every code's value is its own rounding, and the codes of a group run in steps of 1/8 of a binade."""
    for which, codes in (("m", np.arange(0, 120)), ("v", np.arange(1, 248))):
        x = value_of(codes, [127 + 4], which)
        assert np.all(np.diff(x) > 0)
        top = np.concatenate([x, [2.0 ** 4 * 1.5]])  # a largest value in binade 4
        low, _, a = neighbours(top, which)
        assert a[0] == 4 and np.array_equal(low[:-1], x)


def test_rounding_has_no_bias():
    x = np.full(256 * 64, 1.03) * np.where(np.arange(256 * 64) % 2, 1, -1)
    um, uv = chances(x.size, 1, 0, 5)
    assert abs(np.mean(np.abs(rounded(x, um, "m"))) - 1.03) < 0.125 * 4 / np.sqrt(x.size)
    assert abs(np.mean(rounded(np.abs(x), uv, "v")) - 1.03) < 0.125 * 4 / np.sqrt(x.size)
    tiny = np.array([1.0] + [1e-12] * 255)
    assert rounded(tiny, np.zeros(256), "v")[1] > 0 and rounded(tiny, np.zeros(256), "m")[1] == 0
