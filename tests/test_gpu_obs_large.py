"""GPU: observations of more elements than one launch's threads hold (2^32 threads of four elements)."""
import pytest
import torch

from paper_1912_06680_amd import o5
from tests.gpu_util import banner, need_gpu, workspace

pytestmark = pytest.mark.gpu


def test_observations_past_2_34():
    """Rows of +2 and -2 in turn have a mean of 0 and a deviation of 2 in every feature: +1 and -1 everywhere."""
    need_gpu()
    N, D = (1 << 20) + 2, 16388
    banner(f"observations {N} x {D}")
    assert N * D > 1 << 34
    obs = torch.empty((N // 2, 2, D), device="cuda")
    obs[:, 0], obs[:, 1] = 2.0, -2.0
    out = torch.full((N // 2, 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
    stats = torch.zeros((3, D), dtype=torch.float64, device="cuda")
    ws = workspace(o5.o5_obs_normalize_workspace_bytes(N, D))
    o5.o5_obs_normalize(o5.O5_BF16, N, D, obs, stats, 5.0, 1e-8, out, ws)
    assert (stats[0] == N).all() and stats[1].abs().max() < 1e-9 and (stats[2] / N - 4.0).abs().max() < 1e-9
    for i in range(0, N // 2, 1 << 15):
        part = out[i:i + (1 << 15)]
        assert (part[:, 0] == 1).all() and (part[:, 1] == -1).all(), i
    del obs, out, part
    torch.cuda.empty_cache()
