"""The binding's adamw_tensor takes the types from the tensors (CPU): it refuses those that a kernel would read past, or as
something else."""
import pytest
import torch

from paper_1912_06680_amd import o5

N = 1000


def _args(bits=8, **kw):
    state = torch.uint8 if bits == 8 else torch.float32
    a = dict(p=torch.zeros(N), g=torch.zeros(N, dtype=torch.bfloat16), m=torch.zeros(N, dtype=state), v=torch.zeros(N, dtype=state),
             m_exp=torch.zeros(4, dtype=torch.uint8), v_exp=torch.zeros(4, dtype=torch.uint8),
             p_bf16=torch.zeros(N, dtype=torch.bfloat16))
    a.update(kw)
    return a


def test_types_from_the_tensors():
    for bits in (8, 32):
        for g in (torch.zeros(N), torch.zeros(20, 50, dtype=torch.bfloat16)):
            t = o5.adamw_tensor(**_args(bits, g=g))
            assert (t.n, t.bits, t.g_dt) == (N, bits, o5.O5_BF16 if g.dtype == torch.bfloat16 else o5.O5_F32)
    t = o5.adamw_tensor(**_args(32, m_exp=None, v_exp=None, p_bf16=None))
    assert t.m_exp is None and t.p_bf16 is None


@pytest.mark.parametrize("bits,bad", [
    (32, dict(p=torch.zeros(N, dtype=torch.bfloat16))), (32, dict(p=torch.zeros(N, 2)[:, 0])),
    (32, dict(g=torch.zeros(N, dtype=torch.float16))), (8, dict(g=torch.zeros(N, dtype=torch.float64))),
    (8, dict(g=torch.zeros(N - 1))), (32, dict(g=torch.zeros(50, 20).t())),
    (32, dict(m=torch.zeros(N, dtype=torch.bfloat16))), (32, dict(m=torch.zeros(N, dtype=torch.int8))),
    (8, dict(v=torch.zeros(N))), (32, dict(v=torch.zeros(N, dtype=torch.uint8))), (32, dict(v=torch.zeros(N // 2))),
    (8, dict(m_exp=torch.zeros(3, dtype=torch.uint8))), (8, dict(v_exp=torch.zeros(4))),
    (8, dict(p_bf16=torch.zeros(N))), (8, dict(p_bf16=torch.zeros(N - 8, dtype=torch.bfloat16))),
])
def test_refusals(bits, bad):
    with pytest.raises(ValueError, match=next(iter(bad))):
        o5.adamw_tensor(**_args(bits, **bad))
