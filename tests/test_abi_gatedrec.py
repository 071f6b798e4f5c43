"""The gated recurrence's entry points on the CPU: host-side refusals and size queries (no GPU: every call below fails before
any HIP call, or only computes sizes)."""
import pytest

from paper_1912_06680_amd import o5

F, BF = o5.O5_F32, o5.O5_BF16
P = 16  # an aligned address that is never read


@pytest.fixture(scope="module")
def lib():
    return o5.lib()


def _put(x, i, v):
    return [*x[:i], v, *x[i + 1:]]


def test_refusals(lib):
    size = [BF, 16, 4, 64]
    ins = [P, 64, P, 192, P, 64, P, 8.0]
    need, bneed = lib.o5_gatedrec_fwd_workspace_bytes(*size), lib.o5_gatedrec_bwd_workspace_bytes(*size)
    assert need > 0 and bneed > 0 and lib.o5_gatedrec_marks_bytes(*size[1:]) >= 4 * 64 * 4

    def fwd(size=size, ins=ins, h0=None, reset=None, h=P, ldh=64, hT=None, marks=None, ws=P, n=need):
        return lib.o5_gatedrec_fwd(*size, *ins, h0, reset, h, ldh, hT, marks, ws, n, None)

    for i, bad, status in ((0, 2, 3), (1, 0, 2), (2, -1, 2), (3, 0, 2), (3, 60, 2), (3, 65544, 2), (1, 2 ** 28, 2), (2, 2 ** 27, 2)):
        assert fwd(size=_put(size, i, bad)) == status, (i, bad, o5.o5_last_error())
        assert lib.o5_gatedrec_fwd_workspace_bytes(*_put(size, i, bad)) == 0
        assert lib.o5_gatedrec_bwd_workspace_bytes(*_put(size, i, bad)) == 0
        if i:
            assert lib.o5_gatedrec_marks_bytes(*_put(size, i, bad)[1:]) == 0
    for i, bad, status in ((0, None, 1), (2, None, 1), (4, None, 1), (6, None, 1), (0, 24, 4), (4, 8, 4), (1, 56, 2), (3, 68, 2),
                           (5, 2 ** 31, 2), (7, float("inf"), 7), (7, 0.0, 7), (7, -1.0, 7), (7, float("nan"), 7)):
        assert fwd(ins=_put(ins, i, bad)) == status, (i, bad, o5.o5_last_error())
    assert fwd(h=None) == 1 and fwd(ldh=56) == 2 and fwd(h0=20) == 4 and fwd(hT=20) == 4 and fwd(marks=20) == 4
    assert fwd(reset=2) == 4 and fwd(ws=None) == 5 and fwd(n=need - 1) == 5

    outs = [P, 64, P, 64, P, 192]

    def bwd(size=size, ins=ins, marks=P, reset=None, dh=P, lddh=64, dhT=None, outs=outs, dlam=P, dh0=None, ws=P, n=bneed):
        return lib.o5_gatedrec_bwd(*size, *ins, marks, reset, dh, lddh, dhT, *outs, dlam, dh0, ws, n, None)

    assert bwd(marks=None) == 1 and bwd(dh=None) == 1 and bwd(dlam=None) == 1 and bwd(lddh=8) == 2 and bwd(dhT=4) == 4
    assert bwd(dh0=4) == 4 and bwd(n=bneed - 1) == 5 and bwd(ws=None) == 5 and bwd(ins=_put(ins, 7, -8.0)) == 7
    for i, bad, status in ((0, None, 1), (1, 32, 2), (2, 8, 4), (4, None, 1), (5, 100, 2)):
        assert bwd(outs=_put(outs, i, bad)) == status

    step = [BF, 4, 64]
    assert lib.o5_gatedrec_step(*step, *ins, None, None, P, 64, None) == 1
    assert lib.o5_gatedrec_step(*step, *ins, 20, P, P, 64, None) == 4
    assert lib.o5_gatedrec_step(*step, *ins, None, P, P, 60, None) == 2
    assert lib.o5_gatedrec_step(*_put(step, 1, 0), *ins, None, P, P, 64, None) == 2


def test_workspaces(lib):
    """Scratch stays small beside the rows, whatever the lengths."""
    for dt in (F, BF):
        for T, B, D in ((1, 1, 8), (16, 2048, 4096), (256, 128, 4096), (10007, 1, 2048), (1 << 20, 1, 64), (5000, 30, 1000)):
            rows = T * B * D * (2 if dt == BF else 4)
            assert 0 < lib.o5_gatedrec_fwd_workspace_bytes(dt, T, B, D) <= max(1 << 16, rows // 4)
            assert 0 < lib.o5_gatedrec_bwd_workspace_bytes(dt, T, B, D) <= max(1 << 16, 2 * rows)
