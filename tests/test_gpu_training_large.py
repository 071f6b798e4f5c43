"""GPU: the gated recurrence and the loss on logits on buffers whose offsets pass 32 bits, and in calls that go out in several
launches, against the same rows in small buffers."""
import pytest
import torch

from paper_1912_06680_amd import o5
from tests.gpu_util import banner, need_gpu, workspace

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


@pytest.mark.parametrize("T,B,D", [(10, 40, 72), (300, 1, 64), (2, 40, 4096)])
def test_gatedrec_rows_far_apart(T, B, D):
    """Row strides of 2^24 elements: hundreds of rows span 13 GB, and a launch takes 32 samples at most."""
    need_gpu()
    banner(f"gatedrec rows far apart {T}x{B}x{D}")
    dt, ld = o5.O5_BF16, 1 << 24
    g = _gen(0)
    small = [torch.randn((T * B, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(4)]
    lam, h0 = torch.randn(D, generator=g, device="cuda") - 3.0, torch.randn((B, D), generator=g, device="cuda")
    dhT = torch.randn((B, D), generator=g, device="cuda")
    reset = (torch.rand((T, B), generator=g, device="cuda") < 0.1).to(torch.uint8)
    wide = torch.empty(T * B * ld, dtype=torch.bfloat16, device="cuda").view(T * B, ld)
    far = [wide[:, i * 8192:i * 8192 + D] for i in range(4)]
    for a, b in zip(far, small):
        a.copy_(b)
    size = (T, B, D)
    ws = workspace(max(o5.o5_gatedrec_fwd_workspace_bytes(dt, *size), o5.o5_gatedrec_bwd_workspace_bytes(dt, *size)))

    def both(x, r, i, dh, ld, outs, ldo):
        marks = torch.empty(o5.o5_gatedrec_marks_bytes(*size) // 4, device="cuda")
        hT, dh0, dlam = torch.empty_like(h0), torch.empty_like(h0), torch.empty_like(lam)
        ins = (x, ld, r, ld, i, ld, lam, 8.0)
        o5.o5_gatedrec_fwd(dt, *size, *ins, h0, reset, outs[0], ldo, hT, marks, ws)
        o5.o5_gatedrec_bwd(dt, *size, *ins, marks, reset, dh, ld, dhT, outs[1], ldo, outs[2], ldo, outs[3], ldo, dlam, dh0, ws)
        return hT, dh0, dlam

    ref = [torch.empty_like(x) for x in small]
    states = both(*small, D, ref, D)
    out = [wide[:, 65536 + i * 8192:65536 + i * 8192 + D] for i in range(4)]
    assert all(torch.equal(a, b) for a, b in zip(states, both(*far, ld, out, ld)))
    assert all(torch.equal(a, b) for a, b in zip(ref, out))
    if T == 2:  # single tokens
        S, S2 = h0.clone(), h0.clone()
        o5.o5_gatedrec_step(dt, B, D, small[0], D, small[1], D, small[2], D, lam, 8.0, None, S, ref[0], D)
        o5.o5_gatedrec_step(dt, B, D, far[0], ld, far[1], ld, far[2], ld, lam, 8.0, None, S2, out[0], ld)
        assert torch.equal(S, S2) and torch.equal(ref[0][:B], out[0][:B])


def test_gatedrec_of_many_samples():
    """2^27 samples of 8 channels: more lanes than offsets of 32 bits take at once; the states of samples at both ends of each
    launch next to the same samples alone."""
    need_gpu()
    banner("gatedrec, 2^27 samples of 8 channels")
    B, D, dt = (1 << 27) - 5, 8, o5.O5_BF16
    g = _gen(1)
    x = torch.randn((B, D), generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    lam = torch.randn(D, generator=g, device="cuda")
    S, h = torch.ones((B, D), device="cuda"), torch.empty((B, D), dtype=torch.bfloat16, device="cuda")
    o5.o5_gatedrec_step(dt, B, D, x, D, x, D, x, D, lam, 8.0, None, S, h, D)
    hT, seq = torch.full((B, D), 7.0, device="cuda"), torch.empty((B, D), dtype=torch.bfloat16, device="cuda")
    ws = workspace(o5.o5_gatedrec_fwd_workspace_bytes(dt, 1, B, D))
    o5.o5_gatedrec_fwd(dt, 1, B, D, x, D, x, D, x, D, lam, 8.0, torch.ones((B, D), device="cuda"), None, seq, D, hT, None, ws)
    assert torch.equal(S, hT) and torch.equal(h, seq)
    for a in (0, (1 << 26) - 64, B - 512):
        a &= ~7
        n = min(512, B - a)
        one, o = torch.ones((n, D), device="cuda"), torch.empty((n, D), dtype=torch.bfloat16, device="cuda")
        xa = x[a:a + n].clone()
        o5.o5_gatedrec_step(dt, n, D, xa, D, xa, D, xa, D, lam, 8.0, None, one, o, D)
        assert torch.equal(one, S[a:a + n]) and torch.equal(o, h[a:a + n])
    del x, S, h, hT, seq
    torch.cuda.empty_cache()


@pytest.mark.parametrize("heads", [(30, 8, 32, 4), (3000,), (70000, 3)])
def test_logits_rows_far_apart(heads):
    """Row strides of 2^24 - 1 elements: 300 rows span 10 GB, at every alignment."""
    need_gpu()
    banner(f"ppo_logits rows far apart {heads}")
    N, A, ld, dt = 300, sum(heads), (1 << 24) - 1, o5.O5_BF16
    g = _gen(2)
    z, y = (torch.randn((N, A + 1), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    act = torch.stack([torch.randint(0, n, (N,), generator=g, device="cuda", dtype=torch.int32) for n in heads], 1).contiguous()
    adv, ret, old = (torch.randn(N, generator=g, device="cuda") for _ in range(3))
    wide = torch.empty(N * ld + (1 << 20), dtype=torch.bfloat16, device="cuda")
    far = [torch.as_strided(wide, (N, A + 1), (ld, 1), i << 18) for i in range(3)]
    far[0].copy_(z)
    far[1].copy_(y)
    ws = workspace(o5.o5_ppo_logits_grad_workspace_bytes(dt, N, heads))

    def run(z, y, ld, dz):
        stats, logp, kl = torch.empty(9, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        o5.o5_ppo_logits_grad(dt, N, heads, z, ld, y, ld, act, old, adv, ret, None, None, None, 0.2, 1.0, 0.01, 0.1, stats, logp, kl,
                              dz, ld, ws)
        return stats, logp, kl

    dz = torch.empty_like(z)
    ref = run(z, y, A + 1, dz)
    assert all(torch.equal(a, b) for a, b in zip(ref, run(far[0], far[1], ld, far[2])))
    assert torch.equal(dz, far[2])
    del wide, far
    torch.cuda.empty_cache()


@pytest.mark.parametrize("heads", [(1 << 24,), (5, (1 << 23) + 1, 3, 1 << 22)])
def test_as_many_logits_as_there_may_be(heads):
    """2^24 choices in one head, and nearly as many in several.

    A probability here is 1e-7 and a sum over a head's has 2^23 terms of like size, added by lanes in runs of at most 2^14 and
    joined in pairs: relative errors of 2^14 2^-24 = 1e-3 at the very most and, as errors of random sign, 2^7 2^-24 = 8e-6.  Of
    log p, near -17, 1e-5 is allowed on top of an exponential's 2^-22 for each; of the gradient, relative to its largest,
    (2^-14 + 2^-8)."""
    need_gpu()
    banner(f"ppo_logits of {sum(heads)} logits")
    N, A, dt = 2, sum(heads), o5.O5_BF16
    g = _gen(3)
    z, y = (torch.randn((N, A), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    act = torch.stack([torch.randint(0, n, (N,), generator=g, device="cuda", dtype=torch.int32) for n in heads], 1).contiguous()
    act[1, -1] = heads[-1] - 1
    adv, w = torch.tensor([1.5, -0.5], device="cuda"), torch.tensor([0.25, 0.75], device="cuda")
    logp = sum(torch.log_softmax(s.double(), -1).gather(1, act[:, k:k + 1].long())[:, 0]
               for k, s in enumerate(z.split(heads, 1)))
    kl = sum((s.double().softmax(-1) * (s.double().log_softmax(-1) - q.double().log_softmax(-1))).sum(-1)
             for s, q in zip(z.split(heads, 1), y.split(heads, 1)))
    old = (logp - 0.1).float()
    stats, got_logp, got_kl = torch.empty(9, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    dz, ws = torch.full((N, A), 7.0, dtype=torch.bfloat16, device="cuda"), workspace(o5.o5_ppo_logits_grad_workspace_bytes(dt, N, heads))
    o5.o5_ppo_logits_grad(dt, N, heads, z, A, y, A, act, old, adv, None, w, None, None, 0.2, 0.0, 0.0, 1.0, stats, got_logp, got_kl,
                          dz, A, ws)
    assert (got_logp.double() - logp).abs().max() <= len(heads) * (1e-5 + 17 * 2.0 ** -22)
    assert (got_kl.double() - kl).abs().max() <= len(heads) * (1e-5 + 17 * 2.0 ** -22)
    ratio = (logp - old.double()).exp()  # 1.1: inside the clip
    at = 0
    for k, n in enumerate(heads):
        s, q = z[:, at:at + n].double(), y[:, at:at + n].double()
        lp = s.log_softmax(-1)
        d = lp - q.log_softmax(-1)
        p = lp.exp()
        ref = p * (ratio * adv.double())[:, None] + p * (d - (p * d).sum(-1, keepdim=True))
        ref.scatter_add_(1, act[:, k:k + 1].long(), -(ratio * adv.double())[:, None])
        ref *= w.double()[:, None]
        got = dz[:, at:at + n].double()
        others = torch.ones_like(ref, dtype=torch.bool).scatter_(1, act[:, k:k + 1].long(), False)
        for m in (others, ~others):  # the action's is near 1, the others' near 1e-7
            assert (got - ref)[m].abs().max() <= (2.0 ** -14 + 2.0 ** -8) * ref[m].abs().max()
        at += n
    torch.cuda.empty_cache()
