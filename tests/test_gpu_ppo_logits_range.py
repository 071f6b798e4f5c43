"""GPU: the policy loss on logits that lie far from 0, and from each other.

Tolerances.  A logit less the largest is rounded to 2^-24 of itself whatever their size, log s is below 32: a log-probability
holds 4e-6 (1 + |log p|), as where the logits are small, and KL that of its terms.  A gradient is p times a sum of terms that
are each rounded so: 3e-5 of the largest of policy gradient, entropy and KL terms of its row; in bf16 2^-8 of itself more."""
import numpy as np
import pytest
import torch

import tests.test_gpu_ppo_logits as base
from oracle.ppo_logits import ppo_logits_grad
from tests.gpu_util import banner, host, need_gpu

pytestmark = pytest.mark.gpu

# heads of every way through the kernels: teams of 4, 8, 16, 64 and more lanes, few slots and many, rows read twice
HEADS = [(3,), (1, 2), (14,), (9, 4), (60,), (30, 8, 32, 4), (100,), (300, 70), (700,), (700, 30), (2600,), (2600, 5), (5000,),
         (7000, 3), (9000,), (9000, 5), (20000,), (70000,), (140000,), (70000, 40)]


def check(c):
    with np.errstate(all="ignore"):
        r_stats, r_dz, r_logp, r_kl = ppo_logits_grad(**c.args())
    stats, dz, logp, kl = c.run()
    logp, kl, dz, got = host(logp), host(kl), host(dz[:, :c.cols]), host(stats)
    assert np.isfinite(r_logp).all() and np.isfinite(r_kl).all() and r_stats[7] == got[7] == 0
    K = len(c.heads)
    worst = lambda a, b: float(np.max(np.abs(a - b) / (1.0 + np.abs(b))))  # noqa: E731
    print(f"    logp {worst(logp, r_logp):.2e} kl {worst(kl, r_kl):.2e}", flush=True)
    assert worst(logp, r_logp) <= K * 4e-6 and worst(kl, r_kl) <= K * 4e-6
    # (the KL terms p (log p - log q - KL) of a gradient cancel where KL is large: their size is KL's)
    w = 1.0 / c.N
    size = np.max(np.abs(r_dz), axis=1) + w * base.HP[3] * np.abs(r_kl) + w * base.HP[2] * np.log(c.A + 1.0)
    err = np.max(np.abs(dz - r_dz) - 2.0 ** -8 * np.abs(r_dz) * c.bf16, axis=1) / size
    print(f"    dlogits {np.max(err):.2e}", flush=True)
    assert np.max(err) <= base.TOL
    assert np.all(np.abs(got - r_stats) <= base.TOL * (1.0 + np.max(np.abs(r_stats[1:4])) + base.HP[3] * r_stats[8]))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "_".join(map(str, h)))
def test_far_logits(bf16, heads):
    """Heads moved by up to 1e38 as a whole, single choices that far above and below the others, in the policy's logits and in
    the reference's."""
    need_gpu()
    banner(f"ppo_logits far logits bf16={bf16} {heads}")
    far = (1e4, 1e5, 1e7, 3e8, 2e9, 1e10, 1e12, 1e20, 1e30, 2e36, 1e38)
    c = base.Case(bf16, 6 * len(far), heads, seed=11)
    h = heads[0]
    for k, v in enumerate(far):
        n = 6 * k
        c.z[n, :h] += v
        c.z[n + 1, :h] -= v
        c.z[n + 2, h - 1] = v                        # one choice far above
        c.act[n + 2, 0] = h - 1
        c.y[n + 2, :h] = 0.0
        c.z[n + 3, :h - 1] = -v                      # all but one filled with a low number
        c.act[n + 3, 0] = h - 1
        c.y[n + 4, :h] += v                          # a reference far away as a whole
        c.y[n + 5, :h] -= v
        c.z[n + 5, 0], c.y[n + 5, 0] = -v, -2.0 * v  # a choice that neither makes
        c.act[n + 5, 0] = h - 1
    # ratios near 1, as where the logits are small
    c.logp_old = torch.zeros_like(c.logp_old)
    with np.errstate(all="ignore"):
        logp = ppo_logits_grad(**c.args())[2]
    g = np.random.Generator(np.random.PCG64(12))
    c.logp_old = torch.from_numpy((np.where(np.abs(logp) < 100.0, logp, 0.0) - 0.03 * g.standard_normal(c.N)).astype(np.float32)).cuda()
    check(c)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads", [(20000,), (70000,), (140000,), (9000, 9000), (40000, 3)], ids=lambda h: "_".join(map(str, h)))
def test_offsets_where_rows_are_read_twice(bf16, heads):
    """The same policy at an offset has the same log-probabilities, also where a lane's largest logit grows as it goes on."""
    need_gpu()
    banner(f"ppo_logits offsets bf16={bf16} {heads}")
    c = base.Case(bf16, 8, heads, seed=13)
    for n, v in enumerate((0.0, 1e3, -1e3, 1e4, -1e4, 1e5, -1e5, 3e6)):
        c.z[n, :c.A] += v
        c.y[n] -= v
    c.z[3, :c.A] += torch.linspace(-20.0, 20.0, c.A, device="cuda").to(c.et)
    c.logp_old = torch.zeros_like(c.logp_old)
    with np.errstate(all="ignore"):
        c.logp_old = torch.from_numpy((ppo_logits_grad(**c.args())[2] + 0.02).astype(np.float32)).cuda()
    check(c)


class Wide(base.Case):
    def check(self, out, ref):
        """As for narrow heads, but for the statistics' size.  A row whose wide head has no choice left lacks that head's
        log-probability, d = ln 70000 = 11 of log r: r = e^d is off by 2^-24 (2 d + 4) < 3e-5 of itself, and r, r - 1 - d and
        the policy loss (r A, where A < 0) are of the size of w r, which the narrow heads' bound takes to be 1."""
        stats, r_stats = host(out[0]), ref[0]
        fine = np.isfinite(r_stats)
        size = 1.0 + abs(r_stats[3]) + abs(r_stats[1]) + abs(r_stats[2]) + abs(r_stats[6])
        assert np.array_equal(np.isfinite(stats), fine) and stats[7] == r_stats[7]
        assert np.max(np.abs(stats - r_stats)[fine]) <= base.TOL * size
        super().check((torch.from_numpy(r_stats).cuda(), *out[1:]), ref)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads", [(70000,), (140000,), (40000, 3), (9000, 9000)], ids=lambda h: "_".join(map(str, h)))
def test_what_masks_hide_where_rows_are_read_twice(monkeypatch, bf16, heads):
    monkeypatch.setattr(base, "Case", Wide)
    base.test_what_masks_hide_may_hold_anything(bf16, heads)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("avail", [False, True])
@pytest.mark.parametrize("heads", [(2, 3), (14,), (9, 4), (300, 70), (2600, 5), (9000, 5), (9000, 9000), (40000, 3), (3, 40000), (70000,)],
                         ids=lambda h: "_".join(map(str, h)))
def test_a_head_of_infinities_adds_nothing(bf16, avail, heads):
    """A head whose available logits are all -infinity is as one without a choice, also where its action could be one."""
    need_gpu()
    banner(f"ppo_logits heads of -infinity bf16={bf16} avail={avail} {heads}")
    c = Wide(bf16, 9, heads, avail=avail, seed=14)
    at, dead = 0, []
    for k, n in enumerate(heads):
        for row in ((1, 4) if k % 2 == 0 else (2, 4)):
            c.z[row, at:at + n] = -float("inf")
            dead.append((row, slice(at, at + n)))
        at += n
    out = c.run()
    c.check(out, ppo_logits_grad(**c.args()))
    for row, cols in dead:
        assert not out[1][row, cols].any()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads", [(70000,), (140000,), (40000, 3), (9000, 9000)], ids=lambda h: "_".join(map(str, h)))
def test_extreme_logits_where_rows_are_read_twice(bf16, heads):
    base.test_extreme_logits(bf16, heads)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "_".join(map(str, h)))
def test_a_reference_near_by(bf16, heads):
    """KL of 1e-5 to 1e-2 a head, to what the terms of its sums hold.

    KL = sum p (d - dy) + log(sr / s), with d and dy what the logits lie below the largest, 10 on the average over p for these
    (ln A and less): each product and the two sums are off by 4e-6 of themselves at most in the worst case, but p's errors are
    the ones that log(sr / s) has with the other sign, so that 4 roundings to 2^-24 of 10 are left, 2.4e-6 a head; 4e-6 with
    log2's and the reciprocal's."""
    need_gpu()
    banner(f"ppo_logits near reference bf16={bf16} {heads}")
    c = base.Case(bf16, 24, heads, seed=15)
    g = np.random.Generator(np.random.PCG64(16))
    near = torch.from_numpy(g.standard_normal((24, c.A)).astype(np.float32)).cuda()
    for n in range(24):
        # (bf16 has neighbours of a logit at 2^-8 of it; in fp32 the reference as near as 1e-5 of KL)
        c.y[n] = (c.z[n, :c.A].float() + (0.005, 0.02, 0.08)[n % 3] * near[n]).to(c.et)
    _, _, _, r_kl = ppo_logits_grad(**c.args())
    kl = host(c.run()[3])
    worst = float(np.max(np.abs(kl - r_kl)))
    print(f"    kl: {worst:.2e} of {np.min(r_kl):.1e} to {np.max(r_kl):.1e}", flush=True)
    assert worst <= len(heads) * 4e-6
    # a KL of 0 would not pass, where there is more than one choice
    assert max(heads) == 1 or np.max(r_kl) > 8 * len(heads) * 4e-6
