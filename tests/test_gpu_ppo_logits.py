"""GPU: the policy loss on logits against its fp64 definition.

Tolerances.  In fp32 a log-probability is a difference of numbers below 32, each rounded to 2^-24 of itself, an exponential of
it and a quotient: 1.5 * 32 * 2^-24 + 4 * 2^-24 < 4e-6 of a probability; the ratio is an exponential of the sum of eight of
them at most: 3e-5 of the largest gradient.  Log-probabilities and KL are such differences: 8 heads * 4e-6 at most.  Sums over
rows hold 3e-5 of the sum of the terms' sizes.  A gradient in bf16 is rounded once more, by at most 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle.ppo_logits import ppo_logits_grad
from paper_1912_06680_amd import o5
from tests.gpu_util import assert_close, banner, host, need_gpu, workspace

pytestmark = pytest.mark.gpu

TOL = 3e-5
TOL_DZ = {False: TOL, True: 2.0 ** -8 + TOL}
HP = (0.2, 0.7, 0.05, 0.3)


class Case:
    """Rows in buffers with columns to spare (which hold NaN and stay), strides of their own."""

    def __init__(self, bf16, N, heads, value=True, ref=True, avail=False, mask=False, weight=False, seed=0, spare=(3, 0, 5)):
        g = np.random.Generator(np.random.PCG64(seed))
        self.bf16, self.N, self.heads, self.A = bf16, N, heads, sum(heads)
        self.dt, self.et = (o5.O5_BF16, torch.bfloat16) if bf16 else (o5.O5_F32, torch.float32)
        self.cols = self.A + value
        f = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731
        self.z = self.rows(self.cols, spare[0], f(2.0 * g.standard_normal((N, self.cols))))
        self.y = self.rows(self.A, spare[1], self.z[:, :self.A].float() + f(0.5 * g.standard_normal((N, self.A)))) if ref else None
        self.dz = torch.full((N, self.cols + spare[2]), 7.0, dtype=self.et, device="cuda")
        self.avail = None
        if avail:
            self.avail = torch.from_numpy((g.random((N, self.A)) < 0.7).astype(np.uint8)).cuda()
        act = np.empty((N, len(heads)), np.int32)
        at = 0
        for k, n in enumerate(heads):
            act[:, k] = g.integers(0, n, N)
            if avail:
                self.avail[torch.arange(N), at + torch.from_numpy(act[:, k]).long()] = 1
            at += n
        self.act = torch.from_numpy(act).cuda()
        self.mask = torch.from_numpy((g.random((N, len(heads))) < 0.8).astype(np.uint8)).cuda() if mask else None
        self.adv, self.ret = f(g.standard_normal(N)), f(g.standard_normal(N)) if value else None
        self.weight = None
        if weight:
            w = g.random(N) * (g.random(N) < 0.7)
            self.weight = f(w / max(w.sum(), 0.1))
        self.logp_old = torch.zeros(N, device="cuda")
        # behaviour's log-probabilities: ratios on all sides of the clip and none within 1e-3 of it
        lr = 0.25 * g.standard_normal(N)
        for edge in np.log([0.8, 1.2]):
            lr = np.where(np.abs(lr - edge) < 2e-3, 0.05, lr)
        logp = ppo_logits_grad(**self.args())[2]
        self.logp_old = f(np.where(np.isfinite(logp), logp, 0.0) - lr)

    def rows(self, cols, spare, x):
        t = torch.full((self.N, cols + spare), float("nan"), dtype=self.et, device="cuda")
        t[:, :cols] = x.to(self.et)
        return t

    def args(self):
        f = lambda t: None if t is None else t.detach().double().cpu().numpy()  # noqa: E731
        i = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
        return dict(logits=f(self.z[:, :self.cols]), act=i(self.act), logp_old=f(self.logp_old), adv=f(self.adv),
                    head_sizes=self.heads, ref=None if self.y is None else f(self.y[:, :self.A]), ret=f(self.ret),
                    weight=f(self.weight), head_mask=i(self.mask), avail=i(self.avail), clip_eps=HP[0], vf_coef=HP[1],
                    ent_coef=HP[2], kl_coef=HP[3] if self.y is not None else 0.0)

    def run(self, hp=HP, rows=True):
        stats = torch.full((9,), 7.0, device="cuda")
        logp, kl = (torch.full((self.N,), 7.0, device="cuda") for _ in range(2)) if rows else (None, None)
        dz = self.dz.clone()
        if not hasattr(self, "ws"):
            self.ws = workspace(o5.o5_ppo_logits_grad_workspace_bytes(self.dt, self.N, self.heads)).fill_(255)
        o5.o5_ppo_logits_grad(self.dt, self.N, self.heads, self.z, self.z.stride(0), self.y,
                              0 if self.y is None else self.y.stride(0), self.act, self.logp_old, self.adv, self.ret, self.weight,
                              self.mask, self.avail, *hp, stats, logp, kl, dz, dz.stride(0), self.ws)
        return stats, dz, logp, kl

    def check(self, out, ref=None):
        stats, dz, logp, kl = out
        r_stats, r_dz, r_logp, r_kl = ppo_logits_grad(**self.args()) if ref is None else ref
        assert (dz[:, self.cols:] == 7).all(), "columns beside the row were written"
        if np.any(r_dz):
            assert_close("dlogits", host(dz[:, :self.cols]), r_dz, TOL_DZ[self.bf16])
        else:
            assert not dz[:, :self.cols].any()
        for name, x, y in (("logp", logp, r_logp), ("kl", kl, r_kl)):
            err = np.abs(host(x) - y)[np.isfinite(y)]
            print(f"    {name}: {np.max(err, initial=0.0):.2e}", flush=True)
            assert np.max(err, initial=0.0) <= 8 * 4e-6
            assert np.array_equal(np.isfinite(host(x)), np.isfinite(y))
        size = 1.0 + abs(r_stats[3]) + abs(r_stats[1]) + abs(r_stats[2])
        got = host(stats)
        assert got[7] == r_stats[7]
        fine = np.isfinite(r_stats)
        err = np.max(np.abs(got[fine] - r_stats[fine]))
        print(f"    stats: {err:.2e}", flush=True)
        assert np.array_equal(np.isfinite(got), fine) and err <= TOL * size


#     N     heads             value  ref    avail  mask   weight
CASES = [
    (1, (1,), False, True, False, False, False),
    (1, (75,), True, True, True, False, False),
    (60, (30, 8, 32, 4), True, True, True, True, False),
    (33, (30, 8, 32, 4), True, False, False, False, True),
    (517, (30, 8, 32, 4), False, True, True, False, True),
    (9000, (3, 5), True, True, False, False, False),
    (40, (1, 1, 1, 2, 3, 5, 8, 128), True, True, True, True, True),
    (37, (129,), False, True, True, False, True),
    (21, (2000, 7, 129), True, True, True, True, False),
    (5, (2048,), True, False, False, False, False),
    (9, (2049, 3), True, True, True, True, True),
    (3, (16384,), False, True, False, False, False),
    (4, (11, 16385), True, True, True, False, True),
    (3, (50257,), True, True, True, False, False),
    (2, (131071, 2), False, True, False, False, False),
    (19, (1, 2), True, True, True, True, True),
    (90, (2, 1), False, False, False, False, False),
    (70, (700,), True, True, True, False, True),
    (5, (9000, 5), True, True, True, True, False),
    (3, (20000,), False, False, True, False, False),
    (77, (3, 1, 9, 2, 1, 8, 5, 4), True, True, True, True, True),
    (1030, (40, 2, 6), False, True, True, True, True),
    (300, (10,), True, True, True, True, True),
    (5000, (3,), False, True, True, False, True),
    (1500, (30,), True, True, True, True, True),
    (1100, (61,), False, True, False, True, True),
    (70, (13,), True, False, True, False, False),
    (41, (1500,), True, True, True, False, True),
    (23, (1200, 130, 1), True, True, True, True, True),
    (23, (2500, 300), False, True, False, True, True),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{'_'.join(map(str, c[1]))}")
def test_loss_and_gradient(bf16, case):
    need_gpu()
    banner(f"ppo_logits bf16={bf16} {case}")
    c = Case(bf16, *case)
    out = c.run()
    c.check(out)
    again = c.run()
    assert all(torch.equal(a, b) for a, b in zip(out, again)), "not the same bits twice"
    stats, dz, _, _ = c.run(rows=False)
    assert torch.equal(stats, out[0]) and torch.equal(dz, out[1])


@pytest.mark.parametrize("N,heads", [(33000, (3, 5)), (140000, (12,)), (70000, (40,)), (9000, (300,)), (2100, (2500,)), (4200, (2000, 600)), (530, (70000, 2))])
def test_more_rows_than_the_chip_takes_at_once(N, heads):
    need_gpu()
    banner(f"ppo_logits {N} rows of {heads}")
    c = Case(True, N, heads, value=False, weight=True, seed=3)
    out = c.run()
    c.check(out)
    assert all(torch.equal(a, b) for a, b in zip(out, c.run())), "not the same bits twice"


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("spare", [(0, 0, 0), (1, 2, 3), (8, 16, 24), (5, 1, 0)])
@pytest.mark.parametrize("heads", [(4099,), (17, 600), (33,), (11,)])
def test_strides(bf16, heads, spare):
    """The same numbers whatever the rows' strides and alignments."""
    need_gpu()
    banner(f"ppo_logits strides bf16={bf16} {heads} {spare}")
    c = Case(bf16, 11, heads, avail=True, spare=spare)
    base = Case(bf16, 11, heads, avail=True, spare=(0, 0, 0))
    out, ref = c.run(), base.run()
    assert all(torch.equal(out[k], ref[k]) for k in (0, 2, 3)) and torch.equal(out[1][:, :c.cols], ref[1])
    c.check(out)


@pytest.mark.parametrize("heads", [(6, 3), (300, 40), (5000,)])
def test_gradient_against_differences(heads):
    """Along a random direction, the loss of the definition in fp64."""
    need_gpu()
    banner(f"ppo_logits gradient against differences {heads}")
    c = Case(False, 12, heads, avail=True, weight=True, seed=5)
    _, dz, _, _ = c.run()
    g = np.random.Generator(np.random.PCG64(6))
    a, v = c.args(), g.standard_normal((12, c.cols))
    J = lambda e: ppo_logits_grad(**{**a, "logits": a["logits"] + e * v})[0][0]  # noqa: E731
    got = host(dz[:, :c.cols])
    assert abs((J(1e-5) - J(-1e-5)) / 2e-5 - np.sum(got * v)) <= TOL * np.sum(np.abs(got * v)) + 1e-9


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads", [(9, 4), (14,), (300, 70), (5000, 3), (20000,)])
def test_what_masks_hide_may_hold_anything(bf16, heads):
    """NaN and infinities in padded rows and in unavailable logits reach nothing; rows without a choice, impossible actions."""
    need_gpu()
    banner(f"ppo_logits masks bf16={bf16} {heads}")
    c = Case(bf16, 12, heads, avail=True, weight=True, seed=7)
    c.weight[2], c.weight[7], c.weight[3] = 0.0, 0.0, 0.1
    c.avail[4, :heads[0]] = 0          # no choice in a head
    c.avail[5] = 0                     # none at all
    c.act[3, 0] = -1
    c.act[6, 0] = heads[0]
    c.avail[9, c.act[9, 0]] = 0        # an action that was not available
    ref = ppo_logits_grad(**c.args())
    for t in (c.z, c.y, c.logp_old, c.adv, c.ret):
        t[2], t[7] = float("nan"), float("inf")
    c.act[2] = 1 << 30
    hidden = c.avail == 0
    c.z[:, :c.A][hidden] = float("nan")
    c.y[:, :c.A][hidden] = float("inf")
    out = c.run()
    c.check(out, ref)
    assert not out[1][[2, 7], :c.cols].any() and not out[1][5, :c.A].any()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("heads", [(9, 4), (14,), (300, 70), (5000,), (20000,)])
def test_extreme_logits(bf16, heads):
    """-infinity, the type's lowest and largest values, offsets of 1e4, choices that only one of the policies excludes."""
    need_gpu()
    banner(f"ppo_logits extreme logits bf16={bf16} {heads}")
    c = Case(bf16, 12, heads, seed=8)
    low, h = float(torch.finfo(c.et).min), heads[0]
    c.z[0, 1:h] = -float("inf")                             # one choice left
    c.act[0, 0] = 0
    c.z[1, :h] = low                                        # all alike, at the lowest
    c.z[2, 1:h // 2] = low                                  # masked by the lowest value in both
    c.y[2, 1:h // 2] = -float("inf")
    c.act[2, 0] = 0
    c.z[3, :h] += 1e4
    c.y[4, :h] -= 1e4
    c.z[5, :h] = -float("inf")                              # as if none were available
    c.z[6, 0], c.act[6, 0] = -float("inf"), 0               # a taken action without probability
    c.z[7, 2], c.act[7, 0] = 3e38, 2                        # one choice far above
    c.y[8, 0] = -float("inf")                               # the reference excludes a choice: KL is infinite
    with np.errstate(all="ignore"):
        r_stats, r_dz, r_logp, r_kl = ppo_logits_grad(**c.args())
    stats, dz, logp, kl = c.run()
    ok = np.array([n for n in range(12) if n not in (8,)])
    dz, kl = host(dz[:, :c.cols]), host(kl)
    assert np.isposinf(kl[8]) and not np.isfinite(dz[8, :h]).all() and float(stats[7]) >= 1 and np.isposinf(r_kl[8])
    assert np.isfinite(dz[ok]).all()
    size = np.max(np.abs(r_dz[ok]))
    assert np.max(np.abs(dz[ok] - r_dz[ok])) <= TOL_DZ[bf16] * size
    assert np.array_equal(np.isfinite(host(logp)), np.isfinite(r_logp))
    fine = [n for n in (0, 1, 2, 9, 10, 11)]
    assert np.max(np.abs(kl - r_kl)[fine] / (1.0 + np.abs(r_kl[fine]))) <= 8 * 4e-6


def test_no_coefficient_no_trace():
    """With kl_coef = 0 a reference is measured and moves nothing, one that excludes choices too; with ref NULL kl is 0."""
    need_gpu()
    banner("ppo_logits without a coefficient")
    c = Case(False, 40, (30, 8), seed=9)
    stats, dz, logp, kl = c.run()
    c.y[3, 2] = -float("inf")
    s0, d0, _, k0 = c.run(hp=(*HP[:3], 0.0))
    c.y = None
    s1, d1, _, k1 = c.run()
    assert torch.equal(d0, d1) and torch.isposinf(k0[3]) and torch.equal(k0[4:], kl[4:]) and not k1.any()
    assert torch.equal(s0[:8], s1[:8]) and float(s1[8]) == 0


def test_it_agrees_with_the_loss_through_the_heads_product():
    """o5_ppo_loss_grad on h = logits and an identity in Wp: the same statistics and bias gradient."""
    need_gpu()
    banner("ppo_logits against ppo_loss_grad")
    heads, N = (30, 8, 21, 4), 300
    c = Case(False, N, heads, ref=False, avail=True, mask=True, spare=(0, 0, 0))
    A1 = c.cols
    assert A1 == 64
    stats, dz, _, _ = c.run()
    s0, dh = torch.empty(8, device="cuda"), torch.empty((N, A1), device="cuda")
    dW, db = torch.empty((A1, A1), device="cuda"), torch.empty(A1, device="cuda")
    ws = workspace(o5.o5_ppo_loss_grad_workspace_bytes(c.dt, N, A1, heads))
    o5.o5_ppo_loss_grad(c.dt, N, A1, heads, c.z, torch.eye(A1, device="cuda"), torch.zeros(A1, device="cuda"), c.act, c.logp_old,
                        c.adv, c.ret, c.mask, *HP[:3], s0, dh, dW, db, ws, avail=c.avail)
    assert_close("stats", host(stats[:8]), host(s0), TOL)
    assert_close("dlogits", host(dz), host(dh), TOL)


def test_another_stream_and_a_graph():
    need_gpu()
    banner("ppo_logits on another stream and in a graph")
    for heads in ((30, 8, 32, 4), (700,), (20000,)):
        c = Case(True, 70, heads, avail=True, weight=True)
        ref = c.run()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            out = c.run()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = c.run()
        for _ in range(3):
            for t in (out[0], out[2], out[3]):
                t.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, ref))
            c.run()
            torch.cuda.synchronize()


def test_refusals():
    need_gpu()
    banner("ppo_logits refusals leave outputs untouched")
    c = Case(False, 4, (6, 3))
    stats = torch.full((9,), 7.0, device="cuda")
    ws = workspace(o5.o5_ppo_logits_grad_workspace_bytes(c.dt, 4, c.heads))

    def call(dt=c.dt, N=4, heads=c.heads, z=c.z, ldl=13, ldr=9, act=c.act, adv=c.adv, eps=0.2, kl=0.1, ldd=15, ws=ws):
        o5.o5_ppo_logits_grad(dt, N, heads, z, ldl, c.y, ldr, act, c.logp_old, adv, c.ret, None, None, None, eps, 1.0, 0.1, kl,
                              stats, None, None, c.dz, ldd, ws)

    for status, bad in ((3, dict(dt=2)), (2, dict(N=0)), (2, dict(heads=(6, 0))), (2, dict(heads=(1,) * 9)), (2, dict(ldl=9)),
                        (2, dict(ldr=8)), (2, dict(ldd=9)), (1, dict(z=None)), (1, dict(act=None)), (4, dict(adv=c.adv[1:])),
                        (7, dict(eps=1.0)), (7, dict(kl=float("inf"))), (5, dict(ws=None)), (2, dict(heads=(1 << 24, 1)))):
        with pytest.raises(o5.O5Error) as e:
            call(**bad)
        assert e.value.status == status, (bad, str(e.value))
    torch.cuda.synchronize()
    assert (stats == 7).all() and (c.dz == 7).all()
