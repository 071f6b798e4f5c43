"""The operators of a recurrent policy's training step, as measurable cases.

Three operators, reached through the ``o5_*`` bindings:

gatedrec  a linear recurrence whose decay and input are gated by the input: over T steps (forward and backward) and for
          single tokens on a state kept in place
logits    the clipped policy loss with value, entropy and KL terms on logits, and its gradient
gradnorm  the global norm of many tensors' gradients, and AdamW on gradients clipped to it

Kinds: ``fwd``, ``bwd`` and ``step`` (gatedrec), ``loss`` (logits), ``norm`` and ``clip`` (gradnorm).  With ``own`` false
``run`` computes the same from elementary torch operations in 32 bits; ``exact`` computes it in 64 bits from the
definitions.
"""
import math

import torch

own = False

DEV = "cuda"
C = 8.0        # the recurrence's factor on its rates
HEADS = (30, 8, 32, 4)  # the action heads of the synthetic configurations
BLOCK = 256    # every tensor of the flat parameter buffers starts at a multiple of it

CLIP_EPS, VF, ENT, KL = 0.2, 1.0, 0.01, 0.1
HP = {"lr": 5e-5, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "clip_k": 0.0, "seed": 7, "step": 20}
STATS = 9      # total, policy, value, entropy, clipped share, approximate KL, ratio, rows not finite, KL


def listed():
    return [
        # one environment's next action at width 1024: a single token, latency
        {"name": "step_1", "kind": "step", "dtype": "bf16", "B": 1, "D": 1024, "resets": False, "fused": True},
        # rollout inference for 4,096 environments at width 4096
        {"name": "step_4096", "kind": "step", "dtype": "bf16", "B": 4096, "D": 4096, "resets": True, "fused": True},
        # whole 256-step segments of the benchmark's batch at width 4096, for training
        {"name": "fwd_segments", "kind": "fwd", "dtype": "bf16", "T": 256, "B": 128, "D": 4096, "resets": True, "fused": True,
         "train": True},
        # one long history: the work has to be split over time
        {"name": "fwd_long", "kind": "fwd", "dtype": "bf16", "T": 10007, "B": 1, "D": 2048, "resets": False, "fused": True,
         "train": False},
        # training on whole segments
        {"name": "bwd_segments", "kind": "bwd", "dtype": "bf16", "T": 256, "B": 64, "D": 4096, "resets": True, "fused": True,
         "train": True},
        # training in full precision on a few environments, with sizes that are no multiple of a tile
        {"name": "bwd_odd_f32", "kind": "bwd", "dtype": "f32", "T": 277, "B": 24, "D": 1000, "resets": True, "fused": False,
         "train": True},
        # the action heads of a few environments' rows: latency
        {"name": "loss_60", "kind": "loss", "dtype": "f32", "N": 60, "heads": "30 8 32 4", "value": True, "ref": True,
         "avail": True, "pad": 0.0},
        # the benchmark's 32,768 rows, heads and value, held near an earlier policy
        {"name": "loss_full", "kind": "loss", "dtype": "bf16", "N": 32768, "heads": "30 8 32 4", "value": True, "ref": True,
         "avail": True, "pad": 0.0},
        # one head of 32,000 choices over a padded batch of token rows
        {"name": "loss_wide", "kind": "loss", "dtype": "bf16", "N": 8192, "heads": "32000", "value": False, "ref": True,
         "avail": False, "pad": 0.1},
        # full precision, an odd number of choices, some of them not available, with a value
        {"name": "loss_odd_f32", "kind": "loss", "dtype": "f32", "N": 1003, "heads": "50257", "value": True, "ref": True,
         "avail": True, "pad": 0.05},
        # the gradients of every tensor of a small policy
        {"name": "norm_small", "kind": "norm", "g": "f32", "width": 512, "layers": 4, "mirror": False},
        # every tensor of a 4096-wide policy: norm, clip and update
        {"name": "clip_full", "kind": "clip", "g": "bf16", "width": 4096, "layers": 2, "mirror": True},
    ]


# ------------------------------------------------------------------ draws


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_any(rng):
    kind = rng.choice(("step", "fwd", "fwd", "bwd", "bwd", "loss", "loss", "loss", "norm", "clip"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("step", "fwd", "bwd"):
        c = {"kind": kind, "dtype": dtype, "B": _log_int(rng, 1, 4096 if kind == "step" else 1024), "D": 8 * _log_int(rng, 1, 1024),
             "resets": rng.random() < 0.6, "fused": rng.random() < 0.5}
        if kind != "step":
            c["T"] = _log_int(rng, 1, 12000)
            c["train"] = kind == "bwd" or rng.random() < 0.5
        return c
    if kind == "loss":
        if rng.random() < 0.5:
            heads = [_log_int(rng, 1, 131072)]
        else:
            heads = [_log_int(rng, 1, 2000) for _ in range(rng.randint(2, 8))]
        return {"kind": kind, "dtype": dtype, "N": _log_int(rng, 1, 32768), "heads": " ".join(map(str, heads)),
                "value": rng.random() < 0.5, "ref": rng.random() < 0.7, "avail": rng.random() < 0.5,
                "pad": rng.choice((0.0, 0.2))}
    return {"kind": kind, "g": rng.choice(("f32", "bf16")), "width": 8 * _log_int(rng, 8, 512), "layers": rng.randint(1, 8),
            "mirror": kind == "clip" and rng.random() < 0.7}


def _cost(c):
    """A rough time in microseconds, to keep draws below the largest listed case."""
    w = work(c)
    return w["bytes"] / 3e6 + w["flops"] / 50e6


def draw(rng):
    most = {kind: max(_cost(c) for c in listed() if c["kind"] in kinds) for kinds in _FAMILIES for kind in kinds}
    while True:
        c = _draw_any(rng)
        if _cost(c) <= most[c["kind"]]:
            return c


_FAMILIES = (("step",), ("fwd", "bwd"), ("loss",), ("norm", "clip"))


# ------------------------------------------------------------------- work


def _es(t):
    return 2 if t == "bf16" else 4


def _heads(c):
    return [int(n) for n in c["heads"].split()]


def work(case):
    c = case
    k = c["kind"]
    if k in ("step", "fwd", "bwd"):
        rows, state = c["B"] * c.get("T", 1), c["B"] * c["D"] * 4
        n, e = rows * c["D"], _es(c["dtype"])
        resets = rows if c["resets"] else 0
        if k == "bwd":  # in: x, r, i, dh, h0, dhT; out: dx, dr, di, dh0, dlam
            return {"bytes": 7 * n * e + 3 * state + resets, "flops": n * 40.0}
        return {"bytes": 4 * n * e + 2 * state + resets, "flops": n * 20.0}  # in: x, r, i, h0; out: h, hT
    if k == "loss":
        heads = _heads(c)
        A = sum(heads)
        cols = A + (1 if c["value"] else 0)
        per = cols * 2 + (A if c["ref"] else 0)  # in: logits, ref; out: the gradient
        rows = 4 * len(heads) + 8 + (4 if c["value"] else 0) + (4 if c["pad"] else 0) + (A if c["avail"] else 0) + 8
        return {"bytes": c["N"] * (per * _es(c["dtype"]) + rows), "flops": c["N"] * A * (30.0 if c["ref"] else 20.0)}
    n = sum(_sizes(c))
    if k == "norm":
        return {"bytes": n * _es(c["g"]), "flops": n * 2.0}
    return {"bytes": n * (24 + _es(c["g"]) + (2 if c["mirror"] else 0)), "flops": n * 18.0}  # p, m, v in and out


# ----------------------------------------------------------------- inputs


class _Rand:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0, dtype="f32"):
        t = torch.randn(shape, generator=self.g, device=DEV)
        t.mul_(std)
        return t.to(torch.bfloat16) if dtype == "bf16" else t

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device=DEV)

    def flags(self, p, *shape):
        return (self.uniform(*shape) < p).to(torch.uint8)


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _sizes(c):
    """Elements of each tensor of a policy of gated blocks: per layer the fused projection of the input, the two gates and
    the output's gate, the output projection, the three vectors of the norms and the residual scale and the rates; then the
    heads and their bias."""
    d, heads = c["width"], sum(HEADS) + 1
    return [4 * d * d, d * d, d, d, d, d] * c["layers"] + [heads * d, heads]


def prepare(case, seed):
    r = _Rand(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind in ("step", "fwd", "bwd"):
        _prepare_gatedrec(case, r, s)
    elif kind == "loss":
        _prepare_loss(case, r, s)
    else:
        _prepare_norm(case, r, s)
    return s


def _prepare_gatedrec(c, r, s):
    T, B, D = c.get("T", 1), c["B"], c["D"]
    dt = _type(c["dtype"])
    if c["fused"]:  # one projection's output: input, gates and output gate of a row beside each other
        s["x"], s["r"], s["i"], _ = r.normal(T, B, 4 * D, dtype=c["dtype"]).split(D, -1)
    else:
        s["x"], s["r"], s["i"] = (r.normal(T, B, D, dtype=c["dtype"]) for _ in range(3))
    # at half-open gates, half-lives from a few steps to a few thousand
    rate = torch.exp2(-2.0 - 9.0 * torch.arange(D, device=DEV) / max(1, D - 1))
    s["lam"] = torch.log(torch.expm1(rate * (2.0 / C)))
    s["reset"] = r.flags(0.01, T, B) if c["resets"] else None
    s["h0"] = r.normal(B, D)
    if c["kind"] == "step":
        s["x"], s["r"], s["i"] = s["x"][0], s["r"][0], s["i"][0]
        s["reset"] = None if s["reset"] is None else s["reset"][0]
        s["h"] = torch.empty(B, D, dtype=dt, device=DEV)
        return
    s["h"] = torch.empty(T, B, D, dtype=dt, device=DEV)
    s["hT"] = torch.empty_like(s["h0"])
    if c["kind"] == "bwd":
        s["dh"] = r.normal(T, B, D, dtype=c["dtype"])
        s["dhT"] = r.normal(B, D)
        if c["fused"]:
            s["dx"], s["dr"], s["di"], _ = torch.empty(T, B, 4 * D, dtype=dt, device=DEV).split(D, -1)
        else:
            s["dx"], s["dr"], s["di"] = (torch.empty(T, B, D, dtype=dt, device=DEV) for _ in range(3))
        s["dlam"], s["dh0"] = torch.empty(D, device=DEV), torch.empty_like(s["h0"])
    if own:
        from paper_1912_06680_amd import o5
        code, size = int(c["dtype"] == "bf16"), (T, B, D)
        need = max(o5.o5_gatedrec_fwd_workspace_bytes(code, *size), o5.o5_gatedrec_bwd_workspace_bytes(code, *size))
        s["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
        s["marks"] = torch.empty(o5.o5_gatedrec_marks_bytes(*size) // 4, device=DEV) if c["train"] else None
        if c["kind"] == "bwd":  # what the forward pass left
            _own_fwd(s)


def _offsets(heads):
    at = [0]
    for n in heads:
        at.append(at[-1] + n)
    return at


def _prepare_loss(c, r, s):
    N, heads = c["N"], _heads(c)
    A, K, at = sum(heads), len(heads), _offsets(_heads(c))
    cols = A + (1 if c["value"] else 0)
    s["z"] = r.normal(N, cols, std=2.0, dtype=c["dtype"])
    s["ref"] = None
    if c["ref"]:  # an earlier policy's, not far away
        s["ref"] = (s["z"][:, :A].float() + r.normal(N, A, std=0.3)).to(_type(c["dtype"]))
    avail = None
    if c["avail"]:
        avail = r.flags(0.8, N, A)
        empty = r.flags(0.02, N, K)  # now and then a head has no choice left
    act, logp = torch.empty(N, K, dtype=torch.int32, device=DEV), torch.zeros(N, device=DEV)
    for k in range(K):
        a, b = at[k], at[k + 1]
        z = s["z"][:, a:b].float()
        if avail is not None:
            avail[:, a:b] *= 1 - empty[:, k:k + 1]
            z = z.masked_fill(avail[:, a:b] == 0, -math.inf)
        noise = -torch.log(-torch.log(r.uniform(N, b - a).clamp(1e-7, 1.0 - 1e-7)))
        act[:, k] = torch.argmax(z + noise, -1)
        if avail is not None:
            open_ = avail[:, a:b].any(-1, keepdim=True)
            z = torch.where(open_, z, torch.zeros((), device=DEV))
            lp = torch.log_softmax(z, -1).gather(1, act[:, k:k + 1].long())
            logp += torch.where(open_, lp, torch.zeros((), device=DEV))[:, 0]
        else:
            logp += torch.log_softmax(z, -1).gather(1, act[:, k:k + 1].long())[:, 0]
    # the behaviour policy's ratio: some rows beyond the clip on either side, none within a hair of it
    lr = r.normal(N, std=0.15)
    for edge in (math.log(1.0 + CLIP_EPS), math.log(1.0 - CLIP_EPS)):
        lr = torch.where((lr - edge).abs() < 2e-3, torch.full_like(lr, 0.05), lr)
    s["act"], s["avail"], s["logp_old"] = act, avail, logp - lr
    s["adv"] = r.normal(N)
    s["ret"] = r.normal(N) if c["value"] else None
    s["weight"] = None
    if c["pad"]:  # a padded batch: the mean over the rows that count
        keep = 1.0 - r.flags(c["pad"], N).float()
        s["weight"] = keep / keep.sum().clamp(min=1.0)
    if own:
        from paper_1912_06680_amd import o5
        s["stats"], s["logp"], s["kl"] = torch.empty(STATS, device=DEV), torch.empty(N, device=DEV), torch.empty(N, device=DEV)
        s["dz"] = torch.empty_like(s["z"])
        size = o5.o5_ppo_logits_grad_workspace_bytes(int(c["dtype"] == "bf16"), N, heads)
        s["ws"] = torch.empty(max(16, size), dtype=torch.uint8, device=DEV)


def _rows(n):
    return (n + BLOCK - 1) // BLOCK


def _prepare_norm(c, r, s):
    sizes = _sizes(c)
    at, total = [], 0
    for n in sizes:
        at.append(total)
        total += _rows(n) * BLOCK
    flat = lambda dt: torch.zeros(total, dtype=dt, device=DEV)  # noqa: E731
    s["flat"] = {"p": flat(torch.float32), "g": flat(_type(c["g"])), "m": flat(torch.float32), "v": flat(torch.float32)}
    if c["mirror"]:
        s["flat"]["p16"] = flat(torch.bfloat16)
    s["views"] = {k: [t[a:a + n] for a, n in zip(at, sizes)] for k, t in s["flat"].items()}
    w = s["views"]
    for p, g, m, v in zip(w["p"], w["g"], w["m"], w["v"]):
        n = p.numel()
        p.copy_(r.normal(n, std=0.02))
        scale = torch.exp(r.normal(n))  # gradients of very different sizes, as of frequent and rare features
        g.copy_(r.normal(n, std=1e-3) * scale)
        m.copy_(r.normal(n, std=3e-4) * scale)
        v.copy_(scale.square() * 1e-6 * (0.5 + r.normal(n).abs()))
    # the gradients' root mean square is about 2.7e-3: their norm is some twice the largest allowed
    s["max_norm"] = 1.35e-3 * math.sqrt(sum(sizes))
    if own:
        from paper_1912_06680_amd import o5
        tensors = [o5.adamw_tensor(*t[:4], p_bf16=t[4]) for t in zip(w["p"], w["g"], w["m"], w["v"],
                                                                    w.get("p16", [None] * len(sizes)))]
        s["plan"] = torch.empty(o5.o5_adamw_plan_bytes(tensors), dtype=torch.uint8)
        o5.o5_adamw_plan(tensors, s["plan"])
        s["plan_dev"] = s["plan"].to(DEV)
        s["clip"] = torch.empty(4, device=DEV)
        s["ws"] = torch.empty(max(16, o5.o5_adamw_grad_norm_workspace_bytes(s["plan"])), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------- the plain forms


def _gates(s):
    """(sigmoid(r), sigmoid(i), x, log a, 1 - a, sqrt(1 - a^2)) in 32 bits."""
    x, r, i = (s[n].float() for n in "xri")
    g, o = 1.0 / (1.0 + torch.exp(-r)), 1.0 / (1.0 + torch.exp(-i))
    la = g * (-C * torch.log1p(torch.exp(s["lam"])))
    w = -torch.expm1(la)
    return g, o, x, la, w, torch.sqrt(w * (2.0 - w))


def _scan(a, b, first):
    """y_t = a_t y_{t-1} + b_t along dimension 0 with y_{-1} = first: step by step, or by doubling where there are many."""
    T = a.shape[0]
    if T <= 1024:
        y, out = first, torch.empty_like(b)
        for t in range(T):
            y = torch.addcmul(b[t], a[t], y, out=out[t])
        return out
    b[0] += a[0] * first  # (both are this pass's own)
    d = 1
    while d < T:
        b[d:] = torch.addcmul(b[d:], a[d:], b[:-d])
        a[d:] = a[d:] * a[:-d]
        d *= 2
    return b


def _carry(s, w):
    a = 1.0 - w
    if s["reset"] is not None:
        a = torch.where((s["reset"] != 0)[..., None], torch.zeros((), device=DEV), a)
    return a


def _plain_fwd(s):
    _, o, x, _, w, beta = _gates(s)
    h = _scan(_carry(s, w), beta * o * x, s["h0"])
    return {"h": h.to(s["x"].dtype), "hT": h[-1].clone()}


def _plain_step(s):
    _, o, x, _, w, beta = _gates(s)
    s["h0"].copy_(_carry(s, w) * s["h0"] + beta * o * x)
    return {"h": s["h0"].to(s["x"].dtype), "state": s["h0"]}


def _plain_bwd(s):
    dt = s["x"].dtype
    g, o, x, la, w, beta = _gates(s)
    a = _carry(s, w)
    h = _scan(a, beta * o * x, s["h0"])
    before = torch.cat([s["h0"][None], h[:-1]])
    # the gradient of the states runs the other way
    after = torch.cat([torch.ones_like(a[:1]), a[1:].flip(0)])
    G = _scan(after, s["dh"].float().flip(0), s["dhT"]).flip(0)
    keep = 1.0 - w
    part = torch.where(beta > 0, la / beta, torch.zeros((), device=DEV))
    e = G * (a * before * la - keep * keep * (o * x) * part)
    du = G * beta
    out = {"dx": (du * o).to(dt), "dr": (e * (1.0 - g)).to(dt), "di": (du * x * o * (1.0 - o)).to(dt)}
    sp = torch.log1p(torch.exp(s["lam"]))
    out["dlam"] = e.sum((0, 1)) / (sp * (1.0 + torch.exp(-s["lam"])))
    out["dh0"] = a[0] * G[0]
    return out


def _plain_loss(s):
    c = s["case"]
    N, heads, at = c["N"], _heads(c), _offsets(_heads(c))
    A, zero = at[-1], torch.zeros((), device=DEV)
    z = s["z"].float()
    weight = torch.full((N,), 1.0 / N, device=DEV) if s["weight"] is None else s["weight"]
    logp, ent, kl = (torch.zeros(N, device=DEV) for _ in range(3))
    kept = []
    for k, n in enumerate(heads):
        zk = z[:, at[k]:at[k + 1]]
        on = torch.ones(N, 1, dtype=torch.bool, device=DEV)
        see = None
        if s["avail"] is not None:
            see = s["avail"][:, at[k]:at[k + 1]] != 0
            on = see.any(-1, keepdim=True)
            zk = torch.where(see | ~on, zk, torch.full((), -math.inf, device=DEV))
        m = zk.amax(-1, keepdim=True)
        e = torch.exp(zk - m)
        sum_e = e.sum(-1, keepdim=True)
        p, lse = e / sum_e, m + torch.log(sum_e)
        lp = zk - lse
        plp = torch.where(p > 0, p * lp, zero)
        S = -plp.sum(-1, keepdim=True)
        a = s["act"][:, k:k + 1].long()
        logp += torch.where(on, lp.gather(1, a), zero)[:, 0]
        ent += torch.where(on, S, zero)[:, 0]
        far, D = None, None
        if s["ref"] is not None:
            y = s["ref"][:, at[k]:at[k + 1]].float()
            if see is not None:
                y = torch.where(see | ~on, y, torch.full((), -math.inf, device=DEV))
            my = y.amax(-1, keepdim=True)
            far = lp - (y - my - torch.log(torch.exp(y - my).sum(-1, keepdim=True)))
            far = torch.where(p > 0, far, zero)
            D = (p * far).sum(-1, keepdim=True)
            kl += torch.where(on, D, zero)[:, 0]
        kept.append((p, lp, S, far, D, a, on))
    ratio = torch.exp(logp - s["logp_old"])
    plain = ratio * s["adv"]
    cut = ratio.clamp(1.0 - CLIP_EPS, 1.0 + CLIP_EPS) * s["adv"]
    flows = torch.where(plain <= cut, -plain, zero) * weight
    dz = torch.zeros_like(z)
    for k, (p, lp, S, far, D, a, on) in enumerate(kept):
        d = -p * flows[:, None]
        d.scatter_add_(1, a, flows[:, None])
        d += torch.where(p > 0, p * (lp + S), zero) * (ENT * weight)[:, None]
        if far is not None:
            d += p * (far - D) * (KL * weight)[:, None]
        dz[:, at[k]:at[k + 1]] = torch.where(on, d, zero)
    err = torch.zeros(N, device=DEV)
    if s["ret"] is not None:
        err = z[:, A] - s["ret"]
        dz[:, A] = 2.0 * VF * weight * err
    lr = logp - s["logp_old"]
    rows = [-torch.minimum(plain, cut), err * err, ent, ((ratio - 1.0).abs() > CLIP_EPS).float(), (ratio - 1.0) - lr, ratio]
    pg, vf, en, share, approx, mean = [(weight * x).sum() for x in rows]
    far = (weight * kl).sum()
    total = pg + VF * vf - ENT * en + KL * far
    stats = torch.stack([total, pg, vf, en, share, approx, mean, torch.zeros((), device=DEV), far])
    on = weight != 0
    return {"stats": stats, "dz": dz.to(s["z"].dtype), "logp": torch.where(on, logp, zero), "kl": torch.where(on, kl, zero)}


def _plain_norm(s):
    total = torch.zeros((), dtype=torch.float64, device=DEV)
    for g in s["views"]["g"]:
        total = total + g.double().square().sum()
    norm = torch.sqrt(total)
    return torch.stack([norm, torch.clamp(s["max_norm"] / norm, max=1.0)]).float()


def _f32(x):
    return torch.tensor(x, dtype=torch.float32).item()


def _plain_clip(s):
    hp = HP
    clip = _plain_norm(s)
    b1, b2, lr = _f32(hp["beta1"]), _f32(hp["beta2"]), _f32(hp["lr"])
    c1, c2 = 1.0 / (1.0 - b1 ** hp["step"]), 1.0 / (1.0 - b2 ** hp["step"])
    f = s["flat"]  # (the gaps between tensors hold zeros and stay so)
    g = f["g"].float() * clip[1]
    f["v"].mul_(b2).addcmul_(g, g, value=1.0 - b2)
    f["m"].mul_(b1).add_(g, alpha=1.0 - b1)
    f["p"].sub_((f["m"] * c1) / (torch.sqrt(f["v"] * c2) + _f32(hp["eps"])) * lr)
    if "p16" in f:
        f["p16"].copy_(f["p"])
    return _clip_out(s, clip)


def _clip_out(s, clip):
    return {"clip": clip, **{k: s["flat"][k] for k in ("p", "m", "v", "p16") if k in s["flat"]}}


# ------------------------------------------------------------------- run


_PLAIN = {"fwd": _plain_fwd, "bwd": _plain_bwd, "step": _plain_step, "loss": _plain_loss, "norm": _plain_norm,
          "clip": _plain_clip}


def _own_fwd(s):
    from paper_1912_06680_amd import o5
    c = s["case"]
    o5.o5_gatedrec_fwd(int(c["dtype"] == "bf16"), c["T"], c["B"], c["D"], s["x"], s["x"].stride(1), s["r"], s["r"].stride(1),
                       s["i"], s["i"].stride(1), s["lam"], C, s["h0"], s["reset"], s["h"], c["D"], s["hT"], s["marks"], s["ws"])


def run(state):
    s = state
    c = s["case"]
    kind = c["kind"]
    if not own:
        return _PLAIN[kind](s)
    from paper_1912_06680_amd import o5
    dt = int(c["dtype"] == "bf16") if "dtype" in c else 0
    if kind == "step":
        o5.o5_gatedrec_step(dt, c["B"], c["D"], s["x"], s["x"].stride(0), s["r"], s["r"].stride(0), s["i"], s["i"].stride(0),
                            s["lam"], C, s["reset"], s["h0"], s["h"], c["D"])
        return {"h": s["h"], "state": s["h0"]}
    if kind == "fwd":
        _own_fwd(s)
        return {"h": s["h"], "hT": s["hT"]}
    if kind == "bwd":
        o5.o5_gatedrec_bwd(dt, c["T"], c["B"], c["D"], s["x"], s["x"].stride(1), s["r"], s["r"].stride(1), s["i"],
                           s["i"].stride(1), s["lam"], C, s["marks"], s["reset"], s["dh"], c["D"], s["dhT"],
                           s["dx"], s["dx"].stride(1), s["dr"], s["dr"].stride(1), s["di"], s["di"].stride(1), s["dlam"],
                           s["dh0"], s["ws"])
        return {k: s[k] for k in ("dx", "dr", "di", "dlam", "dh0")}
    if kind == "loss":
        o5.o5_ppo_logits_grad(dt, c["N"], _heads(c), s["z"], s["z"].stride(0), s["ref"],
                              0 if s["ref"] is None else s["ref"].stride(0), s["act"], s["logp_old"], s["adv"], s["ret"],
                              s["weight"], None, s["avail"], CLIP_EPS, VF, ENT, KL, s["stats"], s["logp"], s["kl"], s["dz"],
                              s["dz"].stride(0), s["ws"])
        return {k: s[k] for k in ("stats", "dz", "logp", "kl")}
    o5.o5_adamw_grad_norm(s["plan"], s["plan_dev"], s["max_norm"], s["clip"], s["ws"])
    if kind == "norm":
        return s["clip"][:2]
    o5.o5_adamw_step_clipped(s["plan"], s["plan_dev"], HP["lr"], HP["beta1"], HP["beta2"], HP["eps"], HP["clip_k"], s["clip"],
                             HP["seed"], HP["step"])
    return _clip_out(s, s["clip"][:2])


# ----------------------------------------------------------------- exact


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("step", "fwd", "bwd"):
        return _exact_gatedrec(case, s)
    if kind == "loss":
        return _exact_loss(case, s)
    return _exact_norm(case, s)


def _exact_gatedrec(c, s):
    """The recurrence step by step, its gradient by the chain rule in each step."""
    T, B, D = c.get("T", 1), c["B"], c["D"]
    row = lambda n, t: (s[n][t] if "T" in c else s[n]).double()  # noqa: E731
    rate = C * torch.nn.functional.softplus(s["lam"].double())
    cut = torch.zeros(T, B, 1, device=DEV) if s["reset"] is None else (s["reset"].view(T, B, 1) != 0).float()
    wide = c["dtype"] == "f32"

    def gates(t):
        g, o = torch.sigmoid(row("r", t)), torch.sigmoid(row("i", t))
        la = -rate * g
        return g, o, row("x", t), la, torch.exp(la), torch.sqrt(-torch.expm1(2.0 * la))

    h, hs = s["h0"].double().clone(), []
    keep = (lambda x: x) if wide or c["kind"] == "bwd" else (lambda x: x.float())
    for t in range(T):
        before = h * (1.0 - cut[t].double())
        if c["kind"] == "bwd":
            hs.append(before)
        g, o, x, la, a, beta = gates(t)
        h = a * before + beta * o * x
        if c["kind"] != "bwd":
            hs.append(keep(h))
    if c["kind"] == "step":
        return {"h": hs[0], "state": h}
    if c["kind"] == "fwd":
        return {"h": torch.stack(hs), "hT": h}
    G, dlam = s["dhT"].double().clone(), torch.zeros(D, dtype=torch.float64, device=DEV)
    dx, dr, di = ([None] * T for _ in range(3))
    out = torch.float64 if wide else torch.float32
    for t in reversed(range(T)):
        G = G + s["dh"][t].double()
        g, o, x, la, a, beta = gates(t)
        dla = G * (a * hs[t] - o * x * a * a / beta)
        dr[t] = (dla * -rate * g * (1.0 - g)).to(out)
        dlam += (dla * -C * g).sum(0)
        dx[t], di[t] = (G * beta * o).to(out), (G * beta * x * o * (1.0 - o)).to(out)
        hs[t] = None
        G = a * G * (1.0 - cut[t].double())
    return {"dx": torch.stack(dx), "dr": torch.stack(dr), "di": torch.stack(di),
            "dlam": dlam * torch.sigmoid(s["lam"].double()), "dh0": G}


def _exact_loss(c, s):
    """The loss of its definition in 64 bits, a few rows at a time, its gradient by automatic differentiation."""
    N, heads, at = c["N"], _heads(c), _offsets(_heads(c))
    A = at[-1]
    weight = torch.full((N,), 1.0 / N, dtype=torch.float64, device=DEV) if s["weight"] is None else s["weight"].double()
    part = max(1, (1 << 27) // (A + 1))
    sums, dz, logps, kls = torch.zeros(STATS, dtype=torch.float64, device=DEV), [], [], []
    for n0 in range(0, N, part):
        n1 = min(N, n0 + part)
        w = weight[n0:n1]
        leaf = s["z"][n0:n1].double().requires_grad_()
        logp, ent, kl = (torch.zeros(n1 - n0, dtype=torch.float64, device=DEV) for _ in range(3))
        for k in range(len(heads)):
            cols = slice(at[k], at[k + 1])
            see = torch.ones(n1 - n0, heads[k], dtype=torch.bool, device=DEV)
            if s["avail"] is not None:
                see = s["avail"][n0:n1, cols] != 0
            some = see.any(-1)
            low = (some[:, None] & ~see).double() * -1e300
            lp = torch.log_softmax(torch.where(see, leaf[:, cols], torch.zeros_like(low)) + low, -1)
            p = lp.exp()
            seen = torch.where(see, lp, torch.zeros_like(lp))
            logp = logp + torch.where(some, lp.gather(1, s["act"][n0:n1, k:k + 1].long())[:, 0], torch.zeros_like(logp))
            ent = ent - torch.where(some, (p * seen).sum(-1), torch.zeros_like(ent))
            if s["ref"] is not None:
                y = torch.where(see, s["ref"][n0:n1, cols].double(), torch.zeros_like(low))
                lq = torch.log_softmax(y + low, -1)
                kl = kl + torch.where(some, (p * (seen - torch.where(see, lq, torch.zeros_like(lq)))).sum(-1), torch.zeros_like(kl))
        lr = logp - s["logp_old"][n0:n1].double()
        ratio, adv = lr.exp(), s["adv"][n0:n1].double()
        pg = -torch.minimum(ratio * adv, ratio.clamp(1.0 - _f32(CLIP_EPS), 1.0 + _f32(CLIP_EPS)) * adv)
        err = leaf[:, A] - s["ret"][n0:n1].double() if s["ret"] is not None else torch.zeros_like(logp)
        total = pg + VF * err ** 2 - _f32(ENT) * ent + _f32(KL) * kl
        dz.append(torch.autograd.grad((w * total).sum(), leaf)[0].to(torch.float32 if c["dtype"] == "bf16" else torch.float64))
        rows = (total, pg, err ** 2, ent, ((ratio - 1.0).abs() > CLIP_EPS).double(), ratio - 1.0 - lr, ratio,
                torch.zeros_like(kl), kl)
        sums += torch.stack([(w * x.detach()).sum() for x in rows])
        on = (w != 0).double()
        logps.append(logp.detach() * on)
        kls.append(kl.detach() * on)
    return {"stats": sums, "dz": torch.cat(dz), "logp": torch.cat(logps), "kl": torch.cat(kls)}


def _exact_norm(c, s):
    square = sum(float((g.double() ** 2).sum()) for g in s["views"]["g"])
    norm = math.sqrt(square)
    factor = min(1.0, s["max_norm"] / norm)
    clip = torch.tensor([norm, factor], dtype=torch.float64, device=DEV)
    if c["kind"] == "norm":
        return clip
    out = {"clip": clip}
    b1, b2, lr, eps = (_f32(HP[k]) for k in ("beta1", "beta2", "lr", "eps"))
    f = {k: t.double() for k, t in s["flat"].items()}
    g = f["g"] * factor
    out["v"] = b2 * f["v"] + (1.0 - b2) * g ** 2
    out["m"] = b1 * f["m"] + (1.0 - b1) * g
    out["p"] = f["p"] - lr * (out["m"] / (1.0 - b1 ** HP["step"])) / ((out["v"] / (1.0 - b2 ** HP["step"])).sqrt() + eps)
    if c["mirror"]:
        out["p16"] = out["p"]
    return {k: out[k] for k in ("clip", "p", "m", "v", "p16") if k in out}
