"""The operators of a recurrent core that is parallel over time, as measurable cases.

Three operators, reached through the ``o5_*`` bindings:

linattn   linear attention with a decay for each head: over T steps (forward
          and backward) and for single tokens on a state kept in place
resnorm   RMS norms before and after a block, fused with the block's gate and
          residual scale (forward and backward)
adamw     AdamW over many tensors at once, its moments in 32 bits or in 8

Kinds: ``fwd``, ``bwd`` and ``step`` (linattn), ``norm_fwd`` and ``norm_bwd``
(resnorm), ``adamw``.  With ``own`` false ``run`` computes the same from
elementary torch operations in 32 bits; ``exact`` computes it in 64 bits from
the recurrences.
"""
import functools
import math

import torch

own = False

DEV = "cuda"
CHUNK = 64     # steps per chunk of the plain chunked form, at most
BLOCK = 256    # elements that share an exponent in the 8-bit moments
EPS = 1e-6     # of the norms
HEADS = 75     # rows of the policy and value heads of the synthetic configurations

HP = {"lr": 5e-5, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "clip_k": 5.0, "wd": 0.01, "seed": 7, "step": 20}


def listed():
    return [
        # one environment's next action: a single token, latency
        {"name": "step_1", "kind": "step", "dtype": "bf16", "B": 1, "nh": 8, "nkv": 8, "dk": 64, "dv": 64, "resets": False},
        # rollout inference for 4,096 environments at width 1024: bound by the states
        {"name": "step_4096", "kind": "step", "dtype": "bf16", "B": 4096, "nh": 8, "nkv": 8, "dk": 128, "dv": 128, "resets": True},
        # whole 256-step segments of the benchmark's batch at width 4096
        {"name": "fwd_segments", "kind": "fwd", "dtype": "bf16", "T": 256, "B": 128, "nh": 32, "nkv": 32, "dk": 128, "dv": 128,
         "resets": True, "fused": True},
        # one long history, few heads that share their states' keys and values: the work has to be split over time
        {"name": "fwd_long", "kind": "fwd", "dtype": "bf16", "T": 10007, "B": 1, "nh": 16, "nkv": 4, "dk": 64, "dv": 128,
         "resets": False, "fused": True},
        # debugging in full precision, with sizes that are no multiple of a tile
        {"name": "fwd_ragged_f32", "kind": "fwd", "dtype": "f32", "T": 77, "B": 24, "nh": 6, "nkv": 3, "dk": 40, "dv": 72,
         "resets": True, "fused": False},
        # training on whole segments at width 2048
        {"name": "bwd_segments", "kind": "bwd", "dtype": "bf16", "T": 256, "B": 64, "nh": 16, "nkv": 16, "dk": 128, "dv": 128,
         "resets": True, "fused": True},
        # training on 16-step samples at width 1024, fp32
        {"name": "bwd_samples_f32", "kind": "bwd", "dtype": "f32", "T": 16, "B": 256, "nh": 16, "nkv": 8, "dk": 64, "dv": 64,
         "resets": True, "fused": False},
        # the norms around a block for a few environments' next tokens: latency
        {"name": "norm_fwd_60", "kind": "norm_fwd", "xt": "bf16", "dtype": "bf16", "N": 60, "D": 1024, "form": "both", "gate": True},
        # the benchmark's 32,768 rows at width 4096, training
        {"name": "norm_bwd_full", "kind": "norm_bwd", "xt": "bf16", "dtype": "bf16", "N": 32768, "D": 4096, "form": "both",
         "gate": True},
        # a residual stream in fp32, an odd number of rows and a width that is no power of two
        {"name": "norm_bwd_odd", "kind": "norm_bwd", "xt": "f32", "dtype": "bf16", "N": 5003, "D": 1000, "form": "both",
         "gate": False},
        # every tensor of a small policy, moments in 32 bits
        {"name": "adamw_small", "kind": "adamw", "bits": 32, "g": "f32", "width": 512, "layers": 4, "mirror": True},
        # every tensor of a 4096-wide policy, moments in 8 bits, and their values as a checkpoint takes them
        {"name": "adamw_full_8bit", "kind": "adamw", "bits": 8, "g": "bf16", "width": 4096, "layers": 2, "mirror": True},
    ]


# ------------------------------------------------------------------ draws


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_any(rng):
    kind = rng.choice(("step", "fwd", "fwd", "bwd", "bwd", "norm_fwd", "norm_bwd", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("step", "fwd", "bwd"):
        group = rng.choice((1, 1, 2, 4))
        nkv = _log_int(rng, 1, 32)
        c = {"kind": kind, "dtype": dtype, "B": _log_int(rng, 1, 4096 if kind == "step" else 256), "nh": nkv * group, "nkv": nkv,
             "dk": rng.choice((64, 128, 8 * rng.randint(2, 16))), "dv": rng.choice((64, 128, 8 * rng.randint(2, 16))),
             "resets": rng.random() < 0.6}
        if kind != "step":
            c["T"] = _log_int(rng, 1, 12000)
            c["fused"] = rng.random() < 0.5
        return c
    if kind in ("norm_fwd", "norm_bwd"):
        form = rng.choice(("both", "both", "pre", "post"))
        return {"kind": kind, "xt": "f32" if dtype == "f32" else rng.choice(("f32", "bf16")), "dtype": dtype,
                "N": _log_int(rng, 1, 40000), "D": 8 * _log_int(rng, 8, 1024), "form": form,
                "gate": form != "pre" and rng.random() < 0.6}
    return {"kind": "adamw", "bits": rng.choice((8, 32)), "g": rng.choice(("f32", "bf16")), "width": 8 * _log_int(rng, 8, 512),
            "layers": rng.randint(1, 8), "mirror": rng.random() < 0.7}


def _cost(c):
    """A rough time in microseconds, to keep draws below the largest listed case."""
    w = work(c)
    return w["bytes"] / 3e6 + w["flops"] / 50e6


def draw(rng):
    most = {kind: max(_cost(c) for c in listed() if c["kind"] in kinds) for kinds in _FAMILIES for kind in kinds}
    while True:
        c = _draw_any(rng)
        if _cost(c) <= most[c["kind"]] and 3072 not in c.values():  # (a size that no configuration here has)
            return c


_FAMILIES = (("step",), ("fwd", "bwd"), ("norm_fwd", "norm_bwd"), ("adamw",))


# ------------------------------------------------------------------- work


def _es(t):
    return 2 if t == "bf16" else 4


def work(case):
    c = case
    k = c["kind"]
    if k in ("step", "fwd", "bwd"):
        e, rows = _es(c["dtype"]), c["B"] * c.get("T", 1)
        qb, kb, vb, ob = (rows * n * e for n in (c["nh"] * c["dk"], c["nkv"] * c["dk"], c["nkv"] * c["dv"], c["nh"] * c["dv"]))
        states = c["B"] * c["nkv"] * c["dk"] * c["dv"] * 4
        resets = rows if c["resets"] else 0
        products = 2.0 * rows * c["dk"] * c["dv"]  # one read or one update of every state
        if k == "bwd":  # in: q, k, v, do, S0, dST; out: dq, dk, dv, dS0; S and G each updated and read, dk, dv read G
            return {"bytes": 2 * (qb + kb + vb) + ob + 3 * states + resets, "flops": products * (2 * c["nh"] + 3 * c["nkv"])}
        return {"bytes": qb + kb + vb + ob + 2 * states + resets, "flops": products * (c["nh"] + c["nkv"])}
    if k in ("norm_fwd", "norm_bwd"):
        n, x, e = c["N"] * c["D"], _es(c["xt"]), _es(c["dtype"])
        post, pre = c["form"] != "pre", c["form"] != "post"
        gate = e if c["gate"] else 0
        if k == "norm_fwd":  # in: x, u, gate; out: x', n
            per = x + (e + gate + x if post else 0) + (e if pre else 0)
            return {"bytes": n * per, "flops": n * 16.0}
        per = 2 * x + (x + e if pre else 0) + (2 * e + 2 * gate if post else 0)  # in: dx', x', dn, u, gate; out: dx, du, dgate
        return {"bytes": n * per, "flops": n * 32.0}
    n = sum(_sizes(c))
    per = 8 + _es(c["g"]) + (2 if c["mirror"] else 0) + (16 if c["bits"] == 32 else 4 + 4 / BLOCK + 2 + 2 / BLOCK + 8)
    return {"bytes": n * per, "flops": n * 16.0}


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

    def flags(self, p, *shape):
        return (torch.rand(shape, generator=self.g, device=DEV) < p).to(torch.uint8)


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _sizes(c):
    """Elements of each tensor of a policy: per layer the fused query, key, value and gate projection, the output
    projection and the three vectors of the norms and the residual scale; then the heads and their bias."""
    d = c["width"]
    return [4 * d * d, d * d, d, d, d] * c["layers"] + [HEADS * d, HEADS]


def _rows(n):
    return (n + BLOCK - 1) // BLOCK


def prepare(case, seed):
    r = _Rand(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind in ("step", "fwd", "bwd"):
        _prepare_linattn(case, r, s)
    elif kind == "adamw":
        _prepare_adamw(case, r, s)
    else:
        _prepare_norm(case, r, s)
    return s


def _prepare_linattn(c, r, s):
    T, B, nh, nkv, dk, dv = c.get("T", 1), c["B"], c["nh"], c["nkv"], c["dk"], c["dv"]
    dt = _type(c["dtype"])
    widths = (nh * dk, nkv * dk, nkv * dv)
    if c.get("fused"):  # one projection's output: q, k and v of a row beside each other
        x = r.normal(T, B, sum(widths), dtype=c["dtype"])
        s["q"], s["k"], s["v"] = x.split(widths, -1)
        grads = torch.empty_like(x).split(widths, -1) if c["kind"] == "bwd" else None
    else:
        s["q"], s["k"], s["v"] = (r.normal(T, B, w, dtype=c["dtype"]) for w in widths)
        grads = [torch.empty_like(s[n]) for n in "qkv"] if c["kind"] == "bwd" else None
    # half-lives from about 20 steps to a few thousand, a decay for each state head
    s["decay"] = 1.0 - torch.exp2(-5.0 - 7.0 * torch.arange(nkv, device=DEV) / max(1, nkv - 1))
    s["scale"] = dk ** -0.5
    s["reset"] = r.flags(0.01, T, B) if c["resets"] else None
    s["S"] = r.normal(B, nkv, dk, dv)
    if c["kind"] == "step":
        s["o"] = torch.empty(B, nh * dv, dtype=dt, device=DEV)
        s["q"], s["k"], s["v"] = s["q"][0], s["k"][0], s["v"][0]
        s["reset"] = None if s["reset"] is None else s["reset"][0]
        return
    if c["kind"] == "bwd":
        s["do"] = r.normal(T, B, nh * dv, dtype=c["dtype"])
        s["dST"] = r.normal(B, nkv, dk, dv)
        s["dq"], s["dk"], s["dv"] = grads
        s["dS"] = torch.empty_like(s["S"])
    else:
        s["o"] = torch.empty(T, B, nh * dv, dtype=dt, device=DEV)
        s["ST"] = torch.empty_like(s["S"])
    if own:
        from paper_1912_06680_amd import o5
        size = o5.o5_linattn_bwd_workspace_bytes if c["kind"] == "bwd" else o5.o5_linattn_fwd_workspace_bytes
        s["ws"] = torch.empty(max(16, size(int(c["dtype"] == "bf16"), T, B, nh, nkv, dk, dv)), dtype=torch.uint8, device=DEV)


def _prepare_norm(c, r, s):
    N, D = c["N"], c["D"]
    post, pre = c["form"] != "pre", c["form"] != "post"
    x, dt = _type(c["xt"]), _type(c["dtype"])
    s["x"] = r.normal(N, D, dtype=c["xt"])
    s["u"] = r.normal(N, D, std=3.0, dtype=c["dtype"]) if post else None
    s["gate"] = r.normal(N, D, dtype=c["dtype"]) if c["gate"] else None
    s["w_post"] = 1.0 + r.normal(D, std=0.1) if post else None
    s["rho"] = 0.5 + r.normal(D, std=0.1) if post else None
    s["w_pre"] = 1.0 + r.normal(D, std=0.1) if pre else None
    row = lambda on: torch.empty(N, device=DEV) if on else None  # noqa: E731
    s["r_post"], s["r_pre"] = row(post), row(pre)
    if c["kind"] == "norm_fwd":
        s["xo"] = torch.empty(N, D, dtype=x, device=DEV) if post else None
        s["n"] = torch.empty(N, D, dtype=dt, device=DEV) if pre else None
        return
    # the backward pass has what the forward pass left: x' in x's place and the rows' inverse norms
    if post:
        s["r_post"] = torch.rsqrt(s["u"].float().square().mean(-1) + EPS)
    if pre:
        s["r_pre"] = torch.rsqrt(s["x"].float().square().mean(-1) + EPS)
    s["dxo"] = r.normal(N, D, dtype=c["xt"])
    s["dn"] = r.normal(N, D, dtype=c["dtype"]) if pre else None
    s["dx"] = torch.empty_like(s["x"])
    s["du"] = torch.empty_like(s["u"]) if post else None
    s["dgate"] = torch.empty_like(s["gate"]) if c["gate"] else None
    s["dw_post"], s["drho"], s["dw_pre"] = (torch.empty(D, device=DEV) if on else None for on in (post, post, pre))
    if own:
        from paper_1912_06680_amd import o5
        size = o5.o5_resnorm_bwd_workspace_bytes(int(c["xt"] == "bf16"), int(c["dtype"] == "bf16"), N, D)
        s["ws"] = torch.empty(max(16, size), dtype=torch.uint8, device=DEV)


def _prepare_adamw(c, r, s):
    sizes = _sizes(c)
    at, total = [], 0
    for n in sizes:  # every tensor starts at a whole block of one flat buffer
        at.append(total)
        total += _rows(n) * BLOCK
    flat = lambda dt: torch.zeros(total, dtype=dt, device=DEV)  # noqa: E731
    views = lambda t: [t[a:a + n] for a, n in zip(at, sizes)]  # noqa: E731
    s["flat"] = {"p": flat(torch.float32), "g": flat(_type(c["g"]))}
    m, v = flat(torch.float32), flat(torch.float32)
    for p, g, mi, vi in zip(views(s["flat"]["p"]), views(s["flat"]["g"]), views(m), views(v)):
        n = p.numel()
        p.copy_(r.normal(n, std=0.02))
        scale = torch.exp(r.normal(n))  # gradients of very different sizes, as of frequent and rare features
        g.copy_(r.normal(n, std=1e-3) * scale)
        mi.copy_(r.normal(n, std=3e-4) * scale)
        vi.copy_(scale.square() * 1e-6 * (0.5 + r.normal(n).abs()))
    if c["bits"] == 8:
        mb, vb = m.view(-1, BLOCK), v.view(-1, BLOCK)
        half = torch.full_like(mb, 0.5)
        s["flat"]["mq"], s["flat"]["me"] = _to_8(mb, half, 13, True)
        s["flat"]["vq"], s["flat"]["ve"] = _to_8(vb, half, 29, False)
        s["flat"]["m"], s["flat"]["v"] = flat(torch.float32), flat(torch.float32)
    else:
        s["flat"]["m"], s["flat"]["v"] = m, v
    if c["mirror"]:
        s["flat"]["p16"] = flat(torch.bfloat16)
    s["views"] = {k: views(t.view(-1)) for k, t in s["flat"].items() if k not in ("me", "ve")}
    if c["bits"] == 8:
        for k in ("me", "ve"):
            s["views"][k] = [s["flat"][k][a // BLOCK:a // BLOCK + _rows(n)] for a, n in zip(at, sizes)]
    # decay on matrices alone
    s["wd"] = [HP["wd"] if n > HEADS and n != c["width"] else 0.0 for n in sizes]
    if own:
        from paper_1912_06680_amd import o5
        w = s["views"]
        mom = ("mq", "vq") if c["bits"] == 8 else ("m", "v")
        none = [None] * len(sizes)
        tensors = [o5.adamw_tensor(p, g, a, b, m_exp=me, v_exp=ve, p_bf16=p16, weight_decay=wd)
                   for p, g, a, b, me, ve, p16, wd in zip(w["p"], w["g"], w[mom[0]], w[mom[1]], w.get("me", none),
                                                          w.get("ve", none), w.get("p16", none), s["wd"])]
        s["plan"] = torch.empty(o5.o5_adamw_plan_bytes(tensors), dtype=torch.uint8)
        o5.o5_adamw_plan(tensors, s["plan"])
        s["plan_dev"] = s["plan"].to(DEV)


# ------------------------------------------------------- the plain forms


def _heads(x, n):
    """[T, B, n d] -> [B, n, T, d] in 32 bits."""
    T, B, w = x.shape
    return x.float().view(T, B, n, w // n).permute(1, 2, 0, 3)


def _flat(x, dt):
    """[B, n, T, d] -> [T, B, n d]."""
    B, n, T, d = x.shape
    return x.permute(2, 0, 1, 3).reshape(T, B, n * d).to(dt)


def _chunked(q, k, v, decay, S, episode, before, late):
    """out_i = decay^(i + late) q_i S + sum over j <= i of the same episode of decay^(i - j) (q_i . k_j) v_j, and the state
    after the last step; q, k, v [B, n, T, .], S [B, n, ., .].  `episode` [B, T] numbers the episodes and `before` [B] is
    the one that S belongs to; late = 1 where S decays once before the first step reads it."""
    B, n, T, dk = q.shape
    dv = v.shape[-1]
    C = min(CHUNK, T)
    nc = (T + C - 1) // C
    pad = nc * C - T
    if pad:
        q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, pad)) for x in (q, k, v))
        episode = torch.cat([episode, episode[:, -1:].expand(B, pad)], 1)
    q, k, v = (x.reshape(B, n, nc, C, -1) for x in (q, k, v))
    ep = episode.view(B, 1, nc, C)
    log = torch.log2(decay).view(1, n, 1, 1)
    i = torch.arange(C, device=DEV, dtype=torch.float32)
    gap = (i[:, None] - i[None, :]).clamp(min=0)
    see = (i[:, None] >= i[None, :]) & (ep[..., :, None] == ep[..., None, :])
    score = torch.matmul(q, k.transpose(-1, -2).contiguous())
    score = torch.where(see, score * torch.exp2(log[..., None] * gap), torch.zeros((), device=DEV))
    # what each chunk adds to the state at its own end
    length = torch.full((nc, 1), float(C), device=DEV)
    length[-1] = C - pad
    left = length - 1 - i if late else length - i
    last = ep[..., -1:]
    w = torch.where(ep == last, torch.exp2(log * left.clamp(min=0).view(1, 1, nc, C)), torch.zeros((), device=DEV))
    add = torch.matmul((k * w[..., None]).transpose(-1, -2).contiguous(), v)
    # the state at each chunk's start and after the last: S and the earlier chunks' parts, decayed
    starts = torch.cat([torch.zeros(1, device=DEV), torch.cumsum(length.view(-1), 0)])
    ends = torch.cat([before.view(B, 1, 1).to(ep.dtype), last.view(B, nc, 1)], 1).view(B, nc + 1)
    c, d = torch.arange(nc + 1, device=DEV)[:, None], torch.arange(nc + 1, device=DEV)[None, :]
    far = (starts[:, None] - starts[None, :]).clamp(min=0)
    keep = (d <= c) & (ends[:, :, None] == ends[:, None, :])
    mix = torch.where(keep[:, None], torch.exp2(log * far), torch.zeros((), device=DEV))
    parts = torch.cat([S[:, :, None], add], 2).view(B, n, nc + 1, -1)
    states = torch.matmul(mix, parts).view(B, n, nc + 1, dk, dv)
    first = ends[:, :-1].reshape(B, 1, nc, 1)
    lead = torch.where(ep == first, torch.exp2(log * (i + late)), torch.zeros((), device=DEV))
    out = torch.matmul(score, v) + torch.matmul(q, states[:, :, :-1]) * lead[..., None]
    return out.view(B, n, nc * C, dv)[:, :, :T], states[:, :, -1]


def _episodes(s, T, B):
    """Counts of the resets up to each step, [B, T]."""
    if s["reset"] is None:
        return torch.zeros(B, T, device=DEV)
    return torch.cumsum((s["reset"] != 0).float().t(), 1)


def _per_query(x, group):
    return x if group == 1 else x.repeat_interleave(group, 1)


def _sum_group(x, group):
    B, n = x.shape[:2]
    return x if group == 1 else x.view(B, n // group, group, *x.shape[2:]).sum(2)


def _plain_fwd(s):
    c = s["case"]
    T, B, g = c["T"], c["B"], c["nh"] // c["nkv"]
    ep = _episodes(s, T, B)
    q, k, v = _heads(s["q"], c["nh"]) * s["scale"], _per_query(_heads(s["k"], c["nkv"]), g), _per_query(_heads(s["v"], c["nkv"]), g)
    o, ST = _chunked(q, k, v, s["decay"].repeat_interleave(g), _per_query(s["S"], g), ep, torch.zeros(B, device=DEV), 1)
    return {"o": _flat(o, s["q"].dtype), "ST": ST[:, ::g].contiguous()}


def _plain_bwd(s):
    c = s["case"]
    T, B, g, dt = c["T"], c["B"], c["nh"] // c["nkv"], s["q"].dtype
    ep = _episodes(s, T, B)
    decay = s["decay"].repeat_interleave(g)
    q, do = _heads(s["q"], c["nh"]) * s["scale"], _heads(s["do"], c["nh"])
    k, v = _per_query(_heads(s["k"], c["nkv"]), g), _per_query(_heads(s["v"], c["nkv"]), g)
    St = _per_query(s["S"], g).transpose(-1, -2).contiguous()
    dq, _ = _chunked(do, v, k, decay, St, ep, torch.zeros(B, device=DEV), 1)
    # the states' gradient runs the other way; a group's first query carries the one that arrives at the end
    qr, kr, vr, dor, epr = q.flip(2), k.flip(2), v.flip(2), do.flip(2), ep.flip(1)
    G = _per_query(s["dST"], g) * (torch.arange(c["nh"], device=DEV) % g == 0).view(1, -1, 1, 1)
    dv, dS = _chunked(kr, qr, dor, decay, G, epr, ep[:, -1], 0)
    dk, _ = _chunked(vr, dor, qr, decay, G.transpose(-1, -2).contiguous(), epr, ep[:, -1], 0)
    dS = torch.where((ep[:, 0] == 0).view(B, 1, 1, 1), _sum_group(dS, g), torch.zeros((), device=DEV))
    return {"dq": _flat(dq * s["scale"], dt), "dk": _flat(_sum_group(dk.flip(2), g), dt),
            "dv": _flat(_sum_group(dv.flip(2), g), dt), "dS0": dS}


def _plain_step(s):
    c = s["case"]
    B, nkv, g = c["B"], c["nkv"], c["nh"] // c["nkv"]
    k, v = s["k"].float().view(B, nkv, -1, 1), s["v"].float().view(B, nkv, 1, -1)
    S = s["S"] * s["decay"].view(1, nkv, 1, 1)
    if s["reset"] is not None:
        S = torch.where((s["reset"] != 0).view(B, 1, 1, 1), torch.zeros((), device=DEV), S)
    s["S"].copy_(S + k * v)
    o = torch.matmul(s["q"].float().view(B, nkv, g, -1) * s["scale"], s["S"])
    return {"o": o.view(B, -1).to(s["q"].dtype), "S": s["S"]}


def _plain_norm_fwd(s):
    out, x = {}, s["x"].float()
    if s["u"] is not None:
        u = s["u"].float()
        r = torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS)
        y = u * r * s["w_post"] * s["rho"]
        if s["gate"] is not None:
            y = y / (1.0 + torch.exp(-s["gate"].float()))
        x = x + y
        out["xo"], out["r_post"] = x.to(s["x"].dtype), r[:, 0]
    if s["w_pre"] is not None:
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        out["n"], out["r_pre"] = (x * r * s["w_pre"]).to(_type(s["case"]["dtype"])), r[:, 0]
    return out


def _plain_norm_bwd(s):
    out, d = {}, s["dxo"].float()
    if s["w_pre"] is not None:
        x, r, dn = s["x"].float(), s["r_pre"][:, None], s["dn"].float()
        a = dn * s["w_pre"]
        d = d + r * (a - x * (r * r) * (a * x).mean(-1, keepdim=True))
        out["dw_pre"] = (dn * x * r).sum(0)
    out["dx"] = d.to(s["x"].dtype)
    if s["u"] is not None:
        u, r = s["u"].float(), s["r_post"][:, None]
        y, t = u * r, d
        if s["gate"] is not None:
            sig = 1.0 / (1.0 + torch.exp(-s["gate"].float()))
            out["dgate"] = (d * y * (s["w_post"] * s["rho"]) * sig * (1.0 - sig)).to(s["gate"].dtype)
            t = d * sig
        ty = t * y
        out["drho"], out["dw_post"] = (ty * s["w_post"]).sum(0), (ty * s["rho"]).sum(0)
        a = t * (s["w_post"] * s["rho"])
        out["du"] = (r * (a - y * (a * y).mean(-1, keepdim=True))).to(s["u"].dtype)
    return out


def _pow2(e):
    """2^e of whole numbers e in [-126, 127], exactly."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _exponent(x):
    """floor(log2 x) of x >= 0 (-127 where x is subnormal or zero)."""
    return (x.view(torch.int32) >> 23) - 127


def _to_8(x, up, low, signed):
    """Codes and shared exponents of the rows of x [rows, BLOCK]: 3 bits of mantissa, the exponents from `low` binades below
    the row's largest value's up to one above it, rounded up with the chance `up` compares to (0.5: to nearest)."""
    mag = x.abs()
    a = _exponent(mag.amax(-1, keepdim=True)).clamp(-90, 126)
    y = mag * _pow2(-a)
    t = _exponent(y).clamp(min=-low)
    code = (t + low) * 8 + torch.floor(y * _pow2(3 - t) + up).to(torch.int32)
    code = code.clamp(max=126 if signed else 254)
    if signed:
        code = torch.where((x < 0) & (code > 0), code + 128, code)
    else:
        code = torch.where(x > 0, code.clamp(min=1), code)
    return code.to(torch.uint8), (a[:, 0] + 127).to(torch.uint8)


def _from_8(q, e, low, signed):
    code = q.to(torch.int32)
    mag = code & 127 if signed else code
    field = mag >> 3
    mant = (mag & 7) + 8 * (field > 0).to(torch.int32)
    x = mant.float() * _pow2(e.to(torch.int32)[:, None] - 127 - low - 3 + field.clamp(min=1) - 1)
    return torch.where(code >= 128, -x, x) if signed else x


def _mulhilo(a, b):
    p = a * b
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _noise(n, step, tensor, seed):
    """Two random numbers of 16 bits in [0, 1) for each of n elements (a whole number of blocks): Philox4x32-7 (Salmon et
    al., SC'11) at the counter (i div 4, 0, step, tensor) and the key seed; element i takes word i mod 4, low and high half."""
    c0 = torch.arange(n // 4, device=DEV)
    c1, c2, c3 = torch.zeros_like(c0), torch.full_like(c0, step), torch.full_like(c0, tensor)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    words = functools.reduce(lambda x, _: _philox_round(*x), range(7), (c0, c1, c2, c3, k0, k1))[:4]
    w = torch.stack(words, 1).view(-1)
    return (w & 0xFFFF).float() * 2.0 ** -16, (w >> 16).float() * 2.0 ** -16


def _philox_round(c0, c1, c2, c3, k0, k1):
    h0, l0 = _mulhilo(c0, 0xD2511F53)
    h1, l1 = _mulhilo(c2, 0xCD9E8D57)
    return h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0, (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF


def _f32(x):
    return torch.tensor(x, dtype=torch.float32).item()


def _blocks(x):
    """[n] -> [rows, BLOCK], filled up with zeros."""
    return torch.nn.functional.pad(x, (0, _rows(x.numel()) * BLOCK - x.numel())).view(-1, BLOCK)


def _plain_adamw_one(s, i):
    w, hp = {k: t[i] for k, t in s["views"].items()}, HP
    bits, n = s["case"]["bits"], w["p"].numel()
    b1, b2, lr = _f32(hp["beta1"]), _f32(hp["beta2"]), _f32(hp["lr"])
    c1, c2 = _f32(1.0 / (1.0 - b1 ** hp["step"])), _f32(1.0 / (1.0 - b2 ** hp["step"]))
    g = w["g"].float()
    if bits == 8:
        m = _from_8(_blocks(w["mq"]), w["me"], 13, True).view(-1)[:n]
        v = _from_8(_blocks(w["vq"]), w["ve"], 29, False).view(-1)[:n]
    else:
        m, v = w["m"], w["v"]
    v = v * b2 + (g * g) * (1.0 - b2)
    root = torch.sqrt(v * c2)
    bound = root * _f32(hp["clip_k"])
    m = m * b1 + torch.minimum(torch.maximum(g, -bound), bound) * (1.0 - b1)
    p = w["p"] * _f32(1.0 - lr * _f32(s["wd"][i])) - (m * c1) / (root + _f32(hp["eps"])) * lr
    w["p"].copy_(p)
    if "p16" in w:
        w["p16"].copy_(p)
    if bits == 8:
        up_m, up_v = _noise(_rows(n) * BLOCK, hp["step"], i, hp["seed"])
        mq, me = _to_8(_blocks(m), up_m.view(-1, BLOCK), 13, True)
        vq, ve = _to_8(_blocks(v), up_v.view(-1, BLOCK), 29, False)
        w["mq"].copy_(mq.view(-1)[:n])
        w["me"].copy_(me)
        w["vq"].copy_(vq.view(-1)[:n])
        w["ve"].copy_(ve)
        m, v = _from_8(mq, me, 13, True).view(-1)[:n], _from_8(vq, ve, 29, False).view(-1)[:n]
    w["m"].copy_(m)
    w["v"].copy_(v)


def _adamw_out(s):
    return {k: s["flat"][k] for k in ("p", "m", "v", "p16") if k in s["flat"]}


def _plain_adamw(s):
    [_plain_adamw_one(s, i) for i in range(len(s["wd"]))]
    return _adamw_out(s)


# ------------------------------------------------------------------- run


_PLAIN = {"fwd": _plain_fwd, "bwd": _plain_bwd, "step": _plain_step, "norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd,
          "adamw": _plain_adamw}


def run(state):
    s = state
    c = s["case"]
    kind = c["kind"]
    if not own:
        return _PLAIN[kind](s)
    from paper_1912_06680_amd import o5
    dt = int(c["dtype"] == "bf16") if "dtype" in c else 0
    if kind == "step":
        o5.o5_linattn_step(dt, c["B"], c["nh"], c["nkv"], c["dk"], c["dv"], s["q"], s["q"].stride(0), s["k"], s["k"].stride(0),
                           s["v"], s["v"].stride(0), s["decay"], s["scale"], s["reset"], s["S"], s["o"], s["o"].stride(0))
        return {"o": s["o"], "S": s["S"]}
    if kind in ("fwd", "bwd"):
        size = (c["T"], c["B"], c["nh"], c["nkv"], c["dk"], c["dv"])
        inputs = (s["q"], s["q"].stride(1), s["k"], s["k"].stride(1), s["v"], s["v"].stride(1), s["decay"], s["scale"], s["S"],
                  s["reset"])
        if kind == "fwd":
            o5.o5_linattn_fwd(dt, *size, *inputs, s["o"], s["o"].stride(1), s["ST"], s["ws"])
            return {"o": s["o"], "ST": s["ST"]}
        o5.o5_linattn_bwd(dt, *size, *inputs, s["do"], s["do"].stride(1), s["dST"], s["dq"], s["dq"].stride(1),
                          s["dk"], s["dk"].stride(1), s["dv"], s["dv"].stride(1), s["dS"], s["ws"])
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"], "dS0": s["dS"]}
    if kind == "norm_fwd":
        o5.o5_resnorm_fwd(int(c["xt"] == "bf16"), dt, c["N"], c["D"], s["x"], s["u"], s["gate"], c["D"], s["w_post"], s["rho"],
                          s["w_pre"], EPS, s["xo"], s["n"], s["r_post"], s["r_pre"])
        return {k: s[k] for k in ("xo", "r_post", "n", "r_pre") if s[k] is not None}
    if kind == "norm_bwd":
        o5.o5_resnorm_bwd(int(c["xt"] == "bf16"), dt, c["N"], c["D"], s["x"], s["u"], s["gate"], c["D"], s["w_post"], s["rho"],
                          s["w_pre"], s["r_post"], s["r_pre"], s["dxo"], s["dn"], s["dx"], s["du"], s["dgate"], c["D"],
                          s["dw_post"], s["drho"], s["dw_pre"], s["ws"])
        return {k: s[k] for k in ("dw_pre", "dx", "dgate", "drho", "dw_post", "du") if s[k] is not None}
    o5.o5_adamw_step(s["plan"], s["plan_dev"], HP["lr"], HP["beta1"], HP["beta2"], HP["eps"], HP["clip_k"], HP["seed"], HP["step"])
    if c["bits"] == 8:
        o5.o5_adamw_moments(s["plan"], s["plan_dev"], s["flat"]["m"], s["flat"]["v"])
    return _adamw_out(s)


# ----------------------------------------------------------------- exact


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("step", "fwd", "bwd"):
        return _exact_linattn(case, s)
    if kind == "adamw":
        return _exact_adamw(case, s)
    return _exact_norm(case, s)


def _exact_linattn(c, s):
    """The recurrence, step by step."""
    T, B, nh, nkv, dk, dv = c.get("T", 1), c["B"], c["nh"], c["nkv"], c["dk"], c["dv"]
    g = nh // nkv
    q = s["q"].reshape(T, B, nkv, g, dk)
    k, v = s["k"].reshape(T, B, nkv, dk), s["v"].reshape(T, B, nkv, dv)
    lam, scale = s["decay"].double().view(1, nkv, 1, 1), s["scale"]
    cut = torch.zeros(T, B, dtype=torch.bool, device=DEV) if s["reset"] is None else s["reset"].view(T, B) != 0
    S = s["S"].double().clone()
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    back = c["kind"] == "bwd"
    do = s["do"].reshape(T, B, nkv, g, dv) if back else None
    outs = []
    for t in range(T):
        S = lam * torch.where(cut[t].view(B, 1, 1, 1), zero, S) + k[t].double()[..., :, None] * v[t].double()[..., None, :]
        if back:
            outs.append(torch.matmul(do[t].double(), S.transpose(-1, -2).contiguous()).float() * scale)
        else:
            outs.append((scale * torch.matmul(q[t].double(), S)).to(torch.float32 if c["dtype"] == "bf16" else torch.float64))
    if c["kind"] == "step":
        return {"o": outs[0].reshape(B, nh * dv), "S": S}
    if not back:
        return {"o": torch.stack(outs).view(T, B, nh * dv), "ST": S}
    G = s["dST"].double().clone()
    dks, dvs = [], []
    for t in reversed(range(T)):
        G = G + scale * torch.matmul(q[t].double().transpose(-1, -2).contiguous(), do[t].double())
        dks.append(torch.matmul(G, v[t].double()[..., None])[..., 0].float())
        dvs.append(torch.matmul(k[t].double()[..., None, :], G)[..., 0, :].float())
        G = torch.where(cut[t].view(B, 1, 1, 1), zero, lam * G)
    return {"dq": torch.stack(outs).view(T, B, nh * dk), "dk": torch.stack(dks[::-1]).view(T, B, nkv * dk),
            "dv": torch.stack(dvs[::-1]).view(T, B, nkv * dv), "dS0": G}


def _exact_norm(c, s):
    """The definition in 64 bits, its gradient by automatic differentiation."""
    wide = {k: None if s[k] is None else s[k].double() for k in ("x", "u", "gate", "w_post", "rho", "w_pre")}
    norm = lambda z: (z * z).mean(-1, keepdim=True).add(EPS).pow(-0.5)  # noqa: E731
    gate = lambda z: 1.0 if z is None else torch.sigmoid(z)  # noqa: E731
    x, u = wide["x"], wide["u"]
    if c["kind"] == "norm_fwd":
        out = {}
        if u is not None:
            x = x + wide["rho"] * gate(wide["gate"]) * (wide["w_post"] * u * norm(u))
            out["xo"], out["r_post"] = x, norm(u)[:, 0]
        if wide["w_pre"] is not None:
            out["n"], out["r_pre"] = wide["w_pre"] * x * norm(x), norm(x)[:, 0]
        return out
    out = {}
    d = s["dxo"].double()
    if wide["w_pre"] is not None:
        x.requires_grad_()
        wide["w_pre"].requires_grad_()
        gx, gw = torch.autograd.grad((wide["w_pre"] * x * norm(x) * s["dn"].double()).sum(), (x, wide["w_pre"]))
        d, out["dw_pre"] = d + gx, gw
    out["dx"] = d
    if u is not None:
        names = [n for n in ("u", "gate", "w_post", "rho") if wide[n] is not None]
        leaves = [wide[n].requires_grad_() for n in names]
        y = wide["rho"] * gate(wide["gate"]) * (wide["w_post"] * u * norm(u))
        out.update(zip(("d" + n for n in names), torch.autograd.grad((y * d).sum(), leaves)))
    return out


def _exact_round(x, up, low, signed):
    """The value that stands for each x [rows, BLOCK] in 8 bits, in 64 bits throughout."""
    mag = x.abs()
    top = torch.floor(torch.log2(mag.amax(-1, keepdim=True).clamp(min=2.0 ** -90)))
    e = torch.floor(torch.log2(mag.clamp(min=2.0 ** -200)))
    step = torch.exp2(torch.maximum(e, top - low) - 3)
    y = torch.floor(mag / step + up) * step
    if not signed:
        y = torch.where(x > 0, torch.maximum(y, torch.exp2(top - low - 3)), y)
    return torch.where(x < 0, -y, y)


def _exact_words(n, step, tensor, seed):
    """The random words of n elements, by products of 16-bit halves."""
    def times(a, b):
        al, ah, bl, bh = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
        mid = ah * bl + ((al * bl) >> 16)
        mid2 = al * bh + (mid & 0xFFFF)
        return ah * bh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((al * bl) & 0xFFFF)

    x = [torch.arange((n + 3) // 4, device=DEV)]
    x += [torch.full_like(x[0], z) for z in (0, step, tensor)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(7):
        (ha, la), (hb, lb) = times(x[0], 0xD2511F53), times(x[2], 0xCD9E8D57)
        x = [hb ^ x[1] ^ key[0], lb, ha ^ x[3] ^ key[1], la]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    return torch.stack(x, -1).reshape(-1)[:n]


def _exact_adamw(c, s):
    out = {k: torch.zeros(t.shape, dtype=torch.float64, device=DEV) for k, t in _adamw_out(s).items()}
    b1, b2, lr, eps, clip = (_f32(HP[k]) for k in ("beta1", "beta2", "lr", "eps", "clip_k"))
    at = 0
    for i, n in enumerate(_sizes(c)):
        w = {k: t[i] for k, t in s["views"].items()}
        full = _rows(n) * BLOCK
        g = w["g"].double()
        if c["bits"] == 8:
            m0 = _from_8(_blocks(w["mq"]), w["me"], 13, True).double().view(-1)[:n]
            v0 = _from_8(_blocks(w["vq"]), w["ve"], 29, False).double().view(-1)[:n]
        else:
            m0, v0 = w["m"].double(), w["v"].double()
        v = b2 * v0 + (1 - b2) * g ** 2
        root = (v / (1 - b2 ** HP["step"])).sqrt()
        m = b1 * m0 + (1 - b1) * torch.clamp(g, -clip * root, clip * root)
        p = w["p"].double() * (1 - lr * _f32(s["wd"][i])) - lr * m / (1 - b1 ** HP["step"]) / (root + eps)
        if c["bits"] == 8:
            words = _exact_words(full, HP["step"], i, HP["seed"])
            m = _exact_round(_blocks(m), (words & 0xFFFF).double().view(-1, BLOCK) / 65536, 13, True).view(-1)[:n]
            v = _exact_round(_blocks(v), (words >> 16).double().view(-1, BLOCK) / 65536, 29, False).view(-1)[:n]
        for name, value in (("p", p), ("m", m), ("v", v), ("p16", p)):
            if name in out:
                out[name][at:at + n] = value
        at += full
    return out
