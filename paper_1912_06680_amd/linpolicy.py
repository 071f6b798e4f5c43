"""A recurrent policy whose core is parallel over time, trained with PPO.

Where the LSTM policy (step.py) runs its steps one after another over short
samples, this one's blocks carry their state by linear attention with a decay
for each head, so that a whole rollout segment is one sample:

    n = norm(x; w_pre);  [q | k | v | g] = n W_in^T
    u = linattn(q, k, v) W_out^T
    x' = x + rho sigmoid(g) norm(u; w_post)

(o5_linattn_*, and o5_resnorm_* for the norms, the gate and the residual sum in
one pass between two blocks), then the heads and the PPO loss on the last
norm's output, the backward pass through the same calls, and one o5_adamw_step
over every tensor, its moments in 8 bits or in 32.  In the rollout the same
weights run one token at a time on states kept in place.

This module allocates device buffers (torch), calls the library in order on
one stream and leaves the plain products with the projections to torch.mm.

    python -m paper_1912_06680_amd.linpolicy      # a few training steps on synthetic segments
"""
import torch

from . import o5

EPS = 1e-6
VECTORS = ("w_pre", "w_post", "rho")


def _decays(heads, device):
    """Half-lives from about 20 steps to a few thousand."""
    i = torch.arange(heads, dtype=torch.float64) / max(1, heads - 1)
    return (1.0 - torch.exp2(-5.0 - 7.0 * i)).float().to(device)


class LinPolicy:
    """Parameters, buffers and call sequence for segments of T steps of B environments.

    D: width, a multiple of 64; heads: of D / heads, a multiple of 8 up to 128; head_sizes: of the action heads.

    self.S0 holds the blocks' states before the segments, zeros at first.  To train on the segments that follow, copy
    self.ST into it, with zeros where the last step's `dones` is set: a segment's resets begin at its second step.
    """

    def __init__(self, T, B, D, layers, heads, head_sizes, dtype="bf16", bits=8, seed=0, lr=5e-5, weight_decay=0.01,
                 device="cuda"):
        assert D % 64 == 0 and D % heads == 0 and layers >= 1
        self.T, self.B, self.D, self.layers, self.heads, self.head_sizes = T, B, D, layers, heads, tuple(head_sizes)
        self.N, self.d = T * B, D // heads
        self.bf16 = dtype == "bf16"
        self.dt, self.et = (o5.O5_BF16, torch.bfloat16) if self.bf16 else (o5.O5_F32, torch.float32)
        self.dev, self.lr, self.seed, self.step_count = device, lr, seed, 0
        self.scale = self.d ** -0.5
        self.decay = _decays(heads, device)
        A1 = sum(self.head_sizes) + 1
        self.shapes = {}
        for i in range(layers):
            self.shapes.update({f"W_in{i}": (4 * D, D), f"W_out{i}": (D, D), f"w_pre{i}": (D,), f"w_post{i}": (D,),
                                f"rho{i}": (D,)})
        self.shapes.update({f"w_pre{layers}": (D,), "Wp": (A1, D), "bp": (A1,)})
        self._parameters(bits, weight_decay)
        N, f32 = self.N, dict(dtype=torch.float32, device=device)
        e = dict(dtype=self.et, device=device)
        # what a forward pass leaves for the backward pass, by block
        self.x = [torch.empty((N, D), **f32) for _ in range(layers + 1)]
        self.n = [torch.empty((N, D), **e) for _ in range(layers + 1)]
        self.r_pre = [torch.empty(N, **f32) for _ in range(layers + 1)]
        self.qkvg = [torch.empty((N, 4 * D), **e) for _ in range(layers)]
        self.o = [torch.empty((N, D), **e) for _ in range(layers)]
        self.u = [torch.empty((N, D), **e) for _ in range(layers)]
        self.r_post = [torch.empty(N, **f32) for _ in range(layers)]
        state = (B, heads, self.d, self.d)
        self.S0 = [torch.zeros(state, **f32) for _ in range(layers)]
        self.ST = [torch.empty(state, **f32) for _ in range(layers)]
        # gradients on their way and scratch
        self.dstream = torch.empty((N, D), **f32)
        self.dh = torch.empty((N, D), **f32)
        self.dn, self.du, self.do = (torch.empty((N, D), **e) for _ in range(3))
        self.dqkvg = torch.empty((N, 4 * D), **e)
        self.stats = torch.empty(8, **f32)
        self.adv, self.ret, self.adv_s, self.ret_s = (torch.empty((T, B), **f32) for _ in range(4))
        self.reset = torch.empty((T, B), dtype=torch.uint8, device=device)
        size = (self.dt, T, B, heads, heads, self.d, self.d)
        need = max(o5.o5_linattn_fwd_workspace_bytes(*size), o5.o5_linattn_bwd_workspace_bytes(*size),
                   o5.o5_resnorm_bwd_workspace_bytes(o5.O5_F32, self.dt, N, D),
                   o5.o5_ppo_loss_grad_workspace_bytes(self.dt, N, D, self.head_sizes),
                   o5.o5_policy_sample_workspace_bytes(self.dt, B, D, self.head_sizes))
        self.ws = torch.empty(need, dtype=torch.uint8, device=device)

    def _parameters(self, bits, weight_decay):
        """Masters in fp32, their copies for the products, gradients and moments; the plan of their update."""
        gen = torch.Generator(device=self.dev).manual_seed(self.seed)
        f32 = dict(dtype=torch.float32, device=self.dev)
        self.P, self.W, self.G, self.moments, tensors = {}, {}, {}, {}, []
        for name, shape in self.shapes.items():
            matrix = len(shape) == 2
            if matrix:
                p = torch.randn(shape, generator=gen, **f32) * shape[1] ** -0.5
                p *= 0.1 if name == "Wp" else 1.0
            else:
                p = torch.full(shape, 0.1 if name.startswith("rho") else 0.0 if name == "bp" else 1.0, **f32)
            self.P[name] = p
            copy = matrix and self.bf16
            self.W[name] = p.to(torch.bfloat16) if copy else p
            # the projections' gradients come out of their products in the products' type
            self.G[name] = torch.empty(shape, dtype=self.et if matrix and name != "Wp" else torch.float32, device=self.dev)
            if bits == 8:
                m, v = (torch.zeros(shape, dtype=torch.uint8, device=self.dev) for _ in range(2))
                me, ve = (torch.zeros((p.numel() + 255) // 256, dtype=torch.uint8, device=self.dev) for _ in range(2))
            else:
                m, v, me, ve = torch.zeros(shape, **f32), torch.zeros(shape, **f32), None, None
            self.moments[name] = (m, v, me, ve)
            tensors.append(o5.adamw_tensor(p, self.G[name], m, v, me, ve, self.W[name] if copy else None,
                                           weight_decay=weight_decay if matrix else 0.0))
        self.plan = torch.empty(o5.o5_adamw_plan_bytes(tensors), dtype=torch.uint8)
        o5.o5_adamw_plan(tensors, self.plan)
        self.plan_dev = self.plan.to(self.dev)

    # -------------------------------------------------------------- training
    def _parts(self, qkvg):
        D = self.D
        return [qkvg[:, i * D:(i + 1) * D] for i in range(4)]

    def forward(self, x, reset=None):
        """x [T, B, D] fp32; leaves the heads' input in self.n[-1] and the last states in self.ST."""
        T, B, D, N, P, W = self.T, self.B, self.D, self.N, self.P, self.W
        self.x[0].copy_(x.view(N, D))
        o5.o5_resnorm_fwd(o5.O5_F32, self.dt, N, D, self.x[0], None, None, 0, None, None, P["w_pre0"], EPS, None, self.n[0],
                          None, self.r_pre[0])
        for i in range(self.layers):
            torch.mm(self.n[i], W[f"W_in{i}"].t(), out=self.qkvg[i])
            q, k, v, g = self._parts(self.qkvg[i])
            o5.o5_linattn_fwd(self.dt, T, B, self.heads, self.heads, self.d, self.d, q, 4 * D, k, 4 * D, v, 4 * D, self.decay,
                              self.scale, self.S0[i], reset, self.o[i], D, self.ST[i], self.ws)
            torch.mm(self.o[i], W[f"W_out{i}"].t(), out=self.u[i])
            o5.o5_resnorm_fwd(o5.O5_F32, self.dt, N, D, self.x[i], self.u[i], g, 4 * D, P[f"w_post{i}"], P[f"rho{i}"],
                              P[f"w_pre{i + 1}"], EPS, self.x[i + 1], self.n[i + 1], self.r_post[i], self.r_pre[i + 1])

    def backward(self, reset=None):
        """Every parameter's gradient into self.G, from the loss's gradient self.dh on the heads' input."""
        T, B, D, N, P, W, G = self.T, self.B, self.D, self.N, self.P, self.W, self.G
        if self.bf16:
            o5.o5_f32_to_bf16(N * D, self.dh, self.dn)
        else:
            self.dn.copy_(self.dh)
        self.dstream.zero_()
        dq, dk, dv, dg = self._parts(self.dqkvg)
        for i in reversed(range(self.layers)):
            q, k, v, g = self._parts(self.qkvg[i])
            o5.o5_resnorm_bwd(o5.O5_F32, self.dt, N, D, self.x[i + 1], self.u[i], g, 4 * D, P[f"w_post{i}"], P[f"rho{i}"],
                              P[f"w_pre{i + 1}"], self.r_post[i], self.r_pre[i + 1], self.dstream, self.dn, self.dstream,
                              self.du, dg, 4 * D, G[f"w_post{i}"], G[f"rho{i}"], G[f"w_pre{i + 1}"], self.ws)
            torch.mm(self.du.t(), self.o[i], out=G[f"W_out{i}"])
            torch.mm(self.du, W[f"W_out{i}"], out=self.do)
            o5.o5_linattn_bwd(self.dt, T, B, self.heads, self.heads, self.d, self.d, q, 4 * D, k, 4 * D, v, 4 * D, self.decay,
                              self.scale, self.S0[i], reset, self.do, D, None, dq, 4 * D, dk, 4 * D, dv, 4 * D, None, self.ws)
            torch.mm(self.dqkvg.t(), self.n[i], out=G[f"W_in{i}"])
            torch.mm(self.dqkvg, W[f"W_in{i}"], out=self.dn)
        o5.o5_resnorm_bwd(o5.O5_F32, self.dt, N, D, self.x[0], None, None, 0, None, None, P["w_pre0"], None, self.r_pre[0],
                          self.dstream, self.dn, self.dstream, None, None, 0, None, None, G["w_pre0"], self.ws)

    def loss(self, act, logp_old, adv, ret, clip_eps=0.2, vf_coef=1.0, ent_coef=0.01):
        o5.o5_ppo_loss_grad(self.dt, self.N, self.D, self.head_sizes, self.n[-1], self.W["Wp"], self.P["bp"], act, logp_old,
                            adv, ret, None, clip_eps, vf_coef, ent_coef, self.stats, self.dh, self.G["Wp"], self.G["bp"],
                            self.ws)

    def train_step(self, x, rewards, dones, values, act, logp_old, gamma=0.998, lam=0.95):
        """One optimizer step on B segments of T steps; self.stats holds the loss, self.ST the states after them.

        x [T, B, D]; rewards, dones [T, B]; values [T + 1, B]; act [T B, heads] int32; logp_old [T B]."""
        T, B = self.T, self.B
        o5.o5_gae(T, B, rewards, values, dones, gamma, lam, self.adv, self.ret)
        # a segment is one sample: this only turns episode ends into the next step's resets
        o5.o5_segments_to_samples(T, B, T, self.adv, self.ret, dones, self.adv_s, self.ret_s, self.reset)
        self.forward(x, self.reset)
        self.loss(act, logp_old, self.adv_s, self.ret_s)
        self.backward(self.reset)
        self.step_count += 1
        o5.o5_adamw_step(self.plan, self.plan_dev, self.lr, 0.9, 0.999, 1e-8, 5.0, self.seed, self.step_count)

    # --------------------------------------------------------------- rollout
    def new_states(self):
        return [torch.zeros_like(s) for s in self.S0]

    def act(self, x, states, seed, counter, reset=None):
        """One step of B environments: x [B, D] fp32, states updated in place; (actions, log-probability, value)."""
        B, D, P, W = self.B, self.D, self.P, self.W
        e = dict(dtype=self.et, device=self.dev)
        x = x.clone()
        n = torch.empty((B, D), **e)
        o = torch.empty((B, D), **e)
        o5.o5_resnorm_fwd(o5.O5_F32, self.dt, B, D, x, None, None, 0, None, None, P["w_pre0"], EPS, None, n, None, None)
        for i in range(self.layers):
            qkvg = torch.mm(n, W[f"W_in{i}"].t())
            q, k, v, g = self._parts(qkvg)
            o5.o5_linattn_step(self.dt, B, self.heads, self.heads, self.d, self.d, q, 4 * D, k, 4 * D, v, 4 * D, self.decay,
                               self.scale, reset, states[i], o, D)
            u = torch.mm(o, W[f"W_out{i}"].t())
            o5.o5_resnorm_fwd(o5.O5_F32, self.dt, B, D, x, u, g, 4 * D, P[f"w_post{i}"], P[f"rho{i}"], P[f"w_pre{i + 1}"], EPS,
                              x, n, None, None)
        act = torch.empty((B, len(self.head_sizes)), dtype=torch.int32, device=self.dev)
        logp, value = torch.empty(B, device=self.dev), torch.empty(B, device=self.dev)
        o5.o5_policy_sample(self.dt, B, D, self.head_sizes, n, W["Wp"], P["bp"], seed, counter, act, logp, value, self.ws)
        return act, logp, value


def rollout(policy, x, seed=1, dones=None):
    """T steps of the policy on the inputs x [T + 1, B, D]: (act [T B, heads], logp [T B], values [T + 1, B])."""
    states, out = policy.new_states(), []
    for t in range(x.shape[0]):
        reset = dones[t - 1].contiguous().clone() if dones is not None and t > 0 else None
        out.append(policy.act(x[t], states, seed, t, reset))
    T = x.shape[0] - 1
    return (torch.stack([o[0] for o in out[:T]]).flatten(0, 1), torch.cat([o[1] for o in out[:T]]),
            torch.stack([o[2] for o in out]))


def main(steps=20):
    """Trains on one synthetic batch, drawn by the untrained policy, and prints the loss."""
    T, B, D = 128, 32, 512
    policy = LinPolicy(T, B, D, layers=2, heads=4, head_sizes=(30, 8, 32, 4), lr=1e-3)
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((T + 1, B, D), generator=gen, device="cuda")
    rewards = torch.randn((T, B), generator=gen, device="cuda")
    dones = (torch.rand((T, B), generator=gen, device="cuda") < 0.01).to(torch.uint8)
    act, logp, values = rollout(policy, x, dones=dones)
    for i in range(steps):
        policy.train_step(x[:T].contiguous(), rewards, dones, values, act, logp)
        total, _, vf, ent = policy.stats[:4].tolist()
        print(f"step {i + 1}: loss {total:.5f} (value {vf:.5f}, entropy {ent:.4f})", flush=True)


if __name__ == "__main__":
    main()
