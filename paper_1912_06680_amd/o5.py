"""Python binding of libo5 (ctypes).

Argument marshalling only: every function below has the name of the C entry
point it calls, takes torch tensors (device memory) where the C call takes
device pointers, and raises ``O5Error`` when the call returns a nonzero
status.  No computation happens here; if ``libo5.so`` has not been built the
first call raises instead of falling back to anything else.

Default stream: the current torch stream of the current device.
"""
import ctypes
import os

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libo5.so")

O5_F32 = 0
O5_BF16 = 1

EXPORTED = (
    "o5_version", "o5_status_str", "o5_last_error",
    "o5_lstm_fwd_workspace_bytes", "o5_lstm_fwd",
    "o5_lstm_bptt_workspace_bytes", "o5_lstm_bptt", "o5_lstm_bptt_factored",
    "o5_gae", "o5_segments_to_samples",
    "o5_reward_process_workspace_bytes", "o5_reward_process",
    "o5_obs_normalize_workspace_bytes", "o5_obs_normalize", "o5_prelstm_fwd",
    "o5_prelstm_bwd_workspace_bytes", "o5_prelstm_bwd",
    "o5_ppo_loss_grad_workspace_bytes", "o5_ppo_loss_grad", "o5_ppo_head_grad_ld", "o5_ppo_loss_grad_factored",
    "o5_ppo_logits_grad_workspace_bytes", "o5_ppo_logits_grad",
    "o5_adam_step",
    "o5_policy_sample_workspace_bytes", "o5_policy_sample", "o5_policy_sample_static",
    "o5_linattn_fwd_workspace_bytes", "o5_linattn_fwd", "o5_linattn_bwd_workspace_bytes", "o5_linattn_bwd",
    "o5_linattn_step",
    "o5_gatedrec_marks_bytes", "o5_gatedrec_fwd_workspace_bytes", "o5_gatedrec_fwd", "o5_gatedrec_bwd_workspace_bytes",
    "o5_gatedrec_bwd", "o5_gatedrec_step",
    "o5_resnorm_fwd", "o5_resnorm_bwd_workspace_bytes", "o5_resnorm_bwd",
    "o5_adamw_plan_bytes", "o5_adamw_plan", "o5_adamw_step", "o5_adamw_moments",
    "o5_adamw_grad_norm_workspace_bytes", "o5_adamw_grad_norm", "o5_adamw_step_clipped",
    "o5_f32_to_bf16",
    "o5_param_count", "o5_surgery_widen", "o5_surgery_fold_input",
    "o5_ktimer_enable", "o5_ktimer_enable_sites", "o5_ktimer_read", "o5_ktimer_site_name",
)

KTIMER_SITES = ("lstm_fwd_gemm", "lstm_fwd_cell", "lstm_dh_gemm", "lstm_bwd_cell", "lstm_dw_gemm",
                "lstm_dx_gemm", "ppo_loss_grad", "adam_step", "gae", "policy_sample", "reward_process",
                "obs_normalize", "prelstm_fwd", "prelstm_bwd", "lstm_fwd_call")


class O5Error(RuntimeError):
    def __init__(self, fn, status, msg):
        super().__init__(f"{fn} failed with status {status}: {msg}")
        self.status = status


class PpoHp(ctypes.Structure):
    _fields_ = [("clip_eps", ctypes.c_float), ("vf_coef", ctypes.c_float), ("ent_coef", ctypes.c_float)]


class AdamHp(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("clip_k", ctypes.c_float)]


class UnitHead(ctypes.Structure):
    _fields_ = [("head", ctypes.c_int), ("d", ctypes.c_int), ("Wq", ctypes.c_void_p), ("bq", ctypes.c_void_p),
                ("E", ctypes.c_void_p), ("dWq", ctypes.c_void_p), ("dbq", ctypes.c_void_p)]


def unit_head(head, d, Wq, bq, E, dWq=None, dbq=None):
    """An o5_unit_head over torch tensors (keep the tensors alive for the call)."""
    return UnitHead(int(head), int(d), _p(Wq), _p(bq), _p(E), _p(dWq), _p(dbq))


def _unit(u):
    return None if u is None else ctypes.byref(u)


class RewardHp(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_float), ("decay_base", ctypes.c_float), ("decay_minutes", ctypes.c_float),
                ("eps", ctypes.c_float)]


class AdamwTensor(ctypes.Structure):
    _fields_ = [("n", ctypes.c_size_t), ("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("p_bf16", ctypes.c_void_p), ("lr_scale", ctypes.c_float), ("weight_decay", ctypes.c_float),
                ("g_dt", ctypes.c_int), ("bits", ctypes.c_int)]


def adamw_tensor(p, g, m, v, m_exp=None, v_exp=None, p_bf16=None, lr_scale=1.0, weight_decay=0.0):
    """An o5_adamw_tensor over torch tensors (keep the tensors alive while the plan is used): g's type by its dtype,
    moments in 8 bits where m is a tensor of bytes.  Refuses tensors that the kernels would read as what they are not."""
    n = p.numel()
    state = torch.uint8 if m.dtype == torch.uint8 else torch.float32
    groups = (n + 255) // 256 if state == torch.uint8 else 0
    for name, t, dtypes, least in (("p", p, (torch.float32,), n), ("g", g, (torch.float32, torch.bfloat16), n),
                                   ("m", m, (state,), n), ("v", v, (state,), n), ("m_exp", m_exp, (torch.uint8,), groups),
                                   ("v_exp", v_exp, (torch.uint8,), groups), ("p_bf16", p_bf16, (torch.bfloat16,), n)):
        if t is not None and (t.dtype not in dtypes or t.numel() < least or not t.is_contiguous()):
            raise ValueError(f"adamw_tensor: {name} must be contiguous, of {' or '.join(map(str, dtypes))} and of at least "
                             f"{least} elements, not {t.dtype} {tuple(t.shape)}")
    return AdamwTensor(p.numel(), _p(p), _p(g), _p(m), _p(v), _p(m_exp), _p(v_exp), _p(p_bf16), float(lr_scale),
                       float(weight_decay), O5_BF16 if g.dtype == torch.bfloat16 else O5_F32,
                       8 if m.dtype == torch.uint8 else 32)


_vp = ctypes.c_void_p
_i = ctypes.c_int
_sz = ctypes.c_size_t
_f = ctypes.c_float
_u64 = ctypes.c_uint64

_SIGS = {
    "o5_version": (_i, []),
    "o5_status_str": (ctypes.c_char_p, [_i]),
    "o5_last_error": (ctypes.c_char_p, []),
    "o5_lstm_fwd_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "o5_lstm_fwd": (_i, [_i, _i, _i, _i, _i] + [_vp] * 11 + [_sz, _vp]),
    "o5_lstm_bptt_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "o5_lstm_bptt": (_i, [_i, _i, _i, _i, _i] + [_vp] * 17 + [_sz, _vp]),
    "o5_lstm_bptt_factored": (_i, [_i, _i, _i, _i, _i] + [_vp] * 11 + [_i] + [_vp] * 7 + [_sz, _vp]),
    "o5_gae": (_i, [_i, _i, _vp, _vp, _vp, _f, _f, _vp, _vp, _vp]),
    "o5_segments_to_samples": (_i, [_i, _i, _i] + [_vp] * 6 + [_vp]),
    "o5_reward_process_workspace_bytes": (_sz, [_i, _i]),
    "o5_reward_process": (_i, [_i, _i, _vp, _vp, _vp, RewardHp, _vp, _vp, _vp, _sz, _vp]),
    "o5_obs_normalize_workspace_bytes": (_sz, [_i, _i]),
    "o5_obs_normalize": (_i, [_i, _i, _i, _vp, _vp, _f, _f, _vp, _vp, _sz, _vp]),
    "o5_prelstm_fwd": (_i, [_i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp]),
    "o5_prelstm_bwd_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "o5_prelstm_bwd": (_i, [_i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "o5_ppo_loss_grad_workspace_bytes": (_sz, [_i, _i, _i, _i, _vp, _vp]),
    "o5_ppo_loss_grad": (_i, [_i, _i, _i, _i, _vp] + [_vp] * 10 + [PpoHp] + [_vp] * 5 + [_sz, _vp]),
    "o5_ppo_head_grad_ld": (_i, [_i, _i, _vp, _vp]),
    "o5_ppo_loss_grad_factored": (_i, [_i, _i, _i, _i, _vp] + [_vp] * 10 + [PpoHp] + [_vp] * 3 + [_i] + [_vp] * 3
                                  + [_sz, _vp]),
    "o5_ppo_logits_grad_workspace_bytes": (_sz, [_i, _i, _i, _vp]),
    "o5_ppo_logits_grad": (_i, [_i, _i, _i, _vp] + [_vp, _sz] * 2 + [_vp] * 7 + [PpoHp, _f] + [_vp] * 4
                           + [_sz, _vp, _sz, _vp]),
    "o5_adam_step": (_i, [_sz, _vp, _vp, _vp, _vp, _vp, AdamHp, _i, _vp]),
    "o5_policy_sample_workspace_bytes": (_sz, [_i, _i, _i, _i, _vp, _vp]),
    "o5_policy_sample": (_i, [_i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _u64, _u64, _vp, _vp, _vp, _vp, _sz,
                              _vp]),
    "o5_policy_sample_static": (_i, [_i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _u64, _u64, _vp, _vp, _vp,
                                     _vp]),
    "o5_linattn_fwd_workspace_bytes": (_sz, [_i] * 7),
    "o5_linattn_fwd": (_i, [_i] * 7 + [_vp, _sz] * 3 + [_vp, _f] + [_vp] * 2 + [_vp, _sz, _vp, _vp, _sz, _vp]),
    "o5_linattn_bwd_workspace_bytes": (_sz, [_i] * 7),
    "o5_linattn_bwd": (_i, [_i] * 7 + [_vp, _sz] * 3 + [_vp, _f] + [_vp] * 2 + [_vp, _sz, _vp] + [_vp, _sz] * 3
                       + [_vp, _vp, _sz, _vp]),
    "o5_linattn_step": (_i, [_i] * 6 + [_vp, _sz] * 3 + [_vp, _f] + [_vp] * 2 + [_vp, _sz, _vp]),
    "o5_gatedrec_marks_bytes": (_sz, [_i] * 3),
    "o5_gatedrec_fwd_workspace_bytes": (_sz, [_i] * 4),
    "o5_gatedrec_fwd": (_i, [_i] * 4 + [_vp, _sz] * 3 + [_vp, _f] + [_vp] * 2 + [_vp, _sz] + [_vp] * 3 + [_sz, _vp]),
    "o5_gatedrec_bwd_workspace_bytes": (_sz, [_i] * 4),
    "o5_gatedrec_bwd": (_i, [_i] * 4 + [_vp, _sz] * 3 + [_vp, _f] + [_vp] * 2 + [_vp, _sz, _vp] + [_vp, _sz] * 3 + [_vp] * 3
                        + [_sz, _vp]),
    "o5_gatedrec_step": (_i, [_i] * 3 + [_vp, _sz] * 3 + [_vp, _f] + [_vp] * 2 + [_vp, _sz, _vp]),
    "o5_resnorm_fwd": (_i, [_i] * 4 + [_vp] * 3 + [_sz] + [_vp] * 3 + [_f] + [_vp] * 5),
    "o5_resnorm_bwd_workspace_bytes": (_sz, [_i] * 4),
    "o5_resnorm_bwd": (_i, [_i] * 4 + [_vp] * 3 + [_sz] + [_vp] * 10 + [_sz] + [_vp] * 4 + [_sz, _vp]),
    "o5_adamw_plan_bytes": (_sz, [_i, _vp]),
    "o5_adamw_plan": (_i, [_i, _vp, _vp, _sz]),
    "o5_adamw_step": (_i, [_vp, _vp, AdamHp, _u64, _i, _vp]),
    "o5_adamw_moments": (_i, [_vp] * 5),
    "o5_adamw_grad_norm_workspace_bytes": (_sz, [_vp]),
    "o5_adamw_grad_norm": (_i, [_vp, _vp, _f, _vp, _vp, _sz, _vp]),
    "o5_adamw_step_clipped": (_i, [_vp, _vp, AdamHp, _vp, _u64, _i, _vp]),
    "o5_f32_to_bf16": (_i, [_sz, _vp, _vp, _vp]),
    "o5_param_count": (_sz, [_i, _i, _i]),
    "o5_surgery_widen": (_i, [_i, _i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _f, _u64, _vp]),
    "o5_surgery_fold_input": (_i, [_i, _i, _i, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "o5_ktimer_enable": (_i, [_i]),
    "o5_ktimer_enable_sites": (_i, [ctypes.c_uint]),
    "o5_ktimer_read": (_i, [_i, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int)]),
    "o5_ktimer_site_name": (ctypes.c_char_p, [_i]),
}

_lib = None


def lib():
    """The loaded libo5 (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                               "or `python -m paper_1912_06680_amd.build`")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _p(t):
    """Device pointer of a tensor (None -> NULL)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:  # (the handle itself: 0.3 us a call, where building a torch.cuda.Stream for it takes 2.8)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(fn, status):
    if status != 0:
        msg = lib().o5_last_error().decode()
        raise O5Error(fn, status, msg)


def _ws(ws):
    if ws is None:
        return None, 0
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _heads(head_sizes):
    arr = (ctypes.c_int * len(head_sizes))(*[int(n) for n in head_sizes])
    return arr


def o5_version():
    return lib().o5_version()


def o5_status_str(status):
    return lib().o5_status_str(status).decode()


def o5_last_error():
    return lib().o5_last_error().decode()


def o5_lstm_fwd_workspace_bytes(dt, T, B, D, H):
    return lib().o5_lstm_fwd_workspace_bytes(dt, T, B, D, H)


def o5_lstm_fwd(dt, T, B, D, H, x, Wx, Wh, b, h0, c0, reset, h, c, gates, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_lstm_fwd", lib().o5_lstm_fwd(
        dt, T, B, D, H, _p(x), _p(Wx), _p(Wh), _p(b), _p(h0), _p(c0), _p(reset),
        _p(h), _p(c), _p(gates), wp, wn, _stream(stream)))


def o5_lstm_bptt_workspace_bytes(dt, T, B, D, H):
    return lib().o5_lstm_bptt_workspace_bytes(dt, T, B, D, H)


def o5_lstm_bptt(dt, T, B, D, H, x, Wx, Wh, h0, c0, reset, h, c, gates, dh, dhT, dcT,
                 dWx, dWh, db, dx, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_lstm_bptt", lib().o5_lstm_bptt(
        dt, T, B, D, H, _p(x), _p(Wx), _p(Wh), _p(h0), _p(c0), _p(reset), _p(h), _p(c),
        _p(gates), _p(dh), _p(dhT), _p(dcT), _p(dWx), _p(dWh), _p(db), _p(dx), wp, wn,
        _stream(stream)))


def o5_lstm_bptt_factored(dt, T, B, D, H, x, Wx, Wh, h0, c0, reset, h, c, gates, P, W, ld, dhT, dcT,
                          dWx, dWh, db, dx, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_lstm_bptt_factored", lib().o5_lstm_bptt_factored(
        dt, T, B, D, H, _p(x), _p(Wx), _p(Wh), _p(h0), _p(c0), _p(reset), _p(h), _p(c),
        _p(gates), _p(P), _p(W), int(ld), _p(dhT), _p(dcT), _p(dWx), _p(dWh), _p(db), _p(dx), wp, wn,
        _stream(stream)))


def o5_gae(L, S, r, v, done, gamma, lam, adv, ret, stream=None):
    _check("o5_gae", lib().o5_gae(L, S, _p(r), _p(v), _p(done), float(gamma), float(lam),
                                  _p(adv), _p(ret), _stream(stream)))


def o5_segments_to_samples(L, S, T, adv, ret, done, adv_s, ret_s, reset, stream=None):
    _check("o5_segments_to_samples", lib().o5_segments_to_samples(
        L, S, T, _p(adv), _p(ret), _p(done), _p(adv_s), _p(ret_s), _p(reset), _stream(stream)))


def o5_reward_process_workspace_bytes(L, G):
    return lib().o5_reward_process_workspace_bytes(L, G)


def o5_reward_process(L, G, shaped, outcome, game_time, tau, decay_base, decay_minutes, eps, stats, r, ws,
                      stream=None):
    wp, wn = _ws(ws)
    hp = RewardHp(tau, decay_base, decay_minutes, eps)
    _check("o5_reward_process", lib().o5_reward_process(L, G, _p(shaped), _p(outcome), _p(game_time), hp,
                                                        _p(stats), _p(r), wp, wn, _stream(stream)))


def o5_obs_normalize_workspace_bytes(N, Do):
    return lib().o5_obs_normalize_workspace_bytes(N, Do)


def o5_obs_normalize(dt, N, Do, obs, stats, clip, eps, o, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_obs_normalize", lib().o5_obs_normalize(dt, N, Do, _p(obs), _p(stats), float(clip), float(eps), _p(o),
                                                      wp, wn, _stream(stream)))


def o5_prelstm_fwd(dt, T, B, Do, D, o, W, b, y, x, stream=None):
    _check("o5_prelstm_fwd", lib().o5_prelstm_fwd(dt, T, B, Do, D, _p(o), _p(W), _p(b), _p(y), _p(x),
                                                  _stream(stream)))


def o5_prelstm_bwd_workspace_bytes(dt, T, B, Do, D):
    return lib().o5_prelstm_bwd_workspace_bytes(dt, T, B, Do, D)


def o5_prelstm_bwd(dt, T, B, Do, D, o, y, dx, dW, db, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_prelstm_bwd", lib().o5_prelstm_bwd(dt, T, B, Do, D, _p(o), _p(y), _p(dx), _p(dW), _p(db), wp, wn,
                                                  _stream(stream)))


def o5_ppo_loss_grad_workspace_bytes(dt, N, H, head_sizes, unit=None):
    return lib().o5_ppo_loss_grad_workspace_bytes(dt, N, H, len(head_sizes), _heads(head_sizes), _unit(unit))


def o5_ppo_loss_grad(dt, N, H, head_sizes, h, Wp, bp, act, logp_old, adv, ret, head_mask,
                     clip_eps, vf_coef, ent_coef, stats, dh, dWp, dbp, ws, stream=None, avail=None, unit=None):
    wp, wn = _ws(ws)
    hp = PpoHp(clip_eps, vf_coef, ent_coef)
    _check("o5_ppo_loss_grad", lib().o5_ppo_loss_grad(
        dt, N, H, len(head_sizes), _heads(head_sizes), _p(h), _p(Wp), _p(bp), _p(act),
        _p(logp_old), _p(adv), _p(ret), _p(head_mask), _p(avail), _unit(unit), hp, _p(stats), _p(dh), _p(dWp),
        _p(dbp), wp, wn, _stream(stream)))


def o5_ppo_head_grad_ld(H, head_sizes, unit=None):
    return lib().o5_ppo_head_grad_ld(H, len(head_sizes), _heads(head_sizes), _unit(unit))


def o5_ppo_loss_grad_factored(dt, N, H, head_sizes, h, Wp, bp, act, logp_old, adv, ret, head_mask,
                              clip_eps, vf_coef, ent_coef, stats, P, W, ld, dWp, dbp, ws, stream=None,
                              avail=None, unit=None):
    wp, wn = _ws(ws)
    hp = PpoHp(clip_eps, vf_coef, ent_coef)
    _check("o5_ppo_loss_grad_factored", lib().o5_ppo_loss_grad_factored(
        dt, N, H, len(head_sizes), _heads(head_sizes), _p(h), _p(Wp), _p(bp), _p(act),
        _p(logp_old), _p(adv), _p(ret), _p(head_mask), _p(avail), _unit(unit), hp, _p(stats), _p(P), _p(W),
        int(ld), _p(dWp), _p(dbp), wp, wn, _stream(stream)))


def o5_ppo_logits_grad_workspace_bytes(dt, N, head_sizes):
    return lib().o5_ppo_logits_grad_workspace_bytes(dt, N, len(head_sizes), _heads(head_sizes))


def o5_ppo_logits_grad(dt, N, head_sizes, logits, ldl, ref, ldr, act, logp_old, adv, ret, weight, head_mask, avail,
                       clip_eps, vf_coef, ent_coef, kl_coef, stats, logp, kl, dlogits, ldd, ws, stream=None):
    wp, wn = _ws(ws)
    hp = PpoHp(clip_eps, vf_coef, ent_coef)
    _check("o5_ppo_logits_grad", lib().o5_ppo_logits_grad(
        dt, N, len(head_sizes), _heads(head_sizes), _p(logits), ldl, _p(ref), ldr, _p(act), _p(logp_old), _p(adv), _p(ret),
        _p(weight), _p(head_mask), _p(avail), hp, float(kl_coef), _p(stats), _p(logp), _p(kl), _p(dlogits), ldd, wp, wn,
        _stream(stream)))


def o5_adam_step(n, p, m, v, g, p_bf16, lr, beta1, beta2, eps, clip_k, step, stream=None):
    hp = AdamHp(lr, beta1, beta2, eps, clip_k)
    _check("o5_adam_step", lib().o5_adam_step(n, _p(p), _p(m), _p(v), _p(g), _p(p_bf16), hp,
                                              int(step), _stream(stream)))


def o5_policy_sample_workspace_bytes(dt, B, H, head_sizes, unit=None):
    return lib().o5_policy_sample_workspace_bytes(dt, B, H, len(head_sizes), _heads(head_sizes), _unit(unit))


def o5_policy_sample(dt, B, H, head_sizes, h, Wp, bp, seed, counter, act, logp, value, ws,
                     stream=None, avail=None, unit=None):
    wp, wn = _ws(ws)
    _check("o5_policy_sample", lib().o5_policy_sample(
        dt, B, H, len(head_sizes), _heads(head_sizes), _p(h), _p(Wp), _p(bp), _p(avail), _unit(unit), int(seed),
        int(counter), _p(act), _p(logp), _p(value), wp, wn, _stream(stream)))


def o5_policy_sample_static(dt, B, H, head_sizes, h, Wp, bp, seed, counter, act, logp, value, stream=None,
                            avail=None, unit=None):
    _check("o5_policy_sample_static", lib().o5_policy_sample_static(
        dt, B, H, len(head_sizes), _heads(head_sizes), _p(h), _p(Wp), _p(bp), _p(avail), _unit(unit), int(seed),
        int(counter), _p(act), _p(logp), _p(value), _stream(stream)))


def o5_param_count(D, H, A1):
    return lib().o5_param_count(D, H, A1)


def o5_surgery_widen(D, H, A1, D2, H2, p_old, m_old, v_old, p_new, m_new, v_new, scale, seed, stream=None):
    _check("o5_surgery_widen", lib().o5_surgery_widen(D, H, A1, D2, H2, _p(p_old), _p(m_old), _p(v_old), _p(p_new),
                                                      _p(m_new), _p(v_new), float(scale), int(seed),
                                                      _stream(stream)))


def o5_surgery_fold_input(D, H, A1, Dk, E, p_old, m_old, v_old, p_new, m_new, v_new, stream=None):
    _check("o5_surgery_fold_input", lib().o5_surgery_fold_input(D, H, A1, Dk, _p(E), _p(p_old), _p(m_old),
                                                                _p(v_old), _p(p_new), _p(m_new), _p(v_new),
                                                                _stream(stream)))


def o5_linattn_fwd_workspace_bytes(dt, T, B, nh, nkv, dk, dv):
    return lib().o5_linattn_fwd_workspace_bytes(dt, T, B, nh, nkv, dk, dv)


def o5_linattn_fwd(dt, T, B, nh, nkv, dk, dv, q, ldq, k, ldk, v, ldv, decay, scale, S0, reset, o, ldo, ST, ws,
                   stream=None):
    wp, wn = _ws(ws)
    _check("o5_linattn_fwd", lib().o5_linattn_fwd(
        dt, T, B, nh, nkv, dk, dv, _p(q), ldq, _p(k), ldk, _p(v), ldv, _p(decay), float(scale), _p(S0), _p(reset),
        _p(o), ldo, _p(ST), wp, wn, _stream(stream)))


def o5_linattn_bwd_workspace_bytes(dt, T, B, nh, nkv, dk, dv):
    return lib().o5_linattn_bwd_workspace_bytes(dt, T, B, nh, nkv, dk, dv)


def o5_linattn_bwd(dt, T, B, nh, nkv, dk, dv, q, ldq, k, ldk, v, ldv, decay, scale, S0, reset, dout, lddo, dST,
                   dq, lddq, dkey, lddk, dval, lddv, dS0, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_linattn_bwd", lib().o5_linattn_bwd(
        dt, T, B, nh, nkv, dk, dv, _p(q), ldq, _p(k), ldk, _p(v), ldv, _p(decay), float(scale), _p(S0), _p(reset),
        _p(dout), lddo, _p(dST), _p(dq), lddq, _p(dkey), lddk, _p(dval), lddv, _p(dS0), wp, wn, _stream(stream)))


def o5_linattn_step(dt, B, nh, nkv, dk, dv, q, ldq, k, ldk, v, ldv, decay, scale, reset, S, o, ldo, stream=None):
    _check("o5_linattn_step", lib().o5_linattn_step(
        dt, B, nh, nkv, dk, dv, _p(q), ldq, _p(k), ldk, _p(v), ldv, _p(decay), float(scale), _p(reset), _p(S),
        _p(o), ldo, _stream(stream)))


def o5_gatedrec_marks_bytes(T, B, D):
    return lib().o5_gatedrec_marks_bytes(T, B, D)


def o5_gatedrec_fwd_workspace_bytes(dt, T, B, D):
    return lib().o5_gatedrec_fwd_workspace_bytes(dt, T, B, D)


def o5_gatedrec_fwd(dt, T, B, D, x, ldx, r, ldr, i, ldi, lam, c, h0, reset, h, ldh, hT, marks, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_gatedrec_fwd", lib().o5_gatedrec_fwd(
        dt, T, B, D, _p(x), ldx, _p(r), ldr, _p(i), ldi, _p(lam), float(c), _p(h0), _p(reset), _p(h), ldh, _p(hT),
        _p(marks), wp, wn, _stream(stream)))


def o5_gatedrec_bwd_workspace_bytes(dt, T, B, D):
    return lib().o5_gatedrec_bwd_workspace_bytes(dt, T, B, D)


def o5_gatedrec_bwd(dt, T, B, D, x, ldx, r, ldr, i, ldi, lam, c, marks, reset, dh, lddh, dhT, dx, lddx, dr, lddr, di, lddi,
                    dlam, dh0, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_gatedrec_bwd", lib().o5_gatedrec_bwd(
        dt, T, B, D, _p(x), ldx, _p(r), ldr, _p(i), ldi, _p(lam), float(c), _p(marks), _p(reset), _p(dh), lddh, _p(dhT),
        _p(dx), lddx, _p(dr), lddr, _p(di), lddi, _p(dlam), _p(dh0), wp, wn, _stream(stream)))


def o5_gatedrec_step(dt, B, D, x, ldx, r, ldr, i, ldi, lam, c, reset, S, h, ldh, stream=None):
    _check("o5_gatedrec_step", lib().o5_gatedrec_step(
        dt, B, D, _p(x), ldx, _p(r), ldr, _p(i), ldi, _p(lam), float(c), _p(reset), _p(S), _p(h), ldh, _stream(stream)))


def o5_resnorm_fwd(xt, dt, N, D, x, u, gate, ldg, w_post, rho, w_pre, eps, xo, n, r_post, r_pre, stream=None):
    _check("o5_resnorm_fwd", lib().o5_resnorm_fwd(
        xt, dt, N, D, _p(x), _p(u), _p(gate), ldg, _p(w_post), _p(rho), _p(w_pre), float(eps), _p(xo), _p(n),
        _p(r_post), _p(r_pre), _stream(stream)))


def o5_resnorm_bwd_workspace_bytes(xt, dt, N, D):
    return lib().o5_resnorm_bwd_workspace_bytes(xt, dt, N, D)


def o5_resnorm_bwd(xt, dt, N, D, xo, u, gate, ldg, w_post, rho, w_pre, r_post, r_pre, dxo, dn, dx, du, dgate, lddg,
                   dw_post, drho, dw_pre, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_resnorm_bwd", lib().o5_resnorm_bwd(
        xt, dt, N, D, _p(xo), _p(u), _p(gate), ldg, _p(w_post), _p(rho), _p(w_pre), _p(r_post), _p(r_pre), _p(dxo),
        _p(dn), _p(dx), _p(du), _p(dgate), lddg, _p(dw_post), _p(drho), _p(dw_pre), wp, wn, _stream(stream)))


def _tensors(tensors):
    return (AdamwTensor * len(tensors))(*tensors)


def o5_adamw_plan_bytes(tensors):
    return lib().o5_adamw_plan_bytes(len(tensors), _tensors(tensors))


def o5_adamw_plan(tensors, plan):
    """Write the plan of a list of adamw_tensor()s into `plan`, a CPU tensor of bytes."""
    _check("o5_adamw_plan", lib().o5_adamw_plan(len(tensors), _tensors(tensors), _p(plan), plan.numel()))


def o5_adamw_step(plan, plan_dev, lr, beta1, beta2, eps, clip_k, seed, step, stream=None):
    hp = AdamHp(lr, beta1, beta2, eps, clip_k)
    _check("o5_adamw_step", lib().o5_adamw_step(_p(plan), _p(plan_dev), hp, int(seed), int(step), _stream(stream)))


def o5_adamw_moments(plan, plan_dev, m, v, stream=None):
    _check("o5_adamw_moments", lib().o5_adamw_moments(_p(plan), _p(plan_dev), _p(m), _p(v), _stream(stream)))


def o5_adamw_grad_norm_workspace_bytes(plan):
    return lib().o5_adamw_grad_norm_workspace_bytes(_p(plan))


def o5_adamw_grad_norm(plan, plan_dev, max_norm, clip, ws, stream=None):
    wp, wn = _ws(ws)
    _check("o5_adamw_grad_norm", lib().o5_adamw_grad_norm(_p(plan), _p(plan_dev), float(max_norm), _p(clip), wp, wn,
                                                          _stream(stream)))


def o5_adamw_step_clipped(plan, plan_dev, lr, beta1, beta2, eps, clip_k, clip, seed, step, stream=None):
    hp = AdamHp(lr, beta1, beta2, eps, clip_k)
    _check("o5_adamw_step_clipped", lib().o5_adamw_step_clipped(_p(plan), _p(plan_dev), hp, _p(clip), int(seed), int(step),
                                                                _stream(stream)))


def o5_f32_to_bf16(n, src, dst, stream=None):
    _check("o5_f32_to_bf16", lib().o5_f32_to_bf16(n, _p(src), _p(dst), _stream(stream)))


def o5_ktimer_enable(on):
    _check("o5_ktimer_enable", lib().o5_ktimer_enable(1 if on else 0))


def o5_ktimer_enable_sites(names):
    """Record only the named sites (an empty list stops recording)."""
    mask = 0
    for nm in names:
        mask |= 1 << KTIMER_SITES.index(nm)
    _check("o5_ktimer_enable_sites", lib().o5_ktimer_enable_sites(mask))


def o5_ktimer_read(site):
    """(total device milliseconds, launches) recorded for one site."""
    t = ctypes.c_double(0.0)
    n = ctypes.c_int(0)
    _check("o5_ktimer_read", lib().o5_ktimer_read(int(site), ctypes.byref(t), ctypes.byref(n)))
    return t.value, n.value


def o5_ktimer_site_name(site):
    return lib().o5_ktimer_site_name(int(site)).decode()
