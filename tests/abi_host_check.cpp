// Host-side checks of the C ABI, built with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host code of every source file (device
// code is not built: nothing here reaches a launch).  Every call below fails
// validation, or is a size query, so no GPU is needed.  Exit status 0 and the
// last line "abi_host_check: all N checks passed" mean that every check held
// and the sanitizers reported nothing (they abort the process on a report).
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "o5.h"

static int g_checks = 0, g_fail = 0;

#define EXPECT(cond)                                                          \
  do {                                                                        \
    ++g_checks;                                                               \
    if (!(cond)) {                                                            \
      ++g_fail;                                                               \
      std::fprintf(stderr, "FAILED %s:%d: %s (last error: %s)\n", __FILE__,    \
                   __LINE__, #cond, o5_last_error());                         \
    }                                                                         \
  } while (0)

// A fake, 16-byte aligned device address: never dereferenced, since every
// call that receives it is rejected before any launch.
static void* P(uintptr_t a = 16) { return reinterpret_cast<void*>(a); }
static float* F(uintptr_t a = 16) { return static_cast<float*>(P(a)); }
static uint8_t* U8(uintptr_t a = 16) { return static_cast<uint8_t*>(P(a)); }

static void check_strings() {
  EXPECT(o5_version() == 100);
  for (int c = -3; c < 12; ++c) EXPECT(o5_status_str(c) != nullptr && std::strlen(o5_status_str(c)) > 0);
  EXPECT(std::strncmp(o5_status_str(0), "O5_OK", 5) == 0);
  EXPECT(o5_last_error() != nullptr);
  for (int s = -2; s < 40; ++s) EXPECT(o5_ktimer_site_name(s) != nullptr);
  double ms = 0.0;
  int n = 0;
  EXPECT(o5_ktimer_read(-1, &ms, &n) != O5_OK);
  EXPECT(o5_ktimer_read(1 << 20, &ms, &n) != O5_OK);
  EXPECT(o5_ktimer_enable(0) == O5_OK);
  EXPECT(o5_ktimer_enable_sites(0) == O5_OK);
}

static void check_gae() {
  EXPECT(o5_gae(16, 8, nullptr, nullptr, nullptr, 0.99f, 0.95f, nullptr, nullptr, nullptr) == O5_E_NULL);
  EXPECT(o5_gae(0, 8, F(), F(), U8(), 0.99f, 0.95f, F(), F(), nullptr) == O5_E_SHAPE);
  EXPECT(o5_gae(-5, 8, F(), F(), U8(), 0.99f, 0.95f, F(), F(), nullptr) == O5_E_SHAPE);
  EXPECT(o5_gae(INT_MAX, INT_MAX, F(), F(), U8(), 0.99f, 0.95f, F(), F(), nullptr) == O5_E_SHAPE);
  EXPECT(o5_gae(16, 8, F(0x1001), F(), U8(), 0.99f, 0.95f, F(), F(), nullptr) == O5_E_ALIGN);
  EXPECT(o5_gae(16, 8, F(), F(), U8(), 1.5f, 0.95f, F(), F(), nullptr) == O5_E_ARG);
  EXPECT(o5_gae(16, 8, F(), F(), U8(), 0.99f, -0.1f, F(), F(), nullptr) == O5_E_ARG);
  EXPECT(o5_segments_to_samples(10, 2, 3, F(), F(), U8(), F(), F(), U8(), nullptr) == O5_E_SHAPE);
  EXPECT(o5_segments_to_samples(INT_MAX, INT_MAX, 16, F(), F(), U8(), F(), F(), U8(), nullptr) == O5_E_SHAPE);
  EXPECT(o5_segments_to_samples(16, 8, 16, nullptr, F(), U8(), F(), F(), U8(), nullptr) == O5_E_NULL);
}

static void check_lstm() {
  for (int dt = 0; dt < 2; ++dt) {
    const o5_dtype d = static_cast<o5_dtype>(dt);
    const size_t need = o5_lstm_fwd_workspace_bytes(d, 16, 8, 64, 128);
    EXPECT(need > 0);
    EXPECT(o5_lstm_fwd(d, 16, 8, 64, 128, P(), P(), P(), F(), F(), F(), U8(), P(), F(), P(), P(), need - 1,
                       nullptr) == O5_E_WORKSPACE);
    EXPECT(o5_lstm_fwd(d, 16, 8, 64, 128, P(), P(), P(), F(), F(), F(), U8(), P(), F(), P(), nullptr, need,
                       nullptr) == O5_E_WORKSPACE);
    EXPECT(o5_lstm_fwd(d, 1, 1, 60, 64, P(), P(), P(), F(), F(), F(), U8(), P(), F(), P(), P(), 1 << 20,
                       nullptr) == O5_E_SHAPE);
    EXPECT(o5_lstm_fwd(d, 16, 8, 64, 128, nullptr, P(), P(), F(), F(), F(), U8(), P(), F(), P(), P(), need,
                       nullptr) == O5_E_NULL);
    EXPECT(o5_lstm_fwd(d, 16, 8, 64, 128, P(0x1002), P(), P(), F(), F(), F(), U8(), P(), F(), P(), P(), need,
                       nullptr) == O5_E_ALIGN);
    const size_t bneed = o5_lstm_bptt_workspace_bytes(d, 16, 8, 64, 128);
    EXPECT(bneed > 0);
    EXPECT(o5_lstm_bptt(d, 16, 8, 64, 128, P(), P(), P(), F(), F(), U8(), P(), F(), nullptr, F(), F(), F(), F(), F(),
                        F(), nullptr, P(), bneed, nullptr) == O5_E_NULL);
    EXPECT(o5_lstm_bptt(d, 16, 8, 64, 128, P(), P(), P(), F(), F(), U8(), P(), F(), P(), F(), F(), F(), F(), F(), F(),
                        nullptr, P(), bneed - 1, nullptr) == O5_E_WORKSPACE);
    // extreme sizes: the queries reject them (0) without overflowing
    const int big[] = {0, -1, 1, 63, 64, 65536, 1 << 20, INT_MAX};
    for (int T : {1, 16, INT_MAX})
      for (int B : big)
        for (int H : big) {
          (void)o5_lstm_fwd_workspace_bytes(d, T, B, H, H);
          (void)o5_lstm_bptt_workspace_bytes(d, T, B, H, H);
          (void)o5_prelstm_bwd_workspace_bytes(d, T, B, H, H);
          ++g_checks;
        }
  }
  EXPECT(o5_lstm_fwd(static_cast<o5_dtype>(9), 1, 1, 64, 64, P(), P(), P(), F(), F(), F(), U8(), P(), F(), P(), P(),
                     1 << 20, nullptr) == O5_E_DTYPE);
  EXPECT(o5_lstm_fwd_workspace_bytes(static_cast<o5_dtype>(9), 16, 8, 64, 128) == 0);
}

static void check_heads_and_sampler() {
  const int heads[4] = {30, 8, 32, 4};
  const int bad[2] = {3, 0};
  const o5_ppo_hp hp{0.2f, 1.0f, 0.01f};
  for (int dt = 0; dt < 2; ++dt) {
    const o5_dtype d = static_cast<o5_dtype>(dt);
    EXPECT(o5_ppo_loss_grad_workspace_bytes(d, 8, 64, 2, bad, nullptr) == 0);
    EXPECT(std::strstr(o5_last_error(), "head_sizes[1]") != nullptr);
    EXPECT(o5_ppo_loss_grad_workspace_bytes(d, 8, 64, 4, nullptr, nullptr) == 0);
    EXPECT(o5_ppo_loss_grad_workspace_bytes(d, 8, 64, 0, heads, nullptr) == 0);
    EXPECT(o5_ppo_loss_grad_workspace_bytes(d, 8, 64, 99, heads, nullptr) == 0);
    const size_t need = o5_ppo_loss_grad_workspace_bytes(d, 2048, 4096, 4, heads, nullptr);
    EXPECT(need > 0);
    EXPECT(o5_ppo_loss_grad(d, 2048, 4096, 4, heads, P(), P(), F(), static_cast<int32_t*>(P()), F(), F(), F(), U8(),
                            nullptr, nullptr, hp, F(), F(), F(), F(), P(), need - 1, nullptr) == O5_E_WORKSPACE);
    EXPECT(o5_ppo_loss_grad(d, 2048, 4096, 4, heads, P(), P(), F(), static_cast<int32_t*>(P()), F(), F(), F(), U8(),
                            nullptr, nullptr, o5_ppo_hp{1.0f, 1.0f, 0.01f}, F(), F(), F(), F(), P(), need,
                            nullptr) == O5_E_ARG);
    EXPECT(o5_ppo_loss_grad(d, 2048, 4096, 4, heads, nullptr, P(), F(), static_cast<int32_t*>(P()), F(), F(), F(),
                            U8(), nullptr, nullptr, hp, F(), F(), F(), F(), P(), need, nullptr) == O5_E_NULL);
    // a unit head with d not a power of two, or pointing at a missing head
    o5_unit_head u{1, 100, P(), F(), P(), F(), F()};
    EXPECT(o5_ppo_loss_grad_workspace_bytes(d, 64, 64, 4, heads, &u) == 0);
    u.d = 128;
    u.head = 7;
    EXPECT(o5_ppo_loss_grad_workspace_bytes(d, 64, 64, 4, heads, &u) == 0);
    u.head = 1;
    EXPECT(o5_ppo_loss_grad_workspace_bytes(d, 32768, 4096, 4, heads, &u) > need);
    const size_t sneed = o5_policy_sample_workspace_bytes(d, 4096, 4096, 4, heads, nullptr);
    EXPECT(sneed > 0);
    EXPECT(o5_policy_sample(d, 4096, 4096, 4, heads, P(), P(), F(), U8(), nullptr, 1, 0, static_cast<int32_t*>(P()),
                            F(), F(), P(), sneed - 1, nullptr) == O5_E_WORKSPACE);
    EXPECT(o5_policy_sample(d, 4096, 4096, 4, heads, nullptr, P(), F(), U8(), nullptr, 1, 0,
                            static_cast<int32_t*>(P()), F(), F(), P(), sneed, nullptr) == O5_E_NULL);
    // the static-scratch sampler rejects before it touches a device
    EXPECT(o5_policy_sample_static(d, 1 << 20, 4096, 4, heads, P(), P(), F(), U8(), nullptr, 1, 0,
                                   static_cast<int32_t*>(P()), F(), F(), nullptr) == O5_E_SHAPE);
    EXPECT(o5_policy_sample_static(d, 64, 4096, 4, heads, nullptr, P(), F(), U8(), nullptr, 1, 0,
                                   static_cast<int32_t*>(P()), F(), F(), nullptr) == O5_E_NULL);
    const int big[] = {0, -1, 1, 64, 65536, 1 << 24, INT_MAX};
    for (int N : big)
      for (int H : big) {
        (void)o5_ppo_loss_grad_workspace_bytes(d, N, H, 4, heads, nullptr);
        (void)o5_ppo_loss_grad_workspace_bytes(d, N, H, 4, heads, &u);
        (void)o5_policy_sample_workspace_bytes(d, N, H, 4, heads, nullptr);
        (void)o5_policy_sample_workspace_bytes(d, N, H, 4, heads, &u);
        ++g_checks;
      }
  }
  // the factored loss and backward calls: bf16 only, ld as the heads need
  {
    const o5_ppo_hp hp{0.2f, 1.0f, 0.01f};
    const int ld = o5_ppo_head_grad_ld(4096, 4, heads, nullptr);
    EXPECT(ld == 256);
    o5_unit_head u{1, 128, P(), F(), P(), F(), F()};
    EXPECT(o5_ppo_head_grad_ld(4096, 4, heads, &u) == 512);
    EXPECT(o5_ppo_head_grad_ld(4096, 4, nullptr, nullptr) == 0);
    EXPECT(o5_ppo_head_grad_ld(-1, 4, heads, nullptr) == 0);
    const size_t need = o5_ppo_loss_grad_workspace_bytes(O5_BF16, 2048, 4096, 4, heads, nullptr);
    uint16_t* p16 = static_cast<uint16_t*>(P());
    EXPECT(o5_ppo_loss_grad_factored(O5_F32, 2048, 4096, 4, heads, P(), P(), F(), static_cast<int32_t*>(P()), F(),
                                     F(), F(), U8(), nullptr, nullptr, hp, F(), p16, p16, ld, F(), F(), P(), need,
                                     nullptr) == O5_E_DTYPE);
    EXPECT(o5_ppo_loss_grad_factored(O5_BF16, 2048, 4096, 4, heads, P(), P(), F(), static_cast<int32_t*>(P()), F(),
                                     F(), F(), U8(), nullptr, nullptr, hp, F(), p16, p16, ld + 64, F(), F(), P(), need,
                                     nullptr) == O5_E_SHAPE);
    EXPECT(o5_ppo_loss_grad_factored(O5_BF16, 2048, 4096, 4, heads, P(), P(), F(), static_cast<int32_t*>(P()), F(),
                                     F(), F(), U8(), nullptr, nullptr, hp, F(), nullptr, p16, ld, F(), F(), P(), need,
                                     nullptr) == O5_E_NULL);
    const size_t bneed = o5_lstm_bptt_workspace_bytes(O5_BF16, 16, 8, 64, 128);
    EXPECT(o5_lstm_bptt_factored(O5_F32, 16, 8, 64, 128, P(), P(), P(), F(), F(), U8(), P(), F(), P(), p16, p16, 256,
                                 nullptr, nullptr, F(), F(), F(), nullptr, P(), bneed, nullptr) == O5_E_DTYPE);
    EXPECT(o5_lstm_bptt_factored(O5_BF16, 16, 8, 64, 128, P(), P(), P(), F(), F(), U8(), P(), F(), P(), p16, p16, 100,
                                 nullptr, nullptr, F(), F(), F(), nullptr, P(), bneed, nullptr) == O5_E_SHAPE);
    EXPECT(o5_lstm_bptt_factored(O5_BF16, 16, 8, 64, 128, P(), P(), P(), F(), F(), U8(), P(), F(), P(), p16, p16, 256,
                                 nullptr, nullptr, F(), F(), F(), nullptr, P(), bneed - 1, nullptr) == O5_E_WORKSPACE);
    EXPECT(o5_lstm_bptt_factored(O5_BF16, 16, 8, 64, 128, P(), P(), P(), F(), F(), U8(), P(), F(), P(), nullptr, p16,
                                 256, nullptr, nullptr, F(), F(), F(), nullptr, P(), bneed, nullptr) == O5_E_NULL);
  }
  // many large heads: the total is capped
  int wide[8];
  for (int& w : wide) w = INT_MAX / 4;
  EXPECT(o5_ppo_loss_grad_workspace_bytes(O5_BF16, 64, 64, 8, wide, nullptr) == 0);
}

static void check_adam_surgery_misc() {
  const o5_adam_hp hp{1e-3f, 0.9f, 0.999f, 1e-8f, 5.0f};
  EXPECT(o5_adam_step(10, F(), F(), F(), F(), nullptr, hp, 0, nullptr) == O5_E_ARG);
  EXPECT(o5_adam_step(10, nullptr, F(), F(), F(), nullptr, hp, 1, nullptr) == O5_E_NULL);
  EXPECT(o5_adam_step(10, F(0x1004), F(), F(), F(), nullptr, hp, 1, nullptr) == O5_E_ALIGN);
  EXPECT(o5_adam_step(10, F(), F(), F(), F(), nullptr, o5_adam_hp{1e-3f, 1.0f, 0.999f, 1e-8f, 5.0f}, 1, nullptr) ==
         O5_E_ARG);
  EXPECT(o5_f32_to_bf16(10, nullptr, static_cast<uint16_t*>(P()), nullptr) == O5_E_NULL);
  EXPECT(o5_param_count(4096, 4096, 75) == 134541387u);
  (void)o5_param_count(INT_MAX, INT_MAX, INT_MAX);
  (void)o5_param_count(-1, -1, -1);
  EXPECT(o5_surgery_widen(64, 64, 9, 32, 64, F(), nullptr, nullptr, F(), F(), F(), 0.01f, 1, nullptr) ==
         O5_E_SHAPE);
  EXPECT(o5_surgery_widen(64, 64, 9, 64, 128, F(), nullptr, nullptr, F(), F(), F(), -1.0f, 1, nullptr) == O5_E_ARG);
  EXPECT(o5_surgery_widen(64, 64, 9, 64, 128, nullptr, nullptr, nullptr, F(), F(), F(), 0.01f, 1, nullptr) ==
         O5_E_NULL);
  EXPECT(o5_surgery_widen(INT_MAX, INT_MAX, INT_MAX, INT_MAX, INT_MAX, F(), nullptr, nullptr, F(), F(), F(), 0.01f, 1,
                          nullptr) != O5_OK);
  EXPECT(o5_surgery_fold_input(64, 64, 9, 64, F(), F(), nullptr, nullptr, F(), F(), F(), nullptr) == O5_E_SHAPE);
  const o5_reward_hp rhp{0.3f, 0.6f, 10.0f, 1e-8f};
  EXPECT(o5_reward_process(0, 4, F(), nullptr, F(), rhp, static_cast<double*>(P()), F(), P(), 1 << 20, nullptr) ==
         O5_E_SHAPE);
  EXPECT(o5_reward_process(4, 4, F(), nullptr, nullptr, rhp, static_cast<double*>(P()), F(), P(), 1 << 20,
                           nullptr) == O5_E_NULL);
  EXPECT(o5_reward_process(4, 4, F(), nullptr, F(), o5_reward_hp{1.5f, 0.6f, 10.0f, 1e-8f}, static_cast<double*>(P()),
                           F(), P(), 1 << 20, nullptr) == O5_E_ARG);
  const size_t rneed = o5_reward_process_workspace_bytes(4, 4);
  EXPECT(rneed > 0);
  EXPECT(o5_reward_process(4, 4, F(), nullptr, F(), rhp, static_cast<double*>(P()), F(), P(), rneed - 1, nullptr) ==
         O5_E_WORKSPACE);
  EXPECT(o5_reward_process_workspace_bytes(0, 1) == 0);
  (void)o5_reward_process_workspace_bytes(INT_MAX, INT_MAX);
  EXPECT(o5_obs_normalize(O5_BF16, 0, 64, F(), static_cast<double*>(P()), 5.0f, 1e-8f, P(), P(), 1 << 20, nullptr) ==
         O5_E_SHAPE);
  EXPECT(o5_obs_normalize(O5_BF16, 10, 64, F(), static_cast<double*>(P()), 0.0f, 1e-8f, P(), P(), 1 << 20, nullptr) ==
         O5_E_ARG);
  (void)o5_obs_normalize_workspace_bytes(INT_MAX, INT_MAX);
  EXPECT(o5_prelstm_fwd(O5_BF16, 2, 7, 64, 64, P(), P(), F(), F(), P(), nullptr) == O5_E_SHAPE);
  EXPECT(o5_prelstm_fwd(O5_BF16, 2, 10, 64, 96, P(), P(), F(), F(), P(), nullptr) == O5_E_SHAPE);
  EXPECT(o5_prelstm_fwd(static_cast<o5_dtype>(5), 2, 10, 64, 64, P(), P(), F(), F(), P(), nullptr) == O5_E_DTYPE);
  EXPECT(o5_prelstm_bwd(O5_BF16, 2, 10, 64, 64, P(), F(), P(), F(), F(), nullptr, 0, nullptr) == O5_E_WORKSPACE);
}

// The parallel recurrent core: linear attention, the norms around a block, AdamW over many tensors.
static void check_linattn() {
  for (int dt = 0; dt < 2; ++dt) {
    const o5_dtype d = static_cast<o5_dtype>(dt);
    const size_t need = o5_linattn_fwd_workspace_bytes(d, 1000, 2, 8, 4, 64, 128);
    const size_t bneed = o5_linattn_bwd_workspace_bytes(d, 1000, 2, 8, 4, 64, 128);
    EXPECT(need > 256 && bneed >= need);
    const auto fwd = [&](int T, int nh, const void* q, size_t ldq, float scale, const float* S0, void* o, void* ws, size_t n) {
      return o5_linattn_fwd(d, T, 2, nh, 4, 64, 128, q, ldq, P(), 256, P(), 512, F(), scale, S0, U8(), o, 1024, F(), ws, n, nullptr);
    };
    EXPECT(fwd(0, 8, P(), 512, 1.0f, F(), P(), P(), need) == O5_E_SHAPE);
    EXPECT(fwd(INT_MAX, 8, P(), 512, 1.0f, F(), P(), P(), need) == O5_E_SHAPE);
    EXPECT(fwd(1000, 6, P(), 512, 1.0f, F(), P(), P(), need) == O5_E_SHAPE);
    EXPECT(fwd(1000, 8, P(), 504, 1.0f, F(), P(), P(), need) == O5_E_SHAPE);
    EXPECT(fwd(1000, 8, P(), SIZE_MAX - 7, 1.0f, F(), P(), P(), need) == O5_E_SHAPE);
    EXPECT(fwd(1000, 8, nullptr, 512, 1.0f, F(), P(), P(), need) == O5_E_NULL);
    EXPECT(fwd(1000, 8, P(0x1002), 512, 1.0f, F(), P(), P(), need) == O5_E_ALIGN);
    EXPECT(fwd(1000, 8, P(), 512, INFINITY, F(), P(), P(), need) == O5_E_ARG);
    EXPECT(fwd(1000, 8, P(), 512, 1.0f, F(0x1004), P(), P(), need) == O5_E_ALIGN);
    EXPECT(fwd(1000, 8, P(), 512, 1.0f, nullptr, nullptr, P(), need) == O5_E_NULL);
    EXPECT(fwd(1000, 8, P(), 512, 1.0f, nullptr, P(), nullptr, need) == O5_E_WORKSPACE);
    EXPECT(fwd(1000, 8, P(), 512, 1.0f, nullptr, P(), P(), need - 1) == O5_E_WORKSPACE);
    const auto bwd = [&](const void* dout, size_t lddq, void* dk, const float* dST, size_t n) {
      return o5_linattn_bwd(d, 1000, 2, 8, 4, 64, 128, P(), 512, P(), 256, P(), 512, F(), 1.0f, nullptr, nullptr, dout, 1024, dST,
                            P(), lddq, dk, 256, P(), 512, F(), P(), n, nullptr);
    };
    EXPECT(bwd(nullptr, 512, P(), F(), bneed) == O5_E_NULL);
    EXPECT(bwd(P(), 510, P(), F(), bneed) == O5_E_SHAPE);
    EXPECT(bwd(P(), 512, nullptr, F(), bneed) == O5_E_NULL);
    EXPECT(bwd(P(), 512, P(), F(0x1008), bneed) == O5_E_ALIGN);
    EXPECT(bwd(P(), 512, P(), nullptr, bneed - 1) == O5_E_WORKSPACE);
    EXPECT(o5_linattn_step(d, 2, 8, 4, 64, 128, P(), 512, P(), 256, P(), 512, F(), 1.0f, nullptr, nullptr, P(), 1024, nullptr) ==
           O5_E_NULL);
    EXPECT(o5_linattn_step(d, -2, 8, 4, 64, 128, P(), 512, P(), 256, P(), 512, F(), 1.0f, nullptr, F(), P(), 1024, nullptr) ==
           O5_E_SHAPE);
    const int big[] = {INT_MIN, -1, 0, 1, 8, 128, 136, 65536, (1 << 24) - 1, 1 << 30, INT_MAX};
    for (int T : big)
      for (int B : big)
        for (int nh : big)
          for (int nkv : {-1, 0, 1, 8, INT_MAX}) {
            (void)o5_linattn_fwd_workspace_bytes(d, T, B, nh, nkv, 64, 128);
            (void)o5_linattn_bwd_workspace_bytes(d, T, B, nh, nkv, 8, T);
            ++g_checks;
          }
  }
  EXPECT(o5_linattn_fwd_workspace_bytes(static_cast<o5_dtype>(9), 1, 1, 1, 1, 8, 8) == 0);
}

static void check_resnorm() {
  const o5_dtype t = O5_BF16;
  const auto fwd = [&](o5_dtype dt, int N, int D, const void* u, const void* gate, size_t ldg, const float* w_pre, float eps) {
    return o5_resnorm_fwd(t, dt, N, D, P(), u, gate, ldg, F(), F(), w_pre, eps, P(), P(), nullptr, F(0x1008), nullptr);
  };
  EXPECT(fwd(O5_F32, 4, 64, P(), P(), 64, F(), 1e-6f) == O5_E_DTYPE);
  EXPECT(fwd(t, 0, 64, P(), P(), 64, F(), 1e-6f) == O5_E_SHAPE);
  EXPECT(fwd(t, INT_MAX, INT_MAX, P(), P(), 64, F(), 1e-6f) == O5_E_SHAPE);
  EXPECT(fwd(t, 4, 64, P(), P(), 60, F(), 1e-6f) == O5_E_SHAPE);
  EXPECT(fwd(t, 4, 64, P(), P(), SIZE_MAX - 7, F(), 1e-6f) == O5_E_SHAPE);
  EXPECT(fwd(t, 4, 64, nullptr, P(), 64, F(), 1e-6f) == O5_E_ARG);
  EXPECT(fwd(t, 4, 64, nullptr, nullptr, 0, nullptr, 1e-6f) == O5_E_ARG);
  EXPECT(fwd(t, 4, 64, P(), P(), 64, F(), NAN) == O5_E_ARG);
  EXPECT(fwd(t, 4, 64, P(), P(), 64, F(), 1e-6f) == O5_E_ALIGN);  // (r_pre above)
  const size_t need = o5_resnorm_bwd_workspace_bytes(t, t, 4, 64);
  EXPECT(need > 0);
  const auto bwd = [&](const float* r_post, void* dgate, size_t lddg, void* ws, size_t n) {
    return o5_resnorm_bwd(t, t, 4, 64, P(), P(), P(), 64, F(), F(), F(), r_post, F(), P(), P(), P(), P(), dgate, lddg, F(), F(),
                          F(), ws, n, nullptr);
  };
  EXPECT(bwd(nullptr, P(), 64, P(), need) == O5_E_NULL);
  EXPECT(bwd(F(), nullptr, 64, P(), need) == O5_E_NULL);
  EXPECT(bwd(F(), P(), 56, P(), need) == O5_E_SHAPE);
  EXPECT(bwd(F(), P(), 64, nullptr, need) == O5_E_WORKSPACE);
  EXPECT(bwd(F(), P(), 64, P(), need - 1) == O5_E_WORKSPACE);
  for (int N : {INT_MIN, -1, 0, 1, 1 << 20, (1 << 30) - 1, 1 << 30, INT_MAX})
    for (int D : {INT_MIN, -8, 0, 4, 8, 8192, 8200, INT_MAX}) {
      (void)o5_resnorm_bwd_workspace_bytes(O5_F32, t, N, D);
      ++g_checks;
    }
}

static void check_adamw() {
  const auto tensor = [](size_t n, int bits) {
    return o5_adamw_tensor{n, F(), P(), P(), P(), U8(), U8(), nullptr, 1.0f, 0.0f, O5_F32, bits};
  };
  EXPECT(o5_adamw_plan_bytes(1, nullptr) == 0);
  EXPECT(o5_adamw_plan_bytes(-1, nullptr) == 0);
  // plans in heap buffers of exactly their size, with whole and partial chunks: a byte past the end is reported
  for (size_t n : {size_t{1}, size_t{1023}, size_t{1024}, size_t{1025}, size_t{1000003}})
    for (int count : {1, 3, 100}) {
      o5_adamw_tensor* t = new o5_adamw_tensor[count];
      for (int i = 0; i < count; ++i) t[i] = tensor(n + i, i % 2 ? 8 : 32);
      const size_t bytes = o5_adamw_plan_bytes(count, t);
      EXPECT(bytes > 0);
      char* plan = new char[bytes];
      EXPECT(o5_adamw_plan(count, t, plan, bytes) == O5_OK);
      EXPECT(o5_adamw_plan(count, t, plan, bytes - 1) == O5_E_WORKSPACE);
      EXPECT(o5_adamw_plan(count, t, plan + 1, bytes) == O5_E_ALIGN);
      const o5_adam_hp hp{1e-3f, 0.9f, 0.999f, 1e-8f, 5.0f};
      EXPECT(o5_adamw_step(plan, nullptr, hp, 1, 1, nullptr) == O5_E_NULL);
      EXPECT(o5_adamw_step(plan, P(), hp, 1, 0, nullptr) == O5_E_ARG);
      EXPECT(o5_adamw_step(plan, P(), o5_adam_hp{NAN, 0.9f, 0.999f, 1e-8f, 5.0f}, 1, 1, nullptr) == O5_E_ARG);
      EXPECT(o5_adamw_moments(plan, P(), nullptr, F(), nullptr) == O5_E_NULL);
      std::memset(plan, 0, 16);
      EXPECT(o5_adamw_step(plan, P(), hp, 1, 1, nullptr) == O5_E_ARG);
      EXPECT(o5_adamw_moments(plan, P(), F(), F(), nullptr) == O5_E_ARG);
      delete[] plan;
      delete[] t;
    }
  o5_adamw_tensor bad[4] = {tensor(0, 32), tensor(SIZE_MAX, 32), tensor(10, 16), tensor(10, 8)};
  bad[3].v_exp = nullptr;
  for (const o5_adamw_tensor& b : bad) {
    char plan[64];
    EXPECT(o5_adamw_plan_bytes(1, &b) == 0);
    EXPECT(o5_adamw_plan(1, &b, plan, sizeof plan) != O5_OK);
  }
  const o5_adamw_tensor huge[3] = {tensor((size_t{1} << 40) - 1, 8), tensor((size_t{1} << 40) - 1, 8), tensor((size_t{1} << 40) - 1, 8)};
  EXPECT(o5_adamw_plan_bytes(3, huge) == 0);
}

static int32_t* I32(uintptr_t a = 16) { return static_cast<int32_t*>(P(a)); }

static const int kInts[] = {INT_MIN, -1, 0, 1, 7, 8, 15, 64, 256, 1000, 4096, 65536, 65544, 1 << 20, 1 << 29, INT_MAX};

static void check_gatedrec() {
  for (o5_dtype dt : {O5_F32, O5_BF16, O5_DTYPE_MAX_ENUM})
    for (int T : kInts)
      for (int B : kInts)
        for (int D : kInts) {
          const bool ok = dt <= O5_BF16 && T >= 1 && B >= 1 && D >= 8 && D <= 65536 && D % 8 == 0 &&
                          static_cast<long long>(T) * B < (1ll << 30);
          EXPECT((o5_gatedrec_fwd_workspace_bytes(dt, T, B, D) > 0) == ok);
          EXPECT((o5_gatedrec_bwd_workspace_bytes(dt, T, B, D) > 0) == ok);
          if (dt == O5_F32) EXPECT((o5_gatedrec_marks_bytes(T, B, D) > 0) == ok);
          if (!ok) {
            EXPECT(o5_gatedrec_fwd(dt, T, B, D, P(), 65536, P(), 65536, P(), 65536, F(), 8.0f, nullptr, nullptr, P(), 65536, nullptr,
                                   nullptr, P(), SIZE_MAX, nullptr) != O5_OK);
          } else {
            EXPECT(o5_gatedrec_fwd(dt, T, B, D, P(), 65536, P(), 65536, P(), 65536, F(), 8.0f, nullptr, nullptr, P(), 65536, nullptr,
                                   nullptr, P(), o5_gatedrec_fwd_workspace_bytes(dt, T, B, D) - 1, nullptr) == O5_E_WORKSPACE);
            EXPECT(o5_gatedrec_bwd(dt, T, B, D, P(), 65536, P(), 65536, P(), 65536, F(), 8.0f, F(), nullptr, P(), 65536, nullptr, P(),
                                   65536, P(), 65536, P(), 65536, F(), nullptr, P(),
                                   o5_gatedrec_bwd_workspace_bytes(dt, T, B, D) - 1, nullptr) == O5_E_WORKSPACE);
          }
        }
  EXPECT(o5_gatedrec_step(O5_F32, 4, 64, P(), 64, P(), 64, P(), SIZE_MAX, F(), 8.0f, nullptr, F(), P(), 64, nullptr) == O5_E_SHAPE);
  EXPECT(o5_gatedrec_step(O5_F32, 4, 64, P(), 64, P(), 64, P(), 64, F(), NAN, nullptr, F(), P(), 64, nullptr) == O5_E_ARG);
  EXPECT(o5_gatedrec_step(O5_F32, 4, 64, P(), 64, P(), 64, P(), 64, F(), 8.0f, nullptr, nullptr, P(), 64, nullptr) == O5_E_NULL);
}

static void check_ppo_logits() {
  const o5_ppo_hp hp{0.2f, 1.0f, 0.01f};
  for (o5_dtype dt : {O5_F32, O5_BF16, O5_DTYPE_MAX_ENUM})
    for (int N : kInts)
      for (int K : {INT_MIN, -1, 0, 1, 2, 8, 9, INT_MAX})
        for (int n : kInts) {
          int heads[8];
          for (int& h : heads) h = n;
          const bool ok = dt <= O5_BF16 && N >= 1 && N < (1 << 30) && K >= 1 && K <= 8 && n >= 1 &&
                          static_cast<long long>(n) * K <= (1 << 24);
          const size_t bytes = o5_ppo_logits_grad_workspace_bytes(dt, N, K, heads);
          EXPECT((bytes > 0) == ok);
          const int st = o5_ppo_logits_grad(dt, N, K, heads, P(), INT_MAX, P(), INT_MAX, I32(), F(), F(), F(), F(), U8(), U8(), hp,
                                            0.1f, F(), F(), F(), P(), INT_MAX, P(), bytes ? bytes - 1 : SIZE_MAX, nullptr);
          EXPECT(ok ? st == O5_E_WORKSPACE : st != O5_OK);
        }
  const int one[1] = {5};
  EXPECT(o5_ppo_logits_grad_workspace_bytes(O5_F32, 1, 1, nullptr) == 0);
  EXPECT(o5_ppo_logits_grad(O5_F32, 1, 1, one, P(), SIZE_MAX, nullptr, 0, I32(), F(), F(), nullptr, nullptr, nullptr, nullptr, hp, 0.0f,
                            F(), nullptr, nullptr, P(), 5, P(), SIZE_MAX, nullptr) == O5_E_SHAPE);
}

static void check_grad_norm() {
  const o5_adamw_tensor t{5000, F(), P(), P(), P(), nullptr, nullptr, nullptr, 1.0f, 0.0f, O5_F32, 32};
  const size_t bytes = o5_adamw_plan_bytes(1, &t);
  char* plan = new char[bytes];
  EXPECT(o5_adamw_plan(1, &t, plan, bytes) == O5_OK);
  const size_t need = o5_adamw_grad_norm_workspace_bytes(plan);
  EXPECT(need > 0 && o5_adamw_grad_norm_workspace_bytes(nullptr) == 0);
  EXPECT(o5_adamw_grad_norm(plan, P(), 1.0f, F(), P(), need - 1, nullptr) == O5_E_WORKSPACE);
  EXPECT(o5_adamw_grad_norm(plan, P(), NAN, F(), P(), need, nullptr) == O5_E_ARG);
  EXPECT(o5_adamw_grad_norm(plan, nullptr, 1.0f, F(), P(), need, nullptr) == O5_E_NULL);
  const o5_adam_hp hp{1e-3f, 0.9f, 0.999f, 1e-8f, 5.0f};
  EXPECT(o5_adamw_step_clipped(plan, P(), hp, nullptr, 1, 1, nullptr) == O5_E_NULL);
  EXPECT(o5_adamw_step_clipped(plan, P(), hp, F(8), 1, 1, nullptr) == O5_E_ALIGN);
  EXPECT(o5_adamw_step_clipped(plan, P(), hp, F(), 1, 0, nullptr) == O5_E_ARG);
  std::memset(plan, 0, 16);
  EXPECT(o5_adamw_grad_norm(plan, P(), 1.0f, F(), P(), need, nullptr) == O5_E_ARG);
  EXPECT(o5_adamw_grad_norm_workspace_bytes(plan) == 0);
  EXPECT(o5_adamw_step_clipped(plan, P(), hp, F(), 1, 1, nullptr) == O5_E_ARG);
  delete[] plan;
}

int main() {
  check_strings();
  check_gae();
  check_lstm();
  check_heads_and_sampler();
  check_adam_surgery_misc();
  check_linattn();
  check_resnorm();
  check_adamw();
  check_gatedrec();
  check_ppo_logits();
  check_grad_norm();
  if (g_fail) {
    std::printf("abi_host_check: %d of %d checks failed\n", g_fail, g_checks);
    return 1;
  }
  std::printf("abi_host_check: all %d checks passed\n", g_checks);
  return 0;
}
