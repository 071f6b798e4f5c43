// Host-side checks of the gated recurrence, the loss on logits and the
// gradients' norm, built with AddressSanitizer and UndefinedBehaviorSanitizer on
// the host code of their source files.  Every call below fails validation, or is
// a size query, so no GPU is needed.  Exit status 0 and the last line
// "abi_training_check: all N checks passed" mean that every check held and the
// sanitizers reported nothing (they abort the process on a report).
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "o5.h"

static int g_checks = 0, g_fail = 0;

#define EXPECT(cond)                                                                                             \
  do {                                                                                                           \
    ++g_checks;                                                                                                  \
    if (!(cond)) {                                                                                               \
      ++g_fail;                                                                                                  \
      std::fprintf(stderr, "FAILED %s:%d: %s (last error: %s)\n", __FILE__, __LINE__, #cond, o5_last_error());   \
    }                                                                                                            \
  } while (0)

// A fake, 16-byte aligned device address: never dereferenced.
static void* P(uintptr_t a = 16) { return reinterpret_cast<void*>(a); }
static float* F(uintptr_t a = 16) { return static_cast<float*>(P(a)); }
static uint8_t* U8(uintptr_t a = 16) { return static_cast<uint8_t*>(P(a)); }
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

static void check_logits() {
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

static void check_norm() {
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
  check_gatedrec();
  check_logits();
  check_norm();
  if (g_fail) {
    std::printf("abi_training_check: %d of %d checks failed\n", g_fail, g_checks);
    return 1;
  }
  std::printf("abi_training_check: all %d checks passed\n", g_checks);
  return 0;
}
