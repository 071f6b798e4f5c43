// Linear attention with a decay for each head, o5_linattn_*.
//
//   S_t = l (reset_t ? 0 : S_{t-1}) + k_t v_t^T,   o_t = scale S_t^T q_t
//
// Every pass is one recurrence of this kind.  With G_t = dJ/dS_t,
//   G_t = scale q_t do_t^T + l (1 - reset_{t+1}) G_{t+1},
// the gradients are dq_t = scale S_t do_t, dk_t = G_t v_t, dv_t = G_t^T k_t:
// the same recurrence with (query, key, value) = (do, v, k) forward in time
// on S^T, and (v, do, q) on G^T and (k, q, do) on G backward in time.
#include "common.h"

namespace o5 {
namespace {

// One recurrence over T steps of B samples.
struct LinPass {
  const void* q;  // [T, B, .] rows of ldq elements: head n at column n * da
  const void* k;  // head n at n * da
  const void* v;  // head n at n * dc
  void* o;        // head n at n * dc
  size_t ldq, ldk, ldv, ldo;
  const float* decay;      // [nkv]
  const uint8_t* reset;    // [T, B] or NULL
  const float* s0;         // [B, nkv, da, dc], or transposed (s0t), or NULL (= 0)
  float* sT;               // the last state, laid out as s0, or NULL
  int T, B, nkv;
  int gq, gk;              // query heads and key/value heads that share a state (one of them is 1)
  int da, dc;              // rows and columns of the state
  float oscale, kscale;    // on the outputs, on what enters the state
  bool s0t, rev;
};

template <typename E>
__device__ __forceinline__ float ld(const void* p, size_t i) {
  return elem<E>::to_f32(static_cast<const E*>(p)[i]);
}

// A wave takes 64 columns of one state and runs the recurrence step by step,
// a column in each lane's registers.
template <typename E, int DA>
__global__ void __launch_bounds__(64) linattn_steps(LinPass p) {
  __shared__ float kq[2][DA];
  const int nout = p.nkv * p.gq;
  const int b = blockIdx.x / nout, hq = blockIdx.x % nout, n = hq / p.gq;
  const int c = blockIdx.y * 64 + threadIdx.x;
  const bool on = c < p.dc;
  const float lam = p.decay[n];
  float S[DA];
  const size_t sbase = (static_cast<size_t>(b) * p.nkv + n) * p.da * p.dc;
  const size_t sa = p.s0t ? 1 : p.dc, sc = p.s0t ? p.da : 1;
#pragma unroll
  for (int a = 0; a < DA; ++a) S[a] = (on && a < p.da && p.s0) ? p.s0[sbase + a * sa + c * sc] : 0.0f;
  for (int u = 0; u < p.T; ++u) {
    const int t = p.rev ? p.T - 1 - u : u;
    const size_t row = static_cast<size_t>(t) * p.B + b;
    bool cut = false;
    if (p.reset) cut = p.rev ? (u > 0 && p.reset[row + p.B] != 0) : p.reset[row] != 0;
    if (!(p.rev && u == 0)) {
#pragma unroll
      for (int a = 0; a < DA; ++a) S[a] = cut ? 0.0f : lam * S[a];
    }
    for (int g = 0; g < p.gk; ++g) {
      const int hk = n * p.gk + g;
      __syncthreads();
      for (int a = threadIdx.x; a < DA; a += 64) {
        kq[0][a] = a < p.da ? p.kscale * ld<E>(p.k, row * p.ldk + static_cast<size_t>(hk) * p.da + a) : 0.0f;
        kq[1][a] = a < p.da ? p.oscale * ld<E>(p.q, row * p.ldq + static_cast<size_t>(hq) * p.da + a) : 0.0f;
      }
      __syncthreads();
      const float v = on ? ld<E>(p.v, row * p.ldv + static_cast<size_t>(hk) * p.dc + c) : 0.0f;
#pragma unroll
      for (int a = 0; a < DA; ++a)
        if (a < p.da) S[a] = fmaf(kq[0][a], v, S[a]);
    }
    float o = 0.0f;
#pragma unroll
    for (int a = 0; a < DA; ++a)
      if (a < p.da) o = fmaf(kq[1][a], S[a], o);
    if (on) static_cast<E*>(p.o)[row * p.ldo + static_cast<size_t>(hq) * p.dc + c] = elem<E>::from_f32(o);
  }
  if (p.sT && on && hq % p.gq == 0) {
    const bool cut = p.rev && p.reset && p.reset[b] != 0;
#pragma unroll
    for (int a = 0; a < DA; ++a)
      if (a < p.da) p.sT[sbase + a * sa + c * sc] = cut ? 0.0f : (p.rev ? lam * S[a] : S[a]);
  }
}

template <typename E>
void launch_steps(const LinPass& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.B) * p.nkv * p.gq, (p.dc + 63) / 64);
  if (p.da <= 32)
    hipLaunchKernelGGL((linattn_steps<E, 32>), grid, dim3(64), 0, s, p);
  else if (p.da <= 64)
    hipLaunchKernelGGL((linattn_steps<E, 64>), grid, dim3(64), 0, s, p);
  else
    hipLaunchKernelGGL((linattn_steps<E, 128>), grid, dim3(64), 0, s, p);
}

void launch_pass(o5_dtype dt, const LinPass& p, hipStream_t s) {
  if (dt == O5_BF16)
    launch_steps<uint16_t>(p, s);
  else
    launch_steps<float>(p, s);
}

// ----------------------------------------------------------- single token

// One token of one state: a block takes CP groups of 4 columns and all rows,
// 256 / CP rows at a time, and keeps its part of the state in registers
// between the update and the group's query heads.
template <typename E, int CP, int DK>
__global__ void __launch_bounds__(256) linattn_token(int nkv, int G, int dk, int dv, const void* __restrict__ q, size_t ldq,
                                                     const void* __restrict__ k, size_t ldk,
                                                     const void* __restrict__ v, size_t ldv,
                                                     const float* __restrict__ decay, float scale,
                                                     const uint8_t* __restrict__ reset, float* __restrict__ S,
                                                     void* __restrict__ o, size_t ldo) {
  constexpr int RP = 256 / CP;       // rows in flight
  constexpr int NR = DK / RP;        // rows of a thread
  __shared__ float ks[DK], qs[DK];
  __shared__ float4 part[4][CP];
  const int b = blockIdx.x / nkv, n = blockIdx.x % nkv;
  const int tid = threadIdx.x, cg = tid % CP, r0 = tid / CP;
  const int c = (blockIdx.y * CP + cg) * 4;
  const bool on = c < dv;
  float* Sb = S + (static_cast<size_t>(b) * nkv + n) * dk * dv;
  const bool cut = reset != nullptr && reset[b] != 0;
  const float lam = decay[n];
  float4 s[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int a = r0 + i * RP;
    s[i] = (on && a < dk && !cut) ? *reinterpret_cast<const float4*>(Sb + static_cast<size_t>(a) * dv + c)
                                  : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
  if (tid < DK) ks[tid] = tid < dk ? ld<E>(k, b * ldk + static_cast<size_t>(n) * dk + tid) : 0.0f;
  float x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = on ? ld<E>(v, b * ldv + static_cast<size_t>(n) * dv + c + j) : 0.0f;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int a = r0 + i * RP;
    const float kk = ks[a];
    s[i] = make_float4(fmaf(kk, x[0], lam * s[i].x), fmaf(kk, x[1], lam * s[i].y), fmaf(kk, x[2], lam * s[i].z),
                       fmaf(kk, x[3], lam * s[i].w));
    if (on && a < dk) *reinterpret_cast<float4*>(Sb + static_cast<size_t>(a) * dv + c) = s[i];
  }
  for (int g = 0; g < G; ++g) {
    const size_t h = static_cast<size_t>(n) * G + g;
    if (tid < DK) qs[tid] = tid < dk ? scale * ld<E>(q, b * ldq + h * dk + tid) : 0.0f;
    __syncthreads();
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int a = r0 + i * RP;
      if (a < dk) {
        const float w = qs[a];
        y = make_float4(fmaf(w, s[i].x, y.x), fmaf(w, s[i].y, y.y), fmaf(w, s[i].z, y.z), fmaf(w, s[i].w, y.w));
      }
    }
#pragma unroll
    for (int w = CP; w < 64; w *= 2) {
      y.x += __shfl_xor(y.x, w);
      y.y += __shfl_xor(y.y, w);
      y.z += __shfl_xor(y.z, w);
      y.w += __shfl_xor(y.w, w);
    }
    if ((tid & 63) < CP) part[tid >> 6][cg] = y;
    __syncthreads();
    if (tid < CP && on) {
      const float4 p0 = part[0][cg], p1 = part[1][cg], p2 = part[2][cg], p3 = part[3][cg];
      E* ob = static_cast<E*>(o) + b * ldo + h * dv + c;
      ob[0] = elem<E>::from_f32((p0.x + p1.x) + (p2.x + p3.x));
      ob[1] = elem<E>::from_f32((p0.y + p1.y) + (p2.y + p3.y));
      ob[2] = elem<E>::from_f32((p0.z + p1.z) + (p2.z + p3.z));
      ob[3] = elem<E>::from_f32((p0.w + p1.w) + (p2.w + p3.w));
    }
  }
}

// ------------------------------------------------------------ validation

constexpr int kMaxHead = 128;

int check_sizes(const char* fn, o5_dtype dt, int T, int B, int nh, int nkv, int dk, int dv) {
  O5_CHECK(dt == O5_F32 || dt == O5_BF16, O5_E_DTYPE, "%s: unknown dtype %d", fn, static_cast<int>(dt));
  O5_CHECK(T >= 1 && B >= 1 && nh >= 1 && nkv >= 1, O5_E_SHAPE, "%s: T, B, nh and nkv must be >= 1", fn);
  O5_CHECK(nh % nkv == 0, O5_E_SHAPE, "%s: nh=%d is not a multiple of nkv=%d", fn, nh, nkv);
  for (int d : {dk, dv})
    O5_CHECK(d >= 8 && d <= kMaxHead && d % 8 == 0, O5_E_SHAPE,
             "%s: dk=%d and dv=%d must be multiples of 8 in 8..%d", fn, dk, dv, kMaxHead);
  O5_CHECK(static_cast<long long>(T) * B < (1ll << 31) && static_cast<long long>(nh) * kMaxHead < (1ll << 31) &&
               static_cast<long long>(B) * nh < (1ll << 24),
           O5_E_SHAPE, "%s: T*B must be below 2^31 and B*nh below 2^24", fn);
  return O5_OK;
}

int check_ld(const char* fn, const char* name, size_t ld, long long width) {
  O5_CHECK(ld >= static_cast<size_t>(width) && ld % 8 == 0 && ld < (1ull << 31), O5_E_SHAPE,
           "%s: %s=%zu must be a multiple of 8, at least %lld and below 2^31", fn, name, ld, width);
  return O5_OK;
}

#define O5_TRY(expr)                  \
  do {                                \
    const int st_ = (expr);           \
    if (st_ != O5_OK) return st_;     \
  } while (0)

int check_inputs(const char* fn, int nh, int nkv, int dk, int dv, const void* q, size_t ldq, const void* k, size_t ldk,
                 const void* v, size_t ldv, const float* decay, float scale) {
  O5_TRY(check_ld(fn, "ldq", ldq, static_cast<long long>(nh) * dk));
  O5_TRY(check_ld(fn, "ldk", ldk, static_cast<long long>(nkv) * dk));
  O5_TRY(check_ld(fn, "ldv", ldv, static_cast<long long>(nkv) * dv));
  O5_CHECK(std::isfinite(scale), O5_E_ARG, "%s: scale must be finite", fn);
  O5_PTR_IN(fn, q, "q");
  O5_PTR_IN(fn, k, "k");
  O5_PTR_IN(fn, v, "v");
  O5_PTR_IN(fn, decay, "decay");
  return O5_OK;
}

}  // namespace
}  // namespace o5

using namespace o5;

extern "C" size_t o5_linattn_fwd_workspace_bytes(o5_dtype dt, int T, int B, int nh, int nkv, int dk, int dv) {
  if (check_sizes("o5_linattn_fwd_workspace_bytes", dt, T, B, nh, nkv, dk, dv) != O5_OK) return 0;
  return 16;
}

extern "C" int o5_linattn_fwd(o5_dtype dt, int T, int B, int nh, int nkv, int dk, int dv, const void* q, size_t ldq,
                              const void* k, size_t ldk, const void* v, size_t ldv, const float* decay, float scale,
                              const float* S0, const uint8_t* reset, void* o, size_t ldo, float* ST, void* ws,
                              size_t ws_bytes, void* stream) {
  const char* fn = "o5_linattn_fwd";
  O5_TRY(check_sizes(fn, dt, T, B, nh, nkv, dk, dv));
  O5_TRY(check_inputs(fn, nh, nkv, dk, dv, q, ldq, k, ldk, v, ldv, decay, scale));
  O5_TRY(check_ld(fn, "ldo", ldo, static_cast<long long>(nh) * dv));
  O5_PTR(o, "o");
  O5_OPT_PTR(S0, "S0");
  O5_OPT_PTR(ST, "ST");
  O5_OPT_PTR(reset, "reset");
  O5_CHECK(ws != nullptr && ws_bytes >= o5_linattn_fwd_workspace_bytes(dt, T, B, nh, nkv, dk, dv), O5_E_WORKSPACE,
           "%s: ws is NULL or ws_bytes=%zu is too small", fn, ws_bytes);
  O5_PTR(ws, "ws");
  const LinPass p = {q, k, v, o, ldq, ldk, ldv, ldo, decay, reset, S0, ST, T, B, nkv, nh / nkv, 1, dk, dv, scale, 1.0f,
                     false, false};
  launch_pass(dt, p, as_stream(stream));
  return check_launch(fn);
}

extern "C" size_t o5_linattn_bwd_workspace_bytes(o5_dtype dt, int T, int B, int nh, int nkv, int dk, int dv) {
  if (check_sizes("o5_linattn_bwd_workspace_bytes", dt, T, B, nh, nkv, dk, dv) != O5_OK) return 0;
  return 16;
}

extern "C" int o5_linattn_bwd(o5_dtype dt, int T, int B, int nh, int nkv, int dk, int dv, const void* q, size_t ldq,
                              const void* k, size_t ldk, const void* v, size_t ldv, const float* decay, float scale,
                              const float* S0, const uint8_t* reset, const void* dout, size_t lddo, const float* dST,
                              void* dq, size_t lddq, void* dkey, size_t lddk, void* dval, size_t lddv, float* dS0,
                              void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "o5_linattn_bwd";
  O5_TRY(check_sizes(fn, dt, T, B, nh, nkv, dk, dv));
  O5_TRY(check_inputs(fn, nh, nkv, dk, dv, q, ldq, k, ldk, v, ldv, decay, scale));
  O5_TRY(check_ld(fn, "lddo", lddo, static_cast<long long>(nh) * dv));
  O5_TRY(check_ld(fn, "lddq", lddq, static_cast<long long>(nh) * dk));
  O5_TRY(check_ld(fn, "lddk", lddk, static_cast<long long>(nkv) * dk));
  O5_TRY(check_ld(fn, "lddv", lddv, static_cast<long long>(nkv) * dv));
  O5_PTR(dout, "dout");
  O5_PTR(dq, "dq");
  O5_PTR(dkey, "dk");
  O5_PTR(dval, "dv");
  O5_OPT_PTR(S0, "S0");
  O5_OPT_PTR(reset, "reset");
  O5_OPT_PTR(dST, "dST");
  O5_OPT_PTR(dS0, "dS0");
  O5_CHECK(ws != nullptr && ws_bytes >= o5_linattn_bwd_workspace_bytes(dt, T, B, nh, nkv, dk, dv), O5_E_WORKSPACE,
           "%s: ws is NULL or ws_bytes=%zu is too small", fn, ws_bytes);
  O5_PTR(ws, "ws");
  const int G = nh / nkv;
  const LinPass pq = {dout, v, k, dq, lddo, ldv, ldk, lddq, decay, reset, S0, nullptr, T, B, nkv, G, 1, dv, dk, scale,
                      1.0f, true, false};
  const LinPass pv = {k, q, dout, dval, ldk, ldq, lddo, lddv, decay, reset, dST, dS0, T, B, nkv, 1, G, dk, dv, 1.0f,
                      scale, false, true};
  const LinPass pk = {v, dout, q, dkey, ldv, lddo, ldq, lddk, decay, reset, dST, nullptr, T, B, nkv, 1, G, dv, dk, 1.0f,
                      scale, true, true};
  for (const LinPass* p : {&pq, &pv, &pk}) launch_pass(dt, *p, as_stream(stream));
  return check_launch(fn);
}

extern "C" int o5_linattn_step(o5_dtype dt, int B, int nh, int nkv, int dk, int dv, const void* q, size_t ldq,
                               const void* k, size_t ldk, const void* v, size_t ldv, const float* decay, float scale,
                               const uint8_t* reset, float* S, void* o, size_t ldo, void* stream) {
  const char* fn = "o5_linattn_step";
  O5_TRY(check_sizes(fn, dt, 1, B, nh, nkv, dk, dv));
  O5_TRY(check_inputs(fn, nh, nkv, dk, dv, q, ldq, k, ldk, v, ldv, decay, scale));
  O5_TRY(check_ld(fn, "ldo", ldo, static_cast<long long>(nh) * dv));
  O5_PTR(S, "S");
  O5_PTR(o, "o");
  O5_OPT_PTR(reset, "reset");
  const dim3 grid(static_cast<unsigned>(B) * nkv, (dv + 31) / 32);
  auto kernel = dt == O5_BF16 ? (dk <= 32 ? linattn_token<uint16_t, 8, 32> : dk <= 64 ? linattn_token<uint16_t, 8, 64> : linattn_token<uint16_t, 8, 128>)
                              : (dk <= 32 ? linattn_token<float, 8, 32> : dk <= 64 ? linattn_token<float, 8, 64> : linattn_token<float, 8, 128>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, as_stream(stream), nkv, nh / nkv, dk, dv, q, ldq, k, ldk, v, ldv, decay,
                     scale, reset, S, o, ldo);
  return check_launch(fn);
}
