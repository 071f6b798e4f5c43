// The clipped policy loss with value, entropy and KL terms and its gradient on
// logits, o5_ppo_logits_grad.
//
// A team of lanes takes a row.  One pass over each head's logits and the
// reference's carries, relative to the largest seen so far (m, and mr of the
// reference),
//
//   s = sum e^(z-m),  t = sum e^(z-m) (z-m),  v = sum e^(z-m) (y-mr),
//   sr = sum e^(y-mr)                            (z logits, y the reference's)
//
// so that log p_j = z_j - m - log s, S = log s - t/s and
// KL = (t - v)/s - log(s/sr), a difference of small numbers where the policies
// are near each other.  A second pass writes
//
//   dz_j = -w A r [unclipped] (1[j = a] - p_j)
//          + w p_j (ent (log p_j + S) + kl (log p_j - log q_j - KL)).
//
// HBM-bound where rows are wide: logits and reference are read once from
// memory (the second pass finds them in a cache) and the gradient written once.
#include "heads.h"
#include "reduce.h"

namespace o5 {
namespace {

constexpr int kSums = 8;  // pg, vf, ent, clipfrac, approx_kl, ratio, nonfinite, kl
constexpr int kMostLogits = 1 << 24;
constexpr int kMaxBlocks = 2048;
constexpr float kLowest = -3.40282346e38f;

struct Loss {  // a call's arrays
  const void *z, *y;
  void* dz;
  size_t ldz, ldy, ldd;
  const int32_t* act;
  const float *logp_old, *adv, *ret, *weight;
  const uint8_t *mask, *avail;
  float *logp, *kl;
  double* part;  // [blocks][kSums]
  int N;
  HeadsMeta heads;
  float clip_eps, vf_coef, ent_coef, kl_coef, even;
};

// ---------------------------------------------------- reductions of a team

// Over the G lanes of a team, the result in each, in a fixed order: within a
// row of 16 lanes, a wave, or the waves of a block through LDS.
template <int G, class Op>
__device__ __forceinline__ float lanes_reduce(float v, float id, Op op) {
  if (G == 16) {
    v = op(v, dpp<0xB1>(id, v));   // quad_perm [1, 0, 3, 2]
    v = op(v, dpp<0x4E>(id, v));   // quad_perm [2, 3, 0, 1]
    v = op(v, dpp<0x124>(id, v));  // row_ror 4
    v = op(v, dpp<0x128>(id, v));  // row_ror 8
    return v;
  }
  return wave_reduce(v, id, op);
}
__device__ __forceinline__ float op_max(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float op_sum(float a, float b) { return a + b; }

// n values at once; red [2][16 waves][n], used in turn.
template <int G, int n, class Op>
__device__ __forceinline__ void team_reduce(float (&v)[n], float id, Op op, float (*red)[n]) {
#pragma unroll
  for (int q = 0; q < n; ++q) v[q] = lanes_reduce<G>(v[q], id, op);
  if (G <= 64) return;
  const int wave = threadIdx.x >> 6;
  __syncthreads();  // (the last reduction's values have been read)
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int q = 0; q < n; ++q) red[wave][q] = v[q];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < n; ++q) v[q] = red[0][q];
  for (int w = 1; w < G / 64; ++w)
#pragma unroll
    for (int q = 0; q < n; ++q) v[q] = op(v[q], red[w][q]);
}

// ------------------------------------------------------------- the columns

// V neighbouring elements, of which n are there (at no alignment but the
// element's).
template <typename E, int V>
struct Cols {
  E v[V];
  __device__ __forceinline__ void load(const E* p, int n) {
    if (n >= V) {
      __builtin_memcpy(v, p, sizeof v);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = j < n ? p[j] : E(0);
    }
  }
  __device__ __forceinline__ void store(E* p, int n) const {
    if (n >= V) {
      __builtin_memcpy(p, v, sizeof v);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < n) p[j] = v[j];
    }
  }
  __device__ __forceinline__ float operator[](int j) const;
};
template <typename E, int V>
__device__ __forceinline__ float Cols<E, V>::operator[](int j) const { return elem<E>::to_f32(v[j]); }

// e^x of x <= 0, the lowest difference of two floats included.
__device__ __forceinline__ float exp_of(float x) { return __expf(x); }
// a - b, where infinities and overflow become the lowest number: its
// exponential is 0, and 0 times it is 0.
__device__ __forceinline__ float below(float a, float b) { return fmaxf(a - b, kLowest); }
// f x, and 0 where f is: what has become negligible may be infinite.
__device__ __forceinline__ float scaled(float f, float x) { return f == 0.0f ? 0.0f : f * x; }

// A head's logs of sums stand apart from the largest logits: beside a large
// one they would be lost.
struct HeadStats {
  float m, ls, mr, lsr;  // log p = z - m - ls, log q = y - mr - lsr
  float S, D;            // entropy, KL
  bool some;             // a logit that counts
};

// One pass over a head of n logits.
template <typename E, int G, int V>
__device__ __forceinline__ HeadStats head_stats(const E* z, const E* y, const uint8_t* av, int n, int lane,
                                                float (*redm)[2], float (*reds)[4]) {
  float m = kLowest, mr = kLowest, s = 0.0f, t = 0.0f, v = 0.0f, sr = 0.0f;
  for (int j = lane * V; j < n; j += G * V) {
    const int have = n - j;
    Cols<E, V> zc, yc;
    Cols<uint8_t, V> ac;
    zc.load(z + j, have);
    if (y) yc.load(y + j, have);
    if (av) ac.load(av + j, have);
    float zz[V], yy[V], mj = m, mrj = mr;
#pragma unroll
    for (int q = 0; q < V; ++q) {
      const bool on = q < have && (!av || ac.v[q] != 0);
      zz[q] = on ? zc[q] : -INFINITY;
      yy[q] = on && y ? yc[q] : -INFINITY;
      mj = fmaxf(mj, zz[q]);
      mrj = fmaxf(mrj, yy[q]);
    }
    const float d = below(m, mj), f = exp_of(d);
    t = scaled(f, fmaf(s, d, t));
    s *= f;
    v = fmaf(s, below(mr, mrj), scaled(f, v));
    sr *= exp_of(below(mr, mrj));
    m = mj;
    mr = mrj;
#pragma unroll
    for (int q = 0; q < V; ++q) {
      const float dz = zz[q] - m, e = exp_of(dz);
      s += e;
      const bool nil = e == 0.0f;  // (NaN is none)
      t += nil ? 0.0f : e * dz;
      if (y) {
        const float dy = yy[q] - mr;
        v += nil ? 0.0f : e * dy;
        sr += exp_of(dy);
      }
    }
  }
  float mm[2] = {m, mr};
  team_reduce<G>(mm, kLowest, op_max, redm);
  const float d = below(m, mm[0]), dr = below(mr, mm[1]), f = exp_of(d);
  float sum[4];
  sum[0] = s * f;
  sum[1] = scaled(f, fmaf(s, d, t));
  sum[2] = fmaf(sum[0], dr, scaled(f, v));
  sum[3] = sr * exp_of(dr);
  team_reduce<G>(sum, 0.0f, op_sum, reds);
  HeadStats h;
  h.some = sum[0] != 0.0f;
  h.m = mm[0];
  h.mr = mm[1];
  h.ls = logf(sum[0]);
  h.lsr = logf(sum[3]);
  h.S = h.ls - sum[1] / sum[0];
  h.D = y ? (sum[1] - sum[2]) / sum[0] - logf(sum[0] / sum[3]) : 0.0f;
  return h;
}

// What a row's gradient needs beside its heads' statistics.
struct RowGrad {
  float pg, ent, kl;
};

template <typename E, int G, int V>
__device__ __forceinline__ void head_grad(const E* z, const E* y, const uint8_t* av, E* dz, int n, int lane, bool use,
                                          const HeadStats& h, int a, const RowGrad& g) {
  for (int j = lane * V; j < n; j += G * V) {
    const int have = n - j;
    Cols<E, V> zc, yc, out;
    Cols<uint8_t, V> ac;
    if (use) {
      zc.load(z + j, have);
      if (y) yc.load(y + j, have);
      if (av) ac.load(av + j, have);
    }
#pragma unroll
    for (int q = 0; q < V; ++q) {
      float d = 0.0f;
      if (use && (!av || ac.v[q] != 0)) {
        const float lp = (zc[q] - h.m) - h.ls, p = exp_of(lp);
        float c = g.ent * (lp + h.S);
        if (y) c = fmaf(g.kl, lp - ((yc[q] - h.mr) - h.lsr) - h.D, c);
        d = p == 0.0f ? 0.0f : p * (c - g.pg);
        if (j + q == a) d += g.pg;
      }
      out.v[q] = elem<E>::from_f32(d);
    }
    out.store(dz + j, have);
  }
}

// ----------------------------------------------------------------- kernels

// A team's lane k holds head k's number.
template <int G>
__device__ __forceinline__ float of_head(float v, int k) { return __shfl(v, k, G < 64 ? G : 64); }

template <typename E, int G, int V>
__global__ void __launch_bounds__(G < 256 ? 256 : G) logits_rows(Loss p) {
  constexpr int kThreads = G < 256 ? 256 : G, kTeams = kThreads / G;
  __shared__ float redm[16][2], reds[16][4];
  __shared__ double sums[kTeams][kSums];
  const int team = threadIdx.x / G, lane = threadIdx.x % G, K = p.heads.K, A = p.heads.A;
  const float kl_coef = p.y ? p.kl_coef : 0.0f;
  double acc[kSums] = {};
  for (int64_t n = static_cast<int64_t>(blockIdx.x) * kTeams + team; n < p.N; n += static_cast<int64_t>(gridDim.x) * kTeams) {
    const E* z = static_cast<const E*>(p.z) + n * p.ldz;
    const E* y = p.y ? static_cast<const E*>(p.y) + n * p.ldy : nullptr;
    E* dz = static_cast<E*>(p.dz) + n * p.ldd;
    const uint8_t* av = p.avail ? p.avail + n * A : nullptr;
    const float w = p.weight ? p.weight[n] : p.even;
    const bool pad = w == 0.0f;
    float logpi = 0.0f, ent = 0.0f, kl = 0.0f;
    // head k's statistics, in lane k (of each wave)
    float m = 0.0f, ls = 0.0f, mr = 0.0f, lsr = 0.0f, S = 0.0f, D = 0.0f;
    int use = 0;
    for (int k = 0; k < K && !pad; ++k) {
      if (p.mask && p.mask[n * K + k] == 0) continue;
      const int o = p.heads.off[k], nk = p.heads.off[k + 1] - o, a = p.act[n * K + k];
      const HeadStats h = head_stats<E, G, V>(z + o, y ? y + o : nullptr, av ? av + o : nullptr, nk, lane, redm, reds);
      if (!h.some) continue;
      const bool taken = a >= 0 && a < nk && (!av || av[o + a] != 0);
      logpi += taken ? (elem<E>::to_f32(z[o + (taken ? a : 0)]) - h.m) - h.ls : -INFINITY;
      ent += h.S;
      kl += h.D;
      use |= 1 << k;
      if ((lane & 63) == k) m = h.m, ls = h.ls, mr = h.mr, lsr = h.lsr, S = h.S, D = h.D;
    }
    const float Ad = pad ? 0.0f : p.adv[n];
    const float dlog = pad ? 0.0f : logpi - p.logp_old[n];
    const float ratio = expf(dlog);
    const float cut = fminf(fmaxf(ratio, 1.0f - p.clip_eps), 1.0f + p.clip_eps);
    const float surr = fminf(ratio * Ad, cut * Ad);
    const bool flow = (Ad >= 0.0f && ratio <= 1.0f + p.clip_eps) || (Ad < 0.0f && ratio >= 1.0f - p.clip_eps);
    const float err = p.ret && !pad ? elem<E>::to_f32(z[A]) - p.ret[n] : 0.0f;
    const RowGrad g = {flow ? -w * ratio * Ad : 0.0f, w * p.ent_coef, w * kl_coef};
    for (int k = 0; k < K; ++k) {
      const int o = p.heads.off[k], nk = p.heads.off[k + 1] - o;
      HeadStats h;
      h.m = of_head<G>(m, k);
      h.ls = of_head<G>(ls, k);
      h.mr = of_head<G>(mr, k);
      h.lsr = of_head<G>(lsr, k);
      h.S = of_head<G>(S, k);
      h.D = of_head<G>(D, k);
      const bool on = (use >> k) & 1;
      head_grad<E, G, V>(z + o, kl_coef != 0.0f ? y + o : nullptr, av ? av + o : nullptr, dz + o, nk, lane, on, h,
                         on ? p.act[n * K + k] : -1, g);
    }
    if (lane == 0) {
      if (p.ret) dz[A] = elem<E>::from_f32(2.0f * p.vf_coef * w * err);
      if (p.logp) p.logp[n] = pad ? 0.0f : logpi;
      if (p.kl) p.kl[n] = pad ? 0.0f : kl;
    }
    if (pad) continue;
    const float loss = -surr + p.vf_coef * err * err - p.ent_coef * ent + (kl_coef != 0.0f ? kl_coef * kl : 0.0f);
    const double wd = w;
    acc[0] -= wd * surr;
    acc[1] += wd * (err * err);
    acc[2] += wd * ent;
    acc[3] += fabsf(ratio - 1.0f) > p.clip_eps ? wd : 0.0;
    acc[4] += wd * (expm1f(dlog) - dlog);  // (r - 1) - log r without the cancellation in r - 1
    acc[5] += wd * ratio;
    acc[6] += isfinite(loss) ? 0.0 : 1.0;
    acc[7] += wd * kl;
  }
  if (lane == 0)
#pragma unroll
    for (int q = 0; q < kSums; ++q) sums[team][q] = acc[q];
  __syncthreads();
  if (threadIdx.x < kSums) {
    double s = 0.0;
    for (int q = 0; q < kTeams; ++q) s += sums[q][threadIdx.x];
    p.part[static_cast<size_t>(blockIdx.x) * kSums + threadIdx.x] = s;
  }
}

// The statistics from the blocks' sums, in a fixed order: thread t takes sum t
// mod 8 of blocks t / 8, t / 8 + 32, ...
__global__ void __launch_bounds__(256) logits_stats(int blocks, const double* __restrict__ part, float vf_coef,
                                                    float ent_coef, float kl_coef, float* __restrict__ stats) {
  __shared__ double red[32][kSums];
  const int q = threadIdx.x % kSums, r = threadIdx.x / kSums;
  double s = 0.0;
#pragma unroll 8
  for (int b = r; b < blocks; b += 32) s += part[b * kSums + q];
  red[r][q] = s;
  __syncthreads();
  if (r == 0) {
    for (int k = 1; k < 32; ++k) s += red[k][q];
    red[0][q] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const double* x = red[0];
    const double kl = kl_coef != 0.0f ? kl_coef * x[7] : 0.0;
    stats[0] = static_cast<float>(x[0] + vf_coef * x[1] - ent_coef * x[2] + kl);
    for (int k = 0; k < 7; ++k) stats[k + 1] = static_cast<float>(x[k]);
    stats[8] = static_cast<float>(x[7]);
  }
}

struct Form {
  int teams, threads;
  void (*f32)(Loss);
  void (*bf16)(Loss);
};

Form form_of(const HeadsMeta& hm) {
  int most = 0;
  for (int k = 0; k < hm.K; ++k) most = std::max(most, hm.off[k + 1] - hm.off[k]);
  if (most <= 128) return {16, 256, logits_rows<float, 16, 1>, logits_rows<uint16_t, 16, 1>};
  if (most <= 2048) return {4, 256, logits_rows<float, 64, 4>, logits_rows<uint16_t, 64, 8>};
  if (most <= 16384) return {1, 256, logits_rows<float, 256, 4>, logits_rows<uint16_t, 256, 8>};
  return {1, 1024, logits_rows<float, 1024, 4>, logits_rows<uint16_t, 1024, 8>};
}

int blocks_of(const Form& f, int N) { return static_cast<int>(std::min<long long>((N + f.teams - 1ll) / f.teams, kMaxBlocks)); }

#define O5_TRY(expr)              \
  do {                            \
    const int st_ = (expr);       \
    if (st_ != O5_OK) return st_; \
  } while (0)

int check_sizes(const char* fn, o5_dtype dt, int N, int K, const int* head_sizes, HeadsMeta* hm) {
  O5_CHECK(dt == O5_F32 || dt == O5_BF16, O5_E_DTYPE, "%s: unknown dtype %d", fn, static_cast<int>(dt));
  O5_CHECK(N >= 1 && N < (1 << 30), O5_E_SHAPE, "%s: N=%d must be in 1..2^30-1", fn, N);
  O5_CHECK(K >= 1 && K <= kMaxHeads, O5_E_SHAPE, "%s: K=%d must be in 1..%d", fn, K, kMaxHeads);
  O5_CHECK(head_sizes != nullptr, O5_E_NULL, "%s: argument 'head_sizes' is NULL", fn);
  hm->K = K;
  long long at = 0;
  for (int k = 0; k < K; ++k) {
    O5_CHECK(head_sizes[k] >= 1, O5_E_SHAPE, "%s: head_sizes[%d]=%d must be >= 1", fn, k, head_sizes[k]);
    hm->off[k] = static_cast<int>(at);
    at += head_sizes[k];
    O5_CHECK(at <= kMostLogits, O5_E_SHAPE, "%s: the heads have more than 2^24 logits", fn);
  }
  for (int k = K; k <= kMaxHeads; ++k) hm->off[k] = static_cast<int>(at);
  hm->A = static_cast<int>(at);
  return O5_OK;
}

int check_rows(const char* fn, const char* name, const void* p, const char* ldname, size_t ld, int cols) {
  O5_CHECK(ld >= static_cast<size_t>(cols) && ld < (1ull << 31), O5_E_SHAPE, "%s: %s=%zu must be at least %d and below 2^31",
           fn, ldname, ld, cols);
  O5_PTR_IN(fn, p, name);
  return O5_OK;
}

}  // namespace
}  // namespace o5

using namespace o5;

extern "C" size_t o5_ppo_logits_grad_workspace_bytes(o5_dtype dt, int N, int K, const int* head_sizes) {
  HeadsMeta hm;
  if (check_sizes("o5_ppo_logits_grad_workspace_bytes", dt, N, K, head_sizes, &hm) != O5_OK) return 0;
  return std::max<size_t>(256, static_cast<size_t>(blocks_of(form_of(hm), N)) * kSums * sizeof(double));
}

extern "C" int o5_ppo_logits_grad(o5_dtype dt, int N, int K, const int* head_sizes, const void* logits, size_t ldl,
                                  const void* ref, size_t ldr, const int32_t* act, const float* logp_old,
                                  const float* adv, const float* ret, const float* weight, const uint8_t* head_mask,
                                  const uint8_t* avail, o5_ppo_hp hp, float kl_coef, float* stats, float* logp, float* kl,
                                  void* dlogits, size_t ldd, void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "o5_ppo_logits_grad";
  Loss p = {};
  O5_TRY(check_sizes(fn, dt, N, K, head_sizes, &p.heads));
  const int A = p.heads.A, cols = A + (ret ? 1 : 0);
  O5_TRY(check_rows(fn, "logits", logits, "ldl", ldl, cols));
  O5_TRY(check_rows(fn, "dlogits", dlogits, "ldd", ldd, cols));
  if (ref) O5_TRY(check_rows(fn, "ref", ref, "ldr", ldr, A));
  O5_PTR(act, "act");
  O5_PTR(logp_old, "logp_old");
  O5_PTR(adv, "adv");
  O5_OPT_PTR(ret, "ret");
  O5_OPT_PTR(weight, "weight");
  O5_OPT_PTR(head_mask, "head_mask");
  O5_OPT_PTR(avail, "avail");
  O5_PTR(stats, "stats");
  O5_OPT_PTR(logp, "logp");
  O5_OPT_PTR(kl, "kl");
  O5_CHECK(hp.clip_eps >= 0.0f && hp.clip_eps < 1.0f, O5_E_ARG, "%s: clip_eps=%g must be in [0, 1)", fn, hp.clip_eps);
  O5_CHECK(std::isfinite(hp.vf_coef) && std::isfinite(hp.ent_coef) && std::isfinite(kl_coef), O5_E_ARG,
           "%s: the coefficients must be finite", fn);
  O5_CHECK(ws != nullptr && ws_bytes >= o5_ppo_logits_grad_workspace_bytes(dt, N, K, head_sizes), O5_E_WORKSPACE,
           "%s: ws is NULL or ws_bytes=%zu is too small", fn, ws_bytes);
  O5_PTR(ws, "ws");
  p.z = logits, p.y = ref, p.dz = dlogits;
  p.ldz = ldl, p.ldy = ldr, p.ldd = ldd;
  p.act = act, p.logp_old = logp_old, p.adv = adv, p.ret = ret, p.weight = weight, p.mask = head_mask, p.avail = avail;
  p.logp = logp, p.kl = kl, p.part = static_cast<double*>(ws), p.N = N;
  p.clip_eps = hp.clip_eps, p.vf_coef = hp.vf_coef, p.ent_coef = hp.ent_coef, p.kl_coef = kl_coef;
  p.even = static_cast<float>(1.0 / N);
  const Form f = form_of(p.heads);
  const int blocks = blocks_of(f, N);
  hipLaunchKernelGGL(dt == O5_BF16 ? f.bf16 : f.f32, dim3(blocks), dim3(f.threads), 0, as_stream(stream), p);
  hipLaunchKernelGGL(logits_stats, dim3(1), dim3(256), 0, as_stream(stream), blocks, p.part, hp.vf_coef, hp.ent_coef,
                     ref ? kl_coef : 0.0f, stats);
  return check_launch(fn);
}
