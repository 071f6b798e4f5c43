// The clipped policy loss with value, entropy and KL terms and its gradient on
// logits, o5_ppo_logits_grad.
//
// With the largest logits m of a head and mr of the reference's,
//
//   s = sum e^(z-m),  t = sum e^(z-m) (z-m),  v = sum e^(z-m) (y-mr),
//   sr = sum e^(y-mr)                            (z logits, y the reference's)
//
// give log p_j = z_j - m - log s, S = log s - t/s and KL = (t - v)/s -
// log(s/sr), a difference of small numbers where the policies are near each
// other, and then
//
//   dz_j = -w A r [unclipped] (1[j = a] - p_j)
//          + w p_j (ent (log p_j + S) + kl (log p_j - log q_j - KL)),
//
// of which all but 1[j = a] is p_j times a linear function of z_j and y_j.
//
// A team of lanes takes a row and holds it in registers, 16 bytes of a head's
// logits and of the reference's to a slot: everything is read once and written
// once.  Rows too wide for that are read twice, the second time from a cache.
// HBM-bound by its bytes; the 33 instructions an element, 3 exponentials among
// them, take nearly as long: 8192 rows of 32000 logits and a reference's in bf16, a
// tenth of them padding, 1.47 GB, 337 us, 4.4 TB/s, with the vector units busy in 84 %
// of the cycles.  1003 rows of 50257 in fp32, which do not fit in a block's registers,
// 175 us, 3.6 TB/s.  Narrow rows are bound by their 690 instructions for four rows: 32768
// rows of 74 logits in 4 heads, 19 MB, 15.8 us; 60 of them in one block 9.4.
#include "heads.h"
#include "reduce.h"

namespace o5 {

// x y, and 0 where one of them is, whatever the other (v_mul_legacy_f32): what has
// probability 0 counts nothing, infinities included.
__device__ __attribute__((const)) float times(float x, float y) __asm("llvm.amdgcn.fmul.legacy");

namespace {

constexpr int kSums = 8;  // pg, vf, ent, clipfrac, approx_kl, ratio, nonfinite, kl
constexpr int kMostLogits = 1 << 24;
constexpr float kLowest = -3.40282346e38f;
constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;

// A call's arrays.  What a call has not is read all the same, from an array that
// it has, and not used (has_*): a branch around a load would wait for it.
struct Loss {
  const void *z, *y;
  void* dz;
  size_t ldz, ldy, ldd, lda;
  const int32_t* act;
  const float *logp_old, *adv, *ret, *weight;
  const uint8_t *mask, *avail;
  float *logp, *kl, *stats;
  double* part;  // [blocks][kSums]
  int N;
  int has_ref, has_ret, has_weight, has_mask, has_avail;
  HeadsMeta heads;
  float clip_eps, vf_coef, ent_coef, kl_coef, even;  // kl_coef: 0 without a reference
};

// ---------------------------------------------------------------- a slot

// 16 bytes of neighbouring columns as they are stored, at no alignment but the
// element's.
template <typename E>
struct Slot {
  static constexpr int V = 16 / sizeof(E);
  uint32_t w[4];

  __device__ __forceinline__ void load(const E* p) { __builtin_memcpy(w, p, 16); }
  // The first n of V, one by one.
  __device__ __forceinline__ void load_some(const E* p, int n) {
    float x[V];
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = j < n ? elem<E>::to_f32(p[j]) : 0.0f;
    set(x);
  }
  // Columns skip to skip + n, V at most, to p + skip ...
  __device__ __forceinline__ void store(E* p, int skip, int n) const {
    if (n >= V) {
      __builtin_memcpy(p, w, 16);
      return;
    }
    if (n <= 0) return;
    constexpr int kBits = 8 * sizeof(E);
    uint64_t lo = w[0] | static_cast<uint64_t>(w[1]) << 32, hi = w[2] | static_cast<uint64_t>(w[3]) << 32;
    if (skip > 0) {
      p += skip;
      lo = skip < V / 2 ? (lo >> (kBits * skip)) | (hi << (64 - kBits * skip)) : hi >> (kBits * (skip - V / 2));
      hi >>= kBits * min(skip, V / 2 - 1);  // (what is left of more is not stored)
    }
    if (n & (V / 2)) {
      __builtin_memcpy(p, &lo, 8);
      p += V / 2;
      lo = hi;
    }
    if (V == 8 && (n & 2)) {
      __builtin_memcpy(p, &lo, 4);
      p += 2;
      lo >>= 32;
    }
    if (n & 1) __builtin_memcpy(p, &lo, sizeof(E));
  }
  __device__ __forceinline__ float operator[](int j) const {
    if (sizeof(E) == 4) return __uint_as_float(w[j % 4]);
    return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&x)[V]) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[k] = sizeof(E) == 4 ? __float_as_uint(x[k]) : f32x2_to_bf16x2(x[2 * k % V], x[(2 * k + 1) % V]);
  }
  // What was computed from the slot before is not kept for what follows, nor is
  // what follows begun before: all columns as floats at once would take more
  // registers than there are.
  __device__ __forceinline__ void hold() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
  }
  // -infinity in place of the columns whose bits in m are 0.
  __device__ __forceinline__ void mask(const uint32_t (&m)[4]) {
    const uint32_t low = sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = (w[k] & m[k]) | (low & ~m[k]);
  }
};

// Where a slot lies: the 16 bytes from column `col` of the row, of which
// columns skip to skip + have are the slot's own.  The last of a row begins
// further left, so that no slot reaches past the row's A logits (there are V of
// them but in tiny rows).
template <typename E>
struct Span {
  static constexpr int V = Slot<E>::V;
  int col, skip, have;
  __device__ __forceinline__ Span() = default;
  __device__ __forceinline__ Span(int start, int left, int A) {
    have = max(0, min(V, left));
    col = max(0, min(start, A - V));  // (a slot of no columns lies somewhere in the row)
    skip = (start - col) & (V - 1);
  }
  // The availability of the slot's columns as it is stored, a byte each.
  template <bool kTiny>
  __device__ __forceinline__ void load(const uint8_t* av, int A, uint32_t (&b)[2]) const {
    b[1] = 0;
    if (!kTiny) {
      __builtin_memcpy(b, av + col, V);
      return;
    }
    uint64_t x = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) x |= static_cast<uint64_t>(j < A ? av[j] : 0) << (8 * j);
    b[0] = static_cast<uint32_t>(x);
    b[1] = static_cast<uint32_t>(x >> 32);
  }
  // All bits of the slot's own columns.
  __device__ __forceinline__ void own(uint32_t (&m)[4]) const {
    const int bits = ((1 << have) - 1) << skip;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (sizeof(E) == 4) {
        m[k] = -((bits >> k) & 1);
      } else {
        const uint32_t lo = -((bits >> (2 * k)) & 1), hi = -((bits >> (2 * k + 1)) & 1);
        m[k] = (lo & 0xffffu) | (hi & 0xffff0000u);
      }
    }
  }
  // ... and of the columns that are available.
  __device__ __forceinline__ static void available(const uint32_t (&b)[2], uint32_t (&m)[4]) {
    uint32_t t[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) t[k] = ((b[k] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | b[k];  // bit 7 of a byte that is not 0
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (sizeof(E) == 4)
        m[k] &= -static_cast<int>((t[0] >> (8 * k + 7)) & 1);
      else  // (selectors 8 to 11 are the signs of bytes 1 and 3 of the second and the first operand)
        m[k] &= __builtin_amdgcn_perm(t[k / 2], t[k / 2] << 8, k & 1 ? 0x0b0b0909u : 0x0a0a0808u);
    }
  }
};

// ------------------------------------------------------------ the formulas

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log_of(float x) { return __builtin_amdgcn_logf(x) * kLn2; }

// Sums and probabilities are of z - m, rounded to 2^-24 of itself and 0 for the largest logit wherever it
// lies.  (One instruction more than fma(z, log2 e, -m log2 e), whose rounding of m log2 e is no longer small
// beside 1 from |m| = 1e7 on, and overflows e^(z-m) from 2^31 on.)
__device__ __forceinline__ float exp_of(float d) { return exp2_of(kLog2e * d); }
// What goes from sums relative to `from` to sums relative to the larger `to`.
__device__ __forceinline__ float between(float from, float to) { return fmaxf(from - to, kLowest); }

// The sums of a head's logits, relative to m and mr.
struct Sums {
  float s, t, v, sr;
  __device__ __forceinline__ void add(float z, float m) {
    const float d = z - m, e = exp_of(d);
    s += e;
    t += times(e, d);
  }
  __device__ __forceinline__ void add(float z, float m, float y, float mr) {
    const float d = z - m, e = exp_of(d), dy = y - mr;
    s += e;
    t += times(e, d);
    v += times(e, dy);
    sr += exp_of(dy);
  }
  // From m, mr to mn, mrn.
  __device__ __forceinline__ void move(float m, float mr, float mn, float mrn) {
    const float d = between(m, mn), dr = between(mr, mrn), f = exp_of(d);
    t = times(f, t + times(s, d));
    s *= f;
    v = times(f, v) + times(s, dr);
    sr *= exp_of(dr);
  }
};

// A head's log-sums (binary), entropy and divergence; the logs stand apart from
// the largest logits, beside which they would be lost.
struct HeadStats {
  float ls, lsr, S, D;
  bool some;  // a logit that counts
  __device__ __forceinline__ HeadStats(const Sums& x, bool ref) {
    some = x.s != 0.0f;
    const float inv = __builtin_amdgcn_rcpf(x.s);
    ls = __builtin_amdgcn_logf(x.s);
    lsr = __builtin_amdgcn_logf(x.sr);
    S = fmaf(kLn2, ls, -x.t * inv);
    D = ref ? fmaf(x.t - x.v, inv, log_of(x.sr * inv)) : 0.0f;
  }
};

// What the row gives its heads' gradients, and a head's p_j (kd d + ky dy + k0)
// of d = z - m and the reference's dy, with log p_j = d - log s.
struct RowGrad {
  float pg, ent, kl;
};
struct HeadGrad {
  float m, mr, ls, kd, ky, k0;
  __device__ __forceinline__ HeadGrad() = default;
  __device__ __forceinline__ HeadGrad(const RowGrad& g, const HeadStats& h, float m_, float mr_) : m(m_), mr(mr_) {
    ls = h.ls;
    kd = g.ent + g.kl;
    ky = -g.kl;
    k0 = fmaf(g.ent, fmaf(-kLn2, h.ls, h.S), -g.pg);
    if (g.kl != 0.0f) k0 = fmaf(g.kl, kLn2 * (h.lsr - h.ls) - h.D, k0);
  }
  __device__ __forceinline__ float p(float d) const { return exp2_of(fmaf(d, kLog2e, -ls)); }
  __device__ __forceinline__ float operator()(float z) const {
    const float d = z - m;
    return times(p(d), fmaf(kd, d, k0));
  }
  __device__ __forceinline__ float operator()(float z, float y) const {
    const float d = z - m;
    return times(p(d), fmaf(kd, d, fmaf(ky, y - mr, k0)));
  }
};

// A row's numbers beside its logits, the same in every lane of its team.
struct Row {
  float w, adv, old, err;
  bool pad;
  template <typename E>
  __device__ __forceinline__ void load(const Loss& p, int64_t n, const E* z, float weight) {
    w = weight;
    pad = w == 0.0f;
    adv = p.adv[n];
    old = p.logp_old[n];
    const float value = elem<E>::to_f32(z[p.has_ret ? p.heads.A : 0]), ret = p.ret[n];
    err = p.has_ret ? value - ret : 0.0f;
  }
};

// What has to be known of a row before its logits are loaded, and is loaded a
// row ahead: its weight and, in lane k, the action and the mask of head k.
struct Ahead {
  float w;
  int a;
  uint8_t active;
  __device__ __forceinline__ void load(const Loss& p, int64_t n, int k) {
    n = n < p.N ? n : p.N - 1;
    w = p.weight[n];
    a = p.act[n * p.heads.K + k];
    active = p.mask[n * p.heads.K + k];
    w = p.has_weight ? w : p.even;
    active = p.has_mask ? active : 1;
  }
};

// (r - 1) - log r of d = log r, without the cancellation near r = 1: the first
// term left out of d^2/2 + d^3/6 + ... is 1e-7 of them at 0.25.
__device__ __forceinline__ float beyond(float d, float r) {
  float s = fmaf(d, 1.0f / 5040.0f, 1.0f / 720.0f);
  s = fmaf(d, s, 1.0f / 120.0f);
  s = fmaf(d, s, 1.0f / 24.0f);
  s = fmaf(d, s, 1.0f / 6.0f);
  s = fmaf(d, s, 0.5f);
  return fabsf(d) < 0.25f ? d * d * s : (r - 1.0f) - d;
}

// The row's loss: the factors of its gradient, and, of the eight sums, the
// row's parts of those that the lane keeps (kParts of them, where a team has fewer than
// eight lanes).
template <int kParts>
__device__ __forceinline__ RowGrad row_loss(const Loss& p, const Row& r, float logpi, float ent, float kl, float kl_coef,
                                            int lane, double (&part)[kParts]) {
  const float dlog = logpi - r.old, ratio = exp2_of(dlog * kLog2e);
  const float cut = fminf(fmaxf(ratio, 1.0f - p.clip_eps), 1.0f + p.clip_eps);
  const float surr = fminf(ratio * r.adv, cut * r.adv);
  const bool flow = (r.adv >= 0.0f && ratio <= 1.0f + p.clip_eps) || (r.adv < 0.0f && ratio >= 1.0f - p.clip_eps);
  const float loss = -surr + p.vf_coef * r.err * r.err - p.ent_coef * ent + (kl_coef != 0.0f ? kl_coef * kl : 0.0f);
#pragma unroll
  for (int j = 0; j < kParts; ++j) {
    const int q = lane % (kSums / kParts) + j * (kSums / kParts);
    float x = -surr;
    x = q == 1 ? r.err * r.err : x;
    x = q == 2 ? ent : x;
    x = q == 3 ? (fabsf(ratio - 1.0f) > p.clip_eps ? 1.0f : 0.0f) : x;
    x = q == 4 ? beyond(dlog, ratio) : x;
    x = q == 5 ? ratio : x;
    x = q == 7 ? kl : x;
    const double d = static_cast<double>(r.w) * x;
    part[j] += q == 6 ? (isfinite(loss) ? 0.0 : 1.0) : d;
  }
  return {flow ? -r.w * ratio * r.adv : 0.0f, r.w * p.ent_coef, r.w * kl_coef};
}

// The statistics from the eight sums.
__device__ __forceinline__ void write_stats(const double* x, float vf_coef, float ent_coef, float kl_coef, float* stats) {
  const double kl = kl_coef != 0.0f ? kl_coef * x[7] : 0.0;
  stats[0] = static_cast<float>(x[0] + vf_coef * x[1] - ent_coef * x[2] + kl);
  for (int k = 0; k < kSums; ++k) stats[k + 1] = static_cast<float>(x[k]);
}

// The block's sums, of which lane q of each team has the team's numbers q, q + G,
// ...; a call's only block writes the statistics itself.
template <int G, int kThreads, int kParts>
__device__ __forceinline__ void block_sums(const Loss& p, double (&part)[kParts]) {
  constexpr int kWaves = kThreads / 64;
  __shared__ double sums[kWaves][kSums];
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < kParts; ++j) {
#pragma unroll
    for (int d = G; d < 64; d *= 2) part[j] += __shfl_xor(part[j], d);
    if (lane < kSums / kParts) sums[threadIdx.x >> 6][lane + j * G] = part[j];
  }
  __syncthreads();
  // (a team of several waves has its numbers in the first)
  constexpr int kStep = G > 64 ? G / 64 : 1;
  double s = 0.0;
  if (threadIdx.x < kSums) {
#pragma unroll
    for (int k = 0; k < kWaves; k += kStep) s += sums[k][threadIdx.x];
    if (gridDim.x > 1) p.part[static_cast<size_t>(blockIdx.x) * kSums + threadIdx.x] = s;
  }
  if (gridDim.x > 1) return;
  __syncthreads();
  if (threadIdx.x < kSums) sums[0][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.x == 0) write_stats(sums[0], p.vf_coef, p.ent_coef, p.kl_coef, p.stats);
}

// ---------------------------------------------------- reductions of a team

// (of numbers that are no NaN, which fmaxf would bring into a form of its own first)
__device__ __forceinline__ float op_max(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }
__device__ __forceinline__ float op_sum(float a, float b) { return a + b; }

template <int ctrl>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), ctrl, 0xf, 0xf, true));
}

// Over 4, 8 or a row of 16 lanes or a wave, the result in each lane, in a fixed order.
template <int G, class Op>
__device__ __forceinline__ float lanes_reduce(float v, float id, Op op) {
  if (G > 16) return wave_reduce(v, id, op);
  v = op(v, moved<0xB1>(v));    // quad_perm [1, 0, 3, 2]
  v = op(v, moved<0x4E>(v));    // quad_perm [2, 3, 0, 1]
  if (G == 4) return v;
  if (G == 8) return op(v, moved<0x141>(v));  // row_half_mirror
  v = op(v, moved<0x124>(v));   // row_ror 4
  return op(v, moved<0x128>(v));  // row_ror 8
}

// Over the lanes of a row of 16 from this one on that have the same head (on[d]: the
// lane 2^d further is one), in a fixed order.
template <class Op>
__device__ __forceinline__ float rest_of_head(float v, const bool (&on)[4], float id, Op op) {
  float x = moved<0x101>(v);  // row_shl 1 (by all lanes)
  v = op(v, on[0] ? x : id);
  x = moved<0x102>(v);
  v = op(v, on[1] ? x : id);
  x = moved<0x104>(v);
  v = op(v, on[2] ? x : id);
  x = moved<0x108>(v);
  return op(v, on[3] ? x : id);
}

// What lane k of each wave of a team has of head k, joined over the team's
// waves (in every lane if there is one head).  n values; red [waves][8][n].
template <int G, int n, bool kOne, class Op>
__device__ __forceinline__ void team_join(float (&v)[n], Op op, float (*red)[kMaxHeads][n]) {
  if (G <= 64) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, k = kOne ? 0 : min(lane, kMaxHeads - 1);
  __syncthreads();  // (what the last call left has been read)
  if (lane < (kOne ? 1 : kMaxHeads))
#pragma unroll
    for (int q = 0; q < n; ++q) red[wave][lane][q] = v[q];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < n; ++q) v[q] = red[0][k][q];
  for (int w = 1; w < G / 64; ++w)
#pragma unroll
    for (int q = 0; q < n; ++q) v[q] = op(v[q], red[w][k][q]);
}

// ------------------------------------------------------- rows in registers

// A team of G lanes, I slots to a lane.  kOne: one head.  With several, lane k
// of each wave (of a row of 16 lanes) keeps head k's numbers, whose reductions take
// head after head; where a lane of 16 has one slot, a head's lanes follow each other,
// all heads are reduced at once and a head's first lane keeps its numbers.  kTiny: fewer
// logits than a slot holds.  kMore: the row (of one head) has more slots than the
// team holds; those behind are read twice, the second time from a cache.
template <typename E, int G, int I, bool kOne, bool kTiny, bool kAvail, bool kMore, int kThreads>
__global__ void __launch_bounds__(kThreads, !kOne && I > 2 && kThreads < 1024 ? 3 : 4) logits_slots(Loss p) {
  constexpr int V = Slot<E>::V, kTeams = kThreads / G, kWidth = G < 64 ? G : 64;
  constexpr bool kRuns = !kOne && G == 16 && I == 1;
  __shared__ float redm[G > 64 ? G / 64 : 1][kMaxHeads][2], reds[G > 64 ? G / 64 : 1][kMaxHeads][4];
  const int lane = threadIdx.x % G, hl = lane % kWidth;
  const int K = kOne ? 1 : p.heads.K, A = p.heads.A;
  const bool ref = p.has_ref != 0, some = kAvail && p.has_avail != 0;
  const float kl_coef = p.kl_coef;
  // the slots' heads and places
  int head[kOne ? 1 : I];
  Span<E> spans[kOne ? 1 : I];
  if (!kOne) {
#pragma unroll
    for (int i = 0; i < I; ++i) {
      int k = 0, s = i * G + lane, n = p.heads.off[1];
      for (; k < K - 1 && s >= (n + V - 1) / V; ++k) {
        s -= (n + V - 1) / V;
        n = p.heads.off[k + 2] - p.heads.off[k + 1];
      }
      head[i] = k;
      spans[i] = Span<E>(p.heads.off[k] + s * V, n - s * V, A);
    }
  }
  // the heads that the wave has slots of
  uint32_t here = 1;
  if (!kOne) {
    here = 0;
    for (int k = 0; k < K; ++k) {
      bool mine = false;
#pragma unroll
      for (int i = 0; i < (kOne ? 1 : I); ++i) mine |= head[i] == k && spans[i].have > 0;
      here |= __builtin_amdgcn_ballot_w64(mine) != 0 ? 1u << k : 0u;
    }
  }
  // the head whose numbers the lane keeps, and (kRuns) its first lane
  int mine = min(hl, K - 1), from = mine;
  bool keeps = hl < K, same[4];
  if (kRuns) {
    mine = head[0];
    from = 0;
    for (int k = 0; k < mine; ++k) from += (p.heads.off[k + 1] - p.heads.off[k] + V - 1) / V;
    keeps = hl == from;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int there = __shfl(mine, min(hl + (1 << d), 15), 16);  // (by all lanes: what a lane out of work has reads as 0)
      same[d] = hl + (1 << d) < 16 && there == mine;
    }
  }
  // what lane `from` of a head has, in the lanes of slot i
  const auto of_head = [&](auto v, int i) { return __shfl(v, kRuns ? from : head[i], kWidth); };
  const auto span = [&](int i) {
    if (!kOne) return spans[i];
    int l = lane;
    asm volatile("" : "+v"(l));  // (formed anew each time, not kept in registers)
    return Span<E>((i * G + l) * V, A - (i * G + l) * V, A);
  };
  const int my_off = p.heads.off[mine], my_size = p.heads.off[mine + 1] - my_off;
  double part[G < kSums ? kSums / G : 1] = {};
  // whether any of the wave's lanes has a slot i
  const int wave_lane = __builtin_amdgcn_readfirstlane(lane & ~63);
  const auto any = [&](int i) {
    if (I == 1) return true;
    return kOne ? (i * G + wave_lane) * V < A : __builtin_amdgcn_ballot_w64(spans[kOne ? 0 : i].have > 0) != 0;
  };
  const int team = G < 64 ? threadIdx.x / G : __builtin_amdgcn_readfirstlane(threadIdx.x / G);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kTeams + team, step = static_cast<int64_t>(gridDim.x) * kTeams;
  Ahead next = {0.0f, -1, 0};
  next.load(p, first, mine);
  for (int64_t n = first; n < p.N; n += step) {
    const E* z = static_cast<const E*>(p.z) + n * p.ldz;
    const E* y = static_cast<const E*>(p.y) + n * p.ldy;
    E* dz = static_cast<E*>(p.dz) + n * p.ldd;
    const uint8_t* av = p.avail + n * p.lda;
    const Ahead now = next;
    next.load(p, n + step, mine);
    Slot<E> zs[I], ys[I];
    if (now.w == 0.0f) {
#pragma unroll
      for (int i = 0; i < I; ++i) {
        zs[i] = {};
        const Span<E> at = span(i);
        zs[i].store(dz + at.col, at.skip, at.have);
      }
      if (kMore)
        for (int j = (I * G + lane) * V; j < A; j += G * V) {
          const Span<E> at(j, A - j, A);
          zs[0].store(dz + at.col, at.skip, at.have);
        }
      if (lane == 0) {
        if (p.has_ret) dz[A] = elem<E>::from_f32(0.0f);
        if (p.logp) p.logp[n] = 0.0f;
        if (p.kl) p.kl[n] = 0.0f;
      }
      continue;
    }
    uint32_t avs[I][2];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const Span<E> at = span(i);
      if (kTiny) {
        zs[i].load_some(z, A);
        ys[i].load_some(y, A);
      } else {
        zs[i].load(z + at.col);
        ys[i].load(y + at.col);
      }
      if (kAvail) at.template load<kTiny>(av, A, avs[i]);
    }
    // the action of the lane's head
    const bool active = (kRuns || keeps) && now.active != 0;
    int a = (kRuns || keeps) && now.a >= 0 && now.a < my_size ? now.a : -1;
    const float za = elem<E>::to_f32(z[my_off + max(a, 0)]);
    if (some && av[my_off + max(a, 0)] == 0) a = -1;
    Row r;
    r.load(p, n, z, now.w);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      if (any(i) && (some || !kOne || (i + 1) * G * V > A)) {
        uint32_t m[4];
        span(i).own(m);
        if (some) Span<E>::available(avs[i], m);
        zs[i].mask(m);
        ys[i].mask(m);
      }
    }
    // the slots behind those held, as they come
    float more_m[2] = {kLowest, kLowest};
    Sums more = {0.0f, 0.0f, 0.0f, 0.0f};
    if (kMore)
      for (int j = (I * G + lane) * V; j < A; j += G * V) {
        const Span<E> at(j, A - j, A);
        Slot<E> zx, yx;
        uint32_t ax[2];
        zx.load(z + at.col);
        yx.load(y + at.col);
        if (kAvail) at.template load<false>(av, A, ax);
        if (some || at.have < V) {
          uint32_t m[4];
          at.own(m);
          if (some) Span<E>::available(ax, m);
          zx.mask(m);
          yx.mask(m);
        }
        float mn[2] = {more_m[0], more_m[1]};
#pragma unroll
        for (int q = 0; q < V; ++q) mn[0] = fmaxf(mn[0], zx[q]);
        if (ref)
#pragma unroll
          for (int q = 0; q < V; ++q) mn[1] = fmaxf(mn[1], yx[q]);
        more.move(more_m[0], more_m[1], mn[0], mn[1]);
        more_m[0] = mn[0];
        more_m[1] = mn[1];
        zx.hold();
        yx.hold();
        if (ref)
#pragma unroll
          for (int q = 0; q < V; ++q) more.add(zx[q], mn[0], yx[q], mn[1]);
        else
#pragma unroll
          for (int q = 0; q < V; ++q) more.add(zx[q], mn[0]);
      }
    // the largest
    constexpr int J = kOne ? 1 : I;
    float zm[J], ym[J];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int to = kOne ? 0 : i;
      if (!kOne || i == 0) zm[to] = more_m[0], ym[to] = more_m[1];
      if (!any(i)) continue;
      zs[i].hold();
      ys[i].hold();
#pragma unroll
      for (int q = 0; q < V; ++q) zm[to] = fmaxf(zm[to], zs[i][q]);
      if (ref)
#pragma unroll
        for (int q = 0; q < V; ++q) ym[to] = fmaxf(ym[to], ys[i][q]);
    }
    float mm[2] = {kLowest, kLowest};
    if (kRuns) {
      mm[0] = of_head(rest_of_head(zm[0], same, kLowest, op_max), 0);
      if (ref) mm[1] = of_head(rest_of_head(ym[0], same, kLowest, op_max), 0);
    }
    for (int k = 0; k < K && !kRuns; ++k) {
      if (!((here >> k) & 1)) continue;
      float u[2] = {kLowest, kLowest};
#pragma unroll
      for (int i = 0; i < J; ++i)
        if (kOne || head[i] == k) u[0] = fmaxf(u[0], zm[i]), u[1] = fmaxf(u[1], ym[i]);
      u[0] = lanes_reduce<G>(u[0], kLowest, op_max);
      if (ref) u[1] = lanes_reduce<G>(u[1], kLowest, op_max);
      if (kOne || hl == k) mm[0] = u[0], mm[1] = u[1];
    }
    team_join<G, 2, kOne>(mm, op_max, redm);
    // the sums
    Sums sum[J];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const float m = kOne || kRuns ? mm[0] : of_head(mm[0], i), mr = kOne || kRuns ? mm[1] : of_head(mm[1], i);
      if (!kOne || i == 0) {
        sum[i] = more;
        if (kMore) sum[i].move(more_m[0], more_m[1], m, mr);
      }
      if (!any(i)) continue;
      Sums& to = sum[kOne ? 0 : i];
      zs[i].hold();
      ys[i].hold();
      if (ref)
#pragma unroll
        for (int q = 0; q < V; ++q) to.add(zs[i][q], m, ys[i][q], mr);
      else
#pragma unroll
        for (int q = 0; q < V; ++q) to.add(zs[i][q], m);
    }
    float all[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (kRuns) {
      all[0] = rest_of_head(sum[0].s, same, 0.0f, op_sum);
      all[1] = rest_of_head(sum[0].t, same, 0.0f, op_sum);
      if (ref) all[2] = rest_of_head(sum[0].v, same, 0.0f, op_sum), all[3] = rest_of_head(sum[0].sr, same, 0.0f, op_sum);
    }
    for (int k = 0; k < K && !kRuns; ++k) {
      if (!((here >> k) & 1)) continue;
      float u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < J; ++i)
        if (kOne || head[i] == k) u[0] += sum[i].s, u[1] += sum[i].t, u[2] += sum[i].v, u[3] += sum[i].sr;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < 2 || ref) u[q] = lanes_reduce<G>(u[q], 0.0f, op_sum);
      if (kOne || hl == k)
#pragma unroll
        for (int q = 0; q < 4; ++q) all[q] = u[q];
    }
    team_join<G, 4, kOne>(all, op_sum, reds);
    // one lane finishes a head; the row's numbers are sums over its heads
    const HeadStats h({all[0], all[1], all[2], all[3]}, ref);
    const bool use = active && h.some && keeps;
    float logpi = use ? (a < 0 ? -INFINITY : fmaf(-kLn2, h.ls, za - mm[0])) : 0.0f, ent = use ? h.S : 0.0f, kl = use ? h.D : 0.0f;
    bool on = use;
    if (kOne) {  // (lane 0 of each wave has the action)
      logpi = __shfl(logpi, 0, kWidth);
      ent = __shfl(ent, 0, kWidth);
      kl = __shfl(kl, 0, kWidth);
      on = __shfl(static_cast<int>(use), 0, kWidth) != 0;
      a = __shfl(a, 0, kWidth);
    } else {
      logpi = lanes_reduce<G>(logpi, 0.0f, op_sum);
      ent = lanes_reduce<G>(ent, 0.0f, op_sum);
      kl = lanes_reduce<G>(kl, 0.0f, op_sum);
    }
    const RowGrad g = row_loss(p, r, logpi, ent, kl, kl_coef, lane, part);
    const HeadGrad hg(g, h, mm[0], mm[1]);
    const int target = (kRuns || on) && a >= 0 ? (kOne ? 0 : my_off) + a : -(1 << 30);
#pragma unroll
    for (int i = 0; i < I; ++i) {
      if (!any(i)) continue;
      zs[i].hold();
      ys[i].hold();
      HeadGrad f = hg;
      int to = target;
      bool live = on;
      if (!kOne) {
        if (!kRuns) {
          f.m = of_head(mm[0], i);
          f.mr = of_head(mm[1], i);
          to = of_head(target, i);
        }
        f.ls = of_head(hg.ls, i);
        f.k0 = of_head(hg.k0, i);
        live = of_head(static_cast<int>(on), i) != 0;
        to = live ? to : -(1 << 30);
      }
      float out[V];
      if (!live) {
#pragma unroll
        for (int q = 0; q < V; ++q) out[q] = 0.0f;
      } else if (kl_coef != 0.0f) {
#pragma unroll
        for (int q = 0; q < V; ++q) out[q] = f(zs[i][q], ys[i][q]);
      } else {
#pragma unroll
        for (int q = 0; q < V; ++q) out[q] = f(zs[i][q]);
      }
      const Span<E> at = span(i);
      to -= at.col;
      if (static_cast<uint32_t>(to) < static_cast<uint32_t>(V))
#pragma unroll
        for (int q = 0; q < V; ++q) out[q] += q == to ? g.pg : 0.0f;
      Slot<E> o;
      o.set(out);
      o.store(dz + at.col, at.skip, at.have);
    }
    if (kMore)
      for (int j = (I * G + lane) * V; j < A; j += G * V) {
        const Span<E> at(j, A - j, A);
        float out[V] = {};
        if (on) {
          Slot<E> zx, yx;
          zx.load(z + at.col);
          yx.load(y + at.col);
          if (some) {
            uint32_t ax[2], m[4] = {~0u, ~0u, ~0u, ~0u};
            at.template load<false>(av, A, ax);
            Span<E>::available(ax, m);
            zx.mask(m);
            yx.mask(m);
          }
#pragma unroll
          for (int q = 0; q < V; ++q) out[q] = kl_coef != 0.0f ? hg(zx[q], yx[q]) : hg(zx[q]);
        }
        const int to = target - at.col;
        if (static_cast<uint32_t>(to) < static_cast<uint32_t>(V))
#pragma unroll
          for (int q = 0; q < V; ++q) out[q] += q == to ? g.pg : 0.0f;
        Slot<E> o;
        o.set(out);
        o.store(dz + at.col, at.skip, at.have);
      }
    if (lane == 0) {
      if (p.has_ret) dz[A] = elem<E>::from_f32(2.0f * p.vf_coef * r.w * r.err);
      if (p.logp) p.logp[n] = logpi;
      if (p.kl) p.kl[n] = kl;
    }
  }
  block_sums<G, kThreads>(p, part);
}

// --------------------------------------------------------- rows read twice

constexpr int kWide = 1024;  // lanes

// A block takes a row, head after head; U slots of a lane are in flight at once.
template <typename E>
__global__ void __launch_bounds__(kWide) logits_stream(Loss p) {
  constexpr int V = Slot<E>::V, U = 16 / V;
  __shared__ float redm[kWide / 64][kMaxHeads][2], reds[kWide / 64][kMaxHeads][4];
  const int lane = threadIdx.x, hl = lane & 63, K = p.heads.K, A = p.heads.A;
  const bool ref = p.has_ref != 0, some = p.has_avail != 0;
  const float kl_coef = p.kl_coef;
  double part[1] = {};
  for (int64_t n = blockIdx.x; n < p.N; n += gridDim.x) {
    const E* z = static_cast<const E*>(p.z) + n * p.ldz;
    const E* y = static_cast<const E*>(p.y) + n * p.ldy;
    E* dz = static_cast<E*>(p.dz) + n * p.ldd;
    const uint8_t* av = p.avail + n * p.lda;
    Row r;
    r.load(p, n, z, p.has_weight ? p.weight[n] : p.even);
    // head k's numbers, in lane k of each wave
    float m = 0.0f, mr = 0.0f, all[4] = {0.0f, 0.0f, 0.0f, 0.0f}, za = -INFINITY;
    int a = -1;
    bool active = false;
    for (int k = 0; k < K && !r.pad; ++k) {
      if (p.has_mask && p.mask[n * K + k] == 0) continue;
      const int o = p.heads.off[k], size = p.heads.off[k + 1] - o;
      float mk[2] = {kLowest, kLowest};
      Sums s = {0.0f, 0.0f, 0.0f, 0.0f};
      for (int j0 = lane * V; j0 < size; j0 += kWide * V * U) {
        Slot<E> zs[U], ys[U];
        uint32_t avs[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const Span<E> at(o + j0 + u * kWide * V, size - j0 - u * kWide * V, A);
          zs[u].load(z + at.col);
          ys[u].load(y + at.col);
          at.template load<false>(av, A, avs[u]);
        }
        float mn[2] = {mk[0], mk[1]};
#pragma unroll
        for (int u = 0; u < U; ++u) {
          zs[u].hold();
          const Span<E> at(o + j0 + u * kWide * V, size - j0 - u * kWide * V, A);
          if (some || at.have < V) {
            uint32_t m[4];
            at.own(m);
            if (some) Span<E>::available(avs[u], m);
            zs[u].mask(m);
            ys[u].mask(m);
          }
#pragma unroll
          for (int q = 0; q < V; ++q) mn[0] = fmaxf(mn[0], zs[u][q]);
          if (ref)
#pragma unroll
            for (int q = 0; q < V; ++q) mn[1] = fmaxf(mn[1], ys[u][q]);
        }
        s.move(mk[0], mk[1], mn[0], mn[1]);
        mk[0] = mn[0];
        mk[1] = mn[1];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          zs[u].hold();
          ys[u].hold();
          if (ref)
#pragma unroll
            for (int q = 0; q < V; ++q) s.add(zs[u][q], mk[0], ys[u][q], mk[1]);
          else
#pragma unroll
            for (int q = 0; q < V; ++q) s.add(zs[u][q], mk[0]);
        }
      }
      float mm[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) mm[q] = wave_reduce(mk[q], kLowest, op_max);
      team_join<kWide, 2, true>(mm, op_max, redm);
      s.move(mk[0], mk[1], mm[0], mm[1]);
      float u[4] = {s.s, s.t, s.v, s.sr};
#pragma unroll
      for (int q = 0; q < 4; ++q) u[q] = wave_reduce(u[q], 0.0f, op_sum);
      team_join<kWide, 4, true>(u, op_sum, reds);
      if (hl == k) {
        m = mm[0];
        mr = mm[1];
#pragma unroll
        for (int q = 0; q < 4; ++q) all[q] = u[q];
        active = true;
        a = p.act[n * K + k];
        if (a < 0 || a >= size || (some && av[o + a] == 0))
          a = -1;
        else
          za = elem<E>::to_f32(z[o + a]);
      }
    }
    const HeadStats h({all[0], all[1], all[2], all[3]}, ref);
    const bool use = active && h.some;
    const float logpi = wave_reduce(use ? (a < 0 ? -INFINITY : fmaf(-kLn2, h.ls, za - m)) : 0.0f, 0.0f, op_sum);
    const float ent = wave_reduce(use ? h.S : 0.0f, 0.0f, op_sum), kl = wave_reduce(use ? h.D : 0.0f, 0.0f, op_sum);
    RowGrad g = {0.0f, 0.0f, 0.0f};
    if (!r.pad) g = row_loss(p, r, logpi, ent, kl, kl_coef, lane, part);
    const HeadGrad hg(g, h, m, mr);
    for (int k = 0; k < K; ++k) {
      const int o = p.heads.off[k], size = p.heads.off[k + 1] - o;
      HeadGrad f;
      f.m = __shfl(m, k);
      f.mr = __shfl(mr, k);
      f.ls = __shfl(hg.ls, k);
      f.k0 = __shfl(hg.k0, k);
      f.kd = hg.kd;
      f.ky = hg.ky;
      const int target = __shfl(use && a >= 0 ? a + p.heads.off[min(hl, K - 1)] : -(1 << 30), k);
      const bool live = __shfl(static_cast<int>(use), k) != 0;
      for (int j0 = lane * V; j0 < size; j0 += kWide * V * U) {
        Slot<E> zs[U], ys[U];
        uint32_t avs[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const Span<E> at(o + j0 + u * kWide * V, size - j0 - u * kWide * V, A);
          zs[u].load(z + at.col);
          ys[u].load(y + at.col);
          at.template load<false>(av, A, avs[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const Span<E> at(o + j0 + u * kWide * V, size - j0 - u * kWide * V, A);
          float out[V] = {};
          if (live) {
            zs[u].hold();
            if (some) {
              uint32_t m[4] = {~0u, ~0u, ~0u, ~0u};
              Span<E>::available(avs[u], m);
              zs[u].mask(m);
              ys[u].mask(m);
            }
#pragma unroll
            for (int q = 0; q < V; ++q) out[q] = kl_coef != 0.0f ? f(zs[u][q], ys[u][q]) : f(zs[u][q]);
          }
          const int to = target - at.col;
          if (static_cast<uint32_t>(to) < static_cast<uint32_t>(V))
#pragma unroll
            for (int q = 0; q < V; ++q) out[q] += q == to ? g.pg : 0.0f;
          Slot<E> d;
          d.set(out);
          d.store(dz + at.col, at.skip, at.have);
        }
      }
    }
    if (lane == 0) {
      if (p.has_ret) dz[A] = elem<E>::from_f32(r.pad ? 0.0f : 2.0f * p.vf_coef * r.w * r.err);
      if (p.logp) p.logp[n] = logpi;
      if (p.kl) p.kl[n] = kl;
    }
  }
  block_sums<kWide, kWide>(p, part);
}

// The statistics from the blocks' sums, in a fixed order: thread t takes sum t
// mod 8 of blocks t / 8, t / 8 + 128, ...
__global__ void __launch_bounds__(1024) logits_stats(int blocks, const double* __restrict__ part, float vf_coef,
                                                     float ent_coef, float kl_coef, float* __restrict__ stats) {
  __shared__ double red[16][kSums];
  const int q = threadIdx.x % kSums, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double s = 0.0;
#pragma unroll 8
  for (int b = threadIdx.x / kSums; b < blocks; b += 128) s += part[b * kSums + q];
#pragma unroll
  for (int d = kSums; d < 64; d *= 2) s += __shfl_xor(s, d);
  if (lane < kSums) red[wave][lane] = s;
  __syncthreads();
  if (threadIdx.x < kSums) {
#pragma unroll
    for (int k = 1; k < 16; ++k) s += red[k][threadIdx.x];
    red[0][threadIdx.x] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) write_stats(red[0], vf_coef, ent_coef, kl_coef, stats);
}

// How a call's rows are taken, by the slots of 16 bytes that a row has.  Narrow
// rows in teams of 4, 8 or 16 lanes, whose reductions cost two to four steps for all of a wave's rows;
// wider ones in as few lanes as hold them, up to a block.  Times in us of one head and of
// two, in bf16, in the form taken and, after the stroke, in the next one:
//
//   300000 x 18 (four lanes) 26 | 80 in 16                30000 x 60 (eight) 14 | 16 in 16
//   30000 x 74 in 4 heads (one slot a lane) 17.5 | 22     10000 x 1700 37, 46 | 53, 64
//   20000 x 220 (two)  17, 18 | 30, 33                    6000 x 3600  47, 56 | 50, 68
//   20000 x 400 (four) 22, 27 | 29, 33 in whole waves     4000 x 7000  50, 65 | 54, 118
//   20000 x 900 40, 48 | 44, 59                           2000 x 15000 52, 89 | 58, 106
//   6000 x 2600 36, 46 | 41, 51                           8192 x 32000 334 | 438
//
// (measured with one instruction a logit less than it takes now: both sides are up to 2 % longer;
// eight slots in 16 lanes: 20000 x 900 38, 81, 5000 x 500 in fp32 17, in whole waves 15;
// four in 128: 6000 x 3600 44, 55, 5000 x 1719 in eight heads in fp32 53, two in 256 51).
// Rows of one head that a block does not hold keep 8 slots a lane and read the others
// twice: 1003 x 50257 in fp32 178, read twice as a whole 192, 2000 x 128000 430 and 445.
struct Form {
  int teams, threads, blocks;  // teams and threads of a block, blocks at most
  void (*kernel)(Loss);
};

template <typename E, int G, int I, bool kOne, bool kTiny = false, bool kAvail = true, bool kMore = false>
Form slots_form(int N) {
  constexpr int kThreads = G <= 64 ? 256 : G;  // (waves of a team meet at barriers, which are a block's)
  // a few rows: one block takes them all and writes the statistics too (60 rows of 74: 9.8 us, in two launches 11.6)
  if constexpr (G <= 64)
    if (N > kThreads / G && N <= 1024 / G) return {1024 / G, 1024, 1, logits_slots<E, G, I, kOne, kTiny, kAvail, kMore, 1024>};
  // (blocks: 32768 rows of 74 with 1024 22.5 us, with 2048 23.4; 300000 of 18 26.1 and 27.4, with 512 31.4)
  return {kThreads / G, kThreads, (G <= 16 ? 1024 : 2048) * 256 / kThreads, logits_slots<E, G, I, kOne, kTiny, kAvail, kMore, kThreads>};
}
template <typename E, int G, int I>
Form slots_form(int N, bool one) {
  return one ? slots_form<E, G, I, true>(N) : slots_form<E, G, I, false>(N);
}

template <typename E, int G, bool kMore = false>
Form wide_form(int N, bool avail) {
  return avail ? slots_form<E, G, 8, true, false, true, kMore>(N) : slots_form<E, G, 8, true, false, false, kMore>(N);
}

template <typename E>
Form form_of(int N, const HeadsMeta& hm, bool avail) {
  constexpr int V = Slot<E>::V;
  int slots = 0;
  for (int k = 0; k < hm.K; ++k) slots += (hm.off[k + 1] - hm.off[k] + V - 1) / V;
  const bool one = hm.K == 1;
  if (hm.A < V) return one ? slots_form<E, 4, 1, true, true>(N) : slots_form<E, 16, 1, false, true>(N);
  if (slots <= 4 && one) return slots_form<E, 4, 1, true>(N);
  if (slots <= 8 && one) return slots_form<E, 8, 1, true>(N);
  if (slots <= 16) return slots_form<E, 16, 1>(N, one);
  if (slots <= 32) return slots_form<E, 16, 2>(N, one);
  if (slots <= 64) return slots_form<E, 16, 4>(N, one);
  if (slots <= 128) return slots_form<E, 64, 2>(N, one);
  if (slots <= 256) return slots_form<E, 64, 4>(N, one);
  if (slots <= 384) return slots_form<E, 128, 3>(N, one);
  if (slots <= 512) return slots_form<E, 256, 2>(N, one);
  if (slots <= 1024) return slots_form<E, 256, 4>(N, one);
  if (slots <= 2048) return one ? wide_form<E, 256>(N, avail) : slots_form<E, 512, 4, false>(N);
  if (slots <= 4096 && one) return wide_form<E, 512>(N, avail);
  if (slots <= 8192 && one) return wide_form<E, 1024>(N, avail);
  if (one) return wide_form<E, 1024, true>(N, avail);
  return {1, kWide, 512, logits_stream<E>};
}
Form form_of(o5_dtype dt, int N, const HeadsMeta& hm, bool avail) {
  return dt == O5_BF16 ? form_of<uint16_t>(N, hm, avail) : form_of<float>(N, hm, avail);
}

int blocks_of(const Form& f, int N) { return static_cast<int>(std::min<long long>((N + f.teams - 1ll) / f.teams, f.blocks)); }

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
  return std::max<size_t>(256, static_cast<size_t>(blocks_of(form_of(dt, N, hm, true), N)) * kSums * sizeof(double));
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
  const uint8_t* bytes = static_cast<const uint8_t*>(logits);  // (a row of logits has more of them than logits)
  p.z = logits, p.y = ref ? ref : logits, p.dz = dlogits;
  p.ldz = ldl, p.ldy = ref ? ldr : ldl, p.ldd = ldd, p.lda = avail ? A : ldl * dtype_size(dt);
  p.act = act, p.logp_old = logp_old, p.adv = adv, p.ret = ret ? ret : logp_old, p.weight = weight ? weight : logp_old;
  p.mask = head_mask ? head_mask : reinterpret_cast<const uint8_t*>(act), p.avail = avail ? avail : bytes;
  p.has_ref = ref != nullptr, p.has_ret = ret != nullptr, p.has_weight = weight != nullptr;
  p.has_mask = head_mask != nullptr, p.has_avail = avail != nullptr;
  p.logp = logp, p.kl = kl, p.stats = stats, p.part = static_cast<double*>(ws), p.N = N;
  p.clip_eps = hp.clip_eps, p.vf_coef = hp.vf_coef, p.ent_coef = hp.ent_coef, p.kl_coef = ref ? kl_coef : 0.0f;
  p.even = static_cast<float>(1.0 / N);
  const Form f = form_of(dt, N, p.heads, avail != nullptr);
  const int blocks = blocks_of(f, N);
  hipLaunchKernelGGL(f.kernel, dim3(blocks), dim3(f.threads), 0, as_stream(stream), p);
  if (blocks > 1)
    hipLaunchKernelGGL(logits_stats, dim3(1), dim3(1024), 0, as_stream(stream), blocks, p.part, hp.vf_coef, hp.ent_coef,
                       p.kl_coef, stats);
  return check_launch(fn);
}
