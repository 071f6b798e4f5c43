// A linear recurrence whose decay and input are gated by the input,
// o5_gatedrec_*.
//
//   g = sigmoid(r), o = sigmoid(i), log a = -c softplus(lam) g
//   h_t = a_t (1 - reset_t) h_{t-1} + beta_t o_t x_t,   beta = sqrt(1 - a^2)
//
// Every channel is a recurrence of its own.  Where samples and channels fill the
// chip, a lane takes two neighbouring channels and walks the steps, the rows of
// some steps in flight while it works on those before.  Where they are fewer,
// short sequences go to blocks of 16 waves with 8 steps each of the same 64
// channels: each forms what its steps leave of the state that enters them and what
// they add, the block joins these in LDS, and each wave finishes its steps from the
// state that enters them, with the gates still in registers.  Long sequences of
// few channels are cut into segments: one launch forms what each segment leaves and
// adds, one joins them if they are many, and one runs the segments.
//
// w = 1 - a is formed without the cancellation near a = 1, and the state is
// taken on as h - w h: a rounded to 24 bits would be off by 2^-25 of itself in
// every step, which over the 1/w steps that a state lasts grows to 2^-25 / w.
// Away from 1 it is taken on as a h, since 1 - w keeps nothing of a small a, to
// which the gates' and the rates' gradients are proportional.  beta is sqrt(w (2 - w)).
//
// HBM-bound by its bytes, with 39 instructions an element forward, 6 of them at half
// rate, that keep the vector units busy for 70 to 80 % of the time.  bf16, D = 4096 unless
// said: T = 256, B = 128 forward for training 250 us, 4.6 TB/s; B = 64 backward 203 us,
// 4.8 TB/s; T = 10007, B = 1, D = 2048 forward 72 us, 2.3 TB/s, since a sequence cut in
// segments computes every step twice; a token of 4096 samples 56 us, 4.8 TB/s; of one
// 6.2 us, which is the call and the launch.
#include "common.h"

namespace o5 {
namespace {

constexpr int kMark = 8;        // steps between the states that the forward pass leaves for the backward pass
constexpr float kMost = 1e38f;  // the largest rate: times a gate that is 0 it is 0
constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596299e-8f;

// An array of rows: the row of step t and sample b is step t + ld b bytes from
// p.  A call goes out in launches of so many samples that a lane's place within
// a step is below 2^32 bytes, while step t is the same for all lanes.
struct Rows {
  char* p;
  uint64_t step;
  uint32_t ld;
};

struct Rec {  // a launch's arrays; the states' pointers are those of its first sample
  Rows x, r, i, h, dh, dx, dr, di;
  const float *lam, *h0, *dhT;
  const uint8_t* reset;
  float *hT, *marks, *dh0, *part;
  float *keep, *add;  // [segments - 1, states]: what a segment leaves of a state (-1: cut off), and what it adds
  float* enter;       // [segments - 1, states]: the states that enter segments 1, 2, ..., or NULL: keep and add give them
  uint64_t states;    // B D of the whole call
  int T, B, nb, D, len;  // len: steps of a segment
  float c;
};

typedef float f2_t __attribute__((ext_vector_type(2)));

// Two neighbouring channels.
template <typename E> struct Pair;
template <> struct Pair<float> {
  f2_t v;
  __device__ __forceinline__ float operator[](int j) const { return v[j]; }
  __device__ __forceinline__ Pair() = default;
  __device__ __forceinline__ Pair(float a, float b) : v{a, b} {}
};
template <> struct Pair<uint16_t> {
  uint32_t v;
  __device__ __forceinline__ float operator[](int j) const { return __uint_as_float(j ? v & 0xffff0000u : v << 16); }
  __device__ __forceinline__ Pair() = default;
  __device__ __forceinline__ Pair(float a, float b) : v(f32x2_to_bf16x2(a, b)) {}
};
template <typename E>
__device__ __forceinline__ Pair<E> load(const Rows& a, int t, uint32_t at) {
  return *reinterpret_cast<const Pair<E>*>(a.p + t * a.step + at);
}
template <typename E>
__device__ __forceinline__ void store(const Rows& a, int t, uint32_t at, float u, float v) {
  *reinterpret_cast<Pair<E>*>(a.p + t * a.step + at) = Pair<E>(u, v);
}

__device__ __forceinline__ float sigmoid2(float x) {  // 1 / (1 + e^-x)
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x));
}
// log(1 + e^x): with u = e^-|x| and s = u / (2 + u), at most 1/3, log(1 + u) is twice the
// series s + s^3/3 + s^5/5 + ..., whose terms from s^15 on are 1e-8 of it (5 steps of
// 2^-24 off at most).  |x| in binary logs is taken in two parts: its rounding would be
// |x| 2^-24 of u.  A lane's two rates take 50 instructions, with expf and log1pf 230
// (a token of 4096 x 4096 59 -> 57.5 us).
__device__ __forceinline__ float softplus(float x) {
  const float b = -fabsf(x) * kLog2e, rest = fmaf(-fabsf(x), kLog2eRest, fmaf(-fabsf(x), kLog2e, -b));
  const float e = __builtin_amdgcn_exp2f(b), u = fabsf(x) < 100.0f ? fmaf(e, 0.693147181f * rest, e) : 0.0f;
  const float s = u * __builtin_amdgcn_rcpf(2.0f + u), q = s * s;
  float y = fmaf(q, 1.0f / 13.0f, 1.0f / 11.0f);
  y = fmaf(q, y, 1.0f / 9.0f);
  y = fmaf(q, y, 1.0f / 7.0f);
  y = fmaf(q, y, 1.0f / 5.0f);
  y = fmaf(q, y, 1.0f / 3.0f);
  y = fmaf(q, y, 1.0f);
  return (x < 0.0f ? 0.0f : x) + 2.0f * s * y;  // (a NaN stays one: the state of a lost rate must not look like one that is kept)
}
__device__ __forceinline__ float rate_of(float c, float lam) {
  const float rate = c * softplus(lam);
  return rate > kMost ? kMost : rate;  // (a NaN stays one)
}

// The decay a = 2^-y, y >= 0, as one number that keeps the last digits of a and of w = 1 - a:
// w, below 0.3 binary logs of e a polynomial, 2e-8 of the value off (a minimax fit; the
// difference would be 3e-7 off), and from there on -a, told by its sign.
struct Decay {
  float s;
  bool near;
  __device__ __forceinline__ explicit Decay(float y) {
    const float a = __builtin_amdgcn_exp2f(-y);
    float q = fmaf(y, 0x1.34893cp-10f, -0x1.3941b2p-7f);
    q = fmaf(y, q, 0x1.c69daep-5f);
    q = fmaf(y, q, -0x1.ebfb9ep-3f);
    q = fmaf(y, q, 0x1.62e430p-1f);
    near = y < 0.3f * kLog2e;
    s = near ? y * q : -a;
  }
  __device__ __forceinline__ Decay(float s_, bool near_) : s(s_), near(near_) {}
  __device__ __forceinline__ float a() const { return near ? 1.0f - s : -s; }
  __device__ __forceinline__ float beta2() const { return __builtin_fmaf(-s, s, near ? s + s : 1.0f); }  // 1 - a^2
  __device__ __forceinline__ float carried(float h) const { return __builtin_fmaf(-s, h, near ? h : 0.0f); }  // a h
};
__device__ __forceinline__ Decay kept(float s) { return Decay(s, __float_as_int(s) >= 0); }  // (-0 is an a of 0)

// What a step takes in, and its state from the one before: rounded the same in
// every kernel (no product is joined with the sum), so that single tokens give
// the bits of a sequence that is not cut.
__device__ __forceinline__ float taken_in(float beta2, float o, float x) {
#pragma clang fp contract(off)
  return __builtin_amdgcn_sqrtf(beta2) * (o * x);
}
__device__ __forceinline__ float next_state(float h, const Decay& a, float v) {
#pragma clang fp contract(off)
  return a.carried(h) + v;
}
__device__ __forceinline__ float next_state(float h, float y, float i, float x) {  // y: the decay in binary logs
  const Decay a(y);
  return next_state(h, a, taken_in(a.beta2(), sigmoid2(i), x));
}

// One step's gradients, from G, that of its state.
struct Grad {
  float dx, dr, di, e;  // e = G d(log a) log a
  __device__ __forceinline__ Grad(float G, float rate, float x, float g, float o, const Decay& d, float v, float before) {
    const float a = d.a();
    // 1 / beta; log a / beta goes to 0 with log a
    const float ib = v < 0x1p-126f ? 0.0f : __builtin_amdgcn_rsqf(v);
    e = G * (a * (-rate * g) * fmaf(-a * ib, o * x, before));
    dx = G * (v * ib) * o;
    dr = fmaf(-e, g, e);
    di = dx * x * (1.0f - o);
  }
};

// A lane's C neighbouring channels of one sample, n-th of its launch, and where
// they lie.
template <int C>
struct Place {
  uint32_t b, d, at;
  bool on;
  float rate[C];  // c softplus(lam)
  __device__ __forceinline__ Place(const Rec& p, uint32_t n) {
    const uint32_t most = static_cast<uint32_t>(p.nb) * (p.D / C), per = p.D / C;
    on = n < most;
    n = min(n, most - 1);
    b = n / per;
    d = (n - b * per) * C;
    at = b * p.D + d;  // within the states
#pragma unroll
    for (int j = 0; j < C; ++j) rate[j] = rate_of(p.c, p.lam[d + j]);
  }
  template <typename E>
  __device__ __forceinline__ uint32_t in(const Rows& a) const {
    return b * a.ld + d * sizeof(E);
  }
};

__device__ __forceinline__ f2_t state_in(const float* p, uint32_t at) { return *reinterpret_cast<const f2_t*>(p + at); }
__device__ __forceinline__ void state_out(float* p, uint32_t at, float a, float b) {
  *reinterpret_cast<f2_t*>(p + at) = f2_t{a, b};
}

// A segment's effect on a state.
__device__ __forceinline__ float pass(float keep, float add, float h) { return keep < 0.0f ? add : fmaf(keep, h, add); }
__device__ __forceinline__ f2_t pass(const Rec& p, uint64_t seg, uint32_t at, f2_t h) {
  const f2_t keep = state_in(p.keep + seg * p.states, at), add = state_in(p.add + seg * p.states, at);
  return f2_t{pass(keep[0], add[0], h[0]), pass(keep[1], add[1], h[1])};
}

// The inputs of U steps; those from `end` on repeat the last and are not used.
template <typename E, int U>
struct Steps {
  Pair<E> x[U], r[U], i[U];
  uint8_t cut[U];
  __device__ __forceinline__ void load(const Rec& p, uint32_t x_at, uint32_t r_at, uint32_t i_at, uint32_t b, int t0, int end) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int t = min(t0 + k, end - 1);
      x[k] = o5::load<E>(p.x, t, x_at);
      r[k] = o5::load<E>(p.r, t, r_at);
      i[k] = o5::load<E>(p.i, t, i_at);
      cut[k] = p.reset ? p.reset[static_cast<uint64_t>(t) * p.B + b] : 0;
    }
  }
};

// Forward, two channels to a lane, over segment blockIdx.y.  kSum: only what the segment leaves of the
// state that enters it, and what it adds.  Four steps are in flight while four are worked on
// (T = 256, B = 128, D = 4096 250 us; eight 264; one channel to a lane is no faster).
template <typename E, bool kSum>
__global__ void __launch_bounds__(256) gatedrec_fwd(Rec p) {
  constexpr int U = 4;
  const Place<2> l(p, blockIdx.x * blockDim.x + threadIdx.x);
  if (!l.on) return;
  const uint32_t x_at = l.in<E>(p.x), r_at = l.in<E>(p.r), i_at = l.in<E>(p.i), h_at = l.in<E>(p.h);
  const float rate[2] = {kLog2e * l.rate[0], kLog2e * l.rate[1]};
  const uint64_t seg = blockIdx.y;
  const int begin = seg * p.len, end = min(begin + p.len, p.T);
  f2_t h = {0.0f, 0.0f}, sum = {0.0f, 0.0f};
  bool whole = true;
  if (!kSum && seg > 0 && p.enter) {
    h = state_in(p.enter + (seg - 1) * p.states, l.at);
  } else if (!kSum) {
    if (p.h0) h = state_in(p.h0, l.at);
#pragma unroll 4
    for (uint64_t s = 0; s < seg; ++s) h = pass(p, s, l.at, h);
  }
  Steps<E, U> next;
  next.load(p, x_at, r_at, i_at, l.b, begin, end);
  for (int t0 = begin; t0 < end; t0 += U) {
    const Steps<E, U> s = next;
    next.load(p, x_at, r_at, i_at, l.b, t0 + U, end);
    if (!kSum && p.marks && t0 % kMark == 0) state_out(p.marks + (t0 / kMark) * p.states, l.at, h[0], h[1]);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (t0 + k >= end) break;
      if (s.cut[k]) {
        h = f2_t{0.0f, 0.0f};
        whole = false;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float y = rate[j] * sigmoid2(s.r[k][j]);
        if (kSum) sum[j] += y;
        h[j] = next_state(h[j], y, s.i[k][j], s.x[k][j]);
      }
      if (!kSum) store<E>(p.h, t0 + k, h_at, h[0], h[1]);
    }
  }
  if (kSum) {
    state_out(p.keep + seg * p.states, l.at, whole ? __builtin_amdgcn_exp2f(-sum[0]) : -1.0f,
              whole ? __builtin_amdgcn_exp2f(-sum[1]) : -1.0f);
    state_out(p.add + seg * p.states, l.at, h[0], h[1]);
  } else if (p.hT && end == p.T) {
    state_out(p.hT, l.at, h[0], h[1]);
  }
}

// The states that enter the segments behind the first, from the one that
// enters the first (forward), or those that enter the ones before the last from
// the right.  A block takes 64 channels; each of its 16 waves joins a run of
// segments first, then all runs before its own.
__global__ void __launch_bounds__(1024) gatedrec_join(const float* __restrict__ keep, const float* __restrict__ add,
                                                      const float* __restrict__ first, float* __restrict__ enter, int n,
                                                      uint64_t states, bool back) {
  __shared__ float ks[16][64], as[16][64];
  const int c = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t at = static_cast<uint64_t>(blockIdx.x) * 64 + c;
  const bool on = at < states;
  const int run = (n + 15) / 16, from = min(wave * run, n), to = min(from + run, n);
  const auto row = [&](int s) { return (back ? n - 1 - s : s) * states + at; };
  float k = 1.0f, a = 0.0f;
  if (on)
#pragma unroll 8
    for (int s = from; s < to; ++s) {
      const float ks = keep[row(s)], as = add[row(s)];
      a = pass(ks, as, a);
      k = ks < 0.0f || k < 0.0f ? -1.0f : k * ks;
    }
  ks[wave][c] = k;
  as[wave][c] = a;
  __syncthreads();
  if (!on) return;
  float h = first ? first[at] : 0.0f;
  for (int w = 0; w < wave; ++w) h = pass(ks[w][c], as[w][c], h);
#pragma unroll 8
  for (int s = from; s < to; ++s) {
    h = pass(keep[row(s)], add[row(s)], h);
    enter[row(s)] = h;
  }
}

// ------------------------------------------------ blocks of 64 channels

constexpr int kWavesOf = 16;  // of a block at most, each kMark steps at a time

template <typename E>
__device__ __forceinline__ float one(const Rows& a, int t, uint32_t at) {
  return elem<E>::to_f32(*reinterpret_cast<const E*>(a.p + t * a.step + at));
}
template <typename E>
__device__ __forceinline__ void put(const Rows& a, int t, uint32_t at, float v) {
  *reinterpret_cast<E*>(a.p + t * a.step + at) = elem<E>::from_f32(v);
}

// What the block's waves leave of a state and add, in the order in which a
// state passes them; two buffers, so that one barrier keeps a wave that is a
// round ahead from what the others still read.
struct Board {
  float keep[2][kWavesOf][64], add[2][kWavesOf][64];
};

// The state s passes the block's waves 0, 1, ... (or, back, ..., 1, 0); what
// enters wave `wave` is left in `in`.
__device__ __forceinline__ float pass_block(const Board& m, int buf, int waves, int wave, int lane, bool back, float s,
                                            float* in) {
#pragma unroll 4
  for (int q = 0; q < waves; ++q) {
    const int w = back ? waves - 1 - q : q;
    *in = w == wave ? s : *in;
    s = pass(m.keep[buf][w][lane], m.add[buf][w][lane], s);
  }
  return s;
}

// Forward.
template <typename E>
__global__ void __launch_bounds__(64 * kWavesOf) gatedrec_fwd_block(Rec p) {
  constexpr int U = kMark;
  __shared__ Board board;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Place<1> l(p, blockIdx.x * 64 + lane);
  const uint32_t x_at = l.in<E>(p.x), r_at = l.in<E>(p.r), i_at = l.in<E>(p.i), h_at = l.in<E>(p.h);
  const float rate = kLog2e * l.rate[0];
  const int end = p.T, round = waves * U;
  float h = p.h0 ? p.h0[l.at] : 0.0f;
  float x[U], r[U], i[U];
  uint32_t cut = 0;
  const auto fetch = [&](int t0) {
    cut = 0;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int t = min(t0 + k, end - 1);
      x[k] = one<E>(p.x, t, x_at);
      r[k] = one<E>(p.r, t, r_at);
      i[k] = one<E>(p.i, t, i_at);
    }
    if (p.reset)
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int t = min(t0 + k, end - 1);
        cut |= t0 + k < end && p.reset[static_cast<uint64_t>(t) * p.B + l.b] != 0 ? 1u << k : 0u;
      }
  };
  fetch(wave * U);
  int buf = 0;
  for (int c0 = 0; c0 < end; c0 += round, buf ^= 1) {
    const int t0 = c0 + wave * U;
    float s[U], v[U], e = 0.0f, y = 0.0f;
    const uint32_t off = cut;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const bool there = t0 + k < end;
      const float yk = there ? rate * sigmoid2(r[k]) : 0.0f;
      const Decay d(yk);
      s[k] = d.s;
      v[k] = there ? taken_in(d.beta2(), sigmoid2(i[k]), x[k]) : 0.0f;
      if ((off >> k) & 1) e = 0.0f;
      e = next_state(e, d, v[k]);
      y += yk;
    }
    if (c0 + round < end) fetch(t0 + round);
    board.keep[buf][wave][lane] = off ? -1.0f : __builtin_amdgcn_exp2f(-y);
    board.add[buf][wave][lane] = e;
    __syncthreads();
    float in = 0.0f;
    h = pass_block(board, buf, waves, wave, lane, false, h, &in);
    if (t0 >= end) continue;
    if (p.marks && l.on) p.marks[(t0 / kMark) * p.states + l.at] = in;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (t0 + k >= end) break;
      if ((off >> k) & 1) in = 0.0f;
      in = next_state(in, kept(s[k]), v[k]);
      if (l.on) put<E>(p.h, t0 + k, h_at, in);
    }
    if (p.hT && t0 + U >= p.T && l.on) p.hT[l.at] = in;
  }
}

// Backward.
template <typename E>
__global__ void __launch_bounds__(64 * kWavesOf) gatedrec_bwd_block(Rec p) {
  constexpr int U = kMark;
  __shared__ Board board;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Place<1> l(p, blockIdx.x * 64 + lane);
  const uint32_t x_at = l.in<E>(p.x), r_at = l.in<E>(p.r), i_at = l.in<E>(p.i), d_at = l.in<E>(p.dh);
  const uint32_t dx_at = l.in<E>(p.dx), dr_at = l.in<E>(p.dr), di_at = l.in<E>(p.di);
  const int end = p.T, round = waves * U;
  float G = p.dhT ? p.dhT[l.at] : 0.0f, sum = 0.0f;
  int buf = 0;
  for (int c0 = (end - 1) / round * round; c0 >= 0; c0 -= round, buf ^= 1) {
    const int t0 = c0 + wave * U;
    float x[U], g[U], o[U], dh[U], s[U], beta2[U], before[U];
    uint32_t cut = 0;
    float h = p.marks[(min(t0, end - 1) / kMark) * p.states + l.at];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int t = min(t0 + k, end - 1);
      g[k] = one<E>(p.r, t, r_at);
      x[k] = one<E>(p.x, t, x_at);
      o[k] = one<E>(p.i, t, i_at);
      dh[k] = one<E>(p.dh, t, d_at);
    }
    if (p.reset)
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int t = min(t0 + k, end - 1);
        cut |= t0 + k < end && p.reset[static_cast<uint64_t>(t) * p.B + l.b] != 0 ? 1u << k : 0u;
      }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if ((cut >> k) & 1) h = 0.0f;
      before[k] = h;
      g[k] = sigmoid2(g[k]);
      o[k] = sigmoid2(o[k]);
      const Decay d(kLog2e * l.rate[0] * g[k]);
      s[k] = d.s;
      beta2[k] = d.beta2();
      h = next_state(h, d, taken_in(beta2[k], o[k], x[k]));
    }
    float e = 0.0f, y = 0.0f;
    bool open = true;
#pragma unroll
    for (int k = U - 1; k >= 0; --k) {
      if (t0 + k >= end) continue;
      e += dh[k];
      e = kept(s[k]).carried(e);
      y += g[k];
      if ((cut >> k) & 1) {
        e = 0.0f;
        open = false;
      }
    }
    board.keep[buf][wave][lane] = open ? __builtin_amdgcn_exp2f(-kLog2e * l.rate[0] * y) : -1.0f;
    board.add[buf][wave][lane] = e;
    __syncthreads();
    float in = 0.0f;
    G = pass_block(board, buf, waves, wave, lane, true, G, &in);
    if (t0 >= end) continue;
#pragma unroll
    for (int k = U - 1; k >= 0; --k) {
      if (t0 + k >= end) continue;
      const Decay a = kept(s[k]);
      const Grad d(in += dh[k], l.rate[0], x[k], g[k], o[k], a, beta2[k], before[k]);
      sum += d.e;
      in = (cut >> k) & 1 ? 0.0f : a.carried(in);
      if (l.on) {
        put<E>(p.dx, t0 + k, dx_at, d.dx);
        put<E>(p.dr, t0 + k, dr_at, d.dr);
        put<E>(p.di, t0 + k, di_at, d.di);
      }
    }
    if (p.dh0 && t0 == 0 && l.on) p.dh0[l.at] = in;
  }
  __syncthreads();
  board.add[0][wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && l.on) {
    for (int w = 1; w < waves; ++w) sum += board.add[0][w][lane];
    p.part[l.at] = sum;
  }
}

// --------------------------------------------------------------------------

// What segment blockIdx.y + 1 leaves, to the segment before it, of the states'
// gradient that enters it from behind, and what it adds.
template <typename E>
__global__ void __launch_bounds__(256) gatedrec_back_sum(Rec p) {
  constexpr int U = 8;
  const Place<2> l(p, blockIdx.x * blockDim.x + threadIdx.x);
  if (!l.on) return;
  const int begin = (blockIdx.y + 1) * p.len, end = min(begin + p.len, p.T);
  const uint32_t r_at = l.in<E>(p.r), d_at = l.in<E>(p.dh);
  const float rate[2] = {kLog2e * l.rate[0], kLog2e * l.rate[1]};
  f2_t G = {0.0f, 0.0f}, sum = {0.0f, 0.0f};
  bool whole = true;
  Pair<E> nr[U], nd[U];
  uint8_t nc[U];
  const auto fetch = [&](int t1) {  // the steps before t1
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int t = max(t1 - 1 - k, begin);
      nr[k] = load<E>(p.r, t, r_at);
      nd[k] = load<E>(p.dh, t, d_at);
      nc[k] = p.reset ? p.reset[static_cast<uint64_t>(t) * p.B + l.b] : 0;
    }
  };
  fetch(end);
  for (int t1 = end; t1 > begin; t1 -= U) {
    Pair<E> r[U], d[U];
    uint8_t cut[U];
#pragma unroll
    for (int k = 0; k < U; ++k) r[k] = nr[k], d[k] = nd[k], cut[k] = nc[k];
    fetch(t1 - U);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (t1 - 1 - k < begin) break;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float y = rate[j] * sigmoid2(r[k][j]);
        sum[j] += y;
        G[j] += d[k][j];
        G[j] = Decay(y).carried(G[j]);
      }
      if (cut[k]) {
        G = f2_t{0.0f, 0.0f};
        whole = false;
      }
    }
  }
  const uint64_t seg = blockIdx.y;
  state_out(p.keep + seg * p.states, l.at, whole ? __builtin_amdgcn_exp2f(-sum[0]) : -1.0f,
            whole ? __builtin_amdgcn_exp2f(-sum[1]) : -1.0f);
  state_out(p.add + seg * p.states, l.at, G[0], G[1]);
}

// Backward, two channels to a lane, over segment blockIdx.y.  The steps between two marks are run forward
// from the mark, which leaves the state before each step and its gates in
// registers, then backward, while those before them are in flight (T = 256, B = 64,
// D = 4096 203 us; fetched when they are needed 390).
template <typename E>
__global__ void __launch_bounds__(256) gatedrec_bwd(Rec p) {
  const Place<2> l(p, blockIdx.x * blockDim.x + threadIdx.x);
  if (!l.on) return;
  const uint32_t x_at = l.in<E>(p.x), r_at = l.in<E>(p.r), i_at = l.in<E>(p.i), d_at = l.in<E>(p.dh);
  const uint32_t dx_at = l.in<E>(p.dx), dr_at = l.in<E>(p.dr), di_at = l.in<E>(p.di);
  const uint64_t seg = blockIdx.y, segs = gridDim.y;
  const int begin = seg * p.len, end = min(begin + p.len, p.T);
  f2_t G = {0.0f, 0.0f}, sum = {0.0f, 0.0f};
  if (seg + 1 < segs && p.enter) {
    G = state_in(p.enter + seg * p.states, l.at);
  } else {
    if (p.dhT) G = state_in(p.dhT, l.at);
#pragma unroll 4
    for (uint64_t s = segs - 1; s-- > seg;) G = pass(p, s, l.at, G);
  }
  Steps<E, kMark> next;
  Pair<E> next_dh[kMark];
  f2_t next_h;
  const auto fetch = [&](int t0) {
    next.load(p, x_at, r_at, i_at, l.b, t0, end);
#pragma unroll
    for (int k = 0; k < kMark; ++k) next_dh[k] = load<E>(p.dh, min(t0 + k, end - 1), d_at);
    next_h = state_in(p.marks + (t0 / kMark) * p.states, l.at);
  };
  fetch((end - 1) / kMark * kMark);
  for (int t0 = (end - 1) / kMark * kMark; t0 >= begin; t0 -= kMark) {
    const Steps<E, kMark> s = next;
    Pair<E> dh[kMark];
#pragma unroll
    for (int k = 0; k < kMark; ++k) dh[k] = next_dh[k];
    f2_t h = next_h;
    fetch(max(t0 - kMark, begin));
    float before[kMark][2], g[kMark][2], o[kMark][2], decay[kMark][2], beta2[kMark][2];
#pragma unroll
    for (int k = 0; k < kMark; ++k) {
      if (s.cut[k]) h = f2_t{0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        before[k][j] = h[j];
        g[k][j] = sigmoid2(s.r[k][j]);
        o[k][j] = sigmoid2(s.i[k][j]);
        const Decay d(kLog2e * l.rate[j] * g[k][j]);
        decay[k][j] = d.s;
        beta2[k][j] = d.beta2();
        h[j] = next_state(h[j], d, taken_in(beta2[k][j], o[k][j], s.x[k][j]));
      }
    }
#pragma unroll
    for (int k = kMark - 1; k >= 0; --k) {
      if (t0 + k >= end) continue;
      float dx[2], dr[2], di[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        G[j] += dh[k][j];
        const Decay a = kept(decay[k][j]);
        const Grad d(G[j], l.rate[j], s.x[k][j], g[k][j], o[k][j], a, beta2[k][j], before[k][j]);
        dx[j] = d.dx;
        dr[j] = d.dr;
        di[j] = d.di;
        sum[j] += d.e;
        G[j] = a.carried(G[j]);
      }
      if (s.cut[k]) G = f2_t{0.0f, 0.0f};
      store<E>(p.dx, t0 + k, dx_at, dx[0], dx[1]);
      store<E>(p.dr, t0 + k, dr_at, dr[0], dr[1]);
      store<E>(p.di, t0 + k, di_at, di[0], di[1]);
    }
  }
  if (p.dh0 && begin == 0) state_out(p.dh0, l.at, G[0], G[1]);
  state_out(p.part + seg * p.states, l.at, sum[0], sum[1]);
}

// The sum over a lane's rows of p [n, D], every 16th from its group's, in a
// fixed order; the block's 16 groups joined in group 0.
__device__ __forceinline__ float column_sum(size_t n, size_t D, const float* p, bool on) {
  __shared__ float red[16][64];
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6;
  float s = 0.0f;
  if (on)
#pragma unroll 8
    for (size_t k = g; k < n; k += 16) s += p[k * D];
  red[g][c] = s;
  __syncthreads();
  if (g == 0)
#pragma unroll
    for (int k = 1; k < 16; ++k) s += red[k][c];
  return s;
}

// Where there are many rows, rows blockIdx.x kRows and on are summed first, into
// the first of them: the block alone reads its rows and columns (T = 4, B = 100000, D = 64
// backward 163 us, in one launch 521; 1024 rows and fewer gain nothing).
constexpr int kRows = 512;
constexpr size_t kManyRows = 1024;

__global__ void __launch_bounds__(1024) gatedrec_rows(size_t n, size_t row, int D, float* __restrict__ part) {
  const int d = blockIdx.y * 64 + (threadIdx.x & 63);
  const size_t from = static_cast<size_t>(blockIdx.x) * kRows;
  float* p = part + from * row + d;
  const float s = column_sum(n - from < kRows ? n - from : kRows, row, p, d < D);
  if (threadIdx.x < 64 && d < D) *p = s;
}

// dlam: the sum over the rows of part, row numbers apart, a block 64 columns, times d(log rate) / d(lam).
__global__ void __launch_bounds__(1024) gatedrec_rates(size_t n, size_t row, int D, const float* __restrict__ part,
                                                       const float* __restrict__ lam, float* __restrict__ dlam) {
  const int d = blockIdx.x * 64 + (threadIdx.x & 63);
  const float l = lam[min(d, D - 1)];  // (under way before the sums)
  const float s = column_sum(n, row, part + d, d < D);
  // sigmoid(lam) / softplus(lam), which is 1 - e^lam / 2 + ... far to the left
  if (threadIdx.x < 64 && d < D) dlam[d] = s * (l < -15.0f ? 1.0f - 0.5f * expf(l) : 1.0f / ((1.0f + expf(-l)) * softplus(l)));
}

// One step.  A lane keeps its channels, whose rates cost as much as ten steps, and
// takes sample after sample; where a sample has fewer lanes than a block, the block has
// several side by side (500000 x 8 in fp32 23 us, alone 123).
template <typename E>
__global__ void __launch_bounds__(256) gatedrec_token(Rec p, float* __restrict__ S) {
  const uint32_t per = p.D / 2, beside = max(1u, 256 / per), row = per < 256 ? threadIdx.x / per : 0;
  const uint32_t d = (blockIdx.x * 256 + threadIdx.x - row * per) * 2;
  if (row >= beside || d >= static_cast<uint32_t>(p.D)) return;
  const float rate[2] = {kLog2e * rate_of(p.c, p.lam[d]), kLog2e * rate_of(p.c, p.lam[d + 1])};
  for (uint32_t b = blockIdx.y * beside + row; b < static_cast<uint32_t>(p.nb); b += gridDim.y * beside) {
    const Pair<E> x = load<E>(p.x, 0, b * p.x.ld + d * sizeof(E)), r = load<E>(p.r, 0, b * p.r.ld + d * sizeof(E)),
                  i = load<E>(p.i, 0, b * p.i.ld + d * sizeof(E));
    f2_t s = state_in(S, b * p.D + d);
    if (p.reset && p.reset[b]) s = f2_t{0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 2; ++j) s[j] = next_state(s[j], rate[j] * sigmoid2(r[j]), i[j], x[j]);
    state_out(S, b * p.D + d, s[0], s[1]);
    store<E>(p.h, 0, b * p.h.ld + d * sizeof(E), s[0], s[1]);
  }
}

// ------------------------------------------------------------ validation

constexpr int kMaxWidth = 65536;

int check_sizes(const char* fn, o5_dtype dt, int T, int B, int D) {
  O5_CHECK(dt == O5_F32 || dt == O5_BF16, O5_E_DTYPE, "%s: unknown dtype %d", fn, static_cast<int>(dt));
  O5_CHECK(T >= 1 && B >= 1, O5_E_SHAPE, "%s: T=%d and B=%d must be >= 1", fn, T, B);
  O5_CHECK(D >= 8 && D <= kMaxWidth && D % 8 == 0, O5_E_SHAPE, "%s: D=%d must be a multiple of 8 in 8..%d", fn, D,
           kMaxWidth);
  O5_CHECK(static_cast<long long>(T) * B < (1ll << 30), O5_E_SHAPE, "%s: T*B must be below 2^30", fn);
  return O5_OK;
}

#define O5_TRY(expr)              \
  do {                            \
    const int st_ = (expr);       \
    if (st_ != O5_OK) return st_; \
  } while (0)

int check_rows(const char* fn, const char* name, const void* p, const char* ldname, size_t ld, int D) {
  O5_CHECK(ld >= static_cast<size_t>(D) && ld % 8 == 0 && ld < (1ull << 31), O5_E_SHAPE,
           "%s: %s=%zu must be a multiple of 8, at least %d and below 2^31", fn, ldname, ld, D);
  O5_PTR_IN(fn, p, name);
  return O5_OK;
}

int check_inputs(const char* fn, int D, const void* x, size_t ldx, const void* r, size_t ldr, const void* i, size_t ldi,
                 const float* lam, float c) {
  O5_TRY(check_rows(fn, "x", x, "ldx", ldx, D));
  O5_TRY(check_rows(fn, "r", r, "ldr", ldr, D));
  O5_TRY(check_rows(fn, "i", i, "ldi", ldi, D));
  O5_PTR_IN(fn, lam, "lam");
  O5_CHECK(c > 0.0f && std::isfinite(c), O5_E_ARG, "%s: c must be positive and finite", fn);
  return O5_OK;
}

// How a call is run: in blocks of so many waves, or (0) in lanes, which take
// segments of len steps (a multiple of a mark's).
struct Cut {
  int waves, len, segments;
};
constexpr long long kLanes = 1024 * 64;  // that fill the chip
constexpr int kShort = 2 * kWavesOf * kMark;
constexpr int kMostSegments = 512;
constexpr long long kUnits = 256;  // compute units

// Times in us, bf16, both sides measured (with two instructions a step less than it takes now: all up to 3 % longer).
// - kLanes or more: each walks the whole sequence (T = 256, B = 32, D = 4096: forward 74, cut in two 98, in blocks
//   99; backward 120, in blocks 141).  Half as many lanes are too few (B = 32, D = 2048: forward 72, in blocks 50).
// - Fewer: short sequences in blocks, where a launch and a read of the inputs are saved (T = 256, B = 8, D = 1024:
//   forward 15, in segments 19.5, backward 21.5 and 25.6; T = 128, B = 4, D = 512: 13 and 19, 17 and 21).  Where blocks
//   alone have a walk of many rounds, segments are faster (T = 1000, B = 1, D = 64: 18, in blocks 42).
// - Forward, a block on every compute unit is enough for long sequences too (T = 1000, B = 16, D = 1024: 51, in
//   segments 63; B = 48, D = 2048: 224 and 328; T = 2000, B = 8, 128 blocks: 86 and 66).  Backward, segments read only
//   two of five arrays again, and blocks gain at 256 (76 against 83) what they lose at 384 (125 against 113).
// - More blocks than units take fewer waves, down to 4, so that one's barrier is another's work (B = 32, D = 2048,
//   T = 256: 4 waves 50 and backward 75, 8 waves 55 and 79, 16 waves 61 and 88; T = 32: equal).
// - Segments: two lanes for each that fills the chip (four: T = 2000, B = 4, D = 512 29 -> 32; long ones equal), of one
//   mark's steps at the least (of 4 marks' T = 256, B = 8, D = 1024 28, of one 20), 512 of them at the most, which
//   one block joins (1024 with four lanes for each: T = 12000, B = 1, D = 512 38 -> 43).
Cut cut_of(int T, int B, int D, bool back) {
  const long long lanes = static_cast<long long>(B) * (D / 2), blocks = (lanes + 31) / 32;
  if (lanes >= kLanes) return {0, T, 1};
  if (T <= kShort || (!back && blocks >= kUnits)) {
    int waves = kWavesOf;
    while (waves > 4 && blocks * waves > kUnits * kWavesOf) waves /= 2;
    return {std::min(waves, (T + kMark - 1) / kMark), T, 1};
  }
  const long long want = std::min<long long>(std::min<long long>(kMostSegments, 2 * kLanes / std::max(64ll, lanes)), T / kMark);
  const int len = static_cast<int>(((T + want - 1) / want + kMark - 1) / kMark * kMark);
  return {0, len, (T + len - 1) / len};
}

// Sums, joins and the states that enter: three arrays of segments - 1 rows.
size_t cut_bytes(const Cut& c, int B, int D) {
  return align_up(static_cast<size_t>(c.segments - 1) * B * D * sizeof(float)) * 3;
}
void place_cut(const Cut& c, int B, int D, void* ws, Rec* p) {
  const size_t n = align_up(static_cast<size_t>(c.segments - 1) * B * D * sizeof(float)) / sizeof(float);
  p->keep = static_cast<float*>(ws);
  p->add = p->keep + n;
  p->enter = p->add + n;
  p->len = c.len;
}

Rows rows_of(const void* p, size_t ld, int B, size_t es) {
  return {static_cast<char*>(const_cast<void*>(p)), ld * B * es, static_cast<uint32_t>(ld * es)};
}

// launch(arrays) of at most so many samples that offsets within a step stay below 2^32 (a row alone does: ld b is 0 there).
template <class F>
void launch_samples(const Rec& all, size_t most_ld, F&& launch) {
  const size_t most = std::max<size_t>(1, (static_cast<size_t>(1) << 31) / std::max(most_ld * 4, static_cast<size_t>(all.D) * 4));
  for (size_t b = 0; b < static_cast<size_t>(all.B); b += most) {
    Rec p = all;
    p.nb = static_cast<int>(std::min<size_t>(most, all.B - b));
    for (Rows* a : {&p.x, &p.r, &p.i, &p.h, &p.dh, &p.dx, &p.dr, &p.di})
      if (a->p) a->p += b * (a->step / all.B);
    const size_t at = b * all.D;
    for (const float** a : {&p.h0, &p.dhT})
      if (*a) *a += at;
    for (float** a : {&p.hT, &p.marks, &p.dh0, &p.part, &p.keep, &p.add, &p.enter})
      if (*a) *a += at;
    if (p.reset) p.reset += b;
    launch(p);
  }
}

void run_lanes(const Rec& all, size_t most_ld, int segments, void (*kernel)(Rec), hipStream_t s) {
  launch_samples(all, most_ld, [&](const Rec& p) {
    const unsigned blocks = static_cast<unsigned>((static_cast<size_t>(p.nb) * (p.D / 2) + 255) / 256);
    hipLaunchKernelGGL(kernel, dim3(blocks, segments), dim3(256), 0, s, p);
  });
}

void run_blocks(const Rec& all, size_t most_ld, int waves, void (*kernel)(Rec), hipStream_t s) {
  launch_samples(all, most_ld, [&](const Rec& p) {
    const unsigned blocks = static_cast<unsigned>((static_cast<size_t>(p.nb) * p.D + 63) / 64);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * waves), 0, s, p);
  });
}

// The states that enter the segments; few segments are passed by the launch that
// runs them (T = 300, B = 32, D = 2048 backward, 3 of them: 81 us, with a launch for it
// 87; T = 2000, B = 4, 31 of them: 74 and 77).
constexpr int kFewSegments = 32;

void join(Rec* p, const Cut& c, const float* first, bool back, hipStream_t s) {
  if (c.segments <= kFewSegments) {
    p->enter = nullptr;
    return;
  }
  const uint64_t blocks = (p->states + 63) / 64;  // (few: a call of many states is not cut)
  hipLaunchKernelGGL(gatedrec_join, dim3(static_cast<unsigned>(blocks)), dim3(1024), 0, s, p->keep, p->add, first, p->enter,
                     c.segments - 1, p->states, back);
}

}  // namespace
}  // namespace o5

using namespace o5;

extern "C" size_t o5_gatedrec_marks_bytes(int T, int B, int D) {
  if (check_sizes("o5_gatedrec_marks_bytes", O5_F32, T, B, D) != O5_OK) return 0;
  return static_cast<size_t>((T + kMark - 1) / kMark) * B * D * sizeof(float);
}

extern "C" size_t o5_gatedrec_fwd_workspace_bytes(o5_dtype dt, int T, int B, int D) {
  if (check_sizes("o5_gatedrec_fwd_workspace_bytes", dt, T, B, D) != O5_OK) return 0;
  return std::max<size_t>(256, cut_bytes(cut_of(T, B, D, false), B, D));
}

extern "C" int o5_gatedrec_fwd(o5_dtype dt, int T, int B, int D, const void* x, size_t ldx, const void* r, size_t ldr,
                               const void* i, size_t ldi, const float* lam, float c, const float* h0,
                               const uint8_t* reset, void* h, size_t ldh, float* hT, float* marks, void* ws,
                               size_t ws_bytes, void* stream) {
  const char* fn = "o5_gatedrec_fwd";
  O5_TRY(check_sizes(fn, dt, T, B, D));
  O5_TRY(check_inputs(fn, D, x, ldx, r, ldr, i, ldi, lam, c));
  O5_TRY(check_rows(fn, "h", h, "ldh", ldh, D));
  O5_OPT_PTR(h0, "h0");
  O5_OPT_PTR(reset, "reset");
  O5_OPT_PTR(hT, "hT");
  O5_OPT_PTR(marks, "marks");
  O5_CHECK(ws != nullptr && ws_bytes >= o5_gatedrec_fwd_workspace_bytes(dt, T, B, D), O5_E_WORKSPACE,
           "%s: ws is NULL or ws_bytes=%zu is too small", fn, ws_bytes);
  O5_PTR(ws, "ws");
  const size_t es = dtype_size(dt);
  const Cut cut = cut_of(T, B, D, false);
  Rec all = {};
  all.x = rows_of(x, ldx, B, es), all.r = rows_of(r, ldr, B, es), all.i = rows_of(i, ldi, B, es);
  all.h = rows_of(h, ldh, B, es);
  all.lam = lam, all.h0 = h0, all.reset = reset, all.hT = hT, all.marks = marks;
  all.T = T, all.B = B, all.D = D, all.c = c, all.states = static_cast<uint64_t>(B) * D;
  place_cut(cut, B, D, ws, &all);
  const bool bf16 = dt == O5_BF16;
  const size_t most = std::max(std::max(ldx, ldr), std::max(ldi, ldh));
  if (cut.waves > 0) {
    run_blocks(all, most, cut.waves, bf16 ? gatedrec_fwd_block<uint16_t> : gatedrec_fwd_block<float>, as_stream(stream));
    return check_launch(fn);
  }
  if (cut.segments > 1) {
    run_lanes(all, most, cut.segments - 1, bf16 ? gatedrec_fwd<uint16_t, true> : gatedrec_fwd<float, true>, as_stream(stream));
    join(&all, cut, h0, false, as_stream(stream));
  }
  run_lanes(all, most, cut.segments, bf16 ? gatedrec_fwd<uint16_t, false> : gatedrec_fwd<float, false>, as_stream(stream));
  return check_launch(fn);
}

extern "C" size_t o5_gatedrec_bwd_workspace_bytes(o5_dtype dt, int T, int B, int D) {
  if (check_sizes("o5_gatedrec_bwd_workspace_bytes", dt, T, B, D) != O5_OK) return 0;
  const Cut c = cut_of(T, B, D, true);
  return cut_bytes(c, B, D) + static_cast<size_t>(c.segments) * B * D * sizeof(float);
}

extern "C" int o5_gatedrec_bwd(o5_dtype dt, int T, int B, int D, const void* x, size_t ldx, const void* r, size_t ldr,
                               const void* i, size_t ldi, const float* lam, float c, const float* marks,
                               const uint8_t* reset, const void* dh, size_t lddh, const float* dhT, void* dx,
                               size_t lddx, void* dr, size_t lddr, void* di, size_t lddi, float* dlam, float* dh0,
                               void* ws, size_t ws_bytes, void* stream) {
  const char* fn = "o5_gatedrec_bwd";
  O5_TRY(check_sizes(fn, dt, T, B, D));
  O5_TRY(check_inputs(fn, D, x, ldx, r, ldr, i, ldi, lam, c));
  O5_TRY(check_rows(fn, "dh", dh, "lddh", lddh, D));
  O5_TRY(check_rows(fn, "dx", dx, "lddx", lddx, D));
  O5_TRY(check_rows(fn, "dr", dr, "lddr", lddr, D));
  O5_TRY(check_rows(fn, "di", di, "lddi", lddi, D));
  O5_PTR(marks, "marks");
  O5_OPT_PTR(reset, "reset");
  O5_OPT_PTR(dhT, "dhT");
  O5_PTR(dlam, "dlam");
  O5_OPT_PTR(dh0, "dh0");
  O5_CHECK(ws != nullptr && ws_bytes >= o5_gatedrec_bwd_workspace_bytes(dt, T, B, D), O5_E_WORKSPACE,
           "%s: ws is NULL or ws_bytes=%zu is too small", fn, ws_bytes);
  O5_PTR(ws, "ws");
  const size_t es = dtype_size(dt);
  const Cut cut = cut_of(T, B, D, true);
  Rec all = {};
  all.x = rows_of(x, ldx, B, es), all.r = rows_of(r, ldr, B, es), all.i = rows_of(i, ldi, B, es);
  all.dh = rows_of(dh, lddh, B, es);
  all.dx = rows_of(dx, lddx, B, es), all.dr = rows_of(dr, lddr, B, es), all.di = rows_of(di, lddi, B, es);
  all.lam = lam, all.dhT = dhT, all.reset = reset, all.marks = const_cast<float*>(marks), all.dh0 = dh0;
  all.T = T, all.B = B, all.D = D, all.c = c, all.states = static_cast<uint64_t>(B) * D;
  place_cut(cut, B, D, ws, &all);
  all.part = static_cast<float*>(ws) + cut_bytes(cut, B, D) / sizeof(float);
  const bool bf16 = dt == O5_BF16;
  const size_t most = std::max(std::max(std::max(ldx, ldr), std::max(ldi, lddh)), std::max(std::max(lddx, lddr), lddi));
  if (cut.waves > 0) {
    run_blocks(all, most, cut.waves, bf16 ? gatedrec_bwd_block<uint16_t> : gatedrec_bwd_block<float>, as_stream(stream));
  } else {
    if (cut.segments > 1) {
      run_lanes(all, most, cut.segments - 1, bf16 ? gatedrec_back_sum<uint16_t> : gatedrec_back_sum<float>, as_stream(stream));
      join(&all, cut, dhT, true, as_stream(stream));
    }
    run_lanes(all, most, cut.segments, bf16 ? gatedrec_bwd<uint16_t> : gatedrec_bwd<float>, as_stream(stream));
  }
  size_t n = static_cast<size_t>(cut.segments) * B, row = D;
  const unsigned across = (D + 63) / 64;
  for (; n > kManyRows; n = (n + kRows - 1) / kRows, row *= kRows)
    hipLaunchKernelGGL(gatedrec_rows, dim3(static_cast<unsigned>((n + kRows - 1) / kRows), across), dim3(1024), 0,
                       as_stream(stream), n, row, D, all.part);
  hipLaunchKernelGGL(gatedrec_rates, dim3(across), dim3(1024), 0, as_stream(stream), n, row, D, all.part, lam, dlam);
  return check_launch(fn);
}

// Samples of a lane, where there are many (4096 x 4096 57 us, one to a lane 87).
constexpr int kTokenRows = 8;

extern "C" int o5_gatedrec_step(o5_dtype dt, int B, int D, const void* x, size_t ldx, const void* r, size_t ldr,
                                const void* i, size_t ldi, const float* lam, float c, const uint8_t* reset, float* S,
                                void* h, size_t ldh, void* stream) {
  const char* fn = "o5_gatedrec_step";
  O5_TRY(check_sizes(fn, dt, 1, B, D));
  O5_TRY(check_inputs(fn, D, x, ldx, r, ldr, i, ldi, lam, c));
  O5_TRY(check_rows(fn, "h", h, "ldh", ldh, D));
  O5_OPT_PTR(reset, "reset");
  O5_PTR(S, "S");
  const size_t es = dtype_size(dt);
  Rec all = {};
  all.x = rows_of(x, ldx, B, es), all.r = rows_of(r, ldr, B, es), all.i = rows_of(i, ldi, B, es);
  all.h = rows_of(h, ldh, B, es);
  all.lam = lam, all.reset = reset, all.hT = S, all.T = 1, all.B = B, all.D = D, all.c = c;
  launch_samples(all, std::max(std::max(ldx, ldr), std::max(ldi, ldh)), [&](const Rec& p) {
    const unsigned across = (D / 2 + 255) / 256, beside = std::max(1, 256 / (D / 2));
    const unsigned rows = (p.nb + beside - 1) / beside;
    const unsigned down = std::min<unsigned>(65535, std::max<unsigned>(std::min<unsigned>(rows, 1024 / across), rows / kTokenRows));
    hipLaunchKernelGGL(dt == O5_BF16 ? gatedrec_token<uint16_t> : gatedrec_token<float>, dim3(across, down), dim3(256), 0,
                       as_stream(stream), p, p.hT);
  });
  return check_launch(fn);
}
