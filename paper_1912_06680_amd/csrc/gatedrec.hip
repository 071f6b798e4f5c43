// A linear recurrence whose decay and input are gated by the input,
// o5_gatedrec_*.
//
//   g = sigmoid(r), o = sigmoid(i), log a = -c softplus(lam) g
//   h_t = a_t (1 - reset_t) h_{t-1} + beta_t o_t x_t,   beta = sqrt(1 - a^2)
//
// Every channel is a recurrence of its own, so that a lane takes two of them
// and walks the steps.  HBM-bound: 4 arrays of rows forward, 7 backward.
//
// w = 1 - a is formed without the cancellation near a = 1, and the state is
// taken on as h - w h there: a rounded to 24 bits would be off by 2^-25 of
// itself in every step, which over the 1/w steps that a state lasts grows to
// 2^-25 / w.  beta is sqrt(w (2 - w)).
#include "common.h"

namespace o5 {
namespace {

constexpr int kMark = 16;        // steps between the states that the forward pass leaves for the backward pass
constexpr float kMost = 3e38f;   // the largest rate: times a gate that is 0 it is 0

struct Rec {  // a call's arrays
  const void *x, *r, *i, *dh;
  void *h, *dx, *dr, *di;
  size_t ldx, ldr, ldi, lddh, ldh, lddx, lddr, lddi;
  const float *lam, *h0, *dhT;
  const uint8_t* reset;
  float *hT, *marks, *dh0, *part;
  int T, B, D;
  float c;
};

// Two neighbouring channels of a row.
template <typename E> struct Pair;
template <> struct Pair<float> {
  float2 v;
  __device__ __forceinline__ void load(const void* p, size_t at) {
    v = *reinterpret_cast<const float2*>(static_cast<const float*>(p) + at);
  }
  __device__ __forceinline__ float operator[](int j) const { return j ? v.y : v.x; }
  __device__ __forceinline__ static void store(void* p, size_t at, float a, float b) {
    *reinterpret_cast<float2*>(static_cast<float*>(p) + at) = make_float2(a, b);
  }
};
template <> struct Pair<uint16_t> {
  uint32_t v;
  __device__ __forceinline__ void load(const void* p, size_t at) {
    v = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p) + at);
  }
  __device__ __forceinline__ float operator[](int j) const { return __uint_as_float(j ? v & 0xffff0000u : v << 16); }
  __device__ __forceinline__ static void store(void* p, size_t at, float a, float b) {
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p) + at) = f32x2_to_bf16x2(a, b);
  }
};

__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.0f) + log1pf(expf(-fabsf(x))); }
__device__ __forceinline__ float rate_of(float c, float lam) { return fminf(c * softplus(lam), kMost); }

// The decay of one step: la = log a <= 0, w = 1 - a.
struct Decay {
  float la, a, w;
  __device__ __forceinline__ Decay(float rate, float g) {
    la = -rate * g;
    a = __expf(la);
    // 1 - e^la = y - y^2/2 + ... of y = -la: the first term left out is 2e-8
    // of it at 0.35, where 1 - a is 2.4e-7 off
    const float y = -la;
    float s = fmaf(y, 1.0f / 5040.0f, -1.0f / 720.0f);
    s = fmaf(y, s, 1.0f / 120.0f);
    s = fmaf(y, s, -1.0f / 24.0f);
    s = fmaf(y, s, 1.0f / 6.0f);
    s = fmaf(y, s, -0.5f);
    s = fmaf(y * y, s, y);
    w = y < 0.35f ? s : 1.0f - a;
  }
  // a h
  __device__ __forceinline__ float times(float h) const { return la > -0.35f ? fmaf(-w, h, h) : a * h; }
};

// A lane's place: two channels of one sample.
struct Place {
  int b, d;
  bool on;
  __device__ __forceinline__ Place(const Rec& p, uint64_t first) {
    const uint64_t at = first + static_cast<uint64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    const uint32_t half = p.D / 2;
    on = at < static_cast<uint64_t>(p.B) * half;
    b = static_cast<int>(at / half);
    d = static_cast<int>(at % half) * 2;
  }
};

template <typename E>
__global__ void __launch_bounds__(256) gatedrec_fwd(Rec p, uint64_t first) {
  const Place l(p, first);
  if (!l.on) return;
  const float rate[2] = {rate_of(p.c, p.lam[l.d]), rate_of(p.c, p.lam[l.d + 1])};
  const size_t state = static_cast<size_t>(l.b) * p.D + l.d, states = static_cast<size_t>(p.B) * p.D;
  float h[2] = {0.0f, 0.0f};
  if (p.h0) h[0] = p.h0[state], h[1] = p.h0[state + 1];
  for (int t = 0; t < p.T; ++t) {
    const size_t row = static_cast<size_t>(t) * p.B + l.b;
    Pair<E> x, r, i;
    x.load(p.x, row * p.ldx + l.d);
    r.load(p.r, row * p.ldr + l.d);
    i.load(p.i, row * p.ldi + l.d);
    if (p.marks && t % kMark == 0) Pair<float>::store(p.marks, (t / kMark) * states + state, h[0], h[1]);
    const bool cut = p.reset != nullptr && p.reset[row] != 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const Decay a(rate[j], sigmoid_f(r[j]));
      const float beta = __builtin_amdgcn_sqrtf(a.w * (2.0f - a.w));
      h[j] = (cut ? 0.0f : a.times(h[j])) + beta * (sigmoid_f(i[j]) * x[j]);
    }
    Pair<E>::store(p.h, row * p.ldh + l.d, h[0], h[1]);
  }
  if (p.hT) Pair<float>::store(p.hT, state, h[0], h[1]);
}

// The steps between two marks are run forward from the mark first, which
// leaves the state before each, then backward.
template <typename E>
__global__ void __launch_bounds__(256) gatedrec_bwd(Rec p, uint64_t first) {
  const Place l(p, first);
  if (!l.on) return;
  const float rate[2] = {rate_of(p.c, p.lam[l.d]), rate_of(p.c, p.lam[l.d + 1])};
  const size_t state = static_cast<size_t>(l.b) * p.D + l.d, states = static_cast<size_t>(p.B) * p.D;
  float G[2] = {0.0f, 0.0f}, sum[2] = {0.0f, 0.0f};
  if (p.dhT) G[0] = p.dhT[state], G[1] = p.dhT[state + 1];
  for (int m = (p.T - 1) / kMark; m >= 0; --m) {
    const int t0 = m * kMark;
    float before[kMark][2], h[2];
    h[0] = p.marks[m * states + state], h[1] = p.marks[m * states + state + 1];
#pragma unroll
    for (int k = 0; k < kMark; ++k) {
      if (t0 + k < p.T) {
        const size_t row = static_cast<size_t>(t0 + k) * p.B + l.b;
        Pair<E> x, r, i;
        x.load(p.x, row * p.ldx + l.d);
        r.load(p.r, row * p.ldr + l.d);
        i.load(p.i, row * p.ldi + l.d);
        const bool cut = p.reset != nullptr && p.reset[row] != 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const Decay a(rate[j], sigmoid_f(r[j]));
          const float beta = __builtin_amdgcn_sqrtf(a.w * (2.0f - a.w));
          before[k][j] = cut ? 0.0f : h[j];
          h[j] = a.times(before[k][j]) + beta * (sigmoid_f(i[j]) * x[j]);
        }
      }
    }
#pragma unroll
    for (int k = kMark - 1; k >= 0; --k) {
      if (t0 + k < p.T) {
        const size_t row = static_cast<size_t>(t0 + k) * p.B + l.b;
        Pair<E> x, r, i, dh;
        x.load(p.x, row * p.ldx + l.d);
        r.load(p.r, row * p.ldr + l.d);
        i.load(p.i, row * p.ldi + l.d);
        dh.load(p.dh, row * p.lddh + l.d);
        const bool cut = p.reset != nullptr && p.reset[row] != 0;
        float dx[2], dr[2], di[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float g = sigmoid_f(r[j]), o = sigmoid_f(i[j]);
          const Decay a(rate[j], g);
          const float v = a.w * (2.0f - a.w), ib = v > 0.0f ? __builtin_amdgcn_rsqf(v) : 0.0f;
          G[j] += dh[j];
          // G d(log a) log a: the quotient log a / beta goes to 0 with log a
          const float e = G[j] * (a.a * before[k][j] * a.la - a.a * a.a * (o * x[j]) * (a.la * ib));
          const float du = G[j] * (v * ib);
          dx[j] = du * o;
          dr[j] = e * (1.0f - g);
          di[j] = du * x[j] * (o * (1.0f - o));
          sum[j] += e;
          G[j] = cut ? 0.0f : a.times(G[j]);
        }
        Pair<E>::store(p.dx, row * p.lddx + l.d, dx[0], dx[1]);
        Pair<E>::store(p.dr, row * p.lddr + l.d, dr[0], dr[1]);
        Pair<E>::store(p.di, row * p.lddi + l.d, di[0], di[1]);
      }
    }
  }
  if (p.dh0) Pair<float>::store(p.dh0, state, G[0], G[1]);
  Pair<float>::store(p.part, state, sum[0], sum[1]);
}

// dlam: the sum over the rows of part [n, D] in a fixed order, a block 64
// columns in 16 groups of rows, times d(log rate) / d(lam).
__global__ void __launch_bounds__(1024) gatedrec_rates(size_t n, int D, const float* __restrict__ part,
                                                       const float* __restrict__ lam, float* __restrict__ dlam) {
  __shared__ float red[16][64];
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6, d = blockIdx.x * 64 + c;
  float s = 0.0f;
  if (d < D)
    for (size_t k = g; k < n; k += 16) s += part[k * D + d];
  red[g][c] = s;
  __syncthreads();
  if (g == 0 && d < D) {
#pragma unroll
    for (int k = 1; k < 16; ++k) s += red[k][c];
    // sigmoid(lam) / softplus(lam), which is 1 - e^lam / 2 + ... far to the left
    const float e = expf(lam[d]);
    dlam[d] = s * (lam[d] < -15.0f ? 1.0f - 0.5f * e : 1.0f / ((1.0f + expf(-lam[d])) * softplus(lam[d])));
  }
}

template <typename E>
__global__ void __launch_bounds__(256) gatedrec_token(Rec p, float* __restrict__ S, uint64_t first) {
  const Place l(p, first);
  if (!l.on) return;
  const size_t row = l.b, state = row * p.D + l.d;
  Pair<E> x, r, i;
  x.load(p.x, row * p.ldx + l.d);
  r.load(p.r, row * p.ldr + l.d);
  i.load(p.i, row * p.ldi + l.d);
  Pair<float> s;
  s.load(S, state);
  const bool cut = p.reset != nullptr && p.reset[row] != 0;
  float h[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const Decay a(rate_of(p.c, p.lam[l.d + j]), sigmoid_f(r[j]));
    const float beta = __builtin_amdgcn_sqrtf(a.w * (2.0f - a.w));
    h[j] = (cut ? 0.0f : a.times(s[j])) + beta * (sigmoid_f(i[j]) * x[j]);
  }
  Pair<float>::store(S, state, h[0], h[1]);
  Pair<E>::store(p.h, row * p.ldh + l.d, h[0], h[1]);
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

// launch(first lane, blocks): a launch holds fewer than 2^32 threads.
template <class F>
void launch_lanes(int B, int D, F&& launch) {
  constexpr uint64_t kBlocks = 0xffffffffu / 256;
  const uint64_t blocks = (static_cast<uint64_t>(B) * (D / 2) + 255) / 256;
  for (uint64_t b = 0; b < blocks; b += kBlocks) launch(b * 256, static_cast<unsigned>(std::min(blocks - b, kBlocks)));
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
  return 256;
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
  Rec p = {};
  p.x = x, p.r = r, p.i = i, p.h = h;
  p.ldx = ldx, p.ldr = ldr, p.ldi = ldi, p.ldh = ldh;
  p.lam = lam, p.h0 = h0, p.reset = reset, p.hT = hT, p.marks = marks;
  p.T = T, p.B = B, p.D = D, p.c = c;
  auto kernel = dt == O5_BF16 ? gatedrec_fwd<uint16_t> : gatedrec_fwd<float>;
  launch_lanes(B, D, [&](uint64_t first, unsigned blocks) {
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, as_stream(stream), p, first);
  });
  return check_launch(fn);
}

extern "C" size_t o5_gatedrec_bwd_workspace_bytes(o5_dtype dt, int T, int B, int D) {
  if (check_sizes("o5_gatedrec_bwd_workspace_bytes", dt, T, B, D) != O5_OK) return 0;
  return static_cast<size_t>(B) * D * sizeof(float);
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
  Rec p = {};
  p.x = x, p.r = r, p.i = i, p.dh = dh, p.dx = dx, p.dr = dr, p.di = di;
  p.ldx = ldx, p.ldr = ldr, p.ldi = ldi, p.lddh = lddh, p.lddx = lddx, p.lddr = lddr, p.lddi = lddi;
  p.lam = lam, p.dhT = dhT, p.reset = reset, p.marks = const_cast<float*>(marks), p.dh0 = dh0;
  p.part = static_cast<float*>(ws);
  p.T = T, p.B = B, p.D = D, p.c = c;
  auto kernel = dt == O5_BF16 ? gatedrec_bwd<uint16_t> : gatedrec_bwd<float>;
  launch_lanes(B, D, [&](uint64_t first, unsigned blocks) {
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, as_stream(stream), p, first);
  });
  hipLaunchKernelGGL(gatedrec_rates, dim3((D + 63) / 64), dim3(1024), 0, as_stream(stream), static_cast<size_t>(B), D,
                     p.part, lam, dlam);
  return check_launch(fn);
}

extern "C" int o5_gatedrec_step(o5_dtype dt, int B, int D, const void* x, size_t ldx, const void* r, size_t ldr,
                                const void* i, size_t ldi, const float* lam, float c, const uint8_t* reset, float* S,
                                void* h, size_t ldh, void* stream) {
  const char* fn = "o5_gatedrec_step";
  O5_TRY(check_sizes(fn, dt, 1, B, D));
  O5_TRY(check_inputs(fn, D, x, ldx, r, ldr, i, ldi, lam, c));
  O5_TRY(check_rows(fn, "h", h, "ldh", ldh, D));
  O5_OPT_PTR(reset, "reset");
  O5_PTR(S, "S");
  Rec p = {};
  p.x = x, p.r = r, p.i = i, p.h = h;
  p.ldx = ldx, p.ldr = ldr, p.ldi = ldi, p.ldh = ldh;
  p.lam = lam, p.reset = reset, p.T = 1, p.B = B, p.D = D, p.c = c;
  auto kernel = dt == O5_BF16 ? gatedrec_token<uint16_t> : gatedrec_token<float>;
  launch_lanes(B, D, [&](uint64_t first, unsigned blocks) {
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), 0, as_stream(stream), p, S, first);
  });
  return check_launch(fn);
}
