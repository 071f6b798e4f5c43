// RMS norms before and after a block, fused with its gate and residual
// scale, o5_resnorm_*.
//
//   x' = x + rho . sigmoid(gate) . (w_post . u r_u),   r_u = (mean u^2 + eps)^(-1/2)
//   n  = w_pre . x' r_x',                             r_x' = (mean x'^2 + eps)^(-1/2)
//
// so the norm after one block, its gate, the residual sum and the norm before
// the next block are one pass over the row: each array is read or written
// once, and a row stays in registers between its two reductions.  HBM-bound.
#include "common.h"
#include "reduce.h"

namespace o5 {
namespace {

constexpr int kMaxWidth = 8192;
// Blocks that walk the rows: two on each compute unit in the forward pass, one
// in the backward pass, which has more of a row in flight and sums to write for
// each block.  us, two / one, forward: the norm before alone, 32768 x 4096 in
// bf16, 91 / 130; with block and gate 4096 x 4096 27.6 / 32.5, 40000 x 1032 91 /
// 136, 40000 x 512 32 / 43, in fp32 61 / 61, 157 / 152 and 79 / 76.  One is
// faster where block and gate come with many wide rows: 32768 x 4096 260 / 231,
// in fp32 514 / 474; 2048 x 8192 32 / 28.  Backward with block and gate, one / two:
// 16384 x 4096 202 / 217, in fp32 400 / 404, fp32 with bf16 blocks 267 / 289; 40000
// x 512 63 / 62, 122 / 129 and 87 / 90.  Two are faster for rows of few lanes: 40000
// x 256 54 / 39, 69 / 63 and 55 / 44; 40000 x 64 53 / 37, 56 / 40 and 54 / 38.
constexpr int kFwdBlocks = 512, kBwdBlocks = 256;

typedef float f4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));

template <typename E> struct Run8;  // 8 consecutive elements as they are stored
template <> struct Run8<float> {
  f4_t a, b;
  __device__ __forceinline__ void load(const void* p, size_t i) {
    const f4_t* q = reinterpret_cast<const f4_t*>(static_cast<const float*>(p) + i);
    a = q[0];
    b = q[1];
  }
  __device__ __forceinline__ float operator[](int j) const { return j < 4 ? a[j] : b[j - 4]; }
};
template <> struct Run8<uint16_t> {
  u4_t a;
  __device__ __forceinline__ void load(const void* p, size_t i) {
    a = *reinterpret_cast<const u4_t*>(static_cast<const uint16_t*>(p) + i);
  }
  __device__ __forceinline__ float operator[](int j) const {
    return __uint_as_float((j & 1) ? (a[j / 2] & 0xffff0000u) : (a[j / 2] << 16));
  }
};

template <typename E> __device__ __forceinline__ void store8(void* p, size_t i, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<float>(void* p, size_t i, const float (&v)[8]) {
  f4_t* q = reinterpret_cast<f4_t*>(static_cast<float*>(p) + i);
  q[0] = f4_t{v[0], v[1], v[2], v[3]};
  q[1] = f4_t{v[4], v[5], v[6], v[7]};
}
template <> __device__ __forceinline__ void store8<uint16_t>(void* p, size_t i, const float (&v)[8]) {
  *reinterpret_cast<u4_t*>(static_cast<uint16_t*>(p) + i) =
      u4_t{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7])};
}

// Sum over the TR threads of a row (whole waves), the same in each of them.
template <int TR>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum(v);
  if (TR == 64) return v;
  const int w = threadIdx.x >> 6, w0 = threadIdx.x / TR * (TR / 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[w] = v;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < TR / 64; ++i) s += red[w0 + i];
  return s;
}

struct NormFwd {
  const void *x, *u, *gate;
  const float *w_post, *rho, *w_pre;
  void *xo, *n;
  float *r_post, *r_pre;
  int N, D;
  size_t ldg;
  float eps;
};

// A row's operands on their way from memory: the next row's are in flight
// while one is worked on.
template <typename X, typename E, int NJ>
struct FwdRow {
  Run8<X> x[NJ];
  Run8<E> u[NJ], gate[NJ];
};

// TR threads of a block of max(256, TR) take a row, 8 elements each in NJ
// runs, and walk the rows with the gains in registers.  HBM-bound: 32768 x 4096
// in bf16 260 us, 5.2 TB/s, in fp32 504 to 514; 60 x 1024 4 us, a row's latency.
template <typename X, typename E, int TR, int NJ>
__global__ void __launch_bounds__(TR < 256 ? 256 : TR) resnorm_fwd(NormFwd p) {
  constexpr int BT = TR < 256 ? 256 : TR;
  __shared__ float red[BT / 64];
  const int group = blockIdx.x * (BT / TR) + threadIdx.x / TR, groups = gridDim.x * (BT / TR), t = threadIdx.x % TR;
  const float inv = 1.0f / static_cast<float>(p.D);
  bool on[NJ];
  float wr[NJ][8], wp[NJ][8];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int c = (t + j * TR) * 8;
    on[j] = c < p.D;
    Run8<float> a = {}, b = {}, w = {};
    if (on[j] && p.u) {
      a.load(p.w_post, c);
      b.load(p.rho, c);
    }
    if (on[j] && p.w_pre) w.load(p.w_pre, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      wr[j][i] = a[i] * b[i];
      wp[j][i] = w[i];
    }
  }
  auto fetch = [&](int row, FwdRow<X, E, NJ>& r) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (t + j * TR) * 8;
      r.x[j] = {};
      r.u[j] = {};
      r.gate[j] = {};
      if (row >= p.N || !on[j]) continue;
      r.x[j].load(p.x, static_cast<size_t>(row) * p.D + c);
      if (p.u) r.u[j].load(p.u, static_cast<size_t>(row) * p.D + c);
      if (p.gate) r.gate[j].load(p.gate, static_cast<size_t>(row) * p.ldg + c);
    }
  };
  const int rounds = (p.N + groups - 1) / groups;
  FwdRow<X, E, NJ> next;
  fetch(group, next);
  for (int k = 0; k < rounds; ++k) {
    const int row = group + k * groups;
    const bool in = row < p.N;
    const size_t base = static_cast<size_t>(row) * p.D;
    const FwdRow<X, E, NJ> r = next;
    if (k + 1 < rounds) fetch(row + groups, next);
    float x[NJ][8];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[j][i] = r.x[j][i];
    if (p.u) {
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(r.u[j][i], r.u[j][i], ss);
      const float ru = 1.0f / sqrtf(row_sum<TR>(ss, red) * inv + p.eps);
      if (p.r_post && t == 0 && in) p.r_post[row] = ru;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float y = r.u[j][i] * ru * wr[j][i];
          if (p.gate) y *= sigmoid_f(r.gate[j][i]);
          x[j][i] += y;
        }
        if (in && on[j]) store8<X>(p.xo, base + (t + j * TR) * 8, x[j]);
      }
    }
    if (p.w_pre) {
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[j][i], x[j][i], ss);
      const float rx = 1.0f / sqrtf(row_sum<TR>(ss, red) * inv + p.eps);
      if (p.r_pre && t == 0 && in) p.r_pre[row] = rx;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[j][i] * rx * wp[j][i];
        if (in && on[j]) store8<E>(p.n, base + (t + j * TR) * 8, y);
      }
    }
  }
}

struct NormBwd {
  const void *x, *u, *gate;
  const float *w_post, *rho, *w_pre, *r_post, *r_pre;
  const void *dxo, *dn;
  void *dx, *du, *dgate;
  float *part;  // [blocks][2][D]: the blocks' column sums for dw_pre, and for drho and dw_post
  int N, D;
  size_t ldg, lddg;
};

template <typename X, typename E, int NJ>
struct BwdRow {
  Run8<X> dxo[NJ], x[NJ];
  Run8<E> dn[NJ], u[NJ], gate[NJ];
  float r_pre, r_post;
};

// The rows' gradients, and each block's sums over its rows:
//   a = dn w_pre,  d = dx' + r_x' (a - x' r_x'^2 mean(a x')),  dx = d
//   s = sigmoid(gate), y = u r_u:  dgate = d y w_post rho s (1 - s),
//   a = d s w_post rho,  du = r_u (a - y mean(a y))
//   dw_pre = sum dn x' r_x',  drho = w_post sum d s y,  dw_post = rho sum d s y
// Every operand of the next row is in flight while a row is worked on, and
// the gains stay in registers (read again for each row they were half as many
// bytes as the row itself).  HBM-bound: 32768 x 4096 in bf16 390 us, 5.5 TB/s,
// in fp32 782 us; 5003 x 1000 in fp32 and bf16 19.5 us, 4.6 TB/s.  The fp32 forms
// above 1024 columns hold 256 registers, one wave a SIMD, and that of 4104 to 8192
// spills 14 more (8192 x 8192: 424 us, 5.1 TB/s).
template <typename X, typename E, int TR, int NJ>
__global__ void __launch_bounds__(TR < 256 ? 256 : TR) resnorm_bwd(NormBwd p) {
  constexpr int BT = TR < 256 ? 256 : TR, ROWS = BT / TR;
  __shared__ float red[BT / 64];
  const int group = blockIdx.x * ROWS + threadIdx.x / TR, groups = gridDim.x * ROWS, t = threadIdx.x % TR;
  const float inv = 1.0f / static_cast<float>(p.D);
  float spre[NJ][8] = {}, spost[NJ][8] = {}, wr[NJ][8], wp[NJ][8];
  bool on[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int c = (t + j * TR) * 8;
    on[j] = c < p.D;
    Run8<float> a = {}, b = {}, w = {};
    if (on[j] && p.u) {
      a.load(p.w_post, c);
      b.load(p.rho, c);
    }
    if (on[j] && p.w_pre) w.load(p.w_pre, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      wr[j][i] = a[i] * b[i];
      wp[j][i] = w[i];
    }
  }
  auto fetch = [&](int row, BwdRow<X, E, NJ>& r) {  // (zeros beyond the rows and columns)
    const bool in = row < p.N;
    const size_t base = static_cast<size_t>(row) * p.D;
    r.r_pre = in && p.w_pre ? p.r_pre[row] : 0.0f;
    r.r_post = in && p.u ? p.r_post[row] : 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (t + j * TR) * 8;
      r.dxo[j] = {};
      r.x[j] = {};
      r.dn[j] = {};
      r.u[j] = {};
      r.gate[j] = {};
      if (!in || !on[j]) continue;
      r.dxo[j].load(p.dxo, base + c);
      if (p.w_pre) {
        r.x[j].load(p.x, base + c);
        r.dn[j].load(p.dn, base + c);
      }
      if (p.u) r.u[j].load(p.u, base + c);
      if (p.gate) r.gate[j].load(p.gate, static_cast<size_t>(row) * p.ldg + c);
    }
  };
  const int rounds = (p.N + groups - 1) / groups;
  BwdRow<X, E, NJ> next;
  fetch(group, next);
  for (int k = 0; k < rounds; ++k) {
    const int row = group + k * groups;
    const bool in = row < p.N;
    const size_t base = static_cast<size_t>(row) * p.D;
    const BwdRow<X, E, NJ> q = next;
    if (k + 1 < rounds) fetch(row + groups, next);
    float d[NJ][8];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) d[j][i] = q.dxo[j][i];
    if (p.w_pre) {
      const float r = q.r_pre;
      float dot = 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dot = fmaf(q.dn[j][i] * wp[j][i], q.x[j][i], dot);
          spre[j][i] = fmaf(q.dn[j][i], q.x[j][i] * r, spre[j][i]);
        }
      const float m = row_sum<TR>(dot, red) * inv * (r * r);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[j][i] += r * (q.dn[j][i] * wp[j][i] - q.x[j][i] * m);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (in && on[j]) store8<X>(p.dx, base + (t + j * TR) * 8, d[j]);
    if (p.u) {
      const float r = q.r_post;
      float dot = 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float dg[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = q.u[j][i] * r;
          if (p.gate) {
            const float s = sigmoid_f(q.gate[j][i]);
            dg[i] = d[j][i] * y * wr[j][i] * s * (1.0f - s);
            d[j][i] *= s;
          }
          spost[j][i] = fmaf(d[j][i], y, spost[j][i]);
          d[j][i] *= wr[j][i];
          dot = fmaf(d[j][i], y, dot);
        }
        if (p.gate && in && on[j]) store8<E>(p.dgate, static_cast<size_t>(row) * p.lddg + (t + j * TR) * 8, dg);
      }
      const float m = row_sum<TR>(dot, red) * inv;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = r * (d[j][i] - q.u[j][i] * r * m);
        if (in && on[j]) store8<E>(p.du, base + (t + j * TR) * 8, o);
      }
    }
  }
  float* part = p.part + static_cast<size_t>(blockIdx.x) * 2 * p.D;
  if (ROWS == 1) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (t + j * TR) * 8;
      if (!on[j]) continue;
      if (p.w_pre) store8<float>(part, c, spre[j]);
      if (p.u) store8<float>(part + p.D, c, spost[j]);
    }
  } else {  // the block's row groups first, in order
    constexpr int WIDTH = TR * NJ * 8;
    __shared__ alignas(16) float sums[ROWS == 1 ? 1 : ROWS][ROWS == 1 ? 8 : WIDTH];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NJ; ++j) store8<float>(sums[threadIdx.x / TR], (t + j * TR) * 8, a == 0 ? spre[j] : spost[j]);
      __syncthreads();
      if (a == 0 ? p.w_pre == nullptr : p.u == nullptr) continue;
      for (int c = threadIdx.x; c < p.D; c += BT) {
        float s = 0.0f;
#pragma unroll
        for (int g = 0; g < ROWS; ++g) s += sums[g][c];
        part[a * p.D + c] = s;
      }
    }
  }
}

// dw_pre, drho and dw_post from the blocks' sums: a block takes 64 columns of
// one of the two sums, wave w adds the blocks w, w + 16, ... in order, and
// the 16 waves' sums are added in order, the same each time.  Bound by its
// launch and one chain of loads: 4 to 5 us.
__global__ void __launch_bounds__(1024) resnorm_columns(int groups, int D, const float* __restrict__ part,
                                                        const float* __restrict__ w_post,
                                                        const float* __restrict__ rho, float* __restrict__ dw_pre,
                                                        float* __restrict__ drho, float* __restrict__ dw_post) {
  __shared__ float red[16][64];
  const int which = blockIdx.y + (dw_pre ? 0 : 1);  // 0: dw_pre, 1: the sum of the other two
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  const float* col = part + static_cast<size_t>(which) * D + c;
  float s = 0.0f;
  if (c < D && w < groups)
    s = ordered_sum((groups - w + 15) / 16, [&](int i) { return col[static_cast<size_t>(w + 16 * i) * 2 * D]; });
  red[w][lane] = s;
  __syncthreads();
  if (w != 0 || c >= D) return;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += red[i][lane];
  if (which == 0) {
    dw_pre[c] = s;
  } else {
    drho[c] = w_post[c] * s;
    dw_post[c] = rho[c] * s;
  }
}

// Threads of a row: 8 or 16 elements each, but a wave at least, most of whose
// lanes have nothing where the row is narrow (40000 x 64 in bf16: 25 us forward and
// 53 backward, where the bytes take 5 and 8).
int row_threads(int D) { return D <= 1024 ? 64 : D <= 2048 ? 128 : D <= 4096 ? 256 : 512; }

int row_blocks(int N, int D, int most) {
  const int tr = row_threads(D), per = tr < 256 ? 256 / tr : 1;
  return std::min((N + per - 1) / per, most);
}

template <typename X, typename E>
void launch_fwd(const NormFwd& p, hipStream_t s) {
  const int tr = row_threads(p.D), bt = tr < 256 ? 256 : tr;
  auto k = tr == 64    ? (p.D <= 512 ? resnorm_fwd<X, E, 64, 1> : resnorm_fwd<X, E, 64, 2>)
           : tr == 128 ? resnorm_fwd<X, E, 128, 2>
           : tr == 256 ? resnorm_fwd<X, E, 256, 2>
                       : resnorm_fwd<X, E, 512, 2>;
  hipLaunchKernelGGL(k, dim3(row_blocks(p.N, p.D, kFwdBlocks)), dim3(bt), 0, s, p);
}

template <typename X, typename E>
void launch_bwd(const NormBwd& p, hipStream_t s) {
  const int tr = row_threads(p.D), bt = tr < 256 ? 256 : tr;
  auto k = tr == 64    ? (p.D <= 512 ? resnorm_bwd<X, E, 64, 1> : resnorm_bwd<X, E, 64, 2>)
           : tr == 128 ? resnorm_bwd<X, E, 128, 2>
           : tr == 256 ? resnorm_bwd<X, E, 256, 2>
                       : resnorm_bwd<X, E, 512, 2>;
  hipLaunchKernelGGL(k, dim3(row_blocks(p.N, p.D, kBwdBlocks)), dim3(bt), 0, s, p);
}

int check_common(const char* fn, o5_dtype xt, o5_dtype dt, int N, int D) {
  O5_CHECK((xt == O5_F32 || xt == O5_BF16) && (dt == O5_F32 || dt == O5_BF16), O5_E_DTYPE, "%s: unknown dtype", fn);
  O5_CHECK(!(xt == O5_BF16 && dt == O5_F32), O5_E_DTYPE, "%s: a bf16 residual stream needs bf16 blocks", fn);
  O5_CHECK(N >= 1 && N < (1 << 30) && D >= 8 && D <= kMaxWidth && D % 8 == 0, O5_E_SHAPE,
           "%s: N=%d must be in 1..2^30-1 and D=%d a multiple of 8 in 8..%d", fn, N, D, kMaxWidth);
  return O5_OK;
}

int check_gate(const char* fn, const char* name, const void* gate, size_t ld, int D) {
  if (gate)
    O5_CHECK(ld >= static_cast<size_t>(D) && ld % 8 == 0 && ld < (1ull << 31), O5_E_SHAPE,
             "%s: %s=%zu must be a multiple of 8, at least D and below 2^31", fn, name, ld);
  return O5_OK;
}

#define O5_TRY(expr)              \
  do {                            \
    const int st_ = (expr);       \
    if (st_ != O5_OK) return st_; \
  } while (0)

}  // namespace
}  // namespace o5

using namespace o5;

extern "C" int o5_resnorm_fwd(o5_dtype xt, o5_dtype dt, int N, int D, const void* x, const void* u, const void* gate,
                              size_t ldg, const float* w_post, const float* rho, const float* w_pre, float eps, void* xo,
                              void* n, float* r_post, float* r_pre, void* stream) {
  const char* fn = "o5_resnorm_fwd";
  O5_TRY(check_common(fn, xt, dt, N, D));
  O5_CHECK(eps > 0.0f && std::isfinite(eps), O5_E_ARG, "%s: eps must be positive", fn);
  O5_CHECK(u != nullptr || w_pre != nullptr, O5_E_ARG, "%s: u and w_pre are both NULL", fn);
  O5_CHECK(u != nullptr || gate == nullptr, O5_E_ARG, "%s: a gate needs u", fn);
  O5_TRY(check_gate(fn, "ldg", gate, ldg, D));
  O5_PTR(x, "x");
  O5_OPT_PTR(gate, "gate");
  O5_OPT_PTR(r_post, "r_post");
  O5_OPT_PTR(r_pre, "r_pre");
  if (u) {
    O5_PTR(u, "u");
    O5_PTR(w_post, "w_post");
    O5_PTR(rho, "rho");
    O5_PTR(xo, "xo");
  }
  if (w_pre) {
    O5_PTR(w_pre, "w_pre");
    O5_PTR(n, "n");
  }
  const NormFwd p = {x, u, gate, w_post, rho, w_pre, xo, n, r_post, r_pre, N, D, ldg, eps};
  if (xt == O5_BF16)
    launch_fwd<uint16_t, uint16_t>(p, as_stream(stream));
  else if (dt == O5_BF16)
    launch_fwd<float, uint16_t>(p, as_stream(stream));
  else
    launch_fwd<float, float>(p, as_stream(stream));
  return check_launch(fn);
}

extern "C" size_t o5_resnorm_bwd_workspace_bytes(o5_dtype xt, o5_dtype dt, int N, int D) {
  if (check_common("o5_resnorm_bwd_workspace_bytes", xt, dt, N, D) != O5_OK) return 0;
  return static_cast<size_t>(row_blocks(N, D, kBwdBlocks)) * 2 * D * sizeof(float);
}

extern "C" int o5_resnorm_bwd(o5_dtype xt, o5_dtype dt, int N, int D, const void* xo, const void* u, const void* gate,
                              size_t ldg, const float* w_post, const float* rho, const float* w_pre,
                              const float* r_post, const float* r_pre, const void* dxo, const void* dn, void* dx,
                              void* du, void* dgate, size_t lddg, float* dw_post, float* drho, float* dw_pre, void* ws,
                              size_t ws_bytes, void* stream) {
  const char* fn = "o5_resnorm_bwd";
  O5_TRY(check_common(fn, xt, dt, N, D));
  O5_CHECK(u != nullptr || w_pre != nullptr, O5_E_ARG, "%s: u and w_pre are both NULL", fn);
  O5_CHECK(u != nullptr || gate == nullptr, O5_E_ARG, "%s: a gate needs u", fn);
  O5_TRY(check_gate(fn, "ldg", gate, ldg, D));
  O5_TRY(check_gate(fn, "lddg", gate, lddg, D));
  O5_PTR(dxo, "dxo");
  O5_PTR(dx, "dx");
  if (u) {
    O5_PTR(u, "u");
    O5_PTR(w_post, "w_post");
    O5_PTR(rho, "rho");
    O5_PTR(r_post, "r_post");
    O5_PTR(du, "du");
    O5_PTR(dw_post, "dw_post");
    O5_PTR(drho, "drho");
  }
  if (gate) {
    O5_PTR(gate, "gate");
    O5_PTR(dgate, "dgate");
  }
  if (w_pre) {
    O5_PTR(xo, "xo");
    O5_PTR(w_pre, "w_pre");
    O5_PTR(r_pre, "r_pre");
    O5_PTR(dn, "dn");
    O5_PTR(dw_pre, "dw_pre");
  }
  O5_CHECK(ws != nullptr && ws_bytes >= o5_resnorm_bwd_workspace_bytes(xt, dt, N, D), O5_E_WORKSPACE,
           "%s: ws is NULL or ws_bytes=%zu is too small", fn, ws_bytes);
  O5_PTR(ws, "ws");
  const NormBwd p = {xo, u, gate, w_post, rho, w_pre, r_post, r_pre, dxo, dn, dx, du, dgate, static_cast<float*>(ws), N, D,
                     ldg, lddg};
  if (xt == O5_BF16)
    launch_bwd<uint16_t, uint16_t>(p, as_stream(stream));
  else if (dt == O5_BF16)
    launch_bwd<float, uint16_t>(p, as_stream(stream));
  else
    launch_bwd<float, float>(p, as_stream(stream));
  const dim3 grid((D + 63) / 64, (u ? 1 : 0) + (w_pre ? 1 : 0));
  hipLaunchKernelGGL(resnorm_columns, grid, dim3(1024), 0, as_stream(stream), row_blocks(N, D, kBwdBlocks), D,
                     static_cast<const float*>(ws), w_post, rho, w_pre ? dw_pre : nullptr, drho, dw_post);
  return check_launch(fn);
}
