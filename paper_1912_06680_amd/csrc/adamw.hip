// AdamW over many tensors in one launch, its moments in 32 bits or in 8,
// o5_adamw_*.
//
// A plan, built on the host and copied to the device once by the caller,
// lists the tensors and cuts them into chunks of kChunk elements; a block
// takes a chunk, so that hundreds of small tensors fill the chip like one
// large one.  HBM-bound.
//
// Moments in 8 bits: 256 consecutive elements share the exponent a =
// floor(log2 max|x|) and each keeps 3 bits of mantissa and its own exponent
// below it: m a sign and 4 bits (13 binades below a, then evenly down to 0), v
// 5 bits (29 binades; v has the square of m's range), never 0 for a positive
// v, so that no step divides by eps alone.  They are rounded up with the
// chance of what is cut off: v changes by (1 - beta2) of itself per step, far
// below half a code (1/16), and nearest rounding would leave it where it is.
// The chances come from a counter-based generator, so results repeat.
#include "common.h"
#include "reduce.h"

namespace o5 {
namespace {

constexpr uint64_t kMagic = 0x316e616c7077616full;  // the plan's first word
constexpr int kGroup = 256;                         // elements that share an exponent
constexpr int kChunk = 1024;                        // elements of a block: 168M parameters with 8-bit moments and their
                                                    // values took 847 us, with 2048 872 and with 4096 905
constexpr int kLowM = 13, kLowV = 29;               // binades below the largest that keep 3 bits
constexpr int kNanM = 0x7f, kNanV = 0xff;

struct Tensor {  // as the device reads it
  float* p;
  const void* g;
  void *m, *v;
  uint8_t *m_exp, *v_exp;
  uint16_t* p16;
  uint64_t n, at;  // elements; place in the flat moments of o5_adamw_moments
  float lr_scale, weight_decay;
  uint32_t g_bf16, bits;
};

struct Chunk {
  uint32_t tensor, index;
};

struct Header {
  uint64_t magic;
  uint32_t tensors, chunks;
  uint64_t bytes, pad;
};

__host__ __device__ inline const Tensor* tensors_of(const void* plan) {
  return reinterpret_cast<const Tensor*>(static_cast<const char*>(plan) + sizeof(Header));
}
__host__ __device__ inline const Chunk* chunks_of(const void* plan, uint32_t tensors) {
  return reinterpret_cast<const Chunk*>(tensors_of(plan) + tensors);
}

struct Consts {
  float lr, b1, b2, one_m_b1, one_m_b2, inv_bc1, inv_bc2, eps, clip_k;
  uint32_t key0, key1, step;
};

// The update of one element; m and v leave in 32 bits.  Every product and sum
// is rounded by itself, so that what is stored in 8 bits does not depend on
// how a compiler joins them.
__device__ __forceinline__ void update(const Consts& c, float lr, float keep, float g, float& p, float& m, float& v) {
#pragma clang fp contract(off)
  v = v * c.b2 + (g * g) * c.one_m_b2;
  const float root = sqrtf(v * c.inv_bc2);
  float gc = g;
  if (c.clip_k > 0.0f) {
    const float bound = root * c.clip_k;
    gc = fminf(fmaxf(g, -bound), bound);
  }
  m = m * c.b1 + gc * c.one_m_b1;
  p = p * keep - (m * c.inv_bc1) / (root + c.eps) * lr;
}

// ---------------------------------------------------------- 8-bit moments

__device__ __forceinline__ float pow2i(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
__device__ __forceinline__ int exponent(float x) { return static_cast<int>(__float_as_uint(x) >> 23) - 127; }

// The exponent that a group with the largest magnitude `top` shares: within
// [-90, 126] every value of a code and every scale here is a normal number.
__device__ __forceinline__ int group_exponent(float top) { return min(max(exponent(top), -90), 126); }

__device__ __forceinline__ int shared_exponent(int e) { return max(e - 127, -90); }

__device__ __forceinline__ float decode(uint32_t code, int a, int low) {
  const int field = code >> 3;
  const int mant = (code & 7) + (field > 0 ? 8 : 0);
  return static_cast<float>(mant) * pow2i(a - low - 3 + max(field, 1) - 1);
}
__device__ __forceinline__ float decode_m(uint32_t c, int a) {
  if ((c & 0x7f) == kNanM) return __uint_as_float(0x7fc00000u);
  const float x = decode(c & 0x7f, a, kLowM);
  return (c & 0x80) ? -x : x;
}
__device__ __forceinline__ float decode_v(uint32_t c, int a) {
  return c == kNanV ? __uint_as_float(0x7fc00000u) : decode(c, a, kLowV);
}

// |x| in steps of its binade's eighth, rounded up if `up` in [0, 1) fills the
// step: a carry past 15 is the next binade's code by itself.
__device__ __forceinline__ uint32_t encode(float mag, int a, int low, float up) {
#pragma clang fp contract(off)
  const float y = mag * pow2i(-a);
  const int t = max(exponent(y), -low);
  return static_cast<uint32_t>((t + low) * 8 + static_cast<int>(floorf(y * pow2i(3 - t) + up)));
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ uint32_t encode_m(float x, int a, float up) {
  if (!finite(x)) return kNanM;
  const uint32_t c = min(encode(fabsf(x), a, kLowM, up), 126u);
  return (x < 0.0f && c > 0) ? c + 128 : c;
}
__device__ __forceinline__ uint32_t encode_v(float x, int a, float up) {
  if (!finite(x)) return kNanV;
  const uint32_t c = min(encode(x, a, kLowV, up), 254u);
  return x > 0.0f ? max(c, 1u) : c;
}

// Philox4x32-7 (Salmon, Moraes, Dror, Shaw, SC'11).
__device__ __forceinline__ void philox4x32_7(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t p0 = static_cast<uint64_t>(c[0]) * 0xD2511F53u, p1 = static_cast<uint64_t>(c[2]) * 0xCD9E8D57u;
    const uint32_t n0 = static_cast<uint32_t>(p1 >> 32) ^ c[1] ^ k0, n2 = static_cast<uint32_t>(p0 >> 32) ^ c[3] ^ k1;
    c[0] = n0;
    c[1] = static_cast<uint32_t>(p1);
    c[2] = n2;
    c[3] = static_cast<uint32_t>(p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// ----------------------------------------------------------------- kernels

// Four elements from i on, as they are stored; the tensor's tail (n < 4 of
// them) one by one.  The stream is touched once per step, hence the
// non-temporal hints.
template <typename V, typename T>
__device__ __forceinline__ V load_run(const T* p, size_t i) {
  return __builtin_nontemporal_load(reinterpret_cast<const V*>(p + i));
}
template <typename V, typename T>
__device__ __forceinline__ void store_run(T* p, size_t i, V v) {
  __builtin_nontemporal_store(v, reinterpret_cast<V*>(p + i));
}
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <bool kFull>
__device__ __forceinline__ f32x4 load4(const float* p, size_t i, int n) {
  if (kFull || n == 4) return load_run<f32x4>(p, i);
  f32x4 x;
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = j < n ? p[i + j] : 0.0f;
  return x;
}
template <bool kFull>
__device__ __forceinline__ u32x2 load4(const uint16_t* p, size_t i, int n) {
  if (kFull || n == 4) return load_run<u32x2>(p, i);
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = j < n ? p[i + j] : 0;
  return u32x2{w[0] | (w[1] << 16), w[2] | (w[3] << 16)};
}
template <bool kFull>
__device__ __forceinline__ uint32_t load4(const uint8_t* p, size_t i, int n) {
  if (kFull || n == 4) return load_run<uint32_t>(p, i);
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) w |= (j < n ? static_cast<uint32_t>(p[i + j]) : 0) << (8 * j);
  return w;
}
__device__ __forceinline__ float element(f32x4 x, int j) { return x[j]; }
__device__ __forceinline__ float element(u32x2 x, int j) {
  return __uint_as_float((j & 1) ? x[j >> 1] & 0xffff0000u : x[j >> 1] << 16);
}

template <bool kFull>
__device__ __forceinline__ void store4(float* p, size_t i, int n, f32x4 x) {
  if (kFull || n == 4) {
    store_run(p, i, x);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[i + j] = x[j];
  }
}
template <bool kFull>
__device__ __forceinline__ void store4(uint16_t* p, size_t i, int n, f32x4 x) {
  if (kFull || n == 4) {
    store_run(p, i, u32x2{f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3])});
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[i + j] = f32_to_bf16_bits(x[j]);
  }
}
template <bool kFull>
__device__ __forceinline__ void store4(uint8_t* p, size_t i, int n, uint32_t w) {
  if (kFull || n == 4) {
    store_run(p, i, w);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[i + j] = static_cast<uint8_t>(w >> (8 * j));
  }
}

// How many of the four elements from i on the tensor has.
__device__ __forceinline__ int count4(uint64_t n, size_t i) { return i >= n ? 0 : n - i < 4 ? static_cast<int>(n - i) : 4; }

constexpr int kRuns = kChunk / 1024;  // of four elements, for a thread

template <bool kFull, typename G>
__device__ __forceinline__ void step32(const Tensor& t, const Consts& c, size_t i0, float lr, float keep) {
  const G* gp = static_cast<const G*>(t.g);
  float *mp = static_cast<float*>(t.m), *vp = static_cast<float*>(t.v);
  f32x4 p[kRuns], m[kRuns], v[kRuns];
  decltype(load4<true>(gp, 0, 4)) g[kRuns];
  int n[kRuns];
#pragma unroll
  for (int k = 0; k < kRuns; ++k) {  // every load before the first use
    const size_t i = i0 + k * 1024;
    n[k] = kFull ? 4 : count4(t.n, i);
    p[k] = load4<kFull>(t.p, i, n[k]);
    g[k] = load4<kFull>(gp, i, n[k]);
    m[k] = load4<kFull>(mp, i, n[k]);
    v[k] = load4<kFull>(vp, i, n[k]);
  }
#pragma unroll
  for (int k = 0; k < kRuns; ++k) {
    const size_t i = i0 + k * 1024;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float pj = p[k][j], mj = m[k][j], vj = v[k][j];
      update(c, lr, keep, element(g[k], j), pj, mj, vj);
      p[k][j] = pj, m[k][j] = mj, v[k][j] = vj;
    }
    store4<kFull>(t.p, i, n[k], p[k]);
    store4<kFull>(mp, i, n[k], m[k]);
    store4<kFull>(vp, i, n[k], v[k]);
    if (t.p16) store4<kFull>(t.p16, i, n[k], p[k]);
  }
}

// A wave's run of 4 x 64 elements is one group.
template <bool kFull, typename G>
__device__ __forceinline__ void step8(const Tensor& t, uint32_t index, const Consts& c, size_t i0, float lr, float keep) {
  const G* gp = static_cast<const G*>(t.g);
  uint8_t *mp = static_cast<uint8_t*>(t.m), *vp = static_cast<uint8_t*>(t.v);
  f32x4 p[kRuns];
  decltype(load4<true>(gp, 0, 4)) g[kRuns];
  uint32_t mc[kRuns], vc[kRuns];
  int n[kRuns], am[kRuns], av[kRuns];
#pragma unroll
  for (int k = 0; k < kRuns; ++k) {
    const size_t i = i0 + k * 1024, group = i / kGroup;
    n[k] = kFull ? 4 : count4(t.n, i);
    const bool any = kFull || group * kGroup < t.n;
    p[k] = load4<kFull>(t.p, i, n[k]);
    g[k] = load4<kFull>(gp, i, n[k]);
    mc[k] = load4<kFull>(mp, i, n[k]);
    vc[k] = load4<kFull>(vp, i, n[k]);
    am[k] = any ? t.m_exp[group] : 127;
    av[k] = any ? t.v_exp[group] : 127;
  }
#pragma unroll
  for (int k = 0; k < kRuns; ++k) {
    const size_t i = i0 + k * 1024, group = i / kGroup;
    const int em = shared_exponent(am[k]), ev = shared_exponent(av[k]);
    float m[4], v[4], tm = 0.0f, tv = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float pj = p[k][j];
      m[j] = decode_m((mc[k] >> (8 * j)) & 0xff, em);
      v[j] = decode_v((vc[k] >> (8 * j)) & 0xff, ev);
      update(c, lr, keep, element(g[k], j), pj, m[j], v[j]);
      p[k][j] = pj;
      if (j >= n[k]) m[j] = v[j] = 0.0f;
      tm = fmaxf(tm, finite(m[j]) ? fabsf(m[j]) : 0.0f);
      tv = fmaxf(tv, finite(v[j]) ? v[j] : 0.0f);
    }
    const int nm = group_exponent(wave_max(tm)), nv = group_exponent(wave_max(tv));
    uint32_t w[4] = {static_cast<uint32_t>(i / 4), static_cast<uint32_t>(i >> 34), c.step, index};
    philox4x32_7(w, c.key0, c.key1);
    uint32_t mo = 0, vo = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      mo |= encode_m(m[j], nm, static_cast<float>(w[j] & 0xffff) * 0x1p-16f) << (8 * j);
      vo |= encode_v(v[j], nv, static_cast<float>(w[j] >> 16) * 0x1p-16f) << (8 * j);
    }
    store4<kFull>(t.p, i, n[k], p[k]);
    store4<kFull>(mp, i, n[k], mo);
    store4<kFull>(vp, i, n[k], vo);
    if (t.p16) store4<kFull>(t.p16, i, n[k], p[k]);
    if ((threadIdx.x & 63) == 0 && (kFull || group * kGroup < t.n)) {
      t.m_exp[group] = static_cast<uint8_t>(nm + 127);
      t.v_exp[group] = static_cast<uint8_t>(nv + 127);
    }
  }
}

// A block takes a chunk, a thread four consecutive elements, so that a wave
// holds one group of 256 and the new exponent is one reduction within it.  HBM-
// bound: 168M parameters with bf16 gradients, 8-bit moments and bf16 copies, 16
// bytes each, 541 to 615 us, 5.0 to 4.4 TB/s; 5.3M with 32-bit moments 27 us, 5.9 TB/s
// (partly from the caches).
__global__ void __launch_bounds__(256) adamw_kernel(const void* __restrict__ plan, uint32_t tensors, uint32_t first,
                                                    Consts c) {
  const Chunk ch = chunks_of(plan, tensors)[first + blockIdx.x];
  const Tensor t = tensors_of(plan)[ch.tensor];
  const float lr = c.lr * t.lr_scale;
  const float keep = static_cast<float>(1.0 - static_cast<double>(lr) * static_cast<double>(t.weight_decay));
  const size_t i = static_cast<size_t>(ch.index) * kChunk + threadIdx.x * 4;
  const bool full = (static_cast<size_t>(ch.index) + 1) * kChunk <= t.n;
  if (t.bits == 32) {
    if (t.g_bf16)
      full ? step32<true, uint16_t>(t, c, i, lr, keep) : step32<false, uint16_t>(t, c, i, lr, keep);
    else
      full ? step32<true, float>(t, c, i, lr, keep) : step32<false, float>(t, c, i, lr, keep);
  } else {
    if (t.g_bf16)
      full ? step8<true, uint16_t>(t, ch.tensor, c, i, lr, keep) : step8<false, uint16_t>(t, ch.tensor, c, i, lr, keep);
    else
      full ? step8<true, float>(t, ch.tensor, c, i, lr, keep) : step8<false, float>(t, ch.tensor, c, i, lr, keep);
  }
}

template <bool kFull>
__device__ __forceinline__ void moments(const Tensor& t, size_t i0, float* mo, float* vo) {
  f32x4 m[kRuns], v[kRuns];
  int n[kRuns];
  if (t.bits == 32) {
#pragma unroll
    for (int k = 0; k < kRuns; ++k) {
      const size_t i = i0 + k * 1024;
      n[k] = kFull ? 4 : count4(t.n, i);
      m[k] = load4<kFull>(static_cast<const float*>(t.m), i, n[k]);
      v[k] = load4<kFull>(static_cast<const float*>(t.v), i, n[k]);
    }
  } else {
    uint32_t mc[kRuns], vc[kRuns];
    int am[kRuns], av[kRuns];
#pragma unroll
    for (int k = 0; k < kRuns; ++k) {
      const size_t i = i0 + k * 1024, group = i / kGroup;
      n[k] = kFull ? 4 : count4(t.n, i);
      const bool any = kFull || group * kGroup < t.n;
      mc[k] = load4<kFull>(static_cast<const uint8_t*>(t.m), i, n[k]);
      vc[k] = load4<kFull>(static_cast<const uint8_t*>(t.v), i, n[k]);
      am[k] = any ? t.m_exp[group] : 127;
      av[k] = any ? t.v_exp[group] : 127;
    }
#pragma unroll
    for (int k = 0; k < kRuns; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[k][j] = decode_m((mc[k] >> (8 * j)) & 0xff, shared_exponent(am[k]));
        v[k][j] = decode_v((vc[k] >> (8 * j)) & 0xff, shared_exponent(av[k]));
      }
  }
#pragma unroll
  for (int k = 0; k < kRuns; ++k) {
    store4<kFull>(mo, i0 + k * 1024, n[k], m[k]);
    store4<kFull>(vo, i0 + k * 1024, n[k], v[k]);
  }
}

// The moments as they are stored, in fp32.  HBM-bound: 168M of 8 bits 272 to 280
// us, 6.0 TB/s, most of it written.
__global__ void __launch_bounds__(256) adamw_moments(const void* __restrict__ plan, uint32_t tensors, uint32_t first,
                                                     float* __restrict__ mo, float* __restrict__ vo) {
  const Chunk ch = chunks_of(plan, tensors)[first + blockIdx.x];
  const Tensor t = tensors_of(plan)[ch.tensor];
  const size_t i = static_cast<size_t>(ch.index) * kChunk + threadIdx.x * 4;
  if ((static_cast<size_t>(ch.index) + 1) * kChunk <= t.n)
    moments<true>(t, i, mo + t.at, vo + t.at);
  else
    moments<false>(t, i, mo + t.at, vo + t.at);
}

// A launch holds fewer than 2^32 threads in a dimension (with more the grid
// wraps and the rest is never run, without an error), so that a plan of more
// chunks goes out in several: launch(first chunk, blocks).
template <class F>
void launch_chunks(uint32_t chunks, F&& launch) {
  constexpr uint32_t kMost = 0xffffffffu / 256;
  for (uint32_t first = 0; first < chunks; first += kMost) launch(first, std::min(chunks - first, kMost));
}

#define O5_TRY(expr)              \
  do {                            \
    const int st_ = (expr);       \
    if (st_ != O5_OK) return st_; \
  } while (0)

int check_tensors(const char* fn, int count, const o5_adamw_tensor* t, uint64_t* chunks) {
  O5_CHECK(count >= 1 && count <= (1 << 20), O5_E_SHAPE, "%s: count=%d must be in 1..2^20", fn, count);
  O5_CHECK(t != nullptr, O5_E_NULL, "%s: argument 'tensors' is NULL", fn);
  uint64_t c = 0;
  for (int i = 0; i < count; ++i) {
    O5_CHECK(t[i].n >= 1 && t[i].n < (1ull << 40), O5_E_SHAPE, "%s: tensor %d: n must be in 1..2^40-1", fn, i);
    O5_CHECK(t[i].g_dt == O5_F32 || t[i].g_dt == O5_BF16, O5_E_DTYPE, "%s: tensor %d: unknown g_dt", fn, i);
    O5_CHECK(t[i].bits == 32 || t[i].bits == 8, O5_E_ARG, "%s: tensor %d: bits=%d must be 32 or 8", fn, i, t[i].bits);
    O5_CHECK(t[i].lr_scale >= 0.0f && std::isfinite(t[i].lr_scale) && t[i].weight_decay >= 0.0f &&
                 std::isfinite(t[i].weight_decay),
             O5_E_ARG, "%s: tensor %d: need lr_scale >= 0 and weight_decay >= 0", fn, i);
    O5_PTR_IN(fn, t[i].p, "p");
    O5_PTR_IN(fn, t[i].g, "g");
    O5_PTR_IN(fn, t[i].m, "m");
    O5_PTR_IN(fn, t[i].v, "v");
    O5_OPT_PTR_IN(fn, t[i].p_bf16, "p_bf16");
    if (t[i].bits == 8)
      O5_CHECK(t[i].m_exp != nullptr && t[i].v_exp != nullptr, O5_E_NULL, "%s: tensor %d: m_exp or v_exp is NULL", fn, i);
    c += (t[i].n + kChunk - 1) / kChunk;
  }
  O5_CHECK(c < (1ull << 31), O5_E_SHAPE, "%s: too many elements", fn);
  *chunks = c;
  return O5_OK;
}

size_t plan_bytes(int count, uint64_t chunks) {
  return align_up(sizeof(Header) + static_cast<size_t>(count) * sizeof(Tensor) + chunks * sizeof(Chunk), 16);
}

int check_plan(const char* fn, const void* plan, const void* plan_dev) {
  O5_PTR_IN(fn, plan, "plan");
  O5_PTR_IN(fn, plan_dev, "plan_dev");
  O5_CHECK(static_cast<const Header*>(plan)->magic == kMagic, O5_E_ARG, "%s: 'plan' was not written by o5_adamw_plan", fn);
  return O5_OK;
}

}  // namespace
}  // namespace o5

using namespace o5;

extern "C" size_t o5_adamw_plan_bytes(int count, const o5_adamw_tensor* tensors) {
  uint64_t chunks = 0;
  if (check_tensors("o5_adamw_plan_bytes", count, tensors, &chunks) != O5_OK) return 0;
  return plan_bytes(count, chunks);
}

extern "C" int o5_adamw_plan(int count, const o5_adamw_tensor* tensors, void* plan, size_t bytes) {
  const char* fn = "o5_adamw_plan";
  uint64_t chunks = 0;
  O5_TRY(check_tensors(fn, count, tensors, &chunks));
  O5_PTR(plan, "plan");
  O5_CHECK(bytes >= plan_bytes(count, chunks), O5_E_WORKSPACE, "%s: bytes=%zu is too small", fn, bytes);
  Header* h = static_cast<Header*>(plan);
  *h = {kMagic, static_cast<uint32_t>(count), static_cast<uint32_t>(chunks), plan_bytes(count, chunks), 0};
  Tensor* out = const_cast<Tensor*>(tensors_of(plan));
  Chunk* ch = const_cast<Chunk*>(chunks_of(plan, h->tensors));
  uint64_t at = 0;
  for (int i = 0; i < count; ++i) {
    const o5_adamw_tensor& t = tensors[i];
    out[i] = {t.p, t.g, t.m, t.v, t.m_exp, t.v_exp, t.p_bf16, t.n, at, t.lr_scale, t.weight_decay,
              t.g_dt == O5_BF16 ? 1u : 0u, static_cast<uint32_t>(t.bits)};
    at += (t.n + kGroup - 1) / kGroup * kGroup;
    const uint64_t k = (t.n + kChunk - 1) / kChunk;
    for (uint64_t j = 0; j < k; ++j) *ch++ = {static_cast<uint32_t>(i), static_cast<uint32_t>(j)};
  }
  return O5_OK;
}

extern "C" int o5_adamw_step(const void* plan, const void* plan_dev, o5_adam_hp hp, uint64_t seed, int step, void* stream) {
  const char* fn = "o5_adamw_step";
  O5_CHECK(step >= 1, O5_E_ARG, "%s: step=%d must be >= 1", fn, step);
  O5_CHECK(hp.beta1 >= 0.0f && hp.beta1 < 1.0f && hp.beta2 >= 0.0f && hp.beta2 < 1.0f, O5_E_ARG,
           "%s: betas must lie in [0, 1)", fn);
  O5_CHECK(hp.eps > 0.0f && hp.lr >= 0.0f, O5_E_ARG, "%s: need eps > 0 and lr >= 0", fn);
  O5_TRY(check_plan(fn, plan, plan_dev));
  const Header* h = static_cast<const Header*>(plan);
  Consts c;
  c.lr = hp.lr;
  c.b1 = hp.beta1;
  c.b2 = hp.beta2;
  c.one_m_b1 = 1.0f - hp.beta1;
  c.one_m_b2 = 1.0f - hp.beta2;
  // bias corrections in double on the host, then rounded once
  c.inv_bc1 = static_cast<float>(1.0 / (1.0 - std::pow(static_cast<double>(hp.beta1), step)));
  c.inv_bc2 = static_cast<float>(1.0 / (1.0 - std::pow(static_cast<double>(hp.beta2), step)));
  c.eps = hp.eps;
  c.clip_k = hp.clip_k;
  c.key0 = static_cast<uint32_t>(seed);
  c.key1 = static_cast<uint32_t>(seed >> 32);
  c.step = static_cast<uint32_t>(step);
  launch_chunks(h->chunks, [&](uint32_t first, uint32_t blocks) {
    hipLaunchKernelGGL(adamw_kernel, dim3(blocks), dim3(256), 0, as_stream(stream), plan_dev, h->tensors, first, c);
  });
  return check_launch(fn);
}

extern "C" int o5_adamw_moments(const void* plan, const void* plan_dev, float* m, float* v, void* stream) {
  const char* fn = "o5_adamw_moments";
  O5_TRY(check_plan(fn, plan, plan_dev));
  O5_PTR(m, "m");
  O5_PTR(v, "v");
  const Header* h = static_cast<const Header*>(plan);
  launch_chunks(h->chunks, [&](uint32_t first, uint32_t blocks) {
    hipLaunchKernelGGL(adamw_moments, dim3(blocks), dim3(256), 0, as_stream(stream), plan_dev, h->tensors, first, m, v);
  });
  return check_launch(fn);
}
