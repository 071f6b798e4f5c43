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

// ------------------------------------------------------------ chunked form
//
// With the state S before a chunk of L steps, r_i the last reset at or before
// its step i (-1 if none) and e = 0 for the passes that run backward in time
// (whose carried state has decayed already), else 1:
//
//   o_i = oscale (r_i < 0) l^(i+e) S^T q_i + sum_{r_i <= j <= i} p_ij v_j
//   p_ij = oscale kscale l^(i-j) q_i . k_j
//   S' = (r_{L-1} < 0) l^L S + sum_{j >= r_{L-1}} kscale l^(L-e-j) k_j v_j^T
//
// A block of 4 waves takes one state and runs through its chunks; a wave owns
// a quarter of the state's columns in its accumulators.  Products are formed
// transposed (o^T = S^T q^T, v^T p^T), so that the accumulators of S and the
// tiles of p are, as they lie, operands of the next product.
//
// The reduction index of every product runs in blocks of 32; of a block, lane
// group g = lane / 16 holds 4 g + r and 16 + 4 g + r (r = 0..3), which is how
// two 16 x 16 accumulators hold their rows.  Rows of q, k and p lie in LDS with
// the runs of 4 of a block in the order 0 4 1 5 2 6 3 7, so that a group's two
// runs are one read.

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kPad = 16;  // bytes after each row in LDS: 16 rows start on 16 different groups of 4 banks

template <typename E> struct Mx;

template <> struct Mx<uint16_t> {
  static constexpr int CL = 64;  // steps of a chunk
  typedef bf16x8 Frag;
  static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ Frag rows(const char* at) { return *reinterpret_cast<const Frag*>(at); }
  // columns: rows 4 g + r and 16 + 4 g + r of column lane % 16, of a tile whose runs of 4 columns lie `run` bytes apart
  template <int STRIDE, int RUN>
  static __device__ __forceinline__ Frag columns(const char* tile, int lane) {
    const char* p = tile + (4 * (lane >> 4) + ((lane & 15) >> 2)) * STRIDE + (lane & 3) * RUN;
    struct {
      s16x4 a, b;
    } f;
    f.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p));
    f.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 16 * STRIDE));
    return __builtin_bit_cast(Frag, f);
  }
  static __device__ __forceinline__ float get(const Frag& f, int i) { return static_cast<float>(f[i]); }
  static __device__ __forceinline__ void set(Frag& f, int i, float v) { f[i] = static_cast<__bf16>(v); }
  static __device__ __forceinline__ void store4(void* p, f32x4 v) {
    *static_cast<u32x2*>(p) = u32x2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
  }
  // 16 bytes of a row into LDS, their runs of 4 in the blocks' order
  static __device__ __forceinline__ void put(char* row, int unit, u32x4 x) {
    const int m = unit & 3;
    char* p = row + (unit >> 2) * 64 + ((m & 1) * 4 + (m >> 1)) * 8;
    *reinterpret_cast<u32x2*>(p) = u32x2{x[0], x[1]};
    *reinterpret_cast<u32x2*>(p + 16) = u32x2{x[2], x[3]};
  }
};

template <> struct Mx<float> {
  static constexpr int CL = 32;
  struct Frag {
    f32x4 h[2];
  };
  static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.h[h][r], b.h[h][r], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ Frag rows(const char* at) {
    return {{*reinterpret_cast<const f32x4*>(at), *reinterpret_cast<const f32x4*>(at + 16)}};
  }
  template <int STRIDE, int RUN>
  static __device__ __forceinline__ Frag columns(const char* tile, int lane) {
    const char* p = tile + 4 * (lane >> 4) * STRIDE + ((lane & 15) >> 2) * RUN + (lane & 3) * 4;
    Frag f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) f.h[h][r] = *reinterpret_cast<const float*>(p + (16 * h + r) * STRIDE);
    return f;
  }
  static __device__ __forceinline__ float get(const Frag& f, int i) { return f.h[i >> 2][i & 3]; }
  static __device__ __forceinline__ void set(Frag& f, int i, float v) { f.h[i >> 2][i & 3] = v; }
  static __device__ __forceinline__ void store4(void* p, f32x4 v) { *static_cast<f32x4*>(p) = v; }
  static __device__ __forceinline__ void put(char* row, int unit, u32x4 x) {
    const int q = unit & 7;
    *reinterpret_cast<u32x4*>(row + (unit >> 3) * 128 + ((q & 3) * 2 + (q >> 2)) * 16) = x;
  }
};

// l^n for n >= 0, exact at 0 (l2 = log2 l, -inf for l = 0).
__device__ __forceinline__ float power(float l2, int n) {
  return n == 0 ? 1.0f : __builtin_amdgcn_exp2f(l2 * static_cast<float>(n));
}

template <typename E, int DA, int DC>
struct Tiles {
  static constexpr int CL = Mx<E>::CL, ES = sizeof(E);
  static constexpr int QS = DA * ES + kPad, VS = DC * ES + kPad, PS = CL * ES + kPad;  // row strides
  alignas(16) char q[CL * QS];
  alignas(16) char k[CL * QS];
  alignas(16) char v[CL * VS];
  alignas(16) char p[CL * PS];
};

// One operand's rows of a chunk on the way from memory to LDS.
template <typename E, int D>
struct Stage {
  static constexpr int CL = Mx<E>::CL, U = D * static_cast<int>(sizeof(E)) / 16, N = CL * U / 256, PER = 16 / sizeof(E);
  u32x4 x[N];
  // rows u0 .. u0 + L - 1 of the pass's order; columns from `d` on are zero
  __device__ __forceinline__ void load(const E* base, size_t ld, const LinPass& p, int b, int u0, int L, int d) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int idx = threadIdx.x + n * 256, row = idx / U, c = (idx % U) * PER;
      x[n] = u32x4{0, 0, 0, 0};
      if (row < L && c < d) {
        const int t = p.rev ? p.T - 1 - (u0 + row) : u0 + row;
        x[n] = *reinterpret_cast<const u32x4*>(base + (static_cast<size_t>(t) * p.B + b) * ld + c);
      }
    }
  }
  template <int STRIDE, bool PERM>
  __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int idx = threadIdx.x + n * 256, row = idx / U, unit = idx % U;
      if (PERM)
        Mx<E>::put(lds + row * STRIDE, unit, x[n]);
      else
        *reinterpret_cast<u32x4*>(lds + row * STRIDE + unit * 16) = x[n];
    }
  }
};

// Where the chunks of a split begin and what it starts from.
struct Split {
  int chunks;       // of one split
  float* states;    // [splits][B * nkv][DA * DC] in the accumulators' order, or NULL: one split
  float* keep;      // [splits][B * nkv]: the factor on the state across the split, -1 where a reset cuts it off
};

// kOut: write the outputs; else only add up each split's own part of the state.
// kMany: gk > 1, the outputs are sums over the group.
template <typename E, int DA, int DC, bool kOut, bool kMany>
__global__ void __launch_bounds__(256, 2) linattn_chunks(LinPass p, Split sp) {
  typedef Mx<E> M;
  typedef typename M::Frag Frag;
  typedef Tiles<E, DA, DC> TL;
  constexpr int CL = M::CL, ES = sizeof(E), NI = CL / 16, NB = CL / 32;
  constexpr int NA = DA / 16, NC = DC / 64, NU = DA / 32;
  __shared__ TL lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g4 = lane >> 4;
  const int heads = kOut ? p.nkv * p.gq : p.nkv;
  const int b = blockIdx.x / heads, hq = blockIdx.x % heads, n = kOut ? hq / p.gq : hq;
  const int chunks = (p.T + CL - 1) / CL;
  const int c0 = blockIdx.y * sp.chunks, c1 = min(chunks, c0 + sp.chunks);
  const float l2 = log2f(p.decay[n]);
  const int e = p.rev ? 0 : 1;
  const int bn = b * p.nkv + n;
  const size_t sbase = static_cast<size_t>(bn) * p.da * p.dc;
  const int cw = wave * (DC / 4);  // the wave's first column

  // the state before the first chunk
  f32x4 S[NA][NC];
  if (kOut && sp.states) {
    const f32x4* st = reinterpret_cast<const f32x4*>(sp.states) +
                      (static_cast<size_t>(blockIdx.y) * p.B * p.nkv + bn) * (DA * DC / 4) + wave * NA * NC * 64;
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int c = 0; c < NC; ++c) S[a][c] = st[(a * NC + c) * 64 + lane];
  } else {
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int row = a * 16 + g4 * 4, col = cw + c * 16 + l16;
        S[a][c] = f32x4{0, 0, 0, 0};
        if (kOut && p.s0 && row < p.da && col < p.dc) {
          if (p.s0t) {
            S[a][c] = *reinterpret_cast<const f32x4*>(p.s0 + sbase + static_cast<size_t>(col) * p.da + row);
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) S[a][c][r] = p.s0[sbase + static_cast<size_t>(row + r) * p.dc + col];
          }
        }
      }
  }

  const E* qb = static_cast<const E*>(p.q) + static_cast<size_t>(hq) * p.da;
  const E* kb = static_cast<const E*>(p.k) + static_cast<size_t>(n) * p.gk * p.da;
  const E* vb = static_cast<const E*>(p.v) + static_cast<size_t>(n) * p.gk * p.dc;
  E* ob = static_cast<E*>(p.o) + static_cast<size_t>(hq) * p.dc;
  Stage<E, DA> sq, sk;
  Stage<E, DC> sv;
  bool cut_any = false;  // a reset in this split so far
  f32x4 acc[kMany ? NI : 1][NC];

  auto fetch = [&](int it) {  // the tiles of flat index it = chunk * gk + g
    const int ch = c0 + (kMany ? it / p.gk : it), g = kMany ? it % p.gk : 0;
    const int u0 = ch * CL, L = min(CL, p.T - u0);
    if (kOut && g == 0) sq.load(qb, p.ldq, p, b, u0, L, p.da);
    sk.load(kb + static_cast<size_t>(g) * p.da, p.ldk, p, b, u0, L, p.da);
    sv.load(vb + static_cast<size_t>(g) * p.dc, p.ldv, p, b, u0, L, p.dc);
  };

  const int total = (c1 - c0) * (kMany ? p.gk : 1);
  fetch(0);
  for (int it = 0; it < total; ++it) {
    const int g = kMany ? it % p.gk : 0, u0 = (c0 + (kMany ? it / p.gk : it)) * CL, L = min(CL, p.T - u0);
    const bool first = g == 0, last = !kMany || g == p.gk - 1;
    const int ni = (L + 15) / 16, nb = (L + 31) / 32;
    if (kOut && first) sq.template store<TL::QS, true>(lds.q);
    sk.template store<TL::QS, true>(lds.k);
    sv.template store<TL::VS, false>(lds.v);
    // bit i: a reset before the chunk's step i
    bool flag = false;
    if (p.reset && lane < L) {
      const int u = u0 + lane;
      if (!p.rev)
        flag = p.reset[static_cast<size_t>(u) * p.B + b] != 0;
      else if (u > 0)
        flag = p.reset[static_cast<size_t>(p.T - u) * p.B + b] != 0;
    }
    const uint64_t resets = __ballot(flag);
    const int rl = resets ? 63 - __builtin_clzll(resets) : -1;  // r of the chunk's last step
    auto last_reset = [&](int i) {
      const uint64_t m = resets & (~0ull >> (63 - i));
      return m ? 63 - __builtin_clzll(m) : -1;
    };
    __syncthreads();
    if (it + 1 < total) fetch(it + 1);

    if (kOut) {  // p, 16 x 16 tiles at and below the diagonal, one after another to the waves
      constexpr int kTiles = NI * (NI + 1) / 2;
      for (int x = wave; x < kTiles + NI / 2; x += 4) {
        int ti, tj;
        if (x < kTiles) {
          ti = x >= 6 ? 3 : x >= 3 ? 2 : x >= 1 ? 1 : 0;
          tj = x - ti * (ti + 1) / 2;
        } else {  // the other half of an even row tile's last block of 32
          ti = (x - kTiles) * 2;
          tj = ti + 1;
        }
        if (ti >= ni) continue;
        f32x4 s = {0, 0, 0, 0};
        const int i = ti * 16 + l16;
        if (tj <= ti) {
#pragma unroll
          for (int u = 0; u < NU; ++u) {
            const Frag fk = M::rows(lds.k + (tj * 16 + l16) * TL::QS + u * 32 * ES + g4 * 8 * ES);
            const Frag fq = M::rows(lds.q + i * TL::QS + u * 32 * ES + g4 * 8 * ES);
            s = M::mma(fk, fq, s);
          }
          const int ri = last_reset(i);
          const float f = p.oscale * p.kscale;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int j = tj * 16 + g4 * 4 + r;
            s[r] = (j <= i && j >= ri) ? s[r] * (f * power(l2, max(i - j, 0))) : 0.0f;
          }
        }
        M::store4(lds.p + i * TL::PS + (tj >> 1) * 32 * ES + (g4 * 2 + (tj & 1)) * 4 * ES, s);
      }
      __syncthreads();
    }

    // the wave's columns of v
    Frag vf[NC][NB];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int u = 0; u < NB; ++u)
        vf[c][u] = M::template columns<TL::VS, 4 * ES>(lds.v + u * 32 * TL::VS + (cw + c * 16) * ES, lane);

    if (kOut) {
      // an infinity or NaN in v may not meet the zeros of p: it is taken out of the product and added one by one
      float odd = 0.0f;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int u = 0; u < NB; ++u)
#pragma unroll
          for (int i = 0; i < 8; ++i) odd = fmaf(M::get(vf[c][u], i), 0.0f, odd);
      const bool any_odd = __any(!(odd == 0.0f));
      Frag vp[NC][NB];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int u = 0; u < NB; ++u) {
          vp[c][u] = vf[c][u];
          if (any_odd) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (!(M::get(vf[c][u], i) * 0.0f == 0.0f)) M::set(vp[c][u], i, 0.0f);
          }
        }
      Frag sf[NC][NU];
      if (first) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) M::set(sf[c][u], i, S[2 * u + (i >> 2)][c][i & 3]);
      }
#pragma unroll
      for (int ti = 0; ti < NI; ++ti) {
        if (ti >= ni) break;
        f32x4(&o)[NC] = acc[kMany ? ti : 0];
        const int i = ti * 16 + l16, ri = last_reset(i);
        if (first) {
#pragma unroll
          for (int c = 0; c < NC; ++c) o[c] = f32x4{0, 0, 0, 0};
#pragma unroll
          for (int u = 0; u < NU; ++u) {
            const Frag fq = M::rows(lds.q + i * TL::QS + u * 32 * ES + g4 * 8 * ES);
#pragma unroll
            for (int c = 0; c < NC; ++c) o[c] = M::mma(sf[c][u], fq, o[c]);
          }
          const float f = p.oscale * power(l2, i + e);
#pragma unroll
          for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[c][r] = ri < 0 ? o[c][r] * f : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < ti / 2 + 1; ++u) {
          const Frag fp = M::rows(lds.p + i * TL::PS + u * 32 * ES + g4 * 8 * ES);
#pragma unroll
          for (int c = 0; c < NC; ++c) o[c] = M::mma(vp[c][u], fp, o[c]);
        }
        if (any_odd) {
#pragma unroll 1
          for (int j = max(ri, 0); j <= i; ++j) {
            const int q = (j >> 2) & 7;
            const E pj = *reinterpret_cast<const E*>(lds.p + i * TL::PS + (j >> 5) * 32 * ES +
                                                     (((q & 3) * 2 + (q >> 2)) * 4 + (j & 3)) * ES);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const E vj = *reinterpret_cast<const E*>(lds.v + j * TL::VS + (cw + c * 16 + g4 * 4 + r) * ES);
                const float x = elem<E>::to_f32(vj);
                if (!(x * 0.0f == 0.0f)) o[c][r] = fmaf(elem<E>::to_f32(pj), x, o[c][r]);
              }
          }
        }
        if (last && i < L) {
          const int t = p.rev ? p.T - 1 - (u0 + i) : u0 + i;
          E* row = ob + (static_cast<size_t>(t) * p.B + b) * p.ldo;
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const int col = cw + c * 16 + g4 * 4;
            if (col < p.dc) M::store4(row + col, o[c]);
          }
        }
      }
    }

    // the state after the chunk
    if (first) {
      const float f = power(l2, L);
#pragma unroll
      for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) S[a][c][r] = rl < 0 ? S[a][c][r] * f : 0.0f;
    }
    cut_any = cut_any || rl >= 0;
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      if (u >= nb) break;
      // what enters: in bf16 as a (hi, lo) pair, which keeps 16 bits of it
      Frag hi[NC], lo[NC];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = u * 32 + (i >> 2) * 16 + g4 * 4 + (i & 3);
        const float w = p.kscale * power(l2, max(L - e - j, 0));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const float x = j >= rl ? M::get(vf[c][u], i) * w : 0.0f;
          M::set(hi[c], i, x);
          if (ES == 2) {
            const float y = M::get(hi[c], i);
            M::set(lo[c], i, (y * 0.0f == 0.0f) ? x - y : 0.0f);
          }
        }
      }
#pragma unroll
      for (int a = 0; a < NA; ++a) {
        Frag kf = M::template columns<TL::QS, 8 * ES>(
            lds.k + u * 32 * TL::QS + (a >> 1) * 32 * ES + (a & 1) * 4 * ES, lane);
        if (rl > u * 32) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (u * 32 + (i >> 2) * 16 + g4 * 4 + (i & 3) < rl) M::set(kf, i, 0.0f);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          S[a][c] = M::mma(kf, hi[c], S[a][c]);
          if (ES == 2) S[a][c] = M::mma(kf, lo[c], S[a][c]);
        }
      }
    }
    __syncthreads();
  }

  if (kOut && sp.states) return;  // the scan has written the last state
  if (!kOut) {
    f32x4* st = reinterpret_cast<f32x4*>(sp.states) +
                (static_cast<size_t>(blockIdx.y) * p.B * p.nkv + bn) * (DA * DC / 4) + wave * NA * NC * 64;
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int c = 0; c < NC; ++c) st[(a * NC + c) * 64 + lane] = S[a][c];
    if (tid == 0)
      sp.keep[static_cast<size_t>(blockIdx.y) * p.B * p.nkv + bn] =
          cut_any ? -1.0f : power(l2, min(p.T, c1 * CL) - c0 * CL);
    return;
  }
  if (p.sT && (kMany || hq % p.gq == 0)) {
    const bool cut = p.rev && p.reset && p.reset[b] != 0;
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int row = a * 16 + g4 * 4, col = cw + c * 16 + l16;
        if (row >= p.da || col >= p.dc) continue;
        const f32x4 x = cut ? f32x4{0, 0, 0, 0} : S[a][c];
        if (p.s0t) {
          *reinterpret_cast<f32x4*>(p.sT + sbase + static_cast<size_t>(col) * p.da + row) = x;
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) p.sT[sbase + static_cast<size_t>(row + r) * p.dc + col] = x[r];
        }
      }
  }
}

// The state before each split, in place of the split's own part, and the last
// state: X_0 = S0, X_{s+1} = keep_s X_s + part_s.  A thread takes 4 rows of a
// column (one accumulator).
template <int DA, int DC>
__global__ void __launch_bounds__(256) linattn_scan(LinPass p, Split sp, int splits) {
  constexpr int NA = DA / 16, NC = DC / 64, Q = DA * DC / 4;
  const size_t idx = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  const int states = p.B * p.nkv;
  const int bn = static_cast<int>(idx / Q), x = static_cast<int>(idx % Q);
  const int lane = x & 63, tile = x >> 6, c = tile % NC, a = tile / NC % NA, wave = tile / (NC * NA);
  const int row = a * 16 + (lane >> 4) * 4, col = wave * (DC / 4) + c * 16 + (lane & 15);
  const bool in = row < p.da && col < p.dc;
  const size_t at = static_cast<size_t>(bn) * p.da * p.dc;
  f32x4 X = {0, 0, 0, 0};
  if (in && p.s0) {
    if (p.s0t) {
      X = *reinterpret_cast<const f32x4*>(p.s0 + at + static_cast<size_t>(col) * p.da + row);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) X[r] = p.s0[at + static_cast<size_t>(row + r) * p.dc + col];
    }
  }
  f32x4* st = reinterpret_cast<f32x4*>(sp.states) + idx;
  const size_t stride = static_cast<size_t>(states) * Q;
  for (int s = 0; s < splits; ++s) {
    const f32x4 part = st[s * stride];
    const float keep = sp.keep[static_cast<size_t>(s) * states + bn];
    st[s * stride] = X;
#pragma unroll
    for (int r = 0; r < 4; ++r) X[r] = keep < 0.0f ? part[r] : fmaf(keep, X[r], part[r]);
  }
  if (in && p.sT) {
    if (p.rev && p.reset && p.reset[bn / p.nkv] != 0) X = f32x4{0, 0, 0, 0};
    if (p.s0t) {
      *reinterpret_cast<f32x4*>(p.sT + at + static_cast<size_t>(col) * p.da + row) = X;
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) p.sT[at + static_cast<size_t>(row + r) * p.dc + col] = X[r];
    }
  }
}

int pad_head(int d) { return d <= 64 ? 64 : 128; }

// Splits of the T steps: where the states and their query heads are too few
// to fill the chip, so many that about 512 blocks (2 on each compute unit)
// run, of 4 chunks at least.
int plan_splits(o5_dtype dt, int T, int B, int nkv, int gq) {
  const int cl = dt == O5_BF16 ? Mx<uint16_t>::CL : Mx<float>::CL;
  const int chunks = (T + cl - 1) / cl;
  const long long blocks = static_cast<long long>(B) * nkv * gq;
  if (blocks >= 256) return 1;
  const int want = static_cast<int>((512 + blocks - 1) / blocks);
  return std::max(1, std::min(want, chunks / 4));
}

size_t pass_workspace(o5_dtype dt, int T, int B, int nkv, int gq, int da, int dc) {
  const int splits = plan_splits(dt, T, B, nkv, gq);
  if (splits == 1) return 0;
  return align_up(static_cast<size_t>(splits) * B * nkv * (pad_head(da) * pad_head(dc) + 1) * sizeof(float));
}

template <typename E, int DA, int DC>
void launch_chunks(o5_dtype dt, const LinPass& p, void* ws, hipStream_t s) {
  const int splits = plan_splits(dt, p.T, p.B, p.nkv, p.gq);
  const int chunks = (p.T + Mx<E>::CL - 1) / Mx<E>::CL;
  const unsigned states = static_cast<unsigned>(p.B) * p.nkv;
  Split sp = {chunks, nullptr, nullptr};
  int used = 1;
  if (splits > 1) {
    sp.chunks = (chunks + splits - 1) / splits;
    used = (chunks + sp.chunks - 1) / sp.chunks;
    sp.states = static_cast<float*>(ws);
    sp.keep = sp.states + static_cast<size_t>(used) * states * DA * DC;
    if (p.gk > 1)
      hipLaunchKernelGGL((linattn_chunks<E, DA, DC, false, true>), dim3(states, used), dim3(256), 0, s, p, sp);
    else
      hipLaunchKernelGGL((linattn_chunks<E, DA, DC, false, false>), dim3(states, used), dim3(256), 0, s, p, sp);
    hipLaunchKernelGGL((linattn_scan<DA, DC>), dim3(states * (DA * DC / 1024)), dim3(256), 0, s, p, sp, used);
  }
  if (p.gk > 1)
    hipLaunchKernelGGL((linattn_chunks<E, DA, DC, true, true>), dim3(states * p.gq, used), dim3(256), 0, s, p, sp);
  else
    hipLaunchKernelGGL((linattn_chunks<E, DA, DC, true, false>), dim3(states * p.gq, used), dim3(256), 0, s, p, sp);
}

template <typename E>
void launch_typed(o5_dtype dt, const LinPass& p, void* ws, hipStream_t s) {
  const bool a = p.da <= 64, c = p.dc <= 64;
  if (a && c)
    launch_chunks<E, 64, 64>(dt, p, ws, s);
  else if (a)
    launch_chunks<E, 64, 128>(dt, p, ws, s);
  else if (c)
    launch_chunks<E, 128, 64>(dt, p, ws, s);
  else
    launch_chunks<E, 128, 128>(dt, p, ws, s);
}

void launch_pass(o5_dtype dt, const LinPass& p, void* ws, hipStream_t s) {
  if (dt == O5_BF16)
    launch_typed<uint16_t>(dt, p, ws, s);
  else
    launch_typed<float>(dt, p, ws, s);
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
  return std::max<size_t>(256, pass_workspace(dt, T, B, nkv, nh / nkv, dk, dv));
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
  launch_pass(dt, p, ws, as_stream(stream));
  return check_launch(fn);
}

extern "C" size_t o5_linattn_bwd_workspace_bytes(o5_dtype dt, int T, int B, int nh, int nkv, int dk, int dv) {
  if (check_sizes("o5_linattn_bwd_workspace_bytes", dt, T, B, nh, nkv, dk, dv) != O5_OK) return 0;
  return std::max<size_t>({256, pass_workspace(dt, T, B, nkv, nh / nkv, dv, dk), pass_workspace(dt, T, B, nkv, 1, dk, dv)});
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
  for (const LinPass* p : {&pq, &pv, &pk}) launch_pass(dt, *p, ws, as_stream(stream));
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
