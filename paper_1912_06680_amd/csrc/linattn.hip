// Linear attention with a decay for each head, o5_linattn_*.
//
//   S_t = l (reset_t ? 0 : S_{t-1}) + k_t v_t^T,   o_t = scale S_t^T q_t
//
// Every pass is one recurrence of this kind.  With G_t = dJ/dS_t,
//   G_t = scale q_t do_t^T + l (1 - reset_{t+1}) G_{t+1},
// the gradients are dq_t = scale S_t do_t, dk_t = G_t v_t, dv_t = G_t^T k_t:
// the same recurrence with (query, key, value) = (do, v, k) forward in time
// on S^T, and (v, do, q) on G^T and (k, q, do) on G backward in time.  So one
// kernel, linattn_chunks, serves the forward pass and the three parts of the
// backward pass, which recompute S instead of having it kept: states of 128 x
// 128 for every 64 steps would be four times the size of q, k, v and o.
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
// A block of 4 or 8 waves takes one state and runs through its chunks; each wave
// owns 16 or 32 of the state's columns in its accumulators.  Products are
// formed transposed (o^T = S^T q^T + v^T p^T), so that the accumulators of S
// are, as they lie, operands of the next product.
//
// In bf16 the scores p and the state S are rounded to bf16 where a product
// reads them, as q, k and v are; the state itself stays in fp32 and what enters
// it, k_j times the fp32 l^(..) v_j, is formed from three bf16 terms of that
// factor (24 bits), so that a state after 10,000 steps is as exact as one summed
// in fp32 (1.2e-7 of its size at T = 256, 2.3e-7 at T = 10007; with two terms
// 2.4e-6, and T = 256, B = 128, 32 x 128 x 128 takes 5 % less).  fp32 runs on
// fp32 matrix instructions throughout, with chunks of 32 steps.  The rounded
// operands leave bf16 outputs 2.35e-3 off in the 2-norm, 1.65e-3 of it their own
// rounding; as two bf16 terms each they would leave 1.66e-3, at 8 to 18 % more time
// (that shape 377 -> 409 us; states of 64 x 128 spill and take twice as long).
//
// Bound: by bytes in the limit (q, k, v read once, o written once, S0 read and
// the last state written), and nearly as much by issue, per chunk and wave about
// 1,000 vector and 150 matrix instructions of 4 and 16 cycles.  With both from
// the L2 that shape takes 279 us, its memory traffic alone 343, together 377 to
// 440 on different cards (4.3 to 3.7 TB/s; a copy runs at 5.1).  The backward
// pass reads each row array where a pass needs it, 12 row arrays moved for the
// 7 of the call: T = 256, B = 64, 16 x 128 x 128 takes 230 to 250 us.  One
// sequence (T = 10007, 4 states of 64 x 128, 16 query heads, 32 splits) is bound
// by the latency of a chunk, five of them a block, and by work done over: 50 us,
// 37 of it the outputs, where each of a state's four query heads repeats its
// updates, and 11 the splits' states, 128 blocks on 256 compute units.
//
// The reduction index of every product runs in blocks of 32; of a block, lane
// group g = lane / 16 holds 4 g + r and 16 + 4 g + r (r = 0..3), which is how
// two 16 x 16 accumulators hold their rows.

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <typename E> struct Mx;

template <> struct Mx<uint16_t> {
  static constexpr int CL = 64;     // steps of a chunk
  static constexpr int TERMS = 3;   // bf16 terms of an fp32 operand: 24 bits
  // Rows in LDS: 8 rows of 32 bytes (a transposing read) then lie on 64 different banks, and with the 16-byte units
  // of every second 8 rows exchanged in pairs so do 16 rows of 16 bytes (a read of rows).
  static constexpr int PAD = 32;
  static __device__ __forceinline__ int swap(int row) { return (row & 8) * 2; }
  typedef u32x4 Frag;
  // c + a b; where `upper`, the block's first 16 are zero and need not be multiplied
  static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c, bool upper = false) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  // 4 g + r and 16 + 4 g + r of a row, `at` pointing to its block's element 4 g
  static __device__ __forceinline__ Frag rows(const char* at) {
    const u32x2 a = *reinterpret_cast<const u32x2*>(at), b = *reinterpret_cast<const u32x2*>(at + 32);
    return Frag{a[0], a[1], b[0], b[1]};
  }
  // rows 4 g + r and 16 + 4 g + r of column lane % 16 of a tile: within 16 lanes, lane j of a transposing read
  // takes 4 elements of row j / 4 from column 4 (j % 4) on and lane i receives the 4 rows of column i
  template <int STRIDE, bool SWAP>
  static __device__ __forceinline__ Frag columns(const char* block, int byte, int lane) {
    const int row = 4 * (lane >> 4) + ((lane & 15) >> 2);
    const char* p = block + row * STRIDE + ((byte + (lane & 3) * 8) ^ (SWAP ? swap(row) : 0));
    struct {
      s16x4 a, b;
    } f;
    f.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p));
    f.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 16 * STRIDE));
    return __builtin_bit_cast(Frag, f);
  }
  static __device__ __forceinline__ float get(const Frag& f, int i) {
    return __uint_as_float((i & 1) ? f[i / 2] & 0xffff0000u : f[i / 2] << 16);
  }
  // whether a value that is not finite went past: the largest magnitude's bits so far
  typedef uint16_t Odd __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ void look(const Frag& f, Odd& odd) {
#pragma unroll
    for (int i = 0; i < 4; ++i) odd = __builtin_elementwise_max(odd, __builtin_bit_cast(Odd, f[i] & 0x7fff7fffu));
  }
  static __device__ __forceinline__ bool found(Odd odd) { return odd[0] >= 0x7f80 || odd[1] >= 0x7f80; }
  static __device__ __forceinline__ Frag pack(const float (&x)[8]) {
    return Frag{f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]), f32x2_to_bf16x2(x[4], x[5]), f32x2_to_bf16x2(x[6], x[7])};
  }
  static __device__ __forceinline__ void store4(void* p, f32x4 v) {
    *static_cast<u32x2*>(p) = u32x2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
  }
};

template <> struct Mx<float> {
  static constexpr int CL = 32;
  static constexpr int TERMS = 1;
  static constexpr int PAD = 16;
  static __device__ __forceinline__ int swap(int) { return 0; }
  struct Frag {
    f32x4 h[2];
  };
  static __device__ __forceinline__ f32x4 mma(const Frag& a, const Frag& b, f32x4 c, bool upper = false) {
    if (!upper) {
#pragma unroll
      for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.h[0][r], b.h[0][r], c, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.h[1][r], b.h[1][r], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ Frag rows(const char* at) {
    return {{*reinterpret_cast<const f32x4*>(at), *reinterpret_cast<const f32x4*>(at + 64)}};
  }
  template <int STRIDE, bool SWAP>
  static __device__ __forceinline__ Frag columns(const char* block, int byte, int lane) {
    const char* p = block + 4 * (lane >> 4) * STRIDE + byte + (lane & 15) * 4;
    Frag f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) f.h[h][r] = *reinterpret_cast<const float*>(p + (16 * h + r) * STRIDE);
    return f;
  }
  static __device__ __forceinline__ float get(const Frag& f, int i) { return f.h[i >> 2][i & 3]; }
  typedef float Odd;
  static __device__ __forceinline__ void look(const Frag& f, Odd& odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) odd = fmaf(get(f, i), 0.0f, odd);
  }
  static __device__ __forceinline__ bool found(Odd odd) { return !(odd == 0.0f); }
  static __device__ __forceinline__ Frag pack(const float (&x)[8]) {
    return {{f32x4{x[0], x[1], x[2], x[3]}, f32x4{x[4], x[5], x[6], x[7]}}};
  }
  static __device__ __forceinline__ void store4(void* p, f32x4 v) { *static_cast<f32x4*>(p) = v; }
};

// log2 of a decay, finite for 0 too, so that l^0 is 1 and l^n 0 without a branch; and l^n for n >= 0 (for other n any
// number).
__device__ __forceinline__ float log2_decay(float l) { return fmaxf(log2f(l), -0x1p100f); }
__device__ __forceinline__ float power(float l2, int n) { return __builtin_amdgcn_exp2f(l2 * static_cast<float>(n)); }
__device__ __forceinline__ float uniform(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

template <typename E, int DA, int DC>
struct Tiles {
  static constexpr int CL = Mx<E>::CL, ES = sizeof(E), PAD = Mx<E>::PAD;
  static constexpr int QS = DA * ES + PAD, VS = DC * ES + PAD, PS = CL * ES + 16;  // row strides
  alignas(16) char q[CL * QS];
  alignas(16) char k[CL * QS];
  alignas(16) char v[CL * VS];
  alignas(16) char p[CL * PS];
};

// One operand's rows of a chunk on the way from memory to LDS, BT threads.
template <typename E, int D, int BT>
struct Stage {
  static constexpr int CL = Mx<E>::CL, U = D * static_cast<int>(sizeof(E)) / 16, N = CL * U / BT, PER = 16 / sizeof(E);
  static_assert(N >= 1 && CL * U % BT == 0, "every thread takes whole units");
  u32x4 x[N];
  // `base`: row 0 of the chunk; `step`: elements between rows; rows before `pad` and columns from d on are zero
  template <bool kFull>
  __device__ __forceinline__ void load(const E* base, ptrdiff_t step, int pad, int d) {
    int row = threadIdx.x / U;
    const int c = threadIdx.x % U * PER;
    asm volatile("" : "+v"(row));  // the address is worked out anew for each chunk: kept, it would cost two registers
    const E* at = base + row * step + c;
    if (kFull) {
#pragma unroll
      for (int n = 0; n < N; ++n) x[n] = *reinterpret_cast<const u32x4*>(at + n * (BT / U) * step);
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        x[n] = u32x4{0, 0, 0, 0};
        if (c < d && row + n * (BT / U) >= pad) x[n] = *reinterpret_cast<const u32x4*>(at + n * (BT / U) * step);
      }
    }
  }
  template <int STRIDE, bool SWAP>
  __device__ __forceinline__ void store(char* lds) const {
    const int row = threadIdx.x / U, byte = threadIdx.x % U * 16;
    static_assert(BT / U % 16 == 0 || !SWAP || Mx<E>::TERMS == 1 || N == 1, "a thread's rows exchange alike");
    char* at = lds + row * STRIDE + (byte ^ (SWAP ? Mx<E>::swap(row) : 0));
#pragma unroll
    for (int n = 0; n < N; ++n) *reinterpret_cast<u32x4*>(at + n * (BT / U) * STRIDE) = x[n];
  }
};

// Adds p_ij v_jc for the j of row i's episode whose v is not finite, columns c .. c + 3.
template <typename E, typename TL>
__device__ __forceinline__ f32x4 odd_terms(const TL& lds, int i, int ri, int c) {
  f32x4 o = {0, 0, 0, 0};
#pragma unroll 1
  for (int j = max(ri, 0); j <= i; ++j) {
    const float pj = elem<E>::to_f32(*reinterpret_cast<const E*>(lds.p + i * TL::PS + j * sizeof(E)));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float x = elem<E>::to_f32(*reinterpret_cast<const E*>(lds.v + j * TL::VS + (c + r) * sizeof(E)));
      if (!finite(x)) o[r] = fmaf(pj, x, o[r]);
    }
  }
  return o;
}

// Where the chunks of a split begin and what it starts from.
struct Split {
  int chunks;       // of one split
  float* states;    // [splits][B * nkv][DA * DC] in the accumulators' order, or NULL: one split
  float* keep;      // [splits][B * nkv]: the factor on the state across the split, -1 where a reset cuts it off
};

// The passes of one launch: alike in T, B, nkv and gq, and in the kernel that runs them.
struct Passes {
  int count;
  unsigned first;  // the call's block that is block 0 of this launch, a multiple of count
  LinPass pass[3];
  Split split[3];
};

// Column tiles of a wave: two where the state's accumulators would else need 8 waves of more registers than they can
// have (128 x 128 with one tile spills: 543 us against 423 at T = 256, B = 128, 32 heads).  With two, the bf16 kernels of
// 128 x 128 hold all 256 registers and spill a few more: 1 (kAlone), 3 (kGroupQueries) and 15 (kManyKeys) with whole
// chunks, 2 in kManyKeys without.
constexpr int tile_columns(int da, int dc, bool many) { return (da == 128 || many) && dc == 128 ? 2 : 1; }
constexpr int block_threads(int da, int dc, bool many) { return dc / 16 / tile_columns(da, dc, many) * 64; }
constexpr int waves_per_simd(int da, int dc, bool many) {
  return block_threads(da, dc, many) == 512 ? 4 : da + dc == 128 ? 3 : 2;
}

// kOut: write the outputs; else only add up each split's own part of the state.
// kLoop: what a block takes in turn within a chunk: kAlone, one query head and
// one key/value head; kManyKeys, the gk key/value heads of a state, whose outputs
// are summed; kGroupQueries, the gq query heads of a state, which then stages the keys
// and values and updates the state once for all of them.
enum Loop { kAlone, kManyKeys, kGroupQueries };
// Where T is no multiple of CL the first chunk is short: it starts `pad` steps
// before step 0, and those rows are zero and not written.
// kFull: T is a multiple of CL and the state fills its tiles, so that every
// access is unconditional and the waits for the next chunk's rows need not
// wait for this chunk's outputs too (a kernel of its own: with both kinds of
// chunk in one, registers spilled and T = 256, B = 128, 32 x 128 x 128 took 441
// us instead of 423).
template <typename E, int DA, int DC, bool kOut, Loop kLoop, bool kFull>
__global__ void __launch_bounds__(block_threads(DA, DC, kLoop == kManyKeys), waves_per_simd(DA, DC, kLoop == kManyKeys))
    linattn_chunks(Passes ps) {
  constexpr bool kMany = kLoop == kManyKeys, kGroup = kLoop == kGroupQueries;
  typedef Mx<E> M;
  typedef typename M::Frag Frag;
  typedef Tiles<E, DA, DC> TL;
  constexpr int NC = tile_columns(DA, DC, kMany), WAVES = DC / 16 / NC, BT = WAVES * 64;
  constexpr int CL = M::CL, ES = sizeof(E), NI = CL / 16, NB = CL / 32, NA = DA / 16, NU = DA / 32;
  __shared__ TL lds;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (the passes of a call read the same rows: side by side, so that they find them in the caches)
  const LinPass& p = ps.pass[blockIdx.x % ps.count];
  const Split& sp = ps.split[blockIdx.x % ps.count];
  const int block = (ps.first + blockIdx.x) / ps.count;
  const int heads = kOut && !kGroup ? p.nkv * p.gq : p.nkv;
  const int b = block / heads, n = kOut && !kGroup ? block % heads / p.gq : block % heads;
  const int hq = kGroup ? n * p.gq : block % heads;  // the block's (first) query head
  const int chunks = (p.T + CL - 1) / CL;
  const int c0 = blockIdx.y * sp.chunks, c1 = min(chunks, c0 + sp.chunks);
  const int e = p.rev ? 0 : 1;
  const int bn = b * p.nkv + n;
  const size_t sbase = static_cast<size_t>(bn) * p.da * p.dc;
  const int col0 = wave * 16 * NC;  // the wave's first column

  // the state before the first chunk
  f32x4 S[NA][NC];
  if (kOut && sp.states) {
    const f32x4* st = reinterpret_cast<const f32x4*>(sp.states) +
                      (static_cast<size_t>(blockIdx.y) * p.B * p.nkv + bn) * (DA * DC / 4) + wave * NA * NC * 64;
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int c = 0; c < NC; ++c) S[a][c] = st[(c * NA + a) * 64 + lane];
  } else {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int a = 0; a < NA; ++a) S[a][c] = f32x4{0, 0, 0, 0};
      const int col = col0 + c * 16 + l16;
      if (!kOut || !p.s0 || col >= p.dc) continue;
      const float* s0 = p.s0 + sbase + (p.s0t ? col * p.da + g4 * 4 : g4 * 4 * p.dc + col);
      if (p.s0t) {
#pragma unroll
        for (int a = 0; a < NA; ++a)
          if (a * 16 + g4 * 4 < p.da) S[a][c] = *reinterpret_cast<const f32x4*>(s0 + a * 16);
      } else {
#pragma unroll
        for (int a = 0; a < NA; ++a)
          if (a * 16 + g4 * 4 < p.da) {
#pragma unroll
            for (int r = 0; r < 4; ++r) S[a][c][r] = s0[(a * 16 + r) * p.dc];
          }
      }
    }
  }

  // powers of the decay
  const float l2 = uniform(log2_decay(p.decay[n]));
  const float l16th = uniform(power(l2, 16)), l32 = uniform(power(l2, 32)), l48 = l16th * l32;
  float in[4];  // the factor on what enters the state from a chunk's last 16 steps
#pragma unroll
  for (int r = 0; r < 4; ++r) in[r] = p.kscale * power(l2, 16 - e - (g4 * 4 + r));
  const float pscale = p.oscale * p.kscale;

  const int pad0 = kFull ? 0 : chunks * CL - p.T;
  const ptrdiff_t dir = p.rev ? -p.B : p.B;
  const ptrdiff_t qstep = dir * static_cast<ptrdiff_t>(p.ldq), kstep = dir * static_cast<ptrdiff_t>(p.ldk);
  const ptrdiff_t vstep = dir * static_cast<ptrdiff_t>(p.ldv), ostep = dir * static_cast<ptrdiff_t>(p.ldo);
  const ptrdiff_t row0 = static_cast<ptrdiff_t>(p.rev ? p.T - 1 : 0) * p.B + b;  // of the pass's step 0
  typedef Stage<E, DA, BT> StQ;
  typedef Stage<E, DC, BT> StV;
  // row 0 of chunk c0 (before the buffer where that chunk starts with padding, which is not read)
  const ptrdiff_t u00 = static_cast<ptrdiff_t>(c0) * CL - pad0;
  const E* qb = static_cast<const E*>(p.q) + row0 * static_cast<ptrdiff_t>(p.ldq) + u00 * qstep + hq * p.da;
  const E* kb = static_cast<const E*>(p.k) + row0 * static_cast<ptrdiff_t>(p.ldk) + u00 * kstep + n * p.gk * p.da;
  const E* vb = static_cast<const E*>(p.v) + row0 * static_cast<ptrdiff_t>(p.ldv) + u00 * vstep + n * p.gk * p.dc;
  E* ob = static_cast<E*>(p.o) + row0 * static_cast<ptrdiff_t>(p.ldo) + u00 * ostep + hq * p.dc;
  StQ sq, sk;
  StV sv;
  bool cut_any = false;  // a reset in this split so far
  f32x4 o[NI][NC];  // the chunk's outputs, transposed

  uint32_t flag = 0;  // of step `lane` of the chunk that is on its way: not 0 for a reset before it
  const int r0 = p.rev ? 1 : 0;  // the first step that a reset can precede
  auto fetch = [&](int ch, int g) {
    const int pad = !kFull && ch == 0 ? pad0 : 0;
    const ptrdiff_t u = static_cast<ptrdiff_t>(ch - c0) * CL;
    if (kOut && (!kMany || g == 0)) sq.template load<kFull>(qb + u * qstep + (kGroup ? g * p.da : 0), qstep, pad, p.da);
    if (!kGroup || g == 0) {
      sk.template load<kFull>(kb + u * kstep + (kMany ? g * p.da : 0), kstep, pad, p.da);
      sv.template load<kFull>(vb + u * vstep + (kMany ? g * p.dc : 0), vstep, pad, p.dc);
    }
    if (p.reset && g == 0) {  // (looked at a chunk later: a branch on it here would wait for every load)
      const int t = max(ch * CL - pad0 + min(lane, CL - 1), min(r0, p.T - 1));
      flag = p.reset[static_cast<size_t>(p.rev && t > 0 ? p.T - t : t) * p.B + b];
    }
  };

  int ch = c0, g = 0;
  fetch(ch, g);
  while (ch < c1) {
    const int pad = !kFull && ch == 0 ? pad0 : 0;
    const bool first = !kMany || g == 0, last = !kMany || g == p.gk - 1;  // of the outputs' sums
    if (kOut && first) sq.template store<TL::QS, true>(lds.q);
    if (!kGroup || g == 0) {
      sk.template store<TL::QS, true>(lds.k);
      sv.template store<TL::VS, false>(lds.v);
    }
    uint64_t resets = 0;  // bit i: a reset before the chunk's step i
    if (p.reset) resets = __ballot(flag != 0 && lane < CL && ch * CL - pad0 + lane >= r0);
    const int rl = resets ? 63 - __builtin_clzll(resets) : -1;  // the last reset
    int lr = -1;  // the last reset at or before step `lane`
    if (resets) {
      int x = 63 - lane;
      asm volatile("" : "+v"(x));  // (else the mask is kept in registers from chunk to chunk)
      const uint64_t m = resets & (~0ull >> x);
      lr = m ? 63 - __builtin_clzll(m) : -1;
    }
    auto last_reset = [&](int ti) { return resets ? __shfl(lr, ti * 16 + l16) : -1; };  // of step 16 ti + l16
    __syncthreads();
    int nch = ch, ng = g + 1;
    if (ng == (kMany ? p.gk : kGroup ? p.gq : 1)) ++nch, ng = 0;
    if (nch < c1) fetch(nch, ng);

    if (kOut) {  // p, 16 x 16 tiles at and below the diagonal, one after another to the waves
      constexpr int kTiles = NI * (NI + 1) / 2;
      for (int x = wave; x < kTiles + NI / 2; x += WAVES) {
        int ti, tj;
        if (x < kTiles) {
          ti = x >= 6 ? 3 : x >= 3 ? 2 : x >= 1 ? 1 : 0;
          tj = x - ti * (ti + 1) / 2;
        } else {  // the other half of an even row tile's last block of 32
          ti = (x - kTiles) * 2;
          tj = ti + 1;
        }
        f32x4 s = {0, 0, 0, 0};
        const int i = ti * 16 + l16;
        if (tj <= ti) {
          const char* kr = lds.k + (tj * 16 + l16) * TL::QS + ((g4 * 4 * ES) ^ M::swap(l16));
          const char* qr = lds.q + i * TL::QS + ((g4 * 4 * ES) ^ M::swap(l16));
#pragma unroll
          for (int u = 0; u < NU; ++u) s = M::mma(M::rows(kr + u * 32 * ES), M::rows(qr + u * 32 * ES), s);
          const int d0 = i - tj * 16 - g4 * 4;
          const float dl = l2 * static_cast<float>(d0);
#pragma unroll
          for (int r = 0; r < 4; ++r) s[r] *= pscale * __builtin_amdgcn_exp2f(fmaf(l2, static_cast<float>(-r), dl));
          if (ti == tj) {  // (selects: outside the mask the product may be anything)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[r] = d0 >= r ? s[r] : 0.0f;
          }
          if (resets) {
            const int ri = last_reset(ti) - tj * 16 - g4 * 4;
#pragma unroll
            for (int r = 0; r < 4; ++r) s[r] = r >= ri ? s[r] : 0.0f;
          }
        }
        M::store4(lds.p + i * TL::PS + (tj * 16 + g4 * 4) * ES, s);
      }
      __syncthreads();
    }

    auto upper = [&](int u) { return !kFull && u * 32 + 16 <= pad; };
    // the wave's columns of v
    Frag vf[NC][NB];
    typename M::Odd odd = {};
    auto read_v = [&](int c, int u) {
      return M::template columns<TL::VS, false>(lds.v + u * 32 * TL::VS, (col0 + c * 16) * ES, lane);
    };
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        vf[c][u] = read_v(c, u);
        M::look(vf[c][u], odd);
      }
    const bool any_odd = __any(M::found(odd));  // an infinity or NaN in them

    if (kOut) {
      if (any_odd) {  // it may not meet the zeros of p: it is taken out of the product and added term by term
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int u = 0; u < NB; ++u) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = finite(M::get(vf[c][u], i)) ? M::get(vf[c][u], i) : 0.0f;
            vf[c][u] = M::pack(x);
          }
      }
      const char* qr = lds.q + l16 * TL::QS + ((g4 * 4 * ES) ^ M::swap(l16));
      const char* pr = lds.p + l16 * TL::PS + g4 * 4 * ES;
      auto skip = [&](int ti) { return !kFull && ti * 16 + 16 <= pad; };
      if (first) {
#pragma unroll
        for (int ti = 0; ti < NI; ++ti)
#pragma unroll
          for (int c = 0; c < NC; ++c) o[ti][c] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          __builtin_amdgcn_sched_barrier(0);
          Frag sf[NC];
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const f32x4 x = S[2 * u][c], y = S[2 * u + 1][c];
            const float z[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
            sf[c] = M::pack(z);
          }
#pragma unroll
          for (int ti = 0; ti < NI; ++ti) {
            if (skip(ti)) continue;
            const Frag fq = M::rows(qr + ti * 16 * TL::QS + u * 32 * ES);
#pragma unroll
            for (int c = 0; c < NC; ++c) o[ti][c] = M::mma(sf[c], fq, o[ti][c]);
          }
        }
#pragma unroll
        for (int ti = 0; ti < NI; ++ti) {
          const float f = p.oscale * power(l2, ti * 16 + l16 - pad + e);
#pragma unroll
          for (int c = 0; c < NC; ++c) o[ti][c] *= f;
          if (resets) {
            const bool carried = last_reset(ti) < 0;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
              for (int r = 0; r < 4; ++r) o[ti][c][r] = carried ? o[ti][c][r] : 0.0f;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ti = 2 * u; ti < NI; ++ti) {
          if (skip(ti)) continue;
          const Frag fp = M::rows(pr + ti * 16 * TL::PS + u * 32 * ES);
#pragma unroll
          for (int c = 0; c < NC; ++c) o[ti][c] = M::mma(vf[c][u], fp, o[ti][c], upper(u));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (kMany && any_odd) {
#pragma unroll
        for (int ti = 0; ti < NI; ++ti)
#pragma unroll
          for (int c = 0; c < NC; ++c)
            o[ti][c] += odd_terms<E>(lds, ti * 16 + l16, last_reset(ti), col0 + c * 16 + g4 * 4);
      }
      int lrow = l16;
      asm volatile("" : "+v"(lrow));
      E* orow = ob + static_cast<ptrdiff_t>(ch - c0) * CL * ostep + lrow * ostep + (kGroup ? g * p.dc : 0) + col0 + g4 * 4;
      if (last) {
#pragma unroll
        for (int ti = 0; ti < NI; ++ti) {
          if (!kFull && ti * 16 + l16 < pad) continue;
#pragma unroll
          for (int c = 0; c < NC; ++c)
            if (kFull || col0 + c * 16 + g4 * 4 < p.dc) M::store4(orow + ti * 16 * ostep + c * 16, o[ti][c]);
        }
      }
      if (any_odd) {
#pragma unroll 1
        for (int x = kMany ? NI * NC : 0; x < NI * NC; ++x) {  // onto what this lane has just written
          const int ti = x / NC, c = x % NC, i = ti * 16 + l16, ri = last_reset(ti);
          if (i < pad || col0 + c * 16 + g4 * 4 >= p.dc) continue;
          E* at = orow + ti * 16 * ostep + c * 16;
          f32x4 o;
#pragma unroll
          for (int r = 0; r < 4; ++r) o[r] = elem<E>::to_f32(at[r]);
          M::store4(at, o + odd_terms<E>(lds, i, ri, col0 + c * 16 + g4 * 4));
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int u = 0; u < NB; ++u) vf[c][u] = read_v(c, u);
      }
    }

    // Where no one takes the state after the last chunk, that chunk has no update (backward, 2 samples of T = 2048 in
    // splits, 16 query heads on 4 states of 128 x 128: 116 -> 103 us; fp32, T = 16, B = 256, 16 on 8 of 64 x 64: 77 -> 75).
    // Not in the kernel of most registers, which the branch costs more where the state is taken (full_kernel).
    const bool update = (kFull && DA + DC == 256) || ch + 1 < c1 || !kOut || (p.sT && !sp.states && hq == n * p.gq);
    if ((!kGroup || g == p.gq - 1) && update) {
      if (rl > 0) {  // a key that is cut off may hold anything, and may not meet the zeros of what enters
        for (int x = tid; x < rl * (TL::QS / 16); x += BT) *reinterpret_cast<u32x4*>(lds.k + x * 16) = u32x4{0, 0, 0, 0};
        __syncthreads();
      }

      // the state after the chunk
      if (first) {
        if (resets) {
          cut_any = true;
#pragma unroll
          for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int c = 0; c < NC; ++c) S[a][c] = f32x4{0, 0, 0, 0};
        } else {
          const float f = uniform(power(l2, CL - pad));
#pragma unroll
          for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int c = 0; c < NC; ++c) S[a][c] *= f;
        }
      }
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        if (!kFull && u * 32 + 32 <= pad) continue;
        __builtin_amdgcn_sched_barrier(0);
        // what enters, in bf16 as a sum of terms
        Frag term[NC][M::TERMS];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int tiles = NI - 1 - (2 * u + (i >> 2));
            x[i] = (M::get(vf[c][u], i) * in[i & 3]) * (tiles == 0 ? 1.0f : tiles == 1 ? l16th : tiles == 2 ? l32 : l48);
          }
          if (rl > u * 32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = u * 32 + (i >> 2) * 16 + g4 * 4 + (i & 3) >= rl ? x[i] : 0.0f;
          }
          term[c][0] = M::pack(x);
#pragma unroll
          for (int t = 1; t < M::TERMS; ++t) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] -= M::get(term[c][t - 1], i);
            term[c][t] = M::pack(x);
          }
        }
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          const Frag kf = M::template columns<TL::QS, true>(lds.k + u * 32 * TL::QS, a * 16 * ES, lane);
#pragma unroll
          for (int t = M::TERMS - 1; t >= 0; --t)
#pragma unroll
            for (int c = 0; c < NC; ++c) S[a][c] = M::mma(kf, term[c][t], S[a][c], upper(u));
        }
      }
    }
    __syncthreads();
    ch = nch;
    g = ng;
  }

  if (kOut && sp.states) return;  // the scan has written the last state
  if (!kOut) {
    f32x4* st = reinterpret_cast<f32x4*>(sp.states) +
                (static_cast<size_t>(blockIdx.y) * p.B * p.nkv + bn) * (DA * DC / 4) + wave * NA * NC * 64;
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int c = 0; c < NC; ++c) st[(c * NA + a) * 64 + lane] = S[a][c];
    if (tid == 0)
      sp.keep[static_cast<size_t>(blockIdx.y) * p.B * p.nkv + bn] =
          cut_any ? -1.0f : power(l2, (c1 - c0) * CL - (c0 == 0 ? pad0 : 0));
    return;
  }
  if (!p.sT || hq != n * p.gq) return;
  const bool cut = p.rev && p.reset && p.reset[b] != 0;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int col = col0 + c * 16 + l16;
    if (col >= p.dc) continue;
    float* sT = p.sT + sbase + (p.s0t ? col * p.da + g4 * 4 : g4 * 4 * p.dc + col);
#pragma unroll
    for (int a = 0; a < NA; ++a) {
      if (a * 16 + g4 * 4 >= p.da) continue;
      const f32x4 x = cut ? f32x4{0, 0, 0, 0} : S[a][c];
      if (p.s0t) {
        *reinterpret_cast<f32x4*>(sT + a * 16) = x;
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) sT[(a * 16 + r) * p.dc] = x[r];
      }
    }
  }
}

// The state before each split, in place of the split's own part, and the last
// state: X_0 = S0, X_{s+1} = keep_s X_s + part_s.  A thread takes 4 rows of a
// column (one accumulator).  Bound by its loads' latency: 32 splits of 4 states
// of 64 x 128 5.6 us.
template <int DA, int DC>
__global__ void __launch_bounds__(256) linattn_scan(Passes ps, int splits) {
  constexpr int NA = DA / 16, Q = DA * DC / 4;
  const LinPass& p = ps.pass[blockIdx.y];
  const Split& sp = ps.split[blockIdx.y];
  const size_t idx = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  const int states = p.B * p.nkv;
  const int bn = static_cast<int>(idx / Q), x = static_cast<int>(idx % Q);
  const int lane = x & 63, tile = x >> 6;
  const int row = tile % NA * 16 + (lane >> 4) * 4, col = tile / NA * 16 + (lane & 15);
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
  // (8 splits' loads in flight together: 32 splits of 4 states took 11 us one after another)
  for (int s0 = 0; s0 < splits; s0 += 8) {
    f32x4 part[8];
    float keep[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int s = min(s0 + i, splits - 1);
      part[i] = st[s * stride];
      keep[i] = sp.keep[static_cast<size_t>(s) * states + bn];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (s0 + i >= splits) break;
      st[(s0 + i) * stride] = X;
#pragma unroll
      for (int r = 0; r < 4; ++r) X[r] = keep[i] < 0.0f ? part[i][r] : fmaf(keep[i], X[r], part[i][r]);
    }
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
// run.  Split, a block goes through its chunks twice (the states, then the
// outputs) and two more launches take about four chunks' time, so a sequence
// of few chunks stays whole.  Chunks are what is counted: where a block takes gk
// heads in each (dk and dv of shared states) it is gk times as long, and a short
// sequence of few states stays whole all the same (backward, T = 256, B = 8, 4
// states of 64 x 64 with 4 heads each: 66 us, its bytes 3.6).
int plan_splits(o5_dtype dt, int T, int B, int nkv, int gq) {
  const int cl = dt == O5_BF16 ? Mx<uint16_t>::CL : Mx<float>::CL;
  const int chunks = (T + cl - 1) / cl;
  const long long blocks = static_cast<long long>(B) * nkv * gq;
  if (blocks >= 256) return 1;
  const int want = std::min<int>(chunks, static_cast<int>((512 + blocks - 1) / blocks));
  const int per = (chunks + want - 1) / want;
  return chunks >= 2 * per + 4 ? (chunks + per - 1) / per : 1;
}

// Workspace of any of a call's launches: `count` passes at most, each with as many splits as if it ran alone.
size_t pass_workspace(o5_dtype dt, int T, int B, int nkv, int gq, int da, int dc, int count) {
  const int splits = plan_splits(dt, T, B, nkv, gq);
  if (splits == 1) return 0;
  const size_t floats = static_cast<size_t>(splits) * B * nkv * (pad_head(da) * pad_head(dc) + 1);
  return align_up(floats, 64) * sizeof(float) * count;
}

size_t pass_floats(const LinPass& p, int splits) {
  return static_cast<size_t>(splits) * p.B * p.nkv * (pad_head(p.da) * pad_head(p.dc) + 1);
}

// Whether a launch takes the kernel of whole chunks.  That of 128 x 128 updates
// the state after every chunk, the last one too; where no pass takes that state
// and it is one of at most 4 updates, the other kernel, which leaves it out, is
// faster.  us, whole chunks -> the other, 16 heads of one or of four to a state:
// backward, one chunk, bf16 143 -> 136 and 179 -> 152, fp32 176 -> 150 and 224 ->
// 170; four chunks, bf16 106.8 -> 107.2 and 178 -> 170, fp32 151 -> 146 and 238 ->
// 226; eight, bf16 107 -> 113 and 222 -> 219, fp32 151 and 252 both.  Where the
// state is taken the kernel of whole chunks stays (forward, one to eight chunks,
// bf16 0 to 9 % and fp32 0 to 5 % faster).  A sequence in splits has no one to take its
// last update, whatever its length.
template <typename E, int DA, int DC>
bool full_kernel(const Passes& ps, int chunks, int splits) {
  if (ps.pass[0].T % Mx<E>::CL != 0) return false;
  bool taken = false;
  for (int i = 0; i < ps.count; ++i) {
    if (ps.pass[i].da != DA || ps.pass[i].dc != DC) return false;
    taken = taken || ps.pass[i].sT != nullptr;
  }
  return DA + DC < 256 || (splits == 1 && (taken || chunks > 4));
}

template <typename E, int DA, int DC, Loop kLoop>
void launch_chunks(Passes& ps, float* ws, int splits, hipStream_t s) {
  constexpr bool kMany = kLoop == kManyKeys;
  constexpr int threads = block_threads(DA, DC, kMany);
  const LinPass& p = ps.pass[0];
  const int chunks = (p.T + Mx<E>::CL - 1) / Mx<E>::CL;
  const unsigned states = static_cast<unsigned>(p.B) * p.nkv;
  const int per = (chunks + splits - 1) / splits, used = (chunks + per - 1) / per;
  for (int i = 0; i < ps.count; ++i) {
    ps.split[i] = {per, nullptr, nullptr};
    if (splits > 1) {
      ps.split[i].states = ws;
      ps.split[i].keep = ws + static_cast<size_t>(used) * states * DA * DC;
      ws += align_up(pass_floats(ps.pass[i], splits), 64);
    }
  }
  if (splits > 1) {
    constexpr Loop kParts = kMany ? kManyKeys : kAlone;
    hipLaunchKernelGGL((linattn_chunks<E, DA, DC, false, kParts, false>), dim3(states * ps.count, used), dim3(threads), 0, s, ps);
    hipLaunchKernelGGL((linattn_scan<DA, DC>), dim3(states * (DA * DC / 1024), ps.count), dim3(256), 0, s, ps, used);
  }
  auto kernel = full_kernel<E, DA, DC>(ps, chunks, splits) ? linattn_chunks<E, DA, DC, true, kLoop, true> : linattn_chunks<E, DA, DC, true, kLoop, false>;
  // A launch holds fewer than 2^32 threads in a dimension (with more the grid wraps and the rest is never run, without an
  // error), so that more blocks go out in several.  (Split sequences have fewer than 256 states and heads.)
  const unsigned blocks = states * (kLoop == kGroupQueries ? 1 : p.gq) * ps.count;
  const unsigned most = 0xffffffffu / threads / ps.count * ps.count;
  for (ps.first = 0; ps.first < blocks; ps.first += most)
    hipLaunchKernelGGL(kernel, dim3(std::min(blocks - ps.first, most), used), dim3(threads), 0, s, ps);
}

template <typename E, int DA, int DC>
void launch_loop(Passes& ps, float* ws, int splits, bool group, hipStream_t s) {
  if (ps.pass[0].gk > 1)
    launch_chunks<E, DA, DC, kManyKeys>(ps, ws, splits, s);
  else if (group)
    launch_chunks<E, DA, DC, kGroupQueries>(ps, ws, splits, s);
  else
    launch_chunks<E, DA, DC, kAlone>(ps, ws, splits, s);
}

template <typename E>
void launch_typed(Passes& ps, float* ws, int splits, bool group, hipStream_t s) {
  const bool a = ps.pass[0].da <= 64, c = ps.pass[0].dc <= 64;
  if (a && c)
    launch_loop<E, 64, 64>(ps, ws, splits, group, s);
  else if (a)
    launch_loop<E, 64, 128>(ps, ws, splits, group, s);
  else if (c)
    launch_loop<E, 128, 64>(ps, ws, splits, group, s);
  else
    launch_loop<E, 128, 128>(ps, ws, splits, group, s);
}

// Whether one kernel runs both passes.
bool alike(const LinPass& x, const LinPass& y) {
  return pad_head(x.da) == pad_head(y.da) && pad_head(x.dc) == pad_head(y.dc) && x.gq == y.gq && x.gk == y.gk;
}

// Whether a block takes a state's query heads in turn: where the states alone
// give each compute unit 2 blocks.  Forward, 256 steps of bf16, us by block a
// head -> block a state: 512 states of 64 x 64, 2 heads each 39.9 -> 35.0; 1024 of
// 128 x 128, 4 heads 297 -> 209; fp32, 100 steps, 386 -> 257.  With 256 states the
// chip is half empty: 64 x 64, 2 heads 24.2 -> 28.4, 4 heads 38.3 -> 43.9; and 4
// states over T = 10007, split further in the heads' place, take 62 for 54.
bool group_queries(const LinPass& p, int count) {
  return p.gq > 1 && static_cast<long long>(p.B) * p.nkv * count >= 512;
}

// Passes of one call in as few launches as they allow.
void launch_passes(o5_dtype dt, const LinPass* p, int count, void* ws, hipStream_t s) {
  bool done[3] = {};
  for (int i = 0; i < count; ++i) {
    if (done[i]) continue;
    Passes ps = {};
    for (int j = i; j < count; ++j)
      if (!done[j] && alike(p[i], p[j])) {
        ps.pass[ps.count++] = p[j];
        done[j] = true;
      }
    const int splits = plan_splits(dt, p[i].T, p[i].B, p[i].nkv, p[i].gq * ps.count);
    const bool group = group_queries(p[i], ps.count);  // (so many states are not split)
    if (dt == O5_BF16)
      launch_typed<uint16_t>(ps, static_cast<float*>(ws), splits, group, s);
    else
      launch_typed<float>(ps, static_cast<float*>(ws), splits, group, s);
  }
}

// ----------------------------------------------------------- single token

// One token of one state, a block's: its rows are CP groups of 4 columns, 256 /
// CP rows at a time, and stay in registers between the update and the group's
// query heads.  Bound by the states, read and written once: 4096 x 8 states of
// 128 x 128 take 861 us, 5.0 TB/s, the rate of a copy (953 us when a block took
// 32 of the columns, an eighth of a page; 64 wide: 201 and 222 us).
template <typename E, int CP, int DK>
__global__ void __launch_bounds__(256) linattn_token(int nkv, int G, int dk, int dv, const void* __restrict__ q, size_t ldq,
                                                     const void* __restrict__ k, size_t ldk,
                                                     const void* __restrict__ v, size_t ldv,
                                                     const float* __restrict__ decay, float scale,
                                                     const uint8_t* __restrict__ reset, float* __restrict__ S,
                                                     void* __restrict__ o, size_t ldo) {
  constexpr int RP = 256 / CP;       // rows in flight
  constexpr int NR = (DK + RP - 1) / RP;  // rows of a thread
  __shared__ float ks[DK], qs[DK];
  __shared__ float4 part[4][CP];
  const int b = blockIdx.x / nkv, n = blockIdx.x % nkv;
  const int tid = threadIdx.x, cg = tid % CP, r0 = tid / CP;
  const int c = cg * 4;
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

// The narrowest groups that hold a row.
template <typename E, int CP>
auto token_kernel_rows(int dk) {
  return dk <= 32 ? linattn_token<E, CP, 32> : dk <= 64 ? linattn_token<E, CP, 64> : linattn_token<E, CP, 128>;
}
template <typename E>
auto token_kernel(int dk, int dv) {
  return dv <= 32 ? token_kernel_rows<E, 8>(dk) : dv <= 64 ? token_kernel_rows<E, 16>(dk) : token_kernel_rows<E, 32>(dk);
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
  O5_CHECK(static_cast<long long>(T) * B < (1ll << 30) && static_cast<long long>(nh) * kMaxHead < (1ll << 31) &&
               static_cast<long long>(B) * nh < (1ll << 24),
           O5_E_SHAPE, "%s: T*B must be below 2^30 and B*nh below 2^24", fn);
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
  return std::max<size_t>(256, pass_workspace(dt, T, B, nkv, nh / nkv, dk, dv, 1));
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
  launch_passes(dt, &p, 1, ws, as_stream(stream));
  return check_launch(fn);
}

extern "C" size_t o5_linattn_bwd_workspace_bytes(o5_dtype dt, int T, int B, int nh, int nkv, int dk, int dv) {
  if (check_sizes("o5_linattn_bwd_workspace_bytes", dt, T, B, nh, nkv, dk, dv) != O5_OK) return 0;
  return std::max<size_t>(256, pass_workspace(dt, T, B, nkv, 1, dk, dv, 3));
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
  const LinPass p[3] = {
      {dout, v, k, dq, lddo, ldv, ldk, lddq, decay, reset, S0, nullptr, T, B, nkv, G, 1, dv, dk, scale, 1.0f, true, false},
      {k, q, dout, dval, ldk, ldq, lddo, lddv, decay, reset, dST, dS0, T, B, nkv, 1, G, dk, dv, 1.0f, scale, false, true},
      {v, dout, q, dkey, ldv, lddo, ldq, lddk, decay, reset, dST, nullptr, T, B, nkv, 1, G, dv, dk, 1.0f, scale, true, true}};
  launch_passes(dt, p, 3, ws, as_stream(stream));
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
  auto kernel = dt == O5_BF16 ? token_kernel<uint16_t>(dk, dv) : token_kernel<float>(dk, dv);
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(B) * nkv), dim3(256), 0, as_stream(stream), nkv, nh / nkv, dk, dv,
                     q, ldq, k, ldk, v, ldv, decay, scale, reset, S, o, ldo);
  return check_launch(fn);
}
