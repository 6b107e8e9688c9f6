// Products with 4-bit weights: packing, and Y = X deq(Q)^T of a few tokens, plain
// or gated.
//
// Packing: one scale = bf16(max |w| * (1 / 7)) for each group of 32, 64 or 128 values of
// a row, code = clamp(rne(w / scale), -7, 7), stored as code + 8. A zero weight has
// code 0, so that pruned entries stay exactly zero.
//
// A chunk of 128 codes is 64 bytes: dword j of the 16-byte block b holds the codes
// 32 j + 8 b .. + 7, the even ones in nibbles 0..3 and the odd ones in nibbles
// 4..7. In the products lane (b, n) of a wave takes block b of row n, and dword j
// of the four blocks is one 16x16x32 MFMA operand, of one group at every group
// size.
//   8-bit activations: the nibbles masked in place are bytes code + 8. The offset comes off
//     through a second MFMA with a constant operand (-8), whose result starts the sum of the
//     group; all of it is exact in int32.
//   16-bit ones: the nibbles are converted to bf16 values code / 16, and the outputs' sums
//     take the 16. No offset here: it would add to the fp32 sums what it takes off again, with
//     its rounding, and turn an infinite token into NaN.
// Sums over a group are fp32 or int32, the sum over groups, each times its scales, is fp32.
//
// The codes come from HBM once per call for up to 64 tokens. Up to 16 tokens a workgroup
// takes 16 rows, its waves batches of their chunks, and the waves' sums are joined in LDS in
// their order; more tokens share what is read of them. One 8-bit token, 4096 -> 2 x 14336:
// 14.5 us, 4.2 TB/s; eight 16-bit ones, 14336 -> 4096 in groups of 64: 10.2 us, 3.1 TB/s (16.9
// and 12.9 from weights that no cache holds). Bound by the latency of the one or two batches of
// loads that each wave has, and with more tokens by their reads out of the L2.
#include <type_traits>

#include "common.h"
#include "vec8.h"

namespace optima {
namespace {

constexpr int kChunk = 128;       // codes
constexpr int kChunkBytes = 64;

typedef int i4 __attribute__((ext_vector_type(4)));

// Sixteen lanes a chunk, one dword (eight codes) each. Bound by HBM: 14336 x 4096 fp32
// 50 us, 5.3 TB/s.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_w4_pack(const T* W, int64_t total, int chunks, int d,
                                                      int group, int groups, uint8_t* Q,
                                                      bf16_t* scales) {
  const int64_t idx = int64_t(blockIdx.x) * (kThreads / 16) + (threadIdx.x >> 4);
  const bool live = idx < total;  // of all 16 lanes
  const int64_t n = live ? idx / chunks : 0;
  const int c = live ? int(idx - n * chunks) : 0;
  const int i = threadIdx.x & 15;
  const int k = c * kChunk + 8 * i;
  Raw8<T> raw;
  load_piece(raw, W + n * d, k, live ? d : 0);
  float w[8];
  values8(raw, w);
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(w[e]) & 0x7FFFFFFFu);
  for (int o = 1; o < group / 8; o <<= 1) m = max(m, uint32_t(__shfl_xor(int(m), o, 64)));
  const uint32_t sb = pack_bf16(__uint_as_float(m) * (1.f / 7.f), 0.f) & 0xFFFFu;
  const float s = bf16_low(sb);
  if (live && (k & (group - 1)) == 0 && k < d) scales[n * groups + k / group].bits = uint16_t(sb);
  // A group with an infinity or NaN has codes 0 and that scale: NaN as values.
  const bool fine = s > 0.f && s < __builtin_inff();
  uint32_t q = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float code = fine ? fminf(fmaxf(rintf(w[e] / s), -7.f), 7.f) : 0.f;
    q |= uint32_t(int(code) + 8) << (4 * ((e >> 1) + 4 * (e & 1)));
  }
  if (live)
    *reinterpret_cast<uint32_t*>(Q + (n * chunks + c) * kChunkBytes + (i & 3) * 16 + (i >> 2) * 4) =
        q;
}

struct W4Args {
  const void* x;
  const float* xs;  // scales of 8-bit x, [n_tok][x_groups]
  const uint8_t* q[2];
  const bf16_t* s[2];
  void* y;
  f4* part;
  int64_t n_tok, d_out, ldx, ldy;
  int d, chunks, group, groups, x_groups, y_f32, act;
};

__device__ inline float w4_act(int act, float z) {
  return act == OPTIMA_ACT_SILU ? z / (1.f + expf(-z)) : z;
}

// Output n of a token from its sum (gated: sums) of products.
template <bool I8, int MATS>
__device__ inline void w4_store(const W4Args& a, int64_t tok, int64_t n, float (&v)[MATS]) {
#pragma unroll
  for (int m = 0; m < MATS; ++m)
    if (!I8)
      v[m] *= 16.f;
    else if (a.x_groups == 1)
      v[m] *= a.xs[tok];
  const float y = MATS == 2 ? w4_act(a.act, v[0]) * v[MATS - 1] : v[0];
  const int64_t at = tok * a.ldy + n;
  if (a.y_f32)
    static_cast<float*>(a.y)[at] = y;
  else
    store1(static_cast<bf16_t*>(a.y) + at, y);
}
// The outputs of a wave's two operands from row n0 on: 16 of both matrices, or 32.
template <bool I8, int MATS, int NT>
__device__ inline void slab_store(const W4Args& a, const f4 (&sum)[2][NT], int64_t n0, int64_t t0) {
  const int b = (threadIdx.x & 63) >> 4, i = threadIdx.x & 15;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t tok = t0 + 16 * t + 4 * b + e;
      if (tok >= a.n_tok) continue;
#pragma unroll
      for (int r = 0; r < 2 / MATS; ++r) {
        const int64_t n = n0 + 16 * r + i;
        if (n >= a.d_out) continue;
        float v[MATS];
#pragma unroll
        for (int m = 0; m < MATS; ++m) v[m] = sum[MATS == 2 ? m : r][t][e];
        w4_store<I8, MATS>(a, tok, n, v);
      }
    }
}

// code / 16 of a signed 4-bit code in the low half of byte BYTE. (The compiler's own builtin
// shifts the byte down first.)
template <int BYTE>
__device__ inline float code_of(uint32_t v) {
  static_assert(BYTE >= 0 && BYTE < 4, "");
  float r;
  if constexpr (BYTE == 0)
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(r) : "v"(v));
  else if constexpr (BYTE == 1)
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(r) : "v"(v));
  else if constexpr (BYTE == 2)
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(r) : "v"(v));
  else
    asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(r) : "v"(v));
  return r;
}
// Eight codes as bf16 values code / 16, in the order of their indices.
__device__ inline bf16x8 codes_bf16(uint32_t w) {
  const uint32_t lo = w ^ 0x88888888u, hi = lo >> 4;  // code + 8 as a signed code
  return __builtin_bit_cast(
      bf16x8, u32x4{pack_bf16(code_of<0>(lo), code_of<2>(lo)), pack_bf16(code_of<0>(hi), code_of<2>(hi)),
                    pack_bf16(code_of<1>(lo), code_of<3>(lo)), pack_bf16(code_of<1>(hi), code_of<3>(hi))});
}
// Eight codes as bytes code + 8, in the order 0 4 1 5, 2 6 3 7.
__device__ inline long codes_i8(uint32_t w) {
  return __builtin_bit_cast(long, u32x2{w & 0x0F0F0F0Fu, (w >> 4) & 0x0F0F0F0Fu});
}
// Eight bytes in that order.
__device__ inline long order_i8(u32x2 x) {
  return __builtin_bit_cast(long, u32x2{__builtin_amdgcn_perm(x[1], x[0], 0x05010400u),
                                        __builtin_amdgcn_perm(x[1], x[0], 0x07030602u)});
}

template <bool I8>
struct XFrag;
template <>
struct XFrag<false> {
  bf16x8 v;
  __device__ inline void load(const void* row, int k, int left) {
    const bf16_t* p = static_cast<const bf16_t*>(row) + k;
    Raw8<bf16_t> r;
    if (left >= 8)
      load8(r, p);
    else
      load_some(r, p, left);
    v = __builtin_bit_cast(bf16x8, r.w);
  }
};
template <>
struct XFrag<true> {
  long v;
  __device__ inline void load(const void* row, int k, int left) {
    const uint8_t* p = static_cast<const uint8_t*>(row) + k;
    u32x2 r = {0, 0};
    if (left >= 8) {
      r = *reinterpret_cast<const u32x2_1*>(p);
    } else if (left > 0 && k + left >= 8) {  // the row's last eight, moved down
      r = *reinterpret_cast<const u32x2_1*>(p + left - 8);
      r = __builtin_bit_cast(u32x2, __builtin_bit_cast(uint64_t, r) >> (8 * (8 - left)));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) r[i >> 2] |= uint32_t(p[i]) << (8 * (i & 3));
    }
    v = order_i8(r);
  }
};

// Lane 4 k + e's value in the four lanes 4 k .. 4 k + 3.
template <int E>
__device__ inline float quad_lane(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), E * 0x55, 0xF, 0xF, true));
}

// N (even) consecutive scales from group g on, two a word; zeros past the row's `groups`.
template <int N>
__device__ inline void load_scales(uint32_t (&v)[N / 2], const bf16_t* row, int g, int groups) {
  if (g + N <= groups) {
    struct __attribute__((packed, aligned(2))) Packed {
      uint32_t w[N / 2];
    } q;
    __builtin_memcpy(&q, row + g, sizeof(q));
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = q.w[i];
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      v[i] = g + 2 * i < groups ? row[g + 2 * i].bits : 0u;
      if (g + 2 * i + 1 < groups) v[i] |= uint32_t(row[g + 2 * i + 1].bits) << 16;
    }
  }
}
__device__ inline float scale_of(uint32_t w, int odd) { return odd ? bf16_high(w) : bf16_low(w); }
template <int N>
__device__ inline void load_scales(float (&v)[N], const float* row, int g, int groups) {
  if (g + N <= groups) {
    struct __attribute__((packed, aligned(4))) Packed {
      float f[N];
    } q;
    __builtin_memcpy(&q, row + g, sizeof(q));
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = q.f[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = g + i < groups ? row[g + i] : 0.f;
  }
}

// The sum of one group's products of 16 tokens with the 16 rows of each of OPS
// operands, of 16-bit tokens 1/16 of it. acc's layout: lane (b, i) holds tokens 4 b + e of row i.
template <bool I8, int OPS, int PER>
__device__ inline void group_sums(typename std::conditional<I8, i4, f4>::type (&acc)[OPS],
                                  const XFrag<I8> (&f)[4], const u32x4 (&w)[OPS], int j0) {
  typename std::conditional<I8, i4, f4>::type base = {};
  if constexpr (I8)
#pragma unroll
    for (int j = 0; j < PER; ++j)
      base = __builtin_amdgcn_mfma_i32_16x16x32_i8(f[j0 + j].v, long(0xF8F8F8F8F8F8F8F8ull), base,
                                                   0, 0, 0);
#pragma unroll
  for (int m = 0; m < OPS; ++m) {
    acc[m] = base;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if constexpr (I8)
        acc[m] = __builtin_amdgcn_mfma_i32_16x16x32_i8(f[j0 + j].v, codes_i8(w[m][j0 + j]), acc[m],
                                                       0, 0, 0);
      else
        acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[j0 + j].v, codes_bf16(w[m][j0 + j]),
                                                         acc[m], 0, 0, 0);
    }
  }
}

// Eight consecutive values of a token as they lie in LDS.
template <bool I8>
__device__ inline void put_x(char* p, const XFrag<I8>& f) {
  *reinterpret_cast<decltype(f.v)*>(p) = f.v;
}
template <bool I8>
__device__ inline void get_x(XFrag<I8>& f, const char* p) {
  f.v = *reinterpret_cast<const decltype(f.v)*>(p);
}

constexpr int kBatch = 4;                 // chunks whose loads go out together
constexpr int kBatchK = kBatch * kChunk;  // 512 values

// ---------------------------------------------------------------------------
// Up to 16 tokens
// ---------------------------------------------------------------------------

constexpr int kFew = 16;
// Waves of a workgroup at most, where a wave loads `rows` tokens at once: four for up to
// four tokens, which leaves the gated kernels registers for more waves a SIMD (one token,
// 4096 -> 2 x 14336, 16-bit: 24.5 us with eight, 19.3 with four), eight for more (8 tokens,
// 2048 -> 2 x 5632, 8.9 against 9.4; 16 tokens, 14336 -> 4096, 18.6 against 19.7; though 8
// tokens at 4096 -> 2 x 14336 25.8 against 22.4).
constexpr int few_waves(int mats, int rows) { return mats == 1 || rows == 4 ? 16 : 8; }
// Bytes of one token's values of a batch in LDS, with 64 bytes between rows that keep
// the reads of several tokens off each other's banks.
constexpr int few_pitch(bool i8) { return kBatchK * (i8 ? 1 : 2) + 64; }

// What lanes of a wave wrote to LDS before is there for its other lanes after. A wave's LDS
// accesses are served in order, so that this only keeps the compiler from moving them.
__device__ inline void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 16 outputs of each of MATS matrices; GP groups a chunk. A wave takes every waves-th
// batch and brings the tokens' values of it through LDS: the operand layout would read
// every value 16 times over, 16 / n_tok times for nothing.
template <bool I8, int MATS, int GP, int ROWS>
__global__ void __launch_bounds__(64 * few_waves(MATS, ROWS)) k_w4_few(W4Args a) {
  constexpr int kPer = 4 / GP, kGroups = kBatch * GP;
  constexpr int kPitch = few_pitch(I8), kEsz = I8 ? 1 : 2;
  typedef typename std::conditional<I8, i4, f4>::type acc_t;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  float* part = reinterpret_cast<float*>(lds);  // [wave][MATS][4][64], at the end
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int b = lane >> 4, i = lane & 15, tokens = int(a.n_tok);
  const int64_t n0 = int64_t(blockIdx.x) * 16;
  const int64_t n = std::min(n0 + i, a.d_out - 1);
  const char* x = static_cast<const char*>(a.x);
  const float* xs = a.xs + std::min(4 * b + (i & 3), tokens - 1) * a.x_groups;
  char* mine = lds + wave * tokens * kPitch;
  f4 sum[MATS];
#pragma unroll
  for (int m = 0; m < MATS; ++m) sum[m] = f4{0.f, 0.f, 0.f, 0.f};
  for (int c0 = kBatch * wave; c0 < a.chunks; c0 += kBatch * waves) {
    u32x4 w[kBatch][MATS];
    uint32_t s[MATS][kGroups / 2];
    float sx[kGroups];
    // Lane l takes values 8 l .. of a token's batch, ROWS tokens at a time.
    XFrag<I8> row[ROWS];
    const int xk = c0 * kChunk + 8 * lane;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (r < tokens) row[r].load(x + r * a.ldx * kEsz, xk, a.d - xk);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      // Past the last chunk: its codes again, with scales and tokens of zeros.
      const int c = std::min(c0 + u, a.chunks - 1);
#pragma unroll
      for (int m = 0; m < MATS; ++m)
        w[u][m] = *reinterpret_cast<const u32x4*>(a.q[m] + (n * a.chunks + c) * kChunkBytes + b * 16);
    }
#pragma unroll
    for (int m = 0; m < MATS; ++m)
      load_scales<kGroups>(s[m], a.s[m] + n * a.groups, c0 * GP, a.groups);
    if constexpr (I8) {
      if (a.x_groups > 1)
        load_scales<kGroups>(sx, xs, c0 * GP, a.groups);
      else
#pragma unroll
        for (int g = 0; g < kGroups; ++g) sx[g] = 1.f;
    }
    for (int r0 = 0;; r0 += ROWS) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
        if (r0 + r < tokens) put_x<I8>(mine + (r0 + r) * kPitch + lane * 8 * kEsz, row[r]);
      if (r0 + ROWS >= tokens) break;
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
        if (r0 + ROWS + r < tokens) row[r].load(x + (r0 + ROWS + r) * a.ldx * kEsz, xk, a.d - xk);
    }
    wave_exchange();
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      XFrag<I8> f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        get_x<I8>(f[j], mine + std::min(i, tokens - 1) * kPitch + (u * kChunk + 32 * j + 8 * b) * kEsz);
#pragma unroll
      for (int g = 0; g < GP; ++g) {
        acc_t acc[MATS];
        group_sums<I8, MATS, kPer>(acc, f, w[u], g * kPer);
        const int gi = u * GP + g;
        float r[4] = {1.f, 1.f, 1.f, 1.f};
        if constexpr (I8) {
          r[0] = quad_lane<0>(sx[gi]);
          r[1] = quad_lane<1>(sx[gi]);
          r[2] = quad_lane<2>(sx[gi]);
          r[3] = quad_lane<3>(sx[gi]);
        }
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
          const float sc = scale_of(s[m][gi >> 1], gi & 1);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[m][e] += float(acc[m][e]) * (I8 ? sc * r[e] : sc);
        }
      }
    }
    wave_exchange();
  }
  constexpr int kPart = MATS * 256;
  __syncthreads();  // the staged values' place
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[wave * kPart + (m * 4 + e) * 64 + lane] = sum[m][e];
  __syncthreads();
  for (int o = threadIdx.x; o < 256; o += blockDim.x) {
    const int nn = o & 15, tok = o >> 4;
    if (tok >= tokens || n0 + nn >= a.d_out) continue;
    float v[MATS];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      const float* p = part + (m * 4 + (tok & 3)) * 64 + (tok >> 2) * 16 + nn;
      v[m] = 0.f;
      for (int w = 0; w < waves; ++w) v[m] += p[w * kPart];
    }
    w4_store<I8, MATS>(a, tok, n0 + nn, v);
  }
}

// ---------------------------------------------------------------------------
// More tokens, 64 at a time
// ---------------------------------------------------------------------------

constexpr int kSlabTokens = 64;
constexpr int kSlabWaves = 8;
constexpr int kSlabBatch = 2;                    // chunks
constexpr int kSlabK = kSlabBatch * kChunk;
constexpr int slab_pitch(bool i8) { return kSlabK * (i8 ? 1 : 2) + 16; }
constexpr int slab_rows(int mats) { return kSlabWaves * 16 * (2 / mats); }  // a workgroup's

// The tokens' values of a batch go through LDS, two batches in turn, for all waves of the
// workgroup; a wave takes two operands of 16 rows (of both matrices, or two blocks of
// one), whose codes it loads a batch ahead. With few rows the chunks are split over
// blockIdx.y, and k_w4_join adds the parts: 16 rows' own read of the tokens, as above,
// would bring every token N / 16 times out of the L2.
// Bound by latency: at 64 tokens, 4096 -> 2 x 14336, the MFMAs are busy for 16 % of 38 us
// (8-bit: 21 % of 42), and the two waves a SIMD wait for loads and barriers for 41 and 50 %.
template <bool I8, int MATS, int NT, int GP>
__global__ void __launch_bounds__(64 * kSlabWaves) k_w4_slab(W4Args a) {
  constexpr int kPer = 4 / GP, kGroups = kSlabBatch * GP, OPS = 2;
  constexpr int kPitch = slab_pitch(I8), kEsz = I8 ? 1 : 2, kTok = 16 * NT;
  typedef typename std::conditional<I8, i4, f4>::type acc_t;
  __shared__ __attribute__((aligned(16))) char xl[2][kTok * kPitch];
  __shared__ __attribute__((aligned(16))) float xsl[2][I8 ? kGroups * kTok : 1];  // [group][token]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = lane >> 4, i = lane & 15;
  const int64_t t0 = int64_t(blockIdx.z) * kSlabTokens;
  const int tokens = int(std::min<int64_t>(a.n_tok - t0, kTok));
  const char* x = static_cast<const char*>(a.x) + t0 * a.ldx * kEsz;
  const float* xs = a.xs + t0 * a.x_groups;
  int64_t n[OPS];
#pragma unroll
  for (int m = 0; m < OPS; ++m)
    n[m] = std::min(int64_t(blockIdx.x) * slab_rows(MATS) + wave * 16 * (2 / MATS) +
                        (MATS == 1 ? 16 * m : 0) + i, a.d_out - 1);
  const int batches = (a.chunks + kSlabBatch - 1) / kSlabBatch;
  const int b0 = int(int64_t(batches) * blockIdx.y / gridDim.y);
  const int b1 = int(int64_t(batches) * (blockIdx.y + 1) / gridDim.y);

  // This thread's share of a batch's tokens: values 8 (thread % 32) .. of every 16th.
  const int xt = threadIdx.x >> 5, xk = 8 * (threadIdx.x & 31);
  XFrag<I8> row[NT];
  float rs[I8 ? (kGroups * kTok + 511) / 512 : 1];
  auto fetch_x = [&](int batch) {
    const int k = batch * kSlabK + xk;
#pragma unroll
    for (int r = 0; r < NT; ++r)
      row[r].load(x + std::min(xt + 16 * r, tokens - 1) * a.ldx * kEsz, k, a.d - k);
    if constexpr (I8)
      if (a.x_groups > 1)
#pragma unroll
        for (int v = 0; v < int(sizeof(rs) / 4); ++v) {
          const int at = threadIdx.x + 512 * v, g = batch * kGroups + at / kTok;
          rs[v] = g < a.groups && at < kGroups * kTok
                      ? xs[std::min(at % kTok, tokens - 1) * a.x_groups + g] : 0.f;
        }
  };
  auto put_batch = [&](int to) {
#pragma unroll
    for (int r = 0; r < NT; ++r) put_x<I8>(xl[to] + (xt + 16 * r) * kPitch + xk * kEsz, row[r]);
    if constexpr (I8)
      if (a.x_groups > 1)
#pragma unroll
        for (int v = 0; v < int(sizeof(rs) / 4); ++v) {
          const int at = threadIdx.x + 512 * v;
          if (at < kGroups * kTok) xsl[to][at] = rs[v];
        }
  };
  u32x4 w[kSlabBatch][OPS];
  uint32_t s[OPS][(kGroups / 2)];
  auto fetch_w = [&](int batch) {
#pragma unroll
    for (int u = 0; u < kSlabBatch; ++u) {
      const int c = std::min(batch * kSlabBatch + u, a.chunks - 1);
#pragma unroll
      for (int m = 0; m < OPS; ++m)
        w[u][m] = *reinterpret_cast<const u32x4*>(a.q[m % MATS] + (n[m] * a.chunks + c) * kChunkBytes +
                                                  b * 16);
    }
#pragma unroll
    for (int m = 0; m < OPS; ++m)
      load_scales<kGroups>(s[m], a.s[m % MATS] + n[m] * a.groups, batch * kGroups, a.groups);
  };

  f4 sum[OPS][NT];
#pragma unroll
  for (int m = 0; m < OPS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[m][t] = f4{0.f, 0.f, 0.f, 0.f};
  if (b0 < b1) {
    fetch_x(b0);
    fetch_w(b0);
    put_batch(0);
  }
  __syncthreads();
  for (int batch = b0; batch < b1; ++batch) {
    const int cur = (batch - b0) & 1;
    u32x4 wc[kSlabBatch][OPS];
    uint32_t sc[OPS][(kGroups / 2)];
#pragma unroll
    for (int u = 0; u < kSlabBatch; ++u)
#pragma unroll
      for (int m = 0; m < OPS; ++m) wc[u][m] = w[u][m];
#pragma unroll
    for (int m = 0; m < OPS; ++m)
#pragma unroll
      for (int g = 0; g < (kGroups / 2); ++g) sc[m][g] = s[m][g];
    if (batch + 1 < b1) {
      fetch_x(batch + 1);
      fetch_w(batch + 1);
    }
#pragma unroll
    for (int u = 0; u < kSlabBatch; ++u)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        XFrag<I8> f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          get_x<I8>(f[j], xl[cur] + (16 * t + i) * kPitch + (u * kChunk + 32 * j + 8 * b) * kEsz);
#pragma unroll
        for (int g = 0; g < GP; ++g) {
          acc_t acc[OPS];
          group_sums<I8, OPS, kPer>(acc, f, wc[u], g * kPer);
          const int gi = u * GP + g;
          f4 r = {1.f, 1.f, 1.f, 1.f};
          if constexpr (I8)
            if (a.x_groups > 1) r = *reinterpret_cast<const f4*>(&xsl[cur][gi * kTok + 16 * t + 4 * b]);
#pragma unroll
          for (int m = 0; m < OPS; ++m) {
            const float q = scale_of(sc[m][gi >> 1], gi & 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[m][t][e] += float(acc[m][e]) * (I8 ? q * r[e] : q);
          }
        }
        // Looking further ahead than this the compiler runs out of registers.
#pragma unroll
        for (int m = 0; m < OPS; ++m) asm volatile("" : "+v"(sum[m][t]));
      }
    if (batch + 1 < b1) put_batch(cur ^ 1);
    __syncthreads();
  }
  if (gridDim.y > 1) {  // [split][64 tokens][workgroup][wave][operand][token block][lane]
    const size_t wg = (size_t(blockIdx.y) * gridDim.z + blockIdx.z) * gridDim.x + blockIdx.x;
    f4* part = a.part + (wg * kSlabWaves + wave) * OPS * NT * 64;
#pragma unroll
    for (int m = 0; m < OPS; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t) part[(m * NT + t) * 64 + lane] = sum[m][t];
    return;
  }
  slab_store<I8, MATS, NT>(a, sum, int64_t(blockIdx.x) * slab_rows(MATS) + wave * 16 * (2 / MATS), t0);
}

// The parts of the outputs, added in their order: one of the slab kernel's waves' outputs
// for 16 tokens a wave. waves: of all tokens; per: of 64 of them.
template <bool I8, int MATS, int NT>
__global__ void __launch_bounds__(kThreads) k_w4_join(W4Args a, int splits, int waves, int per) {
  const int lane = threadIdx.x & 63, at = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int wave = at / NT, t = at - wave * NT;
  if (wave >= waves) return;
  const int z = wave / per;
  const f4* part = a.part + (size_t(wave) * 2 * NT + t) * 64 + lane;
  const size_t step = size_t(waves) * 2 * NT * 64;
  f4 sum[2][1] = {{{0.f, 0.f, 0.f, 0.f}}, {{0.f, 0.f, 0.f, 0.f}}};
#pragma unroll 8
  for (int sp = 0; sp < splits; ++sp)
#pragma unroll
    for (int m = 0; m < 2; ++m) sum[m][0] += part[sp * step + m * NT * 64];
  slab_store<I8, MATS, 1>(a, sum, int64_t(wave - z * per) * 16 * (2 / MATS),
                          int64_t(z) * kSlabTokens + 16 * t);
}

// Ranges that the chunks of a product of more than kFew tokens are split into: as many
// as give every CU a workgroup (14336 -> 2 x 4096, 128 tokens: 186 us in one, 62 in
// four). Beyond eight they have two batches at least: 4096 -> 4096, 64 tokens, 16.6 us in
// 8 ranges, 19.7 in 16. Two batches of up to 32 tokens stay whole: 512 -> 2048, 17 tokens,
// 6.9 us and 7.4.
int64_t slab_splits(int64_t n_tok, int64_t d, int64_t d_out, int mats) {
  const int64_t wgs = ceil_div(d_out, slab_rows(mats)) * ceil_div(n_tok, kSlabTokens);
  const int64_t batches = ceil_div(d, kSlabK);
  if (batches <= 2 && n_tok <= 32) return 1;
  return std::max<int64_t>(1, std::min(256 / wgs, std::max(batches / 2, std::min<int64_t>(batches, 8))));
}

template <bool I8, int MATS, int NT, int GP>
void launch_slab(const W4Args& a, hipStream_t s) {
  const unsigned wgs = unsigned(ceil_div(a.d_out, slab_rows(MATS)));
  const unsigned tiles = unsigned(ceil_div(a.n_tok, kSlabTokens));
  const int splits = int(slab_splits(a.n_tok, a.d, a.d_out, MATS));
  hipLaunchKernelGGL((k_w4_slab<I8, MATS, NT, GP>), dim3(wgs, unsigned(splits), tiles),
                     dim3(64 * kSlabWaves), 0, s, a);
  if (splits > 1) {
    const unsigned per = wgs * kSlabWaves, waves = per * tiles;
    hipLaunchKernelGGL((k_w4_join<I8, MATS, NT>), dim3(waves * NT / (kThreads / 64)),
                       dim3(kThreads), 0, s, a, splits, int(waves), int(per));
  }
}

template <bool I8, int MATS, int GP, int ROWS>
void launch_few(const W4Args& a, hipStream_t s) {
  // Few enough waves that each has a batch of chunks to load together, and whose tokens the
  // CU's LDS holds: 12 tokens, 14336 -> 4096, 14.9 us with 12 waves, 15.8 with 10.
  const size_t each = std::max(size_t(a.n_tok) * few_pitch(I8), size_t(MATS) * 1024);
  constexpr size_t kLds = 160 << 10;
  const int most = int(std::min<size_t>(few_waves(MATS, ROWS), kLds / each));
  const int waves = int(std::min<int64_t>(ceil_div(a.chunks, kBatch), most));
  hipLaunchKernelGGL((k_w4_few<I8, MATS, GP, ROWS>), dim3(unsigned(ceil_div(a.d_out, 16))),
                     dim3(64 * waves), waves * each, s, a);
}

template <bool I8, int MATS, int GP>
void launch_w4(const W4Args& a, hipStream_t s) {
  if (a.n_tok > 32) launch_slab<I8, MATS, 4, GP>(a, s);
  else if (a.n_tok > kFew) launch_slab<I8, MATS, 2, GP>(a, s);
  else if (a.n_tok > 4) launch_few<I8, MATS, GP, 8>(a, s);
  else launch_few<I8, MATS, GP, 4>(a, s);
}
template <bool I8, int MATS>
void launch_w4(const W4Args& a, hipStream_t s) {
  if (a.group == 32) launch_w4<I8, MATS, 4>(a, s);
  else if (a.group == 64) launch_w4<I8, MATS, 2>(a, s);
  else launch_w4<I8, MATS, 1>(a, s);
}

}  // namespace

optima_status w4_pack(const void* W, int dtype, int64_t n, int64_t d, int64_t group, void* Q,
                      void* scales, hipStream_t s) {
  const int chunks = int(ceil_div(d, kChunk)), groups = int(ceil_div(d, group));
  const int64_t total = n * chunks;
  const dim3 grid(unsigned(ceil_div(total, kThreads / 16)));
  if (dtype == OPTIMA_DTYPE_BF16)
    hipLaunchKernelGGL(k_w4_pack<bf16_t>, grid, dim3(kThreads), 0, s,
                       static_cast<const bf16_t*>(W), total, chunks, int(d), int(group), groups,
                       static_cast<uint8_t*>(Q), static_cast<bf16_t*>(scales));
  else
    hipLaunchKernelGGL(k_w4_pack<float>, grid, dim3(kThreads), 0, s, static_cast<const float*>(W),
                       total, chunks, int(d), int(group), groups, static_cast<uint8_t*>(Q),
                       static_cast<bf16_t*>(scales));
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

size_t w4_workspace_bytes(int64_t n_tok, int64_t d, int64_t d_out, int mats) {
  if (n_tok <= kFew) return 0;
  // The most of any number of tokens up to these, so that more need no less.
  const int64_t wgs = ceil_div(d_out, slab_rows(mats)), tiles = ceil_div(n_tok, kSlabTokens);
  int64_t parts = 0;
  for (int64_t t = 1; t <= std::min(tiles, 128 / wgs); ++t) {
    const int64_t splits = slab_splits(t * kSlabTokens, d, d_out, mats);
    if (splits > 1) parts = std::max(parts, splits * t);
  }
  return size_t(parts) * size_t(wgs) * kSlabWaves * 2 * (kSlabTokens / 16) * 64 * sizeof(f4);
}

// With Q2 and s2, act(X deq(Q)^T) o (X deq(Q2)^T).
optima_status w4_linear(const void* X, int64_t ldx, const float* x_scales, int64_t x_group,
                        int64_t n_tok, int64_t d, const void* Q, const void* sc, const void* Q2,
                        const void* sc2, int64_t group, int64_t d_out, int act, void* Y,
                        int64_t ldy, int y_dtype, void* ws, hipStream_t s) {
  W4Args a{};
  a.part = static_cast<f4*>(ws);
  a.x = X;
  a.xs = x_scales;
  a.q[0] = static_cast<const uint8_t*>(Q);
  a.q[1] = static_cast<const uint8_t*>(Q2);
  a.s[0] = static_cast<const bf16_t*>(sc);
  a.s[1] = static_cast<const bf16_t*>(sc2);
  a.y = Y;
  a.n_tok = n_tok;
  a.d_out = d_out;
  a.ldx = ldx;
  a.ldy = ldy;
  a.d = int(d);
  a.chunks = int(ceil_div(d, kChunk));
  a.group = int(group);
  a.groups = int(ceil_div(d, group));
  // One group covers the row: the same as one scale a token.
  a.x_groups = x_scales ? int(x_group ? ceil_div(d, x_group) : 1) : 0;
  a.y_f32 = y_dtype == OPTIMA_DTYPE_F32;
  a.act = act;
  if (x_scales) {
    if (Q2) launch_w4<true, 2>(a, s);
    else launch_w4<true, 1>(a, s);
  } else {
    if (Q2) launch_w4<false, 2>(a, s);
    else launch_w4<false, 1>(a, s);
  }
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

}  // namespace optima
