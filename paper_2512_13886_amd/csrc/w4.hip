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
// size. Masking the nibbles in place gives pairs of bf16 (16-bit activations) or
// bytes (8-bit ones) without any further movement:
//   bf16: a nibble m in the upper mantissa bits of 2^4 is 16 + m = code + 24;
//   int8: m = code + 8.
// The offset comes off through a second MFMA with a constant operand (-24, -8),
// whose result starts the sum of the group. Sums over a group are fp32 (int8: exact
// in int32), the sum over groups, each times its scales, is fp32.
//
// Bound by the codes' way from HBM, once per call for up to 64 tokens: a workgroup
// takes 16 rows, its eight waves every eighth chunk of them, and the waves' sums
// are joined in LDS in their order.
#include <type_traits>

#include "common.h"
#include "vec8.h"

namespace optima {
namespace {

constexpr int kChunk = 128;       // codes
constexpr int kChunkBytes = 64;
constexpr int kW4Tokens = 64;     // a workgroup's

typedef int i4 __attribute__((ext_vector_type(4)));

// Sixteen lanes a chunk, one dword (eight codes) each.
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
  load_upto8(raw, W + n * d + k, live ? d - k : 0);
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
  int64_t n_tok, d_out, ldx, ldy;
  int d, chunks, group, groups, x_groups, y_f32, act;
};

__device__ inline float w4_act(int act, float z) {
  return act == OPTIMA_ACT_SILU ? z / (1.f + expf(-z)) : z;
}

// Eight codes as bf16 values code + 24, in the order of their indices.
__device__ inline bf16x8 codes_bf16(uint32_t w) {
  constexpr uint32_t kMask = 0x00780078u, kBase = 0x41804180u;
  return __builtin_bit_cast(bf16x8, u32x4{((w << 3) & kMask) | kBase, ((w >> 1) & kMask) | kBase,
                                          ((w >> 5) & kMask) | kBase, ((w >> 9) & kMask) | kBase});
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
    Raw8<bf16_t> r;
    load_upto8(r, static_cast<const bf16_t*>(row) + k, left);
    v = __builtin_bit_cast(bf16x8, r.w);
  }
};
template <>
struct XFrag<true> {
  long v;
  __device__ inline void load(const void* row, int k, int left) {
    const uint8_t* p = static_cast<const uint8_t*>(row) + k;
    u32x2 r = {0, 0};
    if (left >= 8)
      r = *reinterpret_cast<const u32x2_1*>(p);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) r[i >> 2] |= uint32_t(p[i]) << (8 * (i & 3));
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

// Chunks that a wave takes at once, their loads together, and waves of a workgroup.
constexpr int w4_batch(int nt) { return nt == 1 ? 4 : nt == 2 ? 2 : 1; }
constexpr int w4_waves(int mats, int nt) { return mats * nt == 1 ? 16 : 8; }  // at most
// Bytes of one token's values of a batch in LDS (NT = 1), with 64 bytes between
// rows that keep the reads of several tokens off each other's banks.
constexpr int w4_x_pitch(bool i8) { return 4 * kChunk * (i8 ? 1 : 2) + 64; }

// 16 outputs of each of MATS matrices for up to 16 NT tokens; GP groups a chunk.
// Up to 16 tokens (NT = 1) a wave brings the tokens' values of its batch through
// LDS: the operand layout would read every value 16 times over, 16 / n_tok times
// for nothing.
template <bool I8, int MATS, int NT, int GP>
__global__ void __launch_bounds__(64 * w4_waves(MATS, NT)) k_w4(W4Args a) {
  constexpr int kBatch = w4_batch(NT), kPer = 4 / GP, kGroups = kBatch * GP;
  constexpr bool kStaged = NT == 1;
  constexpr int kPitch = w4_x_pitch(I8), kEsz = I8 ? 1 : 2;
  typedef typename std::conditional<I8, i4, f4>::type acc_t;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  float* part = reinterpret_cast<float*>(lds);  // [wave][MATS][NT][4][64], at the end
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int b = lane >> 4, i = lane & 15;
  const int64_t n0 = int64_t(blockIdx.x) * 16, t0 = int64_t(blockIdx.y) * kW4Tokens;
  const int64_t n = std::min(n0 + i, a.d_out - 1);
  const int tokens = int(std::min<int64_t>(a.n_tok - t0, 16 * NT));
  const char* x = static_cast<const char*>(a.x) + t0 * a.ldx * kEsz;
  const char* rows[NT];
  const float* xs[NT];  // of token 4 b + i % 4
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    rows[t] = x + std::min(16 * t + i, tokens - 1) * a.ldx * kEsz;
    xs[t] = a.xs + (t0 + std::min(16 * t + 4 * b + (i & 3), tokens - 1)) * a.x_groups;
  }
  char* mine = lds + wave * tokens * kPitch;
  f4 sum[MATS][NT];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[m][t] = f4{0.f, 0.f, 0.f, 0.f};
  for (int c0 = kBatch * wave; c0 < a.chunks; c0 += kBatch * waves) {
    u32x4 w[kBatch][MATS];
    uint32_t s[MATS][(kGroups + 1) / 2];
    float sx[NT][kGroups];
    // Lane l takes values 8 l .. of a token's batch, eight tokens at a time.
    XFrag<I8> row[kStaged ? 8 : 1];
    const int xk = c0 * kChunk + 8 * lane;
    if constexpr (kStaged)
#pragma unroll
      for (int r = 0; r < 8; ++r)
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
      load_scales<(kGroups + 1) / 2 * 2>(s[m], a.s[m] + n * a.groups, c0 * GP, a.groups);
    if constexpr (I8)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (a.x_groups > 1)
          load_scales<kGroups>(sx[t], xs[t], c0 * GP, a.groups);
        else
#pragma unroll
          for (int g = 0; g < kGroups; ++g) sx[t][g] = 1.f;
      }
    if constexpr (kStaged) {
      for (int r0 = 0;; r0 += 8) {
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (r0 + r < tokens)
            *reinterpret_cast<decltype(row[r].v)*>(mine + (r0 + r) * kPitch + lane * 8 * kEsz) = row[r].v;
        if (r0 + 8 >= tokens) break;
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (r0 + 8 + r < tokens) row[r].load(x + (r0 + 8 + r) * a.ldx * kEsz, xk, a.d - xk);
      }
      // The wave's own rows: its LDS accesses are served in order.
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      XFrag<I8> f[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (kStaged) {
            f[t][j].v = *reinterpret_cast<const decltype(f[t][j].v)*>(
                mine + std::min(i, tokens - 1) * kPitch + (u * kChunk + 32 * j + 8 * b) * kEsz);
          } else {
            const int k = (c0 + u) * kChunk + 32 * j + 8 * b;
            f[t][j].load(rows[t], k, a.d - k);
          }
        }
#pragma unroll
      for (int g = 0; g < GP; ++g)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc_t acc[MATS], base = {};
#pragma unroll
          for (int j = g * kPer; j < (g + 1) * kPer; ++j) {
            if constexpr (I8) {
              base = __builtin_amdgcn_mfma_i32_16x16x32_i8(
                  f[t][j].v, long(0xF8F8F8F8F8F8F8F8ull), base, 0, 0, 0);
            } else {
              const bf16x8 k24 = __builtin_bit_cast(
                  bf16x8, u32x4{0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u});
              base = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[t][j].v, k24, base, 0, 0, 0);
            }
          }
#pragma unroll
          for (int m = 0; m < MATS; ++m) {
            acc[m] = base;
#pragma unroll
            for (int j = g * kPer; j < (g + 1) * kPer; ++j) {
              if constexpr (I8)
                acc[m] = __builtin_amdgcn_mfma_i32_16x16x32_i8(f[t][j].v, codes_i8(w[u][m][j]),
                                                               acc[m], 0, 0, 0);
              else
                acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    f[t][j].v, codes_bf16(w[u][m][j]), acc[m], 0, 0, 0);
            }
          }
          const int gi = u * GP + g;
          float sc[MATS];
#pragma unroll
          for (int m = 0; m < MATS; ++m) sc[m] = scale_of(s[m][gi >> 1], gi & 1);
          float r[4] = {1.f, 1.f, 1.f, 1.f};
          if constexpr (I8) {
            r[0] = quad_lane<0>(sx[t][gi]);
            r[1] = quad_lane<1>(sx[t][gi]);
            r[2] = quad_lane<2>(sx[t][gi]);
            r[3] = quad_lane<3>(sx[t][gi]);
          }
#pragma unroll
          for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sum[m][t][e] += float(acc[m][e]) * (I8 ? sc[m] * r[e] : sc[m]);
        }
    }
    if constexpr (kStaged) __builtin_amdgcn_wave_barrier();
  }
  constexpr int kPart = MATS * NT * 256;
  __syncthreads();  // the staged values' place
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        part[wave * kPart + ((m * NT + t) * 4 + e) * 64 + lane] = sum[m][t][e];
  __syncthreads();
  for (int o = threadIdx.x; o < 256 * NT; o += blockDim.x) {
    const int nn = o & 15, m16 = (o >> 4) & 15, t = o >> 8;
    const int64_t tok = t0 + 16 * t + m16;
    if (tok >= a.n_tok || n0 + nn >= a.d_out) continue;
    float v[MATS];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      const float* p = part + ((m * NT + t) * 4 + (m16 & 3)) * 64 + (m16 >> 2) * 16 + nn;
      v[m] = 0.f;
      for (int w = 0; w < waves; ++w) v[m] += p[w * kPart];
      if (I8 && a.x_groups == 1) v[m] *= a.xs[tok];
    }
    const float y = MATS == 2 ? w4_act(a.act, v[0]) * v[MATS - 1] : v[0];
    const int64_t at = tok * a.ldy + n0 + nn;
    if (a.y_f32)
      static_cast<float*>(a.y)[at] = y;
    else
      store1(static_cast<bf16_t*>(a.y) + at, y);
  }
}

template <bool I8, int MATS, int NT, int GP>
void launch_w4(const W4Args& a, hipStream_t s) {
  // Few enough waves that each has a batch of chunks to load together.
  const int64_t batches = ceil_div(a.chunks, w4_batch(NT));
  const size_t stage = NT == 1 ? size_t(std::min<int64_t>(a.n_tok, 16)) * w4_x_pitch(I8) : 0;
  const size_t each = std::max(stage, size_t(MATS) * NT * 1024);
  constexpr size_t kLds = 136 << 10;
  const int most = int(std::min<size_t>(w4_waves(MATS, NT), kLds / each));
  const int waves = int(std::min<int64_t>(std::max<int64_t>(batches, 1), most));
  const dim3 grid(unsigned(ceil_div(a.d_out, 16)), unsigned(ceil_div(a.n_tok, kW4Tokens)));
  hipLaunchKernelGGL((k_w4<I8, MATS, NT, GP>), grid, dim3(64 * waves), waves * each, s, a);
}
template <bool I8, int MATS, int NT>
void launch_w4(const W4Args& a, hipStream_t s) {
  if (a.group == 32) launch_w4<I8, MATS, NT, 4>(a, s);
  else if (a.group == 64) launch_w4<I8, MATS, NT, 2>(a, s);
  else launch_w4<I8, MATS, NT, 1>(a, s);
}
template <bool I8, int MATS>
void launch_w4(const W4Args& a, hipStream_t s) {
  if (a.n_tok <= 16) launch_w4<I8, MATS, 1>(a, s);
  else if (a.n_tok <= 32) launch_w4<I8, MATS, 2>(a, s);
  else launch_w4<I8, MATS, 4>(a, s);
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

// With Q2 and s2, act(X deq(Q)^T) o (X deq(Q2)^T).
optima_status w4_linear(const void* X, int64_t ldx, const float* x_scales, int64_t x_group,
                        int64_t n_tok, int64_t d, const void* Q, const void* sc, const void* Q2,
                        const void* sc2, int64_t group, int64_t d_out, int act, void* Y,
                        int64_t ldy, int y_dtype, hipStream_t s) {
  W4Args a{};
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
