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
constexpr int kW4Waves = 8;
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

// 16 outputs of each of MATS matrices for up to 16 NT tokens.
template <bool I8, int MATS, int NT>
__global__ void __launch_bounds__(64 * kW4Waves) k_w4(W4Args a) {
  __shared__ float part[kW4Waves][MATS][NT][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b = lane >> 4, i = lane & 15;
  const int64_t n0 = int64_t(blockIdx.x) * 16, t0 = int64_t(blockIdx.y) * kW4Tokens;
  const int64_t n = std::min(n0 + i, a.d_out - 1);
  const char* x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
    x[t] = static_cast<const char*>(a.x) +
           std::min(t0 + 16 * t + i, a.n_tok - 1) * a.ldx * (I8 ? 1 : 2);
  f4 sum[MATS][NT];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[m][t] = f4{0.f, 0.f, 0.f, 0.f};
  const int per = a.group / 32;  // dwords of a chunk in a group: 1, 2 or 4
  for (int c = wave; c < a.chunks; c += kW4Waves) {
    u32x4 w[MATS];
#pragma unroll
    for (int m = 0; m < MATS; ++m)
      w[m] = *reinterpret_cast<const u32x4*>(a.q[m] + (n * a.chunks + c) * kChunkBytes + b * 16);
    XFrag<I8> f[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = c * kChunk + 32 * j + 8 * b;
        f[t][j].load(x[t], k, a.d - k);
      }
    typedef typename std::conditional<I8, i4, f4>::type acc_t;
    acc_t acc[MATS][NT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        acc_t base = {};
        if constexpr (I8) {
          base = __builtin_amdgcn_mfma_i32_16x16x32_i8(f[t][j].v, long(0xF8F8F8F8F8F8F8F8ull), base,
                                                       0, 0, 0);
        } else {
          const bf16x8 k24 = __builtin_bit_cast(
              bf16x8, u32x4{0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u});
          base = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[t][j].v, k24, base, 0, 0, 0);
        }
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
          acc_t v = base;
          if constexpr (I8)
            v = __builtin_amdgcn_mfma_i32_16x16x32_i8(f[t][j].v, codes_i8(w[m][j]), v, 0, 0, 0);
          else
            v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[t][j].v, codes_bf16(w[m][j]), v, 0, 0, 0);
          acc[m][t] = j % per == 0 ? v : acc[m][t] + v;
        }
      }
      if ((j + 1) % per) continue;
      const int g = (c * 4 + j) / per;  // the group that ends here
      if (g >= a.groups) continue;      // padding
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float xs[4] = {1.f, 1.f, 1.f, 1.f};
        if (I8 && a.x_groups > 1)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            xs[e] = a.xs[std::min(t0 + 16 * t + 4 * b + e, a.n_tok - 1) * a.x_groups + g];
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
          const float s = bf16_low(a.s[m][n * a.groups + g].bits);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[m][t][e] += float(acc[m][t][e]) * (s * xs[e]);
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[wave][m][t][e][lane] = sum[m][t][e];
  __syncthreads();
  for (int o = threadIdx.x; o < 256 * NT; o += 64 * kW4Waves) {
    const int nn = o & 15, m16 = (o >> 4) & 15, t = o >> 8;
    const int64_t tok = t0 + 16 * t + m16;
    if (tok >= a.n_tok || n0 + nn >= a.d_out) continue;
    float v[MATS];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
      v[m] = 0.f;
#pragma unroll
      for (int w = 0; w < kW4Waves; ++w) v[m] += part[w][m][t][m16 & 3][(m16 >> 2) * 16 + nn];
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

template <bool I8, int MATS>
void launch_w4(const W4Args& a, hipStream_t s) {
  const dim3 grid(unsigned(ceil_div(a.d_out, 16)), unsigned(ceil_div(a.n_tok, kW4Tokens)));
  const dim3 wg(64 * kW4Waves);
  if (a.n_tok <= 16) hipLaunchKernelGGL((k_w4<I8, MATS, 1>), grid, wg, 0, s, a);
  else if (a.n_tok <= 32) hipLaunchKernelGGL((k_w4<I8, MATS, 2>), grid, wg, 0, s, a);
  else hipLaunchKernelGGL((k_w4<I8, MATS, 4>), grid, wg, 0, s, a);
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
