// The gated feed-forward product of a decoder block and its gradient.
//
// Forward: g = X Wg^T, u = X Wu^T, h = act(g) o u, with X [n_tok][d] and Wg, Wu
// [ff][d] in bf16. A tile multiplies the same token rows with rows of both weights,
// so that g and u of an output meet in one lane's registers.
// Up to 64 tokens: bound by the weights' way from HBM, k_gated_few streams them once.
// One token, 4096 -> 14336: 38.5 us, 6.1 TB/s.
//
// Backward: dU = dH o act(g), dG = dH o u o act'(g), then
//   dX = [dG dU] [Wg; Wu],  [dWg; dWu] = [dG dU]^T X  (o masks).
// The matrix instructions take P = [dG dU] in bf16: it comes in two bf16 parts, 16 bits of
// mantissa, with twice the instructions. Rounded to one, 4096 tokens, 4096 -> 14336: fp32
// gradients 1.7e-3 off in place of 5e-6, bf16 ones 2.35e-3 in place of the 1.66e-3 that their own
// rounding makes; 1.58 ms in place of 3.07.
#include "common.h"
#include "gated_plan.h"
#include "gemm128.h"
#include "gemm256.h"
#include "gemm_core.h"
#include "vec8.h"

namespace optima {
namespace {

__device__ inline int cdiv(int64_t a, int b) { return int((a + b - 1) / b); }

__device__ inline float gate_act(int act, float z) {
  return act == OPTIMA_ACT_SILU ? z / (1.f + expf(-z)) : z;
}
// act(z) and its derivative.
__device__ inline void gate_act_slope(int act, float z, float* a, float* slope) {
  if (act == OPTIMA_ACT_SILU) {
    const float sig = 1.f / (1.f + expf(-z));
    *a = z * sig;
    *slope = sig * (1.f + z * (1.f - sig));
  } else {
    *a = z;
    *slope = 1.f;
  }
}

struct GatedArgs {
  const char *x, *wg, *wu;  // rows of bf16
  void* h;
  bf16_t *g, *u;                // or NULL
  int64_t n_tok, d, ff;
  int64_t ldx, ldw, ldh, ldg, ldu;  // in elements
  int h_f32, act;
  int splits;   // ranges of the sum over d (k_gated_ring) ..
  float* part;  // .. whose parts go here: [split][tile][128][g: 64, u: 64]
  // The outputs from n on.
  void skip(int64_t n) {
    wg += 2 * n * ldw;
    wu += 2 * n * ldw;
    h = static_cast<char*>(h) + (h_f32 ? 4 : 2) * n;
    if (g) g += n;
    if (u) u += n;
    ff -= n;
  }
};

// Four or eight consecutive outputs of a token from their sums g and u.
template <int N>
__device__ inline void gated_store(const GatedArgs& a, int64_t tok, int64_t n, const float (&g)[N],
                                   const float (&u)[N]) {
  const int left = int(std::max<int64_t>(std::min<int64_t>(a.ff - n, N), 0));
  float h[N];
#pragma unroll
  for (int e = 0; e < N; ++e) h[e] = gate_act(a.act, g[e]) * u[e];
  auto put = [left](auto* p, const float (&v)[N]) {
    if constexpr (N == 8)
      store_upto8(p, v, left);
    else
      store_upto4(p, v, left);
  };
  if (a.g) put(a.g + tok * a.ldg + n, g);
  if (a.u) put(a.u + tok * a.ldu + n, u);
  if (a.h_f32)
    put(static_cast<float*>(a.h) + tok * a.ldh + n, h);
  else
    put(static_cast<bf16_t*>(a.h) + tok * a.ldh + n, h);
}

// ---------------------------------------------------------------------------
// Few tokens: the waves of a workgroup take the 64-value pieces of its weight rows in
// turn, and their sums are joined in LDS in their order. Lane (q, i) reads
// values 16 q .. + 15 of a piece of row i: two MFMA operands, and with the other
// lanes whole 128-byte lines. The 16 rows of an operand are MATS = 1: 8 of Wg and
// the same 8 of Wu; MATS = 2: 16 of each, in two operands that share the tokens'.
// ---------------------------------------------------------------------------
constexpr int few_waves(int mats) { return mats == 1 ? 16 : 8; }  // at most
// Pieces that a wave loads together.
constexpr int few_batch(int nt) { return nt <= 2 ? 2 : 1; }

__device__ inline f4 few_mfma(const Raw8<bf16_t>& x, const Raw8<bf16_t>& w, const f4& acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.w),
                                                 __builtin_bit_cast(bf16x8, w.w), acc, 0, 0, 0);
}

// 16 values of a row. Where ODD, rows may lie at odd elements: a 16-byte load whose address
// is no multiple of 4 is slow, so that these are loaded from one element earlier, and moved
// (4097 -> 14336: one token 95 us as they lie, 51 moved, 64 tokens 295 and 139; 1001 ->
// 2731, 13 tokens 10.4 and 7.5). Kernels with more waves to wait for gained nothing.
template <bool ODD>
struct FewRaw {
  Raw8<bf16_t> half[2];
  uint32_t last;
  __device__ inline void load(const bf16_t* p, int shift) {
    if (ODD) {
      last = p[15].bits;
      p -= shift / 16;
    }
    load8(half[0], p);
    load8(half[1], p + 8);
  }
  __device__ inline Raw8<bf16_t> get(int e, int shift) const {
    if (!ODD) return half[e];
    const u32x4 w = half[e].w;
    const uint32_t next = e == 0 ? half[1].w[0] : last;
    return Raw8<bf16_t>{u32x4{__builtin_amdgcn_alignbit(w[1], w[0], shift),
                              __builtin_amdgcn_alignbit(w[2], w[1], shift),
                              __builtin_amdgcn_alignbit(w[3], w[2], shift),
                              __builtin_amdgcn_alignbit(next, w[3], shift)}};
  }
};
// Bits by which a row's values are moved. The element before the first row is not there.
__device__ inline int row_shift(const bf16_t* row, int64_t index) {
  return index > 0 && (reinterpret_cast<uintptr_t>(row) & 2) ? 16 : 0;
}

template <int MATS, int NT, bool ODD>
__global__ void __launch_bounds__(64 * few_waves(MATS)) k_gated_few(GatedArgs a) {
  constexpr int kBatch = few_batch(NT), kOut = 8 * MATS;
  __shared__ float part[few_waves(MATS)][MATS][NT][4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int q = lane >> 4, i = lane & 15;
  const int64_t n0 = int64_t(blockIdx.x) * kOut;
  const int64_t n = std::min(n0 + (i & (kOut - 1)), a.ff - 1);
  const bf16_t* w[MATS];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
    w[m] = reinterpret_cast<const bf16_t*>((MATS == 1 ? i >= 8 : m) ? a.wu : a.wg) + n * a.ldw;
  const bf16_t* x[NT];
  int shift_w[MATS], shift_x[NT];
#pragma unroll
  for (int m = 0; m < MATS; ++m) shift_w[m] = row_shift(w[m], n);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t tok = std::min<int64_t>(16 * t + i, a.n_tok - 1);
    x[t] = reinterpret_cast<const bf16_t*>(a.x) + tok * a.ldx;
    shift_x[t] = row_shift(x[t], tok);
  }
  f4 acc[MATS][NT];
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[m][t] = f4{0.f, 0.f, 0.f, 0.f};
  const int pieces = int(a.d / 64);  // whole ones
  for (int c0 = wave; c0 < pieces; c0 += waves * kBatch) {
    FewRaw<ODD> rw[kBatch][MATS], rx[kBatch][NT];
#pragma unroll
    for (int v = 0; v < kBatch; ++v) {
      const int k = 64 * (c0 + v * waves) + 16 * q;
      if (c0 + v * waves >= pieces) break;
#pragma unroll
      for (int m = 0; m < MATS; ++m) rw[v][m].load(w[m] + k, shift_w[m]);
#pragma unroll
      for (int t = 0; t < NT; ++t) rx[v][t].load(x[t] + k, shift_x[t]);
    }
#pragma unroll
    for (int v = 0; v < kBatch; ++v) {
      if (c0 + v * waves >= pieces) break;
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int m = 0; m < MATS; ++m)
            acc[m][t] = few_mfma(rx[v][t].get(e, shift_x[t]), rw[v][m].get(e, shift_w[m]), acc[m][t]);
    }
  }
  if (a.d % 64 && wave == pieces % waves) {  // the rest, by the wave whose turn it is
    const int k = 64 * pieces + 16 * q, d = int(a.d);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      Raw8<bf16_t> rw[MATS], rx;
#pragma unroll
      for (int m = 0; m < MATS; ++m) load_piece(rw[m], w[m], k + 8 * e, d);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        load_piece(rx, x[t], k + 8 * e, d);
#pragma unroll
        for (int m = 0; m < MATS; ++m) acc[m][t] = few_mfma(rx, rw[m], acc[m][t]);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MATS; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[wave][m][t][e][lane] = acc[m][t][e];
  __syncthreads();
  for (int o = threadIdx.x; o < 16 * kOut * NT; o += blockDim.x) {
    const int nn = o % kOut, m16 = o / kOut & 15, t = o / (16 * kOut);
    const int64_t tok = 16 * t + m16, at = n0 + nn;
    if (tok >= a.n_tok || at >= a.ff) continue;
    float v[2] = {0.f, 0.f};
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int m = 0; m < 2; ++m)
        v[m] += part[w][MATS == 1 ? 0 : m][t][m16 & 3][(m16 >> 2) * 16 + (MATS == 1 ? 8 * m : 0) + nn];
    const float h = gate_act(a.act, v[0]) * v[1];
    if (a.h_f32)
      static_cast<float*>(a.h)[tok * a.ldh + at] = h;
    else
      store1(static_cast<bf16_t*>(a.h) + tok * a.ldh + at, h);
    if (a.g) store1(a.g + tok * a.ldg + at, v[0]);
    if (a.u) store1(a.u + tok * a.ldu + at, v[1]);
  }
}

template <int MATS, int NT>
void launch_few(const GatedArgs& a, hipStream_t s) {
  // Enough pieces for sixteen waves to have a batch each.
  const int waves = MATS == 1 && a.d >= 2048 ? 16 : 8;
  const dim3 grid(unsigned(ceil_div(a.ff, 8 * MATS))), block(64 * waves);
  if (a.ldw % 2 || (a.n_tok > 1 && a.ldx % 2))
    hipLaunchKernelGGL((k_gated_few<MATS, NT, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((k_gated_few<MATS, NT, false>), grid, block, 0, s, a);
}

// ---------------------------------------------------------------------------
// Tiles. Operand rows are 16-byte aligned with whole 64-value stages.
// ---------------------------------------------------------------------------

// 256 tokens x 128 outputs on the 256 x 256 tile: half B0 holds rows of Wg, half
// B1 the same rows of Wu, so quadrants (qa, 0) and (qa, 1) of a lane are g and u of
// the same outputs. Bound by MFMA: 8192 tokens, 4096 -> 14336, g and u kept, 1430 us,
// 1.35 PFLOP/s.
__global__ void __launch_bounds__(Tile256::kThreads) k_gated256(GatedArgs a) {
  __shared__ __attribute__((aligned(1024))) char l0[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l1[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l2[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l3[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l4[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l5[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l6[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l7[Tile256::kHalfBytes];
  const int tiles_m = cdiv(a.n_tok, 256), tiles_n = cdiv(a.ff, 128);
  int tm, tn;
  tile_of_block(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, &tm, &tn);
  const int64_t m0 = int64_t(tm) * 256, n0 = int64_t(tn) * 128;
  Operands256 src;
#pragma unroll
  for (int i = 0; i < Tile256::kHalfLoads; ++i) {
    const int r = t256_load_row(i), seg = t256_seg_bytes(i);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      src.a[h][i] = a.x + std::min(m0 + 128 * h + r, a.n_tok - 1) * (2 * a.ldx) + seg;
      src.b[h][i] = (h ? a.wu : a.wg) +
                    std::min(n0 + t256_rows_source(r), a.ff - 1) * (2 * a.ldw) + seg;
    }
  }
  Acc256 acc;
  gemm256_mainloop<Bf16Rows<false>>(acc, src, int(a.d / 64), l0, l1, l2, l3, l4, l5, l6, l7, [] {});

  const int64_t n = n0 + t256_rows_col(0);
#pragma unroll
  for (int qa = 0; qa < 2; ++qa)
#pragma unroll
    for (int mi = 0; mi < 4; ++mi) {
      const int64_t tok = m0 + t256_rows_row(qa, mi);
      if (tok >= a.n_tok) continue;
      float g[8], u[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[e] = acc.q[qa][0][mi][e >> 2][e & 3];
        u[e] = acc.q[qa][1][mi][e >> 2][e & 3];
      }
      gated_store<8>(a, tok, n, g, u);
    }
}

struct SplitSteps {
  int s0;  // the workgroup's first stage
  __device__ inline int64_t a(int s) const { return int64_t(s0 + s) * 128; }
  __device__ inline int64_t b(int s) const { return int64_t(s0 + s) * 128; }
};

// 128 tokens x 64 outputs on the 128 x 128 ring tile: 16-row blocks of B are rows
// of Wg and Wu in turn, so that blocks 0 and 1 of a wave are g and u. With few tiles the
// sum is split, and k_gated_join adds its parts: 256 tokens, 4032 -> 83, 32 us in one piece
// and 12 split.
__global__ void __launch_bounds__(Ring128::kThreads) k_gated_ring(GatedArgs a) {
  __shared__ __attribute__((aligned(1024))) char b0[Ring128::kBufBytes];
  __shared__ __attribute__((aligned(1024))) char b1[Ring128::kBufBytes];
  __shared__ __attribute__((aligned(1024))) char b2[Ring128::kBufBytes];
  __shared__ __attribute__((aligned(1024))) char b3[Ring128::kBufBytes];
  const int tiles_m = cdiv(a.n_tok, 128), tiles_n = cdiv(a.ff, 64), tiles = tiles_m * tiles_n;
  const int sp = blockIdx.x / tiles, stages = int(a.d / 64);
  const int s0 = int(int64_t(stages) * sp / a.splits);
  const int s1 = int(int64_t(stages) * (sp + 1) / a.splits);
  int tm, tn;
  tile_of_block(blockIdx.x - sp * tiles, tiles, tiles_m, tiles_n, &tm, &tn);
  const int64_t m0 = int64_t(tm) * 128, n0 = int64_t(tn) * 64;
  OperandsR128 src;
#pragma unroll
  for (int i = 0; i < Ring128::kLoads; ++i) {
    const int r = t256_load_row(i), seg = t256_seg_bytes(i);
    src.a[i] = a.x + std::min(m0 + r, a.n_tok - 1) * (2 * a.ldx) + seg;
    const int64_t n = n0 + 16 * (r >> 5) + (r & 15);
    src.b[i] = ((r & 16) ? a.wu : a.wg) + std::min(n, a.ff - 1) * (2 * a.ldw) + seg;
  }
  AccR128<false> acc;
  r128_mainloop<Bf16Rows<false>>(acc, src, SumShape{0, 0, 0}, s1 - s0, b0, b1, b2, b3, [] {},
                                 SplitSteps{s0});

  const int col = 16 * ((threadIdx.x >> 6) & 3) + 4 * ((threadIdx.x >> 4) & 3);
#pragma unroll
  for (int mi = 0; mi < 4; ++mi) {
    const int row = t256_rows_row(0, mi);
    if (a.splits > 1) {
      float* p = a.part + size_t(blockIdx.x) * 16384 + row * 128 + col;
      *reinterpret_cast<f4*>(p) = acc.q[mi][0];
      *reinterpret_cast<f4*>(p + 64) = acc.q[mi][1];
      continue;
    }
    if (m0 + row >= a.n_tok) continue;
    float g[4], u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) g[e] = acc.q[mi][0][e], u[e] = acc.q[mi][1][e];
    gated_store<4>(a, m0 + row, n0 + col, g, u);
  }
}

// The outputs from the parts of their sums, in their order: 16 tokens of a tile a
// workgroup, four outputs a thread.
__global__ void __launch_bounds__(kThreads) k_gated_join(GatedArgs a) {
  const int tiles_m = cdiv(a.n_tok, 128), tiles_n = cdiv(a.ff, 64), tiles = tiles_m * tiles_n;
  const int tile = blockIdx.x >> 3;
  int tm, tn;
  tile_of_block(tile, tiles, tiles_m, tiles_n, &tm, &tn);
  const int row = (blockIdx.x & 7) * 16 + (threadIdx.x >> 4), col = 4 * (threadIdx.x & 15);
  const int64_t tok = int64_t(tm) * 128 + row;
  if (tok >= a.n_tok) return;
  const float* p = a.part + size_t(tile) * 16384 + row * 128 + col;
  f4 sg = {0.f, 0.f, 0.f, 0.f}, su = sg;
#pragma unroll 4
  for (int sp = 0; sp < a.splits; ++sp) {
    sg += *reinterpret_cast<const f4*>(p + size_t(sp) * tiles * 16384);
    su += *reinterpret_cast<const f4*>(p + size_t(sp) * tiles * 16384 + 64);
  }
  const float g[4] = {sg[0], sg[1], sg[2], sg[3]}, u[4] = {su[0], su[1], su[2], su[3]};
  gated_store<4>(a, tok, int64_t(tn) * 64 + col, g, u);
}

// ---------------------------------------------------------------------------
// Layout
// ---------------------------------------------------------------------------

// dst [rows_out][pitch] = src [rows][cols] with zeros around it; pitch is a multiple of 8.
struct PadRows {
  const bf16_t* src;
  int64_t ld, rows, cols, rows_out, pitch;
  bf16_t* dst;
  int64_t blocks() const { return src ? ceil_div(rows_out * (pitch / 8), kThreads) : 0; }
};
__device__ inline void pad_rows(const PadRows& a, int64_t block) {
  const int64_t i = block * kThreads + threadIdx.x;
  const int64_t per = a.pitch / 8, r = i / per, c = 8 * (i - r * per);
  if (r >= a.rows_out) return;
  Raw8<bf16_t> v;
  load_piece(v, a.src + r * a.ld, int(c), r < a.rows ? int(a.cols) : 0);
  *reinterpret_cast<u32x4*>(a.dst + r * a.pitch + c) = v.w;
}

// 64 x 64 values of a tile in LDS, rows 66 apart: the transposing reads below
// (eight rows of a column a lane) are free of bank conflicts.
constexpr int kTrPitch = 66;

__device__ inline void tr_put(uint16_t* tile, int r, int c, const u32x4& w) {
  uint32_t* p = reinterpret_cast<uint32_t*>(tile + r * kTrPitch + c);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = w[i];
}
__device__ inline u32x4 tr_get(const uint16_t* tile, int r, int c) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = tile[(r + 2 * i) * kTrPitch + c] | (uint32_t(tile[(r + 2 * i + 1) * kTrPitch + c]) << 16);
  return w;
}

// dst [cols][pitch] = src^T, src [rows][cols], with zeros from `rows` up to the
// next multiple of 64 of a dst row. pitch and dst are multiples of 8 values.
struct Transpose {
  const bf16_t* src;
  int64_t ld, rows, cols, pitch;
  bf16_t* dst;
  int64_t blocks() const { return src ? ceil_div(rows, 64) * ceil_div(cols, 64) : 0; }
};
__device__ inline void transpose_tile(const Transpose& a, int block, uint16_t* tile) {
  const int tiles_c = cdiv(a.cols, 64), tr = block / tiles_c;
  const int64_t r0 = int64_t(tr) * 64, c0 = int64_t(block - tr * tiles_c) * 64;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int p = threadIdx.x + k * kThreads, r = p >> 3, c = 8 * (p & 7);
    Raw8<bf16_t> v;
    load_piece(v, a.src + (r0 + r) * a.ld, int(c0) + c, r0 + r < a.rows ? int(a.cols) : 0);
    tr_put(tile, r, c, v.w);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int p = threadIdx.x + k * kThreads, c = p >> 3, r = 8 * (p & 7);
    if (c0 + c < a.cols)
      *reinterpret_cast<u32x4*>(a.dst + (c0 + c) * a.pitch + r0 + r) = tr_get(tile, r, c);
  }
}

struct GateGradArgs {
  const bf16_t *g, *u, *dh;
  int64_t ldg, ldu, lddh, n_tok, ff;
  // Upper parts, then lower ones:
  bf16_t* p;   // [n_tok][2][2 ffp]: dG, dU, each with zeros up to ffp, or NULL
  bf16_t* pt;  // [2 ff][2][tp]: their transpose with zeros from n_tok to tp, or NULL
  int64_t ffp, tp;
  int act;
  int64_t blocks() const { return ffp / 64 * (tp / 64); }
};

// Eight values rounded to bf16.
__device__ inline u32x4 rounded(const float (&v)[8]) {
  u32x4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
  return w;
}
// Eight values as sums of two bf16 parts: cut to bf16, and the rest rounded, off by at most 2^-16
// of the value. The parts have one sign and neither is 0 beside the other (a rest of 0 becomes
// 2^-20 of the value), so that products with an infinity are those of the value.
__device__ inline void two_parts(const float (&v)[8], u32x4* upper, u32x4* lower) {
  float hi[8], lo[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t bits = __float_as_uint(v[e]);
    const bool finite = (bits & 0x7F800000u) != 0x7F800000u;
    hi[e] = finite ? __uint_as_float(bits & 0xFFFF0000u) : v[e];
    lo[e] = finite ? v[e] - hi[e] : v[e];
    if (lo[e] == 0.f) lo[e] = hi[e] * 0x1p-20f;
  }
  *upper = rounded(hi);
  *lower = rounded(lo);
}

// 64 tokens x 64 values of dG and dU. Bound by HBM: 22 bytes a value, 270 us for 4096 x
// 14336.
__device__ inline void gate_grad_tile(const GateGradArgs& a, int block,
                                      uint16_t (&tile)[2][64 * kTrPitch]) {
  const int tiles_f = int(a.ffp / 64), tt = block / tiles_f;
  const int64_t t0 = int64_t(tt) * 64, f0 = int64_t(block - tt * tiles_f) * 64;
  u32x4 lg[2], lu[2];  // the lower parts
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = threadIdx.x + k * kThreads, r = i >> 3, c = 8 * (i & 7);
    const int64_t t = t0 + r, f = f0 + c;
    const int ff = t < a.n_tok ? int(a.ff) : 0;
    Raw8<bf16_t> rg, ru, rh;
    load_piece(rg, a.g + t * a.ldg, int(f), ff);
    load_piece(ru, a.u + t * a.ldu, int(f), ff);
    load_piece(rh, a.dh + t * a.lddh, int(f), ff);
    float g[8], u[8], dh[8], dg[8], du[8];
    values8(rg, g);
    values8(ru, u);
    values8(rh, dh);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float act, slope;
      gate_act_slope(a.act, g[e], &act, &slope);
      du[e] = dh[e] * act;
      dg[e] = dh[e] * u[e] * slope;
    }
    u32x4 hg, hu;
    two_parts(dg, &hg, &lg[k]);
    two_parts(du, &hu, &lu[k]);
    if (a.p && t < a.n_tok) {
      bf16_t* row = a.p + t * (4 * a.ffp) + f;
      *reinterpret_cast<u32x4*>(row) = hg;
      *reinterpret_cast<u32x4*>(row + a.ffp) = hu;
      *reinterpret_cast<u32x4*>(row + 2 * a.ffp) = lg[k];
      *reinterpret_cast<u32x4*>(row + 3 * a.ffp) = lu[k];
    }
    if (a.pt) {
      tr_put(tile[0], r, c, hg);
      tr_put(tile[1], r, c, hu);
    }
  }
  if (!a.pt) return;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = threadIdx.x + k * kThreads, c = i >> 3, r = 8 * (i & 7);
      if (f0 + c >= a.ff) continue;
      bf16_t* to = a.pt + (2 * (f0 + c) + part) * a.tp + t0 + r;
      *reinterpret_cast<u32x4*>(to) = tr_get(tile[0], r, c);
      *reinterpret_cast<u32x4*>(to + 2 * a.ff * a.tp) = tr_get(tile[1], r, c);
    }
    if (part == 1) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = threadIdx.x + k * kThreads, r = i >> 3, c = 8 * (i & 7);
      tr_put(tile[0], r, c, lg[k]);
      tr_put(tile[1], r, c, lu[k]);
    }
  }
}

// All that the products wait for, in one launch: P and P^T, X^T, and copies of weights
// whose rows do not suit them.
struct GradPrep {
  GateGradArgs gate;
  Transpose x;
  PadRows w[2];
  int64_t gate_blocks, x_blocks, w_blocks;
};
__global__ void __launch_bounds__(kThreads) k_gated_grad_prep(GradPrep a) {
  __shared__ uint16_t tile[2][64 * kTrPitch];
  int64_t b = blockIdx.x;
  if (b < a.gate_blocks) return gate_grad_tile(a.gate, int(b), tile);
  b -= a.gate_blocks;
  if (b < a.x_blocks) return transpose_tile(a.x, int(b), tile[0]);
  b -= a.x_blocks;
  const int k = b >= a.w_blocks;
  pad_rows(a.w[k], k ? b - a.w_blocks : b);
}

// The operands of the forward product whose rows do not suit wide loads.
struct ForwardPrep {
  PadRows m[3];
  int64_t first[3];  // block of the launch
};
__global__ void __launch_bounds__(kThreads) k_gated_prep(ForwardPrep a) {
  const int64_t b = blockIdx.x;
  const int k = b >= a.first[2] ? 2 : b >= a.first[1] ? 1 : 0;
  pad_rows(a.m[k], b - a.first[k]);
}

// ---------------------------------------------------------------------------
// The gradient's products, dX = P [Wg; Wu] and [dWg; dWu] = P^T X. A is P or P^T, both
// written by k_gated_grad_prep, with the contraction contiguous in its rows. dX takes the
// weights as they are, with the contraction along their rows, through the transposing
// LDS reads of gemm256.h (TB); dW takes X^T, transposed in memory.
// Measured at 4096 tokens, 4096 -> 14336, with one part of P, 962 GFLOP each: dX 701 us with TB, 670 and
// 114 for the transposed weights without; dW 767 us with TB, 670 and 14 for X^T without,
// and 840 us with both operands read through LDS that way (46 us less to write before).
// Both run in one launch, the longer sums first, so that the tiles of one fill the CUs
// that the other leaves. Long sums over few tiles are split, and joined by k_grad_join.
// ---------------------------------------------------------------------------

// Rows of the product below `part` go to y[0], those from `split` to split + part to
// y[1]. A zero in a mask makes the product's value +0 there. accumulate adds to what
// the output holds.
struct GradOut {
  void* y[2];
  const uint8_t* mask[2];
  int64_t split, part, ld, cols;
  int f32, accumulate;
};
struct GradArgs {
  const char *a, *b;
  int64_t pitch_a, pitch_b;  // bytes, multiples of 16
  int64_t rows, cols8;       // of the product; its columns rounded up to 8
  int64_t stages;            // of 64 values of the contraction, over both parts of A
  int64_t period;            // stages of one part: B is the same for each
  int64_t s1, jump;          // TB: from its stage s1 on B continues `jump` bytes further
  GradOut out;
};

template <bool TB>
struct GradSteps {
  int64_t pitch_b, jump;
  int period, s1, s0;  // s0: the workgroup's first stage
  __device__ inline int64_t a(int s) const { return int64_t(s0 + s) * 128; }
  __device__ inline int64_t b(int s) const {
    const int t = s0 + s < period ? s0 + s : s0 + s - period;
    return TB ? int64_t(t) * 64 * pitch_b + (t >= s1 ? jump : 0) : int64_t(t) * 128;
  }
};

template <typename T, int N>
__device__ inline void grad_put(T* y, float (&v)[N], int left, int accumulate) {
  if (accumulate) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 2)
          v[i] += bf16_low(y[i].bits);
        else
          v[i] += y[i];
      }
  }
  if constexpr (N == 8)
    store_upto8(y, v, left);
  else
    store_upto4(y, v, left);
}

// N consecutive values of a row of the product.
template <int N>
__device__ inline void grad_store(const GradOut& o, int64_t row, int64_t col, float (&v)[N]) {
  const int which = row >= o.split;
  const int64_t r = which ? row - o.split : row, at = r * o.ld + col;
  const int left = int(std::min<int64_t>(o.cols - col, N));
  if (r >= o.part || left <= 0) return;
  if (o.mask[which]) {
    const uint8_t* m = o.mask[which] + r * o.cols + col;
    uint8_t keep[N];
    if (left == N)
      __builtin_memcpy(keep, m, N);
    else
#pragma unroll
      for (int i = 0; i < N; ++i) keep[i] = i < left ? m[i] : 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!keep[i]) v[i] = 0.f;
  }
  if (o.f32)
    grad_put(static_cast<float*>(o.y[which]) + at, v, left, o.accumulate);
  else
    grad_put(static_cast<bf16_t*>(o.y[which]) + at, v, left, o.accumulate);
}
// The two blocks of a wave's 32 columns from c0 on, of one row.
template <bool TB>
__device__ inline void grad_store_blocks(const GradOut& o, int64_t row, int64_t c0,
                                         const f4 (&c)[2]) {
  const int q = (threadIdx.x >> 4) & 3;
  if (TB) {
#pragma unroll
    for (int ni = 0; ni < 2; ++ni) {
      float v[4] = {c[ni][0], c[ni][1], c[ni][2], c[ni][3]};
      grad_store<4>(o, row, c0 + 16 * ni + 4 * q, v);
    }
  } else {
    float v[8] = {c[0][0], c[0][1], c[0][2], c[0][3], c[1][0], c[1][1], c[1][2], c[1][3]};
    grad_store<8>(o, row, c0 + 8 * q, v);
  }
}

// This thread's first-stage address of load i of A's rows from r0 on, and of B's
// columns from c0 on.
__device__ inline const char* grad_a(const GradArgs& a, int64_t r0, int i) {
  return a.a + std::min(r0 + t256_load_row(i), a.rows - 1) * a.pitch_a + t256_seg_bytes(i);
}
template <bool TB>
__device__ inline const char* grad_b(const GradArgs& a, int64_t c0, int i) {
  if (TB)
    return a.b + tr_load_row(i) * a.pitch_b +
           2 * std::min<int64_t>(c0 + tr_seg_bytes() / 2, a.cols8 - 8);
  return a.b + std::min(c0 + t256_rows_source(t256_load_row(i)), a.out.cols - 1) * a.pitch_b +
         t256_seg_bytes(i);
}

struct GradPair {
  GradArgs a[2];         // dX, dW; of a product that is not wanted, no tiles
  int first;             // the product whose blocks come first, ..
  int64_t first_blocks;  // .. and how many: tiles, times the ranges of its sum
  int splits[2];
  float* part[2];        // [split][tile][side][side] where there are several
};

#define GRAD_LDS(name, bytes) __shared__ __attribute__((aligned(1024))) char name[bytes]

// What a block does: a product, its tile and stages [s0, s1) of the sum; to `part` where
// that is not NULL.
struct GradBlock {
  int which, tile, s0, s1;
  float* part;
};
__device__ inline GradBlock grad_block(const GradPair& p, int side) {
  GradBlock g;
  const bool head = blockIdx.x < p.first_blocks;
  g.which = head ? p.first : 1 - p.first;
  const int b = head ? int(blockIdx.x) : int(blockIdx.x - p.first_blocks);
  const GradArgs& a = p.a[g.which];
  const int tiles = cdiv(a.rows, side) * cdiv(a.out.cols, side), splits = p.splits[g.which];
  const int sp = b / tiles;
  g.tile = b - sp * tiles;
  g.s0 = int(a.stages * sp / splits);
  g.s1 = int(a.stages * (sp + 1) / splits);
  g.part = splits > 1 ? p.part[g.which] + size_t(b) * side * side : nullptr;
  return g;
}

// The two blocks of a wave's 32 columns of one row of a tile's partial sums.
template <bool TB>
__device__ inline void grad_part_blocks(float* row, const f4 (&c)[2]) {
  const int q = (threadIdx.x >> 4) & 3;
#pragma unroll
  for (int ni = 0; ni < 2; ++ni)
    *reinterpret_cast<f4*>(row + (TB ? 16 * ni + 4 * q : 8 * q + 4 * ni)) = c[ni];
}

template <bool TB>
__device__ inline void grad256_tile(const GradArgs& a, const GradBlock& g, char* l0, char* l1,
                                    char* l2, char* l3, char* l4, char* l5, char* l6, char* l7) {
  const int tiles_m = cdiv(a.rows, 256), tiles_n = cdiv(a.out.cols, 256);
  int tm, tn;
  tile_of_block(g.tile, tiles_m * tiles_n, tiles_m, tiles_n, &tm, &tn);
  const int64_t m0 = int64_t(tm) * 256, n0 = int64_t(tn) * 256;
  Operands256 src;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < Tile256::kHalfLoads; ++i) {
      src.a[h][i] = grad_a(a, m0 + 128 * h, i);
      src.b[h][i] = grad_b<TB>(a, n0 + 128 * h, i);
    }
  Acc256 acc;
  const GradSteps<TB> steps{a.pitch_b, a.jump, int(a.period), int(a.s1), g.s0};
  gemm256_mainloop<Bf16Rows<TB>>(acc, src, g.s1 - g.s0, l0, l1, l2, l3, l4, l5, l6, l7, [] {}, steps);
  const int wn = (threadIdx.x >> 6) & 3;
#pragma unroll
  for (int qa = 0; qa < 2; ++qa)
#pragma unroll
    for (int mi = 0; mi < 4; ++mi)
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) {
        const int row = t256_rows_row(qa, mi), col = 128 * qb + 32 * wn;
        if (g.part)
          grad_part_blocks<TB>(g.part + row * 256 + col, acc.q[qa][qb][mi]);
        else
          grad_store_blocks<TB>(a.out, m0 + row, n0 + col, acc.q[qa][qb][mi]);
      }
}

__global__ void __launch_bounds__(Tile256::kThreads) k_grad256(GradPair p) {
  GRAD_LDS(l0, Tile256::kHalfBytes);
  GRAD_LDS(l1, Tile256::kHalfBytes);
  GRAD_LDS(l2, Tile256::kHalfBytes);
  GRAD_LDS(l3, Tile256::kHalfBytes);
  GRAD_LDS(l4, Tile256::kHalfBytes);
  GRAD_LDS(l5, Tile256::kHalfBytes);
  GRAD_LDS(l6, Tile256::kHalfBytes);
  GRAD_LDS(l7, Tile256::kHalfBytes);
  const GradBlock g = grad_block(p, 256);
  if (g.which == 0)
    grad256_tile<true>(p.a[0], g, l0, l1, l2, l3, l4, l5, l6, l7);
  else
    grad256_tile<false>(p.a[1], g, l0, l1, l2, l3, l4, l5, l6, l7);
}

template <bool TB>
__device__ inline void grad_ring_tile(const GradArgs& a, const GradBlock& g, char* b0, char* b1,
                                      char* b2, char* b3) {
  const int tiles_m = cdiv(a.rows, 128), tiles_n = cdiv(a.out.cols, 128);
  int tm, tn;
  tile_of_block(g.tile, tiles_m * tiles_n, tiles_m, tiles_n, &tm, &tn);
  const int64_t m0 = int64_t(tm) * 128, n0 = int64_t(tn) * 128;
  OperandsR128 src;
#pragma unroll
  for (int i = 0; i < Ring128::kLoads; ++i) {
    src.a[i] = grad_a(a, m0, i);
    src.b[i] = grad_b<TB>(a, n0, i);
  }
  AccR128<false> acc;
  const GradSteps<TB> steps{a.pitch_b, a.jump, int(a.period), int(a.s1), g.s0};
  r128_mainloop<Bf16Rows<TB>>(acc, src, SumShape{0, 0, 0}, g.s1 - g.s0, b0, b1, b2, b3, [] {}, steps);
  const int wn = (threadIdx.x >> 6) & 3;
#pragma unroll
  for (int mi = 0; mi < 4; ++mi) {
    const int row = t256_rows_row(0, mi), col = 32 * wn;
    if (g.part)
      grad_part_blocks<TB>(g.part + row * 128 + col, acc.q[mi]);
    else
      grad_store_blocks<TB>(a.out, m0 + row, n0 + col, acc.q[mi]);
  }
}

__global__ void __launch_bounds__(Ring128::kThreads) k_grad_ring(GradPair p) {
  GRAD_LDS(b0, Ring128::kBufBytes);
  GRAD_LDS(b1, Ring128::kBufBytes);
  GRAD_LDS(b2, Ring128::kBufBytes);
  GRAD_LDS(b3, Ring128::kBufBytes);
  const GradBlock g = grad_block(p, 128);
  if (g.which == 0)
    grad_ring_tile<true>(p.a[0], g, b0, b1, b2, b3);
  else
    grad_ring_tile<false>(p.a[1], g, b0, b1, b2, b3);
}
#undef GRAD_LDS

// The outputs of split sums from the ranges' parts, in their order: four values a
// thread, 1024 of a tile a workgroup. blocks0 of them are dX's.
__global__ void __launch_bounds__(kThreads) k_grad_join(GradPair p, int side, int64_t blocks0) {
  const int which = blockIdx.x >= blocks0, per = side * side / 1024;
  const GradArgs& a = p.a[which];
  const int64_t b = which ? blockIdx.x - blocks0 : blockIdx.x;
  const int tiles_m = cdiv(a.rows, side), tiles_n = cdiv(a.out.cols, side);
  const int tiles = tiles_m * tiles_n, tile = int(b / per);
  int tm, tn;
  tile_of_block(tile, tiles, tiles_m, tiles_n, &tm, &tn);
  const int at = int(b % per) * 1024 + 4 * threadIdx.x;
  const int64_t row = int64_t(tm) * side + at / side, col = int64_t(tn) * side + at % side;
  if (row >= a.rows) return;
  f4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int sp = 0; sp < p.splits[which]; ++sp)
    sum += *reinterpret_cast<const f4*>(p.part[which] + (size_t(sp) * tiles + tile) * side * side + at);
  float v[4] = {sum[0], sum[1], sum[2], sum[3]};
  grad_store<4>(a.out, row, col, v);
}

// A product that is not wanted has no rows.
optima_status grad_products(GradPair& p, const GradPlan& plan, float* part, hipStream_t s) {
  const int64_t area = int64_t(plan.side) * plan.side;
  int64_t tiles[2], joined[2];
  for (int k = 0; k < 2; ++k) {
    tiles[k] = ceil_div(p.a[k].rows, plan.side) * ceil_div(p.a[k].out.cols, plan.side);
    p.splits[k] = plan.splits[k];
    p.part[k] = part;
    const bool split = plan.splits[k] > 1;
    if (split) part += tiles[k] * plan.splits[k] * area;
    joined[k] = split ? tiles[k] * (area / 1024) : 0;
  }
  p.first = ceil_div(p.a[0].stages, p.splits[0]) >= ceil_div(p.a[1].stages, p.splits[1]) ? 0 : 1;
  p.first_blocks = tiles[p.first] * p.splits[p.first];
  const dim3 grid(unsigned(tiles[0] * p.splits[0] + tiles[1] * p.splits[1]));
  if (plan.side == 256)
    hipLaunchKernelGGL(k_grad256, grid, dim3(Tile256::kThreads), 0, s, p);
  else
    hipLaunchKernelGGL(k_grad_ring, grid, dim3(Ring128::kThreads), 0, s, p);
  OPTIMA_LAUNCH_CHECK();
  if (joined[0] + joined[1]) {
    hipLaunchKernelGGL(k_grad_join, dim3(unsigned(joined[0] + joined[1])), dim3(kThreads), 0, s, p,
                       plan.side, joined[0]);
    OPTIMA_LAUNCH_CHECK();
  }
  return OPTIMA_OK;
}

struct GatedLayout {
  bf16_t *x, *wg, *wu;
  float* part;
};
GatedLayout carve_gated(void* ws, int64_t n_tok, int64_t d, int64_t ff, size_t* bytes) {
  Carver c(ws);
  GatedLayout l{};
  // Sized for tiles wherever more tokens may take them.
  if (!few_tokens(n_tok, d, ff)) {
    const int64_t dp = round_up(d, 64);
    l.x = c.take<bf16_t>(size_t(n_tok) * size_t(dp));
    if (dp != d) {
      l.wg = c.take<bf16_t>(size_t(ff) * size_t(dp));
      l.wu = c.take<bf16_t>(size_t(ff) * size_t(dp));
    }
    // Split sums: no more parts than stages.
    const int64_t parts = ceil_div(n_tok, 128) * ceil_div(ff, 64) * (dp / 64);
    l.part = c.take<float>(16384 * size_t(std::min(kPartTiles, parts)));
  }
  if (bytes) *bytes = c.bytes();
  return l;
}

struct GradLayout {
  bf16_t *p, *pt, *xt, *wg, *wu;
  float* part;
};
// Whether the weights' rows suit the products as they are: whole stages of rows,
// 16-byte pieces.
bool weights_suit(int64_t d, int64_t ff) { return ff % 64 == 0 && d % 8 == 0; }
GradLayout carve_grad(void* ws, int64_t n_tok, int64_t d, int64_t ff, size_t* bytes) {
  Carver c(ws);
  GradLayout l{};
  const size_t ffp = size_t(round_up(ff, 64)), tp = size_t(round_up(n_tok, 64));
  const size_t dp = size_t(round_up(d, 8));
  l.p = c.take<bf16_t>(size_t(n_tok) * 4 * ffp);
  l.pt = c.take<bf16_t>(4 * size_t(ff) * tp);
  l.xt = c.take<bf16_t>(size_t(d) * tp);
  if (!weights_suit(d, ff)) {
    l.wg = c.take<bf16_t>(ffp * dp);
    l.wu = c.take<bf16_t>(ffp * dp);
  }
  // Split sums: no more ranges than stages, of tiles of up to 256 x 256.
  const int64_t cols = 4 * ceil_div(d, 256);
  const int64_t parts = cols * (ceil_div(n_tok, 256) * int64_t(4 * ffp / 64) +
                                ceil_div(2 * ff, 256) * int64_t(2 * tp / 64));
  l.part = c.take<float>(16384 * size_t(std::min(kPartTiles, parts)));
  if (bytes) *bytes = c.bytes();
  return l;
}

}  // namespace

size_t gated_forward_workspace_bytes(int64_t n_tok, int64_t d, int64_t ff) {
  size_t b = 0;
  carve_gated(nullptr, n_tok, d, ff, &b);
  return b;
}

optima_status gated_forward(const void* X, int64_t ldx, int64_t n_tok, int64_t d, const void* Wg,
                            const void* Wu, int64_t ff, int act, void* H, int64_t ldh, int h_dtype,
                            void* G, int64_t ldg, void* U, int64_t ldu, void* ws, hipStream_t s) {
  GatedArgs a{static_cast<const char*>(X), static_cast<const char*>(Wg),
              static_cast<const char*>(Wu), H, static_cast<bf16_t*>(G), static_cast<bf16_t*>(U),
              n_tok, d, ff, ldx, d, ldh, ldg, ldu, h_dtype == OPTIMA_DTYPE_F32, act, 1, nullptr};
  if (few_tokens(n_tok, d, ff)) {
    // Half the outputs a workgroup where that makes the launch, or its reads of the
    // tokens are few: 4096 -> 2048, 16 tokens, 10.3 against 13.9 us, 4096 -> 14336, 4
    // tokens, 39.4 against 45.1; but 1024 -> 8192, 16 tokens, 11.9 against 8.7.
    if (n_tok <= 16 && (n_tok <= 8 || ff < 4096)) launch_few<1, 1>(a, s);
    else if (n_tok <= 16) launch_few<2, 1>(a, s);
    else if (n_tok <= 32) launch_few<2, 2>(a, s);
    else launch_few<2, 4>(a, s);
    OPTIMA_LAUNCH_CHECK();
    return OPTIMA_OK;
  }
  const GatedLayout l = carve_gated(ws, n_tok, d, ff, nullptr);
  const int64_t dp = round_up(d, 64);
  ForwardPrep prep{};
  int64_t blocks = 0;
  if (dp != d || !aligned16(X) || ldx % 8) {
    prep.m[0] = PadRows{static_cast<const bf16_t*>(X), ldx, n_tok, d, n_tok, dp, l.x};
    blocks = prep.m[0].blocks();
    a.x = reinterpret_cast<const char*>(l.x);
    a.ldx = dp;
  }
  prep.first[1] = prep.first[2] = blocks;
  if (dp != d) {
    prep.m[1] = PadRows{static_cast<const bf16_t*>(Wg), d, ff, d, ff, dp, l.wg};
    prep.m[2] = PadRows{static_cast<const bf16_t*>(Wu), d, ff, d, ff, dp, l.wu};
    prep.first[2] += prep.m[1].blocks();
    blocks = prep.first[2] + prep.m[2].blocks();
    a.wg = reinterpret_cast<const char*>(l.wg);
    a.wu = reinterpret_cast<const char*>(l.wu);
    a.ldw = dp;
  }
  if (blocks) {
    // Without weights to copy, no block is theirs.
    if (dp == d) prep.first[1] = prep.first[2] = INT64_MAX;
    hipLaunchKernelGGL(k_gated_prep, dim3(unsigned(blocks)), dim3(kThreads), 0, s, prep);
  }
  a.d = dp;
  OPTIMA_LAUNCH_CHECK();
  const GatedPlan plan = plan_gated(n_tok, d, ff);
  a.splits = plan.splits;
  a.part = l.part;
  if (plan.wide) {
    GatedArgs w = a;
    w.ff = plan.wide;
    const int64_t tiles = ceil_div(n_tok, 256) * ceil_div(w.ff, 128);
    hipLaunchKernelGGL(k_gated256, dim3(unsigned(tiles)), dim3(Tile256::kThreads), 0, s, w);
  }
  if (plan.wide < ff) {
    a.skip(plan.wide);
    const int64_t tiles = ceil_div(n_tok, 128) * ceil_div(a.ff, 64);
    hipLaunchKernelGGL(k_gated_ring, dim3(unsigned(tiles * plan.splits)), dim3(Ring128::kThreads), 0,
                       s, a);
    if (plan.splits > 1)
      hipLaunchKernelGGL(k_gated_join, dim3(unsigned(tiles * 8)), dim3(kThreads), 0, s, a);
  }
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

size_t gated_backward_workspace_bytes(int64_t n_tok, int64_t d, int64_t ff) {
  size_t b = 0;
  carve_grad(nullptr, n_tok, d, ff, &b);
  return b;
}

optima_status gated_backward(const void* X, int64_t ldx, int64_t n_tok, int64_t d, const void* Wg,
                             const void* Wu, int64_t ff, int act, const void* G, int64_t ldg,
                             const void* U, int64_t ldu, const void* dH, int64_t lddh, void* dX,
                             int64_t lddx, int dx_dtype, void* dWg, void* dWu, int dw_dtype,
                             const uint8_t* mask_g, const uint8_t* mask_u, int accumulate, void* ws,
                             hipStream_t s) {
  const GradLayout l = carve_grad(ws, n_tok, d, ff, nullptr);
  const int64_t ffp = round_up(ff, 64), tp = round_up(n_tok, 64), dp = round_up(d, 8);
  GradPrep prep{};
  GradPair pair{};
  const void *wg = Wg, *wu = Wu;
  if (dX && n_tok > 0) {
    if (!weights_suit(d, ff)) {
      prep.w[0] = PadRows{static_cast<const bf16_t*>(Wg), d, ff, d, ffp, dp, l.wg};
      prep.w[1] = PadRows{static_cast<const bf16_t*>(Wu), d, ff, d, ffp, dp, l.wu};
      wg = l.wg;
      wu = l.wu;
    }
    // P [dG dU] times Wg, then Wu.
    const int64_t s1 = ffp / 64;
    const int64_t jump = static_cast<const char*>(wu) - static_cast<const char*>(wg) - 2 * ffp * dp;
    pair.a[0] = GradArgs{reinterpret_cast<const char*>(l.p), static_cast<const char*>(wg),
                      8 * ffp, 2 * dp, n_tok, dp, 4 * s1, 2 * s1, s1, jump,
                      GradOut{{dX, nullptr}, {nullptr, nullptr}, INT64_MAX, n_tok, lddx, d,
                              dx_dtype == OPTIMA_DTYPE_F32, 0}};
  }
  if (dWg) {
    // No tokens: no stages, and the products are zero.
    if (n_tok > 0) prep.x = Transpose{static_cast<const bf16_t*>(X), ldx, n_tok, d, tp, l.xt};
    pair.a[1] = GradArgs{reinterpret_cast<const char*>(l.pt), reinterpret_cast<const char*>(l.xt),
                      4 * tp, 2 * tp, 2 * ff, dp, tp / 32, tp / 64, 0, 0,
                      GradOut{{dWg, dWu}, {mask_g, mask_u}, ff, ff, d, d,
                              dw_dtype == OPTIMA_DTYPE_F32, accumulate}};
  }
  if (n_tok > 0) {
    prep.gate = GateGradArgs{static_cast<const bf16_t*>(G), static_cast<const bf16_t*>(U),
                             static_cast<const bf16_t*>(dH), ldg, ldu, lddh, n_tok, ff,
                             dX ? l.p : nullptr, dWg ? l.pt : nullptr, ffp, tp, act};
    prep.gate_blocks = prep.gate.blocks();
    prep.x_blocks = prep.x.blocks();
    prep.w_blocks = prep.w[0].blocks();
    const int64_t blocks = prep.gate_blocks + prep.x_blocks + 2 * prep.w_blocks;
    hipLaunchKernelGGL(k_gated_grad_prep, dim3(unsigned(blocks)), dim3(kThreads), 0, s, prep);
    OPTIMA_LAUNCH_CHECK();
  }
  if (n_tok == 0 && !dWg) return OPTIMA_OK;
  return grad_products(pair, plan_grad(n_tok, d, ff), l.part, s);
}

}  // namespace optima
