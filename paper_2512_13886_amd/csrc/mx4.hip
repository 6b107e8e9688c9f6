// Microscaled 4-bit floating point: packing rows, the values they stand for, and products
// Y = X W^T with packed weights, of 16-bit tokens or packed ones.
//
// A block of 32 values v has the scale 2^(e - 2), e = floor(log2 max |v|), kept as a biased
// exponent in a byte, and codes of v / scale: sign, two bits of exponent and one of mantissa
// (0, 0.5, 1, 1.5, 2, 3, 4, 6), nearest even, at most 6. A zero has code 0, so that pruned
// entries stay exactly zero.
//
// Rows of codes are padded to whole 256 values (128 bytes) and lie in the order of the values:
// in the products lane (b, i) of a wave holds the 16 bytes of block b of 128 values of row i,
// which is an operand of the 16x16x128 block-scaled MFMA as it lies, and four of the 16x16x32
// bf16 one. The scales of four such 128s lie together for each b: a lane's four are one dword,
// and the MFMA picks the byte, so that scales cost no instructions.
//   packed tokens: products of codes and scales are exact, the sum is the MFMA's fp32.
//   16-bit tokens: codes times scale are exact in bf16 (one instruction for two).
#include <type_traits>

#include "common.h"
#include "vec8.h"
#include "mx4_plan.h"
#include "mx4_tile.h"

namespace optima {
namespace {

constexpr int kChunk = 128;  // values of an operand
constexpr int kChunkBytes = 64;

using mx4::i8x32;

int64_t row_bytes(int64_t d) { return ceil_div(d, 256) * 128; }
int64_t scale_bytes(int64_t d) { return ceil_div(d, 512) * 16; }

// ---------------------------------------------------------------------------
// Packing, and back
// ---------------------------------------------------------------------------

// Largest of m over the four lanes of a block.
__device__ inline uint32_t quad_max(uint32_t m) {
  m = max(m, uint32_t(__builtin_amdgcn_mov_dpp(int(m), 0xB1, 0xF, 0xF, true)));  // lanes 1 0 3 2
  return max(m, uint32_t(__builtin_amdgcn_mov_dpp(int(m), 0x4E, 0xF, 0xF, true)));  // 2 3 0 1
}

// Eight values to codes, by the four lanes of a block; s: the block's scale.
__device__ inline uint32_t codes8(const float (&v)[8], uint32_t& s) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  m = quad_max(m);
  // The exponent's field of the largest less 2, within 0 .. 252; 255 with infinity or NaN, whose
  // block has codes 0: NaN as values.
  const uint32_t top = m >> 23;
  const bool fine = top < 255u;
  s = fine ? max(top, 2u) - 2u : 255u;
  const float inv = __uint_as_float((254u - s) << 23);  // 2^(127 - s): the quotients are exact
  uint32_t q = 0;
  if (fine) {
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0] * inv, v[1] * inv, 1.f, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2] * inv, v[3] * inv, 1.f, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4] * inv, v[5] * inv, 1.f, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6] * inv, v[7] * inv, 1.f, 3);
  }
  return q;
}

// Thirty-two lanes for H pieces of 256 values, eight codes of each a lane: a block's largest takes two
// exchanges of neighbouring lanes, and its scale, a power of two, leaves the quotients exact, so that
// one rounding is all there is. Bound by HBM: 14336 x 4096 in 52 us from fp32, 5.1 TB/s, and 28 from bf16,
// 5.3 TB/s. Two pieces, for bf16 rows of more than one: 8192 x 4096 19.8 to 17.9 us; but fp32 at
// 14336 x 4096 51.9 to 52.9, and 100000 x 64 13.9 to 17.6.
template <typename T, int H>
__global__ void __launch_bounds__(kThreads) k_mx4_pack(const T* X, int64_t ldx, uint32_t total,
                                                       uint32_t each, int d, uint8_t* Q, int row,
                                                       uint8_t* scales, int srow) {
  const uint32_t idx = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const bool live = idx < total;  // of all 32 lanes
  const int64_t n = live ? idx / each : 0u;
  const int at = live ? int(idx % each) * H : 0, pieces = row / 128;
  const int i = threadIdx.x & 31;
  Raw8<T> raw[H];
#pragma unroll
  for (int h = 0; h < H; ++h) load_piece(raw[h], X + n * ldx, 256 * (at + h) + 8 * i, live ? d : 0);
  uint32_t q[H], sc = 0;
#pragma unroll
  for (int h = 0; h < H; ++h) {
    float v[8];
    values8(raw[h], v);
    uint32_t s;
    q[h] = codes8(v, s);
    // Lanes 0 .. 15 hold the first 128 values, 16 .. 31 the second, whose scales are neighbours. A
    // piece past the row's has the padding's scales of 0.
    s |= uint32_t(__shfl_xor(int(s), 16, 64)) << 8;
    if (at + h < pieces) sc |= s << (16 * h);
  }
  if (!live) return;
#pragma unroll
  for (int h = 0; h < H; ++h)
    if (at + h < pieces) *reinterpret_cast<uint32_t*>(Q + n * row + (at + h) * 128 + 4 * i) = q[h];
  if (i < 16 && (i & 3) == 0) {
    uint8_t* to = scales + n * srow + 16 * (at >> 1) + i + 2 * (at & 1);
    if (H == 2 || ((at & 1) == 0 && at + 1 == pieces))  // with the padding's
      *reinterpret_cast<uint32_t*>(to) = sc;
    else
      *reinterpret_cast<uint16_t*>(to) = uint16_t(sc);
  }
}
template <typename T, int H>
void launch_pack(const void* X, int64_t ldx, int64_t n, int64_t d, void* Q, void* scales, hipStream_t s) {
  const uint32_t each = uint32_t(ceil_div(d, 256 * H)), total = uint32_t(n * each);  // below 2^27
  hipLaunchKernelGGL((k_mx4_pack<T, H>), dim3(unsigned(ceil_div(total, kThreads / 32))), dim3(kThreads), 0,
                     s, static_cast<const T*>(X), ldx, total, each, int(d), static_cast<uint8_t*>(Q),
                     int(row_bytes(d)), static_cast<uint8_t*>(scales), int(scale_bytes(d)));
}

// The values, exact in either type. Bound by HBM's writes: 14336 x 4096 to bf16 in 23 us, 6.5 TB/s with
// the codes partly in a cache.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_mx4_unpack(const uint8_t* Q, const uint8_t* scales,
                                                         int srow, uint32_t total, uint32_t pieces,
                                                         int d, T* Y, int64_t ldy) {
  const uint32_t idx = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (idx >= total) return;
  const int64_t n = idx / pieces;
  const int h = int(idx % pieces);
  const int i = threadIdx.x & 31, k = 256 * h + 8 * i;
  if (k >= d) return;
  const uint32_t q = *reinterpret_cast<const uint32_t*>(Q + (n * pieces + h) * 128 + 4 * i);
  const uint32_t s = scales[n * srow + 16 * (h >> 1) + (i & 12) + 2 * (h & 1) + (i >> 4)];
  const float scale = __uint_as_float(s << 23);  // its exponent alone counts
  const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 0);
  const f2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 1);
  const f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 2);
  const f2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, scale, 3);
  const float v[8] = {a[0], a[1], b[0], b[1], c[0], c[1], e[0], e[1]};
  store_upto8(Y + n * ldy + k, v, d - k);
}

// ---------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------

struct Mx4Args {
  const void* x;      // bf16 [n_tok][ldx], or codes
  const uint8_t* xs;  // scales of codes
  const uint8_t *q, *s;
  void* y;
  f4* part;
  int64_t n_tok, d_out, ldx, ldy;
  int d, chunks, row, srow, y_f32;  // chunks of 128 values; bytes of a row of codes, of scales
};

// Eight codes of a block times its scale (a float of which the exponent counts).
__device__ inline bf16x8 weights8(uint32_t w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Byte U of a lane's scales as such a float.
template <int U>
__device__ inline float scale_at(uint32_t s) {
  return __uint_as_float(((s >> (8 * U)) & 255u) << 23);
}
// c += W X^T for 128 values of 16 rows and 16 packed tokens; byte U of the lanes' scales.
template <int U>
__device__ inline void mfma_mx4(f4& c, const u32x4& w, uint32_t sw, const u32x4& x, uint32_t sx) {
  const i8x32 a = {int(w[0]), int(w[1]), int(w[2]), int(w[3]), 0, 0, 0, 0};
  const i8x32 b = {int(x[0]), int(x[1]), int(x[2]), int(x[3]), 0, 0, 0, 0};
  c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, U, int(sw), U, int(sx));
}
// The same with 16-bit tokens: x[j] holds values 8 j .. of the lane's block.
template <int U>
__device__ inline void mfma_bf16(f4& c, const u32x4& w, uint32_t sw, const bf16x8 (&x)[4]) {
  const float scale = scale_at<U>(sw);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(weights8(w[j], scale), x[j], c, 0, 0, 0);
}

// Values k .. k + 7 of rows of d 16-bit values, zeros past their end: loaded as they lie or, of a row's
// last piece, from eight values before its end, without a branch, so that the loads of several rows
// go out together; and moved afterwards. (In load_piece each row's end waits for its own load: 13
// tokens, 1001 -> 2731, 7.1 us and 5.7.)
struct TokenPiece {
  int at, shift, d;
  __device__ inline TokenPiece(int k, int d) : at(max(min(k, d - 8), 0)), shift(k - at), d(d) {}
  __device__ inline u32x4 load(const bf16_t* row) const {
    Raw8<bf16_t> r;
    if (d >= 8)
      load8(r, row + at);
    else
      load_some(r, row, d);
    return r.w;
  }
  __device__ inline u32x4 moved(const u32x4& v) const {
    if (shift >= 8) return u32x4{0, 0, 0, 0};
    Raw8<bf16_t> r{v};
    shift_down(r, shift);
    return r.w;
  }
};

// 16 tokens from tok0 on and 32 outputs from n0 on, of which lane (b, i) has those from 8 b on of token i.
// They are stored by lane 4 i + b, so that neighbouring lanes store neighbouring bytes.
__device__ inline void store_block(const Mx4Args& a, int64_t tok0, int64_t n0, const f4& v, const f4& w) {
  const int lane = threadIdx.x & 63, from = ((lane & 3) * 16 + (lane >> 2)) * 4;
  const int64_t tok = tok0 + (lane >> 2), n = n0 + 8 * (lane & 3);
  auto moved = [from](uint32_t u) { return uint32_t(__builtin_amdgcn_ds_bpermute(from, int(u))); };
  const int left = int(std::min<int64_t>(a.d_out - n, 8));
  const bool live = tok < a.n_tok && left > 0;
  const int64_t at = tok * a.ldy + n;
  if (a.y_f32) {
    float u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = __uint_as_float(moved(__float_as_uint(e < 4 ? v[e] : w[e - 4])));
    if (live) store_upto8(static_cast<float*>(a.y) + at, u, left);
  } else {
    Raw8<bf16_t> r{u32x4{moved(pack_bf16(v[0], v[1])), moved(pack_bf16(v[2], v[3])),
                         moved(pack_bf16(w[0], w[1])), moved(pack_bf16(w[2], w[3]))}};
    bf16_t* y = static_cast<bf16_t*>(a.y) + at;
    if (!live) return;
    if (left == 8)
      *reinterpret_cast<u32x4_2*>(y) = r.w;
    else
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) y[e].bits = uint16_t(r.w[e >> 1] >> (16 * (e & 1)));
  }
}

constexpr int kBatch = 4;                 // chunks that a wave's loads go out together for
constexpr int kBatchK = kBatch * kChunk;  // 512 values, whose scales are one dword a lane

// What lanes of a wave wrote to LDS before is there for its other lanes after. A wave's LDS
// accesses are served in order, so that this only keeps the compiler from moving them.
__device__ inline void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Up to 16 tokens (of packed ones blockIdx.y's). A workgroup takes 16 outputs, its waves every waves-th
// batch of 512 values, and the waves' sums are joined in LDS in their order. Bound by the latency of one or two batches of
// loads a wave, which nothing hides: one 16-bit token, 14336 -> 4096 (31 MB) 8.2 us, 3.8 TB/s, with
// weights that no cache holds 9.5. Twice the outputs a workgroup took 12.8, codes loaded a batch ahead 12.2.
static_assert(kMx4FewPitch == kBatchK * 2 + 64, "a token's batch, with 64 bytes between rows");

// A batch's codes and scales of row n: zeros for chunks past the row's end.
__device__ inline void load_codes(u32x4 (&w)[kBatch], uint32_t& s, const uint8_t* q,
                                  const uint8_t* sc, const Mx4Args& a, int64_t n, int batch, int b) {
  const uint8_t* p = q + n * a.row + b * 16;
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const int c = batch * kBatch + u;
    w[u] = u32x4{0, 0, 0, 0};
    if (c < a.chunks) w[u] = *reinterpret_cast<const u32x4*>(p + c * kChunkBytes);
  }
  s = *reinterpret_cast<const uint32_t*>(sc + n * a.srow + batch * 16 + 4 * b);
}

// ROWS: tokens that a lane loads values of together; RB: blocks of 16 outputs; RAGGED: 16-bit tokens of
// a width that is no multiple of 8.
template <bool PACKED, int ROWS, int RB, bool RAGGED>
__global__ void __launch_bounds__(64 * kMx4FewWaves) k_mx4_few(Mx4Args a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  float* part = reinterpret_cast<float*>(lds);  // [wave][lane][4], at the end
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t t0 = PACKED ? int64_t(blockIdx.y) * kMx4Few : 0;
  const int b = lane >> 4, i = lane & 15, tokens = int(std::min<int64_t>(a.n_tok - t0, kMx4Few));
  const int64_t n0 = int64_t(blockIdx.x) * 16 * RB;
  const int tok = std::min(i, tokens - 1), batches = (a.chunks + kBatch - 1) / kBatch;
  const bf16_t* x = static_cast<const bf16_t*>(a.x);
  char* mine = lds + wave * tokens * kMx4FewPitch;
  f4 sum[RB];
#pragma unroll
  for (int m = 0; m < RB; ++m) sum[m] = f4{0.f, 0.f, 0.f, 0.f};
  for (int batch = wave; batch < batches; batch += waves) {
    u32x4 w[RB][kBatch];
    uint32_t s[RB];
#pragma unroll
    for (int m = 0; m < RB; ++m)
      load_codes(w[m], s[m], a.q, a.s, a, std::min(n0 + 16 * m + i, a.d_out - 1), batch, b);
    if constexpr (PACKED) {
      u32x4 f[kBatch];
      uint32_t sx;
      load_codes(f, sx, static_cast<const uint8_t*>(a.x), a.xs, a, t0 + tok, batch, b);
#pragma unroll
      for (int m = 0; m < RB; ++m) {
        mfma_mx4<0>(sum[m], w[m][0], s[m], f[0], sx);
        mfma_mx4<1>(sum[m], w[m][1], s[m], f[1], sx);
        mfma_mx4<2>(sum[m], w[m][2], s[m], f[2], sx);
        mfma_mx4<3>(sum[m], w[m][3], s[m], f[3], sx);
      }
    } else {
      // The tokens' values come through LDS: the operands would read each 16 times over.
      const TokenPiece piece(batch * kBatchK + 8 * lane, a.d);
      for (int r0 = 0; r0 < tokens; r0 += ROWS) {
        u32x4 v[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
          if (r0 + r < tokens) {
            const bf16_t* row = x + (r0 + r) * a.ldx;
            if constexpr (RAGGED)
              v[r] = piece.load(row);
            else
              v[r] = piece.shift ? u32x4{0, 0, 0, 0} : *reinterpret_cast<const u32x4_2*>(row + piece.at);
          }
        if (RAGGED && piece.shift)
#pragma unroll
          for (int r = 0; r < ROWS; ++r) v[r] = piece.moved(v[r]);
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
          if (r0 + r < tokens)
            *reinterpret_cast<u32x4*>(mine + (r0 + r) * kMx4FewPitch + 16 * lane) = v[r];
      }
      wave_exchange();
      auto chunk = [&](auto u) {
        constexpr int U = decltype(u)::value;
        bf16x8 f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          f[j] = *reinterpret_cast<const bf16x8*>(mine + tok * kMx4FewPitch +
                                                  (U * kChunk + 32 * b + 8 * j) * 2);
#pragma unroll
        for (int m = 0; m < RB; ++m) mfma_bf16<U>(sum[m], w[m][U], s[m], f);
      };
      chunk(std::integral_constant<int, 0>());
      chunk(std::integral_constant<int, 1>());
      chunk(std::integral_constant<int, 2>());
      chunk(std::integral_constant<int, 3>());
      wave_exchange();
    }
  }
  __syncthreads();  // the staged values' place
#pragma unroll
  for (int m = 0; m < RB; ++m) *reinterpret_cast<f4*>(part + ((wave * RB + m) * 64 + lane) * 4) = sum[m];
  __syncthreads();
  for (int o = threadIdx.x; o < 256 * RB; o += blockDim.x) {
    const int nn = o % (16 * RB), t = o / (16 * RB);
    if (t >= tokens || n0 + nn >= a.d_out) continue;
    const float* p = part + ((nn >> 4) * 64 + (nn >> 2 & 3) * 16 + t) * 4 + (nn & 3);
    float v = 0.f;
    for (int w = 0; w < waves; ++w) v += p[w * RB * 256];
    const int64_t at = (t0 + t) * a.ldy + n0 + nn;
    if (a.y_f32)
      static_cast<float*>(a.y)[at] = v;
    else
      store1(static_cast<bf16_t*>(a.y) + at, v);
  }
}

// More 16-bit tokens, 16 NT at a time. The tokens' values of a batch go through LDS, two batches in
// turn, for all waves of a workgroup; a wave takes 32 outputs, whose codes it loads a batch ahead, in
// the order in which a lane's sums of both blocks are eight consecutive outputs (stored as they
// came out of the MFMA, four by four, 8192 tokens took 1126 us in place of 1083). With few outputs the
// batches are split over blockIdx.y, and k_mx4_join adds the parts. 64 tokens, 4096 -> 128000 (279 MB) 105
// us, 4096 -> 14336 24 us, where packed tokens take 54 and 12; 8192 tokens, 4096 -> 14336 0.89 PFLOP/s. Bound
// by waits: two waves a SIMD with a barrier a batch spend 39 to 46 % of their time on loads, LDS and
// barriers, while the matrix instructions are busy for 28, 12 and 37 % of it, all vector instructions (the
// conversion of codes, which every 64 tokens repeat, is a part) for 21, 14 and 27, and LDS for 32, 13 and 42.
constexpr int kSlabWaves = kMx4SlabRows / 32;

template <int NT>
__global__ void __launch_bounds__(64 * kSlabWaves) k_mx4_slab(Mx4Args a) {
  constexpr int kTok = 16 * NT, kXBytes = kBatchK * 2, kPitch = kXBytes + 16;
  constexpr int kPieces = kXBytes / 16;                      // of 16 bytes, of a token's batch
  constexpr int kEach = (kTok * kPieces + 511) / 512;        // that a thread brings
  __shared__ __attribute__((aligned(16))) char xl[2][kTok * kPitch];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = lane >> 4, i = lane & 15;
  const int64_t t0 = int64_t(blockIdx.z) * kTok;
  const int tokens = int(std::min<int64_t>(a.n_tok - t0, kTok));
  const int64_t n0 = int64_t(blockIdx.x) * kMx4SlabRows + wave * 32;
  int64_t n[2];
#pragma unroll
  for (int m = 0; m < 2; ++m) n[m] = std::min(n0 + 8 * (i >> 2) + 4 * m + (i & 3), a.d_out - 1);
  const int batches = (a.chunks + kBatch - 1) / kBatch;
  const int b0 = int(int64_t(batches) * blockIdx.y / gridDim.y);
  const int b1 = int(int64_t(batches) * (blockIdx.y + 1) / gridDim.y);

  u32x4 xv[kEach];
  auto fetch_x = [&](int batch) {
    static_assert(512 % kPieces == 0, "one place in all rows of a thread");
    const TokenPiece piece(batch * kBatchK + 8 * (int(threadIdx.x) % kPieces), a.d);
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
      const int64_t t = t0 + std::min(int(threadIdx.x + 512 * r) / kPieces, tokens - 1);
      xv[r] = piece.load(static_cast<const bf16_t*>(a.x) + t * a.ldx);
    }
  };
  auto put_x = [&](int to, int batch) {
    const TokenPiece piece(batch * kBatchK + 8 * (int(threadIdx.x) % kPieces), a.d);
    if (piece.shift)
#pragma unroll
      for (int r = 0; r < kEach; ++r) xv[r] = piece.moved(xv[r]);
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
      const int at = threadIdx.x + 512 * r;
      if (kTok * kPieces % 512 == 0 || at < kTok * kPieces)
        *reinterpret_cast<u32x4*>(xl[to] + at / kPieces * kPitch + at % kPieces * 16) = xv[r];
    }
  };
  u32x4 w[2][kBatch];
  uint32_t s[2];
  auto fetch_w = [&](int batch) {
#pragma unroll
    for (int m = 0; m < 2; ++m) load_codes(w[m], s[m], a.q, a.s, a, n[m], batch, b);
  };

  f4 sum[2][NT];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[m][t] = f4{0.f, 0.f, 0.f, 0.f};
  if (b0 < b1) {
    fetch_x(b0);
    fetch_w(b0);
    put_x(0, b0);
  }
  __syncthreads();
  for (int batch = b0; batch < b1; ++batch) {
    const int cur = (batch - b0) & 1;
    u32x4 wc[2][kBatch];
    uint32_t sc[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) wc[m][u] = w[m][u];
      sc[m] = s[m];
    }
    if (batch + 1 < b1) {
      fetch_x(batch + 1);
      fetch_w(batch + 1);
    }
    const char* xc = xl[cur] + i * kPitch;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (batch * kBatch + u >= a.chunks) break;  // past the row's end
      bf16x8 v[2][4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float scale = __uint_as_float(((sc[m] >> (8 * u)) & 255u) << 23);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[m][j] = weights8(wc[m][u][j], scale);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8 f =
              *reinterpret_cast<const bf16x8*>(xc + 16 * t * kPitch + (u * kChunk + 32 * b + 8 * j) * 2);
#pragma unroll
          for (int m = 0; m < 2; ++m)
            sum[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[m][j], f, sum[m][t], 0, 0, 0);
        }
    }
    if (batch + 1 < b1) put_x(cur ^ 1, batch + 1);
    __syncthreads();
  }
  if (gridDim.y > 1) {  // [split][64 tokens][workgroup][wave][row block][token block][lane]
    const size_t wg = (size_t(blockIdx.y) * gridDim.z + blockIdx.z) * gridDim.x + blockIdx.x;
    f4* part = a.part + (wg * kSlabWaves + wave) * 2 * NT * 64;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t) part[(m * NT + t) * 64 + lane] = sum[m][t];
    return;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) store_block(a, t0 + 16 * t, n0, sum[0][t], sum[1][t]);
}

// The parts of the outputs, added in their order. blocks: 16 x 32 outputs, of all splits' one.
template <int NT>
__global__ void __launch_bounds__(kThreads) k_mx4_join(Mx4Args a, int splits, int64_t blocks,
                                                       int64_t per) {
  const int lane = threadIdx.x & 63;
  const int64_t at = int64_t(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (at >= blocks) return;
  const int64_t z = at / per, in = at - z * per;  // of 16 NT tokens
  const int64_t wave = at / NT;
  const int t = int(in % NT);
  const f4* part = a.part + (wave * 2 * NT + t) * 64 + lane;
  f4 c[2] = {};
#pragma unroll 8
  for (int sp = 0; sp < splits; ++sp)
#pragma unroll
    for (int m = 0; m < 2; ++m) c[m] += part[(sp * blocks * 2 + m * NT) * 64];
  store_block(a, z * 16 * NT + 16 * t, in / NT * 32, c[0], c[1]);
}

template <int NT>
void launch_slab(const Mx4Args& a, int splits, hipStream_t s) {
  const unsigned wgs = unsigned(ceil_div(a.d_out, kMx4SlabRows));
  const unsigned tiles = unsigned(ceil_div(a.n_tok, 16 * NT));
  hipLaunchKernelGGL((k_mx4_slab<NT>), dim3(wgs, unsigned(splits), tiles),
                     dim3(64 * kSlabWaves), 0, s, a);
  if (splits > 1) {
    const int64_t per = int64_t(wgs) * kSlabWaves * NT, blocks = per * tiles;
    hipLaunchKernelGGL((k_mx4_join<NT>), dim3(unsigned(ceil_div(blocks, kThreads / 64))),
                       dim3(kThreads), 0, s, a, splits, blocks, per);
  }
}

// ---------------------------------------------------------------------------
// Many packed tokens
// ---------------------------------------------------------------------------

// A 256 x 256 tile of outputs, or with gridDim.y > 1 a range of its sum's pairs of stages.
__global__ void __launch_bounds__(Tile256::kThreads) k_mx4_tile(Mx4Args a) {
  __shared__ __attribute__((aligned(1024))) char l0[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l1[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l2[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l3[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l4[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l5[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l6[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char l7[Tile256::kHalfBytes];
  __shared__ __attribute__((aligned(1024))) char s0[mx4::kScaleBytes];
  __shared__ __attribute__((aligned(1024))) char s1[mx4::kScaleBytes];
  const int tiles_m = int((a.n_tok + 255) / 256), tiles_n = int((a.d_out + 255) / 256);
  int tm, tn;
  tile_of_block(blockIdx.x, tiles_m * tiles_n, tiles_m, tiles_n, &tm, &tn);
  const int64_t m0 = int64_t(tm) * 256, n0 = int64_t(tn) * 256;
  const int stages = a.row / Tile256::kSRB, pairs = (stages + 1) / 2;
  const int p0 = int(int64_t(pairs) * blockIdx.y / gridDim.y);
  const int p1 = int(int64_t(pairs) * (blockIdx.y + 1) / gridDim.y);
  Operands256 src;
#pragma unroll
  for (int i = 0; i < Tile256::kHalfLoads; ++i) {
    const int r = t256_load_row(i);
    const int64_t at = int64_t(2 * p0) * Tile256::kSRB + t256_seg_bytes(i);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      src.a[h][i] = static_cast<const char*>(a.x) + std::min(m0 + 128 * h + r, a.n_tok - 1) * a.row + at;
      src.b[h][i] = reinterpret_cast<const char*>(a.q) +
                    std::min(n0 + 128 * h + t256_rows_source(r), a.d_out - 1) * a.row + at;
    }
  }
  const int r = threadIdx.x & 255;
  const char* scales = reinterpret_cast<const char*>(
      threadIdx.x < 256 ? a.xs + std::min(m0 + r, a.n_tok - 1) * a.srow
                        : a.s + std::min(n0 + (r & 128) + t256_rows_source(r & 127), a.d_out - 1) * a.srow);
  Acc256 acc;
  mx4::mainloop(acc, src, scales + 16 * p0, std::min(2 * p1, stages) - 2 * p0, l0, l1, l2, l3, l4, l5,
                l6, l7, s0, s1);
  const int wm = threadIdx.x >> 8, wn = (threadIdx.x >> 6) & 3;
  f4* part = gridDim.y > 1
                 ? a.part + ((size_t(blockIdx.y) * gridDim.x + blockIdx.x) * Tile256::kWaves +
                             (threadIdx.x >> 6)) * 32 * 64 + (threadIdx.x & 63)
                 : nullptr;
#pragma unroll
  for (int qa = 0; qa < 2; ++qa)
#pragma unroll
    for (int mi = 0; mi < 4; ++mi)
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) {
        const f4 *c = acc.q[qa][qb][mi];
        if (part) {
          part[((qa * 4 + mi) * 4 + 2 * qb) * 64] = c[0];
          part[((qa * 4 + mi) * 4 + 2 * qb + 1) * 64] = c[1];
        } else {
          store_block(a, m0 + qa * 128 + wm * 64 + mi * 16, n0 + qb * 128 + wn * 32, c[0], c[1]);
        }
      }
}

// The parts of the tiles' outputs, added in their order: 16 rows of a wave's a wave.
__global__ void __launch_bounds__(kThreads) k_mx4_tile_join(Mx4Args a, int splits, int tiles) {
  const int lane = threadIdx.x & 63;
  const int64_t at = int64_t(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (at >= int64_t(tiles) * 64) return;
  const int tile = int(at >> 6), wave = int(at >> 3) & 7, qa = int(at >> 2) & 1, mi = int(at & 3);
  const f4* part = a.part + at * 4 * 64 + lane;
  const size_t step = size_t(tiles) * 64 * 4 * 64;
  f4 c[4] = {};
#pragma unroll 4
  for (int sp = 0; sp < splits; ++sp)
#pragma unroll
    for (int q = 0; q < 4; ++q) c[q] += part[sp * step + q * 64];
  const int tiles_m = int((a.n_tok + 255) / 256);
  int tm, tn;
  tile_of_block(tile, tiles, tiles_m, tiles / tiles_m, &tm, &tn);
  const int64_t tok = int64_t(tm) * 256 + qa * 128 + (wave >> 2) * 64 + mi * 16;
  const int64_t n = int64_t(tn) * 256 + (wave & 3) * 32;
  store_block(a, tok, n, c[0], c[1]);
  store_block(a, tok, n + 128, c[2], c[3]);
}

// Smaller tiles. Workgroups of one XCD (index modulo 8) take consecutive tiles, the tiles of one
// column of outputs first, so that its L2 reads the weights once.
template <typename R>
__global__ void __launch_bounds__(R::kThreads) k_mx4_ring(Mx4Args a) {
  __shared__ __attribute__((aligned(1024))) char b0[R::kBufBytes];
  __shared__ __attribute__((aligned(1024))) char b1[R::kBufBytes];
  __shared__ __attribute__((aligned(1024))) char b2[R::NBUF == 4 ? R::kBufBytes : 16];
  __shared__ __attribute__((aligned(1024))) char b3[R::NBUF == 4 ? R::kBufBytes : 16];
  __shared__ __attribute__((aligned(1024))) char s0[R::kScaleBytes];
  __shared__ __attribute__((aligned(1024))) char s1[R::kScaleBytes];
  const int tiles_m = int((a.n_tok + R::TM - 1) / R::TM), tiles_n = int((a.d_out + R::TN - 1) / R::TN);
  const int tile = int(blockIdx.x & 7) * int(gridDim.x >> 3) + int(blockIdx.x >> 3);
  if (tile >= tiles_m * tiles_n) return;
  const int tn = tile / tiles_m;
  const int64_t m0 = int64_t(tile - tn * tiles_m) * R::TM, n0 = int64_t(tn) * R::TN;
  const int stages = a.row / 128, pairs = (stages + 1) / 2;
  const int p0 = int(int64_t(pairs) * blockIdx.y / gridDim.y);
  const int p1 = int(int64_t(pairs) * (blockIdx.y + 1) / gridDim.y);
  auto token = [&](int r) { return std::min(m0 + r, a.n_tok - 1); };
  auto output = [&](int r) { return std::min(n0 + t256_rows_source(r), a.d_out - 1); };
  mx4::RingSource<R> src;
#pragma unroll
  for (int i = 0; i < R::kLoads; ++i) {
    const int r = mx4::ring_load_row(i);
    src.row[i] = (r < R::TM ? static_cast<const char*>(a.x) + token(r) * a.row
                            : reinterpret_cast<const char*>(a.q) + output(r - R::TM) * a.row) +
                 int64_t(2 * p0) * 128 + ((int(threadIdx.x & 7) ^ (r & 7)) * 16);
  }
  const int r = std::min(int(threadIdx.x), R::TM + R::TN - 1);
  src.scales = reinterpret_cast<const char*>(r < R::TM ? a.xs + token(r) * a.srow
                                                       : a.s + output(r - R::TM) * a.srow) + 16 * p0;
  f4 acc[R::MB][R::NB];
  mx4::ring_mainloop<R>(acc, src, std::min(2 * p1, stages) - 2 * p0, b0, b1, b2, b3, s0, s1);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (gridDim.y > 1) {  // [split][tile][wave][block][lane]
    f4* part = a.part + ((size_t(blockIdx.y) * (tiles_m * tiles_n) + tile) * 4 + wave) * R::MB * R::NB * 64 +
               lane;
#pragma unroll
    for (int mi = 0; mi < R::MB; ++mi)
#pragma unroll
      for (int ni = 0; ni < R::NB; ++ni) part[(mi * R::NB + ni) * 64] = acc[mi][ni];
    return;
  }
#pragma unroll
  for (int mi = 0; mi < R::MB; ++mi)
#pragma unroll
    for (int ni = 0; ni < R::NB; ni += 2)
      store_block(a, m0 + ((wave / R::WN) * R::MB + mi) * 16, n0 + (wave % R::WN) * R::NB * 16 + ni * 16,
                  acc[mi][ni], acc[mi][ni + 1]);
}

template <typename R>
__global__ void __launch_bounds__(kThreads) k_mx4_ring_join(Mx4Args a, int splits, int tiles, int tiles_m) {
  constexpr int kPairs = R::MB * R::NB / 2;  // of blocks, of a wave
  const int lane = threadIdx.x & 63;
  const int64_t at = int64_t(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (at >= int64_t(tiles) * 4 * kPairs) return;
  const f4* part = a.part + at * 2 * 64 + lane;
  const size_t step = size_t(tiles) * 4 * kPairs * 2 * 64;
  f4 c[2] = {};
#pragma unroll 4
  for (int sp = 0; sp < splits; ++sp)
#pragma unroll
    for (int q = 0; q < 2; ++q) c[q] += part[sp * step + q * 64];
  const int tile = int(at / (4 * kPairs)), wave = int(at / kPairs) & 3, pair = int(at % kPairs);
  const int tn = tile / tiles_m, mi = pair / (R::NB / 2), ni = pair % (R::NB / 2) * 2;
  store_block(a, int64_t(tile - tn * tiles_m) * R::TM + ((wave / R::WN) * R::MB + mi) * 16,
              int64_t(tn) * R::TN + (wave % R::WN) * R::NB * 16 + ni * 16, c[0], c[1]);
}

using Ring128x128 = mx4::Ring<128, 128, 2, 2, 2>;
using Ring64x128 = mx4::Ring<64, 128, 1, 4, 2>;
using Ring64x64 = mx4::Ring<64, 64, 2, 2, 4>;

template <typename R>
void launch_ring(const Mx4Args& a, const Mx4Plan& p, hipStream_t s) {
  hipLaunchKernelGGL(k_mx4_ring<R>, dim3(unsigned(round_up(p.tiles, 8)), unsigned(p.splits)),
                     dim3(R::kThreads), 0, s, a);
  if (p.splits > 1)
    hipLaunchKernelGGL(k_mx4_ring_join<R>,
                       dim3(unsigned(ceil_div(p.tiles * 2 * R::MB * R::NB, kThreads / 64))),
                       dim3(kThreads), 0, s, a, p.splits, int(p.tiles), int(ceil_div(a.n_tok, R::TM)));
}

void launch_tile(const Mx4Args& a, hipStream_t s) {
  const Mx4Plan p = mx4_plan(a.n_tok, a.d, a.d_out);
  if (p.tile == kMx4Tile128) return launch_ring<Ring128x128>(a, p, s);
  if (p.tile == kMx4Tile64x128) return launch_ring<Ring64x128>(a, p, s);
  if (p.tile == kMx4Tile64) return launch_ring<Ring64x64>(a, p, s);
  hipLaunchKernelGGL(k_mx4_tile, dim3(unsigned(p.tiles), unsigned(p.splits)), dim3(Tile256::kThreads), 0,
                     s, a);
  if (p.splits > 1)
    hipLaunchKernelGGL(k_mx4_tile_join, dim3(unsigned(p.tiles) * 16), dim3(kThreads), 0, s, a, p.splits,
                       int(p.tiles));
}

template <bool PACKED, int ROWS, int RB, bool RAGGED>
void launch_few(const Mx4Args& a, int waves, hipStream_t s) {
  const size_t each = std::max<size_t>(PACKED ? 0 : size_t(a.n_tok) * kMx4FewPitch, RB * 1024);
  const dim3 grid(unsigned(ceil_div(a.d_out, 16 * RB)), unsigned(ceil_div(a.n_tok, kMx4Few)));
  hipLaunchKernelGGL((k_mx4_few<PACKED, ROWS, RB, RAGGED>), grid, dim3(64 * waves), waves * each, s, a);
}
template <int ROWS, int RB>
void launch_few_16bit(const Mx4Args& a, int waves, hipStream_t s) {
  if (a.d % 8) launch_few<false, 4, RB, true>(a, waves, s);
  else launch_few<false, ROWS, RB, false>(a, waves, s);
}

void launch_packed(const Mx4Args& a, hipStream_t s) {
  if (mx4_packed_tiles(a.n_tok, a.d_out, aligned16(a.xs) && aligned16(a.s))) return launch_tile(a, s);
  const int64_t most = int64_t(65535) * kMx4Few;  // of a launch
  for (int64_t t = 0; t < a.n_tok; t += most) {
    Mx4Args b = a;
    b.x = static_cast<const uint8_t*>(a.x) + t * a.row;
    b.xs = a.xs + t * a.srow;
    b.y = static_cast<char*>(a.y) + t * a.ldy * (a.y_f32 ? 4 : 2);
    b.n_tok = std::min(a.n_tok - t, most);
    const Mx4FewPlan p = mx4_few_plan(std::min<int64_t>(b.n_tok, kMx4Few), a.d, a.d_out, true);
    if (p.blocks == 2) launch_few<true, 4, 2, false>(b, p.waves, s);
    else launch_few<true, 4, 1, false>(b, p.waves, s);
  }
}
void launch_16bit(const Mx4Args& a, hipStream_t s) {
  const Mx4SlabPlan p = mx4_slab_plan(a.n_tok, a.d, a.d_out);
  const Mx4FewPlan few = mx4_few_plan(a.n_tok, a.d, a.d_out, false);
  if (p.tokens == 16) launch_slab<1>(a, p.splits, s);
  else if (p.tokens == 32) launch_slab<2>(a, p.splits, s);
  else if (p.tokens == 64) launch_slab<4>(a, p.splits, s);
  else if (a.n_tok > 4 && few.blocks == 2) launch_few_16bit<8, 2>(a, few.waves, s);
  else if (a.n_tok > 4) launch_few_16bit<8, 1>(a, few.waves, s);
  else if (few.blocks == 2) launch_few_16bit<4, 2>(a, few.waves, s);
  else launch_few_16bit<4, 1>(a, few.waves, s);
}

}  // namespace

size_t mx4_row_bytes(int64_t d) { return size_t(row_bytes(d)); }
size_t mx4_scale_bytes(int64_t d) { return size_t(scale_bytes(d)); }

optima_status mx4_pack(const void* X, int64_t ldx, int dtype, int64_t n, int64_t d, void* Q,
                       void* scales, hipStream_t s) {
  if (dtype == OPTIMA_DTYPE_F32) launch_pack<float, 1>(X, ldx, n, d, Q, scales, s);
  else if (d <= 256) launch_pack<bf16_t, 1>(X, ldx, n, d, Q, scales, s);
  else launch_pack<bf16_t, 2>(X, ldx, n, d, Q, scales, s);
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

optima_status mx4_unpack(const void* Q, const void* scales, int64_t n, int64_t d, void* Y,
                         int64_t ldy, int dtype, hipStream_t s) {
  const uint32_t pieces = uint32_t(ceil_div(d, 256)), total = uint32_t(n * pieces);  // below 2^27
  const int srow = int(scale_bytes(d));
  const dim3 grid(unsigned(ceil_div(total, kThreads / 32)));
  const uint8_t *q = static_cast<const uint8_t*>(Q), *sc = static_cast<const uint8_t*>(scales);
  if (dtype == OPTIMA_DTYPE_BF16)
    hipLaunchKernelGGL(k_mx4_unpack<bf16_t>, grid, dim3(kThreads), 0, s, q, sc, srow, total, pieces,
                       int(d), static_cast<bf16_t*>(Y), ldy);
  else
    hipLaunchKernelGGL(k_mx4_unpack<float>, grid, dim3(kThreads), 0, s, q, sc, srow, total, pieces,
                       int(d), static_cast<float*>(Y), ldy);
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

size_t mx4_workspace_bytes(int64_t n_tok, int64_t d, int64_t d_out) {
  return mx4_room(n_tok, d, d_out);
}

optima_status mx4_linear(const void* X, int64_t ldx, const void* x_scales, int64_t n_tok, int64_t d,
                         const void* Q, const void* scales, int64_t d_out, void* Y, int64_t ldy,
                         int y_dtype, void* ws, hipStream_t s) {
  Mx4Args a{};
  a.x = X;
  a.xs = static_cast<const uint8_t*>(x_scales);
  a.q = static_cast<const uint8_t*>(Q);
  a.s = static_cast<const uint8_t*>(scales);
  a.y = Y;
  a.part = static_cast<f4*>(ws);
  a.n_tok = n_tok;
  a.d_out = d_out;
  a.ldx = ldx;
  a.ldy = ldy;
  a.d = int(d);
  a.chunks = int(ceil_div(d, kChunk));
  a.row = int(row_bytes(d));
  a.srow = int(scale_bytes(d));
  a.y_f32 = y_dtype == OPTIMA_DTYPE_F32;
  if (x_scales) launch_packed(a, s);
  else launch_16bit(a, s);
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

}  // namespace optima
