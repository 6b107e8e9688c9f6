// RMS norm of token rows with the residual's addition, and its gradient.
//
// Forward: s = x + r, y_i = s_i w_i rstd with rstd = (mean(s^2) + eps)^(-1/2).
// Backward: with xh = s rstd, p = w dy and c = mean(p xh),
// dx = dS + rstd (p - c xh) and dw = sum over tokens of dy xh.
//
// Both read each row once and keep it in registers between the sum over the row
// and the outputs, so that they are bound by HBM: 32768 bf16 rows of 4096 with the
// residual 181 us, 5.95 TB/s; the gradient of 16384 of them 104 us, 5.2 TB/s; 20001 fp32
// rows of 1001 to 8 bits 25 us, 3.9 TB/s; one row 3.7 us. A row belongs to a group of threads
// as large as it needs (by_width): part of a wave (up to 256 values), a wave, or a whole
// workgroup; thread t of them holds pieces t, t + THREADS, .. of 8 values. All sums are
// fp32.
#include <type_traits>

#include "common.h"
#include "vec8.h"

namespace optima {
namespace {

// Sum of v[0 .. N-1] over the THREADS threads of a row (up to 64: of a wave; else the
// whole workgroup). red: N * THREADS / 64 floats that no earlier call still reads.
template <int THREADS, int N>
__device__ inline void row_sums(float (&v)[N], float* red) {
#pragma unroll
  for (int o = (THREADS < 64 ? THREADS : 64) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], o, 64);
  if constexpr (THREADS > 64) {
    constexpr int W = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[i * W + wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) v[i] += red[i * W + w];
    }
  }
}

// Largest of the absolute values' bit patterns over groups of LANES lanes. Among
// bit patterns NaN ranks above infinity, so that neither is lost.
__device__ inline uint32_t lanes_max(uint32_t m, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) m = max(m, uint32_t(__shfl_xor(int(m), o, 64)));
  return m;
}

template <int THREADS>
__device__ inline uint32_t row_max(uint32_t m, uint32_t* red) {
  m = lanes_max(m, THREADS < 64 ? THREADS : 64);
  if constexpr (THREADS > 64) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) red[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) m = max(m, red[w]);
  }
  return m;
}

struct NormArgs {
  const void *x, *r, *w;
  void *s, *y;
  float* scales;
  int64_t n, row0, ldx, ldr, lds, ldy;  // row0: the launch's first row
  int d, group, groups, w_bf16;
  float eps;
};

__device__ inline void load_weights(const void* w, int w_bf16, int at, int d, float (&v)[8]) {
  if (w_bf16) {
    Raw8<bf16_t> raw;
    load_piece(raw, static_cast<const bf16_t*>(w), at, d);
    values8(raw, v);
  } else {
    Raw8<float> raw;
    load_piece(raw, static_cast<const float*>(w), at, d);
    values8(raw, v);
  }
}

// Rows of a workgroup, and this thread's of them and place in it.
template <int THREADS>
struct RowGroup {
  static constexpr int kRows = THREADS <= 64 ? 256 / THREADS : 1;
  static constexpr int kWg = THREADS <= 64 ? 256 : THREADS;
  static constexpr int kWaves = (THREADS + 63) / 64;  // of a row
  __device__ static inline int row() { return THREADS <= 64 ? threadIdx.x / THREADS : 0; }
  __device__ static inline int at() { return THREADS <= 64 ? threadIdx.x % THREADS : threadIdx.x; }
};

// One row a group of THREADS threads, CH chunks a thread. T: type of x, r and s;
// O: type of y (int8_t: with scales).
template <typename T, typename O, int THREADS, int CH>
__global__ void __launch_bounds__(RowGroup<THREADS>::kWg) k_rms_norm(NormArgs a) {
  using Rows = RowGroup<THREADS>;
  __shared__ float red[Rows::kWaves];
  __shared__ uint32_t red_max[Rows::kWaves];
  const int t = Rows::at();
  const int64_t row = a.row0 + int64_t(blockIdx.x) * Rows::kRows + Rows::row();
  if (row >= a.n) return;  // all threads of the row
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* r = a.r ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;
  Raw8<T> raw[CH], res[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = 8 * (t + c * THREADS);
    load_piece(raw[c], x, at, a.d);
  }
  if (r)
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = 8 * (t + c * THREADS);
      load_piece(res[c], r, at, a.d);
    }
  float v[CH][8];
  float sq[1] = {0.f};
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    values8(raw[c], v[c]);
    if (r) {
      float u[8];
      values8(res[c], u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] += u[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sq[0] += v[c][i] * v[c][i];
  }
  if (a.s) {
    // The norm is taken of the fp32 sum; s is its rounded copy.
    T* s = static_cast<T*>(a.s) + row * a.lds;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = 8 * (t + c * THREADS);
      store_upto8(s + at, v[c], a.d - at);
    }
  }
  row_sums<THREADS>(sq, red);
  const float rstd = 1.f / sqrtf(sq[0] / float(a.d) + a.eps);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = 8 * (t + c * THREADS);
    float w[8];
    load_weights(a.w, a.w_bf16, at, a.d, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * rstd * w[i];
  }
  O* y = static_cast<O*>(a.y) + row * a.ldy;
  if constexpr (sizeof(O) == 1) {
    float* scales = a.scales + row * a.groups;
    uint32_t m[CH], all = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      m[c] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m[c] = max(m[c], __float_as_uint(v[c][i]) & 0x7FFFFFFFu);
      all = max(all, m[c]);
    }
    if (!a.group) all = row_max<THREADS>(all, red_max);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      // Groups are 4, 8 or 16 aligned lanes, or what a narrow row has.
      const int at = 8 * (t + c * THREADS);
      const float top = __uint_as_float(a.group ? lanes_max(m[c], min(a.group / 8, THREADS)) : all);
      float scale = top / 127.f;
      if (scale < 0x1p-126f) scale = 0.f;
      if (a.group) {
        if ((at & (a.group - 1)) == 0 && at < a.d) scales[at / a.group] = scale;
      } else if (c == 0 && t == 0) {
        scales[0] = scale;
      }
      // A group with an infinity or NaN has codes 0 and that scale: NaN as values.
      const bool fine = scale > 0.f && scale < __builtin_inff();
      const float inv = 1.f / scale;  // |y| inv stays below 127.5
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = fine ? rintf(v[c][i] * inv) : 0.f;
      store_upto8(y + at, v[c], a.d - at);
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = 8 * (t + c * THREADS);
      store_upto8(y + at, v[c], a.d - at);
    }
  }
}

struct NormGradArgs {
  const void *s, *w, *dy, *ds;
  void* dx;
  float* part;  // [blocks][d] sums of dy xh, or NULL; of one block, dw itself
  int add;      // .. to which they are added
  int64_t n, lds, lddy, ldds, lddx;
  int d, w_bf16;
  float eps;
};

// Rows blockIdx, blockIdx + gridDim, .. in groups of kRows; each thread keeps the
// sums of its columns of dw over them.
template <typename T, int THREADS, int CH>
__global__ void __launch_bounds__(RowGroup<THREADS>::kWg) k_rms_norm_grad(NormGradArgs a) {
  using Rows = RowGroup<THREADS>;
  constexpr int kRows = Rows::kRows, kWaves = Rows::kWaves;
  // Two sets, taken in turn: a row's sums are not written before every wave has
  // read those of the row before the last.
  __shared__ float red[2][2 * kWaves];
  __shared__ float cross[kRows == 1 ? 1 : 256 * 8 * CH];
  const int t = Rows::at(), sub = Rows::row();
  // 1024 threads have no registers to keep the weights in: they load them again.
  constexpr bool kKeep = THREADS < 1024;
  float kept[kKeep ? CH : 1][8], dw[CH][8];
  auto weights = [&](int c, float (&w)[8]) {
    if constexpr (kKeep) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = kept[c][i];
    } else {
      load_weights(a.w, a.w_bf16, 8 * (t + c * THREADS), a.d, w);
    }
  };
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if constexpr (kKeep) load_weights(a.w, a.w_bf16, 8 * (t + c * THREADS), a.d, kept[c]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[c][i] = 0.f;
  }
  int turn = 0;
  for (int64_t row = int64_t(blockIdx.x) * kRows + sub; row < a.n;
       row += int64_t(gridDim.x) * kRows, turn ^= 1) {
    Raw8<T> rs[CH], rd[CH], rr[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = 8 * (t + c * THREADS);
      load_piece(rs[c], static_cast<const T*>(a.s) + row * a.lds, at, a.d);
      load_piece(rd[c], static_cast<const T*>(a.dy) + row * a.lddy, at, a.d);
      if (a.ds) load_piece(rr[c], static_cast<const T*>(a.ds) + row * a.ldds, at, a.d);
    }
    float sums[2] = {0.f, 0.f};  // s^2, p s
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float s[8], dy[8], w[8];
      values8(rs[c], s);
      values8(rd[c], dy);
      weights(c, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sums[0] += s[i] * s[i];
        sums[1] += w[i] * dy[i] * s[i];
      }
    }
    row_sums<THREADS>(sums, red[turn]);
    const float rstd = 1.f / sqrtf(sums[0] / float(a.d) + a.eps);
    const float k = sums[1] / float(a.d) * rstd * rstd;  // c xh = k s
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = 8 * (t + c * THREADS);
      float s[8], dy[8], dx[8], w[8];
      values8(rs[c], s);
      values8(rd[c], dy);
      weights(c, w);
      if (a.ds)
        values8(rr[c], dx);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) dx[i] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dx[i] += rstd * (w[i] * dy[i] - k * s[i]);
        dw[c][i] += dy[i] * (s[i] * rstd);
      }
      store_upto8(static_cast<T*>(a.dx) + row * a.lddx + at, dx, a.d - at);
    }
  }
  if (!a.part) return;
  if constexpr (kRows > 1) {
    // The rows' sums, in their order: [value][row][thread of the row].
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) cross[(c * 8 + i) * 256 + threadIdx.x] = dw[c][i];
    __syncthreads();
    if (sub > 0) return;
#pragma unroll 1
    for (int u = 1; u < kRows; ++u)
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] += cross[(c * 8 + i) * 256 + u * THREADS + t];
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = 8 * (t + c * THREADS);
    float* part = a.part + size_t(blockIdx.x) * size_t(a.d);
    if (a.add) {
      Raw8<float> was;
      load_piece(was, part, at, a.d);
      float old[8];
      values8(was, old);
#pragma unroll
      for (int i = 0; i < 8; ++i) dw[c][i] += old[i];
    }
    store_upto8(part + at, dw[c], a.d - at);
  }
}

// dw (+)= sum of the blocks' partial sums: 64 columns a workgroup, whose 16
// waves take every 16th partial and are added in their order. 512 parts of 4096: 4 us.
__global__ void __launch_bounds__(1024) k_norm_dw(const float* part, int blocks, int d, float* dw,
                                                  int accumulate) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (col < d)
#pragma unroll 8
    for (int b = wave; b < blocks; b += 16) s += part[size_t(b) * size_t(d) + col];
  red[wave][lane] = s;
  __syncthreads();
  if (wave || col >= d) return;
  for (int k = 1; k < 16; ++k) s += red[k][lane];
  dw[col] = accumulate ? dw[col] + s : s;
}

// Threads, and pieces of 8 values a thread, of a row of d values. Few threads with
// several pieces spare a row the barriers of its sums, which the 8-bit output has two
// of, and a third piece spares rows of 5000 to 6144 values the idle fourth. 128 million
// bf16 values to 8 bits: d = 2048 113 us in 256 threads, 93 in 64 (to bf16 174 and 181, so
// that only the former take them); d = 8192 145 in 1024, 93 in 256; d = 5000 207 in 1024,
// 135 and 103 in 256 with four and three pieces.
template <int N>
using Int = std::integral_constant<int, N>;
template <bool TO_8_BITS, typename F>
void by_width(int64_t d, F f) {
  if (d <= 64) f(Int<8>(), Int<1>());
  else if (d <= 128) f(Int<16>(), Int<1>());
  else if (d <= 256) f(Int<32>(), Int<1>());
  else if (d <= 512) f(Int<64>(), Int<1>());
  else if (d <= 1024) f(Int<64>(), Int<2>());
  else if (d <= 2048) f(Int<TO_8_BITS ? 64 : 256>(), Int<TO_8_BITS ? 4 : 1>());
  else if (d <= 4096) f(Int<256>(), Int<2>());
  else if (d <= 6144) f(Int<256>(), Int<3>());
  else if (d <= 8192) f(Int<256>(), Int<4>());
  else if (d <= 12288) f(Int<512>(), Int<3>());
  else f(Int<512>(), Int<4>());
}
static_assert(OPTIMA_NORM_MAX_DIM == 512 * 4 * 8, "the widest row that by_width covers");

// The same for the gradient, which keeps more of each value.
template <typename F>
void grad_by_width(int64_t d, F f) {
  if (d <= 64) f(Int<8>(), Int<1>());
  else if (d <= 128) f(Int<16>(), Int<1>());
  else if (d <= 256) f(Int<32>(), Int<1>());
  else if (d <= 512) f(Int<64>(), Int<1>());
  else if (d <= 1024) f(Int<64>(), Int<2>());
  else if (d <= 2048) f(Int<256>(), Int<1>());
  else if (d <= 4096) f(Int<256>(), Int<2>());
  else if (d <= 8192) f(Int<512>(), Int<2>());
  else f(Int<1024>(), Int<2>());
}

template <typename T, typename O>
void launch_norm(NormArgs a, hipStream_t s) {
  by_width<sizeof(T) == 2 && sizeof(O) == 1>(a.d, [&](auto threads, auto ch) {
    constexpr int kT = decltype(threads)::value, kCh = decltype(ch)::value;
    using Rows = RowGroup<kT>;
    // A launch has fewer than 2^32 threads.
    constexpr int64_t kMost = (int64_t(1) << 22) * Rows::kRows;
    for (; a.row0 < a.n; a.row0 += kMost)
      hipLaunchKernelGGL((k_rms_norm<T, O, kT, kCh>),
                         dim3(unsigned(ceil_div(std::min(a.n - a.row0, kMost), Rows::kRows))),
                         dim3(Rows::kWg), 0, s, a);
  });
}

// Rows that one workgroup takes one after the other, so that it has dw by itself and
// nothing has to be joined: d = 2048, one row 4.7 to 2.6 us, two rows 4.7 to 3.5, but four
// 4.7 to 5.1.
constexpr int64_t kOneBlock = 2;
// Workgroups of the gradient, by the sizes alone, so that the order of dw's sums is too.
// 128 million bf16 values, with 256, 512, 1024 and 2048 of them: d = 1024 218, 196, 205 and
// 209 us, d = 4096 230, 193, 212 and 220.
int grad_blocks(int64_t n, int64_t d) {
  int64_t rows = 0;
  grad_by_width(d, [&](auto threads, auto) { rows = RowGroup<decltype(threads)::value>::kRows; });
  if (n > 0 && n <= kOneBlock * rows) return 1;
  return int(std::min<int64_t>(ceil_div(n, rows), d <= 2048 ? 1024 : d <= 8192 ? 512 : 256));
}

}  // namespace

optima_status rms_norm(const void* X, int64_t ldx, const void* R, int64_t ldr, int dtype, int64_t n,
                       int64_t d, const void* w, int w_dtype, float eps, void* S, int64_t lds,
                       void* Y, int64_t ldy, int y_dtype, float* scales, int64_t group,
                       hipStream_t s) {
  NormArgs a{X, R, w, S, Y, scales, n, 0, ldx, ldr, lds, ldy, int(d), int(group),
             int(group ? ceil_div(d, group) : 1), w_dtype == OPTIMA_DTYPE_BF16, eps};
  if (dtype == OPTIMA_DTYPE_BF16) {
    if (y_dtype == OPTIMA_DTYPE_BF16) launch_norm<bf16_t, bf16_t>(a, s);
    else if (y_dtype == OPTIMA_DTYPE_F32) launch_norm<bf16_t, float>(a, s);
    else launch_norm<bf16_t, int8_t>(a, s);
  } else {
    if (y_dtype == OPTIMA_DTYPE_BF16) launch_norm<float, bf16_t>(a, s);
    else if (y_dtype == OPTIMA_DTYPE_F32) launch_norm<float, float>(a, s);
    else launch_norm<float, int8_t>(a, s);
  }
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

size_t rms_norm_backward_workspace_bytes(int64_t n, int64_t d) {
  return size_t(grad_blocks(n, d)) * size_t(d) * sizeof(float);
}

optima_status rms_norm_backward(const void* S, int64_t lds, const void* w, int w_dtype,
                                const void* dY, int64_t lddy, const void* dS, int64_t ldds,
                                int dtype, int64_t n, int64_t d, float eps, void* dX, int64_t lddx,
                                float* dweight, int accumulate, void* ws, hipStream_t s) {
  const int blocks = grad_blocks(n, d);
  if (n > 0) {
    float* part = blocks == 1 ? dweight : static_cast<float*>(ws);
    NormGradArgs a{S, w, dY, dS, dX, dweight ? part : nullptr, blocks == 1 && accumulate, n, lds,
                   lddy, ldds, lddx, int(d), w_dtype == OPTIMA_DTYPE_BF16, eps};
    grad_by_width(d, [&](auto threads, auto ch) {
      constexpr int kT = decltype(threads)::value, kCh = decltype(ch)::value;
      const dim3 wg(RowGroup<kT>::kWg);
      if (dtype == OPTIMA_DTYPE_BF16)
        hipLaunchKernelGGL((k_rms_norm_grad<bf16_t, kT, kCh>), dim3(blocks), wg, 0, s, a);
      else
        hipLaunchKernelGGL((k_rms_norm_grad<float, kT, kCh>), dim3(blocks), wg, 0, s, a);
    });
    OPTIMA_LAUNCH_CHECK();
  }
  if (dweight && blocks != 1) {
    hipLaunchKernelGGL(k_norm_dw, dim3(unsigned(ceil_div(d, 64))), dim3(1024), 0, s,
                       static_cast<const float*>(ws), blocks, int(d), dweight, accumulate);
    OPTIMA_LAUNCH_CHECK();
  }
  return OPTIMA_OK;
}

}  // namespace optima
