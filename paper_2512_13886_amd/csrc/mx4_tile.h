// MFMA main loop of a 256 x 256 tile of outputs Y = X W^T of packed tokens and weights. Buffers,
// swizzle and the offset of half the waves by one part are those of gemm256.h, whose stage of 128
// bytes a row is 256 codes here and whose two K steps are two block-scaled 16x16x128 MFMAs. A
// stage has two phases in place of four:
//   1: read A0, B0, B1   A0 B0, A0 B1   fetch A1 of the next stage
//   2: read A1           A1 B1, A1 B0   fetch A0, B0 and B1 of the stage after it
// so that there are half the barriers, and an MFMA part (32 of 16 cycles) is longer than the other
// group's LDS reads (up to 64 KiB). Every load has a stage's time: both waits leave the newest four
// half tiles in flight, one phase's A1 and the other's three.
//
// Bound by the direct loads, 64 KiB a stage, 18 bytes a clock and CU (of which the L2 caches serve 83 to 85 % of
// the requests, far below their rate: it is the loads' time in flight), and what of the MFMAs does not run
// beside them: 8192 tokens, 4096 -> 14336 250 us (3.8 PFLOP/s), 30 of them the outputs' stores at the
// tiles' ends; 4096 tokens, 14336 -> 4096 105 us (4.6). Of 265 and 112 us it took 195 and 76 without its
// MFMAs, 224 and 89 without its loads, 243 and 103 without the scales. The matrix instructions are busy
// for 47 and 54 % of the time at 1.9 GHz; alone in registers they reach 7.4 PFLOP/s with random codes and
// 9.2 with constant ones. Four phases took the same time as two. All operands of the next half stage read
// while one multiplies would need about 240 registers beside the addresses, and spilled.
//
// The scales of two stages are 16 bytes a row: one direct load a thread brings those of the 256
// rows of X and of W into LDS, first in phase 1 of every even stage, for the two stages after the
// present pair, and each lane keeps the twelve dwords of its rows for both stages (the MFMA picks
// the byte). The waits of an even stage leave that load in flight too, those of the odd one do
// not. Its buffer was last read two stages before.
#pragma once

#include "gemm256.h"

namespace optima {
namespace mx4 {

typedef int i8x32 __attribute__((ext_vector_type(8)));

constexpr int kScaleBytes = 512 * 16;  // of a pair of stages: 256 rows of X, then 256 of W

template <int U>
__device__ inline void mfma(f4& c, const bf16x8& w, uint32_t sw, const bf16x8& x, uint32_t sx) {
  typedef int i4x __attribute__((ext_vector_type(4)));
  const i4x p = __builtin_bit_cast(i4x, w), q = __builtin_bit_cast(i4x, x);
  const i8x32 a = {p[0], p[1], p[2], p[3], 0, 0, 0, 0}, b = {q[0], q[1], q[2], q[3], 0, 0, 0, 0};
  c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, U, int(sw), U, int(sx));
}

struct Scales {
  uint32_t a[2][4], b[2][2];  // of this lane's rows: [half][16-row block]
};

__device__ inline void read_scales(Scales& s, const char* l) {
  const int lane = threadIdx.x & 63, wm = threadIdx.x >> 8, wn = (threadIdx.x >> 6) & 3;
  const char* p = l + (lane & 15) * 16 + (lane >> 4) * 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int m = 0; m < 4; ++m)
      s.a[h][m] = *reinterpret_cast<const uint32_t*>(p + (h * 128 + wm * 64 + m * 16) * 16);
#pragma unroll
    for (int m = 0; m < 2; ++m)
      s.b[h][m] = *reinterpret_cast<const uint32_t*>(p + (256 + h * 128 + wn * 32 + m * 16) * 16);
  }
}

template <int U0>
__device__ inline void quadrant(f4 (&c)[4][2], const bf16x8 (&a)[4][2], const uint32_t (&sa)[4],
                                const bf16x8 (&b)[2][2], const uint32_t (&sb)[2]) {
#pragma unroll
  for (int mi = 0; mi < 4; ++mi)
#pragma unroll
    for (int ni = 0; ni < 2; ++ni) mfma<U0>(c[mi][ni], b[ni][0], sb[ni], a[mi][0], sa[mi]);
#pragma unroll
  for (int mi = 0; mi < 4; ++mi)
#pragma unroll
    for (int ni = 0; ni < 2; ++ni) mfma<U0 + 1>(c[mi][ni], b[ni][1], sb[ni], a[mi][1], sa[mi]);
}

__device__ inline void fetch_scales(const char* src, char* l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)(l + (threadIdx.x >> 6) * 1024),
                                   16, 0, 0);
}

// One stage from buffers a0, a1, b0, b1; na1 is the other A1 buffer. In an even one (U0 = 0) the
// scales `now` are read and those at `src_s` fetched into `next`.
template <int U0>
__device__ inline void stage(Acc256& acc, Scales& sc, const Operands256& src, int64_t off1,
                             int64_t off2, char* a0, char* a1, char* b0, char* b1, char* na1,
                             const char* now, const char* src_s, char* next) {
  constexpr int kFlight = 4 * Tile256::kHalfLoads + (U0 == 0);
  const int wm = threadIdx.x >> 8, wn = (threadIdx.x >> 6) & 3;
  bf16x8 fa[4][2], fb0[2][2], fb1[2][2];
  if constexpr (U0 == 0) fetch_scales(src_s, next);
  t256::fetch(src.a[1], off1, na1);
  t256::read<4>(fa, a0, wm * 64);
  t256::read<2>(fb0, b0, wn * 32);
  t256::read<2>(fb1, b1, wn * 32);
  if constexpr (U0 == 0) read_scales(sc, now);
  t256::end_memory<kFlight>();
  quadrant<U0>(acc.q[0][0], fa, sc.a[0], fb0, sc.b[0]);
  quadrant<U0>(acc.q[0][1], fa, sc.a[0], fb1, sc.b[1]);
  t256::barrier();
  t256::fetch(src.a[0], off2, a0);
  t256::fetch(src.b[0], off2, b0);
  t256::fetch(src.b[1], off2, b1);
  t256::read<4>(fa, a1, wm * 64);
  t256::end_memory<kFlight>();
  quadrant<U0>(acc.q[1][1], fa, sc.a[1], fb1, sc.b[1]);
  quadrant<U0>(acc.q[1][0], fa, sc.a[1], fb0, sc.b[0]);
  t256::barrier();
}

// n stages (n >= 1) from an even one on. l: the eight half tiles; s: two buffers of kScaleBytes;
// scales: this thread's row's at the first stage.
__device__ inline void mainloop(Acc256& acc, const Operands256& src, const char* scales, int n,
                                char* a00, char* a01, char* b00, char* b01, char* a10, char* a11,
                                char* b10, char* b11, char* s0, char* s1) {
#pragma unroll
  for (int i = 0; i < 32; ++i) acc.q[i >> 4][(i >> 3) & 1][(i >> 1) & 3][i & 1] = f4{0.f, 0.f, 0.f, 0.f};
  const int pairs = (n + 1) >> 1;
  auto at = [n](int s) { return int64_t(s < n ? s : n - 1) * Tile256::kSRB; };
  auto at_s = [pairs, scales](int p) { return scales + 16 * (p < pairs ? p : pairs - 1); };
  fetch_scales(at_s(0), s0);
  t256::fetch(src.a[0], at(0), a00);
  t256::fetch(src.b[0], at(0), b00);
  t256::fetch(src.b[1], at(0), b01);
  t256::fetch(src.a[1], at(0), a01);
  t256::fetch(src.a[0], at(1), a10);
  t256::fetch(src.b[0], at(1), b10);
  t256::fetch(src.b[1], at(1), b11);
  t256::end_memory<4 * Tile256::kHalfLoads>();
  const bool behind = threadIdx.x >= 256;  // waves 4-7
  if (behind) t256::barrier();
  Scales sc;
  // The buffers by name: through a pointer the compiler loses track of the array and waits for
  // the loads in flight into the others.
  auto even = [&](int s, const char* now, char* next) {
    stage<0>(acc, sc, src, at(s + 1), at(s + 2), a00, a01, b00, b01, a11, now, at_s(s / 2 + 1), next);
  };
  auto odd = [&](int s) {
    stage<2>(acc, sc, src, at(s + 1), at(s + 2), a10, a11, b10, b11, a01, nullptr, nullptr, nullptr);
  };
  int s = 0;
  for (; s + 3 < n; s += 4) {
    even(s, s0, s1);
    odd(s + 1);
    even(s + 2, s1, s0);
    odd(s + 3);
  }
  if (s < n) even(s, s0, s1);
  if (s + 1 < n) odd(s + 1);
  if (s + 2 < n) even(s + 2, s1, s0);
  if (!behind) t256::barrier();
  // No load may still be writing LDS when the workgroup moves on.
  wait_vmcnt<0>();
  __syncthreads();
}

// ---------------------------------------------------------------------------
// Smaller tiles: four waves, a ring of NBUF stages, one barrier a stage
// ---------------------------------------------------------------------------

// A tile of TM tokens and TN outputs; waves of a WM x WN grid own MB x NB blocks of 16 x 16.
template <int TM_, int TN_, int WM_, int WN_, int NBUF_>
struct Ring {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, NBUF = NBUF_;
  static constexpr int MB = TM / WM / 16, NB = TN / WN / 16;
  static constexpr int kThreads = 256;
  static constexpr int kBufBytes = (TM + TN) * 128;       // rows of X, then of W
  static constexpr int kScaleBytes = 256 * 16;            // of a pair of stages
  static constexpr int kLoads = (TM + TN) / 8 / 4;        // wave loads of a stage
  static_assert(WM * WN == 4 && NB % 2 == 0 && TM + TN <= 256, "");
};

// Row of the tile (X's, then W's from TM on) that load i of this thread fetches, 16 bytes of it.
__device__ inline int ring_load_row(int i) {
  return (i * 4 + int(threadIdx.x >> 6)) * 8 + int((threadIdx.x & 63) >> 3);
}

template <typename R>
struct RingSource {
  const char* row[R::kLoads];  // this thread's addresses at the first stage
  const char* scales;
};

template <typename R>
struct RingScales {
  uint32_t a[R::MB], b[R::NB];
};

// One stage: what it reads of has landed in every wave once the barrier is passed, and the buffer
// `to`, of the stage before, has been read. The newest loads, of the NBUF - 2 stages after this one
// and in an odd stage the scales that were fetched between them, stay in flight.
template <typename R, int U0>
__device__ inline void ring_stage(f4 (&acc)[R::MB][R::NB], RingScales<R>& sc, const RingSource<R>& src,
                                  int s, int n, const char* cur, char* to, const char* now, char* next) {
  constexpr int kFlight = (R::NBUF - 2) * R::kLoads + (U0 != 0 && R::NBUF > 2);
  __builtin_amdgcn_sched_barrier(0);
  if (s + R::NBUF - 2 < n)
    __builtin_amdgcn_s_waitcnt((kFlight & 15) | ((kFlight >> 4) << 14) | 0x0F70);  // vmcnt
  else
    __builtin_amdgcn_s_waitcnt(0x0F70);
  t256::barrier();
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4;
  auto fetch = [&] {
    if (U0 == 0 && s + 2 < n)
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(src.scales + 8 * (s + 2)),
          (__attribute__((address_space(3))) void*)(next + wave * 1024), 16, 0, 0);
    if (s + R::NBUF - 1 < n)
  #pragma unroll
      for (int i = 0; i < R::kLoads; ++i)
        __builtin_amdgcn_global_load_lds(
            (const __attribute__((address_space(1))) void*)(src.row[i] + int64_t(s + R::NBUF - 1) * 128),
            (__attribute__((address_space(3))) void*)(to + (i * 4 + wave) * 1024), 16, 0, 0);
  };
  // With two buffers the next stage's loads have no time to lose; with four the reads go first, and the
  // loads' addresses are worked out behind them (64 tokens, 4096 -> 14336 13.8 to 11.9 us).
  if constexpr (R::NBUF == 2) fetch();
  const int ra = (wave / R::WN) * R::MB * 16 + (lane & 15);
  const int rb = R::TM + (wave % R::WN) * R::NB * 16 + (lane & 15);
  if constexpr (U0 == 0) {
#pragma unroll
    for (int m = 0; m < R::MB; ++m)
      sc.a[m] = *reinterpret_cast<const uint32_t*>(now + (ra + 16 * m) * 16 + 4 * g);
#pragma unroll
    for (int m = 0; m < R::NB; ++m)
      sc.b[m] = *reinterpret_cast<const uint32_t*>(now + (rb + 16 * m) * 16 + 4 * g);
  }
  bf16x8 fa[2][R::MB], fb[2][R::NB];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    auto frag = [cur, g, k](int r) {
      return *reinterpret_cast<const bf16x8*>(cur + r * 128 + (((4 * k + g) ^ (r & 7)) * 16));
    };
#pragma unroll
    for (int m = 0; m < R::NB; ++m) fb[k][m] = frag(rb + 16 * m);
#pragma unroll
    for (int m = 0; m < R::MB; ++m) fa[k][m] = frag(ra + 16 * m);
  }
  if constexpr (R::NBUF > 2) {
    __builtin_amdgcn_sched_barrier(0);
    fetch();
  }
#pragma unroll
  for (int mi = 0; mi < R::MB; ++mi)
#pragma unroll
    for (int ni = 0; ni < R::NB; ++ni)
      mfma<U0>(acc[mi][ni], fb[0][ni], sc.b[ni], fa[0][mi], sc.a[mi]);
#pragma unroll
  for (int mi = 0; mi < R::MB; ++mi)
#pragma unroll
    for (int ni = 0; ni < R::NB; ++ni)
      mfma<U0 + 1>(acc[mi][ni], fb[1][ni], sc.b[ni], fa[1][mi], sc.a[mi]);
}

// n stages (n >= 1) from an even one on. b0 .. b3: the ring's buffers, the first NBUF of them.
template <typename R>
__device__ inline void ring_mainloop(f4 (&acc)[R::MB][R::NB], const RingSource<R>& src, int n, char* b0,
                                     char* b1, char* b2, char* b3, char* s0, char* s1) {
  static_assert(R::NBUF == 2 || R::NBUF == 4, "stages in fours");
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int m = 0; m < R::MB; ++m)
#pragma unroll
    for (int k = 0; k < R::NB; ++k) acc[m][k] = f4{0.f, 0.f, 0.f, 0.f};
  auto first = [&](int s, char* to) {
#pragma unroll
    for (int i = 0; i < R::kLoads; ++i)
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(src.row[i] + int64_t(s) * 128),
          (__attribute__((address_space(3))) void*)(to + (i * 4 + wave) * 1024), 16, 0, 0);
  };
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src.scales,
                                   (__attribute__((address_space(3))) void*)(s0 + wave * 1024), 16, 0, 0);
  first(0, b0);
  if constexpr (R::NBUF == 4) {
    if (1 < n) first(1, b1);
    if (2 < n) first(2, b2);
  }
  RingScales<R> sc;
  for (int s = 0; s < n; s += 4) {
    if constexpr (R::NBUF == 4) {
      ring_stage<R, 0>(acc, sc, src, s, n, b0, b3, s0, s1);
      if (s + 1 < n) ring_stage<R, 2>(acc, sc, src, s + 1, n, b1, b0, nullptr, nullptr);
      if (s + 2 < n) ring_stage<R, 0>(acc, sc, src, s + 2, n, b2, b1, s1, s0);
      if (s + 3 < n) ring_stage<R, 2>(acc, sc, src, s + 3, n, b3, b2, nullptr, nullptr);
    } else {
      ring_stage<R, 0>(acc, sc, src, s, n, b0, b1, s0, s1);
      if (s + 1 < n) ring_stage<R, 2>(acc, sc, src, s + 1, n, b1, b0, nullptr, nullptr);
      if (s + 2 < n) ring_stage<R, 0>(acc, sc, src, s + 2, n, b0, b1, s1, s0);
      if (s + 3 < n) ring_stage<R, 2>(acc, sc, src, s + 3, n, b1, b0, nullptr, nullptr);
    }
  }
}

}  // namespace mx4
}  // namespace optima
