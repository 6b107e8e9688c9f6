// MFMA main loop of a 256x256 output tile of C = A B^T (both operands row-major
// with the contraction contiguous, as in gemm_core.h) by 8 waves, one workgroup
// per CU.
//
// Stages of 128 bytes a row: 64 bf16 values, or 32 columns of split planes (64
// bytes of hi, 64 of lo). A stage is four half tiles of 128 rows, A0, A1, B0
// and B1, 16 KiB each, in LDS arrays of their own (two of each, 128 KiB). Wave
// (wm, wn) of a 2 x 4 grid owns 64 x 32 outputs of each of the four quadrants
// (A half, B half), and multiplies a stage in four phases, one quadrant each:
//   1: read A0, B0   A0 B0      fetch A1 of the next stage
//   2: read B1       A0 B1      fetch A0 of the stage after it
//   3: read A1       A1 B1      fetch B0 of the stage after it
//   4:               A1 B0      fetch B1 of the stage after it
// so every half tile is fetched again as soon as all waves have read it, and
// six to eight 1-KiB loads a wave stay in flight across each stage's end.
//
// A phase is a memory part (LDS reads, the fetch) and an MFMA part, each ended
// by a barrier, and waves 4-7 run one part behind waves 0-3. Waves w and w + 4
// share a SIMD, so in every interval one of them multiplies while the other
// reads. What makes it safe, with parts numbered along the barriers:
//   - a wave's LDS reads have returned before the barrier that ends its memory
//     part, and a half tile is refilled in a later part of either group;
//   - a wave waits for its fetches of the next stage (all but the newest three
//     half tiles) in the memory part of phase 4. The group behind does so in
//     the part before the one in which the group ahead first reads them.
//
// Bound by the MFMAs and, in phase 1, the LDS reads (24 KiB a wave and stage).
// bf16, 32768 x 4096 outputs: each further 4096 of the contraction takes 715 us
// (1.54 PFLOP/s; the 4-wave 128 x 128 loop runs at 0.96). Without the half-phase
// offset between the groups the whole product takes 10 % longer; raising the
// wave's priority around its MFMAs changes nothing.
#pragma once

#include "gemm_core.h"

namespace optima {

struct Tile256 {
  static constexpr int BM = 256, BN = 256, kWaves = 8, kThreads = 512;
  static constexpr int kSRB = 128;                  // bytes per row and stage
  static constexpr int kHalfBytes = 128 * kSRB;     // one half tile
  static constexpr int kHalfLoads = kHalfBytes / 1024 / kWaves;  // wave loads per half tile
};

// Source addresses of this thread's loads at the first stage: half tile h of A
// or B, load i, fetches tile row 128 h + t256_load_row(i), at byte
// t256_seg_bytes(i) of the row's stage. 16-byte aligned.
struct Operands256 {
  const char* a[2][Tile256::kHalfLoads];
  const char* b[2][Tile256::kHalfLoads];
};

__device__ inline int t256_load_row(int i) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  return (i * Tile256::kWaves + wave) * 8 + (lane >> 3);
}
// 16-byte segment g of row r sits at physical segment g ^ (r % 8).
__device__ inline int t256_seg_bytes(int i) {
  return (int(threadIdx.x & 7) ^ (t256_load_row(i) & 7)) * 16;
}

// Bytes from a thread's first-stage addresses to those of stage s.
struct RowSteps {
  __device__ inline int64_t a(int s) const { return int64_t(s) * Tile256::kSRB; }
  __device__ inline int64_t b(int s) const { return int64_t(s) * Tile256::kSRB; }
};

// Half tiles of a B with the contraction along its rows: 64 rows (k) of 128 columns,
// 256 bytes each. Load i of this thread fetches row tr_load_row(i), byte
// tr_seg_bytes() of its 256. 16-byte segment g of row r sits at physical segment
// g ^ tr_swz(r), so that the transposing reads meet no bank twice.
__device__ inline int tr_load_row(int i) {
  return (i * Tile256::kWaves + int(threadIdx.x >> 6)) * 4 + int((threadIdx.x & 63) >> 4);
}
__device__ inline int tr_swz(int r) { return 2 * ((r & 3) | (((r >> 3) & 1) << 2)); }
__device__ inline int tr_seg_bytes() {
  return (int(threadIdx.x & 15) ^ tr_swz(tr_load_row(0))) * 16;  // the same for every i
}

struct Acc256 {
  f4 q[2][2][4][2];  // [A half][B half][16-row block][16-column block]
};

// Row and column, within the tile, of element e of block (mi, ni) of quadrant
// (qa, qb) of this thread.
__device__ inline int t256_row(int qa, int mi, int e) {
  const int lane = threadIdx.x & 63, wm = threadIdx.x >> 8;
  return qa * 128 + wm * 64 + mi * 16 + 4 * (lane >> 4) + e;
}
__device__ inline int t256_col(int qb, int ni) {
  const int lane = threadIdx.x & 63, wn = (threadIdx.x >> 6) & 3;
  return qb * 128 + wn * 32 + ni * 16 + (lane & 15);
}

// The same with Bf16Rows. A lane holds row t256_rows_row(qa, mi), and of the two
// blocks of a wave's 32 columns eight consecutive ones from t256_rows_col(qb) on,
// block 0's four first, if LDS row r of a half tile of B is fetched from column
// t256_rows_source(r) of the half.
__device__ inline int t256_rows_row(int qa, int mi) {
  return qa * 128 + int(threadIdx.x >> 8) * 64 + mi * 16 + int(threadIdx.x & 15);
}
__device__ inline int t256_rows_col(int qb) {
  return qb * 128 + int((threadIdx.x >> 6) & 3) * 32 + 8 * int((threadIdx.x >> 4) & 3);
}
__device__ inline int t256_rows_source(int r) {
  return (r & ~31) + 8 * ((r >> 2) & 3) + 4 * ((r >> 4) & 1) + (r & 3);
}

namespace t256 {

__device__ inline void fetch(const char* const (&src)[Tile256::kHalfLoads], int64_t off, char* half) {
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < Tile256::kHalfLoads; ++i)
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void*)(src[i] + off),
        (__attribute__((address_space(3))) void*)(half + (i * Tile256::kWaves + wave) * 1024), 16, 0,
        0);
}

// Fragments of NBLK 16-row blocks from row r0 of a half tile: segments g and
// 4 + g of the rows (the two 32-value K steps of bf16, or the hi and lo planes).
template <int NBLK>
__device__ inline void read(bf16x8 (&f)[NBLK][2], const char* half, int r0) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int r = r0 + (lane & 15);
  const char* p0 = half + r * Tile256::kSRB + ((g ^ (r & 7)) * 16);
  const char* p1 = half + r * Tile256::kSRB + (((4 + g) ^ (r & 7)) * 16);
#pragma unroll
  for (int m = 0; m < NBLK; ++m) {
    f[m][0] = *reinterpret_cast<const bf16x8*>(p0 + m * 16 * Tile256::kSRB);
    f[m][1] = *reinterpret_cast<const bf16x8*>(p1 + m * 16 * Tile256::kSRB);
  }
}

// The same of a half tile with the contraction along its rows: columns c0 on.
// ds_read_b64_tr_b16 treats the eight-byte reads of 16 lanes as a 4 x 16 matrix of
// 16-bit values (lane j supplies row j / 4, columns 4 (j % 4) .. + 3) and returns
// column i to lane i: two of them give a lane eight consecutive k of its column.
template <int NBLK>
__device__ inline void read_tr(bf16x8 (&f)[NBLK][2], const char* half, int c0) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63, g = lane >> 4, j = lane & 15;
  const int row = 8 * g + (j >> 2), sw = tr_swz(row);
  // One offset from the array: through a chain of them the compiler loses track of the
  // array and waits for the other arrays' loads in flight.
  auto at = [half](int off) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(half + off));
  };
#pragma unroll
  for (int m = 0; m < NBLK; ++m) {
    const int off = row * 256 + 8 * (j & 1) + (((c0 >> 3) + 2 * m + ((j & 3) >> 1)) ^ sw) * 16;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const v4s lo = at(off + k * 8192), hi = at(off + k * 8192 + 1024);
      f[m][k] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
}
template <int NBLK, bool TR>
__device__ inline void read_operand(bf16x8 (&f)[NBLK][2], const char* half, int r0) {
  if constexpr (TR)
    read_tr<NBLK>(f, half, r0);
  else
    read<NBLK>(f, half, r0);
}

// The second and third products of split planes go to `cross`, which may be c.
template <typename T>
__device__ inline void quadrant(f4 (&c)[4][2], f4 (&cross)[4][2], const bf16x8 (&a)[4][2],
                                const bf16x8 (&b)[2][2]) {
  constexpr bool kSplit = std::is_same<T, Bf16x3Tag>::value;
  constexpr bool kRows = MfmaOperands<T>::kRows;
#pragma unroll
  for (int p = 0; p < (kSplit ? 3 : 2); ++p) {
    // bf16: both K steps; split planes: hi hi, hi lo, lo hi.
    const int pa = kSplit ? p >> 1 : p, pb = kSplit ? p & 1 : p;
    f4 (&to)[4][2] = kSplit && p > 0 ? cross : c;
#pragma unroll
    for (int mi = 0; mi < 4; ++mi)
#pragma unroll
      for (int ni = 0; ni < 2; ++ni)
        to[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kRows ? b[ni][pb] : a[mi][pa],
                                                             kRows ? a[mi][pa] : b[ni][pb],
                                                             to[mi][ni], 0, 0, 0);
  }
}

__device__ inline void barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// End of a memory part: LDS reads back, and all but N loads landed (N < 0: no
// wait for loads).
template <int N>
__device__ inline void end_memory() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  if constexpr (N >= 0)
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x70);  // vmcnt(N) lgkmcnt(0)
  else
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  barrier();
}

// One stage from buffers a0, a1, b0, b1; na1 is the other A1 buffer.
template <typename T>
__device__ inline void stage(Acc256& acc, const Operands256& src, int64_t a_off1, int64_t a_off2,
                             int64_t b_off2, char* a0, char* a1, char* b0, char* b1, char* na1) {
  constexpr bool kTb = MfmaOperands<T>::kTb;
  const int wm = threadIdx.x >> 8, wn = (threadIdx.x >> 6) & 3;
  bf16x8 fa[4][2], fb0[2][2], fb1[2][2];
  read<4>(fa, a0, wm * 64);
  read_operand<2, kTb>(fb0, b0, wn * 32);
  fetch(src.a[1], a_off1, na1);
  end_memory<-1>();
  quadrant<T>(acc.q[0][0], acc.q[0][0], fa, fb0);
  barrier();
  read_operand<2, kTb>(fb1, b1, wn * 32);
  fetch(src.a[0], a_off2, a0);
  end_memory<-1>();
  quadrant<T>(acc.q[0][1], acc.q[0][1], fa, fb1);
  barrier();
  read<4>(fa, a1, wm * 64);
  fetch(src.b[0], b_off2, b0);
  end_memory<-1>();
  quadrant<T>(acc.q[1][1], acc.q[1][1], fa, fb1);
  barrier();
  fetch(src.b[1], b_off2, b1);
  end_memory<3 * Tile256::kHalfLoads>();
  quadrant<T>(acc.q[1][0], acc.q[1][0], fa, fb0);
  barrier();
}

}  // namespace t256

// n stages (n >= 0) of tile products. The LDS arguments are distinct
// __shared__ arrays of Tile256::kHalfBytes; fetches past the last stage repeat
// it, into buffers that nobody reads again. `aside` runs once the first fetches
// are out. `steps` says where a stage's operands are.
template <typename T, typename Aside, typename Steps = RowSteps>
__device__ inline void gemm256_mainloop(Acc256& acc, const Operands256& src, int n, char* a00,
                                        char* a01, char* b00, char* b01, char* a10, char* a11,
                                        char* b10, char* b11, Aside aside,
                                        const Steps& steps = Steps{}) {
#pragma unroll
  for (int i = 0; i < 32; ++i) acc.q[i >> 4][(i >> 3) & 1][(i >> 1) & 3][i & 1] = f4{0.f, 0.f, 0.f, 0.f};
  if (n <= 0) return;
  auto a_at = [n, &steps](int s) { return steps.a(s < n ? s : n - 1); };
  auto b_at = [n, &steps](int s) { return steps.b(s < n ? s : n - 1); };
  t256::fetch(src.a[0], a_at(0), a00);
  t256::fetch(src.b[0], b_at(0), b00);
  t256::fetch(src.b[1], b_at(0), b01);
  t256::fetch(src.a[1], a_at(0), a01);
  t256::fetch(src.a[0], a_at(1), a10);
  t256::fetch(src.b[0], b_at(1), b10);
  t256::fetch(src.b[1], b_at(1), b11);
  aside();
  t256::end_memory<3 * Tile256::kHalfLoads>();
  const bool behind = threadIdx.x >= 256;  // waves 4-7
  if (behind) t256::barrier();
  int s = 0;
  for (; s + 1 < n; s += 2) {
    t256::stage<T>(acc, src, a_at(s + 1), a_at(s + 2), b_at(s + 2), a00, a01, b00, b01, a11);
    t256::stage<T>(acc, src, a_at(s + 2), a_at(s + 3), b_at(s + 3), a10, a11, b10, b11, a01);
  }
  if (s < n)
    t256::stage<T>(acc, src, a_at(s + 1), a_at(s + 2), b_at(s + 2), a00, a01, b00, b01, a11);
  if (!behind) t256::barrier();
  // No load may still be writing LDS when the workgroup moves on.
  wait_vmcnt<0>();
  __syncthreads();
}

// Epilogue staging of 256 rows x 128 columns of fp32 through the eight buffers:
// 512 bytes a row, rows 32 h .. 32 h + 31 in buffer h; 16-byte column chunk c
// of row r at physical chunk c ^ (r & 31), free of bank conflicts for the
// MFMA-layout writes and the row-chunk reads.
__device__ inline char* t256_stage_row(char* l0, char* l1, char* l2, char* l3, char* l4, char* l5,
                                       char* l6, char* l7, int r) {
  const int h = r >> 5;
  char* lo = h & 2 ? (h & 1 ? l3 : l2) : (h & 1 ? l1 : l0);
  char* hi = h & 2 ? (h & 1 ? l7 : l6) : (h & 1 ? l5 : l4);
  return (h & 4 ? hi : lo) + (r & 31) * 512;
}

}  // namespace optima
