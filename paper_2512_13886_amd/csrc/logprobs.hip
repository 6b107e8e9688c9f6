// Log probabilities of given tokens, with the entropy and the most probable alternatives, and
// their gradient.
//
// With z = scale x over a row of the vocabulary, m = max x, y = scale (x - m), S = sum exp(y) and
// T = sum exp(y) y: lse = scale m + ln S, logp = scale (x_t - m) - ln S, H = ln S - T / S. S and T
// are kept for a running m, so that a row is read once; parts of a row (m, S, T) join to the
// whole's.
//
// The k largest come out of the same pass. Each thread keeps the largest of its values and the
// first group of eight that holds it; groups compare by value and then by their place. The k
// largest of a row lie in the k best threads' values (a value elsewhere has k larger ones before
// it), which are read again, and those that reach the k-th best thread's are ranked.
#include <type_traits>

#include "common.h"
#include "vec8.h"

namespace optima {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct LogprobArgs {
  const void* x;
  const int64_t* tokens;
  float *logp, *lse, *entropy, *top_logp;
  int64_t* top_index;
  float* stat;     // of parts: [row][part][m, S, T]
  uint64_t* keys;  // of parts: [row][part][k], largest first, 0 for none
  int64_t ldx, n, row0;  // row0: the launch's first row
  int vocab, k, parts, part_len;
  float scale;
};

// ---------------------------------------------------------------------------
// Values in their order: larger values, and of equal ones earlier places, have larger keys. -0 is
// 0, and NaN is -inf.
// ---------------------------------------------------------------------------

__device__ inline uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x == x ? x + 0.f : -__builtin_inff());
  return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ inline float value_of(uint32_t o) {
  return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

// v of another lane of the same 16: rotated by 8, 4, 2 and 1 lanes in turn, every lane gets a sum or
// maximum of all 16.
template <int CTRL>
__device__ inline uint32_t rotated(uint32_t v) {
  return uint32_t(__builtin_amdgcn_mov_dpp(int(v), CTRL, 0xF, 0xF, true));
}
constexpr int kBy8 = 0x128, kBy4 = 0x124, kBy2 = 0x122, kBy1 = 0x121;
template <int CTRL>
__device__ inline float rotated(float v) {
  return __uint_as_float(rotated<CTRL>(__float_as_uint(v)));
}
__device__ inline float lane_value(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
__device__ inline uint32_t wave_max(uint32_t v) {
  v = max(v, rotated<kBy8>(v));
  v = max(v, rotated<kBy4>(v));
  v = max(v, rotated<kBy2>(v));
  v = max(v, rotated<kBy1>(v));
  auto of = [v](int lane) { return uint32_t(__builtin_amdgcn_readlane(int(v), lane)); };
  return max(max(of(0), of(16)), max(of(32), of(48)));
}

__device__ inline float max3(float a, float b, float c) {
  // NaN loses. (The builtin maximum makes every operand canonical first, at an instruction each.)
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// ---------------------------------------------------------------------------
// S and T for a running m
// ---------------------------------------------------------------------------

struct Sums {
  float m, s, t;  // t in units of log 2: sum of 2^y y
};
// Of 2^((x - m) c) = exp(scale (x - m)); finite for every scale, so that the largest values have 2^0.
__device__ inline float exponent_scale(float scale) { return fminf(scale * kLog2e, 3.4028235e38f); }
// The reference of the exponents: any finite one for a row that has only -inf yet.
__device__ inline float finite_max(float m) { return m > -__builtin_inff() ? m : 0.f; }
// to the maximum m (not smaller). c: exponent_scale.
__device__ inline void rebase(Sums& a, float m, float c) {
  // Above 0 only from -inf, with sums of 0.
  const float d = fminf(fmaxf((finite_max(a.m) - finite_max(m)) * c, -1e30f), 0.f);
  const float r = __builtin_amdgcn_exp2f(d);
  a.t = r * (a.t + d * a.s);
  a.s *= r;
  a.m = m;
}
// Of the LANES (16 or 64) lanes of a row, in every lane (of 16, s and t in the first).
template <int LANES>
__device__ inline Sums lanes_sums(Sums a, float c) {
  float m = a.m;
  m = max3(m, rotated<kBy8>(m), m);
  m = max3(m, rotated<kBy4>(m), m);
  m = max3(m, rotated<kBy2>(m), m);
  m = max3(m, rotated<kBy1>(m), m);
  if constexpr (LANES == 64)
    m = max3(max3(lane_value(m, 0), lane_value(m, 16), lane_value(m, 32)), lane_value(m, 48), m);
  rebase(a, m, c);
  auto sum = [](float v) {
    v += rotated<kBy8>(v);
    v += rotated<kBy4>(v);
    v += rotated<kBy2>(v);
    v += rotated<kBy1>(v);
    if constexpr (LANES == 64)
      v = (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
    return v;
  };
  a.s = sum(a.s);
  a.t = sum(a.t);
  return a;
}

// The row's outputs of its sums, by one thread.
__device__ inline float logp_of(float x, const Sums& a, float scale) {
  return a.m == -__builtin_inff() && a.s == 0.f ? -__builtin_inff() : scale * (x - a.m) - logf(a.s);
}
template <typename T>
__device__ inline float value1(const T* p);
template <>
__device__ inline float value1(const float* p) { return *p; }
template <>
__device__ inline float value1(const bf16_t* p) { return bf16_low(p->bits); }

template <typename T>
__device__ inline void write_row(const LogprobArgs& a, int64_t row, const Sums& s) {
  // Nothing left of the row: lse and its log probabilities are -inf, its entropy 0.
  const bool none = s.m == -__builtin_inff() && s.s == 0.f;
  if (a.lse) a.lse[row] = none ? -__builtin_inff() : a.scale * s.m + logf(s.s);
  if (a.entropy) a.entropy[row] = none ? 0.f : logf(s.s) - s.t / s.s * kLn2;
  if (a.logp) {
    const int64_t t = a.tokens[row];
    float v = 0.f;
    if (t >= a.vocab)
      v = __builtin_nanf("");
    else if (t >= 0)
      v = logp_of(value1(static_cast<const T*>(a.x) + row * a.ldx + t), s, a.scale);
    a.logp[row] = v;
  }
}
__device__ inline void write_top(const LogprobArgs& a, int64_t row, int j, uint64_t key,
                                 const Sums& s) {
  const int64_t at = row * a.k + j;
  if (a.top_index) a.top_index[at] = int64_t(uint32_t(~uint32_t(key)));
  if (a.top_logp) a.top_logp[at] = logp_of(value_of(uint32_t(key >> 32)), s, a.scale);
}

// What lanes of a wave wrote to LDS before is there for its other lanes after.
__device__ inline void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
template <int LANES>
__device__ inline void group_sync() {
  if constexpr (LANES > 64)
    __syncthreads();
  else
    wave_exchange();
}

constexpr int kGroups = 4;         // of eight values that a thread loads together
constexpr int kTopSteps = 16;      // groups of a thread, at most, where alternatives are wanted
constexpr int kPartLen = kTopSteps * 256 * 8;

// How many of a wave's values, W a lane, are v or more.
template <int W>
__device__ inline int count_from(const uint32_t (&value)[W], uint32_t v) {
  int c = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) c += __builtin_popcountll(__builtin_amdgcn_ballot_w64(value[w] >= v));
  return c;
}
// A v that `need` of the values are or exceed, and no more unless they equal the last of them: its bits
// from `bit` (even) down to LOW, two at a time; `from` has those above. reach: how many reach v.
template <int LOW, int W>
__device__ inline uint32_t reached_by(const uint32_t (&value)[W], int need, uint32_t from, int bit,
                                      int& reach) {
  for (; bit >= LOW && reach != need; bit -= 2) {
    const int c1 = count_from(value, from | 1u << bit), c2 = count_from(value, from | 2u << bit);
    const int c3 = count_from(value, from | 3u << bit);
    const int more = (c1 >= need) + (c2 >= need) + (c3 >= need);
    from |= uint32_t(more) << bit;
    reach = more == 3 ? c3 : more == 2 ? c2 : more == 1 ? c1 : reach;
  }
  return from;
}

// What reaches the k best of the values `order` (0: none; LOW zero bits or as many ones in all of
// them) with their different places below 2^place_bits (even): a value, and with that value a place
// that is not later. With no more than k of them 0 is reached by all.
struct Border {
  uint32_t value, place;
  __device__ inline bool reached(uint32_t order, uint32_t at) const {
    return order > value || (order == value && at <= place);
  }
};
template <int LOW, int W>
__device__ inline Border border_of(const uint32_t (&order)[W], const uint32_t (&place)[W], int k,
                                   int place_bits) {
  Border r{0u, ~0u};
  int reach = count_from(order, 1u);
  if (reach <= k) return r;
  uint32_t most = 0, least = ~0u;
#pragma unroll
  for (int w = 0; w < W; ++w) most = max(most, order[w]), least = min(least, order[w] - 1);  // not of 0
  most = wave_max(most);
  least = ~wave_max(~least) + 1;
  const int bit = (31 - __builtin_clz((most ^ least) | 1)) & ~1;  // the highest that they differ in
  r.value = reached_by<LOW>(order, k, most & ~((4u << bit) - 1), bit, reach);
  if (LOW > 0 && !(r.value >> 31)) r.value |= (1u << LOW) - 1;  // a negative value's low bits
  if (reach > k) {  // equal ones: the earliest of them
    uint32_t equal[W];
    int above = 0;
    reach = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const bool is = order[w] == r.value;
      equal[w] = is ? (1u << place_bits) - place[w] : 0u;
      above += __builtin_popcountll(__builtin_amdgcn_ballot_w64(!is && order[w] > r.value));
      reach += __builtin_popcountll(__builtin_amdgcn_ballot_w64(is));
    }
    r.place = (1u << place_bits) - reached_by<0>(equal, k - above, 0u, place_bits, reach);
  }
  return r;
}

// The first k of `count` different keys in LDS, by LANES threads: each counts what is larger.
template <int LANES, typename F>
__device__ inline void ranked(const uint64_t* list, int count, int k, int t, F out) {
  for (int q = t; q < count; q += LANES) {
    const uint64_t key = list[q];
    int rank = 0;
#pragma unroll 4
    for (int r = 0; r < count; ++r) rank += list[r] > key;
    if (rank < k) out(rank, key);
  }
}

// Which of a workgroup's rows a thread has: the same for a wave of 64 or more, and known to be.
template <int LANES>
__device__ inline int row_of_thread() {
  if constexpr (LANES >= 256) return 0;
  const int sub = threadIdx.x / LANES;
  return LANES == 64 ? __builtin_amdgcn_readfirstlane(sub) : sub;
}

// A part of a row by LANES lanes (256: a workgroup; 64 and 16: more rows a workgroup). Bound by HBM's
// reads where there are many values: 8192 rows of 128000 in bf16 370 us, 5.7 TB/s, with about a dozen
// vector instructions a value beside them (8192 x 4000 17 us, 65536 x 100 11); by the latency of
// its steps for one row: 128000 values 6.6 us, 14.3 with 20 alternatives, 5 of which join the parts.
template <typename T, int LANES, bool TOP>
__global__ void __launch_bounds__(256) k_logprobs(LogprobArgs a, int list_len) {
  static_assert(!TOP || LANES >= 64, "alternatives are chosen by waves");
  constexpr int kStep = 8 * LANES, kSub = 256 / LANES, kWaves = LANES > 64 ? LANES / 64 : 1;
  constexpr int kLow = sizeof(T) == 2 ? 16 : 0;
  __shared__ float red[kWaves][3];
  __shared__ uint32_t best_of[TOP && LANES > 64 ? 256 : 1], base_of[TOP && LANES > 64 ? 256 : 1];
  __shared__ int chosen[kSub][OPTIMA_TOP_MAX];
  __shared__ Border borders[kSub];
  __shared__ int found[kSub], picked[kSub];
  extern __shared__ uint64_t lists[];
  const int sub = row_of_thread<LANES>(), t = threadIdx.x % LANES;
  const uint32_t task = blockIdx.x * kSub + sub, parts = a.parts;
  const int64_t row = a.row0 + task / parts;
  if (row >= a.n) return;  // all threads of the row
  const int part = int(task % parts), p0 = part * a.part_len;
  const int len = std::min(a.part_len, a.vocab - p0);
  const T* x = static_cast<const T*>(a.x) + row * a.ldx + p0;
  const float c = exponent_scale(a.scale);

  Sums s = {-__builtin_inff(), 0.f, 0.f};
  float best = -__builtin_inff();
  int base = 8 * t;
  // Groups from at0 on, of the `left` values that the row's lanes have before them.
  auto groups = [&](int at0, int left, auto whole) {
    Raw8<T> raw[kGroups];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      if (whole)
        load8(raw[u], x + at0 + u * kStep);
      else if (u * kStep < left)
        load_piece(raw[u], x, at0 + u * kStep, len);
    }
    float v[kGroups][8], m = s.m;
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      if (!whole && u * kStep >= left) break;
      values8(raw[u], v[u]);
      if (!whole && (u + 1) * kStep > left) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at0 + u * kStep + e >= len) v[u][e] = -__builtin_inff();
      }
      float g = max3(max3(v[u][0], v[u][1], v[u][2]), v[u][3], v[u][4]);
      g = max3(max3(g, v[u][5], v[u][6]), v[u][7], v[u][7]);
      if (TOP && g > best) {
        best = g;
        base = at0 + u * kStep;
      }
      m = max3(m, g, g);
    }
    if (m > s.m) rebase(s, m, c);
    const float ref = finite_max(m);
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      if (!whole && u * kStep >= left) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = (v[u][e] - ref) * c;
        const float p = __builtin_amdgcn_exp2f(y);
        s.s += p;
        s.t += p * max3(y, -1e4f, -1e4f);  // 0 for p = 0; NaN comes in by p
      }
    }
  };
  int at = 8 * t, left = len;
  for (; left >= kGroups * kStep; left -= kGroups * kStep, at += kGroups * kStep)
    groups(at, left, std::true_type());
  if (left > 0) groups(at, left, std::false_type());

  s = lanes_sums<(LANES < 64 ? LANES : 64)>(s, c);
  if constexpr (LANES > 64) {
    const int wave = threadIdx.x >> 6;
    if ((t & 63) == 0) red[wave][0] = s.m, red[wave][1] = s.s, red[wave][2] = s.t;
    __syncthreads();
    float m = red[0][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = max3(m, red[w][0], m);
    Sums all = {m, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      Sums one = {red[w][0], red[w][1], red[w][2]};
      rebase(one, m, c);
      all.s += one.s;
      all.t += one.t;
    }
    s = all;
  }
  if (t == 0) {
    if (a.parts == 1) {
      write_row<T>(a, row, s);
    } else {
      float* to = a.stat + (row * a.parts + part) * 3;
      to[0] = s.m, to[1] = s.s, to[2] = s.t;
    }
  }
  if constexpr (TOP) {
    const uint32_t mine = 8 * t < len ? order_of(best) : 0u, from = uint32_t(base) >> 3;
    if constexpr (LANES > 64) {
      best_of[t] = mine;
      base_of[t] = from;
      __syncthreads();
    }
    if (t < 64) {
      uint32_t order[kWaves], place[kWaves];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        order[w] = LANES > 64 ? best_of[t + 64 * w] : mine;
        place[w] = LANES > 64 ? base_of[t + 64 * w] : from;
      }
      const Border r = border_of<kLow>(order, place, a.k, 12);
      static_assert(kPartLen / 8 <= 4096, "places of groups");
      int at = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const bool in = order[w] > 0 && r.reached(order[w], place[w]);
        const uint64_t mask = __builtin_amdgcn_ballot_w64(in);
        if (in) chosen[sub][at + __popcll(mask & ((uint64_t(1) << t) - 1))] = t + 64 * w;
        at += __popcll(mask);
      }
      if (t == 0) {
        found[sub] = 0;
        picked[sub] = at;
        borders[sub] = r;
      }
    }
    group_sync<LANES>();
    const Border limit = borders[sub];
    uint64_t* list = lists + sub * list_len;
    const int steps = (len + kStep - 1) / kStep, tasks = picked[sub] * steps;
    for (int q = t; q < tasks; q += LANES) {
      const int j = q / steps, g = 8 * chosen[sub][j] + (q - j * steps) * kStep;
      if (g >= len) continue;
      Raw8<T> r;
      load_piece(r, x, g, len);
      float v[8];
      values8(r, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t o = order_of(v[e]);
        if (g + e < len && limit.reached(o, uint32_t(g) >> 3))
          list[atomicAdd(&found[sub], 1)] = uint64_t(o) << 32 | uint32_t(~uint32_t(p0 + g + e));
      }
    }
    group_sync<LANES>();
    const int count = found[sub];
    uint64_t* to = a.keys + (row * a.parts + part) * a.k;
    ranked<LANES>(list, count, a.k, t, [&](int rank, uint64_t key) {
      if (a.parts == 1)
        write_top(a, row, rank, key, s);
      else
        to[rank] = key;
    });
    if (a.parts > 1)
      for (int q = count + t; q < a.k; q += LANES) to[q] = 0;
  }
}

// The parts of a row, by LANES threads (64 or 256): lane p of each wave has the sums of part p and
// the m-th of its keys, which are sorted: m keys of k / m parts reach the k / m best of these (both
// rounded up). Of all keys those that do are ranked; m is such that half of the parts do, not all. The
// keys come from other XCDs, so that all loads of a thread go out together.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) k_logprobs_join(LogprobArgs a) {
  constexpr int kSub = 256 / LANES, kEach = LANES > 64 ? 8 : 4, kLow = sizeof(T) == 2 ? 16 : 0;
  extern __shared__ uint64_t lists[];
  __shared__ int found[kSub];
  const int sub = row_of_thread<LANES>(), t = threadIdx.x % LANES, lane = threadIdx.x & 63;
  const int64_t row = a.row0 + int64_t(blockIdx.x) * kSub + sub;
  if (row >= a.n) return;
  const float c = exponent_scale(a.scale);
  const int keys = a.parts * a.k;
  const uint64_t* all = a.keys + row * keys;
  uint64_t key[kEach] = {}, mth = 0;
  const int m = a.k ? std::min((2 * a.k + a.parts - 1) / a.parts, a.k) : 1;
  if (a.k)
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (t + i * LANES < keys) key[i] = all[t + i * LANES];
  Sums s = {-__builtin_inff(), 0.f, 0.f};
  if (lane < a.parts) {
    const float* p = a.stat + (row * a.parts + lane) * 3;
    s = Sums{p[0], p[1], p[2]};
    if (a.k) mth = all[lane * a.k + m - 1];
  }
  if (t == 0) found[sub] = 0;
  s = lanes_sums<64>(s, c);
  if (t == 0) write_row<T>(a, row, s);
  if (!a.k) return;
  const uint32_t order[1] = {uint32_t(mth >> 32)}, place[1] = {~uint32_t(mth)};
  const Border limit = border_of<kLow>(order, place, (a.k + m - 1) / m, 20);
  group_sync<LANES>();
  uint64_t* list = lists + sub * keys;
  for (int q = 0;;) {
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (key[i] && limit.reached(uint32_t(key[i] >> 32), ~uint32_t(key[i])))
        list[atomicAdd(&found[sub], 1)] = key[i];
    q += kEach * LANES;
    if (q >= keys) break;
#pragma unroll
    for (int i = 0; i < kEach; ++i) key[i] = q + t + i * LANES < keys ? all[q + t + i * LANES] : 0;
  }
  group_sync<LANES>();
  ranked<LANES>(list, found[sub], a.k, t,
                [&](int rank, uint64_t best) { write_top(a, row, rank, best, s); });
}

struct LogprobGradArgs {
  const void* x;
  const int64_t* tokens;
  const float *lse, *entropy, *dlogp, *dentropy, *dlse;
  void* dx;
  int64_t ldx, lddx, n, row0;
  int vocab, parts;
  float scale;
};

// p = exp(z - lse) has the error of lse, |lse| 2^-24 at least. Past this |lse| (2^-16 of p) it comes from
// the row itself: z - lse = scale (x - m) - ln S.
constexpr float kFarLse = 256.f;

// m and S (in every lane) of a row of the gradient, read again.
template <typename T, int LANES>
__device__ inline Sums row_sums(const T* x, int vocab, int t, float c) {
  constexpr int kStep = 8 * LANES, kMany = LANES > 64 ? kGroups / 2 : 1;
  Sums s = {-__builtin_inff(), 0.f, 0.f};
  for (int at = 8 * t; at - 8 * t < vocab; at += kMany * kStep) {
    Raw8<T> raw[kMany];
#pragma unroll
    for (int u = 0; u < kMany; ++u) load_piece(raw[u], x, at + u * kStep, vocab);
#pragma unroll
    for (int u = 0; u < kMany; ++u) {
      float v[8], m = s.m;
      values8(raw[u], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (at + u * kStep + e >= vocab) v[e] = -__builtin_inff();
        m = max3(m, v[e], v[e]);
      }
      if (m > s.m) rebase(s, m, c);
      const float ref = finite_max(m);
#pragma unroll
      for (int e = 0; e < 8; ++e) s.s += __builtin_amdgcn_exp2f((v[e] - ref) * c);
    }
  }
  s = lanes_sums<(LANES < 64 ? LANES : 64)>(s, c);
  if constexpr (LANES < 64) s.s = __shfl(s.s, 0, LANES);
  if constexpr (LANES > 64) {
    __shared__ float red[LANES / 64][2];
    if ((t & 63) == 0) red[t >> 6][0] = s.m, red[t >> 6][1] = s.s;
    __syncthreads();
    float m = red[0][0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) m = max3(m, red[w][0], m);
    Sums all = {m, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) {
      Sums one = {red[w][0], red[w][1], 0.f};
      rebase(one, m, c);
      all.s += one.s;
    }
    s = all;
  }
  return s;
}

// dx = scale (g at the token + p (dlse - g - dH (ln p + H))), p = exp(z - lse). A thread loads its 32
// values before it uses any. Bound by HBM: 4096 x 128000 in bf16, read and written, 399 us, 5.3 TB/s, the
// rate of a copy; 65536 x 100 11.5 us. 301 x 50001 fp32 out of wider rows takes 23 us (5.3 TB/s).
// A row of large |lse| is one workgroup's alone, which reads all of it before it writes any: where all
// rows are such, 4096 x 128000 takes 716 us, one row of 128000 44 in place of 8.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) k_logprobs_grad(LogprobGradArgs a) {
  constexpr int kStep = 8 * LANES, kSub = 256 / LANES;
  const int sub = row_of_thread<LANES>(), t = threadIdx.x % LANES;
  const uint32_t task = blockIdx.x * kSub + sub, parts = a.parts;
  const int64_t row = a.row0 + task / parts;
  if (row >= a.n) return;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  T* dx = static_cast<T*>(a.dx) + row * a.lddx;
  Raw8<T> raw[kGroups];
  auto load = [&](int part) {
    const int first = part * kGroups * kStep;
#pragma unroll
    for (int u = 0; u < kGroups; ++u)
      if (first + u * kStep < a.vocab) load_piece(raw[u], x, first + 8 * t + u * kStep, a.vocab);
  };
  const int own_part = int(task % parts);
  const float lse = a.lse[row];
  const int64_t token = a.tokens ? a.tokens[row] : -1;
  float g = a.dlogp && token >= 0 ? a.dlogp[row] : 0.f;
  if (token >= a.vocab) g = __builtin_nanf("");
  const float gh = a.dentropy ? a.dentropy[row] : 0.f, h = a.dentropy ? a.entropy[row] : 0.f;
  const float gl = (a.dlse ? a.dlse[row] : 0.f) - g;
  // Nothing left of the row: no gradient. A row of the lowest finite value counts as such.
  const bool none = lse < -1e30f;
  // The loaded part's gradient, ln p = scale (x - ref) - rest.
  auto store = [&](int part, float ref, float rest) {
    const int at0 = part * kGroups * kStep + 8 * t;
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      const int at = at0 + u * kStep;
      if (at >= a.vocab) break;
      float v[8];
      values8(raw[u], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float lp = (v[e] - ref) * a.scale - rest;
        const float p = __builtin_amdgcn_exp2f(lp * kLog2e);
        float d = p * (gl - gh * (max3(lp, -1e4f, -1e4f) + h));
        if (at + e == token) d += g;
        v[e] = none ? 0.f : d * a.scale;
      }
      store_upto8(dx + at, v, a.vocab - at);
    }
  };
  if (!none && (lse > kFarLse || lse < -kFarLse)) {
    // Neighbouring rows take different places of theirs, which are on different XCDs.
    if (own_part != int(uint32_t(row) % parts)) return;
    const Sums s = row_sums<T, LANES>(x, a.vocab, t, exponent_scale(a.scale));
    // Not where the caller's lse is of more than this row: then it counts as it is.
    const float ln = logf(s.s), own = a.scale * s.m + ln;
    const bool is = own == lse || fabsf(own - lse) <= fabsf(lse) * 0x1p-22f;
    for (int part = 0; part < int(parts); ++part) {
      load(part);
      store(part, is ? s.m : 0.f, is ? ln : lse);
    }
    return;
  }
  load(own_part);
  store(own_part, 0.f, lse);
}

constexpr int64_t kMostTasks = int64_t(1) << 22;  // of a launch, in workgroups

// Lanes of a row: 16 for up to 128 values without alternatives, a wave, or a workgroup.
//
// Parts of a workgroup's row: for few rows as many as give every second CU a workgroup, of 8192
// values at least, since the join is a launch (one row of 128000 14.6 us in one part, 6.6 in 15; 100
// of 9000 with 5 alternatives 9 and 13 in two), or of 16384 bf16 ones with alternatives, whose search
// takes as long for fewer (64 rows of 32000 with 20 15.3 to 13.4, one of 20000 with 5 11.1 to 8.8; but one
// of 128000 in fp32 with 32 14.9 to 17.5); of 16384 where the last rows would otherwise leave CUs
// idle for long (8192 rows of 128000 420 us in one, 370 in seven); and of kPartLen at most with
// alternatives, whose groups of eight have places below 4096 and whose list (k ceil(len / 2048) 64 bytes
// of LDS, 32 KB at k = 32) is kept for a part.
struct LogprobPlan {
  int lanes, parts, len;
};
constexpr int64_t kFewRows = 512, kFewLen = 8192, kManyValues = int64_t(1) << 29, kManyLen = 16384;
LogprobPlan plan(int64_t n, int64_t vocab, int k, int dtype) {
  if (vocab <= 128 && !k) return {16, 1, int(vocab)};
  if (vocab <= (n >= 4096 ? 8192 : 2048)) return {64, 1, int(vocab)};
  const int64_t least = k && dtype == OPTIMA_DTYPE_BF16 ? 2 * kFewLen : kFewLen;
  int64_t parts = std::min<int64_t>({kFewRows / std::max<int64_t>(n, 1), vocab / least, 64});
  if (n * vocab >= kManyValues) parts = std::max(parts, vocab / kManyLen);
  if (k) parts = std::max(parts, ceil_div(vocab, kPartLen));
  const int64_t len = round_up(ceil_div(vocab, std::max<int64_t>(parts, 1)), 8);
  return {256, int(ceil_div(vocab, len)), int(len)};
}

template <typename T, int LANES, bool TOP>
void launch_logprobs(LogprobArgs a, hipStream_t s) {
  constexpr int kSub = 256 / LANES;
  const int64_t rows = kMostTasks * kSub / a.parts;
  const int list = a.k * int(ceil_div(a.part_len, 8 * LANES)) * 8;
  for (; a.row0 < a.n; a.row0 += rows) {
    const int64_t now = std::min(a.n - a.row0, rows);
    LogprobArgs b = a;
    b.n = a.row0 + now;
    hipLaunchKernelGGL((k_logprobs<T, LANES, TOP>), dim3(unsigned(ceil_div(now * a.parts, kSub))),
                       dim3(256), size_t(list) * kSub * 8, s, b, list);
    const size_t keys = size_t(a.parts) * size_t(a.k) * 8;
    if (a.parts > 1 && keys > 2048)
      hipLaunchKernelGGL((k_logprobs_join<T, 256>), dim3(unsigned(now)), dim3(256), keys, s, b);
    else if (a.parts > 1)
      hipLaunchKernelGGL((k_logprobs_join<T, 64>), dim3(unsigned(ceil_div(now, 4))), dim3(256), 4 * keys,
                         s, b);
  }
}
template <typename T>
void launch_logprobs(const LogprobArgs& a, int lanes, hipStream_t s) {
  if (lanes == 16) launch_logprobs<T, 16, false>(a, s);
  else if (lanes == 64 && a.k) launch_logprobs<T, 64, true>(a, s);
  else if (lanes == 64) launch_logprobs<T, 64, false>(a, s);
  else if (a.k) launch_logprobs<T, 256, true>(a, s);
  else launch_logprobs<T, 256, false>(a, s);
}

template <typename T, int LANES>
void launch_grad(LogprobGradArgs a, hipStream_t s) {
  constexpr int kSub = 256 / LANES;
  a.parts = int(ceil_div(a.vocab, kGroups * 8 * LANES));
  const int64_t rows = std::max<int64_t>(1, kMostTasks * kSub / a.parts);
  for (; a.row0 < a.n; a.row0 += rows) {
    LogprobGradArgs b = a;
    b.n = std::min(a.n, a.row0 + rows);
    hipLaunchKernelGGL((k_logprobs_grad<T, LANES>),
                       dim3(unsigned(ceil_div((b.n - a.row0) * a.parts, kSub))), dim3(256), 0, s, b);
  }
}
// The gradient's lanes of a row.
template <typename T>
void launch_grad(const LogprobGradArgs& a, hipStream_t s) {
  if (a.vocab <= 256) launch_grad<T, 16>(a, s);
  else if (a.vocab <= 2048) launch_grad<T, 64>(a, s);
  else launch_grad<T, 256>(a, s);
}

}  // namespace

size_t token_logprobs_workspace_bytes(int64_t n, int64_t vocab, int64_t k) {
  // The parts of any number of rows up to these, so that more need no less.
  int64_t parts = std::min(n, kFewRows) * (vocab / kFewLen);
  parts = std::min(parts, kFewRows);
  if (n * vocab >= kManyValues) parts = std::max(parts, n * (vocab / kManyLen));
  if (k && vocab > kPartLen) parts = std::max(parts, n * ceil_div(vocab, kPartLen));
  return size_t(parts) * size_t(12 + 8 * k);
}

optima_status token_logprobs(const void* X, int64_t ldx, int dtype, int64_t n, int64_t vocab,
                             const int64_t* tokens, float scale, float* logp, float* lse,
                             float* entropy, int64_t k, int64_t* top_index, float* top_logp,
                             void* ws, hipStream_t s) {
  const LogprobPlan p = plan(n, vocab, int(k), dtype);
  uint64_t* keys = static_cast<uint64_t*>(ws);
  float* stat = keys ? reinterpret_cast<float*>(keys + size_t(n) * p.parts * size_t(k)) : nullptr;
  LogprobArgs a{X, tokens, logp, lse, entropy, top_logp, top_index, stat, keys, ldx, n, 0,
                int(vocab), int(k), p.parts, p.len, scale};
  if (dtype == OPTIMA_DTYPE_BF16) launch_logprobs<bf16_t>(a, p.lanes, s);
  else launch_logprobs<float>(a, p.lanes, s);
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

optima_status token_logprobs_backward(const void* X, int64_t ldx, int dtype, int64_t n,
                                      int64_t vocab, const int64_t* tokens, float scale,
                                      const float* lse, const float* entropy, const float* dlogp,
                                      const float* dentropy, const float* dlse, void* dX,
                                      int64_t lddx, hipStream_t s) {
  LogprobGradArgs a{X, tokens, lse, entropy, dlogp, dentropy, dlse, dX, ldx, lddx, n, 0,
                    int(vocab), 0, scale};
  if (dtype == OPTIMA_DTYPE_BF16) launch_grad<bf16_t>(a, s);
  else launch_grad<float>(a, s);
  OPTIMA_LAUNCH_CHECK();
  return OPTIMA_OK;
}

}  // namespace optima
