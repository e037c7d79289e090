// Distributions cut by temperature, top-k, top-p and min-p: a token drawn from a given random number, or the scores without what is cut off.
//
// A row has scores x, m = max x, weights w = 2^((x - m) rate), rate = log2(e) / T.  In order of falling score, equal ones by rising index, the first k stay; of them the
// least number whose weights sum to p of theirs or more (one at least); of them those with w >= min_p.  So what stays is a front of that order: everything before a border
// (score, index).  The drawn token is the least index whose weights up to it, of what stays, exceed u of all of that.
//
// Weights are whole numbers of 2^-S, S = min(51, 62 - log2 of the vocabulary): w is rounded to nearest and to 1 at least (what a double has no number for is 0), and all of a
// row sum to less than 2^63.  Whole sums are exact, so neither atomics nor the launch's shape change a border or a token, and p Z and u Z are compared exactly.  What rounding moves a border by,
// 2^-S a token, is some 10^-12 of the sum at most: a drawn number falls there once in 10^8 draws.
//
// One workgroup a row.  A border is found by histograms: of all scores in steps of T / 16 below the maximum, then, of the step that holds it, of equal parts of the
// floating point numbers between its least and its largest, until few enough are left to be ranked by comparing each with each, or all are equal and their indices decide.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "ad_device.h"
#include "ad_truncate.h"

namespace ad {

typedef unsigned long long u64;

constexpr int kBins = 1024;   // of a histogram
constexpr int kList = 256;    // scores that are ranked by comparing each with each

template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ u64 dpp_move_u64(u64 v) {
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true), hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, true);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 lane_u64(u64 v, int lane) {
  return (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}
// sums over lanes up to this one
__device__ __forceinline__ u64 wave_scan_u64(u64 v) {
  v += dpp_move_u64<0x111>(v);
  v += dpp_move_u64<0x112>(v);
  v += dpp_move_u64<0x114>(v);
  v += dpp_move_u64<0x118>(v);
  v += dpp_move_u64<0x142, 0xa>(v);
  v += dpp_move_u64<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ u64 wave_sum_u64(u64 v) { return lane_u64(wave_scan_u64(v), 63); }

// floor(f z) and ceil(f z), exactly, for 0 <= f < 1
__device__ __forceinline__ unsigned __int128 part_of(float f, u64 z, int& shift) {
  int e;
  const unsigned m = (unsigned)(frexpf(f, &e) * 16777216.f);
  shift = 24 - e;
  return (unsigned __int128)m * z;   // < 2^87
}
__device__ __forceinline__ u64 floor_part(float f, u64 z) {
  int s;
  const unsigned __int128 v = part_of(f, z, s);
  return s > 100 ? 0 : (u64)(v >> s);
}
__device__ __forceinline__ u64 ceil_part(float f, u64 z) {
  int s;
  const unsigned __int128 v = part_of(f, z, s);
  if (s > 100) return v != 0;
  return (u64)((v + (((unsigned __int128)1 << s) - 1)) >> s);
}

// what stays so far: scores above x, and those equal to x up to index i
struct Border {
  float x;
  int i;
  __device__ __forceinline__ bool holds(float v, int at) const { return (v > x) | ((v == x) & (at <= i)); }
};

// floats in their order as whole numbers, -0 as 0
__device__ __forceinline__ unsigned order_of(float v) {
  const unsigned b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A row's weights
struct Weigh {
  float m;
  double rate, least;   // least: 2's exponent of min_p (-inf: none)
  int bits;             // S
  __device__ __forceinline__ double power(float v) const { return ((double)v - (double)m) * rate; }   // (the difference is exact; at temperatures near 0 a rounded product would not do)
  // 2^(t + S) for t <= 0 in whole numbers: 2^f, |f| <= 1/2, by its series to f^11 (7e-15 relative), the whole part straight into the exponent
  __device__ __forceinline__ u64 of(double t) const {
    const double c = fmax(t, -100.0), big = c + 6755399441055744.0, f = c - (big - 6755399441055744.0);
    double p = 4.44553827187081149760e-10;   // ln(2)^k / k!, k = 11 .. 0
    p = fma(p, f, 7.05491162080112332988e-9);
    p = fma(p, f, 1.01780860092396997275e-7);
    p = fma(p, f, 1.32154867901443094884e-6);
    p = fma(p, f, 1.52527338040598402800e-5);
    p = fma(p, f, 1.54035303933816099544e-4);
    p = fma(p, f, 1.33335581464284434234e-3);
    p = fma(p, f, 9.61812910762847716197e-3);
    p = fma(p, f, 5.55041086648215799532e-2);
    p = fma(p, f, 2.40226506959100712334e-1);
    p = fma(p, f, 6.93147180559945309417e-1);
    p = fma(p, f, 1.0);
    const long long b = __builtin_bit_cast(long long, p);
    const unsigned hi = (unsigned)(b >> 32) + ((unsigned)(__builtin_bit_cast(long long, big) + bits) << 20);
    const double w = __builtin_bit_cast(double, (long long)((u64)hi << 32 | (unsigned)b));   // <= 2^51
    const u64 n = __builtin_bit_cast(u64, w + 4503599627370496.0) & 0xfffffffffffffull;     // (to nearest)
    return t < -1074.0 ? 0 : n < 1 ? 1 : n;
  }
};

// A row's scores, 16 bytes at a time from the 16-byte boundary at or before the first: wave w of a workgroup has pieces (w per .. (w + 1) per - 1) of 64 vectors, a lane one of each
template <typename T, int THREADS> struct TruncateRow {
  static constexpr int kVec = 16 / (int)sizeof(T), kWaves = THREADS / 64;
  const T* x;
  int vocab, skew, per, first;   // per: vectors of a lane; first: this lane's first one
  __device__ __forceinline__ TruncateRow(const TruncateArgs& a, int row) {
    x = (const T*)a.x + (size_t)row * a.stride;
    vocab = a.vocab;
    skew = (int)((uintptr_t)x & 15) / (int)sizeof(T);
    per = ((vocab + skew + kVec - 1) / kVec + THREADS - 1) / THREADS;
    first = (int)(threadIdx.x >> 6) * per * 64 + (int)(threadIdx.x & 63);
  }
  __device__ __forceinline__ int index(int c) const { return (first + 64 * c) * kVec - skew; }   // of vector c's first score
  __device__ __forceinline__ bool whole(int i) const { return i >= 0 && i + kVec <= vocab; }
  // (-inf off the row)
  __device__ __forceinline__ void load(int c, float (&v)[kVec]) const {
    const int i = index(c);
    if (whole(i)) {
      const uint4 w = ldg16(x + i);
      if constexpr (sizeof(T) == 4) {
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
      } else {
        v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u); v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
        v[4] = __uint_as_float(w.z << 16); v[5] = __uint_as_float(w.z & 0xffff0000u); v[6] = __uint_as_float(w.w << 16); v[7] = __uint_as_float(w.w & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = i + e >= 0 && i + e < vocab ? Store<T>::load(x + i + e) : -INFINITY;
    }
  }
  template <typename F> __device__ __forceinline__ void each(const F& f) const {   // f(score, index) over this thread's
    for (int c = 0; c < per; ++c) {
      float v[kVec];
      load(c, v);
#pragma unroll
      for (int e = 0; e < kVec; ++e) f(v[e], index(c) + e);
    }
  }
};

template <int THREADS> struct TruncateShared {
  u64 hist[kBins];
  u64 part[THREADS / 64];
  float lo[THREADS / 64], hi[THREADS / 64];
  float list_x[kList];
  int list_i[kList];
  u64 list_w[kList];
  u64 above;      // before the bin that holds the border
  int bin, n;
  Border border;
  float found_x;
};

// The least index whose f(score, index) up to it sum to want(sum of all) or more; thread by thread in the row's order, so the winning wave looks for it alone.  Left in
// s.border: its score and index.
template <typename T, int THREADS, typename F, typename W>
__device__ __forceinline__ u64 truncate_find(TruncateShared<THREADS>& s, const TruncateRow<T, THREADS>& x, const F& f, const W& want) {
  constexpr int kWaves = THREADS / 64, kVec = TruncateRow<T, THREADS>::kVec;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  u64 sum = 0;
  x.each([&](float v, int i) { sum += f(v, i); });
  sum = wave_sum_u64(sum);
  __syncthreads();
  if (lane == 0) s.part[wave] = sum;
  __syncthreads();
  u64 before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const u64 p = s.part[w];
    if (w < wave) before += p;
    all += p;
  }
  const u64 target = want(all);
  if (before < target && before + sum >= target) {   // (one wave)
    for (int c = 0; c < x.per; ++c) {
      float v[kVec];
      u64 e[kVec], own = 0;
      x.load(c, v);
#pragma unroll
      for (int j = 0; j < kVec; ++j) { e[j] = f(v[j], x.index(c) + j); own += e[j]; }
      const u64 up = wave_scan_u64(own), total = lane_u64(up, 63);
      if (before + total < target) {
        before += total;
        continue;
      }
      u64 at = before + up - own;
      if (at < target && at + own >= target) {   // (one lane)
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
          if (at < target && at + e[j] >= target) s.border = Border{v[j], x.index(c) + j};
          at += e[j];
        }
      }
      break;
    }
  }
  __syncthreads();
  return all;
}

// The border of the least front of what `had` holds that sums to the target (its own part of it: `had` itself).  WEIGHTS: sums of weights, target part p of
// all of them; else of ones, target k.
template <bool WEIGHTS, typename T, int THREADS>
__device__ __forceinline__ Border truncate_select(TruncateShared<THREADS>& s, const TruncateRow<T, THREADS>& x, const Weigh& weigh, const Border& had, float p, int k) {
  constexpr int kWaves = THREADS / 64, kEach = kBins / THREADS;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  auto one = [&](float v) -> u64 { return WEIGHTS ? weigh.of(weigh.power(v)) : 1; };
  float lo = -INFINITY, hi = weigh.m;    // the scores among which the border lies
  const float step = fminf(fmaxf((float)(weigh.rate * (16 * 0.69314718055994530942)), 1e-30f), 1e30f);
  u64 above = 0, target = k;
  for (bool top = true;; top = false) {
    int shift = 0;
    if (!top) shift = max(0, 32 - __clz(order_of(hi) - order_of(lo)) - 10);
    auto bin_of = [&](float v) -> int {
      return top ? (int)fminf((weigh.m - v) * step, (float)(kBins - 1)) : (int)((order_of(hi) - order_of(v)) >> shift);
    };
    auto here = [&](float v, int i) { return v >= lo && v <= hi && had.holds(v, i); };
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j) s.hist[t + j * THREADS] = 0;
    if (t == 0) { s.n = 0; s.bin = -1; }
    __syncthreads();
    x.each([&](float v, int i) {
      if (here(v, i)) atomicAdd(&s.hist[bin_of(v)], one(v));
    });
    __syncthreads();
    u64 own = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) own += s.hist[t * kEach + j];
    const u64 up = wave_scan_u64(own);
    if (lane == 63) s.part[wave] = up;
    __syncthreads();
    u64 at = above + up - own, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const u64 q = s.part[w];
      if (w < wave) at += q;
      all += q;
    }
    if (top) {
      if constexpr (WEIGHTS) target = max(ceil_part(fmaxf(p, 0.f), all), (u64)1);
      else if (all <= target) return had;   // (uniform: no more than k)
    }
    if (at < target && at + own >= target) {
      for (int j = 0; j < kEach; ++j) {
        const u64 h = s.hist[t * kEach + j];
        if (at < target && at + h >= target) { s.bin = t * kEach + j; s.above = at; }
        at += h;
      }
    }
    __syncthreads();
    const int bin = s.bin;
    above = s.above;
    // that bin's scores
    float least = INFINITY, most = -INFINITY;
    x.each([&](float v, int i) {
      if (here(v, i) && bin_of(v) == bin) {
        least = fminf(least, v); most = fmaxf(most, v);
        const int n = atomicAdd(&s.n, 1);
        if (n < kList) { s.list_x[n] = v; s.list_i[n] = i; s.list_w[n] = one(v); }
      }
    });
    least = -wave_max(-least); most = wave_max(most);
    if (lane == 0) { s.lo[wave] = least; s.hi[wave] = most; }
    __syncthreads();
    const int n = s.n;
    if (n <= kList) {
      for (int r = t; r < n; r += THREADS) {
        const float v = s.list_x[r];
        const int i = s.list_i[r];
        u64 up = above;
        for (int j = 0; j < n; ++j)
          if (Border{v, i}.holds(s.list_x[j], s.list_i[j])) up += s.list_w[j];
        if (up >= target && up - s.list_w[r] < target) s.border = Border{v, i};
      }
      __syncthreads();
      return s.border;
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { least = fminf(least, s.lo[w]); most = fmaxf(most, s.hi[w]); }
    lo = least; hi = most;
    if (lo == hi) {
      const u64 each = one(lo), nth = (target - above + each - 1) / each;
      truncate_find(s, x, [&](float v, int i) -> u64 { return v == lo && had.holds(v, i); }, [&](u64) { return nth; });
      return s.border;
    }
  }
}

// the sequence of packed row `row` (-1: none): the last one that starts there or before, found by each wave for itself: every 64th start at once, then those between two of them
__device__ __forceinline__ int truncate_owner(const TruncateArgs& a, int row) {
  if (!a.row_start) return row;
  const int lane = threadIdx.x & 63, apart = (a.n_seq + 63) / 64;
  int q = __popcll(__ballot(lane * apart < a.n_seq && a.row_start[min(lane * apart, a.n_seq - 1)] <= row)) - 1;
  if (q < 0) return -1;
  q *= apart;
  if (apart > 1) q += __popcll(__ballot(lane < apart && q + lane < a.n_seq && a.row_start[min(q + lane, a.n_seq - 1)] <= row)) - 1;
  return q >= 0 && a.row_start[q] <= row && row < a.row_start[q + 1] ? q : -1;
}

template <typename T, int THREADS, bool SAMPLE>
__global__ __launch_bounds__(THREADS) void k_truncate(TruncateArgs a) {
  __shared__ TruncateShared<THREADS> s;
  constexpr int kWaves = THREADS / 64, kVec = 16 / (int)sizeof(T);
  const int row = blockIdx.x, t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int b = truncate_owner(a, row);
  if (b < 0) return;
  const TruncateRow<T, THREADS> x(a, row);
  const float temp = a.temperature ? a.temperature[b] : 1.f, top_p = a.top_p ? a.top_p[b] : 1.f, min_p = a.min_p ? a.min_p[b] : 0.f;
  const int top_k = a.top_k ? a.top_k[b] : 0;
  float m = -INFINITY;
  bool bad = !(temp > 0.f && temp < INFINITY) || top_p != top_p || min_p != min_p;
  x.each([&](float v, int) {
    bad = bad || !(v < INFINITY);
    m = fmaxf(m, v);
  });
  m = wave_max(m);
  if (lane == 0) s.hi[wave] = m;
  bad = __syncthreads_or(bad);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s.hi[w]);
  bad = bad || m == -INFINITY;   // no distribution
  Border border{bad ? INFINITY : -INFINITY, -1};
  Weigh weigh{m, 1.44269504088896340736 / (double)temp, -INFINITY, min(51, 62 - (32 - __clz(a.vocab)))};
  if (!bad) {
    if (top_k > 0 && top_k < a.vocab) border = truncate_select<false>(s, x, weigh, border, 0.f, top_k);
    if (top_p < 1.f) border = truncate_select<true>(s, x, weigh, border, top_p, 0);
    if (min_p > 0.f) weigh.least = log2((double)fminf(min_p, 1.f));
  }
  if constexpr (SAMPLE) {
    if (bad) {
      if (t == 0) {
        a.tokens[row] = AD_NEVER;
        if (a.log_probs) a.log_probs[row] = __uint_as_float(0x7fc00000u);
      }
      return;
    }
    const float u = a.u[row];
    const u64 all = truncate_find(
        s, x,
        [&](float v, int i) -> u64 {
          if (!border.holds(v, i)) return 0;
          const double power = weigh.power(v);
          return power >= weigh.least ? weigh.of(power) : 0;
        },
        [&](u64 z) { return !(u > 0.f) ? (u64)1 : u >= 1.f ? z : floor_part(u, z) + 1; });
    if (t == 0) {
      a.tokens[row] = s.border.i;
      if (a.log_probs) a.log_probs[row] = (float)((weigh.power(s.border.x) + (double)weigh.bits) * 0.69314718055994530942 - log((double)all));
    }
  } else {
    T* out = (T*)a.out + (size_t)row * a.out_stride;
    const bool wide = (((uintptr_t)out ^ (uintptr_t)x.x) & 15) == 0;
    for (int c = 0; c < x.per; ++c) {
      float v[kVec];
      x.load(c, v);
      const int i = x.index(c);
      // (selected without a branch: the compiler lost the -inf of a branch's other side)
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        const bool stays = border.holds(v[j], i + j) & (weigh.power(v[j]) >= weigh.least);
        v[j] = __uint_as_float(stays ? __float_as_uint(v[j]) : 0xff800000u);
      }
      if (wide && x.whole(i)) {
        uint4 w;
        if constexpr (sizeof(T) == 4) {
          w = uint4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        } else {   // (every value is a bf16 number)
          auto two = [&](int j) { return __float_as_uint(v[j]) >> 16 | (__float_as_uint(v[j + 1]) & 0xffff0000u); };
          w = uint4{two(0), two(2), two(4), two(6)};
        }
        gstore((uint4*)(out + i), w);
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          if (i + j >= 0 && i + j < a.vocab) Store<T>::store(out + i + j, v[j]);
      }
    }
  }
}

template <bool SAMPLE> static void launch(int dtype, const TruncateArgs& a, hipStream_t s) {
  auto go = [&](auto type) {
    using T = decltype(type);
    if (a.vocab <= 4096) k_truncate<T, 256, SAMPLE><<<a.rows, 256, 0, s>>>(a);
    else k_truncate<T, 1024, SAMPLE><<<a.rows, 1024, 0, s>>>(a);
  };
  if (dtype == AD_BF16) go(bf16_t{});
  else go(float{});
}
void launch_sample(int dtype, const TruncateArgs& a, hipStream_t s) { launch<true>(dtype, a, s); }
void launch_truncate(int dtype, const TruncateArgs& a, hipStream_t s) { launch<false>(dtype, a, s); }

}  // namespace ad
