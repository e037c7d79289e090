// Acceptance of drafted tokens under sampled decoding, from given random numbers.
//
// Row i of a sequence has scores x over the vocabulary, p = softmax(x / T), a drafted token d and the drafter's probabilities q (none: all on d).
// d stands where u_i q(d) < p(d).  The first row i whose token does not stand takes another: r = max(p - q, 0) (a drafter without
// probabilities: p without d; no token drafted: p), and the token is the least t with r(0) + .. + r(t) > v (r(0) + .. + r(V - 1)).
// Tokens so accepted are distributed as p.
//
// A drawn number may lie next to the border between two tokens, so sums over the vocabulary and what goes into them have 64 bits, and the tokens of a row are the same
// to the bit in every call that it may be part of (where a call is large a row's test is tried in 32 bits first: kNear):
//   k_accept_stats   a workgroup per 8 KB of scores of a row: their maximum, and sum of exp2((x - max) log2(e) / T) (without d where q is none).  It reads everything
//                    once and is bound by that; 64-bit exponentials cost 20 instructions a score.
//   k_accept_rows    (q given, or many or large rows) a wave per row: its test.  A row whose number is too close for sums in 32 bits, of random ones p in 16,000, is summed
//                    again by its wave: 46 us more for a call over 32,000 fp32 scores, 121 over 100,003 in bf16 (all of 304 and 90 rows: 59 and 147).
//   k_accept_rest    (then) a workgroup per 8 KB of scores of each sequence's deciding row: sum of r
//   k_accept_pick    a workgroup per sequence: the rows' tests if they have not been made, the piece of the deciding row that holds the wanted sum, the token in it
// One sentence of 8 rows over 32,000 scores: 3.9 and 4.8 us, launches and chains of waits.  32 blocks of up to 25 rows over 32,000 with probabilities (57 MB): 19.5,
// 4.5, 6.2 and 7.2 us; 64 blocks of 3 to 8 rows over 100,003 bf16 scores (70 MB): 18.2, 4.7, 9.0 and 7.8.  The first of them reads at 3 to 3.8 TB/s with its
// exponentials; the three behind it wait for each other more than for memory.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "ad_accept.h"
#include "ad_device.h"

namespace ad {

constexpr int kAcceptThreads = 256;
constexpr int kRowsY = 32768;                                       // rows along y of a launch, the others along z
constexpr int kDecideThreads = 1024;                                // where a sequence's rows are tested, a wave a row
// scores of a workgroup (8 KB: 32 blocks with the drafter's probabilities 39 us with 16 KB, 35 with 8; 64 of bf16 41 with 4 KB, 39 with 8) and of a thread
template <typename T> constexpr int kPiece = 8192 / (int)sizeof(T);
template <typename T> constexpr int kEach = kPiece<T> / kAcceptThreads;

// What weighs less than this beside the row's most likely token weighs nothing: a piece counts only if one of its tokens will (exp2_down ends at 2^-1000).
constexpr double kNothing = 0x1p-900;

// 2^t for t <= 0 (NaN stays): nearest whole number and the Taylor series of 2^f, |f| <= 1/2, to f^11: 7e-15 relative
__device__ __forceinline__ double exp2_down(double t) {
  if (t < -1000.0) return 0.0;
  const double n = rint(t), f = (t - n) * 0.69314718055994530942;
  double p = 2.50521083854417187751e-8;   // 1 / 11!
  p = fma(p, f, 2.75573192239858906526e-7);
  p = fma(p, f, 2.75573192239858906526e-6);
  p = fma(p, f, 2.48015873015873015873e-5);
  p = fma(p, f, 1.98412698412698412698e-4);
  p = fma(p, f, 1.38888888888888888889e-3);
  p = fma(p, f, 8.33333333333333333333e-3);
  p = fma(p, f, 4.16666666666666666667e-2);
  p = fma(p, f, 1.66666666666666666667e-1);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.0);
  p = fma(p, f, 1.0);
  return ldexp(p, (int)n);
}
// The same for the bulk of the scores, 17 instructions: t = (x - m) rate (the difference first, which is exact: at temperatures near 0 a rounded product of the maximum
// would be no small part of what is left of it) held to [-1020, ..] (what is smaller weighs nothing beside the 1 of the maximum; a NaN is
// the caller's to see), the whole part through the low word of t + 1.5 * 2^52 straight into the exponent, and 2^f to f^9 (7e-12 relative: a drawn number falls
// between this and the exact border once in 10^11 / vocab draws).
__device__ __forceinline__ double exp2_bulk(float x, double rate, double m) {
  const double t = fmax(((double)x - m) * rate, -1020.0);
  const double big = t + 6755399441055744.0, f = t - (big - 6755399441055744.0);
  double p = 1.01780860092396997275e-7;    // ln(2)^k / k!, k = 9 .. 0
  p = fma(p, f, 1.32154867901443094884e-6);
  p = fma(p, f, 1.52527338040598402800e-5);
  p = fma(p, f, 1.54035303933816099544e-4);
  p = fma(p, f, 1.33335581464284434234e-3);
  p = fma(p, f, 9.61812910762847716197e-3);
  p = fma(p, f, 5.55041086648215799532e-2);
  p = fma(p, f, 2.40226506959100712334e-1);
  p = fma(p, f, 6.93147180559945309417e-1);
  p = fma(p, f, 1.0);
  const long long bits = __builtin_bit_cast(long long, p);
  const unsigned hi = (unsigned)(bits >> 32) + ((unsigned)__builtin_bit_cast(long long, big) << 20);
  return __builtin_bit_cast(double, (long long)((unsigned long long)hi << 32 | (unsigned)bits));
}
// and to f^11, nothing below 2^-1000, for the rows that are drawn from
__device__ __forceinline__ double exp2_weight(float x, double rate, double m) {
  const double u = ((double)x - m) * rate, t = fmax(u, -1020.0);
  const double big = t + 6755399441055744.0, f = t - (big - 6755399441055744.0);
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
  const long long bits = __builtin_bit_cast(long long, p);
  const unsigned hi = (unsigned)(bits >> 32) + ((unsigned)__builtin_bit_cast(long long, big) << 20);
  return u < -1000.0 ? 0.0 : __builtin_bit_cast(double, (long long)((unsigned long long)hi << 32 | (unsigned)bits));
}
// Sums in 32 bits, what a row's test may be tried with: z off by less than 2^-15.9 of itself.  A weight 2^t, |t| <= 126, has three roundings in t (difference, rate,
// product), 3 * 2^-24 |t|, that is ln(2) * 378 * 2^-24 = 262 * 2^-24 of the weight, the exponential's own 2 * 2^-24, and at most 7 * 2^-24 by additions; what is smaller
// is 2^-125 at most, of which 2^24 are nothing beside z >= 1.  Within this part of u z, u < p is looked at again with the sums in 64 bits.
constexpr double kNear = 0x1p-15;
// sum over the wave, the same in every lane: lane moves as wave_sum's
template <int CTRL> __device__ __forceinline__ double dpp_move_f64(double v) {
  const long long b = __builtin_bit_cast(long long, v);
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, true), hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (long long)((unsigned long long)hi << 32 | lo));
}
__device__ __forceinline__ double lane_f64(double v, int lane) {
  const long long b = __builtin_bit_cast(long long, v);
  const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)b, lane), hi = (unsigned)__builtin_amdgcn_readlane((int)(b >> 32), lane);
  return __builtin_bit_cast(double, (long long)((unsigned long long)hi << 32 | lo));
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  v += dpp_move_f64<0xB1>(v);
  v += dpp_move_f64<0x4E>(v);
  v += dpp_move_f64<0x141>(v);
  v += dpp_move_f64<0x140>(v);
  return (lane_f64(v, 0) + lane_f64(v, 16)) + (lane_f64(v, 32) + lane_f64(v, 48));
}

template <typename T> struct AcceptRow {
  const T* x;
  int vocab, skew;   // skew: scores before the first 16-byte boundary
  static constexpr int kVec = 16 / (int)sizeof(T);
  __device__ __forceinline__ AcceptRow(const AcceptArgs& a, int row) {
    x = (const T*)a.logits + (size_t)row * a.stride;
    vocab = a.vocab;
    skew = (int)((16 - ((uintptr_t)x & 15)) & 15) / (int)sizeof(T);
  }
  __device__ __forceinline__ float at(int i) const { return Store<T>::load(x + i); }
  // Piece c holds the scores from skew + kPiece c on (and, the first one, the skew's): thread t's element j.
  __device__ __forceinline__ int index(int c, int t, int j) const { return skew + c * kPiece<T> + ((j / kVec) * kAcceptThreads + t) * kVec + j % kVec; }
  __device__ __forceinline__ int heads(int c) const { return c == 0 ? min(skew, vocab) : 0; }
  // (-inf past the end)
  __device__ __forceinline__ void load(int c, int t, float (&v)[kEach<T>]) const {
#pragma unroll
    for (int j = 0; j < kEach<T>; j += kVec) {
      const int i = index(c, t, j);
      if (i + kVec <= vocab) {
        const uint4 w = ldg16(x + i);
        if constexpr (sizeof(T) == 4) {
          v[j] = __uint_as_float(w.x); v[j + 1] = __uint_as_float(w.y); v[j + 2] = __uint_as_float(w.z); v[j + 3] = __uint_as_float(w.w);
        } else {
          v[j] = __uint_as_float(w.x << 16); v[j + 1] = __uint_as_float(w.x & 0xffff0000u);
          v[j + 2] = __uint_as_float(w.y << 16); v[j + 3] = __uint_as_float(w.y & 0xffff0000u);
          v[j + 4] = __uint_as_float(w.z << 16); v[j + 5] = __uint_as_float(w.z & 0xffff0000u);
          v[j + 6] = __uint_as_float(w.w << 16); v[j + 7] = __uint_as_float(w.w & 0xffff0000u);
        }
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[j + e] = i + e < vocab ? at(i + e) : -INFINITY;
      }
    }
  }
};

// Takes score `skip` (-1: none) out of what thread t holds of piece c: it is one thread's, there, and only there, it is looked for.  Whether it was a NaN.
template <typename T> __device__ __forceinline__ bool accept_drop(const AcceptRow<T>& x, int c, int t, int skip, float (&v)[kEach<T>]) {
  constexpr int kVec = AcceptRow<T>::kVec;
  const int in = skip - x.index(c, t, 0);
  bool nan = false;
  if (skip >= 0 && in >= 0 && in % (kAcceptThreads * kVec) < kVec && in / (kAcceptThreads * kVec) < kEach<T> / kVec) {
#pragma unroll
    for (int j = 0; j < kEach<T>; ++j)
      if (x.index(c, t, j) == skip) { nan = v[j] != v[j]; v[j] = -INFINITY; }
  }
  return nan;
}

// Weights of what thread t holds of piece c, whose largest score is m, in 64 bits and without score `skip`; NaN where one of the scores is
template <typename T> __device__ __forceinline__ double accept_wide(const AcceptRow<T>& x, int c, int t, int skip, float (&v)[kEach<T>], float head, double rate, float m) {
  bool nan = accept_drop(x, c, t, skip, v) || head != head;
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < kEach<T>; ++j) {
    nan = nan || v[j] != v[j];
    s += exp2_bulk(v[j], rate, (double)m);
  }
  if (t < x.heads(c) && t != skip) s += exp2_bulk(head, rate, (double)m);
  return nan ? (double)NAN : s;
}
// A piece's sum as it is kept, of its four waves'
__device__ __forceinline__ double accept_piece(double s0, double s1, double s2, double s3) {
  const double sum = (s0 + s1) + (s2 + s3);
  return sum < kNothing ? 0.0 : sum;
}
// What a piece of largest score mc and sum s weighs beside a row's maximum m (s is 0 where mc is -inf, or NaN).  (No product is fused into a sum, here or where it is added up:
// the same roundings in every kernel.)
__device__ __forceinline__ double accept_share(float mc, double s, float m, double rate) {
#pragma clang fp contract(off)
  return mc > -INFINITY ? s * exp2_down(((double)mc - (double)m) * rate) : s;
}

struct AcceptSeq { int row0, n; };
__device__ __forceinline__ AcceptSeq accept_seq(const AcceptArgs& a, int b) {
  AcceptSeq s;
  s.row0 = a.row_start[b];
  s.n = min(min(a.row_start[b + 1] - s.row0, a.max_rows), a.rows - s.row0);
  if (s.row0 < 0 || s.row0 > a.rows) s.n = 0;
  return s;
}
// The sequence of packed row `row` (-1: none, or the row is one too many of it): the last one that starts there or before (of several, those before it are empty), found by
// each wave for itself: every 64th start at once, then those between two of them.
__device__ __forceinline__ int accept_owner(const AcceptArgs& a, int row) {
  const int lane = threadIdx.x & 63, apart = (a.n_seq + 63) / 64;
  int q = __popcll(__ballot(lane * apart < a.n_seq && a.row_start[min(lane * apart, a.n_seq - 1)] <= row)) - 1;
  if (q < 0 || row >= a.rows) return -1;
  q *= apart;
  if (apart > 1) q += __popcll(__ballot(lane < apart && q + lane < a.n_seq && a.row_start[min(q + lane, a.n_seq - 1)] <= row)) - 1;
  if (q < 0) return -1;   // (starts that do not ascend)
  const AcceptSeq sq = accept_seq(a, q);
  return row >= sq.row0 && row - sq.row0 < sq.n ? q : -1;
}
// Row i of sequence b, or (PACKED) packed row b kRowsY + i and its sequence, to `b` and `row`; whether there is such a row.
template <bool PACKED> __device__ __forceinline__ bool accept_find(const AcceptArgs& a, int i, int& b, int& row) {
  if constexpr (PACKED) {
    row = b * kRowsY + i;
    b = accept_owner(a, row);
    return b >= 0;
  } else {
    const AcceptSeq sq = accept_seq(a, b);
    row = sq.row0 + i;
    return i < sq.n;
  }
}
// log2(e) / T; NaN where T is no positive number
__device__ __forceinline__ double accept_rate(const AcceptArgs& a, int b) {
  const float t = a.temperature ? a.temperature[b] : 1.f;
  return t > 0.f && t < INFINITY ? 1.44269504088896340736 / (double)t : (double)NAN;
}
__device__ __forceinline__ bool accept_drafted(const AcceptArgs& a, int d) { return d >= 0 && d < a.vocab; }

template <typename T, bool WIDE, bool PACKED>
__global__ __launch_bounds__(kAcceptThreads) void k_accept_stats(AcceptArgs a) {
  __shared__ float ms[kAcceptThreads / 64];
  __shared__ double ss[kAcceptThreads / 64];
  const int c = blockIdx.x, t = threadIdx.x;
  int b = blockIdx.z, row;
  if (!accept_find<PACKED>(a, blockIdx.y, b, row)) return;
  const AcceptRow<T> x(a, row);
  float v[kEach<T>];
  x.load(c, t, v);
  const float head = t < x.heads(c) ? x.at(t) : -INFINITY;
  const int skip = a.probs ? -1 : a.draft[row];   // (point mass: summed apart, so that what is left beside it is not a difference)
  const double rate = accept_rate(a, b);
  float m = head;
#pragma unroll
  for (int j = 0; j < kEach<T>; ++j) m = __builtin_amdgcn_fmed3f(m, v[j], INFINITY);   // (the larger; fmaxf would quiet NaN first)
  m = wave_max(m);
  if ((t & 63) == 0) ms[t >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
  double s = 0.0;
  bool nan = head != head || !(m < INFINITY) || rate != rate;   // (no distribution)
  if (m > -INFINITY) {
    if constexpr (WIDE) {
      s = accept_wide(x, c, t, skip, v, head, rate, m);
    } else {
      // (a row's first test alone rests on these sums)
      const bool here = t < x.heads(c) && t != skip;
      nan = accept_drop(x, c, t, skip, v) || nan;
      const float r = fminf((float)rate, 0x1.fffffep127f);   // (of a temperature below 2^-127 no infinity, which times a difference of 0 would be NaN)
      float e[4] = {here ? __builtin_amdgcn_exp2f((head - m) * r) : 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kEach<T>; ++j) e[j % 4] += __builtin_amdgcn_exp2f((v[j] - m) * r);
      s = (double)((e[0] + e[1]) + (e[2] + e[3]));
    }
  } else {
#pragma unroll
    for (int j = 0; j < kEach<T>; ++j) nan = nan || v[j] != v[j];
  }
  if (nan) s = (double)NAN;
  s = wave_sum_f64(s);
  if ((t & 63) == 0) ss[t >> 6] = s;
  __syncthreads();
  if (t == 0) {
    a.piece_sum[(size_t)row * a.pieces + c] = accept_piece(ss[0], ss[1], ss[2], ss[3]);
    a.piece_max[(size_t)row * a.pieces + c] = m;
  }
}

// A row's maximum and the sum over its vocabulary relative to it (without the drafted token: wd), by one wave
struct AcceptSums { float m; double z, wd; };
template <typename T> __device__ __forceinline__ AcceptSums accept_sums(const AcceptArgs& a, int row, double rate) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63;
  const float* pm = a.piece_max + (size_t)row * a.pieces;
  const double* ps = a.piece_sum + (size_t)row * a.pieces;
  // (what the row needs is requested at once: the drafted token's score behind its id, the first 64 pieces beside them)
  const int d = a.draft[row];
  const float m0 = lane < a.pieces ? pm[lane] : -INFINITY;
  const double s0 = lane < a.pieces ? ps[lane] : 0.0;
  const float xd = accept_drafted(a, d) ? AcceptRow<T>(a, row).at(d) : -INFINITY;
  AcceptSums r;
  r.m = m0;
  for (int c = lane + 64; c < a.pieces; c += 64) r.m = fmaxf(r.m, pm[c]);
  r.m = wave_max(r.m);
  double z = accept_share(m0, s0, r.m, rate);
  for (int c = lane + 64; c < a.pieces; c += 64) z += accept_share(pm[c], ps[c], r.m, rate);
  r.z = wave_sum_f64(z);
  r.wd = accept_drafted(a, d) ? exp2_down(((double)xd - (double)r.m) * rate) : 0.0;
  if (!a.probs) r.z += r.wd;
  return r;
}
__device__ __forceinline__ bool accept_broken(double z) { return !(z > 0.0 && z < (double)INFINITY); }

// A row's sums over its pieces in 64 bits in place of those in 32, by one wave: the same sums in the same order as four waves', left where this lane will look for them
template <typename T> __device__ __forceinline__ void accept_widen(const AcceptArgs& a, int row, double rate) {
  const int lane = threadIdx.x & 63, skip = a.draft[row];
  const AcceptRow<T> x(a, row);
  for (int c = 0; c < a.pieces; ++c) {
    const float m = a.piece_max[(size_t)row * a.pieces + c];
    if (!(m > -INFINITY)) continue;
    double s[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int t = 64 * w + lane;
      float v[kEach<T>];
      x.load(c, t, v);
      s[w] = wave_sum_f64(accept_wide(x, c, t, skip, v, t < x.heads(c) ? x.at(t) : -INFINITY, rate, m));
    }
    if (lane == c % 64) a.piece_sum[(size_t)row * a.pieces + c] = accept_piece(s[0], s[1], s[2], s[3]);
  }
}
// A row's test, by one wave.  NARROW: its sums have 32 bits.  Their error is bounded (kNear) while scores and 1 / T are far from the ends of fp32.
template <typename T, bool NARROW> __device__ __forceinline__ AcceptRowInfo accept_decide(const AcceptArgs& a, int row, double rate) {
  const int d = a.draft[row];
  const float u = a.accept_u[row], q = !a.probs ? 1.f : accept_drafted(a, d) ? a.probs[(size_t)row * a.probs_stride + d] : 0.f;
  AcceptSums r = accept_sums<T>(a, row, rate);
  if constexpr (NARROW) {
    const double uz = (double)u * r.z;
    const bool bounded = rate >= 0x1p-100 && rate <= 0x1p100 && r.m <= 0x1p100f;
    if (accept_drafted(a, d) && rate == rate && (!bounded || (uz > 0.0 && fabs(uz - r.wd) <= kNear * uz))) {
      accept_widen<T>(a, row, rate);
      r = accept_sums<T>(a, row, rate);
    }
  }
  return AcceptRowInfo{r.z, r.m, accept_drafted(a, d) && !accept_broken(r.z) && (double)u * (double)q < r.wd / r.z};
}
// The first row whose drafted token does not stand (n: all do), by the whole workgroup
template <typename T> __device__ __forceinline__ int accept_first(const AcceptArgs& a, const AcceptSeq& sq, double rate, int* first) {
  const int wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) *first = sq.n;
  __syncthreads();
  for (int i0 = 0; i0 < sq.n; i0 += kDecideThreads / 64) {
    const int i = i0 + wave;
    if (i < sq.n) {
      const bool stands = accept_decide<T, false>(a, sq.row0 + i, rate).stands;
      if (!stands && (threadIdx.x & 63) == 0) atomicMin(first, i);
    }
    __syncthreads();
    const int f = *first;
    __syncthreads();
    if (f < sq.n) break;
  }
  return *first;
}

// The test of all rows at once, a wave a row
template <typename T, bool PACKED, bool NARROW>
__global__ __launch_bounds__(kAcceptThreads) void k_accept_rows(AcceptArgs a) {
  int b = blockIdx.y, row;
  if (!accept_find<PACKED>(a, blockIdx.x * (kAcceptThreads / 64) + (threadIdx.x >> 6), b, row)) return;
  const AcceptRowInfo r = accept_decide<T, NARROW>(a, row, accept_rate(a, b));
  if ((threadIdx.x & 63) == 0) a.row_info[row] = r;
}
// The first row whose token does not stand, with its maximum and sum, from there, by each wave for itself
struct AcceptFirst { int i; float m; double z; };
__device__ __forceinline__ AcceptFirst accept_first_of(const AcceptArgs& a, const AcceptSeq& sq) {
  const int lane = threadIdx.x & 63;
  for (int i0 = 0; i0 < sq.n; i0 += 64) {
    const AcceptRowInfo r = gload(a.row_info + sq.row0 + i0 + min(lane, sq.n - 1 - i0));
    const unsigned long long falls = __ballot(i0 + lane < sq.n && !r.stands);
    if (falls) {
      const int l = __ffsll(falls) - 1;
      return AcceptFirst{i0 + l, __int_as_float(__builtin_amdgcn_readlane(__float_as_int(r.m), l)), lane_f64(r.z, l)};
    }
  }
  return AcceptFirst{sq.n, 0.f, 0.0};
}

// What a token of the deciding row weighs in the draw, relative to the row's maximum, or (PROBS) as a probability.  Without the drafter's probabilities the
// drafted token weighs nothing: its score is made -inf (accept_drop).
template <bool PROBS> struct AcceptWeight {
  const float* q;
  float drafted;   // 0: nothing was drafted, q does not count
  int skip;
  double rate, m, inv_z;
  __device__ __forceinline__ AcceptWeight(const AcceptArgs& a, int row, float m_, double z, double rate_) {
    const int d = a.draft[row];
    const bool is = accept_drafted(a, d);
    q = PROBS ? a.probs + (size_t)row * a.probs_stride : nullptr;
    drafted = is ? 1.f : 0.f;
    skip = !PROBS && is ? d : -1;
    rate = rate_; m = m_; inv_z = 1.0 / z;
  }
  __device__ __forceinline__ double operator()(int i, float x) const {
    const double e = exp2_weight(x, rate, m);
    if constexpr (PROBS) return fmax(fma(e, inv_z, -(double)(drafted != 0.f ? q[i] : 0.f)), 0.0);
    return e;
  }
  __device__ __forceinline__ double head(int i, float x) const { return i == skip ? 0.0 : (*this)(i, x); }
};

template <typename T, bool PROBS>
__global__ __launch_bounds__(kAcceptThreads) void k_accept_rest(AcceptArgs a) {
  __shared__ double ss[kAcceptThreads / 64];
  const int c = blockIdx.x, b = blockIdx.y, t = threadIdx.x;
  const AcceptSeq sq = accept_seq(a, b);
  if (sq.n <= 0) return;
  const double rate = accept_rate(a, b);
  const AcceptFirst f = accept_first_of(a, sq);
  if (f.i >= sq.n) return;
  const int row = sq.row0 + f.i;
  const AcceptRow<T> x(a, row);
  float v[kEach<T>];
  x.load(c, t, v);
  double s = 0.0;
  float mc = -INFINITY;
  if constexpr (PROBS) {
    const AcceptWeight<PROBS> w(a, row, f.m, f.z, rate);
#pragma unroll
    for (int j = 0; j < kEach<T>; ++j) {
      const int at = x.index(c, t, j);
      if (at < a.vocab) s += w(at, v[j]);
    }
    if (t < x.heads(c)) s += w.head(t, x.at(t));
  } else {   // (the sums that a small call has of every row)
    mc = a.piece_max[(size_t)row * a.pieces + c];
    if (mc > -INFINITY) s = accept_wide(x, c, t, a.draft[row], v, t < x.heads(c) ? x.at(t) : -INFINITY, rate, mc);
  }
  s = wave_sum_f64(s);
  if ((t & 63) == 0) ss[t >> 6] = s;
  __syncthreads();
  if (t == 0) {
    double sum = (ss[0] + ss[1]) + (ss[2] + ss[3]);
    if constexpr (!PROBS) {
      sum = accept_share(mc, accept_piece(ss[0], ss[1], ss[2], ss[3]), f.m, rate);
      if (sum < kNothing) sum = 0.0;
    }
    a.rest_sum[(size_t)b * a.pieces + c] = sum;
  }
}

// DECIDED: k_accept_rows has been over the rows
template <typename T, bool DECIDED, bool PROBS>
__global__ __launch_bounds__(DECIDED ? kAcceptThreads : kDecideThreads) void k_accept_pick(AcceptArgs a) {
  constexpr int kThreads = DECIDED ? kAcceptThreads : kDecideThreads;
  constexpr int kVec = AcceptRow<T>::kVec, kGroups = kEach<T> / kVec;
  __shared__ int first, token;
  __shared__ double round[kGroups * 4];
  const int b = blockIdx.x, t = threadIdx.x, lane = t & 63;
  const AcceptSeq sq = accept_seq(a, b);
  const double rate = accept_rate(a, b);
  // (requested at once with what decides the row)
  const double rest0 = DECIDED && lane < a.pieces ? a.rest_sum[(size_t)b * a.pieces + lane] : 0.0, pick_u = a.pick_u[b];
  AcceptFirst f{0, 0.f, 0.0};
  int i = 0;
  if (sq.n > 0) {
    if constexpr (DECIDED) { f = accept_first_of(a, sq); i = f.i; }
    else i = accept_first<T>(a, sq, rate, &first);
    if (t == 0) token = AD_NEVER;
    __syncthreads();
  }
  if (i < sq.n) {
    const int row = sq.row0 + i;
    float m;
    double z;
    if constexpr (DECIDED) {
      m = f.m; z = f.z;
    } else {
      const AcceptSums sums = accept_sums<T>(a, row, rate);
      m = sums.m; z = sums.z;
    }
    if (!accept_broken(z)) {
      const AcceptRow<T> x(a, row);
      const AcceptWeight<PROBS> w(a, row, m, z, rate);
      // (the drafted token is left out of the pieces' sums where the drafter gave no probabilities)
      auto piece = [&](int c) -> double {
        if constexpr (DECIDED) return c == lane ? rest0 : a.rest_sum[(size_t)b * a.pieces + c];
        const double s = accept_share(a.piece_max[(size_t)row * a.pieces + c], a.piece_sum[(size_t)row * a.pieces + c], m, rate);
        return s < kNothing ? 0.0 : s;
      };
      // the piece in which the sum passes the wanted part of the whole: every wave finds it by itself, 64 pieces at a time
      double total = 0.0;
      for (int c = lane; c < a.pieces; c += 64) total += piece(c);
      total = wave_sum_f64(total);
      if (total > 0.0) {
        const double want = pick_u * total;
        double before = 0.0, base = 0.0;
        int at = -1, last = 0;
        double last_base = 0.0;
        for (int c0 = 0; c0 < a.pieces && at < 0; c0 += 64) {
          const double own = c0 + lane < a.pieces ? piece(c0 + lane) : 0.0;
          double upto = own;
#pragma unroll
          for (int s = 1; s < 64; s *= 2) {
            const double o = __shfl_up(upto, s);
            if (lane >= s) upto += o;
          }
          const unsigned long long some = __ballot(own > 0.0), over = __ballot(before + upto > want) & some;
          if (over) {
            const int l = __ffsll(over) - 1;
            at = c0 + l;
            base = before + __shfl(upto - own, l);
          }
          if (some) {
            const int l = 63 - __clzll(some);
            last = c0 + l;
            last_base = before + __shfl(upto - own, l);
          }
          before += __shfl(upto, 63);
        }
        if (at < 0) { at = last; base = last_base; }   // (rounding: the last piece that holds anything)
        // Its weights: sums of kVec scores side by side by thread, in kGroups rounds of the workgroup's four waves, which is the order of their indices; the round and
        // wave, the thread, the score in which the running sum passes `want` (else the last that weighs anything).
        double each[kEach<T>], own[kGroups];
        if (t < kAcceptThreads) {
          float v[kEach<T>];
          x.load(at, t, v);
          accept_drop(x, at, t, w.skip, v);
#pragma unroll
          for (int j = 0; j < kEach<T>; j += kVec) {
            double s = 0.0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
              const int n = x.index(at, t, j + e);
              each[j + e] = n < a.vocab ? w(n, v[j + e]) : 0.0;
              s += each[j + e];
            }
            own[j / kVec] = s;
            const double all = wave_sum_f64(s);
            if (lane == 0) round[(j / kVec) * 4 + (t >> 6)] = all;
          }
        }
        __syncthreads();
        int hit = -1, heavy = -1;
        double run = base;
        {
          const int n = x.heads(at);
          const double e = lane < n ? w.head(lane, x.at(lane)) : 0.0;
          for (int i = 0; i < n && hit < 0; ++i) {
            const double g = lane_f64(e, i);
            run += g;
            if (g > 0.0) {
              heavy = i;
              if (run > want) hit = i;
            }
          }
        }
        if (hit < 0) {
          int in = -1;
          double in_run = run;
          for (int n = 0; n < kGroups * 4; ++n) {
            const double s = round[n];
            if (s > 0.0) { in = n; in_run = run; }
            run += s;
            if (run > want && s > 0.0) break;
          }
          if (in >= 0) {
            if (t >> 6 == in % 4) {   // (one wave; it has the round's sums)
              run = in_run;
              double mine = own[0];
#pragma unroll
              for (int j = 1; j < kGroups; ++j) mine = in / 4 == j ? own[j] : mine;
              double upto = mine;
#pragma unroll
              for (int s = 1; s < 64; s *= 2) {
                const double o = __shfl_up(upto, s);
                if (lane >= s) upto += o;
              }
              const unsigned long long some = __ballot(mine > 0.0), over = __ballot(run + upto > want) & some;
              const int l = over ? __ffsll(over) - 1 : 63 - __clzll(some);
              run += upto - mine;
#pragma unroll
              for (int j = 0; j < kEach<T>; ++j)
                if (j / kVec == in / 4) {   // (every thread its own scores: the thread's that was found counts)
                  run += each[j];
                  if (each[j] > 0.0 && hit < 0) {
                    heavy = x.index(at, t, j);
                    if (run > want) hit = heavy;
                  }
                }
              if (lane == l) token = hit >= 0 ? hit : heavy;
            }
          } else if (t == 0) {
            token = heavy;
          }
        } else if (t == 0) {
          token = hit;
        }
      } else {
        if (t == 0) token = a.draft[row];   // p and q alike: nothing is left over, the drafted token stands
      }
    }
    __syncthreads();
  }
  const int tok = sq.n > 0 && i < sq.n ? token : AD_NEVER;
  for (int n = t; n < sq.n; n += kThreads) {
    const int to = n < i ? a.draft[sq.row0 + n] : n == i ? tok : AD_NEVER;
    if (!a.keep || (n <= i && to >= 0)) a.tokens[sq.row0 + n] = to;
  }
  if (t == 0 && a.n_accept) a.n_accept[b] = max(sq.n, 0) == 0 ? 0 : i >= sq.n ? sq.n : tok >= 0 ? i + 1 : i;
}

__global__ __launch_bounds__(64) void k_accept_inputs(const int* __restrict__ draft, const float* __restrict__ u, const float* __restrict__ v,
                                                      const float* __restrict__ t, int k_max, const int* __restrict__ row_start, int* __restrict__ draft_out,
                                                      float* __restrict__ u_out, float* __restrict__ v_out, float* __restrict__ t_out) {
  const int b = blockIdx.x, r0 = row_start[b], n = min(row_start[b + 1] - r0, k_max);
  for (int i = threadIdx.x; i < n; i += 64) {
    draft_out[r0 + i] = draft[(size_t)b * k_max + i];
    u_out[r0 + i] = u[(size_t)b * k_max + i];
  }
  if (threadIdx.x == 0) { v_out[b] = v[b]; t_out[b] = t[b]; }
}
void launch_accept_inputs(const int* draft, const float* u, const float* v, const float* t, int k_max, const int* row_start, int n_seq, int* draft_out,
                          float* u_out, float* v_out, float* t_out, hipStream_t s) {
  k_accept_inputs<<<n_seq, 64, 0, s>>>(draft, u, v, t, k_max, row_start, draft_out, u_out, v_out, t_out);
}

static int pieces_of(int vocab, int piece) { return (vocab + piece - 1) / piece; }
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }
size_t accept_bytes(int n_seq, int rows, int vocab) {
  const size_t p = pieces_of(vocab, kPiece<float>);   // (bf16 has half as many)
  return up256(rows * p * 8) + up256(rows * p * 4) + up256((size_t)n_seq * p * 8) + up256(rows * sizeof(AcceptRowInfo));
}
void launch_accept_nothing(const AcceptArgs& a, hipStream_t s) { k_accept_pick<float, false, false><<<a.n_seq, kDecideThreads, 0, s>>>(a); }
void launch_accept_sampled(int dtype, AcceptArgs a, void* ws, hipStream_t s) {
  a.pieces = pieces_of(a.vocab, dtype == AD_BF16 ? kPiece<bf16_t> : kPiece<float>);
  // Sums in 64 bits of every row serve the draw as well as the test, and the draw is the second and last launch.  Where all rows together are large, only the deciding
  // ones and those whose test is close (accept_decide) get them, in launches of their own (us, all rows / the deciding ones: 8 rows of 32,000 6.8 / 9.5, 128 rows 15.0 / 16.5, 263 rows 19.6 / 22.1,
  // 800 rows 38.4 / 30.5, 352 rows of 100,003 in bf16 43.0 / 34.8).
  const bool wide = a.probs || (size_t)a.rows * a.vocab < ((size_t)1 << 23);
  a.rest = a.probs || !wide;
  // Rows by sequence (max_rows of every one), or packed, which costs each workgroup the search for its sequence, where that would be mostly rows that are not there (us, by
  // sequence / packed: 32 blocks of up to 25 rows 35.2 / 36.1, 64 of 8 rows of 100,003 45.8 / 47; 256 of 8 rows of 32,000 and max_rows = 8 62 / 69, without a bound 2041 / 69).
  const bool packed = accept_packed(a.n_seq, a.rows, a.max_rows);
  const dim3 by = packed ? dim3(1, std::min(a.rows, kRowsY), (a.rows + kRowsY - 1) / kRowsY) : dim3(1, a.max_rows, a.n_seq);
  char* w = (char*)ws;
  a.piece_sum = (double*)w;
  a.piece_max = (float*)(w + up256((size_t)a.rows * a.pieces * 8));
  a.rest_sum = (double*)((char*)a.piece_max + up256((size_t)a.rows * a.pieces * 4));
  a.row_info = (AcceptRowInfo*)((char*)a.rest_sum + up256((size_t)a.n_seq * a.pieces * 8));
  auto go = [&](auto one, auto pk) {
    typedef decltype(one) T;
    constexpr bool PK = pk.value;
    const dim3 grid(a.pieces, by.y, by.z);
    if (wide) k_accept_stats<T, true, PK><<<grid, kAcceptThreads, 0, s>>>(a);
    else k_accept_stats<T, false, PK><<<grid, kAcceptThreads, 0, s>>>(a);
    if (a.rest) {
      const dim3 of_four((by.y + 3) / 4, by.z);
      if (wide) k_accept_rows<T, PK, false><<<of_four, kAcceptThreads, 0, s>>>(a);
      else k_accept_rows<T, PK, true><<<of_four, kAcceptThreads, 0, s>>>(a);
      auto draw = [&](auto probs) {
        k_accept_rest<T, probs.value><<<dim3(a.pieces, a.n_seq), kAcceptThreads, 0, s>>>(a);
        k_accept_pick<T, true, probs.value><<<a.n_seq, kAcceptThreads, 0, s>>>(a);
      };
      if (a.probs) draw(std::true_type{});
      else draw(std::false_type{});
    } else {
      k_accept_pick<T, false, false><<<a.n_seq, kDecideThreads, 0, s>>>(a);
    }
  };
  auto of_type = [&](auto pk) {
    if (dtype == AD_BF16) go(bf16_t{}, pk);
    else go(float{}, pk);
  };
  if (packed) of_type(std::true_type{});
  else of_type(std::false_type{});
}

}  // namespace ad
