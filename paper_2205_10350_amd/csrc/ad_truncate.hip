// Distributions cut by temperature, top-k, top-p and min-p: a token drawn from a given random number, or the scores without what is cut off.
//
// A row has scores x, m = max x, weights w = 2^((x - m) rate), rate = log2(e) / T.  In order of falling score, equal ones by rising index, the first k stay; of them the
// least number whose weights sum to p of theirs or more (one at least); of them those with w >= min_p.  So what stays is a front of that order: everything before a border
// (score, index).  The drawn token is the least index whose weights up to it, of what stays, exceed u of all of that.
//
// Weights are whole numbers of 2^-S, S = min(51, 64 - the bits of the vocabulary): w rounded to nearest, so 0 below half of that (such a token stays where no cut takes it, and is never drawn), and all of a
// row sum to less than 2^64.  Whole sums are exact, so neither atomics nor the launch's shape change a border or a token, and p Z and u Z are compared exactly.  Rounding moves a sum, and so a border, by
// V 2^-(S + 1) of the largest weight at most for V tokens (3.3e-13 of it more by the exponential): 2.8e-11 for 32,000 tokens, 3.6e-10 for 100,003,
// and for 2^20, the most that are accepted, 2^-24, half a step of the fp32 numbers p and u below 1.
//
// One workgroup a row, which it keeps in LDS as far as that goes (32,768 fp32 scores, 65,536 bf16).  With top_k the k-th largest of the largest scores of 2048 parts of the row bounds the border from below; else
// a histogram of all weights in steps of T / 28 below the maximum says which step holds it.  What lies up to there is gathered, in its order, into a list in LDS, where everything else is done: up to
// 256 scores are ranked by comparing each with each; of more the step that holds the border is cut into equal parts of the floating point numbers between its least and its largest until 256 are left, or all are
// equal and their indices decide.  Where the list has no room (2048) it takes the border's step alone, and the token is looked for over the row.
//
// What bounds it: a row of 32,000 scores with top_k 50 and top_p takes 12 us, 2 of them to read it and the rest eight steps of 0.5 to 2 us between barriers of 16 waves; with top_p alone 16.0 us, 6.0 of them the
// histogram, 28 instructions a score, 10 of them in 64 bits, on one compute unit.  32 rows 12.9 us; 416 rows of blocks truncated 47.8, where two turns of 256 rows overlap little (53 MB read and
// written, 20 us at a copy's rate); 256 rows of 100,003 scores, settings of each row's own, 98.5 us: the slowest rows', where thousands of tokens stay and weights are taken twice (the others take 25; 102 MB).
// (Steps on the way, us, 32,000 scores top_p / 256 x 100,003 / 416 rows truncated; workgroups of 512 threads, 6 vectors of a lane in LDS, 25.6 / 138 / 59; of 256 39 / 344 / 121; of 1024, as here, 21.4 / 107 / 53.  Weights of the
// histogram in 32 bits first, and in 64 where a border lies near: 19.3 / 129 / 57 where these were 19.8 / 103 / 49.)
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
// what every lane has alike, told to the compiler
__device__ __forceinline__ int alike(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float alike(float v) { return __uint_as_float((unsigned)__builtin_amdgcn_readfirstlane((int)__float_as_uint(v))); }
__device__ __forceinline__ u64 alike(u64 v) { return lane_u64(v, 0); }
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
  return (unsigned __int128)m * z;   // < 2^88
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
  __device__ __forceinline__ bool holds(float v, int at) const { return (int)(v > x) | ((int)(v == x) & (int)(at <= i)); }
};

// floats in their order as whole numbers, -0 as 0
__device__ __forceinline__ unsigned order_of(float v) {
  const unsigned b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// 2^(-j / 128)
__device__ const double kPowers[128] = {
    1.0, 0x1.fd3c22b8f71f1p-1, 0x1.fa7c1819e90d8p-1, 0x1.f7bfdad9cbe14p-1, 0x1.f50765b6e4540p-1, 0x1.f252b376bba97p-1,
    0x1.efa1bee615a27p-1, 0x1.ecf482d8e67f1p-1, 0x1.ea4afa2a490dap-1, 0x1.e7a51fbc74c83p-1, 0x1.e502ee78b3ff6p-1, 0x1.e264614f5a129p-1,
    0x1.dfc97337b9b5fp-1, 0x1.dd321f301b460p-1, 0x1.da9e603db3285p-1, 0x1.d80e316c98398p-1, 0x1.d5818dcfba487p-1, 0x1.d2f87080d89f2p-1,
    0x1.d072d4a07897cp-1, 0x1.cdf0b555dc3fap-1, 0x1.cb720dcef9069p-1, 0x1.c8f6d9406e7b5p-1, 0x1.c67f12e57d14bp-1, 0x1.c40ab5fffd07ap-1,
    0x1.c199bdd85529cp-1, 0x1.bf2c25bd71e09p-1, 0x1.bcc1e904bc1d2p-1, 0x1.ba5b030a1064ap-1, 0x1.b7f76f2fb5e47p-1, 0x1.b59728de5593ap-1,
    0x1.b33a2b84f15fbp-1, 0x1.b0e07298db666p-1, 0x1.ae89f995ad3adp-1, 0x1.ac36bbfd3f37ap-1, 0x1.a9e6b5579fdbfp-1, 0x1.a799e1330b358p-1,
    0x1.a5503b23e255dp-1, 0x1.a309bec4a2d33p-1, 0x1.a0c667b5de565p-1, 0x1.9e86319e32323p-1, 0x1.9c49182a3f090p-1, 0x1.9a0f170ca07bap-1,
    0x1.97d829fde4e50p-1, 0x1.95a44cbc8520fp-1, 0x1.93737b0cdc5e5p-1, 0x1.9145b0b91ffc6p-1, 0x1.8f1ae99157736p-1, 0x1.8cf3216b5448cp-1,
    0x1.8ace5422aa0dbp-1, 0x1.88ac7d98a6699p-1, 0x1.868d99b4492edp-1, 0x1.8471a4623c7adp-1, 0x1.82589994cce13p-1, 0x1.80427543e1a12p-1,
    0x1.7e2f336cf4e62p-1, 0x1.7c1ed0130c132p-1, 0x1.7a11473eb0187p-1, 0x1.780694fde5d3fp-1, 0x1.75feb564267c9p-1, 0x1.73f9a48a58174p-1,
    0x1.71f75e8ec5f74p-1, 0x1.6ff7df9519484p-1, 0x1.6dfb23c651a2fp-1, 0x1.6c012750bdabfp-1, 0x1.6a09e667f3bcdp-1, 0x1.68155d44ca973p-1,
    0x1.6623882552225p-1, 0x1.6434634ccc320p-1, 0x1.6247eb03a5585p-1, 0x1.605e1b976dc09p-1, 0x1.5e76f15ad2148p-1, 0x1.5c9268a5946b7p-1,
    0x1.5ab07dd485429p-1, 0x1.58d12d497c7fdp-1, 0x1.56f4736b527dap-1, 0x1.551a4ca5d920fp-1, 0x1.5342b569d4f82p-1, 0x1.516daa2cf6642p-1,
    0x1.4f9b2769d2ca7p-1, 0x1.4dcb299fddd0dp-1, 0x1.4bfdad5362a27p-1, 0x1.4a32af0d7d3dep-1, 0x1.486a2b5c13cd0p-1, 0x1.46a41ed1d0057p-1,
    0x1.44e086061892dp-1, 0x1.431f5d950a897p-1, 0x1.4160a21f72e2ap-1, 0x1.3fa4504ac801cp-1, 0x1.3dea64c123422p-1, 0x1.3c32dc313a8e5p-1,
    0x1.3a7db34e59ff7p-1, 0x1.38cae6d05d866p-1, 0x1.371a7373aa9cbp-1, 0x1.356c55f929ff1p-1, 0x1.33c08b26416ffp-1, 0x1.32170fc4cd831p-1,
    0x1.306fe0a31b715p-1, 0x1.2ecafa93e2f56p-1, 0x1.2d285a6e4030bp-1, 0x1.2b87fd0dad990p-1, 0x1.29e9df51fdee1p-1, 0x1.284dfe1f56381p-1,
    0x1.26b4565e27cddp-1, 0x1.251ce4fb2a63fp-1, 0x1.2387a6e756238p-1, 0x1.21f49917ddc96p-1, 0x1.2063b88628cd6p-1, 0x1.1ed5022fcd91dp-1,
    0x1.1d4873168b9aap-1, 0x1.1bbe084045cd4p-1, 0x1.1a35beb6fcb75p-1, 0x1.18af9388c8deap-1, 0x1.172b83c7d517bp-1, 0x1.15a98c8a58e51p-1,
    0x1.1429aaea92de0p-1, 0x1.12abdc06c31ccp-1, 0x1.11301d0125b51p-1, 0x1.0fb66affed31bp-1, 0x1.0e3ec32d3d1a2p-1, 0x1.0cc922b7247f7p-1,
    0x1.0b5586cf9890fp-1, 0x1.09e3ecac6f383p-1, 0x1.0874518759bc8p-1, 0x1.0706b29ddf6dep-1, 0x1.059b0d3158574p-1, 0x1.04315e86e7f85p-1,
    0x1.02c9a3e778061p-1, 0x1.0163da9fb3335p-1};

// A row's weights
struct Weigh {
  float m, half, step;  // half: of m; step: of the histograms, bins two units of the scores
  double rate, most;    // 128 log2(e) / T; the most that a score of min_p's weight lies below the maximum (inf: no min_p)
  int bits;             // S
  const double* table;  // kPowers
  // 128 times the power of two that a score's weight lies below the maximum's 1 (the difference is exact; at temperatures near 0 a difference of rounded products would not do)
  __device__ __forceinline__ double below(float v) const { return ((double)m - (double)v) * rate; }
  // The weight 2^(S - t / 128), 0 <= t <= 12800, in whole numbers: 2^(-f / 128), 0 <= f < 1, by a polynomial (1 at 0 and off by 3.3e-13 at most: least maximum error), the other 127 parts by
  // a table, the whole part straight into the exponent, and the product rounded to a whole number as it is added to 2^52.
  __device__ __forceinline__ u64 near(double t) const {
    const int n = (int)t;
    const double f = __builtin_amdgcn_fract(t);
    double p = -2.6397700221988634e-08;
    p = fma(p, f, 1.466222257317361e-05);
    p = fma(p, f, -0.005415212341565815);
    p = fma(p, f, 1.0);
    const long long b = __builtin_bit_cast(long long, table[n & 127]);
    const unsigned hi = (unsigned)(b >> 32) + ((unsigned)(bits - (n >> 7)) << 20);
    return __builtin_bit_cast(u64, fma(p, __builtin_bit_cast(double, (long long)((u64)hi << 32 | (unsigned)b)), 4503599627370496.0)) & 0xfffffffffffffull;   // (<= 2^51)
  }
  __device__ __forceinline__ u64 of(double t) const { return near(fmin(t, 12800.0)); }   // (2^-100 of the largest is nothing)
  // The histogram's bin: 28 to a T, so that what falls into the last one lies 36.5 T or more below the maximum and weighs nothing (half of 2^-51 is 36.04 T below it).
  // (by halves: the difference itself may be beyond fp32)
  __device__ __forceinline__ float place(float v) const { return fmaf(v, -0.5f, half) * step; }
  __device__ __forceinline__ int bin(float v) const { return (int)fminf(place(v), (float)(kBins - 1)); }
};

template <int THREADS, int EACH> struct TruncateShared {
  static constexpr int kMost = EACH * THREADS;   // scores of the list
  u64 hist[kBins];
  double table[128];
  u64 part[THREADS / 64];
  float lo[THREADS / 64], hi[THREADS / 64];
  float list_x[kMost];   // in the row's order
  int list_i[kMost];
  uint4 rank[kList];     // score, index, weight
  // of the ranked, where the histogram was: the weights up to it, how many are before it
  __device__ __forceinline__ u64& sum(int i) { return hist[i]; }
  __device__ __forceinline__ int& order(int i) { return ((int*)(hist + kList))[i]; }
  u64 above;      // before the bin that holds the border
  int bin, n;
  Border border;
  // what the waves before this one have of `part`, and all of them
  __device__ __forceinline__ u64 before(u64& all) const {
    const int lane = threadIdx.x & 63, wave = alike((int)(threadIdx.x >> 6));
    const u64 own = lane < THREADS / 64 ? part[lane] : 0, up = wave_scan_u64(own);
    all = lane_u64(up, 63);
    return lane_u64(up - own, wave);
  }
};

// A row's scores, 16 bytes at a time from the 16-byte boundary at or before the first: wave w of a workgroup has pieces (w per .. (w + 1) per - 1) of 64 vectors, a lane one of each.  The
// first KEEP of a lane stay in LDS, where each lane reads what it wrote; in find, behind barriers, all waves read what one of them wrote.
template <typename T, int THREADS, int KEEP> struct TruncateRow {
  static constexpr int kVec = 16 / (int)sizeof(T);
  const T* x;
  uint4* kept;
  int vocab, skew, per, first;   // per: vectors of a lane; first: this lane's first one
  __device__ __forceinline__ TruncateRow(const TruncateArgs& a, int row, uint4* lds) {
    x = (const T*)a.x + (size_t)row * a.stride;
    kept = lds + threadIdx.x;
    vocab = a.vocab;
    skew = (int)((uintptr_t)x & 15) / (int)sizeof(T);
    per = ((vocab + skew + kVec - 1) / kVec + THREADS - 1) / THREADS;
    first = (int)(threadIdx.x >> 6) * per * 64 + (int)(threadIdx.x & 63);
  }
  __device__ __forceinline__ int index(int c) const { return (first + 64 * c) * kVec - skew; }   // of vector c's first score
  // the same row as another wave has it
  __device__ __forceinline__ TruncateRow of_wave(int wave) const {
    TruncateRow x = *this;
    const int lane = threadIdx.x & 63;
    x.first = wave * per * 64 + lane;
    x.kept = kept - threadIdx.x + wave * 64 + lane;
    return x;
  }
  __device__ __forceinline__ bool whole(int i) const { return i >= 0 && i + kVec <= vocab; }
  __device__ __forceinline__ uint4 fetch(int c) const {   // (-inf off the row)
    const int i = index(c);
    if (whole(i)) return ldg16(x + i);
    // (an edge: score by score, each read where there is one)
    auto one = [&](int e) -> unsigned {
      const int at = min(max(i + e, 0), vocab - 1);
      if constexpr (sizeof(T) == 4) {
        const unsigned w = __float_as_uint(gload((const float*)x + at));
        return at == i + e ? w : 0xff800000u;
      } else {
        const unsigned w = gload((const bf16_t*)x + at);
        return at == i + e ? w : 0xff80u;
      }
    };
    uint4 w;
    if constexpr (sizeof(T) == 4) w = uint4{one(0), one(1), one(2), one(3)};
    else w = uint4{one(0) | one(1) << 16, one(2) | one(3) << 16, one(4) | one(5) << 16, one(6) | one(7) << 16};
    return w;
  }
  static __device__ __forceinline__ void unpack(const uint4& w, float (&v)[kVec]) {
    if constexpr (sizeof(T) == 4) {
      v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
    } else {
      v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u); v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
      v[4] = __uint_as_float(w.z << 16); v[5] = __uint_as_float(w.z & 0xffff0000u); v[6] = __uint_as_float(w.w << 16); v[7] = __uint_as_float(w.w & 0xffff0000u);
    }
  }
  __device__ __forceinline__ uint4 again(int c) const { return c < KEEP ? kept[c * THREADS] : fetch(c); }
  __device__ __forceinline__ void load(int c, float (&v)[kVec]) const { unpack(again(c), v); }
  // the first time: f(scores) of each vector, eight on their way
  template <typename F> __device__ __forceinline__ void take(const F& f) const {
#pragma clang loop unroll(disable)
    for (int c = 0; c < per; c += 8) {
      uint4 w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < per) w[j] = fetch(c + j);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (c + j >= per) break;
        if (c + j < KEEP) kept[(c + j) * THREADS] = w[j];
        float v[kVec];
        unpack(w[j], v);
        f(v, j);
      }
    }
  }
  template <typename F> __device__ __forceinline__ void vectors(const F& f) const {   // f(vector, scores), the next two on their way
    uint4 w = again(0), w1 = per > 1 ? again(1) : w;
#pragma clang loop unroll(disable)
    for (int c = 0; c < per; ++c) {
      const uint4 w2 = c + 2 < per ? again(c + 2) : w1;
      float v[kVec];
      unpack(w, v);
      f(c, v);
      w = w1; w1 = w2;
    }
  }
  template <typename F> __device__ __forceinline__ void each(const F& f) const {   // f(score, index) over this thread's
    vectors([&](int c, const float (&v)[kVec]) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) f(v[e], index(c) + e);
    });
  }
  // Weights of all, bin by bin.  What would go into the last bin weighs nothing.
  template <typename S> __device__ __forceinline__ void weigh_all(S& s, const Weigh& weigh) const {
    // (a score's weight is a chain of ten steps in 64 bits: the table's numbers of four are looked up together)
    vectors([&](int, const float (&v)[kVec]) {
#pragma unroll
      for (int h = 0; h < kVec; h += 4) {
        u64 w[4];
        float at[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = weigh.of(weigh.below(v[h + e]));   // (at temperatures below 56e-30 a bin is wider than T / 28: what lies in the first ones may weigh nothing, too)
          at[e] = weigh.place(v[h + e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at[e] < (float)(kBins - 1)) atomicAdd(&s.hist[(int)at[e]], w[e]);
      }
    });
  }
  // Those with pred(score) into the list, in their order, if they go there; how many there are.  may(score) of the largest of every eighth vector: whether one of these may have one.
  template <typename S, typename M, typename P> __device__ __forceinline__ int gather(S& s, const float (&most)[8], const M& may, const P& pred) const {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int mine = 0, groups = 0;
    u64 some = 0;   // vectors with one
#pragma unroll
    for (int j = 0; j < 8; ++j) groups |= __any(may(most[j])) ? 1 << j : 0;
#pragma clang loop unroll(disable)
    for (int c = 0; c < per; ++c) {
      if (!(groups >> (c & 7) & 1)) continue;
      float v[kVec];
      load(c, v);
      int n = 0;
#pragma unroll
      for (int e = 0; e < kVec; ++e) n += pred(v[e]);
      mine += n;
      if (__any(n)) some |= (u64)1 << min(c, 63);
    }
    const u64 count = wave_sum_u64(mine);
    __syncthreads();
    if (lane == 0) s.part[wave] = count;
    __syncthreads();
    u64 sum;
    int at = (int)s.before(sum);
    const int all = (int)sum;
    if (all <= S::kMost) {
#pragma clang loop unroll(disable)
      for (int c = 0; c < per; ++c) {
        if (!(some >> min(c, 63) & 1)) continue;
        float v[kVec];
        load(c, v);
        int n = at;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const u64 b = __ballot(pred(v[e]));
          n += __builtin_amdgcn_mbcnt_hi((unsigned)(b >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)b, 0));
          at += __popcll(b);
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (pred(v[e])) { s.list_x[n] = v[e]; s.list_i[n] = index(c) + e; ++n; }
      }
    }
    __syncthreads();
    return all;
  }
  // f(scores' weights, those that do not stay 0) of each vector that has one that stays; weight(score) of four at once, without a branch
  template <typename P, typename G> __device__ __forceinline__ bool weights(int c, const float (&v)[kVec], const P& stays, const G& weight, u64 (&e)[kVec]) const {
    bool in[kVec];
    int some = 0;
#pragma unroll
    for (int j = 0; j < kVec; ++j) { in[j] = stays(v[j], index(c) + j); some |= (int)in[j]; }
    if (!__any(some)) return false;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const u64 w = weight(v[j]);
      e[j] = in[j] ? w : 0;
    }
    return true;
  }
  // The least index up to which the weights of those that stay sum to want(sum of all) or more.  Left in s.border: its score and index.
  template <typename S, typename P, typename G, typename W> __device__ __forceinline__ u64 find(S& s, const P& stays, const G& weight, const W& want) const {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    u64 sum = 0;
    vectors([&](int c, const float (&v)[kVec]) {
      u64 e[kVec];
      if (!weights(c, v, stays, weight, e)) return;
#pragma unroll
      for (int j = 0; j < kVec; ++j) sum += e[j];
    });
    sum = wave_sum_u64(sum);
    __syncthreads();
    if (lane == 0) s.part[wave] = sum;
    __syncthreads();
    u64 all, before = s.before(all);
    const u64 target = want(all);
    if (lane == 0 && before < target && before + sum >= target) { s.bin = wave; s.above = before; }
    __syncthreads();
    const TruncateRow x = of_wave(min(max(alike(s.bin), 0), THREADS / 64 - 1));
    before = alike(s.above);
    // every wave takes some of the winner's vectors (64 at a time, whose sums lie where the histogram was), then each looks for the one that holds the target
    for (int c0 = 0;; c0 += 64) {
      const int n = min(per - c0, 64);
      for (int c = wave; c < n; c += THREADS / 64) {
        float v[kVec];
        u64 e[kVec], own = 0;
        x.load(c0 + c, v);
        if (x.weights(c0 + c, v, stays, weight, e)) {
#pragma unroll
          for (int j = 0; j < kVec; ++j) own += e[j];
        }
        own = wave_sum_u64(own);
        if (lane == 0) s.hist[c] = own;
      }
      __syncthreads();
      const u64 own = lane < n ? s.hist[lane] : 0, up = wave_scan_u64(own);
      const u64 here = __ballot(before + up >= target);
      if (here != 0) {
        const int c = __ffsll(here) - 1;
        if (c % (THREADS / 64) == wave) {
          u64 at = before + lane_u64(up, c) - lane_u64(own, c);
          float v[kVec];
          u64 e[kVec], mine = 0;
          x.load(c0 + c, v);
          if (x.weights(c0 + c, v, stays, weight, e)) {
#pragma unroll
            for (int j = 0; j < kVec; ++j) mine += e[j];
            at += wave_scan_u64(mine) - mine;
            if (at < target && at + mine >= target) {   // (one lane)
#pragma unroll
              for (int j = 0; j < kVec; ++j) {
                if (at < target && at + e[j] >= target) s.border = Border{v[j], x.index(c0 + c) + j};
                at += e[j];
              }
            }
          }
        }
        break;
      }
      before += lane_u64(up, 63);
      if (c0 + 64 >= per) break;   // (not reached: the winner has it)
      __syncthreads();
    }
    __syncthreads();
    return all;
  }
  // weight(score) of those that stay into the histogram's bin(score)
  template <typename S, typename P, typename G, typename B> __device__ __forceinline__ void into(S& s, const P& stays, const G& weight, const B& bin) const {
    vectors([&](int c, const float (&v)[kVec]) {
      u64 e[kVec];
      if (!weights(c, v, stays, weight, e)) return;
#pragma unroll
      for (int j = 0; j < kVec; ++j)
        if (e[j]) atomicAdd(&s.hist[bin(v[j])], e[j]);
    });
  }
};

// The same over the list: wave w has its scores 64 EACH w .., a lane every 64th of them
template <int THREADS, int EACH> struct TruncateList {
  const TruncateShared<THREADS, EACH>& s;
  int n, first, per;
  __device__ __forceinline__ TruncateList(const TruncateShared<THREADS, EACH>& s, int n) : s(s), n(n), first((int)(threadIdx.x >> 6) * 64 * EACH + (int)(threadIdx.x & 63)) {
    per = min(EACH, max(0, (n - alike(first) + 63) / 64));
  }
  __device__ __forceinline__ float at(int j) const { return first + 64 * j < n ? s.list_x[first + 64 * j] : -INFINITY; }
  template <typename F> __device__ __forceinline__ void each(const F& f) const {
#pragma clang loop unroll(disable)
    for (int j = 0; j < per; ++j) f(at(j), s.list_i[first + 64 * j]);
  }
  template <typename S, typename P, typename G, typename B> __device__ __forceinline__ void into(S& s, const P& stays, const G& weight, const B& bin) const {
    each([&](float v, int i) {
      if (stays(v, i)) atomicAdd(&s.hist[bin(v)], weight(v));
    });
  }
  template <typename S, typename P, typename G, typename W> __device__ __forceinline__ u64 find(S& s, const P& stays, const G& weight, const W& want) const {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    u64 sum = 0;
    each([&](float v, int i) { sum += stays(v, i) ? weight(v) : 0; });
    sum = wave_sum_u64(sum);
    __syncthreads();
    if (lane == 0) s.part[wave] = sum;
    __syncthreads();
    u64 all, before = s.before(all);
    const u64 target = want(all);
    if (before < target && before + sum >= target) {   // (one wave)
#pragma clang loop unroll(disable)
      for (int j = 0; j < per; ++j) {
        const float v = at(j);
        const int i = s.list_i[first + 64 * j];
        const u64 own = stays(v, i) ? weight(v) : 0, up = wave_scan_u64(own);
        if (before + up >= target && before + up - own < target) s.border = Border{v, i};
        before += lane_u64(up, 63);
        if (before >= target) break;
      }
    }
    __syncthreads();
    return all;
  }
};

template <int THREADS, int EACH> __device__ __forceinline__ void truncate_clear(TruncateShared<THREADS, EACH>& s) {
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kBins / THREADS; ++j) s.hist[threadIdx.x + j * THREADS] = 0;
  if (threadIdx.x == 0) { s.n = 0; s.bin = -1; }
  __syncthreads();
}
// The bin of the histogram where the sums from `above` on reach want(sum of all) (0: none does); left in s.bin and, what is before it, s.above.  The target.
template <int THREADS, int EACH, typename W> __device__ __forceinline__ u64 truncate_bin(TruncateShared<THREADS, EACH>& s, u64 above, const W& want) {
  constexpr int kEach = kBins / THREADS;
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  __syncthreads();
  u64 h[kEach], own = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) own += h[j] = s.hist[t * kEach + j];
  const u64 up = wave_scan_u64(own);
  if (lane == 63) s.part[wave] = up;
  __syncthreads();
  u64 all, at = above + up - own + s.before(all);
  const u64 target = want(all);
  if (at < target && at + own >= target) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      if (at < target && at + h[j] >= target) { s.bin = t * kEach + j; s.above = at; }
      at += h[j];
    }
  }
  __syncthreads();
  return target;
}

// Ranks s.rank[0 .. n), n <= kList: how many come before each, and the sums of weights up to it, by all waves: each takes 64 of them and compares them with its share of all.
template <int THREADS, int EACH> __device__ __forceinline__ void truncate_rank(TruncateShared<THREADS, EACH>& s, int n) {
  const int t = threadIdx.x, lane = t & 63, wave = alike(t >> 6);
  for (int i = t; i < n; i += THREADS) { s.order(i) = 0; s.sum(i) = 0; }
  __syncthreads();
  const int groups = (n + 63) / 64, shares = THREADS / 64 / groups, group = wave % groups, share = wave / groups, e = group * 64 + lane;
  if (share < shares && e < n) {
    const uint4 own = s.rank[e];
    const Border b{__uint_as_float(own.x), (int)own.y};
    int before = 0;
    u64 up = 0;
    const int end = (share + 1) * n / shares;
#pragma clang loop unroll_count(4)
    for (int j = share * n / shares; j < end; ++j) {
      const uint4 r = s.rank[j];
      if (b.holds(__uint_as_float(r.x), (int)r.y)) { ++before; up += (u64)r.w << 32 | r.z; }
    }
    atomicAdd(&s.order(e), before);   // (with itself)
    atomicAdd(&s.sum(e), up);
  }
  __syncthreads();
}
__device__ __forceinline__ uint4 truncate_entry(float v, int i, u64 w) { return uint4{__float_as_uint(v), (unsigned)i, (unsigned)w, (unsigned)(w >> 32)}; }

// The border of the least front of what `had` holds that sums to the target, from the bin of the first histogram on that holds it.  Sums of weights, or of ones.
template <int THREADS, int EACH, typename X>
__device__ __forceinline__ Border truncate_refine(TruncateShared<THREADS, EACH>& s, const X& x, const Weigh& weigh, bool weights, const Border& had, u64 target) {
  const int t = threadIdx.x, wave = t >> 6, lane = t & 63;
  auto one = [&](float v) -> u64 { return weights ? weigh.of(weigh.below(v)) : 1; };
  float lo = -INFINITY, hi = weigh.m;    // the scores among which the border lies
  int shift = -1;                        // below 0: the first histogram
  auto bin_of = [&](float v) -> int { return shift < 0 ? weigh.bin(v) : (int)((order_of(hi) - order_of(v)) >> max(shift, 0)); };
  auto here = [&](float v, int i) -> bool { return (int)(v >= lo) & (int)(v <= hi) & (int)had.holds(v, i); };
#pragma clang loop unroll(disable)
  for (;;) {
    const int bin = alike(s.bin);
    const u64 above = alike(s.above);
    // that bin's scores
    float least = INFINITY, most = -INFINITY;
    x.each([&](float v, int i) {
      if (here(v, i) && bin_of(v) == bin) {
        least = fminf(least, v); most = fmaxf(most, v);
        const int n = atomicAdd(&s.n, 1);
        if (n < kList) s.rank[n] = truncate_entry(v, i, one(v));
      }
    });
    least = -wave_max(-least); most = wave_max(most);
    if (lane == 0) { s.lo[wave] = least; s.hi[wave] = most; }
    __syncthreads();
    const int n = alike(s.n);
    if (n <= kList) {
      truncate_rank(s, n);
      if (t < n) {
        const uint4 r = s.rank[t];
        const u64 up = above + s.sum(t);
        if (up >= target && up - ((u64)r.w << 32 | r.z) < target) s.border = Border{__uint_as_float(r.x), (int)r.y};
      }
      break;
    }
    lo = alike(-wave_max(-s.lo[lane % (THREADS / 64)])); hi = alike(wave_max(s.hi[lane % (THREADS / 64)]));
    if (lo == hi) {
      const u64 each = alike(one(lo)), nth = (target - above + each - 1) / each;
      x.find(s, [&](float v, int i) -> bool { return (int)(v == lo) & (int)had.holds(v, i); }, [&](float) -> u64 { return 1; }, [&](u64) { return nth; });
      break;
    }
    shift = max(0, 32 - __clz(order_of(hi) - order_of(lo)) - 10);
    truncate_clear(s);
    x.into(s, here, one, bin_of);
    truncate_bin(s, above, [&](u64) { return target; });
  }
  __syncthreads();
  return Border{alike(s.border.x), alike(s.border.i)};
}
__device__ __forceinline__ u64 truncate_part(float p, u64 all) { return max(ceil_part(fmaxf(p, 0.f), all), (u64)1); }
// The border of the first k of what `had` holds, or of its least front with part p of its weights.  k >= what x has: all of that.
template <int THREADS, int EACH, typename X>
__device__ __forceinline__ Border truncate_select(TruncateShared<THREADS, EACH>& s, const X& x, const Weigh& weigh, bool weights, const Border& had, int k, float p) {
  truncate_clear(s);
  x.into(s, [&](float v, int i) { return had.holds(v, i); }, [&](float v) { return weights ? weigh.of(weigh.below(v)) : (u64)1; }, [&](float v) { return weigh.bin(v); });
  const u64 target = truncate_bin(s, 0, [&](u64 all) { return weights ? truncate_part(p, all) : min(all, (u64)k); });
  return truncate_refine(s, x, weigh, weights, had, target);
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

__device__ __forceinline__ u64 pick(bool p, u64 a, u64 b) { return p ? a : b; }
// A list of n <= kList scores, all at once: ranked by all waves, the rest by the first one alone, four neighbours a lane, so without a barrier.  The border of the first k of them; of those, of the front
// with `target` of the weights (0: with part p of theirs); left in s.border.  SAMPLE: then of what stays, and weighs enough for min_p, the least index up to which weights sum to want(sum of all) or more:
// draw(its score, its index, the sum of all), by one lane.
template <bool SAMPLE, int THREADS, int EACH, typename W, typename D>
__device__ __forceinline__ void truncate_short(TruncateShared<THREADS, EACH>& s, int n, const Weigh& weigh, int k, float p, u64 target, const W& want, const D& draw) {
  const int t = threadIdx.x, lane = t & 63;
  if (t < n) {
    const float v = s.list_x[t];
    s.rank[t] = truncate_entry(v, s.list_i[t], weigh.of(weigh.below(v)));
  }
  truncate_rank(s, n);
  if (t >= 64) return;
  k = min(k, n);
  uint4 r[4];
  int place[4];   // (from 1)
  u64 up[4], w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int at = 4 * lane + j;
    const bool mine = at < n;
    r[j] = s.rank[min(at, n - 1)];
    place[j] = mine ? s.order(min(at, n - 1)) : INT_MAX;
    up[j] = s.sum(min(at, n - 1));
    w[j] = (u64)r[j].w << 32 | r[j].z;
  }
  // the one of all lanes' for which f(j): its place and the weights up to it, its score and index
  struct { int place; u64 up; Border b; } found;
  auto only = [&](auto f) {
    int at = -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) at = f(j) ? j : at;
    const int src = max(__ffsll(__ballot(at >= 0)) - 1, 0);
    int pl = place[0];
    u64 u = up[0];
    unsigned x = r[0].x, i = r[0].y;
#pragma unroll
    for (int j = 1; j < 4; ++j) {
      pl = at == j ? place[j] : pl;
      u = pick(at == j, up[j], u);
      x = at == j ? r[j].x : x;
      i = at == j ? r[j].y : i;
    }
    found.place = __builtin_amdgcn_readlane(pl, src);
    found.up = lane_u64(u, src);
    found.b = Border{__uint_as_float((unsigned)__builtin_amdgcn_readlane((int)x, src)), __builtin_amdgcn_readlane((int)i, src)};
  };
  only([&](int j) { return place[j] == k; });
  if (p < 1.f) {
    if (target == 0) target = truncate_part(p, found.up);
    only([&](int j) { return place[j] <= k && up[j] >= target && up[j] - w[j] < target; });
  }
  if constexpr (!SAMPLE) {
    if (lane == 0) s.border = found.b;
  } else {
    u64 e[4], own = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int stays = (int)(place[j] <= found.place) & (int)(weigh.below(__uint_as_float(r[j].x)) <= weigh.most);
      own += e[j] = stays ? w[j] : 0;
    }
    const u64 sums = wave_scan_u64(own), all = lane_u64(sums, 63), to = want(all);
    u64 at = sums - own;
    if (at < to && at + own >= to) {   // (one lane)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (at < to && at + e[j] >= to) draw(__uint_as_float(r[j].x), (int)r[j].y, all);
        at += e[j];
      }
    }
  }
}

// KEEP: vectors of a lane that stay in LDS; EACH: scores of a thread that the list has room for
template <typename T, int THREADS, int KEEP, int EACH, bool SAMPLE>
__global__ __launch_bounds__(THREADS) void k_truncate(TruncateArgs a) {
  __shared__ TruncateShared<THREADS, EACH> s;
  __shared__ uint4 kept[KEEP ? KEEP * THREADS : 1];
  using List = TruncateList<THREADS, EACH>;
  using Row = TruncateRow<T, THREADS, KEEP>;
  constexpr int kWaves = THREADS / 64, kVec = Row::kVec;
  const int row = blockIdx.x, t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const int b = truncate_owner(a, row);
  if (b < 0) return;
  const Row x(a, row, kept);
  const float temp = a.temperature ? a.temperature[b] : 1.f, top_p = a.top_p ? a.top_p[b] : 1.f, min_p = a.min_p ? a.min_p[b] : 0.f;
  const int top_k = a.top_k ? a.top_k[b] : 0;
  const double rate = 128 * 1.44269504088896340736 / (double)temp;
  if (t < 128) s.table[t] = kPowers[t];
  bool clear = true;   // the histogram
#pragma unroll
  for (int j = 0; j < kBins / THREADS; ++j) s.hist[t + j * THREADS] = 0;
  if (t == 0) { s.n = 0; s.bin = -1; }
  float most[8];   // of every eighth of this thread's vectors
#pragma unroll
  for (int j = 0; j < 8; ++j) most[j] = -INFINITY;
  bool bad = !(temp > 0.f && temp < INFINITY) || top_p != top_p || min_p != min_p;
  x.take([&](const float (&v)[kVec], int j) {
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      bad = bad || !(v[e] < INFINITY);
      most[j] = fmaxf(most[j], v[e]);
    }
  });
  constexpr int kLargest = THREADS >= 1024 ? 2 : 8;
  float largest[kLargest];   // of 2048 parts of the row
#pragma unroll
  for (int j = 0; j < kLargest; ++j) {
    largest[j] = most[j];
#pragma unroll
    for (int i = j + kLargest; i < 8; i += kLargest) largest[j] = fmaxf(largest[j], most[i]);
  }
  float m = largest[0];
#pragma unroll
  for (int j = 1; j < kLargest; ++j) m = fmaxf(m, largest[j]);
  m = wave_max(m);
  bad = __any(bad);
  if (lane == 0) { s.hi[wave] = m; s.lo[wave] = bad ? 1.f : 0.f; }
  __syncthreads();
  m = wave_max(s.hi[lane % kWaves]);
  bad = __any(s.lo[lane % kWaves] != 0.f);
  bad = bad || m == -INFINITY;   // no distribution
  m = alike(m);
  Weigh weigh{m, 0.5f * m, fminf((float)(rate * (56 * 0.69314718055994530942 / 128)), 1e30f), rate, INFINITY, min(51, 64 - (32 - __clz(a.vocab))), s.table};
  if (min_p > 0.f) weigh.most = -128.0 * log2((double)fminf(min_p, 1.f));
  Border border{bad ? INFINITY : -INFINITY, -1};
  constexpr int kMost = EACH * THREADS;
  const float u = SAMPLE ? a.u[row] : 0.f;
  auto want = [&](u64 z) { return !(u > 0.f) ? (u64)1 : u >= 1.f ? z : floor_part(u, z) + 1; };
  auto draw = [&](float v, int i, u64 all) {   // the drawn score, its index, the weights of all that stay
    a.tokens[row] = i;
    if (a.log_probs) a.log_probs[row] = (float)(((double)weigh.bits - weigh.below(v) / 128) * 0.69314718055994530942 - log((double)all));
  };
  int n = INT_MAX;   // of the list, once that has all that stays
#pragma clang loop unroll(disable)
  for (int stage = 0; stage < 2; ++stage) {   // top_k, top_p
    const bool weights = stage == 1, first = top_k > 0 && top_k < a.vocab;
    if (bad || !(weights ? top_p < 1.f : first)) continue;
    u64 target = 0;
    if (!weights || !first) {   // (of the first k scores the list has all, or they do not go there)
      if (!clear) truncate_clear(s);
      clear = false;
      if (weights) {
        x.weigh_all(s, weigh);
      } else if (top_k <= kMost) {
#pragma unroll
        for (int j = 0; j < kLargest; ++j)
          if (largest[j] > -INFINITY) atomicAdd(&s.hist[weigh.bin(largest[j])], (u64)1);
      }
      target = alike(truncate_bin(s, 0, [&](u64 all) { return weights ? truncate_part(top_p, all) : all < (u64)top_k ? 0 : (u64)top_k; }));
      const int bin = alike(s.bin);
      // What is in the bins up to the border's goes into the list (the last bin's are not told from what is not there), or, where that has no room for it, what is in the border's alone.
      if (target != 0 && bin < kBins - 1) {
        const float begin = (float)bin, end = begin + 1.f;
        auto near = [&](float v) { return weigh.place(v) < end; };
        n = alike(x.gather(s, most, near, near));
        if (weights && n > kMost) {
          const int among = alike(x.gather(s, most, near, [&](float v) { return weigh.place(v) >= begin && weigh.place(v) < end; }));
          if (among <= kMost) {
            border = truncate_refine(s, List(s, among), weigh, true, border, target);
            break;
          }
        }
      }
      if (!weights) target = 0;
    }
    if (n <= kList) {   // (both at once)
      truncate_short<SAMPLE>(s, n, weigh, first ? top_k : INT_MAX, top_p, target, want, draw);
      if (SAMPLE) return;
      __syncthreads();
      border = Border{alike(s.border.x), alike(s.border.i)};
      break;
    }
    if (n <= kMost) {
      const List list(s, n);
      border = target != 0 ? truncate_refine(s, list, weigh, true, border, target) : truncate_select(s, list, weigh, weights, border, top_k, top_p);
    } else {
      border = target != 0 ? truncate_refine(s, x, weigh, true, border, target) : truncate_select(s, x, weigh, weights, border, top_k, top_p);
    }
  }
  if (SAMPLE && !bad && n == INT_MAX && border.i < 0 && min_p > 0.f) {
    auto stays = [&](float v) { return weigh.below(v) <= weigh.most; };
    n = alike(x.gather(s, most, stays, stays));
  }
  if constexpr (SAMPLE) {
    if (bad) {
      if (t == 0) {
        a.tokens[row] = AD_NEVER;
        if (a.log_probs) a.log_probs[row] = __uint_as_float(0x7fc00000u);
      }
      return;
    }
    auto stays = [&](float v, int i) -> bool { return (int)border.holds(v, i) & (int)(weigh.below(v) <= weigh.most); };
    auto weight = [&](float v) { return weigh.of(weigh.below(v)); };
    const u64 all = n <= kMost ? List(s, n).find(s, stays, weight, want) : x.find(s, stays, weight, want);
    if (t == 0) draw(s.border.x, s.border.i, all);
  } else {
    T* out = (T*)a.out + (size_t)row * a.out_stride;
    const bool wide = (((uintptr_t)out ^ (uintptr_t)x.x) & 15) == 0;
    x.vectors([&](int c, const float (&v)[kVec]) {
      const int i = x.index(c);
      unsigned w[kVec];
      int heavy[kVec];
#pragma unroll
      for (int j = 0; j < kVec; ++j) heavy[j] = 1;
      if (min_p > 0.f) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) heavy[j] = weigh.below(v[j]) <= weigh.most;
      }
      // (selected without a branch: the compiler lost the -inf of a branch's other side)
#pragma unroll
      for (int j = 0; j < kVec; ++j) w[j] = ((int)border.holds(v[j], i + j) & heavy[j]) != 0 ? __float_as_uint(v[j]) : 0xff800000u;
      if (wide && x.whole(i)) {
        uint4 o;
        if constexpr (sizeof(T) == 4) {
          o = uint4{w[0], w[1], w[2], w[3]};
        } else {   // (every value is a bf16 number)
          auto two = [&](int j) { return w[j] >> 16 | w[j + 1]; };
          o = uint4{two(0), two(2), two(4), two(6)};
        }
        gstore((uint4*)(out + i), o);
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          if (i + j >= 0 && i + j < a.vocab) {
            if constexpr (sizeof(T) == 4) gstore((unsigned*)out + i + j, w[j]);
            else gstore((bf16_t*)out + i + j, (bf16_t)(w[j] >> 16));
          }
      }
    });
  }
}

template <bool SAMPLE> static void launch(int dtype, const TruncateArgs& a, hipStream_t s) {
  auto go = [&](auto type) {
    using T = decltype(type);
    constexpr int kVec = 16 / (int)sizeof(T);
    // (256 threads keep as many scores as they have room for in LDS, and four rows share a compute unit)
    if (a.vocab <= 1024 * kVec) k_truncate<T, 256, 4, 2, SAMPLE><<<a.rows, 256, 0, s>>>(a);
    else k_truncate<T, 1024, 8, 2, SAMPLE><<<a.rows, 1024, 0, s>>>(a);
  };
  if (dtype == AD_BF16) go(bf16_t{});
  else go(float{});
}
void launch_sample(int dtype, const TruncateArgs& a, hipStream_t s) { launch<true>(dtype, a, s); }
void launch_truncate(int dtype, const TruncateArgs& a, hipStream_t s) { launch<false>(dtype, a, s); }

}  // namespace ad
