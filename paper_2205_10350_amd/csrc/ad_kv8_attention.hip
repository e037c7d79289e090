// Attention of packed query rows over 8-bit caches (ad_kv8.h has the layout).
//
// One pass over the keys with the running maximum and denominator of the softmax, products transposed: S^T = K Q^T and O^T = V^T P^T, so that a
// lane holds one query row (lane % 16) throughout and its probabilities are the right operand of the second product as they are.
//  * A wave takes 16 R query rows of a (sequence, head), those of the query heads that share the head among them, and every fourth block of
//    a split's keys: four waves of a workgroup, then the splits, each an online softmax of its own, joined in their order.
//  * Two blocks (8 or 16 KB a wave) are on their way while one is worked on, from memory to operand registers without LDS.
//  * Bytes become bf16 operands in registers, exactly; the keys' scale multiplies the scores, the values' the probabilities before they are rounded (e4m3: a
//    power of two, which the conversion of the values applies).
//  * Blocks of 8 bits first, those that every row of the tile sees without a mask; then the rows' own blocks from the bf16 ring.
// A row's sums depend on the cache's sizes and the row's position alone: not on the call's other rows, nor on R, nor on how many splits are launched (blocks and
// splits that a row does not see change nothing in it, to the bit).
//
// What bounds it: few rows over many keys, memory (8 sequences of 16,000 to 32,000 keys, 8 heads of width 128, 4 query heads each: 394 MB in 80 us, 4.9 TB/s, where
// a large copy reaches 5.2; 32 sequences of 1 to 8192 keys, 16 heads of width 64, 1 to 25 rows: 272 MB in 67 us); one sequence, a chain of waits for memory (41 keys
// 4 us, 8216 keys of 16 heads 12); 512 rows, the exponentials and what surrounds them, 130 vector instructions (17 of them exponentials) for 16 matrix
// instructions over 32 rows and 32 keys (26 GFLOP in 65 us, 400 TFLOP/s; a library product reaches 1160).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ad_device.h"
#include "ad_kv8_device.h"

namespace ad {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kStep = 8.f;

// what a launch needs beyond the cache
struct Kv8Attend {
  const bf16_t* q;
  bf16_t* out;
  float *part_o, *part_ml;   // [packed row, query head, split][width], [..][2]; unused with one split
  size_t q_stride, out_stride;
  Kv8Rows rows;
  int group;                 // query heads that share a head
  int split_blocks, n_split; // blocks of a split; splits launched
  Kv8Deal tiles;             // how tiles of 16 R rows are dealt out
  float scale;               // of the scores, times log2(e)
};

// (splits that the join fetches together)
constexpr int kGroup = 4;
struct Kv8Sum { float top, sum; };
// (top, sum) of what came before and of what comes next, and the factors of their outputs
__device__ __forceinline__ Kv8Sum kv8_join(Kv8Sum a, Kv8Sum b, float& fa, float& fb) {
  const float t = fmaxf(a.top, b.top), base = t == -INFINITY ? 0.f : t;
  fa = __builtin_amdgcn_exp2f(a.top - base);
  fb = __builtin_amdgcn_exp2f(b.top - base);
  return Kv8Sum{t, fmaf(b.sum, fb, a.sum * fa)};
}

// the larger of two (of a NaN and a number the number), one instruction where fmaxf first makes signalling NaNs quiet: the middle one of them and infinity, which the
// compiler must not know to be it, or it makes that a maximum again
__device__ __forceinline__ float kv8_max(float a, float b, float inf) { return __builtin_amdgcn_fmed3f(a, b, inf); }
__device__ __forceinline__ float kv8_inf() {
  float v = INFINITY;
  asm("" : "+v"(v));
  return v;
}
// maximum / sum over the four lane groups that hold a row's keys
__device__ __forceinline__ float kv8_rows_max(float m, float inf) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  m = kv8_max(__uint_as_float(p[0]), __uint_as_float(p[1]), inf);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return kv8_max(__uint_as_float(p[0]), __uint_as_float(p[1]), inf);
}
__device__ __forceinline__ float kv8_rows_sum(float v) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// waves a SIMD should hold (its registers are shared out accordingly)
constexpr int kv8_waves(int dh, int r) { return dh == 128 ? 3 - r : 5 - r; }

template <int DH, int R> struct Kv8State {
  bf16x8 q[R][DH / 32];
  f32x4 o[R][DH / 16];
  float inf;          // kv8_inf()
  float m[R], l[R];   // of this lane's row: the exponents' reference (all lane groups alike), the denominator's part of this lane's keys
};

// One block: kf(kt, s) and vf(c) give operands; c1 >= 0: what the raw scores are multiplied by; cv: what the probabilities are, if VSCALE.
// seen(rt): bits of the eight keys of this lane (4 kt + i) that its row sees; MASK false: all.
// (fused multiply-adds are written out: with and without a mask the same roundings)
template <int DH, int R, bool MASK, bool VSCALE, typename KF, typename VF, typename SEEN>
__device__ __forceinline__ void kv8_block(Kv8State<DH, R>& st, const KF& kf, const VF& vf, float c1, float cv, const SEEN& seen) {
  f32x4 sc[R][2];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
    for (int rt = 0; rt < R; ++rt) sc[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < DH / 32; ++s) {
      const bf16x8 a = kf(kt, s);
#pragma unroll
      for (int rt = 0; rt < R; ++rt) sc[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, st.q[rt][s], sc[rt][kt], 0, 0, 0);
    }
  }
  bf16x8 pf[R];
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    unsigned bits = 0xffu;
    if constexpr (MASK) bits = seen(rt);
    auto score = [&](int i) { return sc[rt][i >> 2][i & 3]; };
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = !MASK || ((bits >> i) & 1) ? score(i) : -INFINITY;
    auto larger = [&](float a, float b) { return kv8_max(a, b, st.inf); };
    float top = larger(larger(larger(x[0], x[1]), larger(x[2], x[3])), larger(larger(x[4], x[5]), larger(x[6], x[7])));
    top = kv8_rows_max(top, st.inf) * c1;   // (the largest product is the product of the largest; NaN: ignored here, in the sums below it is not)
    // The reference that a row's exponents are taken from follows its maximum in steps of 2^kStep or more: sums stay far from the ends of fp32 either way, and the
    // sums so far need no rescaling in most blocks.  Which blocks do is a row's own affair; a tile does it for all of its rows, by one for the others.
    const bool step = top > st.m[rt] + kStep;
    if (__any(step)) {
      const float to = step ? top : st.m[rt];
      const float f = __builtin_amdgcn_exp2f(st.m[rt] - (to == -INFINITY ? 0.f : to));
      st.m[rt] = to;
      st.l[rt] *= f;
#pragma unroll
      for (int c = 0; c < DH / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[rt][c][i] *= f;
    }
    const float off = st.m[rt] == -INFINITY ? 0.f : st.m[rt];   // (a row that has seen nothing yet)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = !MASK || ((bits >> i) & 1) ? __builtin_amdgcn_exp2f(fmaf(score(i), c1, -off)) : 0.f;
    if constexpr (VSCALE) {
      st.l[rt] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= cv;
    }
    // (the probabilities of the output product have 8 bits, half a step of 2^-8 relative each, as in every attention of bf16 here; the denominator has 24, of the rounded
    // ones where they are what the values are multiplied by: two to an instruction)
    const uint4 w = uint4{f2bf_pair(x[0], x[1]), f2bf_pair(x[2], x[3]), f2bf_pair(x[4], x[5]), f2bf_pair(x[6], x[7])};
    if constexpr (!VSCALE) {
      auto two = [](unsigned v) { return __builtin_bit_cast(kv8_bf16x2, v); };
      const kv8_bf16x2 one = two(0x3f803f80u);
      st.l[rt] = __builtin_amdgcn_fdot2_f32_bf16(two(w.w), one, __builtin_amdgcn_fdot2_f32_bf16(two(w.z), one, __builtin_amdgcn_fdot2_f32_bf16(two(w.y), one, __builtin_amdgcn_fdot2_f32_bf16(two(w.x), one, st.l[rt], false), false), false), false);
    }
    pf[rt] = __builtin_bit_cast(bf16x8, w);
  }
#pragma unroll
  for (int c = 0; c < DH / 16; ++c) {
    const bf16x8 a = vf(c);
#pragma unroll
    for (int rt = 0; rt < R; ++rt) st.o[rt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[rt], st.o[rt][c], 0, 0, 0);
  }
}

// a block's bytes on their way: DH / 32 pieces of 16 bytes a lane each of keys and values, and the scales
template <int DH> struct Kv8Bytes {
  uint4 k[DH / 32], v[DH / 32];
  float2 scale;
};
template <int DH> __device__ __forceinline__ void kv8_fetch(Kv8Bytes<DH>& x, const unsigned char* blocks, const float2* scales, int blk, int lane) {
  const unsigned char* p = blocks + (size_t)blk * (2 * kKv8Block * DH) + lane * 16;
#pragma unroll
  for (int s = 0; s < DH / 32; ++s) x.k[s] = ldg16(p + s * 1024);
#pragma unroll
  for (int s = 0; s < DH / 32; ++s) x.v[s] = ldg16(p + kKv8Block * DH + s * 1024);
  x.scale = scales[blk];
}

// The state of rows row0 .. last of a (sequence, head) over a split's blocks of this wave, two blocks on their way while one is worked on.
template <int DH, int R, int FMT, bool CLOSED>
__device__ __forceinline__ void kv8_wave(Kv8State<DH, R>& st, const unsigned char* cache, const Kv8Attend& a, const Kv8Dims& dm, const Kv8Seq& sq, size_t bh, int h,
                                         int row0, int last, int own_lo, int own_hi, int blk0, int blk1, int wave) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const unsigned char* blocks = cache + bh * dm.blocks * (2 * kKv8Block * DH);
  const float2* scales = (const float2*)(cache + dm.scales) + bh * dm.blocks;
  const int whole = min(blk1, own_lo), end = min(blk1, own_hi);
  int blk = blk0 + wave;
  constexpr int kAhead = 2;
  Kv8Bytes<DH> x[kAhead + 1];
#pragma unroll
  for (int n = 0; n < kAhead; ++n)
    if (blk + 4 * n < whole) kv8_fetch(x[n], blocks, scales, blk + 4 * n, lane);
  int pos[R];   // position of this lane's row (closed: the length; rows past the last one repeat it)
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    const int m = min(row0 + 16 * rt + r, last), i = m / a.group, hq = h * a.group + m % a.group;
    pos[rt] = CLOSED ? sq.base : sq.base + i;
    const bf16_t* qp = a.q + (size_t)(sq.row0 + i) * a.q_stride + (size_t)hq * DH + 8 * g;
#pragma unroll
    for (int s = 0; s < DH / 32; ++s) {
      uint4 w = ldg16(qp + 32 * s);
      if (a.scale < 0.f) { w.x ^= 0x80008000u; w.y ^= 0x80008000u; w.z ^= 0x80008000u; w.w ^= 0x80008000u; }
      st.q[rt][s] = __builtin_bit_cast(bf16x8, w);
    }
    st.m[rt] = -INFINITY;
    st.l[rt] = 0.f;
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) st.o[rt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  st.inf = kv8_inf();
  const float scale = fabsf(a.scale);
  auto take = [&](auto mask, const Kv8Bytes<DH>& x, int blk) {
    auto kf = [&](int kt, int s) { return kv8_operand<FMT>(kt == 0 ? uint2{x.k[s].x, x.k[s].y} : uint2{x.k[s].z, x.k[s].w}, 1.f); };
    auto vf = [&](int c) { return kv8_operand<FMT>((c & 1) == 0 ? uint2{x.v[c >> 1].x, x.v[c >> 1].y} : uint2{x.v[c >> 1].z, x.v[c >> 1].w}, x.scale.y); };
    auto seen = [&](int rt) -> unsigned {
      if constexpr (!mask.value) return 0xffu;
      if constexpr (CLOSED) {
        unsigned bits = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) bits |= (blk * kKv8Block + kv8_key(g, j) < pos[rt] ? 1u : 0u) << j;
        return bits;
      } else {
        return blk < pos[rt] / kKv8Block ? 0xffu : 0u;
      }
    };
    kv8_block<DH, R, mask.value, FMT == AD_KV_I8>(st, kf, vf, x.scale.x * scale, x.scale.y, seen);
  };
  const std::false_type all{};
  const std::true_type some{};
  while (blk < whole) {
#pragma unroll
    for (int n = 0; n <= kAhead; ++n) {
      if (blk + 4 * kAhead < whole) kv8_fetch(x[(n + kAhead) % (kAhead + 1)], blocks, scales, blk + 4 * kAhead, lane);
      take(all, x[n], blk);
      blk += 4;
      if (blk >= whole) break;
    }
  }
  for (; blk < end; blk += 4) {   // blocks that some of the rows see
    kv8_fetch(x[0], blocks, scales, blk, lane);
    take(some, x[0], blk);
  }
  if constexpr (!CLOSED) {
    const bf16_t* ring = (const bf16_t*)(cache + dm.rings) + bh * dm.ring * (2 * kKv8Block * DH);
    int own = max(own_lo, blk0);
    own += (wave - own % 4 + 4) % 4;   // (a split's blocks are dealt to the waves from a multiple of four on)
    for (; own <= own_hi && own < blk1; own += 4) {
      const bf16_t* kp = ring + (size_t)(own % dm.ring) * (2 * kKv8Block * DH) + lane * 8;
      const bf16_t* vp = kp + kKv8Block * DH;
      uint4 kr[DH / 16], vr[DH / 16];
#pragma unroll
      for (int c = 0; c < DH / 16; ++c) { kr[c] = ldg16(kp + c * 512); vr[c] = ldg16(vp + c * 512); }
      kv8_block<DH, R, true, false>(
          st, [&](int kt, int s) { return __builtin_bit_cast(bf16x8, kr[2 * s + kt]); }, [&](int c) { return __builtin_bit_cast(bf16x8, vr[c]); }, scale, 1.f,
          [&](int rt) -> unsigned {
            unsigned bits = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) bits |= (own * kKv8Block + kv8_key(g, j) <= pos[rt] ? 1u : 0u) << j;
            return own == pos[rt] / kKv8Block ? bits : 0u;
          });
    }
  }
}

// The four waves' states of a tile, in their order: to the output, or to the join's workspace.
template <int DH, int R>
__device__ __forceinline__ void kv8_merge(const Kv8State<DH, R>& st, float (*Os)[16 * (DH + 4)], float (*Ms)[16][2], const Kv8Attend& a, const Kv8Dims& dm,
                                          const Kv8Seq& sq, int h, int row0, int last, int split, int wave) {
  constexpr int kPad = DH + 4;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    if (rt) __syncthreads();
    const float l = kv8_rows_sum(st.l[rt]);
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) *(f32x4*)&Os[wave][r * kPad + 16 * c + 4 * g] = st.o[rt][c];
    if (g == 0) { Ms[wave][r][0] = st.m[rt]; Ms[wave][r][1] = l; }
    __syncthreads();
    const int row = threadIdx.x >> 4, m = row0 + 16 * rt + row;   // 16 threads a row
    if (m > last) continue;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, Ms[w][row][0]);
    float f[4], sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[w] = __builtin_amdgcn_exp2f(Ms[w][row][0] - (top == -INFINITY ? 0.f : top));
      sum = fmaf(f[w], Ms[w][row][1], sum);
    }
    float o[DH / 16];
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) {
      const int col = 32 * (c / 2) + 2 * (threadIdx.x & 15) + (c & 1);
      o[c] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) o[c] = fmaf(f[w], Os[w][row * kPad + col], o[c]);
    }
    const int i = m / a.group, hq = h * a.group + m % a.group;
    const size_t at = ((size_t)(sq.row0 + i) * (dm.heads * a.group) + hq) * a.n_split + split;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int c = 0; c < DH / 16; c += 2) {
      const int col = 16 * c + 2 * (threadIdx.x & 15);
      if (a.n_split == 1) gstore((unsigned*)(a.out + (size_t)(sq.row0 + i) * a.out_stride + (size_t)hq * DH + col), f2bf_pair(o[c] * inv, o[c + 1] * inv));
      else gstore((float2*)(a.part_o + at * DH + col), float2{o[c], o[c + 1]});
    }
    if (a.n_split > 1 && (threadIdx.x & 15) == 0) gstore((float2*)(a.part_ml + at * 2), float2{top, sum});
  }
}

// One workgroup per 16 R rows, (sequence, head) and split.  Of 32 rows where there are no more than 16, half the work (a batch's blocks are ragged).
template <int DH, int R, int FMT, bool CLOSED>
__global__ __launch_bounds__(256, kv8_waves(DH, R)) void k_kv8_attend(const unsigned char* __restrict__ cache, Kv8Attend a, Kv8Dims dm) {
  __shared__ float Os[4][16 * (DH + 4)];
  __shared__ float Ms[4][16][2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // workgroup -> ((split, row tile), (sequence, head)): those of one (sequence, head) lie a multiple of n_seq * heads apart, on one XCD where that is
  // a multiple of 8, so that row tiles read the keys from one L2
  int b, h, tile, split;
  if (a.tiles.packed) {
    const int rest = blockIdx.x / dm.heads;
    h = blockIdx.x % dm.heads;
    tile = rest % a.tiles.pieces; split = rest / a.tiles.pieces;
    b = kv8_owner(a.rows, a.tiles, tile);
    if (b < 0) return;
    tile -= kv8_first(a.rows, a.tiles, b);
    if (tile < 0) return;
  } else {
    const int pairs = a.rows.n_seq * dm.heads, pair = blockIdx.x % pairs, rest = blockIdx.x / pairs;
    tile = rest % a.tiles.pieces; split = rest / a.tiles.pieces;
    b = pair / dm.heads; h = pair % dm.heads;
  }
  const Kv8Seq sq = kv8_seq(a.rows, b, dm.capacity, !CLOSED);
  const int m_rows = sq.n * a.group, row0 = tile * 16 * R;
  if (row0 >= m_rows) return;
  const int last = min(row0 + 16 * R, m_rows) - 1;
  // blocks: every row sees [0, own_lo) in 8 bits; a row at t sees [0, t / 32) so and its own in bf16 (closed: all in 8 bits, up to the length)
  const int own_lo = CLOSED ? sq.base / kKv8Block : (sq.base + row0 / a.group) / kKv8Block;
  const int own_hi = CLOSED ? (sq.base + kKv8Block - 1) / kKv8Block : (sq.base + last / a.group) / kKv8Block;
  const int blk0 = split * a.split_blocks, blk1 = blk0 + a.split_blocks;
  if (blk0 >= (CLOSED ? max(own_hi, 1) : own_hi + 1)) return;   // nothing here for any row (of an empty memory the first split writes the zeros)
  const size_t bh = (size_t)b * dm.heads + h;
  auto go = [&](auto tiles) {
    Kv8State<DH, tiles.value> st;
    kv8_wave<DH, tiles.value, FMT, CLOSED>(st, cache, a, dm, sq, bh, h, row0, last, own_lo, own_hi, blk0, blk1, wave);
    kv8_merge<DH, tiles.value>(st, Os, Ms, a, dm, sq, h, row0, last, split, wave);
  };
  if constexpr (R == 2) {
    if (last - row0 < 16) {
      go(std::integral_constant<int, 1>{});
      return;
    }
  }
  go(std::integral_constant<int, R>{});
}

// The splits of a (row, query head): one wave, DH / 4 lanes a group of kGroup and 256 / DH groups at once; joined group by group, a group's in their order.
template <int DH>
__global__ __launch_bounds__(256) void k_kv8_join(Kv8Attend a, Kv8Deal one, Kv8Dims dm) {
  constexpr int kLanes = DH / 4, kAtOnce = 64 / kLanes;
  const int lane = threadIdx.x & 63, part = lane / kLanes, col = 4 * (lane % kLanes);
  const int heads = dm.heads * a.group, m = blockIdx.x * 4 + (threadIdx.x >> 6), hq = m % heads;
  const int b = one.packed ? kv8_owner(a.rows, one, m / heads) : blockIdx.y;
  if (b < 0) return;
  const Kv8Seq sq = kv8_seq(a.rows, b, dm.capacity, !dm.closed);
  const int i = m / heads - (one.packed ? kv8_first(a.rows, one, b) : 0);
  if (i < 0 || i >= sq.n) return;
  // a tile's splits are written up to its last row's block; a row's own end is enough, what lies behind holds nothing of it
  const int end = dm.closed ? (sq.base + kKv8Block - 1) / kKv8Block : (sq.base + i) / kKv8Block + 1;
  const int n = min(max(1, (end + a.split_blocks - 1) / a.split_blocks), a.n_split);
  const size_t at = ((size_t)(sq.row0 + i) * heads + hq) * a.n_split;
  const float2* ml = (const float2*)a.part_ml + at;
  const float* po = a.part_o + at * DH + col;
  Kv8Sum all{-INFINITY, 0.f};
  float4 o = float4{0.f, 0.f, 0.f, 0.f};
  auto add = [](Kv8Sum& s, float4& o, Kv8Sum n, float4 x) {
    float fa, fb;
    s = kv8_join(s, n, fa, fb);
    o.x = fmaf(x.x, fb, o.x * fa); o.y = fmaf(x.y, fb, o.y * fa); o.z = fmaf(x.z, fb, o.z * fa); o.w = fmaf(x.w, fb, o.w * fa);
  };
  const int groups = (n + kGroup - 1) / kGroup;
  for (int g = part; g < groups; g += kAtOnce) {
    float2 w[kGroup];
    float4 x[kGroup];
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      const int s = min(g * kGroup + j, n - 1);   // (past the last one: read again, counted as nothing)
      w[j] = gload(ml + s);
      x[j] = gload((const float4*)(po + (size_t)s * DH));
      if (g * kGroup + j >= n) { w[j] = float2{-INFINITY, 0.f}; x[j] = float4{0.f, 0.f, 0.f, 0.f}; }
    }
    Kv8Sum s{w[0].x, w[0].y};
    float4 y = x[0];
#pragma unroll
    for (int j = 1; j < kGroup; ++j) add(s, y, Kv8Sum{w[j].x, w[j].y}, x[j]);
    add(all, o, s, y);
  }
#pragma unroll
  for (int step = kLanes; step < 64; step *= 2) {
    const Kv8Sum other{__shfl_xor(all.top, step), __shfl_xor(all.sum, step)};
    const float4 x{__shfl_xor(o.x, step), __shfl_xor(o.y, step), __shfl_xor(o.z, step), __shfl_xor(o.w, step)};
    // (both sides of a pair do the same sum in the same order)
    if (lane & step) {
      Kv8Sum s = other;
      float4 y = x;
      add(s, y, all, o);
      all = s; o = y;
    } else {
      add(all, o, other, x);
    }
  }
  if (part) return;
  const float inv = all.sum == 0.f ? 0.f : 1.f / all.sum;
  gstore((uint2*)(a.out + (size_t)(sq.row0 + i) * a.out_stride + (size_t)hq * DH + col),
         uint2{f2bf_pair(o.x * inv, o.y * inv), f2bf_pair(o.z * inv, o.w * inv)});
}

// The split of the keys.  It goes by the cache's own sizes, so that a row's sums do not depend on a call: few rows over one output want short splits, many rows or
// sequences long ones, and the rule lies between them.  512 keys where sequences and heads are few, more where all of them together
// would have over 2048 splits, which fill the card, or where a call may bring many rows, which fill it too.  Measured in caches for calls of up to 512 rows, us a replay by keys of a split (512, 1024, 2048, 4096, 8192; in
// brackets what the rule takes): 25 rows over 8216 keys, 16 heads 12.1 [13.6] 17.5 25.4 42.3; 2 prompts' pieces of 512 rows over up to 8000 keys 83.6 [71.5] 65.0 65.0
// 57.7; 32 sequences of up to 8192 keys, i8, 66.2 59.5 [58.8] 56.2 67.0; 8 sequences of up to 32,000 keys, 8 heads of width 128, 89.7 [84.1] 83.5 80.7 75.5.
int kv8_split_keys(const Kv8Dims& d) {
  const size_t pairs = (size_t)d.n_seq * d.heads;
  size_t keys = 512;
  while (keys < 8192 && ((!d.closed && keys < 2 * (size_t)d.k_max) || keys * 2048 < pairs * d.capacity)) keys *= 2;
  return (int)keys;
}
static int splits_of(const Kv8Dims& d, int max_keys) {
  const int keys = kv8_split_keys(d);
  return std::max(1, (std::min(max_keys, d.capacity) + keys - 1) / keys);
}
size_t kv8_attend_bytes(const Kv8Dims& d, int q_heads, int rows, int max_keys) {
  const size_t n = splits_of(d, max_keys);
  return n == 1 ? 0 : ((size_t)rows * q_heads * n * 2 * 4 + 255) / 256 * 256 + (size_t)rows * q_heads * n * d.width * 4;
}
// 16 or 32 rows of a wave.  (64, two waves a SIMD instead of three: 512 rows over 32 keys 11.3 us, with 32 7.3; over 1024 21.1 and 17.6, over 8192 47.3 and
// 45.3: a row tile more reads its keys from L2, and the third wave fills the other two's waits.)
static bool one_tile(const Kv8Rows& r, int group) { return (size_t)r.max_rows * group <= 16; }
static Kv8Deal tiles_of(const Kv8Rows& r, int group) {
  const int shift = one_tile(r, group) ? 4 : 5;
  return kv8_deal(r, group, shift, 1, (((size_t)r.max_rows * group - 1) >> shift) + 1);
}
static size_t of_all(const Kv8Deal& d, const Kv8Rows& r) { return d.packed ? d.pieces : (size_t)d.pieces * r.n_seq; }
// a launch takes less than 2^32 lanes along x: 2^24 workgroups of 256
bool kv8_attend_fits(const Kv8Dims& d, const Kv8Rows& r, int q_heads, int max_keys) {
  return of_all(tiles_of(r, q_heads / d.heads), r) * d.heads * splits_of(d, max_keys) < (1u << 24) && (size_t)kv8_deal(r, 1, 0, 0, r.max_rows).pieces * q_heads < (1u << 26);
}

template <int DH, int FMT>
static void attend_for(const Kv8Dims& d, const unsigned char* cache, Kv8Attend& a, hipStream_t s) {
  auto go = [&](auto r, auto closed) {
    k_kv8_attend<DH, r.value, FMT, closed.value><<<(unsigned)(of_all(a.tiles, a.rows) * d.heads * a.n_split), 256, 0, s>>>(cache, a, d);
  };
  auto by_rows = [&](auto closed) {
    if (one_tile(a.rows, a.group)) go(std::integral_constant<int, 1>{}, closed);
    else go(std::integral_constant<int, 2>{}, closed);
  };
  if (d.closed) by_rows(std::true_type{});
  else by_rows(std::false_type{});
  if (a.n_split > 1) {
    const Kv8Deal one = kv8_deal(a.rows, 1, 0, 0, a.rows.max_rows);
    k_kv8_join<DH><<<dim3((unsigned)(((size_t)one.pieces * d.heads * a.group + 3) / 4), one.packed ? 1 : a.rows.n_seq), 256, 0, s>>>(a, one, d);
  }
}
void launch_kv8_attend(const Kv8Dims& d, const void* cache, const void* q, size_t q_stride, void* out, size_t out_stride, int q_heads,
                       const Kv8Rows& r, int max_keys, float scale, void* ws, hipStream_t s) {
  Kv8Attend a;
  a.q = (const bf16_t*)q; a.out = (bf16_t*)out; a.q_stride = q_stride; a.out_stride = out_stride;
  a.rows = r; a.group = q_heads / d.heads; a.scale = scale * kLog2e;
  a.split_blocks = kv8_split_keys(d) / kKv8Block;
  a.n_split = splits_of(d, max_keys);
  a.tiles = tiles_of(r, a.group);
  a.part_ml = (float*)ws;
  a.part_o = (float*)((char*)ws + ((size_t)r.rows * q_heads * a.n_split * 2 * 4 + 255) / 256 * 256);
  kv8_dispatch(d, [&](auto width, auto fmt) { attend_for<width.value, fmt.value>(d, (const unsigned char*)cache, a, s); });
}

}  // namespace ad
