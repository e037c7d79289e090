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
#include "ad_kv8_attend_device.h"

namespace ad {

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

// The splits of a (row, query head), a wave each.
template <int DH>
__global__ __launch_bounds__(256) void k_kv8_join(Kv8Attend a, Kv8Deal one, Kv8Dims dm) {
  const int col = 4 * ((threadIdx.x & 63) % (DH / 4));
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
  Kv8Sum all;
  float4 o;
  if (!kv8_join_splits<DH>((const float2*)a.part_ml + at, a.part_o + at * DH, n, [](int s) { return s; }, all, o)) return;
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
