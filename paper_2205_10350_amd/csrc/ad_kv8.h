// Key/value caches held in 8 bits: layout and launchers (ad_kv8.hip: written and read back, ad_kv8_attention.hip: attention).
//
// A block is 32 tokens of one (sequence, head) with one fp32 scale for its keys and one for its values.  It lies in memory as the matrix
// instruction of the attention reads it (v_mfma_f32_16x16x32_bf16, keys and transposed values as left operands), so that a wave fetches a
// block by loads of 1 KB, 16 bytes a lane, straight into operand registers:
//   keys:   chunk s (of head width / 32), lane slot l: bytes 0-7 the columns 32 s + 8 (l / 16) .. + 7 of key l % 16, bytes 8-15 the same
//           of key 16 + l % 16
//   values: chunk c (of head width / 32), lane slot l, byte 8 t + j: column 16 (2 c + t) + l % 16 of key kv8_key(l / 16, j)
// kv8_key is the order in which the scores' accumulators of a lane hold the keys, 4 g + j and 16 + 4 g + j - 4: the probabilities become the right operand
// of the output product without leaving their lane.
// The bf16 ring of a growing cache holds the blocks that the last call wrote to: the same order, 16 bits an element, with
//   keys:   chunk 2 s + t, lane slot l: columns 32 s + 8 (l / 16) .. of key 16 t + l % 16
//   values: chunk c (of head width / 16), lane slot l, element j: column 16 c + l % 16 of key kv8_key(l / 16, j)
#pragma once

#include <limits.h>

#include <algorithm>

#include "ad_internal.h"

namespace ad {

constexpr int kKv8Block = 32;

struct Kv8Dims {
  int n_seq, heads, width, capacity, k_max, format, closed;
  int blocks;   // of a (sequence, head): ceil(capacity / 32)
  int ring;     // bf16 blocks of a (sequence, head): as many as k_max tokens can touch (closed: none)
  size_t scales, rings, bytes;   // offsets of the scales (float2: keys, values) and of the ring; size of it all
};
// (cfg checked: ad_kv8_check)
inline Kv8Dims kv8_dims(const ad_kv8_config& c) {
  Kv8Dims d;
  d.n_seq = c.n_seq; d.heads = c.n_heads; d.width = c.head_width; d.capacity = c.capacity;
  d.format = c.format; d.closed = c.closed;
  d.k_max = c.closed ? c.capacity : c.k_max;
  d.blocks = (c.capacity + kKv8Block - 1) / kKv8Block;
  d.ring = c.closed ? 0 : (d.k_max + kKv8Block - 2) / kKv8Block + 1;
  const size_t n = (size_t)c.n_seq * c.n_heads;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  d.scales = up(n * d.blocks * 2 * kKv8Block * c.head_width);
  d.rings = d.scales + up(n * d.blocks * 8);
  d.bytes = d.rings + up(n * d.ring * 4 * kKv8Block * c.head_width);
  return d;
}

// Which packed rows each of n_seq sequences has in a call and how many tokens it had before: entries `stride` ints apart; count == nullptr:
// start[b + 1] - start[b], base == nullptr: 0.
// What the tables say is held to [0, rows) packed rows, max_rows rows a sequence and the capacity, so that a wrong table cannot reach past a buffer.
struct Kv8Rows {
  const int *start, *count, *base;
  int stride, rows, max_rows, n_seq;
};
// How a launch deals out a sequence's pieces of 2^shift / mul rows: as many to every sequence as max_rows have, or, where most of those would not be there, packed:
// sequence b's begin at (start[b] mul >> shift) + extra b, and each workgroup looks its sequence up.  (256 sequences of 25 rows over closed caches of 400 tokens, us without a bound:
// by sequence 653, packed 57, with max_rows = 25 and by sequence 50.)
struct Kv8Deal { int packed, pieces, mul, shift, extra; };   // pieces: of a sequence; packed: of all
inline Kv8Deal kv8_deal(const Kv8Rows& r, int mul, int shift, int extra, size_t of_one) {
  const size_t all = ((size_t)r.rows * mul >> shift) + (size_t)extra * r.n_seq;
  const bool packed = of_one * r.n_seq > 4 * all && all < ((size_t)1 << 23);
  return Kv8Deal{packed, (int)std::min(packed ? all : of_one, (size_t)INT_MAX), mul, shift, extra};
}

// Keys and values of the rows (bf16, [rows, heads, width] with row strides in elements) behind base[b] tokens.
void launch_kv8_append(const Kv8Dims& d, void* cache, const void* k, const void* v, size_t k_stride, size_t v_stride, const Kv8Rows& r, hipStream_t s);
// Tokens base[b] .. of sequences that hold length[b], as the row behind them reads them, to packed rows [rows, heads, width].
void launch_kv8_read(const Kv8Dims& d, const void* cache, const Kv8Rows& r, const int* length, int dtype, void* k_out, void* v_out, hipStream_t s);
// Keys of one split: the keys of a (sequence, head) are cut there whatever the call, so that a row's sums do not depend on it.
int kv8_split_keys(const Kv8Dims& d);
// Attention of the rows over the cache; q_heads / heads query heads share a head.  ws: kv8_attend_bytes().
size_t kv8_attend_bytes(const Kv8Dims& d, int q_heads, int rows, int max_keys);
bool kv8_attend_fits(const Kv8Dims& d, const Kv8Rows& r, int q_heads, int max_keys);   // its workgroups are fewer than a launch may have
void launch_kv8_attend(const Kv8Dims& d, const void* cache, const void* q, size_t q_stride, void* out, size_t out_stride, int q_heads,
                       const Kv8Rows& r, int max_keys, float scale, void* ws, hipStream_t s);

}  // namespace ad
