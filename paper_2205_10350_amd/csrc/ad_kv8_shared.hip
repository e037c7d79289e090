// Attention of continuations that share a text: packed query rows over the text's cache, once for all continuations of it, and over each sequence's own (ad_kv8.h has the layouts).
//
// softmax(scale q [K; K']^T) [V; V'] over the keys K of the text and K' of the row's own sequence is two softmaxes, each with its maximum and denominator, joined:
//   m = max(m1, m2), l = l1 2^(m1 - m) + l2 2^(m2 - m), o = (o1 2^(m1 - m) + o2 2^(m2 - m)) / l.
// A text's part takes the rows of all of its continuations together, which lie next to each other, as the rows of one sequence over a closed cache: its keys are fetched once for 32
// rows (of the query heads that share a head among them) instead of once for every continuation.  Both parts are one launch, cut into splits of the keys; a second joins the splits of a row, the text's first.
// A row's sums depend on the caches' sizes, the query heads and the row's own tokens alone.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ad_kv8_attend_device.h"

namespace ad {

// a text's part: the rows of the sequences of group g, and its split of the keys
struct Kv8Shared {
  const unsigned char* cache;
  Kv8Texts texts;
  int split_blocks, n_split;
  unsigned blocks;   // workgroups of it, the launch's first
  Kv8Deal tiles;
};

__device__ __forceinline__ int shared_row(const Kv8Rows& t, const Kv8Texts& x, int g) {   // the first packed row of group g
  return t.start[min(max(x.seq_start[g], 0), t.n_seq)];
}
__device__ __forceinline__ Kv8Seq shared_seq(const Kv8Rows& t, const Kv8Texts& x, int g, const Kv8Dims& d) {
  Kv8Seq s;
  s.row0 = shared_row(t, x, g);
  s.n = shared_row(t, x, g + 1) - s.row0;
  if (s.row0 < 0 || s.row0 > t.rows) s.n = 0;
  s.n = min(min(s.n, x.max_rows), t.rows - s.row0);
  s.base = min(max(x.length[g], 0), d.capacity);
  if (!d.closed) s.base = s.base / kKv8Block * kKv8Block;   // (whole blocks, those in 8 bits)
  return s;
}
__device__ __forceinline__ int shared_first(const Kv8Rows& t, const Kv8Texts& x, const Kv8Deal& d, int g) {   // where the packed tiles of group g begin
  return (int)((long long)min(max(shared_row(t, x, g), 0), t.rows) * d.mul >> d.shift) + d.extra * g;
}
// the last of n things that begins at `at` or before (-1: none): every 64th at once, then those between two of them
template <typename F> __device__ __forceinline__ int shared_owner(int n, int at, const F& first) {
  const int lane = threadIdx.x & 63, apart = (n + 63) / 64;
  int g = __popcll(__ballot(lane * apart < n && first(min(lane * apart, n - 1)) <= at)) - 1;
  if (g < 0) return -1;
  g *= apart;
  if (apart > 1) g += __popcll(__ballot(lane < apart && g + lane < n && first(min(g + lane, n - 1)) <= at)) - 1;
  return g;
}

template <int DH, int FMT>
__global__ __launch_bounds__(256, kv8_waves(DH, 2)) void k_kv8_attend_shared(const unsigned char* __restrict__ cache, Kv8Attend a, Kv8Dims dm, Kv8Shared sh, Kv8Dims ds) {
  __shared__ float Os[4][16 * (DH + 4)];
  __shared__ float Ms[4][16][2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool text = blockIdx.x < sh.blocks;
  const int at = text ? blockIdx.x : blockIdx.x - sh.blocks;
  const Kv8Deal& deal = text ? sh.tiles : a.tiles;
  // workgroup -> ((split, row tile), (sequence, head)), as in the attention over one cache
  int b, h, tile, split;
  if (deal.packed) {
    const int rest = at / dm.heads;
    h = at % dm.heads;
    tile = rest % deal.pieces; split = rest / deal.pieces;
    b = text ? shared_owner(sh.texts.n, tile, [&](int g) { return shared_first(a.rows, sh.texts, sh.tiles, g); }) : kv8_owner(a.rows, a.tiles, tile);
    if (b < 0) return;
    tile -= text ? shared_first(a.rows, sh.texts, sh.tiles, b) : kv8_first(a.rows, a.tiles, b);
    if (tile < 0) return;
  } else {
    const int pairs = (text ? sh.texts.n : a.rows.n_seq) * dm.heads, pair = at % pairs, rest = at / pairs;
    tile = rest % deal.pieces; split = rest / deal.pieces;
    b = pair / dm.heads; h = pair % dm.heads;
  }
  const Kv8Seq sq = text ? shared_seq(a.rows, sh.texts, b, ds) : kv8_seq(a.rows, b, dm.capacity);
  const int m_rows = sq.n * a.group, row0 = tile * 32;
  if (row0 >= m_rows) return;
  const int last = min(row0 + 32, m_rows) - 1;
  const int own_lo = text ? sq.base / kKv8Block : (sq.base + row0 / a.group) / kKv8Block;
  const int own_hi = text ? (sq.base + kKv8Block - 1) / kKv8Block : (sq.base + last / a.group) / kKv8Block;
  const int each = text ? sh.split_blocks : a.split_blocks, blk0 = split * each, blk1 = blk0 + each;
  if (blk0 >= (text ? own_hi : own_hi + 1)) return;   // nothing here for any row
  const size_t bh = (size_t)b * dm.heads + h;
  auto go = [&](auto tiles) {
    Kv8State<DH, tiles.value> st;
    if (text) kv8_wave<DH, tiles.value, FMT, true>(st, sh.cache, a, ds, sq, bh, h, row0, last, own_lo, own_hi, blk0, blk1, wave);
    else kv8_wave<DH, tiles.value, FMT, false>(st, cache, a, dm, sq, bh, h, row0, last, own_lo, own_hi, blk0, blk1, wave);
    kv8_merge<DH, tiles.value>(st, Os, Ms, a, dm, sq, h, row0, last, text ? split : sh.n_split + split, wave);
  };
  if (last - row0 < 16) go(std::integral_constant<int, 1>{});
  else go(std::integral_constant<int, 2>{});
}

// The splits of a (row, query head), a wave each: the text's, then the sequence's own.
template <int DH>
__global__ __launch_bounds__(256) void k_kv8_join_shared(Kv8Attend a, Kv8Deal one, Kv8Dims dm, Kv8Shared sh, Kv8Dims ds) {
  const int col = 4 * ((threadIdx.x & 63) % (DH / 4));
  const int heads = dm.heads * a.group, m = blockIdx.x * 4 + (threadIdx.x >> 6), hq = m % heads;
  const int b = one.packed ? kv8_owner(a.rows, one, m / heads) : blockIdx.y;
  if (b < 0) return;
  const Kv8Seq sq = kv8_seq(a.rows, b, dm.capacity);
  const int i = m / heads - (one.packed ? kv8_first(a.rows, one, b) : 0);
  if (i < 0 || i >= sq.n) return;
  const int row = sq.row0 + i;
  int of_text = 0;
  const int g = shared_owner(sh.texts.n, b, [&](int g) { return sh.texts.seq_start[g]; });
  if (g >= 0 && b < sh.texts.seq_start[g + 1]) {
    const Kv8Seq t = shared_seq(a.rows, sh.texts, g, ds);
    const int blocks = (t.base + kKv8Block - 1) / kKv8Block;
    if (row < t.row0 || row - t.row0 >= t.n) return;   // (beyond the bound on a text's rows: left as it was)
    of_text = min((blocks + sh.split_blocks - 1) / sh.split_blocks, sh.n_split);
  }
  const int own = min(((sq.base + i) / kKv8Block + a.split_blocks) / a.split_blocks, a.n_split - sh.n_split);
  const size_t at = ((size_t)row * heads + hq) * a.n_split;
  Kv8Sum all;
  float4 o;
  if (!kv8_join_splits<DH>((const float2*)a.part_ml + at, a.part_o + at * DH, of_text + own, [&](int s) { return s < of_text ? s : sh.n_split + s - of_text; }, all, o)) return;
  const float inv = all.sum == 0.f ? 0.f : 1.f / all.sum;
  gstore((uint2*)(a.out + (size_t)row * a.out_stride + (size_t)hq * DH + col), uint2{f2bf_pair(o.x * inv, o.y * inv), f2bf_pair(o.z * inv, o.w * inv)});
}

// Keys of a split of a text: by the caches' sizes and the query heads alone, so that a row's sums do not depend on a call.
static int text_split_keys(const Kv8Dims& d, const Kv8Dims& texts, int group) {
  const size_t rows = (size_t)((d.n_seq + texts.n_seq - 1) / texts.n_seq) * group, parts = (size_t)texts.n_seq * d.heads * ((rows + 31) / 32);
  size_t keys = 512;
  while (keys < 8192 && keys * 2048 < parts * texts.capacity) keys *= 2;
  return (int)keys;
}
static int splits(int capacity, int max_keys, int keys) { return (std::min(max_keys, capacity) + keys - 1) / keys; }
static int own_splits(const Kv8Dims& d, int max_keys) { return std::max(1, splits(d.capacity, max_keys, kv8_split_keys(d))); }
static int text_splits(const Kv8Dims& d, const Kv8Dims& texts, int group, int max_keys) { return splits(texts.capacity, max_keys, text_split_keys(d, texts, group)); }
static size_t ml_bytes(size_t parts) { return (parts * 2 * 4 + 255) / 256 * 256; }
size_t kv8_attend_shared_bytes(const Kv8Dims& d, const Kv8Dims& texts, int q_heads, int rows, int max_keys, int max_text_keys) {
  const size_t n = own_splits(d, max_keys) + text_splits(d, texts, q_heads / d.heads, max_text_keys), parts = (size_t)rows * q_heads * n;
  return n == 1 ? 0 : ml_bytes(parts) + parts * d.width * 4;
}
static Kv8Deal tiles_of(const Kv8Rows& r, int group) { return kv8_deal(r, group, 5, 1, (((size_t)r.max_rows * group - 1) >> 5) + 1); }
static size_t of_all(const Kv8Deal& d, size_t n_seq) { return d.packed ? d.pieces : d.pieces * n_seq; }
static Kv8Deal text_tiles(const Kv8Rows& r, const Kv8Texts& x, int group) {
  Kv8Rows t = r;
  t.n_seq = x.n; t.max_rows = std::min(x.max_rows, r.rows);
  return tiles_of(t, group);
}
static size_t text_blocks(const Kv8Dims& d, const Kv8Dims& texts, const Kv8Rows& r, const Kv8Texts& x, int group, int max_text_keys) {
  return x.max_rows == 0 ? 0 : of_all(text_tiles(r, x, group), x.n) * d.heads * text_splits(d, texts, group, max_text_keys);
}
static size_t own_blocks(const Kv8Dims& d, const Kv8Rows& r, int group, int max_keys) { return of_all(tiles_of(r, group), r.n_seq) * d.heads * own_splits(d, max_keys); }
// (a launch takes less than 2^32 lanes along x: 2^24 workgroups of 256)
bool kv8_attend_shared_fits(const Kv8Dims& d, const Kv8Dims& texts, const Kv8Rows& r, const Kv8Texts& x, int q_heads, int max_keys, int max_text_keys) {
  const int group = q_heads / d.heads;
  return text_blocks(d, texts, r, x, group, max_text_keys) + own_blocks(d, r, group, max_keys) < (1u << 24) && (size_t)kv8_deal(r, 1, 0, 0, r.max_rows).pieces * q_heads < (1u << 26);
}

void launch_kv8_attend_shared(const Kv8Dims& d, const void* cache, const Kv8Dims& texts, const void* text_cache, const void* q, size_t q_stride, void* out, size_t out_stride,
                              int q_heads, const Kv8Rows& r, const Kv8Texts& x, int max_keys, int max_text_keys, float scale, void* ws, hipStream_t s) {
  Kv8Attend a;
  a.q = (const bf16_t*)q; a.out = (bf16_t*)out; a.q_stride = q_stride; a.out_stride = out_stride;
  a.rows = r; a.group = q_heads / d.heads; a.scale = scale * kLog2e;
  a.split_blocks = kv8_split_keys(d) / kKv8Block;
  a.tiles = tiles_of(r, a.group);
  Kv8Shared sh;
  sh.cache = (const unsigned char*)text_cache; sh.texts = x;
  sh.split_blocks = text_split_keys(d, texts, a.group) / kKv8Block;
  sh.n_split = text_splits(d, texts, a.group, max_text_keys);
  sh.tiles = text_tiles(r, x, a.group);
  sh.blocks = (unsigned)text_blocks(d, texts, r, x, a.group, max_text_keys);
  a.n_split = sh.n_split + own_splits(d, max_keys);
  const size_t parts = (size_t)r.rows * q_heads * a.n_split;
  a.part_ml = (float*)ws;
  a.part_o = (float*)((char*)ws + ml_bytes(parts));
  const unsigned blocks = sh.blocks + (unsigned)own_blocks(d, r, a.group, max_keys);
  const Kv8Deal one = kv8_deal(r, 1, 0, 0, r.max_rows);
  const dim3 rows((unsigned)(((size_t)one.pieces * q_heads + 3) / 4), one.packed ? 1 : r.n_seq);
  kv8_dispatch(d, [&](auto width, auto fmt) {
    k_kv8_attend_shared<width.value, fmt.value><<<blocks, 256, 0, s>>>((const unsigned char*)cache, a, d, sh, texts);
    if (a.n_split > 1) k_kv8_join_shared<width.value><<<rows, 256, 0, s>>>(a, one, d, sh, texts);
  });
}

}  // namespace ad
