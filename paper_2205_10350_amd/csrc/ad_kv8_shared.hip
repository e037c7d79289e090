// Attention of continuations that share a text: packed query rows over the text's cache, once for all continuations of it, and over each sequence's own (ad_kv8.h has the layouts).
//
// softmax(scale q [K; K']^T) [V; V'] over the keys K of the text and K' of the row's own sequence is two softmaxes, each with its maximum and denominator, joined:
//   m = max(m1, m2), l = l1 2^(m1 - m) + l2 2^(m2 - m), o = (o1 2^(m1 - m) + o2 2^(m2 - m)) / l.
// A text's part takes the rows of all of its continuations together, which lie next to each other, as the rows of one sequence over a closed cache: its keys are fetched once for 32
// rows (of the query heads that share a head among them) instead of once for every continuation.  Both parts are one launch, cut into splits of the keys; a second joins the splits of a row, the text's first.
// Where a text has 32 continuations (times the query heads that share a head) or more, a workgroup takes 128 of its rows, 32 a wave: all waves go over the same keys, whose operands they unpack
// together, once, into LDS.  Else the waves take every fourth block of keys each for the same rows, as over one cache.  Where texts are short and continuations few, all of it is one launch: a workgroup takes
// 16 rows of a continuation over the text and its own tokens.
// A row's sums depend on the caches' sizes, the query heads and the row's own tokens alone.
//
// Four texts of 8000 tokens, 16 heads of width 64, e4m3, us a replay with a workgroup of 32 rows / of 128, by continuations of each and rows of a continuation: 4 x 1 21.5 / 27.9, 10 x 1 21.4 / 28.3,
// 10 x 8 34.7 / 37.1, 16 x 1 23.0 / 29.2, 16 x 8 46.0 / 43.5, 32 x 1 34.9 / 30.5, 32 x 8 79.9 / 69.5, 64 x 1 56.0 / 44.8, 64 x 25 382 / 376 (210 GFLOP, 560 TFLOP/s); in i8 32 x 8 95.7 / 78.8.
// What bounds it with many rows: vector instructions, 176 (32 of them exponentials, at a quarter of the rate) for 36 matrix instructions over 32 rows and 64 keys, busy two thirds of the time; the
// partial results of the splits (one text of 8192 tokens, 96 continuations of 8 rows: 27 MB written and read, 11 us of 58 for the join).
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
  s.n = kv8_held(s.row0, kv8_range(s.row0, shared_row(t, x, g + 1)), t.rows, x.max_rows);
  s.row0 = min(max(s.row0, 0), t.rows);   // (rows are told from a text's by differences)
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

// workgroup -> ((split, row tile), (sequence, head)), as in the attention over one cache; whether it has one
template <typename O, typename F>
__device__ __forceinline__ bool kv8_where(int at, const Kv8Deal& deal, int n_seq, int heads, const O& owner, const F& first, int& b, int& h, int& tile, int& split) {
  if (deal.packed) {
    const int rest = at / heads;
    h = at % heads;
    tile = rest % deal.pieces; split = rest / deal.pieces;
    b = owner(tile);
    if (b < 0) return false;
    tile -= first(b);
    return tile >= 0;
  }
  const int pairs = n_seq * heads, pair = at % pairs, rest = at / pairs;
  tile = rest % deal.pieces; split = rest / deal.pieces;
  b = pair / heads; h = pair % heads;
  return true;
}

template <int DH, int FMT>
__global__ __launch_bounds__(256, kv8_waves(DH, 2)) void k_kv8_attend_shared(const unsigned char* __restrict__ cache, Kv8Attend a, Kv8Dims dm, Kv8Shared sh, Kv8Dims ds) {
  __shared__ float Os[4][16 * (DH + 4)];
  __shared__ float Ms[4][16][2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool text = blockIdx.x < sh.blocks;
  int b, h, tile, split;
  if (!kv8_where(text ? blockIdx.x : blockIdx.x - sh.blocks, text ? sh.tiles : a.tiles, text ? sh.texts.n : a.rows.n_seq, dm.heads,
                 [&](int at) { return text ? shared_owner(sh.texts.n, at, [&](int g) { return shared_first(a.rows, sh.texts, sh.tiles, g); }) : kv8_owner(a.rows, a.tiles, at); },
                 [&](int b) { return text ? shared_first(a.rows, sh.texts, sh.tiles, b) : kv8_first(a.rows, a.tiles, b); }, b, h, tile, split))
    return;
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

// kv8_block of NB blocks at once, half the reductions and looks at the reference where there are two.  f[j]: block j's operands in LDS; c1, cv: its scales, of the keys times that of the scores and of
// the values (VSCALE); bits: of the eight keys of this lane that rows see (MASK; all see the same).  The denominator of e4m3 is a product of the rounded probabilities with ones, l[rt][0] the
// whole row's; of i8, whose values' scale is in the rounded ones, this lane's part in st.l.
template <int DH, int NB, bool MASK, bool VSCALE>
__device__ __forceinline__ void kv8_text_blocks(Kv8State<DH, 2>& st, f32x4 (&l)[2], const uint4* const (&f)[NB], const float (&c1)[NB], const float (&cv)[NB], unsigned bits) {
  const int lane = threadIdx.x & 63;
  auto of = [&](int j, int op) { return __builtin_bit_cast(bf16x8, f[j][op * 64 + lane]); };
  f32x4 sc[2][2 * NB];   // [row tile][16 keys]
#pragma unroll
  for (int kt = 0; kt < 2 * NB; ++kt) {
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) sc[rt][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < DH / 32; ++s) {
      const bf16x8 a = of(kt / 2, 2 * s + kt % 2);
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) sc[rt][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, st.q[rt][s], sc[rt][kt], 0, 0, 0);
    }
  }
  bf16x8 pf[NB][2];   // [block][row tile]
#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    auto larger = [&](float a, float b) { return kv8_max(a, b, st.inf); };
    auto score = [&](int j, int i) { return !MASK || ((bits >> i) & 1) ? sc[rt][2 * j + (i >> 2)][i & 3] : -INFINITY; };
    auto most = [&](int j) {
      return larger(larger(larger(score(j, 0), score(j, 1)), larger(score(j, 2), score(j, 3))), larger(larger(score(j, 4), score(j, 5)), larger(score(j, 6), score(j, 7)))) * c1[j];
    };
    float top = most(0);
    if constexpr (NB == 2) top = larger(top, most(1));
    top = kv8_rows_max(top, st.inf);
    const bool step = top > st.m[rt] + kStep;
    if (__builtin_expect(__any(step), 0)) {
      const float to = step ? top : st.m[rt];
      const float by = __builtin_amdgcn_exp2f(st.m[rt] - (to == -INFINITY ? 0.f : to));
      st.m[rt] = to;
      if constexpr (VSCALE) st.l[rt] *= by;
      else l[rt][0] *= by;
#pragma unroll
      for (int c = 0; c < DH / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[rt][c][i] *= by;
    }
    const float off = st.m[rt] == -INFINITY ? 0.f : st.m[rt];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = !MASK || ((bits >> i) & 1) ? __builtin_amdgcn_exp2f(fmaf(sc[rt][2 * j + (i >> 2)][i & 3], c1[j], -off)) : 0.f;
      if constexpr (VSCALE) {
        st.l[rt] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= cv[j];
      }
      pf[j][rt] = __builtin_bit_cast(bf16x8, uint4{f2bf_pair(x[0], x[1]), f2bf_pair(x[2], x[3]), f2bf_pair(x[4], x[5]), f2bf_pair(x[6], x[7])});   // (roundings as kv8_block's)
    }
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    if constexpr (!VSCALE) {
      const bf16x8 ones = __builtin_bit_cast(bf16x8, uint4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) l[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[j][rt], l[rt], 0, 0, 0);
    }
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) {
      const bf16x8 a = of(j, DH / 16 + c);
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) st.o[rt][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf[j][rt], st.o[rt][c], 0, 0, 0);
    }
  }
}

// A text's blocks blk0 .. blk1 - 1 for the rows of this wave (none: it only unpacks): two blocks after the other through LDS, where all waves put their operands, in the order that a wave
// reads them in; the next two are on their way from memory.
template <int DH, int FMT>
__device__ __forceinline__ void kv8_text(Kv8State<DH, 2>& st, f32x4 (&l)[2], uint4* lds, const unsigned char* blocks, const float2* scales, float scale, int length, int blk0, int blk1, bool rows) {
  constexpr int kOps = DH / 8, kMine = DH >= 64 ? DH / 64 : 1;   // operands of a block, 1 KB each; a thread's 16 bytes of a block's 2 DH / 32 chunks
  constexpr bool kV = FMT == AD_KV_I8;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4;
  const bool unpacks = DH >= 64 || wave < 2;
  uint4 x[2][kMine];
  float2 sc[2];
  float c1[2], cv[2];
  auto fetch = [&](int blk) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int at = min(blk + n, blk1 - 1);   // (past the last one: again, unused)
      const unsigned char* p = blocks + (size_t)at * (2 * kKv8Block * DH) + t * 16;
      if (unpacks) {
#pragma unroll
        for (int j = 0; j < kMine; ++j) x[n][j] = ldg16(p + j * 4096);
      }
      sc[n] = scales[at];
    }
  };
  uint4* buf = lds;
  auto stage = [&](int blk) {   // blocks blk and blk + 1 into the buffer, and those behind them on their way
    buf = lds + (blk >> 1 & 1) * 2 * kOps * 64;   // (a split begins at a multiple of two blocks)
    if (unpacks) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
          const int chunk = wave + 4 * j;
          const float by = chunk >= DH / 32 ? sc[n].y : 1.f;   // (e4m3: the values' scale)
          uint4* to = buf + (n * kOps + 2 * chunk) * 64 + lane;
          to[0] = __builtin_bit_cast(uint4, kv8_operand<FMT>(uint2{x[n][j].x, x[n][j].y}, by));
          to[64] = __builtin_bit_cast(uint4, kv8_operand<FMT>(uint2{x[n][j].z, x[n][j].w}, by));
        }
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) { c1[n] = sc[n].x * scale; cv[n] = sc[n].y; }
    fetch(blk + 2);
    __syncthreads();   // (one for two blocks: the other buffer's readers are past it)
  };
  fetch(blk0);
  int blk = blk0;
  for (const int whole = min(blk1, length / kKv8Block) - 1; blk < whole; blk += 2) {
    stage(blk);
    if (rows) kv8_text_blocks<DH, 2, false, kV>(st, l, {buf, buf + kOps * 64}, c1, cv, 0xffu);
  }
  if (blk >= blk1) return;
  stage(blk);   // the last one or two, of which the very last may be incomplete
  if (!rows) return;
  for (int n = 0; n < 2 && blk + n < blk1; ++n) {
    unsigned bits = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) bits |= ((blk + n) * kKv8Block + kv8_key(g, j) < length ? 1u : 0u) << j;
    kv8_text_blocks<DH, 1, true, kV>(st, l, {buf + n * kOps * 64}, {n ? c1[1] : c1[0]}, {n ? cv[1] : cv[0]}, bits);
  }
}

// As k_kv8_attend_shared, with 128 rows of a text a workgroup and 16 of a sequence.
template <int DH, int FMT>
__global__ __launch_bounds__(256, DH == 128 ? 2 : 4) void k_kv8_attend_many(const unsigned char* __restrict__ cache, Kv8Attend a, Kv8Dims dm, Kv8Shared sh, Kv8Dims ds) {
  constexpr int kStage = 4 * (DH / 8) * 64 * 16, kMerge = 4 * 16 * (DH + 4) * 4 + 4 * 16 * 2 * 4;
  __shared__ __align__(16) unsigned char lds[kStage > kMerge ? kStage : kMerge];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x >= sh.blocks) {
    int b, h, tile, split;
    if (!kv8_where(blockIdx.x - sh.blocks, a.tiles, a.rows.n_seq, dm.heads, [&](int at) { return kv8_owner(a.rows, a.tiles, at); }, [&](int b) { return kv8_first(a.rows, a.tiles, b); }, b, h, tile, split)) return;
    const Kv8Seq sq = kv8_seq(a.rows, b, dm.capacity);
    const int m_rows = sq.n * a.group, row0 = tile * 16;
    if (row0 >= m_rows) return;
    const int last = min(row0 + 16, m_rows) - 1, own_lo = (sq.base + row0 / a.group) / kKv8Block, own_hi = (sq.base + last / a.group) / kKv8Block;
    const int blk0 = split * a.split_blocks, blk1 = blk0 + a.split_blocks;
    if (blk0 >= own_hi + 1) return;
    Kv8State<DH, 1> st;
    kv8_wave<DH, 1, FMT, false>(st, cache, a, dm, sq, (size_t)b * dm.heads + h, h, row0, last, own_lo, own_hi, blk0, blk1, wave);
    float(*Os)[16 * (DH + 4)] = (float(*)[16 * (DH + 4)])lds;
    kv8_merge<DH, 1>(st, Os, (float(*)[16][2])(lds + 4 * 16 * (DH + 4) * 4), a, dm, sq, h, row0, last, sh.n_split + split, wave);
    return;
  }
  int b, h, tile, split;
  auto first = [&](int g) { return shared_first(a.rows, sh.texts, sh.tiles, g); };
  if (!kv8_where(blockIdx.x, sh.tiles, sh.texts.n, dm.heads, [&](int at) { return shared_owner(sh.texts.n, at, first); }, first, b, h, tile, split)) return;
  const Kv8Seq sq = shared_seq(a.rows, sh.texts, b, ds);
  const int m_rows = sq.n * a.group, row0 = tile * 128 + wave * 32;
  if (tile * 128 >= m_rows) return;
  const int blk0 = split * sh.split_blocks, blk1 = min(blk0 + sh.split_blocks, (sq.base + kKv8Block - 1) / kKv8Block);
  if (blk0 >= blk1) return;
  const bool rows = row0 < m_rows;
  const int last = min(row0 + 32, m_rows) - 1;
  const size_t bh = (size_t)b * dm.heads + h;
  Kv8State<DH, 2> st;
  int pos[2];
  kv8_start<DH, 2>(st, a, sq, h, rows ? row0 : m_rows - 1, rows ? last : m_rows - 1, pos);
  f32x4 sum[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  kv8_text<DH, FMT>(st, sum, (uint4*)lds, sh.cache + bh * ds.blocks * (2 * kKv8Block * DH), (const float2*)(sh.cache + ds.scales) + bh * ds.blocks, fabsf(a.scale), sq.base, blk0, blk1, rows);
  if (!rows) return;
  const int lane = threadIdx.x & 63, g = lane >> 4;
#pragma unroll
  for (int rt = 0; rt < 2; ++rt) {
    const float l = FMT == AD_KV_I8 ? kv8_rows_sum(st.l[rt]) : sum[rt][0];
    const int m = row0 + 16 * rt + (lane & 15);
    if (m > last) continue;
    const size_t at = ((size_t)(sq.row0 + m / a.group) * (dm.heads * a.group) + h * a.group + m % a.group) * a.n_split + split;
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) gstore((f32x4*)(a.part_o + at * DH + 16 * c + 4 * g), st.o[rt][c]);
    if (g == 0) gstore((float2*)(a.part_ml + at * 2), float2{st.m[rt], l});
  }
}

// Short texts and sequences, one split of each and few continuations: a workgroup takes 16 rows of a sequence over its text and its own tokens, and is done.
template <int DH, int FMT>
__global__ __launch_bounds__(256, kv8_waves(DH, 1)) void k_kv8_attend_short(const unsigned char* __restrict__ cache, Kv8Attend a, Kv8Dims dm, Kv8Shared sh, Kv8Dims ds) {
  __shared__ float Os[4][16 * (DH + 4)];
  __shared__ float Ms[4][16][2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int b, h, tile, split;
  if (!kv8_where(blockIdx.x, a.tiles, a.rows.n_seq, dm.heads, [&](int at) { return kv8_owner(a.rows, a.tiles, at); }, [&](int b) { return kv8_first(a.rows, a.tiles, b); }, b, h, tile, split)) return;
  Kv8Seq sq = kv8_seq(a.rows, b, dm.capacity), text{sq.row0, sq.n, 0};
  const int g = __builtin_amdgcn_readfirstlane(shared_owner(sh.texts.n, b, [&](int g) { return sh.texts.seq_start[g]; }));
  if (g >= 0 && b < sh.texts.seq_start[g + 1]) {
    const Kv8Seq t = shared_seq(a.rows, sh.texts, g, ds);
    text.base = min(t.base, sh.split_blocks * kKv8Block);
    sq.n = sq.row0 < t.row0 ? 0 : max(min(sq.n, t.row0 + t.n - sq.row0), 0);   // (beyond the bound on a text's rows: left as they were)
  }
  const int m_rows = sq.n * a.group, row0 = tile * 16;
  if (row0 >= m_rows) return;
  const int last = min(row0 + 16, m_rows) - 1;
  Kv8State<DH, 1> st;
  kv8_wave<DH, 1, FMT, true>(st, sh.cache, a, ds, text, (size_t)max(g, 0) * ds.heads + h, h, row0, last, text.base / kKv8Block, (text.base + kKv8Block - 1) / kKv8Block, 0, sh.split_blocks, wave);
  kv8_wave<DH, 1, FMT, false, false>(st, cache, a, dm, sq, (size_t)b * dm.heads + h, h, row0, last, (sq.base + row0 / a.group) / kKv8Block, (sq.base + last / a.group) / kKv8Block, 0, a.split_blocks, wave);
  kv8_merge<DH, 1>(st, Os, Ms, a, dm, sq, h, row0, last, 0, wave);
}

// The splits of a (row, query head), a wave each: the text's, then the sequence's own.  (Two heads a wave, their tables looked up once: 768 rows of 16 heads the same, 4 of 8 1 us longer.)
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

// What goes by the caches' sizes and the query heads alone, so that a row's sums do not depend on a call: whether a workgroup takes 128 rows of a text, and the keys of a split of it.
static size_t text_fan(const Kv8Dims& d, const Kv8Dims& texts, int group) { return (size_t)((d.n_seq + texts.n_seq - 1) / texts.n_seq) * group; }
// (32 from the table above, in e4m3; i8, whose bytes cost more to unpack, was measured beyond it alone, 32 x 8.)
static bool text_many(const Kv8Dims& d, const Kv8Dims& texts, int group) { return text_fan(d, texts, group) >= 32; }
// (us by keys of a split, 512, 1024, 2048, 4096: workgroups of 32 rows, 40 continuations of 13 rows of 4 texts of 2000 to 8000 tokens in i8 61, 54, 50, 54; of 128, 96 continuations of 8 rows of a text
// of 8192 69, 60, 69, -, 64 of 4 query heads of 2 texts of 16,000 to 32,000 72, 62, 67, -)
static int text_split_keys(const Kv8Dims& d, const Kv8Dims& texts, int group) {
  const bool many = text_many(d, texts, group);
  const size_t rows = text_fan(d, texts, group) * (many ? 1 : std::min(d.k_max, 8)), parts = (size_t)texts.n_seq * d.heads * (many ? (rows + 127) / 128 : (rows + 31) / 32);
  size_t keys = many ? 1024 : 512;
  while (keys < 8192 && keys * 1024 < parts * texts.capacity) keys *= 2;
  return (int)keys;
}
// Short texts and few continuations: each continuation's workgroups read the text for themselves.  (Four texts, 16 heads of width 64, continuations with up to 300 tokens, us a replay in one launch / in two, by
// continuations of a text, rows and tokens of a text: 2 x 1, 512 6.9 / 9.5, 1024 8.4 / 9.5, 2048 11.2 / 10.6; 8 x 1, 512 8.5 / 10.6, 1024 11.6 / 11.5; 8 x 8, 1024 12.2 / 14.9; 16 x 1, 512 11.9 / 13.7, 1024
// 16.5 / 14.9; 16 x 8, 1024 17.3 / 23.4; 31 x 1, 512 19.6 / 19.8; 31 x 8, 512 20.0 / 32.7; 64 x 1, 512 33.7 / 27.2.
// A continuation's rows in a call may not decide, so that a row's sums do not depend on it: 16 x 1 and 8 x 1 over 1024 tokens lose 1.6 and 0.1 us for the 6.1 that 16 x 8 gains.)
static bool text_short(const Kv8Dims& d, const Kv8Dims& texts, int group) {
  return !text_many(d, texts, group) && texts.capacity <= 1024 && text_fan(d, texts, group) * texts.capacity <= 16384 && kv8_split_keys(d) >= d.capacity;
}
static int splits(int capacity, int max_keys, int keys) { return (std::min(max_keys, capacity) + keys - 1) / keys; }
static int own_splits(const Kv8Dims& d, int max_keys) { return std::max(1, splits(d.capacity, max_keys, kv8_split_keys(d))); }
static int text_splits(const Kv8Dims& d, const Kv8Dims& texts, int group, int max_keys) { return splits(texts.capacity, max_keys, text_split_keys(d, texts, group)); }
static size_t ml_bytes(size_t parts) { return (parts * 2 * 4 + 255) / 256 * 256; }
size_t kv8_attend_shared_bytes(const Kv8Dims& d, const Kv8Dims& texts, int q_heads, int rows, int max_keys, int max_text_keys) {
  if (text_short(d, texts, q_heads / d.heads)) return 0;
  const size_t n = own_splits(d, max_keys) + text_splits(d, texts, q_heads / d.heads, max_text_keys), parts = (size_t)rows * q_heads * n;
  return n == 1 ? 0 : ml_bytes(parts) + parts * d.width * 4;
}
static Kv8Deal tiles_of(const Kv8Rows& r, int group, int shift) { return kv8_deal(r, group, shift, 1, (((size_t)r.max_rows * group - 1) >> shift) + 1); }   // of 2^shift rows
static Kv8Deal own_tiles(const Kv8Rows& r, int group, bool small) { return tiles_of(r, group, small ? 4 : 5); }
static size_t of_all(const Kv8Deal& d, size_t n_seq) { return d.packed ? d.pieces : d.pieces * n_seq; }
static Kv8Deal text_tiles(const Kv8Rows& r, const Kv8Texts& x, int group, bool many) {
  Kv8Rows t = r;
  t.n_seq = x.n; t.max_rows = std::min(x.max_rows, r.rows);
  return tiles_of(t, group, many ? 7 : 5);
}
static bool small_tiles(const Kv8Dims& d, const Kv8Dims& texts, int group) { return text_many(d, texts, group) || text_short(d, texts, group); }   // 16 rows of a sequence
static size_t text_blocks(const Kv8Dims& d, const Kv8Dims& texts, const Kv8Rows& r, const Kv8Texts& x, int group, int max_text_keys) {
  return x.max_rows == 0 || text_short(d, texts, group) ? 0 : of_all(text_tiles(r, x, group, text_many(d, texts, group)), x.n) * d.heads * text_splits(d, texts, group, max_text_keys);
}
static size_t own_blocks(const Kv8Dims& d, const Kv8Rows& r, int group, bool small, int max_keys) { return of_all(own_tiles(r, group, small), r.n_seq) * d.heads * own_splits(d, max_keys); }
// (a launch takes less than 2^32 lanes along x: 2^24 workgroups of 256)
bool kv8_attend_shared_fits(const Kv8Dims& d, const Kv8Dims& texts, const Kv8Rows& r, const Kv8Texts& x, int q_heads, int max_keys, int max_text_keys) {
  const int group = q_heads / d.heads;
  return text_blocks(d, texts, r, x, group, max_text_keys) + own_blocks(d, r, group, small_tiles(d, texts, group), max_keys) < (1u << 24) && (size_t)kv8_deal(r, 1, 0, 0, r.max_rows).pieces * q_heads < (1u << 26);
}

void launch_kv8_attend_shared(const Kv8Dims& d, const void* cache, const Kv8Dims& texts, const void* text_cache, const void* q, size_t q_stride, void* out, size_t out_stride,
                              int q_heads, const Kv8Rows& r, const Kv8Texts& x, int max_keys, int max_text_keys, float scale, void* ws, hipStream_t s) {
  Kv8Attend a;
  a.q = (const bf16_t*)q; a.out = (bf16_t*)out; a.q_stride = q_stride; a.out_stride = out_stride;
  a.rows = r; a.group = q_heads / d.heads; a.scale = scale * kLog2e;
  a.split_blocks = kv8_split_keys(d) / kKv8Block;
  const bool many = text_many(d, texts, a.group), one_launch = text_short(d, texts, a.group), small = small_tiles(d, texts, a.group);
  a.tiles = own_tiles(r, a.group, small);
  Kv8Shared sh;
  sh.cache = (const unsigned char*)text_cache; sh.texts = x;
  sh.split_blocks = text_split_keys(d, texts, a.group) / kKv8Block;
  sh.n_split = text_splits(d, texts, a.group, max_text_keys);
  sh.tiles = text_tiles(r, x, a.group, many);
  sh.blocks = (unsigned)text_blocks(d, texts, r, x, a.group, max_text_keys);
  a.n_split = one_launch ? 1 : sh.n_split + own_splits(d, max_keys);
  if (one_launch) sh.split_blocks = (std::min(max_text_keys, texts.capacity) + kKv8Block - 1) / kKv8Block;
  const size_t parts = (size_t)r.rows * q_heads * a.n_split;
  a.part_ml = (float*)ws;
  a.part_o = (float*)((char*)ws + ml_bytes(parts));
  const unsigned blocks = sh.blocks + (unsigned)own_blocks(d, r, a.group, small, max_keys);
  const Kv8Deal one = kv8_deal(r, 1, 0, 0, r.max_rows);
  const dim3 rows((unsigned)(((size_t)one.pieces * q_heads + 3) / 4), one.packed ? 1 : r.n_seq);
  kv8_dispatch(d, [&](auto width, auto fmt) {
    if (one_launch) k_kv8_attend_short<width.value, fmt.value><<<blocks, 256, 0, s>>>((const unsigned char*)cache, a, d, sh, texts);
    else if (many) k_kv8_attend_many<width.value, fmt.value><<<blocks, 256, 0, s>>>((const unsigned char*)cache, a, d, sh, texts);
    else k_kv8_attend_shared<width.value, fmt.value><<<blocks, 256, 0, s>>>((const unsigned char*)cache, a, d, sh, texts);
    if (a.n_split > 1) k_kv8_join_shared<width.value><<<rows, 256, 0, s>>>(a, one, d, sh, texts);
  });
}

}  // namespace ad
