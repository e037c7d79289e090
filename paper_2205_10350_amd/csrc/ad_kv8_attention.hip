// Attention of packed query rows over 8-bit caches (ad_kv8.h has the layout).
//
// One pass over the keys with the running maximum and denominator of the softmax, products transposed: S^T = K Q^T and O^T = V^T P^T, so that a
// lane holds one query row (lane % 16) throughout and its probabilities are the right operand of the second product as they are.
//  * A wave takes 16 R query rows of a (sequence, head), those of the query heads that share the head among them, and every fourth block of
//    a split's keys: four waves of a workgroup, then the splits, each an online softmax of its own, joined in their order.
//  * Bytes become bf16 operands in registers, exactly; the keys' scale multiplies the scores, the values' the probabilities before they are rounded.
//  * Blocks of 8 bits first, those that every row of the tile sees without a mask; then the rows' own blocks from the bf16 ring.
// A row's sums depend on the cache's sizes and the row's position alone: not on the call's other rows, nor on R, nor on how many splits are launched (blocks and
// splits that a row does not see change nothing in it, to the bit).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ad_device.h"
#include "ad_kv8_device.h"

namespace ad {

constexpr float kLog2e = 1.44269504088896340736f;

// what a launch needs beyond the cache
struct Kv8Attend {
  const bf16_t* q;
  bf16_t* out;
  float *part_o, *part_ml;   // [packed row, query head, split][width], [..][2]; unused with one split
  size_t q_stride, out_stride;
  Kv8Rows rows;
  int group;                 // query heads that share a head
  int split_blocks, n_split; // blocks of a split; splits launched
  int row_tiles;             // workgroups of 16 R rows for a (sequence, head)
  float scale;               // of the scores, times log2(e)
};

// maximum / sum over the four lane groups that hold a row's keys
__device__ __forceinline__ float kv8_rows_max(float m) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  m = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float kv8_rows_sum(float v) {
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

template <int DH, int R> struct Kv8State {
  bf16x8 q[R][DH / 32];
  f32x4 o[R][DH / 16];
  float m[R], l[R];   // of this lane's row: the maximum (all lane groups alike), the denominator's part of this lane's keys
};

// One block: kf(kt, s) and vf(c) give operands; c1: what the raw scores are multiplied by, cv: the values' scale.
// seen(rt): bits of the eight keys of this lane (4 kt + i) that its row sees; MASK false: all.
// (fused multiply-adds are written out: with and without a mask the same roundings)
template <int DH, int R, bool MASK, typename KF, typename VF, typename SEEN>
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
    for (int i = 0; i < 8; ++i) x[i] = !MASK || ((bits >> i) & 1) ? score(i) * c1 : -INFINITY;
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    top = fmaxf(st.m[rt], kv8_rows_max(top));
    const float off = top == -INFINITY ? 0.f : top;   // (a row that has seen nothing yet)
    if (__any(top != st.m[rt])) {
      const float f = __builtin_amdgcn_exp2f(st.m[rt] - off);
      st.m[rt] = top;
      st.l[rt] *= f;
#pragma unroll
      for (int c = 0; c < DH / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[rt][c][i] *= f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = !MASK || ((bits >> i) & 1) ? __builtin_amdgcn_exp2f(fmaf(score(i), c1, -off)) : 0.f;
      st.l[rt] += x[i];
    }
    // (the probabilities of the output product have 8 bits, half a step of 2^-8 relative each, as in every attention of bf16 here; the denominator has 24)
    const uint4 w = uint4{f2bf_pair(x[0] * cv, x[1] * cv), f2bf_pair(x[2] * cv, x[3] * cv), f2bf_pair(x[4] * cv, x[5] * cv), f2bf_pair(x[6] * cv, x[7] * cv)};
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

template <int DH, int R, int FMT, bool CLOSED>
__global__ __launch_bounds__(256) void k_kv8_attend(const unsigned char* __restrict__ cache, Kv8Attend a, Kv8Dims dm) {
  constexpr int kPad = DH + 4;
  __shared__ float Os[4][16 * kPad];
  __shared__ float Ms[4][16][2];
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // workgroup -> ((split, row tile), (sequence, head)): those of one (sequence, head) lie a multiple of n_seq * heads apart, on one XCD where that is
  // a multiple of 8, so that row tiles read the keys from one L2
  const int pairs = a.rows.n_seq * dm.heads;
  const int pair = blockIdx.x % pairs, rest = blockIdx.x / pairs;
  const int tile = rest % a.row_tiles, split = rest / a.row_tiles;
  const int b = pair / dm.heads, h = pair % dm.heads;
  const Kv8Seq sq = kv8_seq(a.rows, b, dm.capacity, !CLOSED);
  const int m_rows = sq.n * a.group, row0 = tile * 16 * R;
  if (row0 >= m_rows) return;
  const int last = min(row0 + 16 * R, m_rows) - 1;
  // blocks: every row sees [0, own_lo) in 8 bits; a row at t sees [0, t / 32) so and its own in bf16 (closed: all in 8 bits, up to the length)
  const int own_lo = CLOSED ? sq.base / kKv8Block : (sq.base + row0 / a.group) / kKv8Block;
  const int own_hi = CLOSED ? (sq.base + kKv8Block - 1) / kKv8Block : (sq.base + last / a.group) / kKv8Block;
  const int blk0 = split * a.split_blocks, blk1 = blk0 + a.split_blocks;
  if (blk0 >= (CLOSED ? max(own_hi, 1) : own_hi + 1)) return;   // nothing here for any row (of an empty memory the first split writes the zeros)

  Kv8State<DH, R> st;
  int pos[R];   // position of this lane's row (closed: the length; rows past the last one repeat it)
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    const int m = min(row0 + 16 * rt + r, last), i = m / a.group, hq = h * a.group + m % a.group;
    pos[rt] = CLOSED ? sq.base : sq.base + i;
    const bf16_t* qp = a.q + (size_t)(sq.row0 + i) * a.q_stride + (size_t)hq * DH + 8 * g;
#pragma unroll
    for (int s = 0; s < DH / 32; ++s) st.q[rt][s] = __builtin_bit_cast(bf16x8, ldg16(qp + 32 * s));
    st.m[rt] = -INFINITY;
    st.l[rt] = 0.f;
#pragma unroll
    for (int c = 0; c < DH / 16; ++c) st.o[rt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const size_t bh = (size_t)b * dm.heads + h;
  {
    const unsigned char* blocks = cache + bh * dm.blocks * (2 * kKv8Block * DH);
    const float2* scales = (const float2*)(cache + dm.scales) + bh * dm.blocks;
    auto take = [&](const Kv8Bytes<DH>& x, int blk) {
      auto kf = [&](int kt, int s) { return kv8_operand<FMT>(kt == 0 ? uint2{x.k[s].x, x.k[s].y} : uint2{x.k[s].z, x.k[s].w}); };
      auto vf = [&](int c) { return kv8_operand<FMT>((c & 1) == 0 ? uint2{x.v[c >> 1].x, x.v[c >> 1].y} : uint2{x.v[c >> 1].z, x.v[c >> 1].w}); };
      const float c1 = x.scale.x * a.scale;
      if (blk < own_lo) {
        kv8_block<DH, R, false>(st, kf, vf, c1, x.scale.y, [](int) { return 0xffu; });
      } else {
        auto seen = [&](int rt) -> unsigned {
          if constexpr (CLOSED) {
            unsigned bits = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) bits |= (blk * kKv8Block + kv8_key(g, j) < pos[rt] ? 1u : 0u) << j;
            return bits;
          } else {
            return blk < pos[rt] / kKv8Block ? 0xffu : 0u;
          }
        };
        kv8_block<DH, R, true>(st, kf, vf, c1, x.scale.y, seen);
      }
    };
    const int end = min(blk1, own_hi);
    int blk = blk0 + wave;
    if (blk < end) {
      Kv8Bytes<DH> x, y;
      kv8_fetch(x, blocks, scales, blk, lane);
      for (; blk < end; blk += 8) {
        if (blk + 4 < end) kv8_fetch(y, blocks, scales, blk + 4, lane);
        take(x, blk);
        if (blk + 4 >= end) break;
        if (blk + 8 < end) kv8_fetch(x, blocks, scales, blk + 8, lane);
        take(y, blk + 4);
      }
    }
  }
  if constexpr (!CLOSED) {
    const bf16_t* ring = (const bf16_t*)(cache + dm.rings) + bh * dm.ring * (2 * kKv8Block * DH);
    int blk = max(own_lo, blk0);
    blk += (wave - blk % 4 + 4) % 4;   // (a split's blocks are dealt to the waves from a multiple of four on)
    for (; blk <= own_hi && blk < blk1; blk += 4) {
      const bf16_t* kp = ring + (size_t)(blk % dm.ring) * (2 * kKv8Block * DH) + lane * 8;
      const bf16_t* vp = kp + kKv8Block * DH;
      uint4 kr[DH / 16], vr[DH / 16];
#pragma unroll
      for (int c = 0; c < DH / 16; ++c) { kr[c] = ldg16(kp + c * 512); vr[c] = ldg16(vp + c * 512); }
      kv8_block<DH, R, true>(
          st, [&](int kt, int s) { return __builtin_bit_cast(bf16x8, kr[2 * s + kt]); }, [&](int c) { return __builtin_bit_cast(bf16x8, vr[c]); }, a.scale, 1.f,
          [&](int rt) -> unsigned {
            unsigned bits = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) bits |= (blk * kKv8Block + kv8_key(g, j) <= pos[rt] ? 1u : 0u) << j;
            return blk == pos[rt] / kKv8Block ? bits : 0u;
          });
    }
  }

  // the four waves' states, in their order
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
    const int i = m / a.group, hq = h * a.group + m % a.group;
    const size_t at = ((size_t)(sq.row0 + i) * (dm.heads * a.group) + hq) * a.n_split + split;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) {
      const int col = 32 * c + 2 * (threadIdx.x & 15);
      float o[2] = {0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        o[0] = fmaf(f[w], Os[w][row * kPad + col], o[0]);
        o[1] = fmaf(f[w], Os[w][row * kPad + col + 1], o[1]);
      }
      if (a.n_split == 1) gstore((unsigned*)(a.out + (size_t)(sq.row0 + i) * a.out_stride + (size_t)hq * DH + col), f2bf_pair(o[0] * inv, o[1] * inv));
      else gstore((float2*)(a.part_o + at * DH + col), float2{o[0], o[1]});
    }
    if (a.n_split > 1 && (threadIdx.x & 15) == 0) gstore((float2*)(a.part_ml + at * 2), float2{top, sum});
  }
}

// The splits of a (row, query head), in their order: one wave, DH / 4 lanes a split and 256 / DH splits at once.
template <int DH>
__global__ __launch_bounds__(256) void k_kv8_join(Kv8Attend a, Kv8Dims dm) {
  constexpr int kLanes = DH / 4, kAtOnce = 64 / kLanes;
  const int lane = threadIdx.x & 63, part = lane / kLanes, col = 4 * (lane % kLanes);
  const int b = blockIdx.y, heads = dm.heads * a.group;
  const Kv8Seq sq = kv8_seq(a.rows, b, dm.capacity, !dm.closed);
  const int m = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= sq.n * heads) return;
  const int i = m / heads, hq = m % heads;
  // a tile's splits are written up to its last row's block; a row's own end is enough, what lies behind holds nothing of it
  const int end = dm.closed ? (sq.base + kKv8Block - 1) / kKv8Block : (sq.base + i) / kKv8Block + 1;
  const int n = min(max(1, (end + a.split_blocks - 1) / a.split_blocks), a.n_split);
  const size_t at = ((size_t)(sq.row0 + i) * heads + hq) * a.n_split;
  float top = -INFINITY, sum = 0.f;
  float4 o = float4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < n; s0 += kAtOnce) {
    const int s = s0 + part;
    if (s >= n) continue;
    const float2 ml = gload((const float2*)(a.part_ml + (at + s) * 2));
    const float4 x = gload((const float4*)(a.part_o + (at + s) * DH + col));
    const float t = fmaxf(top, ml.x), base = t == -INFINITY ? 0.f : t;
    const float f0 = __builtin_amdgcn_exp2f(top - base), f1 = __builtin_amdgcn_exp2f(ml.x - base);
    top = t;
    sum = sum * f0 + ml.y * f1;
    o.x = o.x * f0 + x.x * f1; o.y = o.y * f0 + x.y * f1; o.z = o.z * f0 + x.z * f1; o.w = o.w * f0 + x.w * f1;
  }
#pragma unroll
  for (int step = kLanes; step < 64; step *= 2) {
    const float ot = __shfl_xor(top, step), os = __shfl_xor(sum, step);
    const float t = fmaxf(top, ot), base = t == -INFINITY ? 0.f : t;
    const float f0 = __builtin_amdgcn_exp2f(top - base), f1 = __builtin_amdgcn_exp2f(ot - base);
    sum = sum * f0 + os * f1;
    o.x = o.x * f0 + __shfl_xor(o.x, step) * f1; o.y = o.y * f0 + __shfl_xor(o.y, step) * f1;
    o.z = o.z * f0 + __shfl_xor(o.z, step) * f1; o.w = o.w * f0 + __shfl_xor(o.w, step) * f1;
    top = t;
  }
  if (part) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  gstore((uint2*)(a.out + (size_t)(sq.row0 + i) * a.out_stride + (size_t)hq * DH + col),
         uint2{f2bf_pair(o.x * inv, o.y * inv), f2bf_pair(o.z * inv, o.w * inv)});
}

// The split of the keys: 256 keys give each wave two blocks, the least that hides a fetch; larger ones where the cache's own sizes (sequences, heads, row tiles
// of its longest call) fill the chip without, since every split costs its rows' state on the way to the join.
int kv8_split_keys(const Kv8Dims& d) {
  const size_t units = (size_t)d.n_seq * d.heads * (d.closed ? 1 : (d.k_max + 63) / 64);
  size_t keys = 256;
  while (keys < 8192 && keys * 1024 < units * d.capacity) keys *= 2;
  return (int)keys;
}
static int splits_of(const Kv8Dims& d, int max_keys) {
  const int keys = kv8_split_keys(d);
  return std::max(1, (std::min(max_keys, d.capacity) + keys - 1) / keys);
}
size_t kv8_attend_bytes(const Kv8Dims& d, int q_heads, int rows, int max_keys) {
  const int n = splits_of(d, max_keys);
  return n == 1 ? 0 : ((size_t)rows * q_heads * n * 2 * 4 + 255) / 256 * 256 + (size_t)rows * q_heads * n * d.width * 4;
}

bool kv8_attend_fits(const Kv8Dims& d, int q_heads, int max_rows, int max_keys) {
  const size_t tiles = ((size_t)max_rows * (q_heads / d.heads) + 15) / 16;
  return tiles * d.n_seq * d.heads * splits_of(d, max_keys) < (1u << 31) && (size_t)max_rows * q_heads / 4 < (1u << 31);
}

template <int DH, int FMT>
static void attend_for(const Kv8Dims& d, const unsigned char* cache, Kv8Attend& a, hipStream_t s) {
  const int m = a.rows.max_rows * a.group;
  auto go = [&](auto r, auto closed) {
    a.row_tiles = (m + 16 * r.value - 1) / (16 * r.value);
    k_kv8_attend<DH, r.value, FMT, closed.value><<<(unsigned)((size_t)a.rows.n_seq * d.heads * a.row_tiles * a.n_split), 256, 0, s>>>(cache, a, d);
  };
  auto by_rows = [&](auto closed) {
    // as few passes over the keys as the rows allow: up to 64 rows of a wave (width 128: 32, more would not fit the registers of two waves)
    if (m <= 16) go(std::integral_constant<int, 1>{}, closed);
    else if (m <= 32 || DH == 128) go(std::integral_constant<int, 2>{}, closed);
    else go(std::integral_constant<int, DH == 128 ? 2 : 4>{}, closed);
  };
  if (d.closed) by_rows(std::true_type{});
  else by_rows(std::false_type{});
  if (a.n_split > 1) k_kv8_join<DH><<<dim3((a.rows.max_rows * d.heads * a.group + 3) / 4, a.rows.n_seq), 256, 0, s>>>(a, d);
}
void launch_kv8_attend(const Kv8Dims& d, const void* cache, const void* q, size_t q_stride, void* out, size_t out_stride, int q_heads,
                       const Kv8Rows& r, int max_keys, float scale, void* ws, hipStream_t s) {
  Kv8Attend a;
  a.q = (const bf16_t*)q; a.out = (bf16_t*)out; a.q_stride = q_stride; a.out_stride = out_stride;
  a.rows = r; a.group = q_heads / d.heads; a.scale = scale * kLog2e;
  a.split_blocks = kv8_split_keys(d) / kKv8Block;
  a.n_split = splits_of(d, max_keys);
  a.row_tiles = 1;
  a.part_ml = (float*)ws;
  a.part_o = (float*)((char*)ws + ((size_t)r.rows * q_heads * a.n_split * 2 * 4 + 255) / 256 * 256);
  kv8_dispatch(d, [&](auto width, auto fmt) { attend_for<width.value, fmt.value>(d, (const unsigned char*)cache, a, s); });
}

}  // namespace ad
