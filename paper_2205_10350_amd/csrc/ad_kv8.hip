// Caches in 8 bits, written and read back (ad_kv8.h has the layout).
//
// A block of 32 tokens and one head, x[32, width] with most = max |x|, is held as
//   e4m3: unit = the least power of two with most <= 448 unit (at least 2^-126): byte = e4m3(x / unit), rounded to nearest, ties to even.  x / unit is
//         exact, and so are byte * unit in bf16 and the products of the attention.
//   i8:   byte = x * 127 / most rounded to nearest, ties to even; scale = most / 127 in fp32.
// once its last token is there; until then, and while a row of the call that wrote it may read it, its tokens lie in the bf16 ring.
// A token whose keys or values of a head are not finite keeps NaN for its keys and 0 for its values there (and so does the whole block's scale of the
// keys): every row that reads it becomes NaN, and no row that must not see it is touched by it (0 * inf in a product).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ad_device.h"
#include "ad_kv8_device.h"

namespace ad {

// scale of a block and the factor pair that brings a value x to its byte
struct Kv8Quant {
  float scale;        // byte -> value
  float shift;        // e4m3: 1 / unit;  i8: the power of two that brings most near 1 (products with 127 stay in range)
  float m;            // i8: most * shift
};
template <int FMT> __device__ __forceinline__ Kv8Quant kv8_quant(float most) {
  Kv8Quant q;
  const int e = __builtin_amdgcn_frexp_expf(most);
  if constexpr (FMT == AD_KV_E4M3) {
    const int u = most == 0.f ? 0 : max(__builtin_amdgcn_frexp_mantf(most) <= 0.875f ? e - 9 : e - 8, -126);   // 448 = 0.875 * 2^9
    q.m = 1.f;
    q.scale = ldexpf(1.f, u);
    q.shift = ldexpf(1.f, -u);
  } else {
    q.scale = most == 0.f ? 1.f : most / 127.f;
    q.shift = ldexpf(1.f, min(max(-e, -126), 126));
    q.m = most == 0.f ? 1.f : most * q.shift;
  }
  return q;
}
template <int FMT> __device__ __forceinline__ unsigned kv8_pack4(const float (&x)[4], const Kv8Quant& q) {
  if constexpr (FMT == AD_KV_E4M3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * q.shift, x[1] * q.shift, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * q.shift, x[3] * q.shift, w, true);
  } else {
    // x * shift * 127 is exact (8 bits times 7), the division correctly rounded: a half between two steps is seen as one
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int v = (int)rintf(x[i] * q.shift * 127.f / q.m);
      w |= ((unsigned)v & 0xffu) << (8 * i);
    }
    return w;
  }
}

// One workgroup per (touched block, head, sequence), 4 * DH threads: the first half takes the keys, the second the values, a thread 16 elements.
// Both sides load rows 8 columns at a time; the values are turned in LDS.  Bound by memory (2 bytes in, 3 out for an element of an
// open block or a ring that a row may read): 8 prompts of 1000 to 2048 rows, 16 heads of width 64, 125 MB in 28 us, 4.5 TB/s; one token 4.4 us, a launch and three waits.
// (A thread's bytes are packed into words by hand: through arrays that were read under another type the compiler put them into scratch memory, 41 us.)
template <int DH, int FMT, bool CLOSED>
__global__ __launch_bounds__(4 * DH) void k_kv8_append(unsigned char* __restrict__ cache, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v,
                                                       size_t k_stride, size_t v_stride, Kv8Rows rt, Kv8Deal deal, Kv8Dims dm) {
  constexpr int kThreads = 4 * DH, kHalf = 2 * DH, kWaves = kThreads / 64, kLdv = DH + 2;
  __shared__ bf16_t Vs[kKv8Block * kLdv];
  __shared__ unsigned bad[kKv8Block];
  __shared__ float most[kWaves];
  const int b = deal.packed ? kv8_owner(rt, deal, blockIdx.x) : blockIdx.z, h = blockIdx.y;
  if (b < 0) return;
  const Kv8Seq sq = kv8_seq(rt, b, dm.capacity);
  if (sq.n <= 0 || (CLOSED && sq.base != 0)) return;
  const int piece = deal.packed ? (int)blockIdx.x - kv8_first(rt, deal, b) : (int)blockIdx.x;
  if (piece < 0) return;
  const int blk = sq.base / kKv8Block + piece, tok0 = blk * kKv8Block, end = sq.base + sq.n;
  if (tok0 >= end) return;
  const int t = threadIdx.x, u = t % kHalf, lane = t & 63, r = lane & 15, g = lane >> 4;
  const bool values = t >= kHalf;   // (whole waves: kHalf is a multiple of 64)
  if (t < kKv8Block) bad[t] = 0;
  const size_t bh = (size_t)b * dm.heads + h;
  bf16_t* ring = CLOSED ? nullptr : (bf16_t*)(cache + dm.rings) + (bh * dm.ring + blk % max(dm.ring, 1)) * (2 * kKv8Block * DH) + (values ? kKv8Block * DH : 0);
  __syncthreads();

  // rows: thread u holds columns 32 s + 8 g .. + 7 of keys r and 16 + r (s = u / 64), as the keys' operand wants them
  const int s = u >> 6;
  uint4 x[2];
  bool spoilt = false;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int p = tok0 + 16 * i + r;
    x[i] = uint4{0, 0, 0, 0};
    if (p >= sq.base && p < end) {
      const bf16_t* src = values ? v + (size_t)(sq.row0 + p - sq.base) * v_stride : k + (size_t)(sq.row0 + p - sq.base) * k_stride;
      x[i] = ldg16(src + (size_t)h * DH + 32 * s + 8 * g);
    } else if (!CLOSED && !values && p < sq.base) {
      x[i] = ldg16(ring + ((2 * s + i) * 64 + lane) * 8);
    }
  }
  // the values kept from earlier calls are in operand order: thread u holds columns 16 c + r, c = 2 s and 2 s + 1, of eight keys each
  uint4 kept[2] = {uint4{0, 0, 0, 0}, uint4{0, 0, 0, 0}};
  const bool keeps = !CLOSED && tok0 < sq.base;
  if (keeps && values) {
#pragma unroll
    for (int i = 0; i < 2; ++i) kept[i] = ldg16(ring + ((2 * s + i) * 64 + lane) * 8);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (kv8_not_finite(x[i])) { bad[16 * i + r] = 1; spoilt = true; }   // (several threads may: all write the same)
    if (values) {
      unsigned* to = (unsigned*)(Vs + (16 * i + r) * kLdv + 32 * s + 8 * g);
      to[0] = x[i].x; to[1] = x[i].y; to[2] = x[i].z; to[3] = x[i].w;
    }
  }
  const bool any_spoilt = __syncthreads_or(spoilt);

  // the 16 elements in operand order, two a word
  unsigned e[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
  if (values) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const int key = kv8_key(g, j), col = 16 * (2 * s + i) + r;
        unsigned w = Vs[key * kLdv + col] | (unsigned)Vs[(key + 1) * kLdv + col] << 16;
        if (keeps) {   // (the same for the whole workgroup)
          const unsigned old = j == 0 ? kept[i].x : j == 2 ? kept[i].y : j == 4 ? kept[i].z : kept[i].w;
          const unsigned from = (tok0 + key < sq.base ? 0xffffu : 0u) | (tok0 + key + 1 < sq.base ? 0xffff0000u : 0u);
          w = (old & from) | (w & ~from);
        }
        if (any_spoilt) w &= (bad[key] ? 0u : 0xffffu) | (bad[key + 1] ? 0u : 0xffff0000u);
        e[4 * i + j / 2] = w;
      }
  } else if (any_spoilt) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (bad[16 * (j / 4) + r]) e[j] = 0x7fc07fc0u;
  }
  if (!CLOSED) {
#pragma unroll
    for (int i = 0; i < 2; ++i) gstore((uint4*)(ring + ((2 * s + i) * 64 + lane) * 8), uint4{e[4 * i], e[4 * i + 1], e[4 * i + 2], e[4 * i + 3]});
    if (tok0 + kKv8Block > end) return;   // (the whole workgroup: the block has tokens to come)
  }
  // The block is complete: its largest value, its bytes.  Magnitudes of bf16 order as whole numbers; a spoilt token's keys are left out of them.
  typedef unsigned short half2 __attribute__((ext_vector_type(2)));
  half2 hi = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (any_spoilt && (e[j] & 0x7fffu) > 0x7f80u) e[j] = 0;
    hi = __builtin_elementwise_max(hi, __builtin_bit_cast(half2, e[j] & 0x7fff7fffu));
  }
  const float mx = wave_max(__uint_as_float((unsigned)(hi.x > hi.y ? hi.x : hi.y) << 16));
  if (lane == 0) most[t >> 6] = mx;
  __syncthreads();
  float top = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves / 2; ++w) top = fmaxf(top, most[(values ? kWaves / 2 : 0) + w]);
  const Kv8Quant q = kv8_quant<FMT>(top);
  auto four = [&](int j) {
    const float f[4] = {__uint_as_float(e[j] << 16), __uint_as_float(e[j] & 0xffff0000u), __uint_as_float(e[j + 1] << 16), __uint_as_float(e[j + 1] & 0xffff0000u)};
    return kv8_pack4<FMT>(f, q);
  };
  gstore((uint4*)(cache + (bh * dm.blocks + blk) * (2 * kKv8Block * DH) + (values ? kKv8Block * DH : 0) + u * 16), uint4{four(0), four(2), four(4), four(6)});
  if (u == 0) gstore((float*)(cache + dm.scales) + (bh * dm.blocks + blk) * 2 + (values ? 1 : 0), any_spoilt && !values ? __uint_as_float(0x7fc00000u) : q.scale);
}

// One workgroup per (block, head, sequence), 4 * DH threads; keys' rows are written as they are held, values turned in LDS.  Bound by memory:
// 75 MB in 14.4 us, 5.2 TB/s; one token 3.3 us.
template <int DH, int FMT, typename T>
__global__ __launch_bounds__(4 * DH) void k_kv8_read(const unsigned char* __restrict__ cache, Kv8Rows rt, const int* __restrict__ length,
                                                     T* __restrict__ k_out, T* __restrict__ v_out, Kv8Deal deal, Kv8Dims dm) {
  constexpr int kHalf = 2 * DH, kLdv = DH + 1;
  __shared__ float Vs[kKv8Block * kLdv];
  const int b = deal.packed ? kv8_owner(rt, deal, blockIdx.x) : blockIdx.z, h = blockIdx.y;
  if (b < 0) return;
  Kv8Seq sq = kv8_seq(rt, b, dm.capacity);
  const int len = min(max(length[(size_t)b * rt.stride], 0), dm.capacity);
  sq.n = min(sq.n, len - sq.base);
  if (sq.n <= 0) return;
  const int piece = deal.packed ? (int)blockIdx.x - kv8_first(rt, deal, b) : (int)blockIdx.x;
  if (piece < 0) return;
  const int blk = sq.base / kKv8Block + piece, tok0 = blk * kKv8Block, end = sq.base + sq.n;
  if (tok0 >= end) return;
  const int t = threadIdx.x, u = t % kHalf, lane = t & 63, r = lane & 15, g = lane >> 4, s = u >> 6;
  const bool values = t >= kHalf;
  const size_t bh = (size_t)b * dm.heads + h;
  float f[16];
  if (dm.closed || blk < len / kKv8Block) {
    const uint4 w = ldg16(cache + (bh * dm.blocks + blk) * (2 * kKv8Block * DH) + (values ? kKv8Block * DH : 0) + u * 16);
    const float scale = gload((const float*)(cache + dm.scales) + (bh * dm.blocks + blk) * 2 + (values ? 1 : 0));
    kv8_unpack<FMT>(w.x, scale, f); kv8_unpack<FMT>(w.y, scale, f + 4); kv8_unpack<FMT>(w.z, scale, f + 8); kv8_unpack<FMT>(w.w, scale, f + 12);
  } else {
    const bf16_t* ring = (const bf16_t*)(cache + dm.rings) + (bh * dm.ring + blk % max(dm.ring, 1)) * (2 * kKv8Block * DH) + (values ? kKv8Block * DH : 0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 w = ldg16(ring + ((2 * s + i) * 64 + lane) * 8);
      const unsigned e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) f[8 * i + j] = __uint_as_float(j & 1 ? e[j / 2] & 0xffff0000u : e[j / 2] << 16);
    }
  }
  if (values) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) Vs[kv8_key(g, j) * kLdv + 16 * (2 * s + i) + r] = f[8 * i + j];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int p = tok0 + 16 * i + r;
    if (p < sq.base || p >= end) continue;
    if (values) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[8 * i + j] = Vs[(16 * i + r) * kLdv + 32 * s + 8 * g + j];
    }
    T* to = (values ? v_out : k_out) + ((size_t)(sq.row0 + p - sq.base) * dm.heads + h) * DH + 32 * s + 8 * g;
    if constexpr (sizeof(T) == 4) {
      gstore((float4*)to, float4{f[8 * i], f[8 * i + 1], f[8 * i + 2], f[8 * i + 3]});
      gstore((float4*)to + 1, float4{f[8 * i + 4], f[8 * i + 5], f[8 * i + 6], f[8 * i + 7]});
    } else {
      gstore((uint4*)to, uint4{f2bf_pair(f[8 * i], f[8 * i + 1]), f2bf_pair(f[8 * i + 2], f[8 * i + 3]),
                               f2bf_pair(f[8 * i + 4], f[8 * i + 5]), f2bf_pair(f[8 * i + 6], f[8 * i + 7])});
    }
  }
}

template <int DH, int FMT>
static void append_for(const Kv8Dims& d, unsigned char* cache, const bf16_t* k, const bf16_t* v, size_t ks, size_t vs, const Kv8Rows& r, const Kv8Deal& deal, dim3 grid, hipStream_t s) {
  if (d.closed) k_kv8_append<DH, FMT, true><<<grid, 4 * DH, 0, s>>>(cache, k, v, ks, vs, r, deal, d);
  else k_kv8_append<DH, FMT, false><<<grid, 4 * DH, 0, s>>>(cache, k, v, ks, vs, r, deal, d);
}
// blocks that rows touch: wherever they begin, one or two more than fill them
static Kv8Deal kv8_blocks(const Kv8Rows& r) { return kv8_deal(r, 1, 5, 2, ((size_t)r.max_rows + kKv8Block - 2) / kKv8Block + 1); }
void launch_kv8_append(const Kv8Dims& d, void* cache, const void* k, const void* v, size_t k_stride, size_t v_stride, const Kv8Rows& r, hipStream_t s) {
  const Kv8Deal deal = kv8_blocks(r);
  const dim3 grid((unsigned)deal.pieces, d.heads, deal.packed ? 1 : r.n_seq);
  kv8_dispatch(d, [&](auto width, auto fmt) {
    append_for<width.value, fmt.value>(d, (unsigned char*)cache, (const bf16_t*)k, (const bf16_t*)v, k_stride, v_stride, r, deal, grid, s);
  });
}

void launch_kv8_read(const Kv8Dims& d, const void* cache, const Kv8Rows& r, const int* length, int dtype, void* k_out, void* v_out, hipStream_t s) {
  const Kv8Deal deal = kv8_blocks(r);
  const dim3 grid((unsigned)deal.pieces, d.heads, deal.packed ? 1 : r.n_seq);
  kv8_dispatch(d, [&](auto width, auto fmt) {
    if (dtype == AD_BF16)
      k_kv8_read<width.value, fmt.value, bf16_t><<<grid, 4 * width.value, 0, s>>>((const unsigned char*)cache, r, length, (bf16_t*)k_out, (bf16_t*)v_out, deal, d);
    else
      k_kv8_read<width.value, fmt.value, float><<<grid, 4 * width.value, 0, s>>>((const unsigned char*)cache, r, length, (float*)k_out, (float*)v_out, deal, d);
  });
}

}  // namespace ad
