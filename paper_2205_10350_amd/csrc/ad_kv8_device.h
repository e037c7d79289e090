// What the kernels over 8-bit caches share.
#pragma once

#include "ad_device.h"
#include "ad_kv8.h"

namespace ad {

// a sequence's rows in this call: [row0, row0 + n) packed, at positions base ..
struct Kv8Seq { int row0, n, base; };
// (`placed`: the rows have places in the cache, behind `base` tokens; else they are queries over a closed one of `base` tokens)
__device__ __forceinline__ Kv8Seq kv8_seq(const Kv8Rows& t, int b, int capacity, bool placed = true) {
  const size_t at = (size_t)b * t.stride;
  Kv8Seq s;
  s.row0 = t.start[at];
  s.n = t.count ? t.count[at] : kv8_range(s.row0, t.start[at + t.stride]);
  s.base = t.base ? t.base[at] : 0;
  if (s.base < 0) s.n = 0;
  s.base = min(max(s.base, 0), capacity);
  s.n = kv8_held(s.row0, s.n, t.rows, t.max_rows);
  if (placed) s.n = min(s.n, capacity - s.base);
  return s;
}

// where the packed pieces of sequence b begin, and the sequence that has packed piece `at` (-1: none), found by each wave for itself: every 64th sequence at once, then
// those between two of them
__device__ __forceinline__ int kv8_first(const Kv8Rows& t, const Kv8Deal& d, int b) {
  return (int)((long long)min(max(t.start[(size_t)b * t.stride], 0), t.rows) * d.mul >> d.shift) + d.extra * b;
}
__device__ __forceinline__ int kv8_owner(const Kv8Rows& t, const Kv8Deal& d, int at) {
  const int lane = threadIdx.x & 63, apart = (t.n_seq + 63) / 64;
  int b = __popcll(__ballot(lane * apart < t.n_seq && kv8_first(t, d, min(lane * apart, t.n_seq - 1)) <= at)) - 1;
  if (b < 0) return -1;
  b *= apart;
  if (apart > 1) b += __popcll(__ballot(lane < apart && b + lane < t.n_seq && kv8_first(t, d, min(b + lane, t.n_seq - 1)) <= at)) - 1;
  return b;
}

// the key that element j of lane group g holds in the values' operand
__device__ __forceinline__ constexpr int kv8_key(int g, int j) { return j < 4 ? 4 * g + j : 16 + 4 * g + j - 4; }

__device__ __forceinline__ bool kv8_not_finite(const uint4& x) {   // any of eight bf16
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned w = i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
    bad = bad || (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
  }
  return bad;
}

typedef __attribute__((ext_vector_type(2))) __bf16 kv8_bf16x2;

// four bytes -> fp32 values
template <int FMT> __device__ __forceinline__ void kv8_unpack(unsigned w, float scale, float* f) {
  if constexpr (FMT == AD_KV_E4M3) {
    // (bytes to bf16 exactly, by the instruction that the attention uses)
    const unsigned lo = __builtin_bit_cast(unsigned, (kv8_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
    const unsigned hi = __builtin_bit_cast(unsigned, (kv8_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
    f[0] = __uint_as_float(lo << 16) * scale; f[1] = __uint_as_float(lo & 0xffff0000u) * scale;
    f[2] = __uint_as_float(hi << 16) * scale; f[3] = __uint_as_float(hi & 0xffff0000u) * scale;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(signed char)(w >> (8 * i)) * scale;
  }
}
// eight bytes -> an operand of eight bf16, exactly (|i8| < 2^8; e4m3 has four significant bits); e4m3: times `scale`, a power of two
template <int FMT> __device__ __forceinline__ bf16x8 kv8_operand(uint2 w, float scale) {
  uint4 o;
  if constexpr (FMT == AD_KV_E4M3) {
    o.x = __builtin_bit_cast(unsigned, (kv8_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, scale, false));
    o.y = __builtin_bit_cast(unsigned, (kv8_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, scale, true));
    o.z = __builtin_bit_cast(unsigned, (kv8_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, scale, false));
    o.w = __builtin_bit_cast(unsigned, (kv8_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, scale, true));
  } else {
    auto two = [](unsigned x, int at) {   // the upper halves of two floats that have nothing in their lower ones
      const unsigned a = __float_as_uint((float)(signed char)(x >> (8 * at))), b = __float_as_uint((float)(signed char)(x >> (8 * at + 8)));
      return __builtin_amdgcn_perm(b, a, 0x07060302u);
    };
    o.x = two(w.x, 0); o.y = two(w.x, 2); o.z = two(w.y, 0); o.w = two(w.y, 2);
  }
  return __builtin_bit_cast(bf16x8, o);
}

// f(head width, format) as compile-time constants
template <typename F> inline void kv8_dispatch(const Kv8Dims& d, const F& f) {
  auto by_fmt = [&](auto width) {
    if (d.format == AD_KV_E4M3) f(width, std::integral_constant<int, AD_KV_E4M3>{});
    else f(width, std::integral_constant<int, AD_KV_I8>{});
  };
  if (d.width == 32) by_fmt(std::integral_constant<int, 32>{});
  else if (d.width == 64) by_fmt(std::integral_constant<int, 64>{});
  else by_fmt(std::integral_constant<int, 128>{});
}

}  // namespace ad
