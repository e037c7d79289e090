// Sequences of 8-bit caches copied: to other places of the same cache or of another (ad_kv8.h has the layouts).
//
// A block's bytes and scales do not depend on where it lies, and copies begin at a block, so they are moved as they are; of a growing cache the incomplete block behind them is
// moved within the bf16 ring, from the slot that it has in one cache to the one that it has in the other.  All entries of a call are read before any is written: a
// workgroup takes the same bytes of the same block and head of all entries at once, holds them in registers, waits, and writes them; what one workgroup reads no other
// writes.  A growing cache holds a block in bf16 only while it is incomplete there: where the copy has no room for all of the source's tokens and would end inside a block that the source holds in 8 bits
// alone, it ends with the block before.  Bound by memory, a byte read and a byte written for a value: 139 MB of 16 sequences, 16 heads, to another cache in 50 to 60 us, 67 MB of 16 sequences of width 128 within one in 28, 4.7 to 5 TB/s;
// three copies of 301 tokens 5.0 us, a launch and two waits for memory.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ad_device.h"
#include "ad_kv8_device.h"

namespace ad {

constexpr int kChunks = 8;   // of 16 bytes, a thread (4 and 16: the same or slower)

// 16 bytes that are not read again soon: caches keep what is written instead (16 sequences of 500 to 8000 tokens copied and read back 161 -> 148 us)
__device__ __forceinline__ uint4 kv8_once(const unsigned char* p) {
  typedef unsigned four __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const AD_GLOBAL four*)p));
}

// (first: the source's first block, first * 32 <= from_capacity.  What the source is to have is held to its cache before the first token is taken off: no table overflows a difference.)
__host__ __device__ int kv8_copied(int first, int end, int from_capacity, int to_capacity, int max_tokens, bool closed) {
  const int have = std::min(std::max(end, 0), from_capacity) - first * kKv8Block, count = std::max(std::min(std::min(have, to_capacity), max_tokens), 0);
  return !closed && count / kKv8Block < have / kKv8Block ? count / kKv8Block * kKv8Block : count;
}

struct Kv8Move { int seqs, count; };   // source | place << 16; tokens (0: nothing)

// blockIdx.x: part of a block, then block, y: head.  2^piece bytes of a block of all entries; behind the blocks of 8 bits the two halves of the ring's.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv8_copy(const unsigned char* origin, unsigned char* cache, Kv8Moves m, Kv8Dims df, Kv8Dims dt, int blocks, int piece, int parts) {
  extern __shared__ int lds[];
  Kv8Move* moves = (Kv8Move*)lds;
  int* taken = lds + 2 * m.n;   // [n_seq] the entry that a place gets
  const int t = threadIdx.x, part = blockIdx.x % parts, blk = blockIdx.x / parts, h = blockIdx.y;
  for (int i = t; i < dt.n_seq; i += THREADS) taken[i] = m.n;
  __syncthreads();
  auto first = [&](int i) { return m.begin ? min(max(m.begin[i], 0), df.capacity) / kKv8Block : 0; };   // the source's first block
  for (int i = t; i < m.n; i += THREADS) {
    const int from = m.source[i], to = m.place[i];
    Kv8Move v{0, 0};
    if (from >= 0 && from < df.n_seq && to >= 0 && to < dt.n_seq) {
      v.seqs = from | to << 16;
      v.count = kv8_copied(first(i), m.end[i], df.capacity, dt.capacity, m.max_tokens, dt.closed);
      atomicMin(&taken[to], i);   // (one of no tokens, too)
    }
    moves[i] = v;
  }
  __syncthreads();
  const int block_bytes = 2 * kKv8Block * dt.width, ring_half = blk - blocks;   // ring_half >= 0: of the ring
  auto whole = [&](int count) { return dt.closed ? (count + kKv8Block - 1) / kKv8Block : count / kKv8Block; };
  // where chunk j of this thread's lies: in the block of its entry, if that has one here
  auto find = [&](int j, const unsigned char*& src, unsigned char*& dst) {
    const int at = t + j * THREADS, i = at >> (piece - 4);
    if (i >= m.n) return false;
    const Kv8Move v = moves[i];
    const int from = v.seqs & 0xffff, to = v.seqs >> 16, b = v.count / kKv8Block;
    if (v.count == 0 || taken[to] != i || (ring_half >= 0 ? v.count % kKv8Block == 0 : blk >= whole(v.count))) return false;
    const size_t in = ((size_t)part << piece) + (at & ((1 << (piece - 4)) - 1)) * 16, hf = (size_t)from * df.heads + h, ht = (size_t)to * dt.heads + h;
    if (ring_half >= 0) {
      src = origin + df.rings + ((hf * df.ring + (first(i) + b) % df.ring) * 2 + ring_half) * block_bytes + in;
      dst = cache + dt.rings + ((ht * dt.ring + b % dt.ring) * 2 + ring_half) * block_bytes + in;
    } else {
      src = origin + (hf * df.blocks + first(i) + blk) * block_bytes + in;
      dst = cache + (ht * dt.blocks + blk) * block_bytes + in;
    }
    return true;
  };
  uint4 x[kChunks];
  const unsigned char* src;
  unsigned char* dst;
#pragma unroll
  for (int j = 0; j < kChunks; ++j)
    if (find(j, src, dst)) x[j] = kv8_once(src);
  // the scales, by the workgroup of a block's first part: a thread those of up to four entries
  const bool scales = part == 0 && ring_half < 0;
  float2 y[4];
  auto find_scale = [&](int j, const float2*& from, float2*& to) {
    const int i = t + j * THREADS;
    if (!scales || i >= m.n) return false;
    const Kv8Move v = moves[i];
    if (v.count == 0 || taken[v.seqs >> 16] != i || blk >= whole(v.count)) return false;
    from = (const float2*)(origin + df.scales) + ((size_t)(v.seqs & 0xffff) * df.heads + h) * df.blocks + first(i) + blk;
    to = (float2*)(cache + dt.scales) + ((size_t)(v.seqs >> 16) * dt.heads + h) * dt.blocks + blk;
    return true;
  };
  const float2* sf;
  float2* st;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (find_scale(j, sf, st)) y[j] = gload(sf);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // everything read has arrived before any wave writes
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kChunks; ++j)
    if (find(j, src, dst)) gstore((uint4*)dst, x[j]);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (find_scale(j, sf, st)) gstore(st, y[j]);
}

// How a copy is launched: blocks of 8 bits that an entry has at most, and the pieces that they are cut into.
struct Kv8CopyShape {
  int threads, blocks, piece, parts;   // 2^piece bytes of a block, `parts` of them
  size_t along;                        // workgroups along x
};
static Kv8CopyShape copy_shape(const Kv8Dims& from, const Kv8Dims& to, int n, int max_tokens) {
  Kv8CopyShape c;
  const int tokens = std::min({max_tokens, from.capacity, to.capacity});
  c.blocks = to.closed ? (tokens + kKv8Block - 1) / kKv8Block : tokens / kKv8Block;
  c.threads = n <= 256 ? 256 : 1024;
  c.piece = to.width == 32 ? 11 : to.width == 64 ? 12 : 13;   // (a block's bytes are 64 a column)
  c.parts = 1;
  while (((size_t)n << c.piece) > (size_t)c.threads * kChunks * 16) { --c.piece; c.parts *= 2; }   // (32 bytes at least: 4096 entries)
  c.along = (size_t)(c.blocks + (to.closed ? 0 : 2)) * c.parts;
  return c;
}
// (a launch takes less than 2^32 lanes along x)
bool kv8_copy_fits(const Kv8Dims& from, const Kv8Dims& to, int n, int max_tokens) {
  const Kv8CopyShape c = copy_shape(from, to, n, max_tokens);
  return c.along * c.threads < ((size_t)1 << 32);
}
void launch_kv8_copy(const Kv8Dims& from, const void* origin, const Kv8Dims& to, void* cache, const Kv8Moves& m, hipStream_t s) {
  const Kv8CopyShape c = copy_shape(from, to, m.n, m.max_tokens);
  const dim3 grid((unsigned)c.along, to.heads);
  const size_t lds = (size_t)m.n * 8 + (size_t)to.n_seq * 4;
  if (c.threads == 256) k_kv8_copy<256><<<grid, 256, lds, s>>>((const unsigned char*)origin, (unsigned char*)cache, m, from, to, c.blocks, c.piece, c.parts);
  else k_kv8_copy<1024><<<grid, 1024, lds, s>>>((const unsigned char*)origin, (unsigned char*)cache, m, from, to, c.blocks, c.piece, c.parts);
}

}  // namespace ad
