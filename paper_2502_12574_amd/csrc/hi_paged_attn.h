// What the kernels of paged attention take.
#pragma once
#include "hi_paged.h"

namespace hi {

// hi_paged_decode.hip: runs of 32-row tiles, one a workgroup (one workgroup for each of the 256 compute units, whose LDS it fills), no
// shorter than a tile for each of its wavefronts; pieces of blocks that lie in several runs, at most two a run; three arrays of counts
constexpr int kPagedRuns = 256;
constexpr int kPagedLeastRun = 4;
template <int BITS> constexpr int kPagedStart = BITS == 8 ? 12 : 6;
constexpr int kPagedArrivals = 3 * kPagedRuns;
constexpr int kPagedPieceFloats = 16 * kPartialFloats;

// hi_paged_chunk.hip: two workgroups of 128 rows a compute unit; a block that is cut leaves an image of its state (64 O^T accumulators, m
// and l for each of 256 lanes) for each piece.  Pieces have at least the tiles of all blocks / (2 x 512), so there are at most twice
// as many images as that (and a few, as that share is worked out in fp32).
constexpr int kPagedSlots = 512;
constexpr int kPagedMostImages = 4 * kPagedSlots + 16;
constexpr int kPagedImageFloats = 66 * 256;
constexpr int kPagedFan = 3, kPagedLevels = 4;   // log2 of the images of a merge; their levels
static_assert(1 << (kPagedFan * kPagedLevels) >= kPagedMostImages, "a block's images");
constexpr int kPagedCounts = kPagedLevels * kPagedMostImages;

// Tiles (and starts) of all blocks, in 31 bits with something to spare for the kernels' fp32 estimates of it.
constexpr float kPagedMostTiles = 2.0e9f;

// Numbers that another workgroup reads: two at a time, by accesses that no L2 keeps a copy of.
__device__ __forceinline__ void store_shared2(float* p, float x, float y) {
  __hip_atomic_store((uint64_t*)p, (uint64_t)__float_as_uint(x) | ((uint64_t)__float_as_uint(y) << 32), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_shared2(const float* p) {
  const uint64_t v = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Values that are not finite.  A weight of zero takes a key out of a row only as long as its value is finite, and in a tile whose keys
// some rows see and others don't no value can be taken out for all of them.  Where such a tile holds a value that is not finite, its
// second product is done with zeros in their place, and a product of ones (of such values) and ones (of keys that are seen) says which
// elements of which rows they belong to: those become NaN.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {                 // bits 15 and 31: of the two bf16 numbers
  return (w & 0x7F807F80u) + 0x00800080u;
}
__device__ __forceinline__ uint32_t spread_halves(uint32_t bits) {           // bits 15 and 31 to all of their halves
  return ((bits >> 15) & 0x00010001u) * 0xFFFFu;
}
struct TwoParts { bf16x8 finite, others; };                                  // the second: ones
__device__ __forceinline__ TwoParts two_parts(bf16x8 v) {
  u32x4 x = __builtin_bit_cast(u32x4, v), y;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t bad = spread_halves(not_finite(x[e]));
    y[e] = bad & 0x3F803F80u;
    x[e] &= ~bad;
  }
  return {__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y)};
}

struct PagedAttnArgs {
  PagedPool pool; PagedSeqs seqs;
  const uint16_t* q; uint16_t* out;
  int group;
  int positions, by_group;       // positions of a block; 65536 / group, rounded up
  float c;                       // what a score is multiplied by before the power of two
  int* arrivals; int* counts; float* pieces; float* images;   // in the workspace
};

hi_status launch_paged_decode(void* stream, const PagedAttnArgs& a);
hi_status launch_paged_chunk(void* stream, const PagedAttnArgs& a, int64_t units);

}  // namespace hi
