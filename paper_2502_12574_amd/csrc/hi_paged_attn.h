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

// Tiles (and starts) of all blocks, in 31 bits with something to spare for the kernels' fp32 estimates of it.
constexpr float kPagedMostTiles = 2.0e9f;

struct PagedAttnArgs {
  PagedPool pool; PagedSeqs seqs;
  const uint16_t* q; uint16_t* out;
  int group;
  int positions, by_group;       // positions of a block; 65536 / group, rounded up
  float c;                       // what a score is multiplied by before the power of two
  int* arrivals; int* plan; float* pieces; float* images;   // in the workspace
};

hi_status launch_paged_decode(void* stream, const PagedAttnArgs& a);
hi_status launch_paged_chunk(void* stream, const PagedAttnArgs& a, int64_t units);

}  // namespace hi
