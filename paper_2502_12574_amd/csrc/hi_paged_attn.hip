// Causal grouped-query attention of many sequences' new rows over a pool of cache pages.
#include "hi_paged_attn.h"

namespace hi {

namespace {

// The workspace: the arrival counts of both kernels, then either the pieces of the one or the images of the other.
constexpr int kArrivalBytes = (kPagedArrivals + kPagedCounts) * 4;
static_assert(kArrivalBytes % 256 == 0, "aligned images");

}  // namespace

}  // namespace hi

using namespace hi;

extern "C" hi_status hi_paged_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int64_t* bytes) {
  if (!bytes || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads != 0) { set_last_error("paged workspace: bad argument"); return HI_ERR_ARG; }
  if (n_q_heads / n_kv_heads > 16) { set_last_error("paged attention: at most 16 query heads a KV head"); return HI_ERR_UNSUPPORTED; }
  const int64_t pieces = (int64_t)2 * kPagedRuns * kPagedPieceFloats * 4, images = (int64_t)kPagedMostImages * kPagedImageFloats * 4;
  *bytes = kArrivalBytes + (pieces > images ? pieces : images);
  return HI_OK;
}

extern "C" hi_status hi_paged_attn(void* stream, const hi_paged_cache* cache, const hi_paged_batch* batch, const void* q_dev,
                                   int32_t n_q_heads, int32_t q_prescaled, void* out_dev, void* workspace_dev) {
  PagedAttnArgs a = {};
  const hi_status st = paged_arguments(cache, batch, "paged attention", a.pool, a.seqs);
  if (st != HI_OK) return st;
  if (!aligned_to(q_dev, 16) || !aligned_to(out_dev, 16) || !aligned_to(workspace_dev, 16)) {
    set_last_error("paged attention: buffers must be 16-byte aligned");
    return HI_ERR_ARG;
  }
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads != 0 || (q_prescaled != 0 && q_prescaled != 1)) { set_last_error("paged attention: bad shape"); return HI_ERR_ARG; }
  const int group = n_q_heads / cache->n_kv_heads;
  if (group > 16) { set_last_error("paged attention: at most 16 query heads a KV head"); return HI_ERR_UNSUPPORTED; }
  // (the scales of all heads of a page lie within 32 bits of bytes)
  if (n_q_heads > 65535) { set_last_error("paged attention: too many heads"); return HI_ERR_RANGE; }
  if (batch->n_seqs == 0 || batch->n_rows == 0) return HI_OK;      // (whose buffers may be null)
  if (!q_dev || !out_dev || !workspace_dev) { set_last_error("paged attention: null buffer"); return HI_ERR_ARG; }
  if (q_dev == out_dev) { set_last_error("paged attention: the output cannot be the queries"); return HI_ERR_ARG; }
  a.q = (const uint16_t*)q_dev; a.out = (uint16_t*)out_dev;
  a.group = group;
  a.c = softmax_scale_log2(q_prescaled != 0);
  a.arrivals = (int*)workspace_dev;
  a.counts = a.arrivals + kPagedArrivals;
  a.pieces = a.images = (float*)((char*)workspace_dev + kArrivalBytes);
  a.by_group = (65536 + group - 1) / group;
  const bool few = (int64_t)batch->max_rows * group <= 16;
  a.positions = (few ? 16 : 128) / group;
  // Blocks of all sequences: each but the last of a sequence is full, and each has a row.  Their tiles, at the table's full length, have
  // to be countable, and there can be no more workgroups than 2^32 lanes.
  const int64_t table_rows = (int64_t)batch->table_pages << a.pool.shift, most = batch->n_rows / a.positions + (int64_t)batch->n_seqs;
  const int64_t units = (most < batch->n_rows ? most : batch->n_rows) * cache->n_kv_heads;
  const int64_t deepest = few ? ceil_div(table_rows, 32) + (a.pool.bits == 8 ? kPagedStart<8> : kPagedStart<16>) : ceil_div(table_rows, 64);
  if ((double)units * (double)deepest > (double)kPagedMostTiles || (!few && units > (1 << 24) - 1 - 2 * kPagedSlots)) {
    set_last_error("paged attention: more tiles than can be counted");
    return HI_ERR_RANGE;
  }
  StreamDevice on(stream);
  return few ? launch_paged_decode(stream, a) : launch_paged_chunk(stream, a, units);
}
