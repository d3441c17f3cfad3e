// Causal grouped-query attention of many sequences' new rows over a pool of cache pages.
#include "hi_paged_attn.h"

namespace hi {

namespace {

// One wavefront for each new row of each query head, a lane for two dims: one pass over the row's keys with a running maximum and sum.
template <int BITS>
__global__ __launch_bounds__(64) void paged_attn_row_kernel(PagedAttnArgs a) {
  const int t = blockIdx.x, head = blockIdx.y, lane = threadIdx.x, kv = head / a.group;
  int before = 0;
  for (int s = lane; s - lane < a.seqs.n_seqs; s += 64)
    before += __popcll(__builtin_amdgcn_ballot_w64(s < a.seqs.n_seqs && a.seqs.starts[s] <= t));
  if (before == 0) return;
  const PagedSeq sq = paged_seq_of(a.seqs, before - 1);
  if (t < sq.first || t >= sq.first + sq.rows) return;
  const int64_t at = ((int64_t)head * a.seqs.n_rows + t) * kHeadDim + 2 * lane;
  const uint32_t qw = *(const uint32_t*)(a.q + at);
  const float q0 = __uint_as_float(qw << 16), q1 = __uint_as_float(qw & 0xFFFF0000u);
  const int64_t sees = (int64_t)sq.past + (t - sq.first) + 1, most = (int64_t)a.seqs.table_pages << a.pool.shift;
  const int n = (int)(sees < most ? sees : most), R = 1 << a.pool.shift;
  float m = kNegBig, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int p = 0; p * R < n; ++p) {
    const int page = a.seqs.table[(int64_t)(before - 1) * a.seqs.table_pages + p];
    if (page < 0 || page >= a.pool.n_pages) continue;
    const int64_t row = paged_row(a.pool, page, kv, 0);
    for (int r = 0; r < R && p * R + r < n; ++r) {
      float k0, k1, v0, v1, ks = 1.f, vs = 1.f;
      if (BITS == 16) {
        const uint32_t kw = *(const uint32_t*)(a.pool.pages + (row + r) * kRowBytes + 4 * lane);
        const uint32_t vw = *(const uint32_t*)(a.pool.pages + (row + R + r) * kRowBytes + 4 * lane);
        k0 = __uint_as_float(kw << 16); k1 = __uint_as_float(kw & 0xFFFF0000u);
        v0 = __uint_as_float(vw << 16); v1 = __uint_as_float(vw & 0xFFFF0000u);
      } else {
        const int kw = *(const uint16_t*)(a.pool.pages + (row + r) * kHeadDim + 2 * lane);
        const int vw = *(const uint16_t*)(a.pool.pages + (row + R + r) * kHeadDim + 2 * lane);
        k0 = __builtin_amdgcn_cvt_f32_fp8(kw, 0); k1 = __builtin_amdgcn_cvt_f32_fp8(kw, 1);
        v0 = __builtin_amdgcn_cvt_f32_fp8(vw, 0); v1 = __builtin_amdgcn_cvt_f32_fp8(vw, 1);
        ks = a.pool.scales[row + r];
        vs = a.pool.scales[row + R + r];
      }
      const float s = over_wave(q0 * k0 + q1 * k1, op_add) * ks;
      const float mn = fmaxf(m, s), alpha = fast_exp2((m - mn) * a.c), w = fast_exp2((s - mn) * a.c);
      l = l * alpha + w;
      o0 = o0 * alpha + w * vs * v0;
      o1 = o1 * alpha + w * vs * v1;
      m = mn;
    }
  }
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  *(uint32_t*)(a.out + at) = pack_bf16(o0 * inv, o1 * inv);
}

constexpr int kArrivalBytes = kPagedRuns * 4;

}  // namespace

}  // namespace hi

using namespace hi;

extern "C" hi_status hi_paged_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int64_t* bytes) {
  if (!bytes || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads != 0) { set_last_error("paged workspace: bad argument"); return HI_ERR_ARG; }
  if (n_q_heads / n_kv_heads > 16) { set_last_error("paged attention: at most 16 query heads a KV head"); return HI_ERR_UNSUPPORTED; }
  *bytes = kArrivalBytes + (int64_t)2 * kPagedRuns * kPagedPieceFloats * 4;
  return HI_OK;
}

extern "C" hi_status hi_paged_attn(void* stream, const hi_paged_cache* cache, const hi_paged_batch* batch, const void* q_dev,
                                   int32_t n_q_heads, int32_t q_prescaled, void* out_dev, void* workspace_dev) {
  PagedAttnArgs a = {};
  const hi_status st = paged_arguments(cache, batch, "paged attention", a.pool, a.seqs);
  if (st != HI_OK) return st;
  if (!q_dev || !out_dev || !workspace_dev) { set_last_error("paged attention: null buffer"); return HI_ERR_ARG; }
  if (!aligned_to(q_dev, 16) || !aligned_to(out_dev, 16) || !aligned_to(workspace_dev, 16)) {
    set_last_error("paged attention: buffers must be 16-byte aligned");
    return HI_ERR_ARG;
  }
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads != 0 || (q_prescaled != 0 && q_prescaled != 1)) { set_last_error("paged attention: bad shape"); return HI_ERR_ARG; }
  const int group = n_q_heads / cache->n_kv_heads;
  if (group > 16) { set_last_error("paged attention: at most 16 query heads a KV head"); return HI_ERR_UNSUPPORTED; }
  if (n_q_heads > 65535) { set_last_error("paged attention: too many heads"); return HI_ERR_RANGE; }
  if (batch->n_seqs == 0 || batch->n_rows == 0) return HI_OK;
  a.q = (const uint16_t*)q_dev; a.out = (uint16_t*)out_dev;
  a.q_heads = n_q_heads; a.group = group;
  a.c = softmax_scale_log2(q_prescaled != 0);
  a.positions = 16 / group;
  a.by_group = (65536 + group - 1) / group;
  a.arrivals = (int*)workspace_dev;
  a.pieces = (float*)((char*)workspace_dev + kArrivalBytes);
  // tiles of 16 rows, at the table's full length, have to be countable in 31 bits
  const int64_t blocks = (int64_t)batch->n_seqs + batch->n_rows / a.positions, tiles = ceil_div((int64_t)batch->table_pages << a.pool.shift, 16);
  if ((double)blocks * (double)tiles * (double)cache->n_kv_heads > 2147483647.0) { set_last_error("paged attention: more tiles than can be counted"); return HI_ERR_RANGE; }
  StreamDevice on(stream);
  if (batch->max_rows * (int64_t)group <= 16) return launch_paged_decode(stream, a);
  const dim3 grid((unsigned)batch->n_rows, (unsigned)n_q_heads);
  if (a.pool.bits == 16) hipLaunchKernelGGL(paged_attn_row_kernel<16>, grid, dim3(64), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(paged_attn_row_kernel<8>, grid, dim3(64), 0, (hipStream_t)stream, a);
  return launched("paged attention");
}
