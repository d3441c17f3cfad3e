// New rows of many sequences into a pool of cache pages: rotary embedding by each row's own position, the queries' scale, and K and V
// into the pages, in bf16 or as e4m3 with a scale a row (scale = max |x| / 448, code = e4m3(x / scale)).
// Pure traffic: each input is read once, each output written once (two prompts, 7922 fp32 rows of 32 + 16 heads into bf16 pages: 48 us, 6 TB/s).
// With few rows the launch and a chain of four latencies (starts, past length, page number, rows) are all of it (48 rows: 4.5 us).
#include "hi_paged.h"

namespace hi {

hi_status paged_arguments(const hi_paged_cache* cache, const hi_paged_batch* batch, const char* what, PagedPool& pool, PagedSeqs& seqs) {
  if (!cache || !batch) { set_last_error("%s: null cache or batch", what); return HI_ERR_ARG; }
  if (cache->kv_bits != 16 && cache->kv_bits != 8) { set_last_error("%s: kv_bits must be 16 or 8", what); return HI_ERR_UNSUPPORTED; }
  if (!cache->pages || (cache->kv_bits == 8 && !cache->scales)) { set_last_error("%s: null cache buffer", what); return HI_ERR_ARG; }
  if (!aligned_to(cache->pages, 16) || !aligned_to(cache->scales, 16)) { set_last_error("%s: cache buffers must be 16-byte aligned", what); return HI_ERR_ARG; }
  if (cache->n_pages < 1 || cache->n_kv_heads < 1) { set_last_error("%s: bad cache shape", what); return HI_ERR_ARG; }
  const int r = cache->page_rows;
  if (r < 16 || r > 1024 || (r & (r - 1)) != 0) { set_last_error("%s: page_rows must be a power of two from 16 to 1024", what); return HI_ERR_UNSUPPORTED; }
  if (batch->n_seqs < 0 || batch->n_rows < 0 || batch->table_pages < 1 || batch->max_rows < 1) { set_last_error("%s: bad batch shape", what); return HI_ERR_ARG; }
  if (batch->n_seqs > 0 && (!batch->page_table || !batch->past_lens || !batch->row_starts)) { set_last_error("%s: null batch array", what); return HI_ERR_ARG; }
  if (!aligned_to(batch->page_table, 4) || !aligned_to(batch->past_lens, 4) || !aligned_to(batch->row_starts, 4)) { set_last_error("%s: batch arrays must be 4-byte aligned", what); return HI_ERR_ARG; }
  int shift = 4;
  while ((1 << shift) < r) ++shift;
  // (rows, and the ends of tiles behind the last one, are counted in 32 bits)
  if (((int64_t)batch->table_pages << shift) > (1 << 30)) { set_last_error("%s: a table of more than 2^30 rows", what); return HI_ERR_RANGE; }
  pool = {(char*)cache->pages, (float*)cache->scales, cache->n_pages, cache->n_kv_heads, shift, cache->kv_bits};
  seqs = {batch->page_table, batch->past_lens, batch->row_starts, batch->n_seqs, batch->table_pages, batch->n_rows};
  return HI_OK;
}

namespace {

struct PagedFreqs { double inv[64]; };

struct AppendArgs {
  PagedPool pool; PagedSeqs seqs;
  const void* q; const void* k; const void* v; uint16_t* q_out;
  int q_heads, rotate;
  float q_scale;
  PagedFreqs f;
};

// 8 consecutive values of a row
template <bool FP32> struct RowPiece;
template <> struct RowPiece<false> {
  u32x4 w;
  __device__ __forceinline__ void load(const void* at, int64_t i) { w = *(const u32x4*)((const uint16_t*)at + i); }
  __device__ __forceinline__ float get(int j) const { return __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16); }
};
template <> struct RowPiece<true> {
  f32x4 w[2];
  __device__ __forceinline__ void load(const void* at, int64_t i) {
    w[0] = *(const f32x4*)((const float*)at + i);
    w[1] = *(const f32x4*)((const float*)at + i + 4);
  }
  __device__ __forceinline__ float get(int j) const { return w[j >> 2][j & 3]; }
};

// the largest of 8 neighbouring lanes, in each of them
__device__ __forceinline__ float max_of_8(float x) {
  auto step = [](float y, auto ctrl) __attribute__((always_inline)) {
    const int u = __builtin_bit_cast(int, y);
    return fmaxf(y, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(u, u, decltype(ctrl)::value, 0xf, 0xf, false)));
  };
  x = step(x, std::integral_constant<int, 0xB1>());        // lane ^ 1
  x = step(x, std::integral_constant<int, 0x4E>());        // lane ^ 2
  return step(x, std::integral_constant<int, 0x141>());    // the other four: mirrored within 8
}

__device__ __forceinline__ void store8_bf16(uint16_t* at, const float (&v)[8]) {
  *(u32x4*)at = (u32x4){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}
__device__ __forceinline__ void store8_e4m3(char* at, const float (&v)[8], float inv) {
  int w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, 0, false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, x, true);
  }
  *(int2*)at = make_int2(w[0], w[1]);
}

constexpr int kAppendMostRows = 4;

// A workgroup takes ROWS new rows and all their heads: 8 lanes a head's row, each with channels 8 c .. 8 c + 7 and the ones 64
// further on, which the rotation pairs with them.  The 64 angles of a row are formed once, in double precision.
template <bool FP32, int ROWS>
__global__ __launch_bounds__(256) void paged_append_kernel(AppendArgs a) {
  static_assert(ROWS <= kAppendMostRows, "a wavefront looks each row up");
  __shared__ float2 turn[ROWS][64];
  __shared__ int place[ROWS][3];                // whether a sequence has the row, page (-1: none), row of the page
  const int t0 = (int)(blockIdx.y * gridDim.x + blockIdx.x) * ROWS, lane = lane_id(), wave = wave_id();
  const int H = a.pool.heads, heads = a.q_heads + 2 * H, tasks = heads * ROWS;
  const int c = threadIdx.x & 7;
  // task i: head i / ROWS (queries, keys, values), row i % ROWS
  auto source = [&](int i, int64_t& at) __attribute__((always_inline)) {
    const int head = i / ROWS, t = t0 + i % ROWS, n = a.seqs.n_rows;
    const int own = head < a.q_heads ? head : head < a.q_heads + H ? head - a.q_heads : head - a.q_heads - H;
    at = ((int64_t)own * n + (t < n ? t : n - 1)) * kHeadDim + 8 * c;
    return head < a.q_heads ? a.q : head < a.q_heads + H ? a.k : a.v;
  };
  int task = threadIdx.x >> 3;
  RowPiece<FP32> lo, hi;
  if (task < tasks) {                           // the first rows are under way while their places are looked up
    int64_t at;
    const void* const src = source(task, at);
    lo.load(src, at);
    hi.load(src, at + 64);
  }
  if (wave < ROWS) {
    const int t = t0 + wave;
    int before = 0;                             // sequences that begin at t or before it
    for (int s = lane; s - lane < a.seqs.n_seqs; s += 64)
      before += __popcll(__builtin_amdgcn_ballot_w64(s < a.seqs.n_seqs && a.seqs.starts[s] <= t));
    bool has = false;
    uint32_t pos = 0;                           // (of two numbers below 2^31: up to 2^32)
    int page = -1;
    if (before > 0 && t < a.seqs.n_rows) {
      const PagedSeq q = paged_seq_of(a.seqs, before - 1);
      has = t >= q.first && t < q.first + q.rows;
      pos = (uint32_t)q.past + (uint32_t)(t - q.first);
      if (has && (pos >> a.pool.shift) < (uint32_t)a.seqs.table_pages) {
        page = a.seqs.table[(int64_t)(before - 1) * a.seqs.table_pages + (pos >> a.pool.shift)];
        if (page >= a.pool.n_pages) page = -1;
      }
    }
    if (a.rotate && has) {
      double s, co;
      sincos((double)pos * a.f.inv[lane], &s, &co);
      turn[wave][lane] = make_float2((float)co, (float)s);
    }
    if (lane == 0) {
      place[wave][0] = has;
      place[wave][1] = page;
      place[wave][2] = (int)(pos & ((1u << a.pool.shift) - 1));
    }
  }
  __syncthreads();
  for (; task < tasks; task += 32) {
    float x[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { x[j] = lo.get(j); y[j] = hi.get(j); }
    const int head = task / ROWS, r = task % ROWS;
    if (task + 32 < tasks) {
      int64_t at;
      const void* const src = source(task + 32, at);
      lo.load(src, at);
      hi.load(src, at + 64);
    }
    const int page = place[r][1];
    if (!place[r][0]) continue;                 // (the 8 lanes of a row go the same way)
    if (a.rotate && head < a.q_heads + H) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 cs = turn[r][8 * c + j];
        const float u = x[j], w = y[j];
        x[j] = u * cs.x - w * cs.y;
        y[j] = w * cs.x + u * cs.y;
      }
    }
    if (head < a.q_heads) {
#pragma unroll
      for (int j = 0; j < 8; ++j) { x[j] *= a.q_scale; y[j] *= a.q_scale; }
      uint16_t* const out = a.q_out + ((int64_t)head * a.seqs.n_rows + t0 + r) * kHeadDim + 8 * c;
      store8_bf16(out, x);
      store8_bf16(out + 64, y);
      continue;
    }
    if (page < 0) continue;
    const bool value = head >= a.q_heads + H;
    const int64_t row = paged_row(a.pool, page, head - a.q_heads - (value ? H : 0), place[r][2]) + (value ? 1 << a.pool.shift : 0);
    if (a.pool.bits == 16) {
      uint16_t* const out = (uint16_t*)a.pool.pages + row * kHeadDim + 8 * c;
      store8_bf16(out, x);
      store8_bf16(out + 64, y);
    } else {
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fmaxf(fabsf(x[j]), fabsf(y[j])));
      top = max_of_8(top);
      const bool any = top >= 0x1p-100f;
      const float inv = any ? 448.0f / top : 0.f;
      if (c == 0) a.pool.scales[row] = any ? top * (1.0f / 448.0f) : 0.f;
      char* const out = a.pool.pages + row * kHeadDim + 8 * c;
      store8_e4m3(out, x, inv);
      store8_e4m3(out + 64, y, inv);
    }
  }
}

}  // namespace

}  // namespace hi

using namespace hi;

extern "C" hi_status hi_paged_append(void* stream, const hi_paged_cache* cache, const hi_paged_batch* batch, const void* q_in_dev,
                                     const void* k_in_dev, const void* v_in_dev, int32_t in_fp32, int32_t n_q_heads,
                                     double rope_theta, float q_scale, void* q_out_dev) {
  AppendArgs a = {};
  const hi_status st = paged_arguments(cache, batch, "append", a.pool, a.seqs);
  if (st != HI_OK) return st;
  if (!aligned_to(q_in_dev, 16) || !aligned_to(k_in_dev, 16) || !aligned_to(v_in_dev, 16) || !aligned_to(q_out_dev, 16)) {
    set_last_error("append: buffers must be 16-byte aligned");
    return HI_ERR_ARG;
  }
  if ((in_fp32 != 0 && in_fp32 != 1) || n_q_heads < (q_in_dev || q_out_dev ? 1 : 0) || n_q_heads > (1 << 20) || cache->n_kv_heads > (1 << 20) ||
      !(rope_theta >= 0) || !(rope_theta < 1e300) || !(q_scale > 0.0f) || !(q_scale < 3.0e38f)) {
    set_last_error("append: bad shape, rope_theta or q_scale");
    return HI_ERR_ARG;
  }
  if (batch->n_seqs == 0 || batch->n_rows == 0) return HI_OK;      // (whose buffers may be null)
  if (!k_in_dev || !v_in_dev || !q_in_dev != !q_out_dev) { set_last_error("append: null buffer"); return HI_ERR_ARG; }
  if (in_fp32 && q_in_dev && q_in_dev == q_out_dev) { set_last_error("append: fp32 queries cannot be rotated in place"); return HI_ERR_ARG; }
  a.q = q_in_dev; a.k = k_in_dev; a.v = v_in_dev; a.q_out = (uint16_t*)q_out_dev;
  a.q_heads = q_in_dev ? n_q_heads : 0;
  a.q_scale = q_scale;
  a.rotate = rope_theta > 0;
  if (a.rotate)
    for (int i = 0; i < 64; ++i) a.f.inv[i] = pow(rope_theta, -(double)i / 64.0);
  StreamDevice on(stream);
  const hipStream_t s = (hipStream_t)stream;
  // One row a workgroup until they fill the chip twice over; from there on four, whose rows of a head lie side by side.
  if (batch->n_rows <= 1024) {
    const dim3 grid((unsigned)batch->n_rows);
    if (in_fp32) hipLaunchKernelGGL((paged_append_kernel<true, 1>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_append_kernel<false, 1>), grid, dim3(256), 0, s, a);
  } else {
    const int64_t n = ceil_div(batch->n_rows, 4), x = n < (1 << 22) ? n : 1 << 22;      // (a dimension of a grid has at most 2^32 lanes)
    const dim3 grid((unsigned)x, (unsigned)ceil_div(n, x));
    if (in_fp32) hipLaunchKernelGGL((paged_append_kernel<true, 4>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_append_kernel<false, 4>), grid, dim3(256), 0, s, a);
  }
  return launched("append");
}
