// Attention of a few new rows of each of many sequences over a pool of cache pages: the read of the cache is the bound.
//
// Work.  A block is the new rows of one sequence that fit 16 columns with the query heads of one KV head (16 / group positions);
// it sweeps its sequence's keys in tiles of 16 rows, which never cross a page.  The tiles of all blocks of all heads of all
// sequences, one after the other, are cut into equal runs, one for each workgroup, whatever the lengths are: every workgroup finds
// its run from the lengths themselves, so nothing is planned on the host and a captured launch follows them.  A block that lies in
// several runs is merged by the workgroup that finishes its piece last (an arrival count for each run in which a block begins).
//
// A workgroup's 4 wavefronts take the tiles of a block in turn, each with a private LDS ring of direct-to-LDS loads and no barrier
// in the loop.  The rows ride as the 16 columns of small MFMA tiles: S^T = K Q^T, O^T += V^T P^T.  8-bit rows are expanded to bf16
// (exactly) on their way from LDS to the matrix pipe; the scale of a K row multiplies its score and that of a V row its weight, in
// fp32.  The V^T operand of 8-bit rows needs no transposed read: dims are dealt to the rows of the MFMA tile so that a lane's 8
// tiles take 8 consecutive bytes of each of its 4 rows.
#include <mutex>
#include "hi_paged_attn.h"

namespace hi {

namespace {

constexpr int kTile = 16;
constexpr int kCols = 16;

template <int BITS> struct Ring;
template <> struct Ring<16> {                                   // 4 loads of K, 4 of V
  static constexpr int kRow = 256, kV = 4096, kStage = 8192, kStages = 4, kLoads = 8;
};
template <> struct Ring<8> {                                    // 2 of K, 2 of V, one of the scales of both
  static constexpr int kRow = 128, kV = 2048, kScales = 4096, kStage = 4352, kStages = 7, kLoads = 5;
};
template <int BITS> constexpr int kWaveLds = Ring<BITS>::kStage * Ring<BITS>::kStages;
constexpr int kPiece = kCols * kPartialFloats;                  // floats of a piece: O[128], m, l for each column
template <int BITS> constexpr int kLds = 4 * kWaveLds<BITS> > 4 * kPiece * 4 ? 4 * kWaveLds<BITS> : 4 * kPiece * 4;
static_assert(kLds<16> <= 160 * 1024 && kLds<8> <= 160 * 1024, "a workgroup's LDS");

// 4 bytes per lane, global -> LDS at lds_uniform + 4 * lane
__device__ __forceinline__ void g2lds4_s(const char* sbase, uint32_t voff, uint32_t lds_uniform_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds_uniform_addr), "v"(voff), "s"(sbase) : "memory");
}

// all but the loads of the `newer` newest tiles have landed
template <int LOADS, int MOST>
__device__ __forceinline__ void wait_tiles(int newer) {
  if constexpr (MOST == 0) wait_vmcnt<0>();
  else if (newer >= MOST) wait_vmcnt<LOADS * MOST>();
  else wait_tiles<LOADS, MOST - 1>(newer);
}

__device__ __forceinline__ void store_shared2(float* p, float x, float y) {
  __hip_atomic_store((uint64_t*)p, (uint64_t)__float_as_uint(x) | ((uint64_t)__float_as_uint(y) << 32), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_shared2(const float* p) {
  const uint64_t v = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

struct RowState {
  float m, l;
  f32x4 o[8];
};

// The lane's byte offsets inside a tile of K, and of V, and of its scales; rows past `last` re-read that row.
template <int BITS>
__device__ __forceinline__ void issue_tile(const PagedPool& pool, int64_t row, int last, uint32_t stage, int lane) {
  const char* const k = pool.pages + row * Ring<BITS>::kRow;
  const char* const v = k + ((int64_t)Ring<BITS>::kRow << pool.shift);
  if constexpr (BITS == 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * i + (lane >> 4), p = lane & 15, at = r < last ? r : last;
      g2lds16_s_stream(k, (uint32_t)(at * 256 + ((p ^ r) << 4)), stage + i * 1024);
      g2lds16_s_stream(v, (uint32_t)(at * 256 + ((p ^ ((r & 7) << 1)) << 4)), stage + Ring<16>::kV + i * 1024);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 8 * i + (lane >> 3), p = lane & 7, at = r < last ? r : last;
      g2lds16_s_stream(k, (uint32_t)(at * 128 + ((p ^ (r & 7)) << 4)), stage + i * 1024);
      g2lds16_s_stream(v, (uint32_t)(at * 128 + (p << 4)), stage + Ring<8>::kV + i * 1024);
    }
    const int r = lane & 15, at = r < last ? r : last;
    g2lds4_s((const char*)(pool.scales + row), (uint32_t)(at * 4 + (((lane >> 4) & 1) << (pool.shift + 2))), stage + Ring<8>::kScales);
  }
}

__device__ __forceinline__ bf16x8 two_words(uint32_t w0, uint32_t w1) {       // 8 e4m3 values as bf16
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  u32x4 x;
  x[0] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, false));
  x[1] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, 1.0f, true));
  x[2] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, false));
  x[3] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, 1.0f, true));
  return __builtin_bit_cast(bf16x8, x);
}

// One tile: keys 16 * tile + 4 * g4 + r of the lane's column, of which those up to `lim` count (hides: some of them may not).
template <int BITS>
__device__ __forceinline__ void attend_tile(lds_char* kt, int lane, const bf16x8 (&qf)[4], RowState& st, float c, bool hides, int key0, int lim) {
  typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  typedef __attribute__((address_space(3))) uint64_t lds_u64;
  const int tok = lane & 15, g4 = lane >> 4;
  lds_char* const vt = kt + Ring<BITS>::kV;
  short4v vop[8];
  f32x4 s = (f32x4){0.f, 0.f, 0.f, 0.f}, vs = (f32x4){1.f, 1.f, 1.f, 1.f};
  if constexpr (BITS == 16) {
    const int v_row = 4 * g4 + (tok >> 2), v_sub = lane & 3;
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const int chunk = (2 * db + (v_sub >> 1)) ^ ((v_row & 7) << 1);
      vop[db] = __builtin_bit_cast(short4v, lds_read_tr8(vt + v_row * 256 + (chunk << 4) + ((v_sub & 1) << 3)));
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_read16(kt + tok * 256 + (((4 * kk + g4) ^ tok) << 4)), qf[kk], s, 0, 0, 0);
  } else {
    u32x4 kw[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) kw[i] = *(lds_u32x4*)(kt + tok * 128 + (((2 * g4 + i) ^ (tok & 7)) << 4));
    uint32_t w[4][4];                                            // [row][pair of dims], bf16
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint64_t b = *(lds_u64*)(vt + (4 * g4 + r) * 128 + tok * 8);
      const u32x4 x = __builtin_bit_cast(u32x4, two_words((uint32_t)b, (uint32_t)(b >> 32)));
#pragma unroll
      for (int e = 0; e < 4; ++e) w[r][e] = x[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint2 lo, hi;
      lo.x = __builtin_amdgcn_perm(w[1][e], w[0][e], 0x05040100); lo.y = __builtin_amdgcn_perm(w[3][e], w[2][e], 0x05040100);
      hi.x = __builtin_amdgcn_perm(w[1][e], w[0][e], 0x07060302); hi.y = __builtin_amdgcn_perm(w[3][e], w[2][e], 0x07060302);
      vop[2 * e] = __builtin_bit_cast(short4v, lo);
      vop[2 * e + 1] = __builtin_bit_cast(short4v, hi);
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(two_words(kw[kk >> 1][2 * (kk & 1)], kw[kk >> 1][2 * (kk & 1) + 1]), qf[kk], s, 0, 0, 0);
    lds_char* const sc = kt + Ring<8>::kScales + 16 * g4;
    s *= *(lds_f32x4*)sc;
    vs = *(lds_f32x4*)(sc + 64);
  }
  const int key = key0 + 4 * g4;
  if (hides) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (key + r > lim) s[r] = kNegBig;
  }
  float mx = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
  mx = over_rows16(mx, op_max);
  const float m_new = fmaxf(st.m, mx);
  if (__builtin_amdgcn_ballot_w64(m_new > st.m) != 0) {
    const float alpha = fast_exp2((st.m - m_new) * c);
    st.l *= alpha;
#pragma unroll
    for (int i = 0; i < 8; ++i) st.o[i] *= alpha;
    st.m = m_new;
  }
  const float mc = st.m * c;
  float p[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) p[r] = fast_exp2(__builtin_fmaf(s[r], c, -mc));
  if (hides) {                                                   // exactly zero while the column has seen nothing, too
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (key + r > lim) p[r] = 0.f;
  }
  st.l += (p[0] + p[1]) + (p[2] + p[3]);
  if constexpr (BITS == 8) {
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] *= vs[r];
  }
  // the weights are rounded to bf16 for the matrix pipe (2^-9 of each at most); their sum is that of the fp32 values
  const uint2 pw = make_uint2(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]));
#pragma unroll
  for (int db = 0; db < 8; ++db) st.o[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vop[db], __builtin_bit_cast(short4v, pw), st.o[db], 0, 0, 0);
}

// The sum of the lanes up to this one.
__device__ __forceinline__ int scan_wave(int x, int lane) {
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const int y = __shfl_up(x, off);
    if (lane >= off) x += y;
  }
  return x;
}

// A sequence's share of the tiles.
struct SeqWork { int tiles, blocks; };          // tiles of a block (the deepest one's), blocks of a head
__device__ __forceinline__ SeqWork seq_work(const PagedAttnArgs& a, const PagedSeq& q) {
  SeqWork w;
  const int64_t len = (int64_t)q.past + q.rows, most = (int64_t)a.seqs.table_pages << a.pool.shift;
  w.tiles = (int)(((len < most ? len : most) + kTile - 1) / kTile);
  w.blocks = q.rows == 0 ? 0 : (q.rows + a.positions - 1) / a.positions;
  return w;
}

// What the 4 wavefronts hold for the columns, from LDS: the workgroup's (m, l) of a column and its weighted sum of dims d, d + 1.
__device__ __forceinline__ float2 merge_waves(const float* red, int col, int d, float c, float& m, float& l) {
  float mw[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) mw[w] = red[w * kPiece + col * kPartialFloats + kHeadDim];
  m = fmaxf(fmaxf(mw[0], mw[1]), fmaxf(mw[2], mw[3]));
  l = 0.f;
  float2 o = make_float2(0.f, 0.f);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float* const x = red + w * kPiece + col * kPartialFloats;
    const float f = fast_exp2((mw[w] - m) * c);
    l += f * x[kHeadDim + 1];
    o.x += f * x[d];
    o.y += f * x[d + 1];
  }
  return o;
}

// Columns of a block to the output: column i is position i / group of the block, query head i % group of the KV head.
__device__ __forceinline__ void write_out(const PagedAttnArgs& a, int kv, int row0, int col, int d, float2 o, float l) {
  const int pos = (col * a.by_group) >> 16, g = col - pos * a.group;
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  *(uint32_t*)(a.out + ((int64_t)(kv * a.group + g) * a.seqs.n_rows + row0 + pos) * kHeadDim + d) = pack_bf16(o.x * inv, o.y * inv);
}

// The last arrival's merge: all pieces of a block, those of runs first .. last; wavefront w takes every fourth, four at a time and four
// columns at a time, so that 32 loads are under way together, and leaves its sums in LDS.
__device__ __forceinline__ void gather_pieces(const float* pieces, int first, int last, int cols, float* red, float c, int lane, int wave) {
  for (int c0 = 0; c0 < cols; c0 += 4) {
    float m[4], l[4];
    float2 o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) { m[j] = kNegBig; l[j] = 0.f; o[j] = make_float2(0.f, 0.f); }
    for (int p0 = first + wave; p0 <= last; p0 += 16) {
      float2 ml[4][4], x[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int p = p0 + 4 * i;
          ml[i][j] = make_float2(kNegBig, 0.f);
          x[i][j] = make_float2(0.f, 0.f);
          if (p <= last && c0 + j < cols) {
            const float* const at = pieces + (int64_t)(2 * p + (p == first)) * kPiece + (c0 + j) * kPartialFloats;
            ml[i][j] = load_shared2(at + kHeadDim);
            x[i][j] = load_shared2(at + 2 * lane);
          }
        }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float mn = fmaxf(fmaxf(fmaxf(ml[0][j].x, ml[1][j].x), fmaxf(ml[2][j].x, ml[3][j].x)), m[j]);
        const float f = fast_exp2((m[j] - mn) * c);
        l[j] *= f; o[j].x *= f; o[j].y *= f;
        m[j] = mn;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = fast_exp2((ml[i][j].x - mn) * c);
          l[j] += e * ml[i][j].y; o[j].x += e * x[i][j].x; o[j].y += e * x[i][j].y;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c0 + j < cols) {
        float* const to = red + wave * kPiece + (c0 + j) * kPartialFloats;
        *(float2*)(to + 2 * lane) = o[j];
        if (lane == 0) *(float2*)(to + kHeadDim) = make_float2(m[j], l[j]);
      }
  }
}

template <int BITS>
__global__ __launch_bounds__(256, 1) void paged_decode_kernel(PagedAttnArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds_raw[];
  __shared__ int arrived;
  const int lane = lane_id(), wave = wave_id(), g4 = lane >> 4, col = lane & 15;
  const int H = a.pool.heads, S = a.seqs.n_seqs;
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_char*)lds_raw + wave * kWaveLds<BITS>;
  float* const red = (float*)lds_raw;

  // all tiles, and the sequence of this run's first one
  int total = 0;
  float about = 0.f;                                               // (a batch whose sequences overlap could overflow the count)
  for (int s0 = 0; s0 < S; s0 += 64) {
    int mine = 0;
    if (s0 + lane < S) {
      const SeqWork w = seq_work(a, paged_seq_of(a.seqs, s0 + lane));
      mine = w.tiles * w.blocks * H;
    }
    total += __builtin_amdgcn_readlane(scan_wave(mine, lane), 63);
    about += over_wave((float)mine, op_add);
  }
  if (about > 2.1e9f) return;
  int run = (total + gridDim.x - 1) / gridDim.x;
  run = run < kPagedLeastRun ? kPagedLeastRun : run;
  int at = blockIdx.x * run;
  if (at >= total) return;
  const int end = at + run < total ? at + run : total;
  int seq = 0, before = 0;
  for (int s0 = 0; s0 < S; s0 += 64) {
    int mine = 0;
    if (s0 + lane < S) {
      const SeqWork w = seq_work(a, paged_seq_of(a.seqs, s0 + lane));
      mine = w.tiles * w.blocks * H;
    }
    const int upto = scan_wave(mine, lane);
    const int n = __popcll(__builtin_amdgcn_ballot_w64(before + upto <= at));      // lanes past the last sequence add nothing
    if (n < 64) {
      seq = s0 + n;
      if (n > 0) before += __builtin_amdgcn_readlane(upto, n - 1);
      break;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  seq = __builtin_amdgcn_readfirstlane(seq);
  before = __builtin_amdgcn_readfirstlane(before);

  while (at < end && seq < S) {
    const PagedSeq sq = paged_seq_of(a.seqs, seq);
    const SeqWork w = seq_work(a, sq);
    const int of_seq = w.tiles * w.blocks * H;
    if (at >= before + of_seq) {                                   // (a sequence without rows has no tiles)
      before += of_seq;
      ++seq;
      continue;
    }
    const int item = (at - before) / w.tiles;
    const int begin = before + item * w.tiles, done = begin + w.tiles;   // the block's tiles among all
    const int kv = item / w.blocks, b = item - kv * w.blocks;
    const int t0 = at - begin, t1 = (end < done ? end : done) - begin;

    const int row0 = sq.first + b * a.positions;
    const int rows = sq.rows - b * a.positions < a.positions ? sq.rows - b * a.positions : a.positions;
    const int cols = rows * a.group;
    const int pos = (col * a.by_group) >> 16, g = col - pos * a.group;
    const int64_t most = (int64_t)a.seqs.table_pages << a.pool.shift, all = (int64_t)sq.past + sq.rows;
    const int len = (int)(all < most ? all : most);
    // the last key that the lane's position sees, and that the block's first one does
    auto sees = [&](int i) __attribute__((always_inline)) {
      const int64_t key = (int64_t)sq.past + b * a.positions + i;
      return (int)(key < len ? key : len - 1);
    };
    const int lim = sees(pos), all_see = sees(0);
    const int* const table = a.seqs.table + (int64_t)seq * a.seqs.table_pages;

    // the wavefront's tiles are t0 + wave, t0 + wave + 4, ..; the pages of the next 64 of them are looked up at once
    const int mine = t1 - t0 > wave ? (t1 - t0 - wave + 3) >> 2 : 0;
    auto tile_of = [&](int j) __attribute__((always_inline)) { return t0 + wave + 4 * j; };
    auto pages_from = [&](int j) __attribute__((always_inline)) {
      const int t = tile_of(j + lane);
      return j + lane < mine ? table[(t * kTile) >> a.pool.shift] : -1;
    };
    int pages = pages_from(0), pages_next = 0, base = 0;
    auto page_of = [&](int j) __attribute__((always_inline)) {
      return j - base < 64 ? __builtin_amdgcn_readlane(pages, j - base) : __builtin_amdgcn_readlane(pages_next, j - base - 64);
    };
    auto there = [&](int page) __attribute__((always_inline)) { return page >= 0 && page < a.pool.n_pages; };
    auto issue = [&](int j, int stage) __attribute__((always_inline)) {
      const int t = tile_of(j), page = page_of(j), last = len - 1 - t * kTile;
      const int64_t row = paged_row(a.pool, there(page) ? page : 0, kv, (t * kTile) & ((1 << a.pool.shift) - 1));
      issue_tile<BITS>(a.pool, row, last < kTile ? last : kTile - 1, ring + stage * Ring<BITS>::kStage, lane);
    };
    constexpr int kAhead = Ring<BITS>::kStages - 1;
    for (int j = 0; j < kAhead; ++j)
      if (j < mine) issue(j, j);

    // Q^T: the lane's column, channels 32 kk + 8 g4 .. (8-bit rows: 32 g4 + 8 kk ..); columns without a row are zeros
    bf16x8 qf[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (col < cols)
        raw = *(const uint4*)(a.q + ((int64_t)(kv * a.group + g) * a.seqs.n_rows + row0 + pos) * kHeadDim + (BITS == 16 ? 32 * kk + 8 * g4 : 32 * g4 + 8 * kk));
      qf[kk] = __builtin_bit_cast(bf16x8, raw);
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) asm volatile("" : "+v"(qf[kk]));

    RowState st;
    st.m = kNegBig;
    st.l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) st.o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    int stage = 0, ahead = kAhead % Ring<BITS>::kStages;
    for (int j = 0; j < mine; ++j) {
      if (j - base == 64 - kAhead) pages_next = pages_from(base + 64);       // before the first look-up beyond the 64
      if (j - base == 64) {
        pages = pages_next;
        base += 64;
      }
      if (j + kAhead < mine) issue(j + kAhead, ahead);
      wait_tiles<Ring<BITS>::kLoads, kAhead>(mine - 1 - j);
      const int t = tile_of(j);
      if (there(page_of(j)))
        attend_tile<BITS>((lds_char*)(uintptr_t)(ring + stage * Ring<BITS>::kStage), lane, qf, st, a.c, t * kTile + kTile - 1 > all_see, t * kTile, lim);
      asm volatile("" ::: "memory");
      stage = stage + 1 < Ring<BITS>::kStages ? stage + 1 : 0;
      ahead = ahead + 1 < Ring<BITS>::kStages ? ahead + 1 : 0;
    }
    st.l = over_rows16(st.l, op_add);

    __syncthreads();                                               // the rings are idle
    if (col < cols) {
      float* const to = red + wave * kPiece + col * kPartialFloats;
#pragma unroll
      for (int db = 0; db < 8; ++db)
#pragma unroll
        for (int r = 0; r < 4; ++r) to[BITS == 16 ? 16 * db + 4 * g4 + r : 8 * (4 * g4 + r) + db] = st.o[db][r];
      if (g4 == 0) {
        to[kHeadDim] = st.m;
        to[kHeadDim + 1] = st.l;
      }
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == w.tiles;
    float* const mine_to = a.pieces + (int64_t)(2 * blockIdx.x + (t0 == 0)) * kPiece;
    for (int i = threadIdx.x; i < cols * 64; i += 256) {
      float m, l;
      const float2 o = merge_waves(red, i >> 6, 2 * (i & 63), a.c, m, l);
      if (whole) {
        write_out(a, kv, row0, i >> 6, 2 * (i & 63), o, l);
      } else {
        float* const to = mine_to + (i >> 6) * kPartialFloats;
        store_shared2(to + 2 * (i & 63), o.x, o.y);
        if ((i & 63) == 0) store_shared2(to + kHeadDim, m, l);
      }
    }
    if (!whole) {
      const int first = begin / run, last = (done - 1) / run;
      // Pieces are written and read by device-scope accesses that no L2 keeps a copy of, so the wait for the stores, the barrier and the
      // count order them; a release or acquire of everything else would walk the whole L2 (1000 rows of 8 heads: 21 us instead of 8).
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (threadIdx.x == 0) arrived = __hip_atomic_fetch_add(a.arrivals + first, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      if (arrived == last - first) {                               // the others' pieces are there
        gather_pieces(a.pieces, first, last, cols, red, a.c, lane, wave);
        __syncthreads();
        for (int i = threadIdx.x; i < cols * 64; i += 256) {
          float m, l;
          const float2 o = merge_waves(red, i >> 6, 2 * (i & 63), a.c, m, l);
          write_out(a, kv, row0, i >> 6, 2 * (i & 63), o, l);
        }
        if (threadIdx.x == 0) __hip_atomic_store(a.arrivals + first, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    __syncthreads();                                               // LDS is free for the next block
    at = begin + t1;
  }
}

template <int BITS>
hi_status decode_go(void* stream, const PagedAttnArgs& a) {
  static std::once_flag once;
  static hipError_t attr = hipSuccess;
  std::call_once(once, [] { attr = hipFuncSetAttribute((const void*)paged_decode_kernel<BITS>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds<BITS>); });
  if (attr != hipSuccess) { set_last_error("paged attention: %s", hipGetErrorString(attr)); return HI_ERR_HIP; }
  hipLaunchKernelGGL(paged_decode_kernel<BITS>, dim3(kPagedRuns), dim3(256), kLds<BITS>, (hipStream_t)stream, a);
  return launched("paged attention");
}

}  // namespace

static_assert(kPagedPieceFloats == kPiece, "the workspace's pieces");

hi_status launch_paged_decode(void* stream, const PagedAttnArgs& a) {
  return a.pool.bits == 16 ? decode_go<16>(stream, a) : decode_go<8>(stream, a);
}

}  // namespace hi
