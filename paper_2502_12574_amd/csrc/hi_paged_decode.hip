// Attention of a few new rows of each of many sequences over a pool of cache pages: the read of the cache is the bound.
// One token, 8 KV heads, 4 query heads each: behind 524211 bf16 rows 316 us (6.8 TB/s), 64 of them behind up to 32000 8-bit rows 212 us
// (6.5 TB/s); behind 1000 rows 8.5 us, a chain of latencies: dispatch, lengths, pages, tiles, pieces, merge.
//
// Work.  A block is the new rows of one sequence that fit 16 columns with the query heads of one KV head (16 / group positions);
// it sweeps its sequence's keys in tiles of 32 rows, two halves that never cross a page.  The tiles of all blocks of all heads of all
// sequences, one after the other, are cut into equal runs, one for each workgroup, whatever the lengths are (a block counts for
// kPagedStart tiles more: its first loads and its merge are not hidden by anything); where there are so few
// that every block can be cut into equal pieces of at most a run without more pieces than workgroups, a workgroup takes such a piece
// instead.  Every workgroup finds its part from the lengths themselves, so nothing is planned on the host and a captured launch
// follows them.  A block that lies in several parts is merged by the workgroup that finishes last: 16 or 32 parts at a time, then those.
//
// A workgroup's 4 wavefronts take the tiles of a block in turn, each with a private LDS ring of direct-to-LDS loads and no barrier
// in the loop.  The rows ride as the 16 columns of small MFMA tiles: S^T = K Q^T, O^T += V^T P^T.  8-bit rows are expanded to bf16
// (exactly) on their way from LDS to the matrix pipe; the scale of a K row multiplies its score and that of a V row its weight, in
// fp32.  The V^T operand of 8-bit rows needs no transposed read: dims are dealt to the rows of the MFMA tile so that a lane's 8
// tiles take 8 consecutive bytes of each of its rows.  One wavefront a SIMD issues an instruction each 7 cycles, and with tiles of 16
// rows (a maximum, a rescale check and a product of their own for every 16 keys) 8-bit pages were bound by that: 4.8 TB/s.
#include <mutex>
#include "hi_paged_attn.h"

namespace hi {

namespace {

constexpr int kTile = 32;
constexpr int kShortTable = 1024;               // entries of a page table that are brought to LDS at once
constexpr int kCols = 16;

// A slot of a ring holds half a tile, 16 rows.
template <int BITS> struct Ring;
template <> struct Ring<16> {                                   // 4 loads of K, 4 of V
  static constexpr int kRow = 256, kV = 4096, kSlot = 8192, kSlots = 4, kLoads = 8;
};
template <> struct Ring<8> {                                    // 2 of K, 2 of V, one of the scales of both
  static constexpr int kRow = 128, kV = 2048, kScales = 4096, kSlot = 4352, kSlots = 8, kLoads = 5;
};
template <int BITS> constexpr int kWaveLds = Ring<BITS>::kSlot * Ring<BITS>::kSlots;
constexpr int kPiece = kCols * kPartialFloats;                  // floats of a piece: O[128], m, l for each column
template <int BITS> constexpr int kLds = 4 * kWaveLds<BITS> > 4 * kPiece * 4 ? 4 * kWaveLds<BITS> : 4 * kPiece * 4;
static_assert(kLds<16> <= 159 * 1024 && kLds<8> <= 159 * 1024, "a workgroup's LDS");

// 4 bytes per lane, global -> LDS at lds_uniform + 4 * lane
__device__ __forceinline__ void g2lds4_s(const char* sbase, uint32_t voff, uint32_t lds_uniform_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds_uniform_addr), "v"(voff), "s"(sbase) : "memory");
}

// all but the loads of the `newer` newest halves have landed
template <int LOADS, int MOST>
__device__ __forceinline__ void wait_halves(int newer) {
  if constexpr (MOST == 0) wait_vmcnt<0>();
  else if (newer >= MOST) wait_vmcnt<LOADS * MOST>();
  else wait_halves<LOADS, MOST - 2>(newer);
}

struct RowState {
  float m, l;
  f32x4 o[8];
};

// The lane's byte offsets in the loads of a half: load i of K lies i loads further on, with the swizzle bits of its rows.
template <int BITS> struct HalfLane { uint32_t k, v, sc; };
template <int BITS>
__device__ __forceinline__ HalfLane<BITS> half_lane(int lane, int shift) {
  if constexpr (BITS == 16) {
    const int r = lane >> 4, p = lane & 15;      // chunk p of row r: chunk p ^ r of a K row, p ^ 2 (r % 8) of a V row
    return {(uint32_t)(r * 256 + ((p ^ r) << 4)), (uint32_t)(r * 256 + ((p ^ (2 * r)) << 4)), 0u};
  } else {
    const int r = lane >> 3, p = lane & 7;       // chunk p ^ (r % 8) of a K row
    return {(uint32_t)(r * 128 + ((p ^ r) << 4)), (uint32_t)(r * 128 + (p << 4)), (uint32_t)((lane & 15) * 4 + (((lane >> 4) & 1) << (shift + 2)))};
  }
}

// The loads of a half tile: K from k on, V from v on, scales from sc on; rows past `last` re-read that row.
template <int BITS>
__device__ __forceinline__ void issue_half(const char* k, const char* v, const char* sc, int last, uint32_t slot, int lane, const HalfLane<BITS>& hl, int shift) {
  if (last >= 15) {
    if constexpr (BITS == 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        g2lds16_s_stream(k, hl.k ^ (uint32_t)(i * 1024 + i * 64), slot + i * 1024);
        g2lds16_s_stream(v, hl.v ^ (uint32_t)(i * 1024 + (i & 1) * 128), slot + Ring<16>::kV + i * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        g2lds16_s_stream(k, hl.k + i * 1024, slot + i * 1024);
        g2lds16_s_stream(v, hl.v + i * 1024, slot + Ring<8>::kV + i * 1024);
      }
      g2lds4_s(sc, hl.sc, slot + Ring<8>::kScales);
    }
  } else {
    if constexpr (BITS == 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * i + (lane >> 4), p = lane & 15, at = r < last ? r : last;
        g2lds16_s_stream(k, (uint32_t)(at * 256 + ((p ^ r) << 4)), slot + i * 1024);
        g2lds16_s_stream(v, (uint32_t)(at * 256 + ((p ^ ((r & 7) << 1)) << 4)), slot + Ring<16>::kV + i * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = 8 * i + (lane >> 3), p = lane & 7, at = r < last ? r : last;
        g2lds16_s_stream(k, (uint32_t)(at * 128 + ((p ^ (r & 7)) << 4)), slot + i * 1024);
        g2lds16_s_stream(v, (uint32_t)(at * 128 + (p << 4)), slot + Ring<8>::kV + i * 1024);
      }
      const int r = lane & 15, at = r < last ? r : last;
      g2lds4_s(sc, (uint32_t)(at * 4 + (((lane >> 4) & 1) << (shift + 2))), slot + Ring<8>::kScales);
    }
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

// One tile, its halves at at[0] and at[1].  Register r of half h of the lane (column lane % 16, g4 = lane / 16) is key 16 h + 4 g4 + r, and
// the contraction of the second product takes them in that order, h, then r.  hides: only the keys up to lim[h] of a half count; later: and
// others may be rows (behind the last row lie only copies of it).
template <int BITS>
__device__ __forceinline__ void attend_tile(lds_char* const (&at)[2], int lane, const bf16x8 (&qf)[4], RowState& st, float c, bool hides, bool later, const int (&lim)[2]) {
  typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  typedef __attribute__((address_space(3))) uint64_t lds_u64;
  const int tok = lane & 15, g4 = lane >> 4;
  bf16x8 vop[8];
  f32x4 s[2], vs[2];
  s[0] = s[1] = (f32x4){0.f, 0.f, 0.f, 0.f};
  if constexpr (BITS == 16) {
    const int v_row = 4 * g4 + (tok >> 2), v_sub = lane & 3;
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const int off = Ring<16>::kV + v_row * 256 + (((2 * db + (v_sub >> 1)) ^ ((v_row & 7) << 1)) << 4) + ((v_sub & 1) << 3);
      vop[db] = (bf16x8)__builtin_shufflevector(lds_read_tr8(at[0] + off), lds_read_tr8(at[1] + off), 0, 1, 2, 3, 4, 5, 6, 7);
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lds_read16(at[h] + tok * 256 + (((4 * kk + g4) ^ tok) << 4)), qf[kk], s[h], 0, 0, 0);
  } else {
    u32x4 kw[2][2];
    uint64_t vb[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) kw[h][i] = *(lds_u32x4*)(at[h] + tok * 128 + (((2 * g4 + i) ^ (tok & 7)) << 4));
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) vb[h][r] = *(lds_u64*)(at[h] + Ring<8>::kV + (4 * g4 + r) * 128 + tok * 8);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t w0 = kw[h][kk >> 1][2 * (kk & 1)], w1 = kw[h][kk >> 1][2 * (kk & 1) + 1];
        s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(two_words(w0, w1), qf[kk], s[h], 0, 0, 0);
      }
    u32x4 x[2][4];                                               // [half][row]: 8 dims as bf16, two to a word
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[h][r] = __builtin_bit_cast(u32x4, two_words((uint32_t)vb[h][r], (uint32_t)(vb[h][r] >> 32)));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      u32x4 lo, hi;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          lo[2 * h + r] = __builtin_amdgcn_perm(x[h][2 * r + 1][e], x[h][2 * r][e], 0x05040100);
          hi[2 * h + r] = __builtin_amdgcn_perm(x[h][2 * r + 1][e], x[h][2 * r][e], 0x07060302);
        }
      vop[2 * e] = __builtin_bit_cast(bf16x8, lo);
      vop[2 * e + 1] = __builtin_bit_cast(bf16x8, hi);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      lds_char* const sc = at[h] + Ring<8>::kScales + 16 * g4;
      s[h] *= *(lds_f32x4*)sc;
      vs[h] = *(lds_f32x4*)(sc + 64);
    }
  }
  if (hides) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * g4 + r > lim[h]) s[h][r] = kNegBig;
  }
  float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
  mx = over_rows16(mx, op_max);
  const float m_new = fmaxf(st.m, mx);
  if (__builtin_amdgcn_ballot_w64(m_new > st.m) != 0) {
    const float alpha = fast_exp2((st.m - m_new) * c);
    st.l *= alpha;
#pragma unroll
    for (int i = 0; i < 8; ++i) st.o[i] *= alpha;
    st.m = m_new;
  }
  const float mc = st.m > kNegBig ? st.m * c : 0.f;              // a column that has seen nothing yet adds weights of zero
  float p[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) p[h][r] = fast_exp2(__builtin_fmaf(s[h][r], c, -mc));
  st.l += ((p[0][0] + p[0][1]) + (p[0][2] + p[0][3])) + ((p[1][0] + p[1][1]) + (p[1][2] + p[1][3]));
  if constexpr (BITS == 8) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) p[h][r] *= vs[h][r];
  }
  // the weights are rounded to bf16 for the matrix pipe (2^-9 of each at most); their sum is that of the fp32 values
  u32x4 pw = {pack_bf16(p[0][0], p[0][1]), pack_bf16(p[0][2], p[0][3]), pack_bf16(p[1][0], p[1][1]), pack_bf16(p[1][2], p[1][3])};
  if (hides && later) {
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (BITS == 8) bad |= not_finite(pw[e]);                   // (a scale that is not)
#pragma unroll
      for (int db = 0; db < 8; ++db) bad |= not_finite(__builtin_bit_cast(u32x4, vop[db])[e]);
    }
    if (__builtin_amdgcn_ballot_w64((bad & 0x80008000u) != 0) != 0) {
      u32x4 seen;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = e >> 1, r = 4 * g4 + 2 * (e & 1);
        const uint32_t shown = (r <= lim[h] ? 0xFFFFu : 0u) | (r + 1 <= lim[h] ? 0xFFFF0000u : 0u);
        pw[e] &= shown;
        seen[e] = 0x3F803F80u & shown;
      }
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const TwoParts v = two_parts(vop[db]);
        const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.others, __builtin_bit_cast(bf16x8, seen), (f32x4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        st.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.finite, __builtin_bit_cast(bf16x8, pw), st.o[db], 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) st.o[db][r] = hit[r] > 0.f ? __builtin_nanf("") : st.o[db][r];
      }
      return;
    }
  }
#pragma unroll
  for (int db = 0; db < 8; ++db) st.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vop[db], __builtin_bit_cast(bf16x8, pw), st.o[db], 0, 0, 0);
}

// A sequence's share of the tiles.
struct SeqWork { int tiles, items; };           // tiles of a block (the deepest one's); blocks of all heads
__device__ __forceinline__ SeqWork seq_work(const PagedAttnArgs& a, const PagedSeq& q) {
  SeqWork w;
  const int64_t len = (int64_t)q.past + q.rows, most = (int64_t)a.seqs.table_pages << a.pool.shift;
  w.tiles = (int)(((len < most ? len : most) + kTile - 1) / kTile);
  w.items = q.rows == 0 ? 0 : (int)((uint32_t)(q.rows + a.positions - 1) / (uint32_t)a.positions) * a.pool.heads;
  return w;
}

// What the 4 wavefronts hold for a column, from LDS: the workgroup's (m, l) and its weighted sum of dims d, d + 1.
__device__ __forceinline__ float2 merge_waves(const float* red, int col, int d, float c, float& m, float& l) {
  float2 ml[4], x[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float* const at = red + w * kPiece + col * kPartialFloats;
    ml[w] = *(const float2*)(at + kHeadDim);
    x[w] = *(const float2*)(at + d);
  }
  m = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
  l = 0.f;
  float2 o = make_float2(0.f, 0.f);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = fast_exp2((ml[w].x - m) * c);
    l += f * ml[w].y;
    o.x += f * x[w].x;
    o.y += f * x[w].y;
  }
  return o;
}

// Columns of a block to the output: column i is position i / group of the block, query head i % group of the KV head.
__device__ __forceinline__ void write_out(const PagedAttnArgs& a, int kv, int row0, int col, int d, float2 o, float l) {
  const int pos = (col * a.by_group) >> 16, g = col - pos * a.group;
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  *(uint32_t*)(a.out + ((int64_t)(kv * a.group + g) * a.seqs.n_rows + row0 + pos) * kHeadDim + d) = pack_bf16(o.x * inv, o.y * inv);
}

// A merge of up to 4 P pieces, piece_at(i) being where piece i lies: wavefront w takes every fourth, for N columns from c0 on (all their
// loads under way together), and leaves its sums in LDS.
template <int P, int N, class At>
__device__ __forceinline__ void gather_columns(int n, At piece_at, int c0, int cols, float* red, float c, int lane, int wave) {
  float2 ml[P][N], x[P][N];
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int p = wave + 4 * i;
      ml[i][j] = make_float2(kNegBig, 0.f);
      x[i][j] = make_float2(0.f, 0.f);
      if (p < n && c0 + j < cols) {
        const float* const at = piece_at(p) + (c0 + j) * kPartialFloats;
        ml[i][j] = load_shared2(at + kHeadDim);
        x[i][j] = load_shared2(at + 2 * lane);
      }
    }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float m = ml[0][j].x, l = 0.f;
#pragma unroll
    for (int i = 1; i < P; ++i) m = fmaxf(m, ml[i][j].x);
    float2 o = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float e = fast_exp2((ml[i][j].x - m) * c);
      l += e * ml[i][j].y; o.x += e * x[i][j].x; o.y += e * x[i][j].y;
    }
    if (c0 + j < cols) {
      float* const to = red + wave * kPiece + (c0 + j) * kPartialFloats;
      *(float2*)(to + 2 * lane) = o;
      if (lane == 0) *(float2*)(to + kHeadDim) = make_float2(m, l);
    }
  }
}
// How many pieces are merged at once: the loads of 32 of up to 4 columns, or of 16 of 8, fit the registers.
__device__ __forceinline__ int fan_of(int cols) { return cols <= 4 ? 32 : 16; }
template <class At>
__device__ __forceinline__ void gather_pieces(int n, At piece_at, int cols, float* red, float c, int lane, int wave) {
  if (cols <= 4) {
    if (n <= 16) gather_columns<4, 4>(n, piece_at, 0, cols, red, c, lane, wave);
    else gather_columns<8, 4>(n, piece_at, 0, cols, red, c, lane, wave);
  } else {
    for (int c0 = 0; c0 < cols; c0 += 8) gather_columns<4, 8>(n, piece_at, c0, cols, red, c, lane, wave);
  }
}

// n / d for quotients of a few hundred at most (by_d: 1 / d, nearly)
__device__ __forceinline__ uint32_t small_quotient(uint32_t n, uint32_t d, float by_d) {
  const uint32_t q = (uint32_t)((float)n * by_d);
  const int rest = (int)(n - q * d);
  return rest < 0 ? q - 1 : rest >= (int)d ? q + 1 : q;
}

template <int BITS>
__global__ __launch_bounds__(256, 2) void paged_decode_kernel(PagedAttnArgs a) {
  using R = Ring<BITS>;
  extern __shared__ __attribute__((aligned(1024))) char lds_raw[];
  __shared__ int arrived, short_table[kShortTable];
  const int lane = lane_id(), wave = wave_id(), g4 = lane >> 4, col = lane & 15;
  const int S = a.seqs.n_seqs, shift = a.pool.shift, page_rows = 1 << shift;
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_char*)lds_raw + wave * kWaveLds<BITS>;
  float* const red = (float*)lds_raw;

  // All tiles, from them the length of a run and how many pieces of at most that length there would be.
  PagedSeq mine = {0, 0, 0};                                       // the lane's sequence (of the last 64 that were looked at)
  SeqWork mw = {0, 0};
  auto look = [&](int s0) __attribute__((always_inline)) {
    mine = s0 + lane < S ? paged_seq_of(a.seqs, s0 + lane) : PagedSeq{0, 0, 0};
    mw = seq_work(a, mine);
  };
  // A short table is brought along with the lengths: the pages of a tile are known one latency earlier.
  const int64_t all_entries = (int64_t)S * a.seqs.table_pages;
  const int entries = all_entries <= kShortTable ? (int)all_entries : 0;
  if (S <= 64) look(0);
  int brought[kShortTable / 256];
#pragma unroll
  for (int i = 0; i < kShortTable / 256; ++i) brought[i] = (int)threadIdx.x + 256 * i < entries ? a.seqs.table[threadIdx.x + 256 * i] : 0;
  constexpr int kStart = kPagedStart<BITS>;
  int tiles_of_all = 0, items_of_all = 0;
  float about = 0.f;                                               // (a batch whose sequences overlap could overflow the count)
  for (int s0 = 0; s0 < S; s0 += 64) {
    if (S > 64) look(s0);
    tiles_of_all += __builtin_amdgcn_readlane(sum_wave(mw.tiles * mw.items), 63);
    items_of_all += __builtin_amdgcn_readlane(sum_wave(mw.items), 63);
    about += over_wave((float)(mw.tiles + kStart) * (float)mw.items, op_add);
  }
  if (about > 1.01f * kPagedMostTiles) return;
  constexpr uint32_t wgs = kPagedRuns;
  // equal pieces: as small as a workgroup each allows, or a quarter larger
  uint32_t piece_tiles = ((uint32_t)tiles_of_all + wgs - 1) / wgs;
  piece_tiles = piece_tiles < kPagedLeastRun ? kPagedLeastRun : piece_tiles;
  int pieces = 0;
  bool by_piece = false;
  float by_tiles = 0.f;
  auto pieces_of = [&](int tiles) __attribute__((always_inline)) { return (int)small_quotient(tiles + piece_tiles - 1, piece_tiles, by_tiles); };
#pragma unroll
  for (int attempt = 0; attempt < 2 && !by_piece; ++attempt) {
    if (attempt == 1) piece_tiles += piece_tiles / 4 + 1;
    pieces = 0;                                                    // (at most as many as tiles; of a block, twice wgs at most)
    by_tiles = __builtin_amdgcn_rcpf((float)piece_tiles);
    for (int s0 = 0; s0 < S; s0 += 64) {
      if (S > 64) look(s0);
      pieces += __builtin_amdgcn_readlane(sum_wave(pieces_of(mw.tiles) * mw.items), 63);
    }
    by_piece = pieces <= (int)wgs;
  }
  const int total = tiles_of_all + kStart * items_of_all, run = (int)(((uint32_t)total + wgs - 1) / wgs);
  // From here on a block has units: its start and its tiles, or its equal pieces if a workgroup takes one of them.
  auto units_of = [&](int tiles) __attribute__((always_inline)) { return by_piece ? pieces_of(tiles) : tiles + kStart; };
  const int step = by_piece ? 1 : run, all = by_piece ? pieces : total, start = by_piece ? 0 : kStart;
  int at = blockIdx.x * step;
  if (at >= all) return;
  const int end = at + step < all ? at + step : all;
  int seq = 0, before = 0;
  for (int s0 = 0; s0 < S; s0 += 64) {
    if (S > 64) look(s0);
    const int upto = sum_wave(units_of(mw.tiles) * mw.items);
    const int n = __popcll(__builtin_amdgcn_ballot_w64(before + upto <= at));      // lanes past the last sequence add nothing
    if (n < 64) {
      seq = s0 + n;
      if (n > 0) before += __builtin_amdgcn_readlane(upto, n - 1);
      break;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
    seq = s0 + 64;
  }
  if (entries != 0) {
#pragma unroll
    for (int i = 0; i < kShortTable / 256; ++i) short_table[threadIdx.x + 256 * i] = brought[i];
    __syncthreads();
  }
  const int looked = S > 64 ? seq & ~63 : 0;                       // the lanes hold the 64 sequences from here on

  const HalfLane<BITS> hl = half_lane<BITS>(lane, shift);
  const uint32_t head_bytes = (uint32_t)(2 * R::kRow) << shift;    // K and V of a head of a page
  const uint64_t page_bytes = (uint64_t)head_bytes * (uint32_t)a.pool.heads;
  while (at < end && seq < S) {
    PagedSeq sq;
    if (seq - looked < 64) {
      sq.first = __builtin_amdgcn_readlane(mine.first, seq - looked);
      sq.rows = __builtin_amdgcn_readlane(mine.rows, seq - looked);
      sq.past = __builtin_amdgcn_readlane(mine.past, seq - looked);
    } else {
      sq = paged_seq_of(a.seqs, seq);
    }
    const SeqWork w = seq_work(a, sq);
    const int units = units_of(w.tiles);
    if (at >= before + units * w.items) {                          // (a sequence without rows has no tiles)
      before += units * w.items;
      ++seq;
      continue;
    }
    const int item = (int)((uint32_t)(at - before) / (uint32_t)units);
    const int begin = before + item * units, done = begin + units;       // the block's units among all
    const int b = (int)((uint32_t)item / (uint32_t)a.pool.heads), kv = item - b * a.pool.heads;
    const int u0 = at - begin, u1 = (end < done ? end : done) - begin;
    if (u1 <= start) return;                                       // (a run that ends in a block's start: the next one begins it)
    int t0 = u0 > start ? u0 - start : 0, t1 = u1 - start;
    if (by_piece) {                                                // (one piece: u1 = u0 + 1)
      const int each = (int)((uint32_t)w.tiles / (uint32_t)units), longer = w.tiles - each * units;
      t0 = each * u0 + (u0 < longer ? u0 : longer);
      t1 = t0 + each + (u0 < longer ? 1 : 0);
    }

    const int row0 = sq.first + b * a.positions;
    const int rows = sq.rows - b * a.positions < a.positions ? sq.rows - b * a.positions : a.positions;
    const int cols = rows * a.group;
    const int pos = (col * a.by_group) >> 16, g = col - pos * a.group;
    const int64_t most = (int64_t)a.seqs.table_pages << shift, length = (int64_t)sq.past + sq.rows;
    const int len = (int)(length < most ? length : most);
    // the last key that the lane's position sees, and that the block's first one does
    auto sees = [&](int i) __attribute__((always_inline)) {
      const int64_t key = (int64_t)sq.past + b * a.positions + i;
      return (int)(key < len ? key : len - 1);
    };
    const int lim = sees(pos), all_see = sees(0);
    const bool later = all_see < len - 1;                          // rows that some column does not see
    const int* const table = a.seqs.table + (int64_t)seq * a.seqs.table_pages;
    const char* const of_head = a.pool.pages + (uint64_t)head_bytes * (uint32_t)kv;
    const char* const scales_of_head = (const char*)a.pool.scales + ((uint64_t)(uint32_t)kv << (shift + 3));

    // the wavefront's tiles are t0 + wave, t0 + wave + 4, ..; the pages of the next 32 of them, 64 halves, are looked up at once
    const int n = t1 - t0 > wave ? (t1 - t0 - wave + 3) >> 2 : 0;
    auto half_row = [&](int h) __attribute__((always_inline)) { return (t0 + wave + 4 * (h >> 1)) * kTile + 16 * (h & 1); };
    auto pages_from = [&](int h) __attribute__((always_inline)) {
      const int row = half_row(h + lane);
      if (h + lane >= 2 * n || row >= len) return -1;
      return entries != 0 ? short_table[seq * a.seqs.table_pages + (row >> shift)] : table[row >> shift];
    };
    int pages = pages_from(0), pages_next = 0, base = 0;

    // Q^T: the lane's column, channels 32 kk + 8 g4 .. (8-bit rows: 32 g4 + 8 kk ..); columns without a row are zeros
    bf16x8 qf[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (col < cols)
        raw = *(const uint4*)(a.q + ((int64_t)(kv * a.group + g) * a.seqs.n_rows + row0 + pos) * kHeadDim + (BITS == 16 ? 32 * kk + 8 * g4 : 32 * g4 + 8 * kk));
      qf[kk] = __builtin_bit_cast(bf16x8, raw);
    }

    auto page_of = [&](int h) __attribute__((always_inline)) {
      return h - base < 64 ? __builtin_amdgcn_readlane(pages, h - base) : __builtin_amdgcn_readlane(pages_next, h - base - 64);
    };
    auto there = [&](int page) __attribute__((always_inline)) { return (uint32_t)page < (uint32_t)a.pool.n_pages; };
    // Both halves of tile j.  A half that is not there is the first row of the other one, and counts for nothing; if neither is,
    // the first page's (nothing of the tile is used).
    auto issue = [&](int j, int slot) __attribute__((always_inline)) {
      const int p0 = page_of(2 * j), p1 = page_of(2 * j + 1), ok0 = there(p0), ok1 = there(p1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool own = h == 0 ? ok0 || !ok1 : ok1 || !ok0, ok = h == 0 ? ok0 : ok1;
        const int row = half_row(2 * j + (own ? h : 1 - h)), in = row & (page_rows - 1);
        const uint32_t page = own ? (ok ? (h == 0 ? p0 : p1) : 0) : (h == 0 ? p1 : p0);
        const int last = ok ? len - 1 - row : 0;
        const char* const k = of_head + page_bytes * page + in * R::kRow;
        const char* const sc = scales_of_head + ((uint64_t)((uint32_t)a.pool.heads << (shift + 3))) * page + in * 4;
        issue_half<BITS>(k, k + (R::kRow << shift), sc, last, ring + (slot + h) * R::kSlot, lane, hl, shift);
      }
    };
    constexpr int kAhead = R::kSlots / 2 - 1;                      // tiles under way besides the one that is waited for
    for (int j = 0; j < kAhead; ++j)
      if (j < n) issue(j, 2 * j);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) asm volatile("" : "+v"(qf[kk]));      // (waited for here, not inside the loop)

    RowState st;
    st.m = kNegBig;
    st.l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) st.o[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
    int slot = 0, ahead = 2 * kAhead;
    for (int j = 0; j < n; ++j) {
      if (2 * j - base == 64 - 2 * kAhead) pages_next = pages_from(base + 64);       // before the first look-up beyond the 64
      if (2 * j - base == 64) {
        pages = pages_next;
        base += 64;
      }
      if (j + kAhead < n) issue(j + kAhead, ahead);
      wait_halves<R::kLoads, 2 * kAhead>(2 * (n - 1 - j));
      const int row = half_row(2 * j);
      const bool ok0 = there(page_of(2 * j)), ok1 = there(page_of(2 * j + 1));
      if (ok0 || ok1) {
        lds_char* const halves[2] = {(lds_char*)(uintptr_t)(ring + slot * R::kSlot), (lds_char*)(uintptr_t)(ring + (slot + 1) * R::kSlot)};
        const int lims[2] = {ok0 ? lim - row : -1, ok1 ? lim - row - 16 : -1};
        attend_tile<BITS>(halves, lane, qf, st, a.c, row + kTile - 1 > all_see || !ok0 || !ok1, later, lims);
      }
      asm volatile("" ::: "memory");
      slot = slot + 2 < R::kSlots ? slot + 2 : 0;
      ahead = ahead + 2 < R::kSlots ? ahead + 2 : 0;
    }
    st.l = over_rows16(st.l, op_add);

    __syncthreads();                                               // the rings are idle
    if (col < cols) {
      float* const to = red + wave * kPiece + col * kPartialFloats;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int db = 0; db < 8; db += 2) {
          if constexpr (BITS == 16) {
            to[16 * db + 4 * g4 + r] = st.o[db][r];
            to[16 * (db + 1) + 4 * g4 + r] = st.o[db + 1][r];
          } else {
            *(float2*)(to + 8 * (4 * g4 + r) + db) = make_float2(st.o[db][r], st.o[db + 1][r]);
          }
        }
      if (g4 == 0) *(float2*)(to + kHeadDim) = make_float2(st.m, st.l);
    }
    __syncthreads();
    // What LDS holds, to the output or to a piece; and whether it was the last of `want` to arrive.
    auto put = [&](float* piece) __attribute__((always_inline)) {
      for (int i = threadIdx.x; i < cols * 64; i += 256) {
        float m, l;
        const float2 o = merge_waves(red, i >> 6, 2 * (i & 63), a.c, m, l);
        if (piece == nullptr) {
          write_out(a, kv, row0, i >> 6, 2 * (i & 63), o, l);
        } else {
          float* const to = piece + (i >> 6) * kPartialFloats;
          store_shared2(to + 2 * (i & 63), o.x, o.y);
          if ((i & 63) == 0) store_shared2(to + kHeadDim, m, l);
        }
      }
    };
    // Pieces are written and read by device-scope accesses that no L2 keeps a copy of, so the wait for the stores, the barrier and the
    // count order them; a release or acquire of everything else would walk the whole L2 (1000 rows of 8 heads: 21 us instead of 13).
    auto last_of = [&](int* count, int want) __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (threadIdx.x == 0) {
        arrived = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
        if (arrived == want) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      return arrived == want;
    };
    if (t0 == 0 && t1 == w.tiles) {
      put(nullptr);
    } else {
      const int first = (begin + start) / step, last = (done - 1) / step, me = blockIdx.x;
      auto piece_of = [&](int p) __attribute__((always_inline)) { return a.pieces + (int64_t)(2 * p + (p == first)) * kPiece; };
      const int most_at_once = fan_of(cols), fan = (me - first) / most_at_once, lead = first + fan * most_at_once;
      const int n_fan = last - lead + 1 < most_at_once ? last - lead + 1 : most_at_once, fans = (last - first) / most_at_once + 1;
      put(piece_of(me));
      // (of a run in which one block ends and another begins, each has a count of its own)
      if (last_of(a.arrivals + (fan == 0 ? 0 : kPagedRuns) + lead, n_fan)) {
        gather_pieces(n_fan, [&](int p) __attribute__((always_inline)) { return piece_of(lead + p); }, cols, red, a.c, lane, wave);
        __syncthreads();
        put(fans == 1 ? nullptr : piece_of(lead));
        if (fans > 1 && last_of(a.arrivals + 2 * kPagedRuns + first, fans)) {
          gather_pieces(fans, [&](int p) __attribute__((always_inline)) { return piece_of(first + p * most_at_once); }, cols, red, a.c, lane, wave);
          __syncthreads();
          put(nullptr);
        }
      }
    }
    __syncthreads();                                               // LDS is free for the next block
    at = begin + u1;
  }
}
static_assert(kPagedRuns <= 16 * 16, "two levels of merges");

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
