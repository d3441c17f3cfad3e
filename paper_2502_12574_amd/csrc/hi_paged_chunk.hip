// Attention of a chunk of new rows of each of many sequences over a pool of cache pages: the matrix rate is the bound.
// 4001 rows of 32 + 8 heads behind 28639: 1850 to 1950 us from box to box, 1.03 to 1.08 PFLOP/s at the clock that the power limit leaves
// (about 1.96 GHz; the matrix pipe is busy 52 % of the time and the vector pipe as long); 8-bit pages 2130 to 2270.
//
// Work.  A block is 128 rows of one sequence and one KV head: 128 / group consecutive positions with the query heads of that KV head,
// so that its rows share the keys.  It sweeps its sequence's keys in tiles of 64; a workgroup takes a block, or, where long blocks alone
// would not fill the chip, one of the equal pieces into which all blocks of the sequence are cut.  Pieces are merged by the workgroups that
// finish last (a launch of its own for that was 3 us dearer where nothing is cut, and nearly as much where few are).  Every workgroup
// works the cut out from the lengths themselves, so a captured launch follows them.  KV heads change fastest in the numbering, then
// blocks, deep ones first: with 8 heads each XCD sweeps one of them, and the workgroups that sweep the same tiles at the same time find
// them in its L2.  (Runs of equal numbers of tiles, as for few rows, would lose that.)
//
// A wavefront holds 32 rows.  S^T = K Q^T (32x32x16 tiles) leaves a row in one lane column: its running maximum and sum are per lane,
// and the weights, rounded to bf16, are the B operand of O^T += V^T P^T as they lie.  bf16 tiles go to LDS by direct loads; rows of
// 8 bits pass through registers, where they become bf16 (exactly) once for the whole workgroup, and their scales multiply scores
// and weights in fp32 (that of a K row in the operation that takes the reference off its scores: it is brought along times c).  Two
// workgroups a compute unit hide each other's softmax.
#include "hi_paged_attn.h"

namespace hi {

namespace {

constexpr int kRows = 128;                       // rows of a block
constexpr int kTileRows = 64;
constexpr int kTileBytes = kTileRows * kRowBytes;   // 16 KiB of K (or V), bf16
constexpr int kStageBytes = 2 * kTileBytes;
constexpr int kScalesAt = 2 * kStageBytes;       // [stage][K|V][64] fp32, then 64 ones
constexpr int kOnesAt = kScalesAt + 2 * 2 * kTileRows * 4;
constexpr float kSumLimit = 4096.f;
template <int BITS> constexpr int kLds = BITS == 8 ? kOnesAt + kTileRows * 4 : kScalesAt;

typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
typedef __attribute__((address_space(3))) float lds_float;

__device__ u32x4 zero_rows[16 * kRowBytes / 16];  // what the rows of a page that is not there hold

// LDS chunk (16 bytes) c of tile row r lies at position c ^ swz: operand reads are free of bank conflicts
__device__ __forceinline__ int swz_k(int row) { return row & 15; }
__device__ __forceinline__ int swz_v(int row) { return ((row & 3) << 2) | (row & 2); }

__device__ __forceinline__ float both_halves(float x, bool max) {      // with the value of lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
  return max ? fmaxf(a, b) : a + b;
}

struct State {
  f32x16 o[4];
  float m, l;
};

struct Lane {
  uint32_t koff[8];  // K operand of contraction step kk (rows 32 .. 63: 8192 further on)
  uint32_t voff[4];  // V^T operand of dims 32 db .. (8 rows on: 2048, 16 rows on: 4096)
};
__device__ __forceinline__ Lane lane_offsets(int lane) {
  Lane lc;
  const int hl = lane >> 5, col = lane & 31, s16 = lane & 15, row = 4 * hl + (s16 >> 2);
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) lc.koff[kk] = (uint32_t)(col * kRowBytes + (((2 * kk + hl) ^ swz_k(col)) << 4));
#pragma unroll
  for (int db = 0; db < 4; ++db)
    lc.voff[db] = (uint32_t)(row * kRowBytes + (((4 * db + 2 * (col >> 4) + ((s16 & 3) >> 1)) ^ swz_v(row)) << 4) + ((s16 & 1) << 3));
  return lc;
}

// 16 e4m3 values as bf16
__device__ __forceinline__ void widen(u32x4 b, u32x4& lo, u32x4& hi) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[i], 1.0f, false));
    const uint32_t y = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[i], 1.0f, true));
    if (i < 2) { lo[2 * i] = x; lo[2 * i + 1] = y; }
    else { hi[2 * i - 4] = x; hi[2 * i - 3] = y; }
  }
}

// A sequence's share: tiles of its deepest block, blocks of a head.
struct SeqBlocks { int tiles, blocks; };
__device__ __forceinline__ SeqBlocks seq_blocks(const PagedAttnArgs& a, const PagedSeq& q) {
  const int64_t len = (int64_t)q.past + q.rows, most = (int64_t)a.seqs.table_pages << a.pool.shift;
  return {(int)(((len < most ? len : most) + kTileRows - 1) / kTileRows), (int)((uint32_t)(q.rows + a.positions - 1) / (uint32_t)a.positions)};
}
__device__ __forceinline__ int pieces_of(int tiles, uint32_t piece) { return (int)((tiles + piece - 1) / piece); }

// What a workgroup does: its block, and the tiles [t0, t1) of it; pieces of the block, the block's first image and the distance of the
// next piece's (number: the workgroup's).
struct ChunkWork { int seq, kv, row0, rows, tiles, t0, t1, sees, len, pieces, piece, image, next_image; bool any; };
// The tiles of a piece: whole blocks, or pieces of an even share of the tiles of all blocks over one round of workgroups, an eighth or a
// quarter more of it (an even share often leaves a few pieces for a round of their own), or over two rounds.  A workgroup costs 6 tiles
// to begin and to end, merges 3 and one for every 70 pieces, and a round ends with its longest piece unless the short ones that
// follow fill its gaps.  0: there is nothing to do.
// (Merges at 6 whatever the pieces: 8 x 512 rows behind 2000 97 us instead of 84.6.)
// 384 rows behind 8000, 96 blocks of 131 tiles: 89 us with even shares (576 pieces), 79 with an eighth more (480).
__device__ __forceinline__ uint32_t chunk_piece(const PagedAttnArgs& a, int lane) {
  const int S = a.seqs.n_seqs;
  float tiles = 0.f, blocks = 0.f, total = 0.f, longest = 0.f;     // (as near as is needed)
  auto look = [&](int s0) __attribute__((always_inline)) {
    const SeqBlocks b = seq_blocks(a, s0 + lane < S ? paged_seq_of(a.seqs, s0 + lane) : PagedSeq{0, 0, 0});
    tiles = b.blocks > 0 ? (float)b.tiles : 0.f;
    blocks = (float)b.blocks * (float)a.pool.heads;
  };
  for (int s0 = 0; s0 < S; s0 += 64) {
    look(s0);
    total += over_wave(tiles * blocks, op_add);
    longest = fmaxf(longest, over_wave(tiles, op_max));
  }
  if (!(total >= 1.f) || total > 1.01f * kPagedMostTiles) return 0;                 // (sequences that overlap could overflow the count)
  float best = longest, least = 0.f;
  const float share = total * (1.f / kPagedSlots);
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    constexpr float kShares[6] = {0.f, 1.f, 1.125f, 1.25f, 0.5f, 0.5625f};
    const float size = i == 0 ? longest : fmaxf(ceilf(share * kShares[i]), 4.f);
    if (i > 0 && size >= longest) continue;
    const float by_size = __builtin_amdgcn_rcpf(size);
    float n = 0.f;
    for (int s0 = 0; s0 < S; s0 += 64) {
      if (S > 64) look(s0);
      n += over_wave(ceilf(tiles * by_size - 1e-3f) * blocks, op_add);
    }
    const float rounds = ceilf(n * (1.f / kPagedSlots)) * (size + 6.f), filled = (total + 6.f * n) * (1.f / kPagedSlots) + size;
    const float cost = fminf(rounds, filled) + (i == 0 ? 0.f : 3.f + n * (1.f / 70.f));
    if (i == 0 || cost < least) {
      least = cost;
      best = size;
    }
  }
  const uint32_t piece = __builtin_amdgcn_readfirstlane((uint32_t)best);
  // (sequences that overlap could have more pieces than there are workgroups: a merge would wait for the next call)
  uint32_t pieces = 0;
  for (int s0 = 0; s0 < S; s0 += 64) {
    if (S > 64) look(s0);
    pieces += __builtin_amdgcn_readlane(sum_wave((int)blocks * pieces_of((int)tiles, piece)), 63);
  }
  return pieces <= gridDim.x ? piece : 0;
}

__device__ __forceinline__ ChunkWork chunk_work(const PagedAttnArgs& a, uint32_t piece, int number, int lane) {
  ChunkWork w;
  w.any = false;
  if (piece == 0) return w;
  const int S = a.seqs.n_seqs, H = a.pool.heads;
  PagedSeq q = {0, 0, 0};
  SeqBlocks sb = {0, 0};
  auto look = [&](int s0) __attribute__((always_inline)) {
    q = s0 + lane < S ? paged_seq_of(a.seqs, s0 + lane) : PagedSeq{0, 0, 0};
    sb = seq_blocks(a, q);
  };
  // the sequence that has the number; images: those of the sequences before it
  int before = 0, images = 0, seq = 0, n_blocks = 0, k = 1;
  for (int s0 = 0; s0 < S; s0 += 64) {
    look(s0);
    const int cut = pieces_of(sb.tiles, piece), here = sb.blocks * H * cut, kept = cut > 1 ? sb.blocks * H * cut : 0;
    const int upto = sum_wave(here), images_upto = sum_wave(kept);
    const int n = __popcll(__builtin_amdgcn_ballot_w64(before + upto <= number));
    if (n < 64) {
      seq = s0 + n;
      if (n > 0) {
        before += __builtin_amdgcn_readlane(upto, n - 1);
        images += __builtin_amdgcn_readlane(images_upto, n - 1);
      }
      w.kv = __builtin_amdgcn_readlane(q.first, n);              // (for now)
      w.rows = __builtin_amdgcn_readlane(q.rows, n);
      w.sees = __builtin_amdgcn_readlane(q.past, n);
      w.tiles = __builtin_amdgcn_readlane(sb.tiles, n);
      n_blocks = __builtin_amdgcn_readlane(sb.blocks, n);
      k = __builtin_amdgcn_readlane(cut, n);
      break;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
    images += __builtin_amdgcn_readlane(images_upto, 63);
    seq = S;
  }
  if (seq >= S) return w;
  const int first = w.kv, rows = w.rows, past = w.sees;
  const uint32_t in = number - before, of_all = in / (uint32_t)H;
  w.seq = seq;
  w.kv = (int)(in - of_all * H);
  w.piece = (int)(of_all / (uint32_t)n_blocks);
  const int nth = (int)of_all - w.piece * n_blocks, b = n_blocks - 1 - nth;      // the deepest first
  w.next_image = n_blocks * H;
  w.image = images + nth * H + w.kv;
  w.row0 = first + b * a.positions;
  w.rows = rows - b * a.positions < a.positions ? rows - b * a.positions : a.positions;
  const int64_t most = (int64_t)a.seqs.table_pages << a.pool.shift, all = (int64_t)past + rows;
  w.len = (int)(all < most ? all : most);
  const int64_t sees = (int64_t)past + b * a.positions, deepest = sees + w.rows;
  w.sees = (int)(sees < w.len ? sees : w.len - 1);                               // the last key of the block's first position
  w.tiles = (int)(((deepest < w.len ? deepest : w.len) + kTileRows - 1) / kTileRows);
  // the pieces are equal; a block of fewer tiles than pieces has that many
  k = k < w.tiles ? k : w.tiles;
  const int each = (int)((uint32_t)w.tiles / (uint32_t)k), longer = w.tiles - each * k;
  w.pieces = k;
  w.t0 = each * w.piece + (w.piece < longer ? w.piece : longer);
  w.t1 = w.t0 + each + (w.piece < longer ? 1 : 0);
  w.any = w.piece < k;
  return w;
}

// The lane's row: position row / group of the block, query head row % group of the KV head.
struct LaneRow { int pos, g; bool live; };
__device__ __forceinline__ LaneRow lane_row(const PagedAttnArgs& a, const ChunkWork& w, int row) {
  LaneRow r;
  r.pos = (row * a.by_group) >> 16;
  r.g = row - r.pos * a.group;
  r.live = r.pos < w.rows;
  return r;
}

__device__ __forceinline__ void write_row(const PagedAttnArgs& a, const ChunkWork& w, const LaneRow& r, int db, int hl, const f32x16& o, float inv) {
  uint16_t* const to = a.out + ((int64_t)(w.kv * a.group + r.g) * a.seqs.n_rows + w.row0 + r.pos) * kHeadDim;
#pragma unroll
  for (int rq = 0; rq < 4; ++rq)
    *(uint2*)(to + 32 * db + 8 * rq + 4 * hl) = make_uint2(pack_bf16(o[4 * rq] * inv, o[4 * rq + 1] * inv), pack_bf16(o[4 * rq + 2] * inv, o[4 * rq + 3] * inv));
}

template <int BITS>
__global__ __launch_bounds__(256, 2) void paged_chunk_kernel(PagedAttnArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds_raw[kLds<BITS>];
  __shared__ int notes[2][4], arrived;
  lds_char* const lds = (lds_char*)lds_raw;
  const int lane = lane_id(), wave = wave_id(), hl = lane >> 5, col = lane & 31;
  const ChunkWork w = chunk_work(a, chunk_piece(a, lane), blockIdx.x, lane);
  if (!w.any) return;
  const int n = w.t1 - w.t0;
  const int* const table = a.seqs.table + (int64_t)w.seq * a.seqs.table_pages;
  const int in_page = (1 << a.pool.shift) - 1;
  auto there = [&](int page) __attribute__((always_inline)) { return page >= 0 && page < a.pool.n_pages; };

  // the wavefront brings rows 16 wave .. 16 wave + 15 of every tile, which lie in one page; the pages of 64 tiles are looked up at once
  auto group_row = [&](int j) __attribute__((always_inline)) { return (w.t0 + j) * kTileRows + 16 * wave; };
  auto pages_from = [&](int j) __attribute__((always_inline)) {
    const int row = group_row(j + lane);
    return j + lane < n && row < w.len ? table[row >> a.pool.shift] : -1;
  };
  // what the piece begins with is asked for at once: the pages of its first tiles, of the search for holes, queries (then the first tile)
  int pages = pages_from(0);
  const int first_page = w.t0 * kTileRows >> a.pool.shift, last_page = ((w.t1 * kTileRows < w.len ? w.t1 * kTileRows : w.len) - 1) >> a.pool.shift;
  const int first_pages = table[first_page + lane < last_page ? first_page + lane : last_page];
  const LaneRow mine = lane_row(a, w, 32 * wave + col);
  bf16x8 qf[8];
  {
    const uint16_t* const q = a.q + ((int64_t)(w.kv * a.group + mine.g) * a.seqs.n_rows + w.row0 + mine.pos) * kHeadDim + 8 * hl;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      uint4 raw = make_uint4(0, 0, 0, 0);
      if (mine.live) raw = *(const uint4*)(q + 16 * kk);
      qf[kk] = __builtin_bit_cast(bf16x8, raw);
    }
  }
  auto page_of = [&](int j) __attribute__((always_inline)) {
    if (j > 0 && (j & 63) == 0) pages = pages_from(j);
    return __builtin_amdgcn_readlane(pages, j & 63);
  };

  u32x4 k_lo = {0, 0, 0, 0}, k_hi = k_lo, v_lo = k_lo, v_hi = k_lo;      // 8-bit rows on their way
  float row_scale = 0.f;
  bool staged = false;
  const uint32_t lds_wave = (uint32_t)(uintptr_t)lds + wave * 4096;
  // bf16 rows: load i brings rows 4 i .. 4 i + 3 of the 16, its offset's i KiB as an immediate (which moves the place in LDS along)
  uint32_t k_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_off[i] = (uint32_t)((lane >> 4) * kRowBytes + (((lane & 15) ^ swz_k(4 * i + (lane >> 4))) << 4));
  const uint32_t v_off = (uint32_t)((lane >> 4) * kRowBytes + (((lane & 15) ^ swz_v(lane >> 4)) << 4));
  auto fetch = [&](int j, int stage) __attribute__((always_inline)) {
    const int page = page_of(j), row = group_row(j), last = w.len - 1 - row;     // rows past the end re-read the last one
    const bool ok = there(page);
    const int64_t at = paged_row(a.pool, ok ? page : 0, w.kv, row & in_page);
    if constexpr (BITS == 16) {
      const char* const k = ok ? a.pool.pages + at * kRowBytes : (const char*)zero_rows;
      const char* const v = ok ? k + ((int64_t)kRowBytes << a.pool.shift) : (const char*)zero_rows;
      const uint32_t to = lds_wave + stage * kStageBytes;
      if (!ok || last >= 15) {
        g2lds16_s<0>(k, k_off[0], to);
        g2lds16_s<1024>(k, k_off[1], to);
        g2lds16_s<2048>(k, k_off[2], to);
        g2lds16_s<3072>(k, k_off[3], to);
        g2lds16_s<0>(v, v_off, to + kTileBytes);
        g2lds16_s<1024>(v, v_off, to + kTileBytes);
        g2lds16_s<2048>(v, v_off, to + kTileBytes);
        g2lds16_s<3072>(v, v_off, to + kTileBytes);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * i + (lane >> 4), p = lane & 15, from = r < last ? r : last;
          g2lds16_s<0>(k, (uint32_t)(from * kRowBytes + ((p ^ swz_k(r)) << 4)), to + i * 1024);
          g2lds16_s<0>(v, (uint32_t)(from * kRowBytes + ((p ^ swz_v(r)) << 4)), to + kTileBytes + i * 1024);
        }
      }
    } else {
      // (of a page that is not there: the first page's, which count for nothing and are made zeros on their way to LDS)
      const char* const k = a.pool.pages + at * kHeadDim;
      const char* const v = k + ((int64_t)kHeadDim << a.pool.shift);
      const int r0 = lane >> 3, r1 = r0 + 8, clip = ok ? last : 15, r = lane & 15;
      const uint32_t at0 = (r0 < clip ? r0 : clip) * kHeadDim + 16 * (lane & 7), at1 = (r1 < clip ? r1 : clip) * kHeadDim + 16 * (lane & 7);
      k_lo = *(const u32x4*)(k + at0);
      k_hi = *(const u32x4*)(k + at1);
      v_lo = *(const u32x4*)(v + at0);
      v_hi = *(const u32x4*)(v + at1);
      row_scale = a.pool.scales[at + (r < clip ? r : clip) + (lane & 16 ? in_page + 1 : 0)];
      staged = ok;
    }
  };
  auto settle = [&](int stage) __attribute__((always_inline)) {        // 8-bit rows into LDS, as bf16
    if constexpr (BITS == 8) {
      lds_char* const to = lds + stage * kStageBytes + wave * 4096;
      const int r0 = lane >> 3, p = lane & 7;
      const uint32_t ka = r0 * kRowBytes + (((2 * p) ^ swz_k(r0)) << 4), va = kTileBytes + r0 * kRowBytes + (((2 * p) ^ swz_v(r0)) << 4);
      if (!staged) {
        k_lo = k_hi = v_lo = v_hi = (u32x4){0, 0, 0, 0};
        row_scale = 0.f;
      }
      // (8 rows on, the swizzle of a K row changes by 8, that of a V row not at all; the second chunk's lies 1 apart)
      auto put = [&](uint32_t off, const u32x4& b) __attribute__((always_inline)) {
        u32x4 lo, hi;
        widen(b, lo, hi);
        *(lds_u32x4*)(to + off) = lo;
        *(lds_u32x4*)(to + (off ^ 16)) = hi;
      };
      put(ka, k_lo);
      put((ka ^ 128) + 8 * kRowBytes, k_hi);
      put(va, v_lo);
      put(va + 8 * kRowBytes, v_hi);
      if (lane < 32) *(lds_float*)(lds + kScalesAt + ((stage * 2 + (lane >> 4)) * kTileRows + 16 * wave + (lane & 15)) * 4) = lane < 16 ? row_scale * a.c : row_scale;
    }
  };
  // Values that are not finite in a tile of keys that some rows of the block see and others don't: each wavefront looks at the rows that it
  // brought before the barrier that begins the tile, and notes it for all (of two tiles in turn, and for good: what it costs is time).
  auto look = [&](int stage) __attribute__((always_inline)) {
    lds_char* const at = lds + stage * kStageBytes + kTileBytes + wave * 4096 + lane * 16;
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 v = *(lds_u32x4*)(at + i * 1024);
#pragma unroll
      for (int e = 0; e < 4; ++e) bad |= not_finite(v[e]);
    }
    bool any = (bad & 0x80008000u) != 0;
    if (BITS == 8) any |= !(fabsf(*(lds_float*)(lds + kScalesAt + ((stage * 2 + 1) * kTileRows + 16 * wave + (lane & 15)) * 4)) < __builtin_inff());
    if (__builtin_amdgcn_ballot_w64(any) != 0 && lane == 0) notes[stage][wave] = 1;
  };
  auto noted = [&](int stage) __attribute__((always_inline)) {
    return __builtin_amdgcn_readfirstlane(notes[stage][0] | notes[stage][1] | notes[stage][2] | notes[stage][3]) != 0;
  };
  auto clean = [&](int stage) __attribute__((always_inline)) {          // zeros in their place, once all wavefronts know them
    __syncthreads();
    lds_char* const at = lds + stage * kStageBytes + kTileBytes + wave * 4096 + lane * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) *(lds_bf16x8*)(at + i * 1024) = two_parts(*(lds_bf16x8*)(at + i * 1024)).finite;
    __syncthreads();
  };
  if (lane == 0) notes[0][wave] = notes[1][wave] = 0;
  fetch(0, 0);
  if (BITS == 8 && threadIdx.x < kTileRows) *(lds_float*)(lds + kOnesAt + threadIdx.x * 4) = 1.f;
  const float unit = BITS == 8 ? 1.f : a.c;      // what scores and maxima are multiplied by before the power of two

  // rows that a piece's tiles lack because their page is not there: looked for once
  bool holes = __builtin_amdgcn_ballot_w64(!there(first_pages)) != 0;
  for (int p = first_page + 64; p <= last_page; p += 64) holes |= __builtin_amdgcn_ballot_w64(!there(table[p + lane < last_page ? p + lane : last_page])) != 0;

  const int lim = w.sees + mine.pos < w.len ? w.sees + mine.pos : w.len - 1;     // the last key the lane's row sees
  const bool works = 32 * wave < w.rows * a.group;
  const Lane lc = lane_offsets(lane);
  State st;
  st.m = kNegBig;
  st.l = 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) st.o[db][r] = 0.f;
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(qf[kk]));
  settle(0);

  for (int j = 0; j < n; ++j) {
    const int stage = j & 1, key0 = (w.t0 + j) * kTileRows;
    if constexpr (BITS == 16) wait_vmcnt<0>();
    const bool hides = key0 + kTileRows - 1 > w.sees;
    if (hides) look(stage);
    __syncthreads();
    if (j + 1 < n) fetch(j + 1, 1 - stage);
    lds_char* const kt = lds + stage * kStageBytes;
    lds_char* const vt = kt + kTileBytes;
    if (!works) {                                // (no row of the wavefront's is a row of the block)
      if (hides && noted(stage)) clean(stage);
      if (j + 1 < n) settle(1 - stage);
      continue;
    }

    // register r of sub-block sb: the lane's row against key 32 sb + 8 (r / 4) + 4 hl + r % 4 of the tile.  Operands are read four
    // ahead of the products that take them: left to itself the compiler reads each where it is needed, and the products wait for LDS.
    constexpr int A = 4;
    bf16x8 op[A + 1];
    f32x16 s[2];
    auto read_k = [&](int i) __attribute__((always_inline)) { op[i % (A + 1)] = *(lds_bf16x8*)(kt + lc.koff[i >> 1] + (i & 1) * 8192); };
    auto v_operand = [&](int i) __attribute__((always_inline)) {
      lds_char* const p = vt + lc.voff[i & 3] + (i >> 2) * 4096;
      const bf16x4 v0 = lds_read_tr8(p), v1 = lds_read_tr8(p + 2048);
      return (bf16x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto read_v = [&](int i) __attribute__((always_inline)) { op[i % (A + 1)] = v_operand(i); };
#pragma unroll
    for (int r = 0; r < 16; ++r) { s[0][r] = 0.f; s[1][r] = 0.f; }
#pragma unroll
    for (int i = 0; i < A; ++i) read_k(i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i + A < 16) read_k(i + A);
      s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i % (A + 1)], qf[i >> 1], s[i & 1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    lds_char* const sc = lds + kScalesAt + stage * 2 * kTileRows * 4 + 16 * hl;
    lds_char* by_key = sc;                       // what the scores are still to be multiplied by
    if (hides || holes) {
      if constexpr (BITS == 8) {
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const f32x4 f = *(lds_f32x4*)(sc + (32 * sb + 8 * q4) * 4);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[sb][4 * q4 + r] *= f[r];
          }
        by_key = lds + kOnesAt + 16 * hl;
      }
      uint64_t shown = lim - key0 >= 63 ? ~0ull : lim < key0 ? 0ull : (2ull << (lim - key0)) - 1;
      if (holes) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = key0 + 16 * i;
          if (row < w.len && !there(table[row >> a.pool.shift])) shown &= ~(0xFFFFull << (16 * i));
        }
      }
      shown >>= 4 * hl;
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const uint32_t t = (uint32_t)__builtin_amdgcn_sbfe((int)(uint32_t)(shown >> (32 * sb)), 8 * (r >> 2) + (r & 3), 1);
          s[sb][r] = __uint_as_float((__float_as_uint(s[sb][r]) & t) | (__float_as_uint(kNegBig) & ~t));
        }
    }
    // The weights, rounded to bf16 for the matrix pipe; their sum is that of the fp32 values.  They are relative to a reference that
    // follows the row's maximum only when it must: the lane's sum bounds each of them, and while it stays below the limit they are as
    // harmless in fp32 and bf16 as weights up to 1.  Otherwise, and where a row has seen nothing yet, the maximum is taken.
    u32x4 pw[2][2];
    auto weights = [&](float mc) __attribute__((always_inline)) {
      float lq[4];
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float p[8];
          if constexpr (BITS == 8) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const f32x4 f = *(lds_f32x4*)(by_key + (32 * sb + 16 * u + 8 * h) * 4);
#pragma unroll
              for (int r = 0; r < 4; ++r) p[4 * h + r] = fast_exp2(__builtin_fmaf(s[sb][8 * u + 4 * h + r], f[r], -mc));
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = fast_exp2(__builtin_fmaf(s[sb][8 * u + e], a.c, -mc));
          }
          lq[2 * sb + u] = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
          if constexpr (BITS == 8) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const f32x4 f = *(lds_f32x4*)(sc + (kTileRows + 32 * sb + 16 * u + 8 * h) * 4);
#pragma unroll
              for (int r = 0; r < 4; ++r) p[4 * h + r] *= f[r];
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) pw[sb][u][e] = pack_bf16(p[2 * e], p[2 * e + 1]);
          if (BITS == 8) __builtin_amdgcn_sched_barrier(0);      // (or all scales would be read at once, into registers that are not there)
        }
      return (lq[0] + lq[1]) + (lq[2] + lq[3]);
    };
    if constexpr (BITS == 16) {
#pragma unroll
      for (int i = 0; i < A; ++i) read_v(i);
      __builtin_amdgcn_sched_barrier(0);
    }
    float sum = weights(st.m > kNegBig ? st.m * unit : 0.f);
    if (__builtin_amdgcn_ballot_w64(!(sum <= kSumLimit) || st.m == kNegBig) != 0) {       // also true for NaN
      float mx = kNegBig;
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          f32x4 f = {1.f, 1.f, 1.f, 1.f};
          if constexpr (BITS == 8) f = *(lds_f32x4*)(by_key + (32 * sb + 8 * q4) * 4);
#pragma unroll
          for (int r = 0; r < 4; ++r) mx = fmaxf(mx, BITS == 8 ? s[sb][4 * q4 + r] * f[r] : s[sb][4 * q4 + r]);
        }
      const float m_new = fmaxf(st.m, both_halves(mx, true)), alpha = fast_exp2((st.m - m_new) * unit);
      st.l *= alpha;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.o[db][r] *= alpha;
      st.m = m_new;
      sum = weights(st.m > kNegBig ? st.m * unit : 0.f);           // (a row that has seen nothing yet adds weights of zero)
    }
    st.l += sum;
    __builtin_amdgcn_sched_barrier(0);
    uint32_t marks[2] = {0, 0};                  // bit 16 (db % 2) + r of db / 2: NaN belongs there
    if (hides && noted(stage)) {
      const uint64_t shown = (lim - key0 >= 63 ? ~0ull : lim < key0 ? 0ull : (2ull << (lim - key0)) - 1) >> (4 * hl);
      const uint32_t upto[2] = {(uint32_t)shown, (uint32_t)(shown >> 32)};
      auto mask_of = [&](int i, int e) __attribute__((always_inline)) {      // of the two keys of a word of the weights
        const uint32_t two = upto[i >> 1] >> (16 * (i & 1) + 8 * (e >> 1) + 2 * (e & 1));
        return (two & 1) * 0xFFFFu | (two & 2) * 0x7FFF8000u;
      };
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        f32x16 hit;
#pragma unroll
        for (int r = 0; r < 16; ++r) hit[r] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x4 seen;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            seen[e] = 0x3F803F80u & mask_of(i, e);
            if (BITS == 8 && db == 0) pw[i >> 1][i & 1][e] &= mask_of(i, e);       // (a scale that is not finite)
          }
          hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(two_parts(v_operand(4 * i + db)).others, __builtin_bit_cast(bf16x8, seen), hit, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) marks[db >> 1] |= (hit[r] > 0.f ? 1u : 0u) << (16 * (db & 1) + r);
      }
      clean(stage);
      if (BITS == 16) {
#pragma unroll
        for (int i = 0; i < A; ++i) read_v(i);
      }
    }
    if constexpr (BITS == 8) {
#pragma unroll
      for (int i = 0; i < A; ++i) read_v(i);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i + A < 16) read_v(i + A);
      st.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i % (A + 1)], __builtin_bit_cast(bf16x8, pw[i >> 3][(i >> 2) & 1]), st.o[i & 3], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (__builtin_amdgcn_ballot_w64((marks[0] | marks[1]) != 0) != 0) {
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) st.o[db][r] = marks[db >> 1] >> (16 * (db & 1) + r) & 1 ? __builtin_nanf("") : st.o[db][r];
    }
    if (j + 1 < n) settle(1 - stage);
  }

  float m = st.m, l = both_halves(st.l, false);
  if (w.pieces > 1) {
    // The block's pieces are merged eight at a time, by the workgroup that finishes last of the eight, then eight of those; in the pieces'
    // order, whoever it is.  An image's numbers are written and read by accesses that no L2 keeps a copy of (the wait for the stores, the
    // barrier and the count order them).
    float* const images = a.images + (int64_t)w.image * kPagedImageFloats + 2 * threadIdx.x;
    const int64_t next = (int64_t)w.next_image * kPagedImageFloats;
    auto keep = [&](int p) __attribute__((always_inline)) {
      float* const to = images + p * next;
#pragma unroll
      for (int i = 0; i < 32; ++i) store_shared2(to + i * 512, st.o[i >> 3][2 * (i & 7)], st.o[i >> 3][2 * (i & 7) + 1]);
      store_shared2(to + 32 * 512, m, l);
    };
    if (works) keep(w.piece);
    for (int level = 0, lead = w.piece;; ++level) {
      const int shift = kPagedFan * level, first = lead >> (shift + kPagedFan) << (shift + kPagedFan);
      const int there = ((w.pieces - first - 1) >> shift) + 1, of = there < (1 << kPagedFan) ? there : 1 << kPagedFan;
      const bool all = w.pieces <= 1 << (shift + kPagedFan);
      lead = first;
      if (of > 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
          int* const count = a.counts + level * kPagedMostImages + w.image + first * w.next_image;
          arrived = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
          if (arrived == of) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (arrived != of) return;
        if (works) {
          const float* const from = images + first * next;
          const int64_t step = next << shift;
          float2 ml[1 << kPagedFan];
          m = kNegBig;
#pragma unroll
          for (int i = 0; i < 1 << kPagedFan; ++i) ml[i] = i < of ? load_shared2(from + i * step + 32 * 512) : make_float2(kNegBig, 0.f);
#pragma unroll
          for (int i = 0; i < 1 << kPagedFan; ++i) m = fmaxf(m, ml[i].x);
          l = 0.f;
#pragma unroll
          for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) st.o[db][r] = 0.f;
          float2 x[2][32];                       // an image, and the next one under way
          auto bring = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 32; ++e) x[i & 1][e] = load_shared2(from + i * step + e * 512);
            __builtin_amdgcn_sched_barrier(0);
          };
          bring(0);
#pragma unroll
          for (int i = 0; i < 1 << kPagedFan; ++i) {
            if (i >= of) break;
            if (i + 1 < of) bring(i + 1);
            const float f = fast_exp2((ml[i].x - m) * unit);
            l += f * ml[i].y;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              st.o[e >> 3][2 * (e & 7)] += f * x[i & 1][e].x;
              st.o[e >> 3][2 * (e & 7) + 1] += f * x[i & 1][e].y;
            }
          }
        }
      }
      if (all) break;
      if (works && of > 1) keep(lead);
    }
  }
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  if (works && mine.live) {
#pragma unroll
    for (int db = 0; db < 4; ++db) write_row(a, w, mine, db, hl, st.o[db], inv);
  }
}

}  // namespace

// units: at least as many as there are blocks; a block that is cut has at most a piece more than its share of the 2 x 512, and the whole
// pieces of all are no more than those
hi_status launch_paged_chunk(void* stream, const PagedAttnArgs& a, int64_t units) {
  const dim3 grid((unsigned)(units + 2 * kPagedSlots));
  if (a.pool.bits == 16) hipLaunchKernelGGL(paged_chunk_kernel<16>, grid, dim3(256), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(paged_chunk_kernel<8>, grid, dim3(256), 0, (hipStream_t)stream, a);
  return launched("paged attention");
}

}  // namespace hi
