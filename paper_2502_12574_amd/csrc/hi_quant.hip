// Products with weights of 4 bits: W^ [n_out][n_in] = zero + code * scale, a scale and a zero for each 128 input channels of a row.
#include <mutex>
#include <type_traits>
#include "hi_device.h"
#include "hi_serve.h"

namespace hi {

namespace {

constexpr int kQGroup = 128;                    // input channels of a scale
constexpr int kQMostIn = 1 << 20;               // 64 rows of x, or 16 of codes, within 32 bits of bytes
constexpr int kQMostOut = 1 << 24;              // (a launch has at most 2^32 lanes)

// ---- bf16 weights to codes: a wavefront takes 16 groups at a time, 4 lanes a group with 32 channels each.  The weights are read
// once and a quarter of them written; run once per matrix (8192 x 8192: 30 us, 5.7 TB/s).
__global__ __launch_bounds__(256) void weight_quant_kernel(const uint16_t* __restrict__ w, int64_t groups, char* __restrict__ codes,
                                                           uint16_t* __restrict__ scales, uint16_t* __restrict__ zeros) {
  const int64_t at = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 2);
  const bool live = at < groups;
  const int64_t g = live ? at : groups - 1;
  const int part = threadIdx.x & 3;
  const uint16_t* const src = w + g * kQGroup + part * 32;
  float x[32];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const u32x4 v = *(const u32x4*)(src + 8 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[8 * i + 2 * j] = __uint_as_float(v[j] << 16);
      x[8 * i + 2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u);
    }
  }
  float mn = x[0], mx = x[0];
#pragma unroll
  for (int i = 1; i < 32; ++i) {
    mn = fminf(mn, x[i]);
    mx = fmaxf(mx, x[i]);
  }
#pragma unroll
  for (int off = 1; off < 4; off *= 2) {
    mn = fminf(mn, __shfl_xor(mn, off));
    mx = fmaxf(mx, __shfl_xor(mx, off));
  }
  const float s32 = __fmul_rn(__fsub_rn(mx, mn), __fdiv_rn(1.0f, 15.0f));
  uint32_t sbits = float_to_bf16_bits(s32);
  float scale = bf16_bits_to_float((uint16_t)sbits);
  if (!(scale >= 0x1p-120f)) {
    scale = 0.f;
    sbits = 0;
  }
  const float inv = scale > 0.f ? __fdiv_rn(1.0f, scale) : 0.f;
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float t = __fmul_rn(__fsub_rn(x[8 * i + j], mn), inv);
      word |= (uint32_t)fminf(rintf(t), 15.0f) << (4 * j);
    }
    out[i] = word;
  }
  if (!live) return;
  *(u32x4*)(codes + g * (kQGroup / 2) + part * 16) = out;
  if (part == 0) {
    scales[g] = (uint16_t)sbits;
    zeros[g] = float_to_bf16_bits(mn);
  }
}

struct LinearArgs {
  const uint16_t* x; const char* codes; const uint16_t* scales; const uint16_t* zeros; uint16_t* y;
  int rows, n_in, n_out, x_heads, y_heads;
};

// A code c becomes the bf16 number 16 + c: 16 .. 31 is an exponent and the code in the upper bits of the fraction.  So with s and z a
// group's scale and zero, and exactly in all but the fp32 sums,
//   sum_k W^_k x_k = s sum_k (16 + c_k) x_k + (z - 16 s) sum_k x_k   over the group's 128 channels:
// no weight is rounded, and scale and zero enter once a group instead of once a weight.
// A byte holds two codes, which belong 12 bits further apart: a product with 2^3 + 2^15 puts both where they have to be, among others
// that the mask takes out.  Two operations for two codes (with shifts, too, but those pair codes that are 4 channels apart, and x had
// to be brought into that order).  The constants are kept in registers: such an instruction cannot carry them.
struct CodeBits {
  uint32_t spread = 0x8008u, mask = 0x00780078u, one = 0x41804180u;
  __device__ __forceinline__ CodeBits() { asm("" : "+v"(spread), "+s"(mask), "+v"(one)); }
};
template <int BYTE>
__device__ __forceinline__ uint32_t codes_pair(uint32_t w, const CodeBits& c) {
  static_assert(BYTE >= 0 && BYTE < 4, "a byte of a word");
  uint32_t x;
  if constexpr (BYTE == 0) asm("v_mul_u32_u24_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0 src1_sel:DWORD" : "=v"(x) : "v"(w), "v"(c.spread));
  else if constexpr (BYTE == 1) asm("v_mul_u32_u24_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1 src1_sel:DWORD" : "=v"(x) : "v"(w), "v"(c.spread));
  else if constexpr (BYTE == 2) asm("v_mul_u32_u24_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2 src1_sel:DWORD" : "=v"(x) : "v"(w), "v"(c.spread));
  else asm("v_mul_u32_u24_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3 src1_sel:DWORD" : "=v"(x) : "v"(w), "v"(c.spread));
  return (x & c.mask) | c.one;
}
__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t w, const CodeBits& c) {
  return __builtin_bit_cast(bf16x8, (u32x4){codes_pair<0>(w, c), codes_pair<1>(w, c), codes_pair<2>(w, c), codes_pair<3>(w, c)});
}
__device__ __forceinline__ bf16x8 bf16_ones() { return __builtin_bit_cast(bf16x8, (u32x4){0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}); }

// the row's 128 channels of group g
__device__ __forceinline__ const uint16_t* x_group(const LinearArgs& a, int row, int g) {
  return a.x + (a.x_heads ? ((int64_t)g * a.rows + row) * kQGroup : (int64_t)row * a.n_in + (int64_t)g * kQGroup);
}
__device__ __forceinline__ uint16_t* y_at(const LinearArgs& a, int row, int n) {
  return a.y + (a.y_heads ? ((int64_t)(n >> 7) * a.rows + row) * kHeadDim + (n & 127) : (int64_t)row * a.n_out + n);
}

// ---- up to 64 rows: the read of the weights is the bound.  A workgroup takes 16 NT outputs and all rows (4 RX of them); its W
// wavefronts take turns of U consecutive groups each and add their sums through LDS.  Codes and x come through a private LDS ring of S
// groups a wavefront, by direct loads: as the matrix tiles want them, 16 neighbouring lanes would touch 16 rows, and the look-up of
// their lines, not the bytes, would be the bound (16 rows of 4096 x 6144: 13.0 us with loads into registers).  One row 5.6 us (2.4 TB/s:
// a chain of launch, ring and join), 29 rows of 8192 x 8192 13.5 us (2.7 TB/s: the feed of the rings).  Sums of x come
// out of the matrix pipe too, against ones.
// A workgroup begins its turns where its number says: the rows of codes lie a power of two apart, and workgroups that all began at
// the first channel would keep to a few memory channels.
template <int RX, int NT, int U, int W, int S>
struct Few {
  static constexpr int kTiles = RX < 4 ? 1 : RX / 4, kLoads = RX + NT, kStage = kLoads * 1024;
  static constexpr int kRing = W * S * kStage, kSums = W * kTiles * NT * 1024, kLds = kRing > kSums ? kRing : kSums;
  static constexpr int kPerSimd = kLds <= 80 * 1024 ? W / 2 : W / 4;          // wavefronts on a SIMD, by LDS
};

template <int RX, int NT, int U, int W, int S>
__global__ __launch_bounds__(64 * W, (Few<RX, NT, U, W, S>::kPerSimd)) void linear_few_kernel(LinearArgs a) {
  using F = Few<RX, NT, U, W, S>;
  constexpr int RT = F::kTiles;
  static_assert((S - 1) * F::kLoads < 64 && F::kLds <= 160 * 1024, "ring");
  extern __shared__ __attribute__((aligned(1024))) char lds_raw[];
  const int lane = lane_id(), wave = wave_id(), c16 = lane & 15, g4 = lane >> 4;
  const int n0 = blockIdx.x * 16 * NT, row0 = blockIdx.y * 4 * RX, groups = a.n_in / kQGroup;
  const int turns = (groups + U - 1) / U, begin = blockIdx.x % turns;
  const uint32_t ring = (uint32_t)(uintptr_t)(lds_char*)lds_raw + wave * (S * F::kStage);

  // a load of codes: 4 lanes an output, 16 outputs (chunk p of output r of the tile is chunk p ^ (r / 4) of its 64 bytes)
  const int cr = lane >> 2;
  const uint32_t code_off = (uint32_t)cr * (uint32_t)(a.n_in / 2) + ((((uint32_t)lane & 3) ^ ((uint32_t)cr >> 2)) << 4);
  const char* codes[NT];
  const uint16_t *sp[NT], *zp[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int n = n0 + 16 * t < a.n_out ? n0 + 16 * t : n0;           // (a tile of outputs is there or not)
    codes[t] = a.codes + (int64_t)n * (a.n_in / 2);
    sp[t] = a.scales + (int64_t)(n + c16) * groups;
    zp[t] = a.zeros + (int64_t)(n + c16) * groups;
  }
  // a load of x: 16 lanes a row, 4 rows (chunk p of row r is chunk p ^ (r % 16) of its 256 bytes)
  uint32_t x_off[RX];
  const uint32_t pitch = a.x_heads ? 2 * kQGroup : 2u * a.n_in;
#pragma unroll
  for (int i = 0; i < RX; ++i) {
    const int r = 4 * i + (lane >> 4), to = row0 + r < a.rows ? r : a.rows - 1 - row0;
    x_off[i] = (uint32_t)to * pitch + (uint32_t)(((lane & 15) ^ (r & 15)) << 4);
  }
  const char* const x0 = (const char*)a.x + (int64_t)row0 * pitch;
  const int64_t x_group_bytes = a.x_heads ? (int64_t)a.rows * (2 * kQGroup) : 2 * kQGroup;

  const int mine = turns > wave ? (turns - wave + W - 1) / W : 0;     // turns of this wavefront: wave, wave + W, ..
  auto first_group = [&](int i) __attribute__((always_inline)) {
    const int turn = wave + W * i + begin;
    return (turn < turns ? turn : turn - turns) * U;
  };
  auto issue = [&](int step, int stage) __attribute__((always_inline)) {      // step: turn and group of it, one after the other
    int g = first_group(step / U) + step % U;
    g = g < groups ? g : groups - 1;                                  // (of a turn that is cut short: loaded, and not used)
    const uint32_t to = ring + stage * F::kStage;
#pragma unroll
    for (int t = 0; t < NT; ++t) g2lds16_s<0>(codes[t] + (int64_t)g * (kQGroup / 2), code_off, to + t * 1024);
#pragma unroll
    for (int i = 0; i < RX; ++i) g2lds16_s<0>(x0 + g * x_group_bytes, x_off[i], to + (NT + i) * 1024);
  };
  struct Scales { uint16_t s[NT][U], z[NT][U]; };
  auto load_scales = [&](Scales& b, int g) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (g + U <= groups) {                     // (2-byte aligned: the hardware takes it in one piece all the same)
        __builtin_memcpy(b.s[t], sp[t] + g, 2 * U);
        __builtin_memcpy(b.z[t], zp[t] + g, 2 * U);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          b.s[t][u] = g + u < groups ? sp[t][g + u] : 0;
          b.z[t][u] = g + u < groups ? zp[t][g + u] : 0;
        }
      }
    }
  };
  Scales now, next;
  if (mine > 0) load_scales(now, first_group(0));
  for (int i = 0; i < S - 1; ++i)
    if (i < mine * U) issue(i, i);

  uint32_t x_at[4];                              // operand reads: row c16 of a tile, channels 32 g4 + 8 k ..
  const int rr = RX < 4 ? c16 & (4 * RX - 1) : c16;
#pragma unroll
  for (int k = 0; k < 4; ++k) x_at[k] = (uint32_t)(NT * 1024 + rr * 256 + (((4 * g4 + k) ^ rr) << 4));
  const uint32_t w_at = (uint32_t)(c16 * 64 + ((g4 ^ (c16 >> 2)) << 4));
  f32x4 y[RT][NT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) y[i][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
  const CodeBits bits;
  int stage = 0, ahead = S - 1;
  for (int turn = 0; turn < mine; ++turn) {
    const int g = first_group(turn);
    if (turn + 1 < mine) load_scales(next, first_group(turn + 1));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int step = turn * U + u;
      if (step + S - 1 < mine * U) {
        issue(step + S - 1, ahead);
        wait_vmcnt<(S - 1) * F::kLoads>();
      } else {
        wait_vmcnt<0>();
      }
      lds_char* const at = (lds_char*)(uintptr_t)(ring + stage * F::kStage);
      if (g + u < groups) {
        u32x4 w[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) w[t] = __builtin_bit_cast(u32x4, lds_read16(at + w_at + t * 1024));
        f32x4 acc[RT][NT], xs[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          xs[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[i][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          bf16x8 wk[NT];
#pragma unroll
          for (int t = 0; t < NT; ++t) wk[t] = codes_to_bf16(w[t][k], bits);
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            const bf16x8 x = lds_read16(at + x_at[k] + i * 4096);
            xs[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, bf16_ones(), xs[i], 0, 0, 0);
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, wk[t], acc[i][t], 0, 0, 0);
          }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float s = bf16_bits_to_float(now.s[t][u]), z = __builtin_fmaf(-16.0f, s, bf16_bits_to_float(now.z[t][u]));
#pragma unroll
          for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) y[i][t][r] = __builtin_fmaf(s, acc[i][t][r], __builtin_fmaf(z, xs[i][r], y[i][t][r]));
        }
      }
      asm volatile("" ::: "memory");
      stage = stage + 1 < S ? stage + 1 : 0;
      ahead = ahead + 1 < S ? ahead + 1 : 0;
    }
    now = next;
  }
  // register r: row 4 g4 + r of the tile, output c16
  float* const part = (float*)lds_raw;           // [wavefront][tile][16 rows][16 outputs]
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[(wave * RT * NT + i * NT + t) * 256 + (4 * g4 + r) * 16 + c16] = y[i][t][r];
  __syncthreads();
  for (int i = threadIdx.x; i < 4 * RX * NT * 8; i += 64 * W) {       // two outputs of a row each
    const int n = 2 * (i % (8 * NT)), r = i / (8 * NT), at = ((r >> 4) * NT + (n >> 4)) * 256 + (r & 15) * 16 + (n & 15);
    if (row0 + r >= a.rows || n0 + n >= a.n_out) continue;
    float2 v = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float2 x = *(const float2*)(part + w * RT * NT * 256 + at);
      v.x += x.x;
      v.y += x.y;
    }
    *(uint32_t*)y_at(a, row0 + r, n0 + n) = pack_bf16(v.x, v.y);
  }
}

// ---- more rows: the matrix rate is the bound.  A workgroup takes 32 RT rows (128; 96 where that fills the chip better) and 128 outputs, a
// group of 128 channels at a time; a wavefront takes all rows and 32 of the outputs, so that no code is expanded twice in a workgroup.
// x goes to LDS by direct loads, a step ahead, the codes into registers.  Operands are read RT ahead of the products that take them (left
// to itself the compiler reads each where it is needed, and the products wait for LDS: 4096 x 4096 and 1500 rows 101 us, with the reads
// ahead 72, in tiles of 96 rows 65).  8192 x 8192 and 4096 rows: 623 us, 880 TFLOP/s; the products and the operations that make and feed
// their operands take turns.
// The sums' part of an output, (z - 16 s) sum x, is a 32x32x16 product of its own for each group: a row's sum as three bf16 numbers
// (24 bits of it), and 16 times them, against z and -s.  Each wavefront forms the sums of 32 rows, from the operands that it reads
// anyway, for all; they are used a step later.
constexpr int kQTile = 128;                              // outputs
template <int RT>
struct Tile {
  static constexpr int kRows = 32 * RT;
  static constexpr int kStage = kRows * 256;             // x of a group
  static constexpr int kSums = 2 * kStage;               // [stage][row] 8 numbers of a row's sum, then 16 bytes of zeros
  static constexpr int kZeros = kSums + 2 * kRows * 16;
  static constexpr int kLds = kZeros + 16;
};

template <int RT>
__global__ __launch_bounds__(256, 2) void linear_tile_kernel(LinearArgs a, int row_tiles) {
  using T = Tile<RT>;
  constexpr int kQStage = T::kStage, kQSums = T::kSums, kQZeros = T::kZeros, kQLds = T::kLds, kRows = T::kRows;
  typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  __shared__ __attribute__((aligned(1024))) char lds_raw[kQLds];
  lds_char* const lds = (lds_char*)lds_raw;
  const int lane = lane_id(), wave = wave_id(), hl = lane >> 5, col = lane & 31, groups = a.n_in / kQGroup;
  // an XCD takes consecutive numbers, of which 64 run at a time: 8 row tiles and 8 of outputs
  const int per = (gridDim.x + 7) / 8, at = (blockIdx.x & 7) * per + (blockIdx.x >> 3), n_tiles = (a.n_out + kQTile - 1) / kQTile;
  const int band = at / (8 * n_tiles), in = at - band * 8 * n_tiles, high = row_tiles - 8 * band < 8 ? row_tiles - 8 * band : 8;
  if (high <= 0) return;
  const int row0 = (8 * band + in % high) * kRows, n0 = in / high * kQTile;
  if (n0 >= a.n_out) return;
  const int n = n0 + 32 * wave + col, nc = n < a.n_out ? n : a.n_out - 1;
  const char* const codes = a.codes + (int64_t)nc * (a.n_in / 2) + 32 * hl;
  const uint16_t* const sp = a.scales + (int64_t)nc * groups;
  const uint16_t* const zp = a.zeros + (int64_t)nc * groups;

  // x: the wavefront brings rows 8 RT wave .. of a tile, 4 to a load (chunk p of row r is chunk p ^ (r % 16) of its 256 bytes)
  const uint32_t pitch = a.x_heads ? 2 * kQGroup : 2u * a.n_in;
  const char* x_now = (const char*)a.x + (int64_t)row0 * pitch;
  const int64_t x_step = a.x_heads ? (int64_t)a.rows * (2 * kQGroup) : 2 * kQGroup;
  const uint32_t lds_wave = (uint32_t)(uintptr_t)lds + wave * (RT * 2048);
  uint32_t x_off[2 * RT];
#pragma unroll
  for (int i = 0; i < 2 * RT; ++i) {
    const int r = 8 * RT * wave + 4 * i + (lane >> 4);
    x_off[i] = (uint32_t)(row0 + r < a.rows ? r : a.rows - 1 - row0) * pitch + (((lane & 15) ^ (r & 15)) << 4);
  }
  struct Codes { u32x4 w[2]; uint32_t s, z; };
  auto fetch = [&](Codes& b, int g, int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i) g2lds16_s<0>(x_now, x_off[i], lds_wave + stage * kQStage + i * 1024);
    x_now += x_step;
    b.w[0] = *(const u32x4*)(codes + (int64_t)g * 64);
    b.w[1] = *(const u32x4*)(codes + (int64_t)g * 64 + 16);
    b.s = sp[g];
    b.z = zp[g];
  };
  if (threadIdx.x == 0) *(lds_u32x4*)(lds + kQZeros) = (u32x4){0, 0, 0, 0};
  // x operand j of channels 64 hl + 8 k ..: the row tiles from the wavefront's own on; bits 4 .. 6 change with k
  auto row_tile = [&](int j) __attribute__((always_inline)) { return wave + j < RT ? wave + j : (wave + j) % RT; };
  uint32_t x_at[RT], sum_at[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    x_at[j] = (uint32_t)((row_tile(j) * 32 + col) * 256 + (((8 * hl) ^ (col & 15)) << 4));
    sum_at[j] = hl ? kQZeros : kQSums + (row_tile(j) * 32 + col) * 16;
  }
  const uint32_t my_sum = kQSums + (row_tile(0) * 32 + col) * 16;      // (two wavefronts write the same sums where RT is 3)
  f32x16 y[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) y[t][r] = 0.f;
  const CodeBits bits;
  u32x4 zs = {0, 0, 0, 0};                       // the last step's z and -s
  auto add_sums = [&](int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < RT; ++j)
      y[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(lds + sum_at[j] + (hl ? 0 : stage * (kRows * 16))), __builtin_bit_cast(bf16x8, zs), y[j], 0, 0, 0);
  };
  auto step = [&](int g, auto parity, Codes& now, Codes& next) __attribute__((always_inline)) {
    constexpr int stage = decltype(parity)::value, A = RT;
    wait_vmcnt<0>();
    asm volatile("" : "+v"(now.w[0]), "+v"(now.w[1]), "+v"(now.s), "+v"(now.z));      // (they were asked for a step ago)
    __syncthreads();
    if (g + 1 < groups) fetch(next, g + 1, 1 - stage);
    lds_char* const xt = lds + stage * kQStage;
    f32x16 acc[RT];
    bf16x8 op[A + 1], b[2];
    float sum = 0.f;
    auto read = [&](int i) __attribute__((always_inline)) { op[i % (A + 1)] = lds_read16(xt + (x_at[i % RT] ^ ((i / RT) << 4))); };
#pragma unroll
    for (int i = 0; i < A; ++i) read(i);
    b[0] = codes_to_bf16(now.w[0][0], bits);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 8 * RT; ++i) {
      const int k = i / RT, j = i % RT;
      if (i + A < 8 * RT) read(i + A);
      f32x16 z;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = 0.f;
      acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i % (A + 1)], b[k & 1], k == 0 ? z : acc[j], 0, 0, 0);
      if (j == 0) {                              // the own rows' sums
        const u32x4 x = __builtin_bit_cast(u32x4, op[i % (A + 1)]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t two = x[q];             // (a vector's element itself would be cast as the vector's first)
          sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
        }
        asm volatile("" : "+v"(sum));            // here, and not where it is used: the operands would be kept until then
      }
      if (j == 1 && k < 7) b[(k + 1) & 1] = codes_to_bf16(now.w[(k + 1) >> 2][(k + 1) & 3], bits);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (g > 0) add_sums(1 - stage);              // of the step before
    const uint32_t minus_s = now.s ^ 0x8000u;
    zs = (u32x4){hl ? 0 : now.z | (now.z << 16), hl ? 0 : now.z | (minus_s << 16), hl ? 0 : minus_s | (minus_s << 16), 0u};
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    sum = __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
    const float h = bf16_bits_to_float((uint16_t)pack_bf16(sum, 0.f)), m = bf16_bits_to_float((uint16_t)pack_bf16(sum - h, 0.f)), l = sum - h - m;
    *(lds_u32x4*)(lds + my_sum + stage * (kRows * 16)) = (u32x4){pack_bf16(h, m), pack_bf16(l, 16.f * h), pack_bf16(16.f * m, 16.f * l), 0u};
    const float s = __uint_as_float(now.s << 16);
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) y[j][r] = __builtin_fmaf(s, acc[j][r], y[j][r]);
  };
  Codes even, odd;
  fetch(even, 0, 0);
  int g = 0;
  for (; g + 1 < groups; g += 2) {
    step(g, std::integral_constant<int, 0>(), even, odd);
    step(g + 1, std::integral_constant<int, 1>(), odd, even);
  }
  if (g < groups) step(g, std::integral_constant<int, 0>(), even, odd);
  __syncthreads();
  add_sums((groups - 1) & 1);
  if (n >= a.n_out) return;
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = row0 + 32 * row_tile(t) + 8 * (r >> 2) + 4 * hl + (r & 3);
      if (row < a.rows) *y_at(a, row, n) = (uint16_t)pack_bf16(y[t][r], 0.f);
    }
}

template <int RX, int NT, int U, int W, int S>
hipError_t few_go(hipStream_t s, const LinearArgs& a) {
  using F = Few<RX, NT, U, W, S>;
  static std::once_flag once;
  static hipError_t attr = hipSuccess;
  std::call_once(once, [] { attr = hipFuncSetAttribute((const void*)linear_few_kernel<RX, NT, U, W, S>, hipFuncAttributeMaxDynamicSharedMemorySize, F::kLds); });
  if (attr != hipSuccess) return attr;
  hipLaunchKernelGGL((linear_few_kernel<RX, NT, U, W, S>), dim3((unsigned)ceil_div(a.n_out, 16 * NT), (unsigned)ceil_div(a.rows, 4 * RX)), dim3(64 * W),
                     F::kLds, s, a);
  return hipSuccess;
}
template <int RT>
hi_status tile_go(hipStream_t s, const LinearArgs& a) {
  const int64_t row_tiles = ceil_div(a.rows, 32 * RT), tiles = row_tiles * ceil_div(a.n_out, kQTile);
  if (tiles > (1 << 24) - 8) { set_last_error("quantised linear: too many rows"); return HI_ERR_RANGE; }
  hipLaunchKernelGGL(linear_tile_kernel<RT>, dim3((unsigned)(8 * ceil_div(tiles, 8))), dim3(256), 0, s, a, (int)row_tiles);
  return launched("quantised linear");
}
// turns of 4 groups, as long as each wavefront has one
template <int RX, int NT, int W, int S>
hipError_t few_turns(hipStream_t s, const LinearArgs& a) {
  const int groups = a.n_in / kQGroup;
  return groups >= 4 * W ? few_go<RX, NT, 4, W, S>(s, a) : groups >= 2 * W ? few_go<RX, NT, 2, W, S>(s, a) : few_go<RX, NT, 1, W, S>(s, a);
}

// Rows of a workgroup: 16, 32 or 64 in the kernel for few rows, 96 or 128 in the other.  Microseconds of each, from the rounds that its
// workgroups take (g: groups of channels; two workgroups of the first and of the last two fit a compute unit, one of the others), fitted
// to hidden sizes of 1024 to 8192 and 1 to 4096 rows.  Measured there, at 4096 x 4096: 64 rows 12.1 with 64 a workgroup; 256 rows 27, with
// 96 and 128 38 and 45; 512 rows 48, 40 and 47; 1024 rows 94, 56 and 50; 1500 rows, 96 and 128: 67 and 72, 2048 rows 97 and 86; at
// 8192 x 8192: 256 rows 88, 72 and 85.
int linear_form(int64_t rows, int64_t n_out, int g) {
  auto few = [&](int64_t r, int64_t outs) { return ceil_div(rows, r) * ceil_div(n_out, outs); };
  auto tiles = [&](int64_t t, double full, double half) {
    const int64_t rest = t % 512;
    const double last = rest == 0 ? 0 : rest <= 256 ? half : half + (full - half) * (0.35 + 0.65 / 256 * (double)(rest - 256));
    return 3 + ((double)(t / 512) * full + last) * g;
  };
  const int64_t w16 = few(16, 16), w32 = few(32, 32), w64 = few(64, 32);
  const int forms[5] = {16, 32, 64, 96, 128};
  const double us[5] = {1.3 + (w16 <= 256 ? 0.11 * g : (double)ceil_div(w16, 512) * 0.18 * g),
                        1.3 + (double)ceil_div(w32, 256) * (0.5 + 0.18 * g),
                        1.5 + (double)ceil_div(w64, 256) * (1.5 + 0.30 * g),
                        tiles(few(96, kQTile), 1.97, 1.12), tiles(few(128, kQTile), 2.48, 1.33)};
  int best = 4;
  for (int i = 3; i >= 0; --i)
    if (us[i] < us[best] && (i == 3 || ceil_div(rows, forms[i]) <= 65535)) best = i;       // (the second dimension of a grid ends there)
  return forms[best];
}

}  // namespace

}  // namespace hi

using namespace hi;

extern "C" hi_status hi_weight_quantize(void* stream, const void* w_dev, int32_t n_out, int32_t n_in, void* codes_dev,
                                        void* scales_dev, void* zeros_dev) {
  if (!w_dev || !codes_dev || !scales_dev || !zeros_dev) { set_last_error("weight quantise: null buffer"); return HI_ERR_ARG; }
  if (!aligned_to(w_dev, 16) || !aligned_to(codes_dev, 16) || !aligned_to(scales_dev, 2) || !aligned_to(zeros_dev, 2)) {
    set_last_error("weight quantise: weights and codes must be 16-byte aligned, scales and zeros 2-byte");
    return HI_ERR_ARG;
  }
  if (n_out < 1 || n_in < 1) { set_last_error("weight quantise: bad shape"); return HI_ERR_ARG; }
  if (n_in % kQGroup != 0) { set_last_error("weight quantise: n_in must be a multiple of %d", kQGroup); return HI_ERR_UNSUPPORTED; }
  const int64_t groups = (int64_t)n_out * (n_in / kQGroup);
  if (ceil_div(groups, 64) >= (1 << 24)) { set_last_error("weight quantise: too many weights"); return HI_ERR_RANGE; }
  StreamDevice on(stream);
  hipLaunchKernelGGL(weight_quant_kernel, dim3((unsigned)ceil_div(groups, 64)), dim3(256), 0, (hipStream_t)stream,
                     (const uint16_t*)w_dev, groups, (char*)codes_dev, (uint16_t*)scales_dev, (uint16_t*)zeros_dev);
  return launched("weight quantise");
}

extern "C" hi_status hi_linear_quantized(void* stream, const void* x_dev, const void* codes_dev, const void* scales_dev,
                                         const void* zeros_dev, int32_t n_rows, int32_t n_in, int32_t n_out, int32_t x_heads,
                                         int32_t y_heads, void* y_dev) {
  if (!aligned_to(x_dev, 16) || !aligned_to(codes_dev, 16) || !aligned_to(scales_dev, 2) || !aligned_to(zeros_dev, 2) || !aligned_to(y_dev, 16)) {
    set_last_error("quantised linear: rows and codes must be 16-byte aligned, scales and zeros 2-byte");
    return HI_ERR_ARG;
  }
  if (n_rows < 0 || n_in < 1 || n_out < 1 || (x_heads != 0 && x_heads != 1) || (y_heads != 0 && y_heads != 1)) {
    set_last_error("quantised linear: bad shape");
    return HI_ERR_ARG;
  }
  if (n_in % kQGroup != 0 || n_out % 16 != 0 || (y_heads && n_out % kHeadDim != 0)) {
    set_last_error("quantised linear: n_in must be a multiple of %d, n_out of 16, and of %d for head-major outputs", kQGroup, kHeadDim);
    return HI_ERR_UNSUPPORTED;
  }
  if (n_in > kQMostIn || n_out > kQMostOut) {
    set_last_error("quantised linear: n_in of more than %d or n_out of more than %d", kQMostIn, kQMostOut);
    return HI_ERR_UNSUPPORTED;
  }
  if (n_rows == 0) return HI_OK;                 // (whose buffers may be null)
  if (!x_dev || !codes_dev || !scales_dev || !zeros_dev || !y_dev) { set_last_error("quantised linear: null buffer"); return HI_ERR_ARG; }
  if (y_dev == x_dev) { set_last_error("quantised linear: y cannot be x"); return HI_ERR_ARG; }
  StreamDevice on(stream);
  const LinearArgs a = {(const uint16_t*)x_dev, (const char*)codes_dev, (const uint16_t*)scales_dev, (const uint16_t*)zeros_dev,
                        (uint16_t*)y_dev, n_rows, n_in, n_out, x_heads, y_heads};
  const hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (n_rows <= 4) e = few_turns<1, 1, 8, 4>(st, a);
  else if (n_rows <= 8) e = few_turns<2, 1, 8, 3>(st, a);
  else switch (linear_form(n_rows, n_out, n_in / kQGroup)) {
    case 16: e = few_turns<4, 1, 8, 2>(st, a); break;
    case 32: e = few_turns<8, 2, 8, 2>(st, a); break;
    case 64: e = few_turns<16, 2, 4, 2>(st, a); break;
    case 96: return tile_go<3>(st, a);
    default: return tile_go<4>(st, a);
  }
  if (e != hipSuccess) { set_last_error("quantised linear: %s", hipGetErrorString(e)); return HI_ERR_HIP; }
  return launched("quantised linear");
}
