// Products with weights of 4 bits: W^ [n_out][n_in] = zero + code * scale, a scale and a zero for each 128 input channels of a row.
#include "hi_device.h"
#include "hi_serve.h"

namespace hi {

namespace {

constexpr int kQGroup = 128;                    // input channels of a scale

// ---- bf16 weights to codes: a wavefront takes 16 groups at a time, 4 lanes a group with 32 channels each.  The weights are read
// once and a quarter of them written; run once per matrix.
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

// One wavefront for an output of a row, two channels a lane at a time.
__global__ __launch_bounds__(64) void linear_simple_kernel(LinearArgs a) {
  const int n = blockIdx.x, lane = threadIdx.x, groups = a.n_in / kQGroup;
  for (int r = blockIdx.y; r < a.rows; r += gridDim.y) {
    float sum = 0.f;
    for (int g = 0; g < groups; ++g) {
      const int64_t at = a.x_heads ? ((int64_t)g * a.rows + r) * kQGroup : (int64_t)r * a.n_in + g * kQGroup;
      const uint32_t xw = *(const uint32_t*)(a.x + at + 2 * lane);
      const uint32_t c = (uint8_t)a.codes[((int64_t)n * groups + g) * (kQGroup / 2) + lane];
      const float x0 = __uint_as_float(xw << 16), x1 = __uint_as_float(xw & 0xFFFF0000u);
      const float s = bf16_bits_to_float(a.scales[(int64_t)n * groups + g]), z = bf16_bits_to_float(a.zeros[(int64_t)n * groups + g]);
      sum += s * (x0 * (float)(c & 15) + x1 * (float)(c >> 4)) + z * (x0 + x1);
    }
    sum = over_wave(sum, op_add);
    const int64_t to = a.y_heads ? ((int64_t)(n >> 7) * a.rows + r) * kHeadDim + (n & 127) : (int64_t)r * a.n_out + n;
    if (lane == 0) a.y[to] = (uint16_t)pack_bf16(sum, 0.f);
  }
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
  if (ceil_div(groups, 64) > 0x7FFFFFFF) { set_last_error("weight quantise: too many weights"); return HI_ERR_RANGE; }
  StreamDevice on(stream);
  hipLaunchKernelGGL(weight_quant_kernel, dim3((unsigned)ceil_div(groups, 64)), dim3(256), 0, (hipStream_t)stream,
                     (const uint16_t*)w_dev, groups, (char*)codes_dev, (uint16_t*)scales_dev, (uint16_t*)zeros_dev);
  return launched("weight quantise");
}

extern "C" hi_status hi_linear_quantized(void* stream, const void* x_dev, const void* codes_dev, const void* scales_dev,
                                         const void* zeros_dev, int32_t n_rows, int32_t n_in, int32_t n_out, int32_t x_heads,
                                         int32_t y_heads, void* y_dev) {
  if (!x_dev || !codes_dev || !scales_dev || !zeros_dev || !y_dev) { set_last_error("quantised linear: null buffer"); return HI_ERR_ARG; }
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
  if (n_rows == 0) return HI_OK;
  StreamDevice on(stream);
  const LinearArgs a = {(const uint16_t*)x_dev, (const char*)codes_dev, (const uint16_t*)scales_dev, (const uint16_t*)zeros_dev,
                        (uint16_t*)y_dev, n_rows, n_in, n_out, x_heads, y_heads};
  hipLaunchKernelGGL(linear_simple_kernel, dim3((unsigned)n_out, (unsigned)(n_rows < 32768 ? n_rows : 32768)), dim3(64), 0,
                     (hipStream_t)stream, a);
  return launched("quantised linear");
}
