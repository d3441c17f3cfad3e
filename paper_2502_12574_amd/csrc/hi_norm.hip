// The residual's addition and the root-mean-square norm between the blocks of a layer: h = x + r, r' = h, y = h / sqrt(mean(h^2) + eps) w.
// One pass over the data: a row stays in registers between the sum of its squares and its outputs, so every input is read once
// and every output written once; bound by HBM (8191 rows of 4096, fp32 residual: 74.5 us, 5.4 TB/s, where a large copy has 4.85) or by the
// launch and two latencies of memory (one row of 4096: 2.6 us).
#include "hi_device.h"
#include "hi_serve.h"

namespace hi {

namespace {

constexpr int kNormMaxD = 16384;

// 8 consecutive values of a row; the pieces of a row are dealt to the lanes one by one, so that a wavefront reads whole lines
template <bool FP32>
__device__ __forceinline__ void norm_load(const void* at, int64_t i, float (&v)[8]) {
  if (FP32) {
    const float4 a = *(const float4*)((const float*)at + i), b = *(const float4*)((const float*)at + i + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    const u32x4 w = *(const u32x4*)((const uint16_t*)at + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
}
template <bool FP32>
__device__ __forceinline__ void norm_store(void* at, int64_t i, const float (&v)[8]) {
  if (FP32) {
    *(float4*)((float*)at + i) = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)((float*)at + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *(u32x4*)((uint16_t*)at + i) = (u32x4){pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
  }
}

struct NormArgs {
  const void* x; const void* res; const uint16_t* w;
  void* res_out; uint16_t* out;
  int rows, d;
  float eps;
};

// LANES lanes a row, N pieces of 8 values a lane (LANES * N >= d / 8).
template <bool XF, bool RF, int LANES, int N>
__global__ __launch_bounds__(256) void add_rmsnorm_kernel(NormArgs a) {
  constexpr int kRows = 256 / LANES;
  const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRows + sub;
  const bool live = row < a.rows;
  const int64_t base = (live ? row : a.rows - 1) * a.d;
  const int pieces = a.d / 8;
  float h[N][8];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = lane + i * LANES;
    if (p < pieces) {
      norm_load<XF>(a.x, base + 8 * p, h[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] = 0.f;
    }
  }
  if (a.res != nullptr) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = lane + i * LANES;
      if (p < pieces) {
        float r[8];
        norm_load<RF>(a.res, base + 8 * p, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] += r[j];
      }
    }
  }
  u32x4 w[N];                                    // asked for before the sum is known
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = lane + i * LANES;
    w[i] = p < pieces ? *(const u32x4*)(a.w + 8 * p) : (u32x4){0, 0, 0, 0};
  }
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float part = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) part = __builtin_fmaf(h[i][j], h[i][j], part);
    sum += part;
  }
  sum = over_wave(sum, op_add);
  if (LANES > 64) {
    __shared__ float waves[256 / 64];
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = (waves[0] + waves[1]) + (waves[2] + waves[3]);
  }
  const float unit = 1.0f / sqrtf(sum / (float)a.d + a.eps);
  if (!live) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int p = lane + i * LANES;
    if (p >= pieces) continue;
    if (a.res_out != nullptr) norm_store<RF>(a.res_out, base + 8 * p, h[i]);
    float y[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      y[2 * j] = h[i][2 * j] * unit * __uint_as_float(w[i][j] << 16);
      y[2 * j + 1] = h[i][2 * j + 1] * unit * __uint_as_float(w[i][j] & 0xFFFF0000u);
    }
    norm_store<false>(a.out, base + 8 * p, y);
  }
}

template <bool XF, bool RF>
void norm_launch(hipStream_t s, const NormArgs& a) {
  const int pieces = a.d / 8;
  // a dimension of a grid has at most 2^32 lanes
  auto grid = [&](int rows) {
    const int64_t n = ceil_div(a.rows, rows), x = n < (1 << 22) ? n : 1 << 22;
    return dim3((unsigned)x, (unsigned)ceil_div(n, x));
  };
  // rows of up to 2048 values take a wavefront each and no barrier, longer ones a workgroup
#define HI_NORM(LANES, N)                                                                                                   \
  if (pieces <= LANES * N) {                                                                                                \
    hipLaunchKernelGGL((add_rmsnorm_kernel<XF, RF, LANES, N>), grid(256 / LANES), dim3(256), 0, s, a);                      \
    return;                                                                                                                 \
  }
  HI_NORM(64, 1) HI_NORM(64, 2) HI_NORM(64, 4) HI_NORM(256, 2) HI_NORM(256, 3) HI_NORM(256, 4) HI_NORM(256, 6) HI_NORM(256, 8)
#undef HI_NORM
}

}  // namespace

}  // namespace hi

using namespace hi;

extern "C" hi_status hi_add_rmsnorm(void* stream, const void* x_dev, int32_t x_fp32, const void* residual_dev,
                                    int32_t residual_fp32, const void* weight_dev, int32_t n_rows, int32_t d, float eps,
                                    void* residual_out_dev, void* out_dev) {
  if (!aligned_to(x_dev, 16) || !aligned_to(residual_dev, 16) || !aligned_to(weight_dev, 16) || !aligned_to(residual_out_dev, 16) ||
      !aligned_to(out_dev, 16)) {
    set_last_error("norm: buffers must be 16-byte aligned");
    return HI_ERR_ARG;
  }
  if (n_rows < 0 || d < 1 || (x_fp32 != 0 && x_fp32 != 1) || (residual_fp32 != 0 && residual_fp32 != 1) || !(eps >= 0.0f) || eps > 3.0e38f) {
    set_last_error("norm: bad shape or eps");
    return HI_ERR_ARG;
  }
  if (d % 8 != 0 || d > kNormMaxD) {
    set_last_error("norm: rows must be a multiple of 8 values and at most %d long", kNormMaxD);
    return HI_ERR_UNSUPPORTED;
  }
  if (n_rows == 0) return HI_OK;                 // (whose buffers may be null)
  if (!x_dev || !weight_dev || !out_dev) { set_last_error("norm: null buffer"); return HI_ERR_ARG; }
  if (x_fp32 && x_dev == out_dev) { set_last_error("norm: an fp32 x cannot be the bf16 output"); return HI_ERR_ARG; }
  if (out_dev == residual_dev || out_dev == residual_out_dev) { set_last_error("norm: the output cannot be the residual"); return HI_ERR_ARG; }
  StreamDevice on(stream);
  const NormArgs a = {x_dev, residual_dev, (const uint16_t*)weight_dev, residual_out_dev, (uint16_t*)out_dev, n_rows, d, eps};
  const hipStream_t s = (hipStream_t)stream;
  if (x_fp32) {
    if (residual_fp32) norm_launch<true, true>(s, a);
    else norm_launch<true, false>(s, a);
  } else {
    if (residual_fp32) norm_launch<false, true>(s, a);
    else norm_launch<false, false>(s, a);
  }
  return launched("norm");
}
