// Few rows times a matrix of 4-bit weights with group scales: the projections
// around the attention of a decode layer (base-model steps that the method
// leaves unchanged).
//   out[t, n] = xs_t sum_g ws[n, g] sum_{k in group g} x[t, k] (q[n, k] - 8)
#include <cuda_fp8.h>

#include <type_traits>

#include "decomoe_internal.cuh"

namespace decomoe {

struct W4Args {
  const void* x;
  const float* xs;
  const uint8_t* w;
  const __nv_bfloat16* ws;
  void* out;
  int64_t T, N, x_stride;
  int K, group, out_f32;
};

// One warp per output column, W4_T rows at a time.
constexpr int W4_T = 8;
template <bool E4M3>
__global__ void __launch_bounds__(256) k_w4_linear(W4Args a) {
  pdl_enter();
  const int lane = threadIdx.x & 31;
  const int64_t n = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (n >= a.N) return;
  const int64_t t0 = static_cast<int64_t>(blockIdx.y) * W4_T;
  const int groups = a.K / a.group;
  float acc[W4_T] = {};
  for (int g = 0; g < groups; ++g) {
    const float s = __bfloat162float(a.ws[n * groups + g]);
    float part[W4_T] = {};
    for (int k = g * a.group + 2 * lane; k < (g + 1) * a.group; k += 64) {
      const uint32_t b = a.w[(n * a.K + k) >> 1];
      const float q0 = static_cast<float>(static_cast<int>(b & 15u) - 8);
      const float q1 = static_cast<float>(static_cast<int>(b >> 4) - 8);
#pragma unroll
      for (int i = 0; i < W4_T; ++i) {
        if (t0 + i >= a.T) break;
        const int64_t at = (t0 + i) * a.x_stride + k;
        float x0, x1;
        if constexpr (E4M3) {
          x0 = static_cast<float>(static_cast<const __nv_fp8_e4m3*>(a.x)[at]);
          x1 = static_cast<float>(static_cast<const __nv_fp8_e4m3*>(a.x)[at + 1]);
        } else {
          x0 = __bfloat162float(static_cast<const __nv_bfloat16*>(a.x)[at]);
          x1 = __bfloat162float(static_cast<const __nv_bfloat16*>(a.x)[at + 1]);
        }
        part[i] = fmaf(x1, q1, fmaf(x0, q0, part[i]));
      }
    }
#pragma unroll
    for (int i = 0; i < W4_T; ++i) acc[i] = fmaf(s, part[i], acc[i]);
  }
#pragma unroll
  for (int i = 0; i < W4_T; ++i) {
    float v = acc[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (lane == 0 && t0 + i < a.T) {
      if (a.xs != nullptr) v *= a.xs[t0 + i];
      const int64_t at = (t0 + i) * a.N + n;
      if (a.out_f32) static_cast<float*>(a.out)[at] = v;
      else static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
    }
  }
}

}  // namespace decomoe

using namespace decomoe;

extern "C" int decomoe_w4_linear(const void* x, int x_dtype, int64_t x_stride, const float* x_scale, int64_t T, int K,
                                 const void* w, const void* w_scale, int group, int64_t N, void* out, int out_dtype,
                                 decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(x_dtype == DECOMOE_BF16 || x_dtype == DECOMOE_E4M3, "w4_linear: x must be bf16 or e4m3");
  DM_ARG_CHECK(out_dtype == DECOMOE_BF16 || out_dtype == DECOMOE_F32, "w4_linear: out must be bf16 or f32");
  DM_ARG_CHECK(group == 32 || group == 64 || group == 128, "w4_linear: group must be 32, 64 or 128");
  DM_ARG_CHECK(T >= 0 && K > 0 && K % group == 0 && N >= 1 && N <= INT_MAX, "w4_linear: bad sizes (K a multiple of group)");
  DM_ARG_CHECK(T <= 65535 * W4_T, "w4_linear: T above %d", 65535 * W4_T);
  if (T == 0) return DECOMOE_OK;
  DM_ARG_CHECK(x && w && w_scale && out, "w4_linear: null pointer");
  DM_ARG_CHECK((x_dtype == DECOMOE_E4M3) == (x_scale != nullptr), "w4_linear: x_scale goes with e4m3 rows, and only with them");
  const int64_t xe = x_dtype == DECOMOE_BF16 ? 2 : 1;
  DM_ARG_CHECK(x_stride >= K && x_stride * xe % 16 == 0 && aligned16(x) && aligned16(w) &&
                   (reinterpret_cast<uintptr_t>(w_scale) & 1u) == 0 &&
                   reinterpret_cast<uintptr_t>(out) % dtype_bytes(out_dtype) == 0,
               "w4_linear: x_stride must be at least K and a multiple of 16 bytes, x and w 16-byte aligned");
  W4Args a = {};
  a.x = x;
  a.xs = x_scale;
  a.w = static_cast<const uint8_t*>(w);
  a.ws = static_cast<const __nv_bfloat16*>(w_scale);
  a.out = out;
  a.T = T;
  a.N = N;
  a.x_stride = x_stride;
  a.K = K;
  a.group = group;
  a.out_f32 = out_dtype == DECOMOE_F32;
  const dim3 grid(static_cast<unsigned>((N + 7) / 8), static_cast<unsigned>((T + W4_T - 1) / W4_T));
  DM_CUDA_CHECK(launch_pdl(x_dtype == DECOMOE_E4M3 ? k_w4_linear<true> : k_w4_linear<false>, grid, dim3(256), 0,
                           reinterpret_cast<cudaStream_t>(stream), a));
  return DECOMOE_OK;
}
