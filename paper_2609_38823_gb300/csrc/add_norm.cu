// Residual addition, RMSNorm with a weight and an 8-bit output with one scale per
// row: the step in front of the projections and of the MoE layer of a decode
// layer (base-model steps that the method leaves unchanged).
#include <cuda_fp8.h>

#include <type_traits>

#include "decomoe_internal.cuh"

namespace decomoe {

constexpr float AN_TINY = 7.888609052210118e-31f;  // 2^-100, the least row maximum that a scale is made for
constexpr float AN_MAX = 448.f;                    // largest e4m3 value
constexpr int AN_NV = 8;                           // 16-byte vectors of a row per lane, at most

struct AddNormArgs {
  const uint4 *x, *res, *w;
  uint4 *sum, *y;
  uint8_t* y8;
  float* scale;
  int64_t T;
  int vec, d;
  float eps;
};

template <bool BF16>
struct NormVec {
  static constexpr int E = BF16 ? 8 : 4;
  float v[E];
};
template <bool BF16>
__device__ __forceinline__ NormVec<BF16> unpack_vec(const uint4& u) {
  const uint32_t a[4] = {u.x, u.y, u.z, u.w};
  NormVec<BF16> r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      r.v[2 * i] = bf16_lo(a[i]);
      r.v[2 * i + 1] = bf16_hi(a[i]);
    } else {
      r.v[i] = __uint_as_float(a[i]);
    }
  }
  return r;
}
template <bool BF16>
__device__ __forceinline__ uint4 pack_vec(const NormVec<BF16>& r) {
  if constexpr (BF16)
    return make_uint4(pack_bf16x2(r.v[0], r.v[1]), pack_bf16x2(r.v[2], r.v[3]), pack_bf16x2(r.v[4], r.v[5]),
                      pack_bf16x2(r.v[6], r.v[7]));
  else
    return make_uint4(__float_as_uint(r.v[0]), __float_as_uint(r.v[1]), __float_as_uint(r.v[2]),
                      __float_as_uint(r.v[3]));
}
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

// One block of 32 W threads per row. Both reductions of a row go together: the
// sum of squares and the largest |s w|, since the row's factor 1 / rms scales
// every |s w| alike. The maximum is taken over the bits of |s w| as integers, in
// which a NaN is larger than everything and so reaches the scale.
template <bool BF16>
__global__ void __launch_bounds__(512) k_add_rmsnorm(AddNormArgs a) {
  __shared__ float red_s[16];
  __shared__ uint32_t red_m[16];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    auto load = [&](int c) {
      NormVec<BF16> s = unpack_vec<BF16>(a.x[t * a.vec + c]);
      if (a.res != nullptr) {
        const NormVec<BF16> r = unpack_vec<BF16>(a.res[t * a.vec + c]);
#pragma unroll
        for (int i = 0; i < s.E; ++i) s.v[i] += r.v[i];
      }
      return s;
    };
    auto weight = [&](int c) {
      if (a.w != nullptr) return unpack_vec<BF16>(a.w[c]);
      NormVec<BF16> w;
#pragma unroll
      for (int i = 0; i < w.E; ++i) w.v[i] = 1.f;
      return w;
    };
    float ss = 0.f;
    uint32_t mx = 0;
    for (int c = threadIdx.x; c < a.vec; c += blockDim.x) {
      const NormVec<BF16> s = load(c), w = weight(c);
#pragma unroll
      for (int i = 0; i < s.E; ++i) {
        ss = fmaf(s.v[i], s.v[i], ss);
        mx = max(mx, __float_as_uint(s.v[i] * w.v[i]) & 0x7fffffffu);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    mx = __reduce_max_sync(0xffffffffu, mx);
    if (lane == 0) {
      red_s[warp] = ss;
      red_m[warp] = mx;
    }
    __syncthreads();
    ss = 0.f;
    for (int i = 0; i < warps; ++i) {
      ss += red_s[i];
      mx = max(mx, red_m[i]);
    }
    __syncthreads();
    const float inv = rsqrtf(ss / static_cast<float>(a.d) + a.eps);
    float m = __uint_as_float(mx) * inv;
    m = m < AN_TINY ? AN_TINY : m;
    const float q = AN_MAX / m;
    for (int c = threadIdx.x; c < a.vec; c += blockDim.x) {
      const NormVec<BF16> s = load(c), w = weight(c);
      NormVec<BF16> v;
#pragma unroll
      for (int i = 0; i < s.E; ++i) v.v[i] = s.v[i] * inv * w.v[i];
      if (a.sum != nullptr) a.sum[t * a.vec + c] = pack_vec<BF16>(s);
      if (a.y != nullptr) a.y[t * a.vec + c] = pack_vec<BF16>(v);
      if (a.y8 != nullptr) {
#pragma unroll
        for (int i = 0; i < s.E; i += 4)
          *reinterpret_cast<uint32_t*>(a.y8 + t * a.d + c * s.E + i) =
              pack_e4m3x4(v.v[i] * q, v.v[i + 1] * q, v.v[i + 2] * q, v.v[i + 3] * q);
      }
    }
    if (a.scale != nullptr && threadIdx.x == 0) a.scale[t] = m / AN_MAX;
  }
}

}  // namespace decomoe

using namespace decomoe;

extern "C" int decomoe_add_rmsnorm_q8(const void* x, const void* residual, const void* weight, int64_t T, int d,
                                      float eps, int dtype, void* sum_out, void* y, void* y8, float* y8_scale,
                                      decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(T >= 0 && d > 0 && eps >= 0.f, "add_rmsnorm_q8: bad sizes");
  DM_ARG_CHECK(dtype == DECOMOE_BF16 || dtype == DECOMOE_F32, "add_rmsnorm_q8: bad dtype");
  if (T == 0) return DECOMOE_OK;
  DM_ARG_CHECK(x && (sum_out || y || y8), "add_rmsnorm_q8: null pointer");
  DM_ARG_CHECK((y8 == nullptr) == (y8_scale == nullptr), "add_rmsnorm_q8: y8 and y8_scale go together");
  DM_ARG_CHECK(sum_out == nullptr || sum_out != y, "add_rmsnorm_q8: sum_out is y");
  const int64_t row_bytes = static_cast<int64_t>(d) * static_cast<int64_t>(dtype_bytes(dtype));
  DM_ARG_CHECK(row_bytes % 16 == 0 && aligned16(x) && aligned16(residual) && aligned16(weight) && aligned16(sum_out) &&
                   aligned16(y) && (reinterpret_cast<uintptr_t>(y8) & 7u) == 0,
               "add_rmsnorm_q8: rows must be 16-byte multiples, pointers aligned");
  AddNormArgs a = {};
  a.x = static_cast<const uint4*>(x);
  a.res = static_cast<const uint4*>(residual);
  a.w = static_cast<const uint4*>(weight);
  a.sum = static_cast<uint4*>(sum_out);
  a.y = static_cast<uint4*>(y);
  a.y8 = static_cast<uint8_t*>(y8);
  a.scale = y8_scale;
  a.T = T;
  a.vec = static_cast<int>(row_bytes / 16);
  a.d = d;
  a.eps = eps;
  const int threads = std::min(512, (a.vec + 31) / 32 * 32);
  const int grid = static_cast<int>(std::min<int64_t>(T, static_cast<int64_t>(sm_count()) * 8));
  DM_CUDA_CHECK(launch_pdl(dtype == DECOMOE_BF16 ? k_add_rmsnorm<true> : k_add_rmsnorm<false>, dim3(grid), dim3(threads),
                           0, reinterpret_cast<cudaStream_t>(stream), a));
  return DECOMOE_OK;
}
