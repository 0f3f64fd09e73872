// Residual addition, RMSNorm with a weight and an 8-bit output with one scale per
// row: the step in front of the projections and of the MoE layer of a decode
// layer (base-model steps that the method leaves unchanged).
#include <cuda_fp8.h>

#include <type_traits>

#include "decomoe_internal.cuh"

namespace decomoe {

constexpr float AN_TINY = 7.888609052210118e-31f;  // 2^-100, the least row maximum that a scale is made for
constexpr float AN_MAX = 448.f;                    // largest e4m3 value
constexpr int AN_NV = 8;                           // 16-byte vectors of a row per thread, at most
constexpr int AN_WARPS = 16;                       // warps of a row, at most

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

// A row is one block's (warps > 1) or one warp's (several rows a block, no barrier).
// Both reductions of a row go together: the sum of squares and the largest |s w|,
// since the row's factor 1 / rms scales every |s w| alike. The maximum is taken over
// the bits of |s w| as integers, in which a NaN is larger than everything and so
// reaches the scale. NV > 0: the row's sum stays in registers, NV vectors of 16 bytes
// a thread, all loads in flight together; NV = 0: longer rows, read twice.
template <bool BF16, int NV>
__global__ void __launch_bounds__(32 * AN_WARPS) k_add_rmsnorm(AddNormArgs a, int warps) {
  constexpr int E = NormVec<BF16>::E;
  constexpr int KEEP = NV > 0 ? NV : 1;
  __shared__ float red_s[2][AN_WARPS];
  __shared__ uint32_t red_m[2][AN_WARPS];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per_block = (blockDim.x >> 5) / warps;  // rows at a time: 1 where warps > 1
  const int in_row = threadIdx.x - (warp / warps) * warps * 32, step = warps * 32;
  int phase = 0;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * per_block + warp / warps; t < a.T;
       t += static_cast<int64_t>(gridDim.x) * per_block, phase ^= 1) {
    const uint4 *xr = a.x + t * a.vec, *rr = a.res != nullptr ? a.res + t * a.vec : nullptr;
    auto sum_of = [&](const uint4& x, const uint4& r) {
      NormVec<BF16> s = unpack_vec<BF16>(x);
      if (a.res != nullptr) {
        const NormVec<BF16> v = unpack_vec<BF16>(r);
#pragma unroll
        for (int i = 0; i < E; ++i) s.v[i] += v.v[i];
      }
      return s;
    };
    auto weight = [&](int c) {
      if (a.w != nullptr) return unpack_vec<BF16>(__ldg(a.w + c));
      NormVec<BF16> w;
#pragma unroll
      for (int i = 0; i < E; ++i) w.v[i] = 1.f;
      return w;
    };
    float ss = 0.f;
    uint32_t mx = 0;
    auto add = [&](const NormVec<BF16>& s, int c) {
      const NormVec<BF16> w = weight(c);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        ss = fmaf(s.v[i], s.v[i], ss);
        mx = max(mx, __float_as_uint(s.v[i] * w.v[i]) & 0x7fffffffu);
      }
    };
    NormVec<BF16> keep[KEEP];
    if constexpr (NV > 0) {
      uint4 x[KEEP], r[KEEP];
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = in_row + k * step;
        x[k] = r[k] = make_uint4(0, 0, 0, 0);
        if (c < a.vec) {
          x[k] = xr[c];
          if (rr != nullptr) r[k] = rr[c];
        }
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        keep[k] = sum_of(x[k], r[k]);
        if (in_row + k * step < a.vec) add(keep[k], in_row + k * step);
      }
    } else {
      for (int c = in_row; c < a.vec; c += step) add(sum_of(xr[c], rr != nullptr ? rr[c] : make_uint4(0, 0, 0, 0)), c);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    mx = __reduce_max_sync(0xffffffffu, mx);
    if (warps > 1) {
      // the next row's values go to the other half, so one barrier a row is enough
      if (lane == 0) {
        red_s[phase][warp] = ss;
        red_m[phase][warp] = mx;
      }
      __syncthreads();
      ss = 0.f;
      for (int i = 0; i < warps; ++i) {
        ss += red_s[phase][i];
        mx = max(mx, red_m[phase][i]);
      }
    }
    const float inv = rsqrtf(ss / static_cast<float>(a.d) + a.eps);
    float m = __uint_as_float(mx) * inv;
    m = m < AN_TINY ? AN_TINY : m;
    const float q = AN_MAX / m;
    auto put = [&](const NormVec<BF16>& s, int c) {
      const NormVec<BF16> w = weight(c);
      NormVec<BF16> v;
#pragma unroll
      for (int i = 0; i < E; ++i) v.v[i] = s.v[i] * inv * w.v[i];
      if (a.sum != nullptr) a.sum[t * a.vec + c] = pack_vec<BF16>(s);
      if (a.y != nullptr) a.y[t * a.vec + c] = pack_vec<BF16>(v);
      if (a.y8 != nullptr) {
        uint32_t b[E / 4];
#pragma unroll
        for (int i = 0; i < E; i += 4)
          b[i / 4] = pack_e4m3x4(v.v[i] * q, v.v[i + 1] * q, v.v[i + 2] * q, v.v[i + 3] * q);
        uint8_t* dst = a.y8 + t * a.d + static_cast<int64_t>(c) * E;
        if constexpr (E == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(b[0], b[1]);
        else *reinterpret_cast<uint32_t*>(dst) = b[0];
      }
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (in_row + k * step < a.vec) put(keep[k], in_row + k * step);
    } else {
      for (int c = in_row; c < a.vec; c += step) put(sum_of(xr[c], rr != nullptr ? rr[c] : make_uint4(0, 0, 0, 0)), c);
    }
    if (a.scale != nullptr && in_row == 0) a.scale[t] = m / AN_MAX;
  }
  pdl_trigger();
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
  // an output may be an input, element for element, but not lie across its rows
  const size_t all = static_cast<size_t>(T) * static_cast<size_t>(row_bytes);
  const Bytes in[] = {{x, all}, {residual, all}, {weight, static_cast<size_t>(row_bytes)}};
  const Bytes outs[] = {{sum_out, all}, {y, all}, {y8, static_cast<size_t>(T) * static_cast<size_t>(d)},
                        {y8_scale, static_cast<size_t>(T) * sizeof(float)}};
  for (int i = 0; i < 4; ++i) {
    bool apart = true;
    for (int j = 0; j < 3; ++j) apart &= !overlaps(outs[i], {in[j]}) || (i < 2 && j < 2 && outs[i].p == in[j].p);
    for (int j = 0; j < i; ++j) apart &= !overlaps(outs[i], {outs[j]});
    DM_ARG_CHECK(apart, "add_rmsnorm_q8: an output overlaps an input or another output");
  }
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
  // Two vectors a thread and many blocks, as few warps as the row then needs: 16384 rows
  // of 2048 bf16 49 us, with one vector (8 warps) 58, four (2 warps) 57; 4 rows of 64
  // vectors a block, 16000 of them 14 us, with a warp more per row 16. At most 16 blocks
  // per SM (4000 rows of 8192 49 us, with a block a row 58). Up to two rows
  // per SM one vector a thread, for latency: 24 rows of 2048 2.3 us, with two 2.7.
  const int first = T <= 2 * static_cast<int64_t>(sm_count()) ? 1 : 2;
  int nv = first;
  while (nv < AN_NV && a.vec > nv * 32 * AN_WARPS) nv *= 2;
  const int warps = std::min(AN_WARPS, (a.vec + nv * 32 - 1) / (nv * 32));
  if (a.vec > nv * 32 * warps) nv = 0;
  const int block = warps > 1 ? warps : 4;  // a row's barrier is the whole block's
  const int64_t want = warps > 1 ? T : (T + block - 1) / block;
  const int grid = static_cast<int>(std::min<int64_t>(want, static_cast<int64_t>(sm_count()) * 16));
  auto go = [&](auto kern) {
    return launch_pdl_late(kern, dim3(grid), dim3(static_cast<unsigned>(32 * block)), 0,
                           reinterpret_cast<cudaStream_t>(stream), a, warps);
  };
  auto pick = [&](auto bf16) {
    constexpr bool B = decltype(bf16)::value;
    switch (nv) {
      case 1: return go(k_add_rmsnorm<B, 1>);
      case 2: return go(k_add_rmsnorm<B, 2>);
      case 4: return go(k_add_rmsnorm<B, 4>);
      case 8: return go(k_add_rmsnorm<B, 8>);
      default: return go(k_add_rmsnorm<B, 0>);
    }
  };
  DM_CUDA_CHECK(dtype == DECOMOE_BF16 ? pick(std::true_type()) : pick(std::false_type()));
  return DECOMOE_OK;
}
