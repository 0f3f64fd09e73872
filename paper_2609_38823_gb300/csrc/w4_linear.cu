// Few rows times a matrix of 4-bit weights with group scales: the projections
// around the attention of a decode layer (base-model steps that the method
// leaves unchanged).
//   out[t, n] = xs_t sum_g ws[n, g] sum_{k in group g} x[t, k] (q[n, k] - 8)
//
// The weights are read once and bound the call (half a byte per product of up to
// 32 rows), so what matters is few instructions per weight and many bytes in
// flight. Products run on the tensor cores (mma.m16n8k16, fp32 accumulate) with
// 16 columns n as the rows of the product and 8 rows t as its columns. A weight
// becomes an operand without a conversion: its four bits are put into the mantissa
// of a 16-bit float of value 16 (bits 3 to 6 in bf16, 6 to 9 in fp16), which
// makes it the exact number 16 + q, one shift and one three-input logic operation
// for two weights. The offset of 24 leaves with 24 sum x, which the tensor
// cores add up too, as the product of the same rows with ones; the difference is
// at most six times what it is taken from, in fp32. Rows in bf16 take bf16
// products, rows in e4m3 fp16 ones (an e4m3 value is exact in fp16), so that every
// product is exact.
//
// The order of k inside a product is free as long as both operands agree: lane l of
// a quad takes 16 / G' consecutive bytes of a group of a weight row (one 16-byte load
// of a group of 128), a word of which holds four pairs (k, k + 4), and picks the
// same pairs of x.
#include <cuda_fp8.h>

#include <type_traits>

#include "decomoe_internal.cuh"

namespace decomoe {

constexpr int W4_WARPS = 8;

struct W4Args {
  const void* x;
  const float* xs;
  const uint8_t* w;
  const __nv_bfloat16* ws;
  void* out;
  int64_t T, N, x_stride;
  int K, groups, out_f32;
};

template <bool E4M3>
__device__ __forceinline__ void w4_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (E4M3)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Pair i (weights i and i + 4) of a word of eight, as two floats 16 + q.
template <bool E4M3>
__device__ __forceinline__ uint32_t w4_pair(uint32_t w, int i) {
  constexpr uint32_t MASK = E4M3 ? 0x03c003c0u : 0x00780078u, SIXTEEN = E4M3 ? 0x4c004c00u : 0x41804180u;
  const int sh = (E4M3 ? 6 : 3) - 4 * i;
  const uint32_t s = sh >= 0 ? w << sh : w >> -sh;
  return (s & MASK) | SIXTEEN;
}

// Eight consecutive values of a row of x as four pairs (k, k + 4).
struct W4X {
  uint32_t p[4];
};
__device__ __forceinline__ W4X w4_x(const uint4& v) {  // bf16
  W4X r;
  r.p[0] = __byte_perm(v.x, v.z, 0x5410);
  r.p[1] = __byte_perm(v.x, v.z, 0x7632);
  r.p[2] = __byte_perm(v.y, v.w, 0x5410);
  r.p[3] = __byte_perm(v.y, v.w, 0x7632);
  return r;
}
__device__ __forceinline__ uint32_t w4_cvt(uint32_t two) {  // two e4m3 in the low 16 bits, as fp16
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  return static_cast<uint32_t>(h.x) | static_cast<uint32_t>(h.y) << 16;
}
__device__ __forceinline__ W4X w4_x(const uint2& v) {  // e4m3
  const uint32_t a = __byte_perm(v.x, v.y, 0x5140), b = __byte_perm(v.x, v.y, 0x7362);
  W4X r;
  r.p[0] = w4_cvt(a & 0xffffu);
  r.p[1] = w4_cvt(a >> 16);
  r.p[2] = w4_cvt(b & 0xffffu);
  r.p[3] = w4_cvt(b >> 16);
  return r;
}

// One block per 16 MT columns and 8 NT rows; its warps take the groups g = warp,
// warp + 8, ... and add up in warp order.
template <bool E4M3, int GROUP, int MT, int NT>
__global__ void __launch_bounds__(32 * W4_WARPS) k_w4_linear(W4Args a) {
  constexpr int WORDS = GROUP / 32;  // words of a group of a weight row per lane
  using XV = std::conditional_t<E4M3, uint2, uint4>;
  __shared__ float red[W4_WARPS][MT * NT][32][4];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane & 3, row = lane >> 2;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * (16 * MT);
  const int64_t t0 = static_cast<int64_t>(blockIdx.y) * (8 * NT);
  const uint8_t* w[MT][2];
  const __nv_bfloat16* ws[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t n = min(n0 + m * 16 + i * 8 + row, a.N - 1);
      w[m][i] = a.w + n * (a.K / 2) + quad * (4 * WORDS);
      ws[m][i] = a.ws + n * a.groups;
    }
  const uint8_t* x[NT];
  bool has[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    has[j] = t0 + j * 8 + row < a.T;
    x[j] = static_cast<const uint8_t*>(a.x) +
           ((has[j] ? t0 + j * 8 + row : 0) * a.x_stride + quad * (8 * WORDS)) * (E4M3 ? 1 : 2);
  }
  float acc[MT][NT][4] = {};
  const uint32_t one = E4M3 ? 0x3c003c00u : 0x3f803f80u;
  const uint32_t ones[4] = {one, one, one, one};
#pragma unroll 2
  for (int g = warp; g < a.groups; g += W4_WARPS) {
    uint32_t q[MT][2][WORDS];
    float s[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint8_t* p = w[m][i] + static_cast<int64_t>(g) * (GROUP / 2);
        if constexpr (WORDS == 4) {
          const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
          q[m][i][0] = v.x, q[m][i][1] = v.y, q[m][i][2] = v.z, q[m][i][3] = v.w;
        } else if constexpr (WORDS == 2) {
          const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
          q[m][i][0] = v.x, q[m][i][1] = v.y;
        } else {
          q[m][i][0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        }
        s[m][i] = __bfloat162float(ws[m][i][g]);
      }
    XV xv[NT][WORDS];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int u = 0; u < WORDS; ++u)
        xv[j][u] = has[j] ? __ldg(reinterpret_cast<const XV*>(x[j] + static_cast<int64_t>(g) * GROUP * (E4M3 ? 1 : 2)) + u)
                          : XV{};
    float c[MT][NT][4] = {}, sum[NT][4] = {};
#pragma unroll
    for (int u = 0; u < WORDS; ++u) {
      W4X xp[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) xp[j] = w4_x(xv[j][u]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint32_t f[4] = {w4_pair<E4M3>(q[m][0][u], 2 * h), w4_pair<E4M3>(q[m][1][u], 2 * h),
                                 w4_pair<E4M3>(q[m][0][u], 2 * h + 1), w4_pair<E4M3>(q[m][1][u], 2 * h + 1)};
#pragma unroll
          for (int j = 0; j < NT; ++j) w4_mma<E4M3>(c[m][j], f, xp[j].p[2 * h], xp[j].p[2 * h + 1]);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) w4_mma<E4M3>(sum[j], ones, xp[j].p[2 * h], xp[j].p[2 * h + 1]);
      }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[m][j][i] = fmaf(s[m][i >> 1], fmaf(-24.f, sum[j][i & 1], c[m][j][i]), acc[m][j][i]);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < NT; ++j)
      *reinterpret_cast<float4*>(red[warp][m * NT + j][lane]) =
          make_float4(acc[m][j][0], acc[m][j][1], acc[m][j][2], acc[m][j][3]);
  __syncthreads();
  // column n (consecutive threads) of row t; its place in the accumulator tiles
  for (int i = threadIdx.x; i < 16 * MT * 8 * NT; i += 32 * W4_WARPS) {
    const int nn = i % (16 * MT), tt = i / (16 * MT);
    const int64_t n = n0 + nn, t = t0 + tt;
    if (n >= a.N || t >= a.T) continue;
    const int tile = (nn >> 4) * NT + (tt >> 3), l = (nn & 7) * 4 + ((tt & 7) >> 1), e = ((nn >> 3) & 1) * 2 + (tt & 1);
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < W4_WARPS; ++k) v += red[k][tile][l][e];
    if (a.xs != nullptr) v *= a.xs[t];
    if (a.out_f32) static_cast<float*>(a.out)[t * a.N + n] = v;
    else static_cast<__nv_bfloat16*>(a.out)[t * a.N + n] = __float2bfloat16_rn(v);
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
  DM_ARG_CHECK(T <= 65535 * 8, "w4_linear: T above %d", 65535 * 8);
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
  a.groups = K / group;
  a.out_f32 = out_dtype == DECOMOE_F32;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto kern, int cols, int rows) -> int {
    const dim3 grid(static_cast<unsigned>((N + cols - 1) / cols), static_cast<unsigned>((T + rows - 1) / rows));
    DM_CUDA_CHECK(launch_pdl(kern, grid, dim3(32 * W4_WARPS), 0, s, a));
    return DECOMOE_OK;
  };
  auto by_rows = [&](auto e4m3, auto grp) -> int {
    constexpr bool E = decltype(e4m3)::value;
    constexpr int G = decltype(grp)::value;
    if (T <= 8) return go(k_w4_linear<E, G, 1, 1>, 16, 8);
    if (T <= 16) return go(k_w4_linear<E, G, 1, 2>, 16, 16);
    return go(k_w4_linear<E, G, 1, 4>, 16, 32);
  };
  auto by_group = [&](auto e4m3) -> int {
    switch (group) {
      case 32: return by_rows(e4m3, std::integral_constant<int, 32>());
      case 64: return by_rows(e4m3, std::integral_constant<int, 64>());
      default: return by_rows(e4m3, std::integral_constant<int, 128>());
    }
  };
  return x_dtype == DECOMOE_E4M3 ? by_group(std::true_type()) : by_group(std::false_type());
}
