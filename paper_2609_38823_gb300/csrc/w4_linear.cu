// Few rows times a matrix of 4-bit weights with group scales: the projections
// around the attention of a decode layer (base-model steps that the method
// leaves unchanged).
//   out[t, n] = xs_t sum_g ws[n, g] sum_{k in group g} x[t, k] (q[n, k] - 8)
//
// The weights are read once and bound the call (half a byte per product of up to
// 32 rows), so what matters is few instructions per weight and many bytes in
// flight. Products run on the tensor cores (mma.m16n8k16, fp32 accumulate) with
// 16 columns n as the rows of the product and 8 rows t as its columns, on bf16 or fp16
// operands that hold the values of x and of the weights as they are, so that every
// product is exact. Weights become operands without a conversion, by their place among the
// bits of a 16-bit float, and less their offset at once. The order of k inside a product is free as long as both
// operands agree: lane l of a quad takes the l-th quarter of a group of a weight row
// (one 16-byte load of a group of 128), a word of which holds four pairs (k, k + 4),
// and picks the same pairs of x.
//
// Two kernels. Up to 2^25 weights the call is a chain of latencies: one block per 16
// columns, rows of x read as they lie (k_w4_direct). Above (and for more than 8 or 16 rows by
// many columns), the weights' stream counts:
// rings of asynchronous copies per warp, x laid out once per block in shared memory
// (k_w4_ring). Measured, bf16 rows, direct / ring, us: 5120 x 2048 T=1 3.2 / 4.9, T=8 3.9
// / 5.5; 2048 x 4096 T=32 6.5 / 10.3; 12000 x 2048 T=8 7.4 / 6.8; 9000 x 4096 T=1 5.9 / 7.0,
// T=8 7.9 / 8.3, T=13 16.2 / 11.3; 32001 x 8192 T=1 38 / 31, T=8 56 / 35, T=32 181 / 79.
#include <cuda_fp8.h>

#include <type_traits>

#include "decomoe_internal.cuh"

namespace decomoe {

constexpr int W4_STAGES = 3;            // units of a warp's ring (with four less of x is staged at a time: T=32 82 us for 79)
constexpr int W4_UNIT = 256;            // values of k of a unit (128 bytes of a weight row)
constexpr int W4_STAGE = 16 * 128;      // bytes of a unit of 16 columns
constexpr int W4_WARPS = 16;            // warps of a ring block, at most
constexpr size_t W4_SMEM = 226 * 1024;

struct W4Args {
  const void* x;
  const float* xs;
  const uint8_t* w;
  const __nv_bfloat16* ws;
  void* out;
  int64_t T, N, x_stride;
  int K, groups, out_f32;
  int wm, wk;      // ring: column tiles and slices of k of a block, wm * wk warps
  int chunk;       // ring: units of x staged at a time
  int64_t tiles;   // tiles of 16 columns in all
};

// c += a b for 16 columns by 8 rows and 16 values of k; w4_mma0 has nothing to add to.
template <bool E4M3>
__device__ __forceinline__ void w4_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (E4M3)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void w4_mma0(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {  // bf16
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
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

// The place of (row t, column n) among the accumulators [column tile][row tile][lane][4]
// of a run of column tiles.
template <int NT>
__device__ __forceinline__ int w4_place(int t, int n) {
  return ((n >> 4) * NT + (t >> 3)) * 128 + ((n & 7) * 4 + ((t & 7) >> 1)) * 4 + ((n >> 3) & 1) * 2 + (t & 1);
}
__device__ __forceinline__ void w4_put(const W4Args& a, int64_t t, int64_t n, float v) {
  if (n >= a.N) return;
  if (a.xs != nullptr) v *= a.xs[t];
  if (a.out_f32) static_cast<float*>(a.out)[t * a.N + n] = v;
  else static_cast<__nv_bfloat16*>(a.out)[t * a.N + n] = __float2bfloat16_rn(v);
}

// ------------------------------------------------------------------ smaller matrices
// Four bits put into the mantissa of a 16-bit float of value 16 (bits 3 to 6 in bf16,
// 6 to 9 in fp16) make it the exact number 16 + q, and less 24 the exact weight q - 8: a shift,
// a three-input logic operation and an addition for two weights. (An offset left in the
// weights, to be taken off a group's sum, would leave there the rounding of large
// values of x that meet the code of zero.)
__device__ __forceinline__ uint32_t w4_const(uint32_t v) {  // a constant that stays in a register
  uint32_t r;
  asm volatile("mov.b32 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// Pair i (weights i and i + 4) of a word of eight, as two floats q - 8.
template <bool E4M3>
__device__ __forceinline__ uint32_t w4_pair(uint32_t w, int i, uint32_t mask, uint32_t sixteen) {
  const int sh = (E4M3 ? 6 : 3) - 4 * i;
  const uint32_t s = sh >= 0 ? w << sh : w >> -sh;
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(s), "r"(mask), "r"(sixteen));  // (s & mask) | sixteen
  if constexpr (E4M3) {
    const __half2 d = __hadd2(*reinterpret_cast<const __half2*>(&r), __half2half2(__ushort_as_half(0xce00)));  // -24
    return *reinterpret_cast<const uint32_t*>(&d);
  } else {
    const __nv_bfloat162 d = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&r),
                                     __bfloat162bfloat162(__ushort_as_bfloat16(0xc1c0)));  // -24
    return *reinterpret_cast<const uint32_t*>(&d);
  }
}

// One block per 16 columns (blockIdx.x) and 8 NT rows (blockIdx.y); its warps take the
// groups g = warp, warp + WARPS, ... and their sums are added in warp order. (Groups of 32 are
// little work each: asked for one block per SM, the compiler keeps more of their loads in
// flight. 4149 x 4960 T=1 6.3 -> 4.9 us, T=32 15.9 -> 9.9; with larger groups fewer blocks
// then fit an SM, 5000 x 4096 by 128 T=1 4.6 -> 5.1, T=8 6.4 -> 7.4.)
template <bool E4M3, int GROUP, int NT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, GROUP == 32 ? 1 : 0) k_w4_direct(W4Args a) {
  constexpr int WORDS = GROUP / 32;  // words of a group of a weight row per lane
  using XV = std::conditional_t<E4M3, uint2, uint4>;
  __shared__ float red[WARPS][NT * 128];
  pdl_wait();
  const uint32_t mask = w4_const(E4M3 ? 0x03c003c0u : 0x00780078u);
  const uint32_t sixteen = w4_const(E4M3 ? 0x4c004c00u : 0x41804180u);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane & 3, row = lane >> 2;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 16;
  const int64_t t0 = static_cast<int64_t>(blockIdx.y) * (8 * NT);
  const uint8_t* w[2];
  const __nv_bfloat16* ws[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t n = min(n0 + i * 8 + row, a.N - 1);
    w[i] = a.w + n * (a.K / 2) + quad * (4 * WORDS);
    ws[i] = a.ws + n * a.groups;
  }
  const uint8_t* x[NT];
  bool has[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    has[j] = t0 + j * 8 + row < a.T;
    x[j] = static_cast<const uint8_t*>(a.x) +
           ((has[j] ? t0 + j * 8 + row : 0) * a.x_stride + quad * (8 * WORDS)) * (E4M3 ? 1 : 2);
  }
  float acc[NT][4] = {};
#pragma unroll 2
  for (int g = warp; g < a.groups; g += WARPS) {
    uint32_t q[2][WORDS];
    float s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* p = w[i] + static_cast<int64_t>(g) * (GROUP / 2);
      if constexpr (WORDS == 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
        q[i][0] = v.x, q[i][1] = v.y, q[i][2] = v.z, q[i][3] = v.w;
      } else if constexpr (WORDS == 2) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
        q[i][0] = v.x, q[i][1] = v.y;
      } else {
        q[i][0] = __ldg(reinterpret_cast<const uint32_t*>(p));
      }
      s[i] = __bfloat162float(ws[i][g]);
    }
    XV xv[NT][WORDS];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int u = 0; u < WORDS; ++u)
        xv[j][u] = has[j] ? __ldg(reinterpret_cast<const XV*>(x[j] + static_cast<int64_t>(g) * GROUP * (E4M3 ? 1 : 2)) + u)
                          : XV{};
    float c[NT][4] = {};
#pragma unroll
    for (int u = 0; u < WORDS; ++u) {
      W4X xp[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) xp[j] = w4_x(xv[j][u]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t f[4] = {w4_pair<E4M3>(q[0][u], 2 * h, mask, sixteen), w4_pair<E4M3>(q[1][u], 2 * h, mask, sixteen),
                               w4_pair<E4M3>(q[0][u], 2 * h + 1, mask, sixteen),
                               w4_pair<E4M3>(q[1][u], 2 * h + 1, mask, sixteen)};
#pragma unroll
        for (int j = 0; j < NT; ++j) w4_mma<E4M3>(c[j], f, xp[j].p[2 * h], xp[j].p[2 * h + 1]);
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = fmaf(s[i >> 1], c[j][i], acc[j][i]);
  }
  pdl_trigger();
#pragma unroll
  for (int j = 0; j < NT; ++j)
    *reinterpret_cast<float4*>(&red[warp][(j * 32 + lane) * 4]) = make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]);
  __syncthreads();
  // a column (consecutive threads) of a row each
  for (int i = threadIdx.x; i < 16 * 8 * NT; i += 32 * WARPS) {
    const int n = i & 15, t = i >> 4;
    if (t0 + t >= a.T) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) v += red[k][w4_place<NT>(t, n)];
    w4_put(a, t0 + t, n0 + n, v);
  }
}

// ------------------------------------------------------------------ larger matrices
// The units that handle logic operations would be the bound with two of them for every
// pair of weights. Four bits at the foot of a bf16 number are the subnormal number
// q 2^-133, the four bits above them 16 q 2^-133, both exact, and one multiply-add of two
// numbers makes (q - 8) / 64 of either, so that a mask and a multiply-add give two operands
// and one shift serves a word of eight. The rows are laid out times 64, rows in e4m3 as
// bf16, which holds their values too; every step is exact.
constexpr float W4_RAISE = 64.f;
__device__ __forceinline__ uint32_t w4_raise(uint32_t v) {  // two bf16, exact below 2^122 (infinite from there)
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&v), __float2bfloat162_rn(W4_RAISE));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t w4_raise_fp16(uint32_t v) {  // two fp16 that were e4m3, to bf16
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
  return pack_bf16x2(f.x * W4_RAISE, f.y * W4_RAISE);
}
// The lowest four bits (UP: the next four) of either half of w as weights over 64.
template <bool UP>
__device__ __forceinline__ uint32_t w4_weights(uint32_t w) {
  const uint32_t bits = w & (UP ? 0x00f000f0u : 0x000f000fu);
  const __nv_bfloat162 f = __bfloat162bfloat162(__ushort_as_bfloat16(UP ? 0x7d00 : 0x7f00));  // 2^123, 2^127
  const __nv_bfloat162 o = __bfloat162bfloat162(__ushort_as_bfloat16(0xbe00));                // -2^-3
  const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&bits), f, o);
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ void w4_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A float at the same place of the shared memory of block `rank` of the cluster.
__device__ __forceinline__ float w4_ld_cluster(uint32_t addr, int rank) {
  uint32_t at;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// A cluster of gridDim.x blocks (one or two) shares the columns of its launch column
// (blockIdx.y), block `rank` of it takes the rank-th part of k, whose x it keeps in
// shared memory for the 8 NT rows of its launch row (blockIdx.z): all of it or, where
// that is too much, `chunk` units at a time. It walks over wm tiles of 16 columns at a
// time, each on wk warps that take its units of k in turn. Every warp streams the
// weights of its tiles through a ring of its own (16-byte asynchronous copies of
// 128-byte pieces of 16 rows, on through the tile's end; no block-wide step but at a
// tile's end). The sums are added over the warps of a block, then over the blocks of
// the cluster through distributed shared memory, both in the order of k.
// 32001 x 8192, T=1: 31 us, 4.4 TB/s; T=8 35 us; the same stream without any product 24.7 us.
// At T=32 (79 us) the reads of x from shared memory bound it: every warp reads all of x for
// 16 columns.
template <bool E4M3, int GROUP, int NT>
__global__ void __launch_bounds__(32 * W4_WARPS, 1) k_w4_ring(W4Args a) {
  constexpr int WORDS = GROUP / 32;            // words of a group of a weight row per lane
  constexpr int GU = W4_UNIT / GROUP;          // groups of a unit
  constexpr int SREG = GU == 8 ? 2 : 1;        // scales of a weight row per lane and unit
  constexpr int TILE = NT * 128;               // floats of a warp's accumulators
  constexpr int XE = E4M3 ? 1 : 2;             // bytes of a value of x
  constexpr int XW = NT * 32;                  // 16-byte places of a word of a group of x
  using XV = std::conditional_t<E4M3, uint2, uint4>;
  extern __shared__ __align__(128) uint8_t w4_smem[];
  const uint32_t xf_at = a.wm * a.wk * (W4_STAGES * W4_STAGE);  // x: [chunk groups][WORDS][NT][32 lanes] uint4
  uint4* xf = reinterpret_cast<uint4*>(w4_smem + xf_at);
  float* red = reinterpret_cast<float*>(xf + a.chunk * (GU * WORDS * XW));  // [warps][NT][32][4]
  pdl_enter();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane & 3, row = lane >> 2;
  const int slice = warp / a.wm, wm = warp - slice * a.wm;
  const int64_t t0 = static_cast<int64_t>(blockIdx.z) * (8 * NT);
  const int rows = static_cast<int>(min(a.T - t0, static_cast<int64_t>(8 * NT)));
  const int ks = static_cast<int>(gridDim.x), rank = static_cast<int>(blockIdx.x);
  const int all_units = (a.K + W4_UNIT - 1) / W4_UNIT;
  const int first = static_cast<int>(static_cast<int64_t>(rank) * all_units / ks);
  const int units = static_cast<int>(static_cast<int64_t>(rank + 1) * all_units / ks) - first;
  const int groups = min(units * GU, a.groups - first * GU);

  // ---- weights: unit after unit of this warp's slice, tile after tile
  const int steps = units > slice ? (units - slice + a.wk - 1) / a.wk : 0;
  const int64_t tile_step = static_cast<int64_t>(gridDim.y) * a.wm;
  const uint32_t kb = static_cast<uint32_t>(a.K / 2);
  const uint32_t ring = warp * (W4_STAGES * W4_STAGE), ring_s = smem_u32(w4_smem) + ring;
  // rows of 128 bytes; the 16-byte pieces of row r are exchanged by the reverse of r's
  // low three bits, which spreads the reads of every group size over all banks
  auto swz = [](int r) { return ((r & 1) << 2) | (r & 2) | ((r >> 2) & 1); };
  int64_t ptile = static_cast<int64_t>(blockIdx.y) * a.wm + wm;
  int pstep = 0, pslot = 0;
  const uint8_t* psrc = nullptr;  // the tile's first row
  uint32_t pat = 0, prow[4];      // place in a row; offsets of the rows that this lane copies
  auto enter = [&]() {
    const int64_t n0 = ptile * 16;
    psrc = a.w + n0 * kb;
    pat = static_cast<uint32_t>(first + slice) * 128u + (lane & 7) * 16u;
    // rows past the last column read it again (their results go nowhere)
    const int last = static_cast<int>(min(a.N - 1 - n0, int64_t{15}));
#pragma unroll
    for (int i = 0; i < 4; ++i) prow[i] = static_cast<uint32_t>(min(i * 4 + (lane >> 3), last)) * kb;
  };
  const uint32_t pdst[2] = {(lane >> 3) * 128u + (((lane & 7) ^ swz(lane >> 3)) << 4),
                            (lane >> 3) * 128u + (((lane & 7) ^ swz(4 + (lane >> 3))) << 4)};
  if (ptile < a.tiles) enter();
  auto issue = [&]() {
    if (ptile < a.tiles && steps > 0) {
      const bool in = pat < kb;  // the last unit of a row may be cut short: zeros
      const uint8_t* src = psrc + (in ? pat : 0u);
      const uint32_t dst = ring_s + pslot * W4_STAGE;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + pdst[i & 1] + i * 512),
                     "l"(src + prow[i]), "r"(in ? 16 : 0)
                     : "memory");
      pat += a.wk * 128u;
      if (++pstep == steps) {
        pstep = 0;
        ptile += tile_step;
        if (ptile < a.tiles) enter();
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    pslot = pslot + 1 == W4_STAGES ? 0 : pslot + 1;
  };
#pragma unroll
  for (int i = 0; i < W4_STAGES - 1; ++i) issue();

  // ---- x: units [u0, u0 + n) of this block's; a thread takes what one lane of a quad
  // reads of a row of a group, the four of them in consecutive threads
  auto stage = [&](int u0, int n) {
    constexpr int U = 8 / WORDS;  // such pieces in flight
    const int g0 = u0 * GU, pieces = min(n * GU, groups - g0) * 4 * rows;
    // v / rows: the reciprocal rounded up is exact for v below 2^32 / rows
    const uint32_t inverse = rows > 1 ? 0xffffffffu / static_cast<uint32_t>(rows) + 1 : 0;
    const uint8_t* x0 = static_cast<const uint8_t*>(a.x) +
                        (t0 * a.x_stride + (static_cast<int64_t>(first) * GU + g0) * GROUP) * XE;
    const int64_t xrow = a.x_stride * XE;
    for (int i0 = tid; i0 - tid < pieces; i0 += U * blockDim.x) {
      XV v[U][WORDS];
      int gs[U], rs[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * blockDim.x, gr = i >> 2;
        gs[u] = rows > 1 ? static_cast<int>(__umulhi(static_cast<uint32_t>(gr), inverse)) : gr;
        rs[u] = gr - gs[u] * rows;
        const XV* src = reinterpret_cast<const XV*>(x0 + rs[u] * xrow + (gs[u] * GROUP + (i & 3) * (8 * WORDS)) * XE);
#pragma unroll
        for (int e = 0; e < WORDS; ++e) {
          v[u][e] = XV{};
          if (i < pieces) v[u][e] = __ldg(src + e);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * blockDim.x;
        if (i >= pieces) break;
        const int at = gs[u] * (WORDS * XW) + (rs[u] >> 3) * 32 + (rs[u] & 7) * 4 + (i & 3);
#pragma unroll
        for (int e = 0; e < WORDS; ++e) {
          W4X p = w4_x(v[u][e]);
#pragma unroll
          for (int k = 0; k < 4; ++k) p.p[k] = E4M3 ? w4_raise_fp16(p.p[k]) : w4_raise(p.p[k]);
          xf[at + e * XW] = make_uint4(p.p[0], p.p[1], p.p[2], p.p[3]);
        }
      }
    }
  };

  // this lane's places in a word of x and in a unit's rows (byte offsets); rows of x
  // that are not there read the first one, and their results go nowhere
  uint32_t xl[NT], wl[GU];
#pragma unroll
  for (int j = 0; j < NT; ++j) xl[j] = xf_at + (j * 8 + row < rows ? j * 32 + lane : quad) * 16;
#pragma unroll
  for (int gg = 0; gg < GU; ++gg)
    wl[gg] = row * 128 + (((gg * WORDS + (quad * WORDS >> 2)) ^ swz(row)) << 4) + (quad * WORDS & 3) * 4;
  const int ends = min(a.chunk, units);  // end of the first chunk
  int c0 = -1;                           // first staged unit
  int slot = 0;
  for (int64_t tile0 = static_cast<int64_t>(blockIdx.y) * a.wm; tile0 < a.tiles; tile0 += tile_step) {
    const bool live = tile0 + wm < a.tiles && steps > 0;
    const int64_t n0 = (tile0 + wm) * 16;
    const unsigned short* ws = reinterpret_cast<const unsigned short*>(a.ws) + n0 * a.groups + first * GU;
    uint32_t so[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      so[i] = static_cast<uint32_t>(max(min(n0 + i * 8 + row, a.N - 1) - n0, int64_t{0})) * static_cast<uint32_t>(a.groups);
    // bf16 scales of even and of odd steps, two steps ahead (a register that a load is on
    // its way to is not moved: that would wait for it); lane l of a quad holds groups l
    // and l + 4 of a unit
    uint32_t s_even[2][SREG] = {}, s_odd[2][SREG] = {};
    auto scales = [&](uint32_t (&d)[2][SREG], int step) {
#pragma unroll
      for (int e = 0; e < SREG; ++e) {
        const int g = min((slice + step * a.wk) * GU + (quad & (GU - 1)) + 4 * e, groups - 1);
#pragma unroll
        for (int i = 0; i < 2; ++i) d[i][e] = __ldg(ws + (so[i] + g));
      }
    };
    if (live) {
      scales(s_even, 0);
      scales(s_odd, 1);
    }
    if (c0 != 0) {
      c0 = 0;
      stage(0, ends);
      __syncthreads();
    }
    float acc[NT][4] = {};
    // chunk after chunk of k (mostly one); every warp goes through every chunk
    for (int step = 0, end = ends;;) {
      const int until = live ? min(steps, (end - slice + a.wk - 1) / a.wk) : 0;
      uint32_t xg = static_cast<uint32_t>((slice + step * a.wk - c0) * GU);  // first group, from the chunk's
      auto unit = [&](uint32_t (&s)[2][SREG]) {
        issue();
        asm volatile("cp.async.wait_group %0;" ::"n"(W4_STAGES - 1) : "memory");
        __syncwarp();
        const uint32_t wq = ring + slot * W4_STAGE;
        const int left = groups - (slice + step * a.wk) * GU;  // the last unit may be cut short
#pragma unroll
        for (int gg = 0; gg < GU; ++gg) {
          if (gg > 0 && gg >= left) break;
          uint32_t q[2][WORDS];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t p = wq + wl[gg] + i * 8 * 128;
            if constexpr (WORDS == 4) {
              const uint4 v = *reinterpret_cast<const uint4*>(w4_smem + p);
              q[i][0] = v.x, q[i][1] = v.y, q[i][2] = v.z, q[i][3] = v.w;
            } else if constexpr (WORDS == 2) {
              const uint2 v = *reinterpret_cast<const uint2*>(w4_smem + p);
              q[i][0] = v.x, q[i][1] = v.y;
            } else {
              q[i][0] = *reinterpret_cast<const uint32_t*>(w4_smem + p);
            }
          }
          float c[NT][4];
          const uint32_t xb = (xg + gg) * (WORDS * XW * 16);
#pragma unroll
          for (int word = 0; word < WORDS; ++word) {
            const uint32_t q0 = q[0][word], q1 = q[1][word], h0 = q0 >> 8, h1 = q1 >> 8;
            const uint32_t f0[4] = {w4_weights<false>(q0), w4_weights<false>(q1), w4_weights<true>(q0), w4_weights<true>(q1)};
            const uint32_t f1[4] = {w4_weights<false>(h0), w4_weights<false>(h1), w4_weights<true>(h0), w4_weights<true>(h1)};
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              const uint4 xp = *reinterpret_cast<const uint4*>(w4_smem + (xl[j] + xb + word * (XW * 16)));
              if (word == 0) w4_mma0(c[j], f0, xp.x, xp.y);
              else w4_mma<false>(c[j], f0, xp.x, xp.y);
              w4_mma<false>(c[j], f1, xp.z, xp.w);
            }
          }
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            f[i] = __uint_as_float(__shfl_sync(0xffffffffu, s[i][gg >> 2], (lane & ~3) + (gg & 3)) << 16);
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] = fmaf(f[i >> 1], c[j][i], acc[j][i]);
        }
        __syncwarp();
        slot = slot + 1 == W4_STAGES ? 0 : slot + 1;
        scales(s, step + 2);
      };
#pragma unroll 1
      for (; step < until; ++step, xg += a.wk * GU) {
        if (step & 1) unit(s_odd);
        else unit(s_even);
      }
      if (end == units) break;
      __syncthreads();
      c0 = end;
      end = min(end + a.chunk, units);
      stage(c0, end - c0);
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
      *reinterpret_cast<float4*>(red + warp * TILE + (j * 32 + lane) * 4) =
          make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]);
    __syncthreads();
    // a column (consecutive threads) of a row each
    const int cols = 16 * a.wm;
    auto of_block = [&](int at) {
      float v = 0.f;
      for (int k = 0; k < a.wk; ++k) v += red[k * a.wm * TILE + at];
      return v;
    };
    if (ks == 1) {
      for (int i = tid; i < cols * rows; i += blockDim.x) {
        const int t = i / cols, n = i - t * cols;
        w4_put(a, t0 + t, tile0 * 16 + n, of_block(w4_place<NT>(t, n)));
      }
      __syncthreads();
    } else {
      if (a.wk > 1)
        for (int i = tid; i < a.wm * TILE; i += blockDim.x) red[i] = of_block(i);
      w4_cluster_sync();
      // each block takes the rank-th part of the (row, column) places
      const int all = cols * rows, per = (all + ks - 1) / ks, i1 = min(all, (rank + 1) * per);
      for (int i = rank * per + tid; i < i1; i += blockDim.x) {
        const int t = i / cols, n = i - t * cols;
        const uint32_t at = smem_u32(red + w4_place<NT>(t, n));
        float v = 0.f;
        for (int k = 0; k < ks; ++k) v += w4_ld_cluster(at, k);
        w4_put(a, t0 + t, tile0 * 16 + n, v);
      }
      w4_cluster_sync();  // nobody leaves, or writes its sums again, before all have read them
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <bool E4M3, int GROUP, int NT>
static int w4_launch(W4Args a, cudaStream_t s) {
  a.tiles = (a.N + 15) / 16;
  const unsigned z = static_cast<unsigned>((a.T + 8 * NT - 1) / (8 * NT));
  // (With more rows x weighs as much as the weights where there are many columns, whatever
  // their length: direct / ring, bf16 T=24 29478 x 512 12.9 / 10.2 us, 8000 x 2048 10.3 / 9.6, T=13
  // 9.0 / 7.3; fewer columns 2000 x 8192 T=24 10.0 / 12.8. Rows in e4m3 weigh half of it: T=13
  // 8000 x 2048 6.2 / 7.2.)
  if (a.N * a.K <= int64_t{1} << 25 && (NT < (E4M3 ? 3 : 2) || a.N < 48 * static_cast<int64_t>(sm_count()))) {
    const dim3 grid(static_cast<unsigned>(a.tiles), z);
    // Sixteen warps a block where every block has an SM to itself and every warp at least
    // two groups: 2048 x 4096 T=1 4.3 -> 3.3 us, T=17 7.4 -> 5.1; not where blocks share SMs
    // (5120 x 2048 T=1 3.1, with sixteen 3.7) or k is short (700 x 1920 T=32 4.2, 4.8).
    if (a.tiles <= sm_count() && a.groups >= 32)
      DM_CUDA_CHECK(launch_pdl_late(k_w4_direct<E4M3, GROUP, NT, 16>, grid, dim3(512), 0, s, a));
    else
      DM_CUDA_CHECK(launch_pdl_late(k_w4_direct<E4M3, GROUP, NT, 8>, grid, dim3(256), 0, s, a));
    return DECOMOE_OK;
  }
  const int units = (a.K + W4_UNIT - 1) / W4_UNIT;
  const size_t per_unit = NT * 32 * 16 * (W4_UNIT / 32);
  const int64_t sms = sm_count();
  // Two blocks share k where x is large beside the columns, so that each lays out half of it
  // and twice as many columns use it: 9000 x 4096 T=32 19.6 -> 17.9 us, T=13 11.7 -> 11.2;
  // not where the columns then no longer go in one pass (20000 x 2048 T=13 13.0 -> 16.7) nor
  // where x is small (9000 x 4096 T=1 7.0 -> 8.0).
  const int ks = units * per_unit > 100 * 1024 && a.tiles <= (sms / 2) * W4_WARPS && sms > 1 ? 2 : 1;
  const int64_t places = sms / ks;
  // as few passes over the column tiles as the warps of all blocks allow, the tiles
  // spread over all blocks, and what is left of the warps over k
  const int64_t passes = (a.tiles + places * W4_WARPS - 1) / (places * W4_WARPS);
  a.wm = static_cast<int>((a.tiles + places * passes - 1) / (places * passes));
  const int part = (units + ks - 1) / ks;
  a.wk = std::max(1, std::min(W4_WARPS / a.wm, part));
  const int warps = a.wm * a.wk;
  const size_t fixed = static_cast<size_t>(warps) * (W4_STAGES * W4_STAGE + NT * 512);
  a.chunk = static_cast<int>(std::min<size_t>(part, (W4_SMEM - fixed) / per_unit));
  const size_t smem = fixed + a.chunk * per_unit;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ks, static_cast<unsigned>(std::min(places, (a.tiles + a.wm - 1) / a.wm)), z);
  cfg.blockDim = dim3(32 * warps);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed =
      pdl_enabled(static_cast<int64_t>(cfg.gridDim.x) * cfg.gridDim.y * cfg.gridDim.z) ? 1 : 0;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ks;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  auto kern = k_w4_ring<E4M3, GROUP, NT>;
  DM_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
  DM_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kern, a));
  return DECOMOE_OK;
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
  DM_ARG_CHECK(K <= 1 << 26, "w4_linear: K above 2^26");
  DM_ARG_CHECK(T <= 65535 * 8, "w4_linear: T above %d", 65535 * 8);
  if (T == 0) return DECOMOE_OK;
  DM_ARG_CHECK(x && w && w_scale && out, "w4_linear: null pointer");
  DM_ARG_CHECK((x_dtype == DECOMOE_E4M3) == (x_scale != nullptr), "w4_linear: x_scale goes with e4m3 rows, and only with them");
  const int64_t xe = x_dtype == DECOMOE_BF16 ? 2 : 1;
  DM_ARG_CHECK(x_stride >= K && x_stride * xe % 16 == 0 && aligned16(x) && aligned16(w) &&
                   (reinterpret_cast<uintptr_t>(w_scale) & 1u) == 0 &&
                   reinterpret_cast<uintptr_t>(out) % dtype_bytes(out_dtype) == 0,
               "w4_linear: x_stride must be at least K and a multiple of 16 bytes, x and w 16-byte aligned");
  DM_ARG_CHECK(!overlaps({out, static_cast<size_t>(T * N) * dtype_bytes(out_dtype)},
                         {{x, static_cast<size_t>(((T - 1) * x_stride + K) * xe)},
                          {x_scale, static_cast<size_t>(T) * sizeof(float)},
                          {w, static_cast<size_t>(N) * static_cast<size_t>(K / 2)},
                          {w_scale, static_cast<size_t>(N) * static_cast<size_t>(K / group) * 2}}),
               "w4_linear: out overlaps an input");
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
  auto by_rows = [&](auto e4m3, auto grp) -> int {
    constexpr bool E = decltype(e4m3)::value;
    constexpr int G = decltype(grp)::value;
    if (T <= 8) return w4_launch<E, G, 1>(a, s);
    if (T <= 16) return w4_launch<E, G, 2>(a, s);
    if (T <= 24) return w4_launch<E, G, 3>(a, s);
    return w4_launch<E, G, 4>(a, s);
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
