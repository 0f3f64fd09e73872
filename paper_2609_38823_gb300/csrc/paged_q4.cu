// A paged key-value cache in 4 bits: new rows quantised into their slots, and rows
// read back in bf16 (decoding on the text-only cache, DecoMoE Section 3.2 and Algorithm
// 2, last step, with a cache of a quarter of the size).
#include "paged_q4.cuh"

namespace decomoe {

struct Q4Rows {
  const int32_t* slots;
  uint8_t* pages;
  int64_t N, rows, k_stride, v_stride, page_stride;  // rows: of the pool; strides of k and v in elements
  int32_t* status;
  int hkv, shift;
};

// Eight features of a row per lane, so that a lane holds a 32-bit word of codes of a key
// or two 16-bit words of a value, D / 8 lanes per (row, KV head, key or value).
template <int D, int G>
struct Q4Lane {
  using T = Q4Tile<D, G>;
  static constexpr int LANES = D / 8, BLOCKS = D / 32, GROUP = D / G, GL = GROUP / 8;  // GL lanes to a group
  int64_t n;      // row of the call; -1: none
  int head, t;    // KV head, lane of the row
  bool value;
  uint8_t* tile;  // its part of the tile: codes of the row, and its parameters
  int codes, params;
  __device__ __forceinline__ Q4Lane(const Q4Rows& a) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    t = static_cast<int>(i % LANES);
    const int64_t part = i / LANES;
    value = part & 1;
    head = static_cast<int>((part >> 1) % a.hkv);
    n = (part >> 1) / a.hkv;
    tile = nullptr;
    if (n >= a.N) {
      n = -1;
      return;
    }
    const int slot = a.slots[n];
    if (slot < 0 || slot >= a.rows) {
      if (slot >= a.rows || slot < -1) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
      n = -1;
      return;
    }
    const int off = slot & ((1 << a.shift) - 1);
    tile = a.pages + (slot >> a.shift) * a.page_stride +
           ((static_cast<int64_t>(head) << a.shift >> 3) + (off >> 3)) * T::BYTES;
    const int row = off & 7;
    codes = (value ? T::V : T::K) + row * T::CODES;
    params = (value ? T::VP : T::KP) + row * T::PARAMS + (t / GL) * 4;
  }
  __device__ __forceinline__ int key_word() const { return codes + ((t & 3) * BLOCKS + (t >> 2)) * 4; }
  __device__ __forceinline__ int value_word() const { return codes + (2 * (t & 3) * BLOCKS + (t >> 2)) * 2; }
};

__device__ __forceinline__ void q4_unpack8(const uint4& u, float (&x)[8]) {
  x[0] = bf16_lo(u.x), x[1] = bf16_hi(u.x), x[2] = bf16_lo(u.y), x[3] = bf16_hi(u.y);
  x[4] = bf16_lo(u.z), x[5] = bf16_hi(u.z), x[6] = bf16_lo(u.w), x[7] = bf16_hi(u.w);
}

template <int D, int G>
__global__ void __launch_bounds__(256) k_paged_append_q4(Q4Rows a, const __nv_bfloat16* k, const __nv_bfloat16* v) {
  using L = Q4Lane<D, G>;
  pdl_wait();
  const L l(a);
  float x[8] = {};
  if (l.n >= 0) {
    const __nv_bfloat16* src = (l.value ? v + l.n * a.v_stride : k + l.n * a.k_stride) + l.head * D + l.t * 8;
    q4_unpack8(*reinterpret_cast<const uint4*>(src), x);
  }
  pdl_trigger();
  // NaN where a value is not finite (a difference of its own is not zero)
  float lo = x[0], hi = x[0], odd = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo = fminf(lo, x[j]);
    hi = fmaxf(hi, x[j]);
    odd += x[j] - x[j];
  }
#pragma unroll
  for (int w = 1; w < L::GL; w <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, w));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, w));
    odd += __shfl_xor_sync(0xffffffffu, odd, w);
  }
  if (l.n < 0) return;
  const float range = hi - lo;
  const bool finite = odd == 0.f && range <= FLT_MAX;
  const __nv_bfloat16 step_b = __float2bfloat16_rn(__fdiv_rn(range, 15.f));
  const float step = __bfloat162float(step_b);
  uint32_t code = 0;
  if (finite && step > 0.f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float q = fminf(rintf(__fdiv_rn(x[j] - lo, step)), 15.f);
      code |= static_cast<uint32_t>(q) << (4 * j);
    }
  }
  if (l.value) {
    uint16_t* dst = reinterpret_cast<uint16_t*>(l.tile + l.value_word());
    dst[0] = static_cast<uint16_t>(code);
    dst[L::BLOCKS] = static_cast<uint16_t>(code >> 16);
  } else {
    *reinterpret_cast<uint32_t*>(l.tile + l.key_word()) = code;
  }
  if (l.t % L::GL == 0)
    *reinterpret_cast<uint32_t*>(l.tile + l.params) = finite ? pack_bf16x2(step, lo) : 0x7fff7fffu;
}

template <int D, int G>
__global__ void __launch_bounds__(256) k_paged_read_q4(Q4Rows a, __nv_bfloat16* k, __nv_bfloat16* v) {
  using L = Q4Lane<D, G>;
  pdl_wait();
  const L l(a);
  if (l.n < 0) return;
  uint32_t code;
  if (l.value) {
    const uint16_t* src = reinterpret_cast<const uint16_t*>(l.tile + l.value_word());
    code = src[0] | static_cast<uint32_t>(src[L::BLOCKS]) << 16;
  } else {
    code = *reinterpret_cast<const uint32_t*>(l.tile + l.key_word());
  }
  const uint32_t p = *reinterpret_cast<const uint32_t*>(l.tile + l.params);
  pdl_trigger();
  const float step = bf16_lo(p), lo = bf16_hi(p);
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = fmaf(step, static_cast<float>((code >> (4 * j)) & 15u), lo);
  __nv_bfloat16* dst = (l.value ? v + l.n * a.v_stride : k + l.n * a.k_stride) + l.head * D + l.t * 8;
  *reinterpret_cast<uint4*>(dst) =
      make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// The checks that the two calls share, and their arguments.
static int q4_rows(const char* name, const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride, int64_t N,
                   int Hkv, int D, int group, const int32_t* slot_map, const void* pages, int64_t num_pages,
                   int page_size, int64_t page_stride, int32_t* status_dev, Q4Rows* a) {
  DM_ARG_CHECK(q4_shape_ok(D, group), "%s: D 64 with groups of 32 or 64, or D 128 with groups of 32, 64 or 128", name);
  DM_ARG_CHECK(N >= 0 && N <= INT_MAX && Hkv >= 1 && Hkv <= 1024, "%s: bad sizes", name);
  DM_ARG_CHECK(page_size >= 8 && (page_size & (page_size - 1)) == 0, "%s: page_size must be a power of two, 8 at least", name);
  DM_ARG_CHECK(num_pages >= 0 && num_pages <= INT_MAX / page_size, "%s: num_pages * page_size must be below 2^31", name);
  const int64_t page = Hkv * (page_size / 8) * q4_tile_bytes(D, group);
  DM_ARG_CHECK(page_stride >= page && page_stride % 16 == 0, "%s: page_stride below a page's bytes, or no multiple of 16", name);
  const int64_t width = static_cast<int64_t>(Hkv) * D;
  DM_ARG_CHECK(k_row_stride >= width && v_row_stride >= width && k_row_stride % 8 == 0 && v_row_stride % 8 == 0,
               "%s: row strides must be at least Hkv * D and multiples of 8", name);
  if (N == 0) return DECOMOE_OK;
  DM_ARG_CHECK(k && v && slot_map && (pages || num_pages == 0), "%s: null pointer", name);
  DM_ARG_CHECK(aligned16(k) && aligned16(v) && aligned16(pages), "%s: pointers must be 16-byte aligned", name);
  a->slots = slot_map;
  a->N = N;
  a->rows = num_pages * page_size;
  a->k_stride = k_row_stride;
  a->v_stride = v_row_stride;
  a->page_stride = page_stride;
  a->status = status_dev;
  a->hkv = Hkv;
  a->shift = __builtin_ctz(static_cast<unsigned>(page_size));
  return DECOMOE_OK;
}

static Bytes q4_pool(const void* pages, int64_t num_pages, int page_size, int64_t page_stride, int Hkv, int D, int group) {
  const int64_t page = Hkv * (page_size / 8) * q4_tile_bytes(D, group);
  return {pages, num_pages == 0 ? 0 : static_cast<size_t>((num_pages - 1) * page_stride + page)};
}

}  // namespace decomoe

using namespace decomoe;

extern "C" {

size_t decomoe_paged_q4_page_bytes(int page_size, int Hkv, int D, int group) {
  if (page_size < 8 || (page_size & (page_size - 1)) != 0 || Hkv < 1 || !q4_shape_ok(D, group)) return 0;
  return static_cast<size_t>(Hkv) * (page_size / 8) * q4_tile_bytes(D, group);
}

int decomoe_paged_append_q4(const void* k_new, int64_t k_row_stride, const void* v_new, int64_t v_row_stride, int64_t N,
                            int Hkv, int D, int group, const int32_t* slot_map, void* pages, int64_t num_pages,
                            int page_size, int64_t page_stride, int32_t* status_dev, decomoe_stream_t stream) {
  clear_error();
  Q4Rows a = {};
  DM_RET(q4_rows("paged_append_q4", k_new, k_row_stride, v_new, v_row_stride, N, Hkv, D, group, slot_map, pages, num_pages,
                 page_size, page_stride, status_dev, &a));
  if (N == 0) return DECOMOE_OK;
  const size_t width = static_cast<size_t>(Hkv) * D;
  DM_ARG_CHECK(!overlaps(q4_pool(pages, num_pages, page_size, page_stride, Hkv, D, group),
                         {{k_new, (static_cast<size_t>(N - 1) * k_row_stride + width) * 2},
                          {v_new, (static_cast<size_t>(N - 1) * v_row_stride + width) * 2},
                          {slot_map, static_cast<size_t>(N) * 4}}),
               "paged_append_q4: the pool overlaps an input");
  a.pages = static_cast<uint8_t*>(pages);
  const int64_t grid = (N * Hkv * 2 * (D / 8) + 255) / 256;
  DM_ARG_CHECK(grid <= INT_MAX, "paged_append_q4: too many rows");
  return q4_dispatch(D, group, [&](auto d, auto g) -> int {
    DM_CUDA_CHECK(launch_pdl_late(k_paged_append_q4<d.value, g.value>, dim3(static_cast<unsigned>(grid)), dim3(256), 0,
                                  reinterpret_cast<cudaStream_t>(stream), a, static_cast<const __nv_bfloat16*>(k_new),
                                  static_cast<const __nv_bfloat16*>(v_new)));
    return DECOMOE_OK;
  });
}

int decomoe_paged_read_q4(const int32_t* slot_map, int64_t N, const void* pages, int64_t num_pages, int page_size,
                          int64_t page_stride, int Hkv, int D, int group, void* k_out, int64_t k_row_stride, void* v_out,
                          int64_t v_row_stride, int32_t* status_dev, decomoe_stream_t stream) {
  clear_error();
  Q4Rows a = {};
  DM_RET(q4_rows("paged_read_q4", k_out, k_row_stride, v_out, v_row_stride, N, Hkv, D, group, slot_map, pages, num_pages,
                 page_size, page_stride, status_dev, &a));
  if (N == 0) return DECOMOE_OK;
  const size_t width = static_cast<size_t>(Hkv) * D;
  const Bytes k = {k_out, (static_cast<size_t>(N - 1) * k_row_stride + width) * 2},
              v = {v_out, (static_cast<size_t>(N - 1) * v_row_stride + width) * 2}, slots = {slot_map, static_cast<size_t>(N) * 4},
              pool = q4_pool(pages, num_pages, page_size, page_stride, Hkv, D, group);
  // k_out and v_out may be slices of the same rows: they must not share an element
  const int64_t apart = (static_cast<const char*>(v_out) - static_cast<const char*>(k_out)) / 2;
  const int64_t w = static_cast<int64_t>(width);
  const int64_t at = k_row_stride == v_row_stride ? ((apart % k_row_stride) + k_row_stride) % k_row_stride : 0;
  const bool side_by_side = k_row_stride == v_row_stride && at >= w && at + w <= k_row_stride;
  DM_ARG_CHECK(!overlaps(k, {slots, pool}) && !overlaps(v, {slots, pool}) && (side_by_side || !overlaps(k, {v})),
               "paged_read_q4: an output overlaps an input or the other output");
  a.pages = const_cast<uint8_t*>(static_cast<const uint8_t*>(pages));
  const int64_t grid = (N * Hkv * 2 * (D / 8) + 255) / 256;
  DM_ARG_CHECK(grid <= INT_MAX, "paged_read_q4: too many rows");
  return q4_dispatch(D, group, [&](auto d, auto g) -> int {
    DM_CUDA_CHECK(launch_pdl_late(k_paged_read_q4<d.value, g.value>, dim3(static_cast<unsigned>(grid)), dim3(256), 0,
                                  reinterpret_cast<cudaStream_t>(stream), a, static_cast<__nv_bfloat16*>(k_out),
                                  static_cast<__nv_bfloat16*>(v_out)));
    return DECOMOE_OK;
  });
}

}  // extern "C"
