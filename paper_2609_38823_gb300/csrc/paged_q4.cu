// A paged key-value cache in 4 bits: new rows quantised into their slots, and rows
// read back in bf16 (decoding on the text-only cache, DecoMoE Section 3.2 and Algorithm
// 2, last step, with a cache of a quarter of the size).
//
// Bound: instructions and latency for long calls, launches for a decode batch. 16381 rows of 8 heads of 64: store
// 13.2 us, 3.4 TB/s (its pool lies in L2), read 9.0 us, 4.9 TB/s; 5000 rows of 8 heads of 128 in groups of 32: 9.9 and
// 6.5 us; 23 rows of 4 heads of 128: 2.1 and 1.5 us (in a graph, six sets of tensors in turn). Steps: the first store
// divided twice a value and found its row by 64-bit division: 33 us; ties between two codes by exact remainders, in a
// branch that 40 % of the warps took: 18.5; values one at a time instead of in packed pairs 13.5, the read 9.6.
#include "paged_q4.cuh"

namespace decomoe {

constexpr int Q4_THREADS = 128;  // of a block (256: 0.2 us slower from 23 rows to 16384)

struct Q4Rows {
  const int32_t* slots;
  uint8_t* pages;
  int64_t N, rows, k_stride, v_stride, page_stride;  // rows: of the pool; strides of k and v in elements
  int32_t* status;
  int hkv, shift, lanes;  // 1 << lanes threads to a row
};

// A lane has eight features of a KV head at a time, of the key and of the value: a 32-bit
// word of the key's codes, two 16-bit words of the value's. 1 << lanes threads (at most a
// warp) walk over a row, CHUNKS pieces of a thread loaded ahead, so that a warp has up to 2 KB in flight.
template <int D, int G>
struct Q4Lane {
  using T = Q4Tile<D, G>;
  static constexpr int LANES = D / 8, BLOCKS = D / 32, GL = D / G / 8;  // lanes of a head's row, and of a group
  static constexpr int CHUNKS = 2;
  // Words of a value's row lie apart (16-bit word (2 (t & 3) + j) BLOCKS + (t >> 2) of lane t's
  // half j): two lanes 4 apart hold the halves of two 32-bit words, one for each of them. The
  // same exchange leads back.
  static __device__ __forceinline__ uint32_t exchange(uint32_t w, int t) {
    const bool odd = (t >> 2) & 1;
    const uint32_t other = __shfl_xor_sync(0xffffffffu, w, 4);
    return odd ? __byte_perm(other, w, 0x7632) : __byte_perm(w, other, 0x5410);
  }
  static __device__ __forceinline__ int key_word(int t) { return ((t & 3) * BLOCKS + (t >> 2)) * 4; }
  static __device__ __forceinline__ int value_word(int t) {  // of exchange()
    return ((2 * (t & 3) + ((t >> 2) & 1)) * BLOCKS + (t >> 3) * 2) * 2;
  }
};

// The eight rows of a head in which a slot lies; null for a slot of -1, or (marked) outside the pool.
template <class T>
__device__ __forceinline__ uint8_t* q4_tile(const Q4Rows& a, int slot, bool mark) {
  if (slot < 0 || slot >= a.rows) {
    if (mark && slot != -1) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
    return nullptr;
  }
  const int off = slot & ((1 << a.shift) - 1);
  return a.pages + (slot >> a.shift) * a.page_stride + static_cast<int64_t>(off >> 3) * T::BYTES;
}

__device__ __forceinline__ void q4_unpack8(const uint4& u, float (&x)[8]) {
  x[0] = bf16_lo(u.x), x[1] = bf16_hi(u.x), x[2] = bf16_lo(u.y), x[3] = bf16_hi(u.y);
  x[4] = bf16_lo(u.z), x[5] = bf16_hi(u.z), x[6] = bf16_lo(u.w), x[7] = bf16_hi(u.w);
}

// Two fp32 numbers at a time.
__device__ __forceinline__ uint64_t q4_two(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t q4_two(uint32_t a, uint32_t b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void q4_split(uint64_t v, uint32_t& a, uint32_t& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t q4_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t q4_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t q4_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Sums >= 0 cut off, but their last digit odd where something was cut off.
__device__ __forceinline__ uint64_t q4_add_odd(uint64_t a, uint64_t b) {
  uint64_t r, up;
  asm("add.rz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  asm("add.rp.f32x2 %0, %1, %2;" : "=l"(up) : "l"(a), "l"(b));
  return r | (up & 0x0000000100000001ull);  // (the two are neighbours where they differ: one of them is odd)
}

__device__ __forceinline__ uint32_t q4_max2(uint32_t a, uint32_t b) {  // of two pairs of bf16 numbers, NaN where one is
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// The codes of eight features of a group that GL lanes share, and the group's parameters.
template <int GL>
__device__ __forceinline__ uint32_t q4_quantise(const uint4& u, uint32_t* params) {
  // the largest of the values (high half) and of their negatives
  const uint32_t big = q4_max2(q4_max2(u.x, u.y), q4_max2(u.z, u.w));
  constexpr uint32_t MINUS = 0x80008000u;
  const uint32_t neg = q4_max2(q4_max2(u.x ^ MINUS, u.y ^ MINUS), q4_max2(u.z ^ MINUS, u.w ^ MINUS));
  uint32_t ends = q4_max2(__byte_perm(neg, big, 0x5410), __byte_perm(neg, big, 0x7632));
#pragma unroll
  for (int w = 1; w < GL; w <<= 1) ends = q4_max2(ends, __shfl_xor_sync(0xffffffffu, ends, w));
  const float lo = -bf16_lo(ends), range = bf16_hi(ends) + bf16_lo(ends);
  // range / 15, to nearest: Markstein's correction of a quotient from the rounded reciprocal
  float step32 = range * (1.f / 15.f);
  step32 = fmaf(fmaf(-15.f, step32, range), 1.f / 15.f, step32);
  const bool small = range < 0x1p-100f;  // where remainders would be subnormal, divide
  if (small) step32 = __fdiv_rn(range, 15.f);
  const float step = __bfloat162float(__float2bfloat16_rn(step32));
  const bool finite = range <= FLT_MAX;  // a value that is not gives NaN or infinity
  *params = finite ? pack_bf16x2(step, lo) : 0x7fff7fffu;
  if (!finite || step == 0.f) return 0;
  float x[8];
  q4_unpack8(u, x);
  uint32_t code = 0;
  // A place half way between two codes is (2 k + 1) step / 2, 13 digits at most. x - lo can need more than fp32's
  // 24: cut off, with an odd last digit where something was lost, it lies on the same side of every such place, and
  // on none; rounded to nearest it could fall on one. (An addition and two operations a pair: 16381 rows 12.8 -> 13.2 us, 5000
  // of 8 heads of 128 8.9 -> 9.9. Held to nine blocks an SM, as many as before, these take 13.4 and 9.3.)
  if (small) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float r = __uint_as_float(__float_as_uint(__fsub_rz(x[j], lo)) | (__float_as_uint(__fsub_ru(x[j], lo)) & 1u));
      code |= static_cast<uint32_t>(fminf(rintf(__fdiv_rn(r, step)), 15.f)) << (4 * j);
    }
    return code;
  }
  // (x - lo) / step to nearest by the same correction, so that a value half way between two codes
  // and no other gives exactly that; adding 3 * 2^22 then rounds to the integer (ties to even), which stands in
  // the low bits. The high ones leave the sum of all eight at once.
  constexpr float MAGIC = 12582912.f;
  constexpr uint32_t HIGH = 0x4b400000u;
  const float inv = __frcp_rn(step);
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const uint64_t r = q4_add_odd(q4_two(x[j], x[j + 1]), q4_two(-lo, -lo)), q = q4_mul(r, q4_two(inv, inv));
    const uint64_t t = q4_add(q4_fma(q4_fma(q4_two(-step, -step), q, r), q4_two(inv, inv), q), q4_two(MAGIC, MAGIC));
    uint32_t t0, t1;
    q4_split(t, t0, t1);
    code += t0 * (1u << (4 * j)) + t1 * (16u << (4 * j));
  }
  return code - (HIGH + (HIGH << 4) + (HIGH << 8) + (HIGH << 12) + (HIGH << 16) + (HIGH << 20) + (HIGH << 24) + (HIGH << 28));
}

template <int D, int G>
__global__ void __launch_bounds__(Q4_THREADS) k_paged_append_q4(Q4Rows a, const __nv_bfloat16* k, const __nv_bfloat16* v) {
  using L = Q4Lane<D, G>;
  using T = Q4Tile<D, G>;
  pdl_wait();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * Q4_THREADS + threadIdx.x, n = i >> a.lanes;
  const int lanes = 1 << a.lanes, sub = static_cast<int>(i) & (lanes - 1), words = a.hkv * L::LANES;
  const int slot = n < a.N ? a.slots[n] : -1;
  uint8_t* tile = q4_tile<T>(a, slot, sub == 0);
  const int row = slot & 7;
  const __nv_bfloat16 *kr = k + n * a.k_stride, *vr = v + n * a.v_stride;
  const int64_t per_head = static_cast<int64_t>(T::BYTES) << a.shift >> 3;
  // (every lane of a warp goes round as often: the groups' exchanges need them all)
  for (int c0 = 0; c0 < words; c0 += L::CHUNKS * lanes) {
    uint4 ku[L::CHUNKS] = {}, vu[L::CHUNKS] = {};
#pragma unroll
    for (int j = 0; j < L::CHUNKS; ++j) {
      const int c = c0 + j * lanes + sub;
      if (tile != nullptr && c < words) {
        ku[j] = *reinterpret_cast<const uint4*>(kr + c * 8);
        vu[j] = *reinterpret_cast<const uint4*>(vr + c * 8);
      }
    }
    if (c0 + L::CHUNKS * lanes >= words) pdl_trigger();
#pragma unroll
    for (int j = 0; j < L::CHUNKS; ++j) {
      const int c = c0 + j * lanes + sub, t = c % L::LANES;
      if (c0 + j * lanes >= words) break;
      uint32_t kp, vp;
      const uint32_t kc = q4_quantise<L::GL>(ku[j], &kp), vc = L::exchange(q4_quantise<L::GL>(vu[j], &vp), t);
      if (tile == nullptr || c >= words) continue;
      uint8_t* at = tile + (c / L::LANES) * per_head;
      *reinterpret_cast<uint32_t*>(at + T::K + row * T::CODES + L::key_word(t)) = kc;
      *reinterpret_cast<uint32_t*>(at + T::V + row * T::CODES + L::value_word(t)) = vc;
      if (t % L::GL == 0) {
        *reinterpret_cast<uint32_t*>(at + T::KP + row * T::PARAMS + t / L::GL * 4) = kp;
        *reinterpret_cast<uint32_t*>(at + T::VP + row * T::PARAMS + t / L::GL * 4) = vp;
      }
    }
  }
}

// low + step * code of eight codes, the lowest bits first, as bf16.
__device__ __forceinline__ uint4 q4_values8(uint32_t code, uint32_t params) {
  const float step = bf16_lo(params), lo = bf16_hi(params);
  float x[8];
  const uint32_t high = code >> 16;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    // 2^23 + code 2^s of a code masked in place, back to the code
    const uint32_t w = j < 4 ? code : high;
    constexpr uint32_t BASE = 0x4b000000u;
    const int s = 4 * (j & 3);
    const float f = 1.f / (1 << s), f1 = f / 16.f;
    const uint64_t at = q4_two((w & (15u << s)) | BASE, (w & (240u << s)) | BASE);
    const uint64_t q = q4_fma(at, q4_two(f, f1), q4_two(-8388608.f * f, -8388608.f * f1));
    uint32_t a, b;
    q4_split(q4_fma(q4_two(step, step), q, q4_two(lo, lo)), a, b);
    x[j] = __uint_as_float(a);
    x[j + 1] = __uint_as_float(b);
  }
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// (sixteen blocks an SM, so 32 registers: with the 40 that it would take 9.8 us for 16381 rows, not 9.25. The store's 50
// squeezed to 40 took 12.6 there, not 13.0, but 9.1, not 8.2, for 5000 rows of 8 heads of 128)
template <int D, int G>
__global__ void __launch_bounds__(Q4_THREADS, 16) k_paged_read_q4(Q4Rows a, __nv_bfloat16* k, __nv_bfloat16* v) {
  using L = Q4Lane<D, G>;
  using T = Q4Tile<D, G>;
  pdl_wait();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * Q4_THREADS + threadIdx.x, n = i >> a.lanes;
  const int lanes = 1 << a.lanes, sub = static_cast<int>(i) & (lanes - 1), words = a.hkv * L::LANES;
  const int slot = n < a.N ? a.slots[n] : -1;
  const uint8_t* tile = q4_tile<T>(a, slot, sub == 0);
  const int row = slot & 7;
  __nv_bfloat16 *kr = k + n * a.k_stride, *vr = v + n * a.v_stride;
  const int64_t per_head = static_cast<int64_t>(T::BYTES) << a.shift >> 3;
  for (int c0 = 0; c0 < words; c0 += L::CHUNKS * lanes) {
    uint32_t kc[L::CHUNKS], vc[L::CHUNKS], kp[L::CHUNKS], vp[L::CHUNKS];
#pragma unroll
    for (int j = 0; j < L::CHUNKS; ++j) {
      const int c = c0 + j * lanes + sub, t = c % L::LANES;
      kc[j] = vc[j] = kp[j] = vp[j] = 0;
      if (tile != nullptr && c < words) {
        const uint8_t* at = tile + (c / L::LANES) * per_head;
        kc[j] = *reinterpret_cast<const uint32_t*>(at + T::K + row * T::CODES + L::key_word(t));
        vc[j] = *reinterpret_cast<const uint32_t*>(at + T::V + row * T::CODES + L::value_word(t));
        kp[j] = *reinterpret_cast<const uint32_t*>(at + T::KP + row * T::PARAMS + t / L::GL * 4);
        vp[j] = *reinterpret_cast<const uint32_t*>(at + T::VP + row * T::PARAMS + t / L::GL * 4);
      }
    }
    if (c0 + L::CHUNKS * lanes >= words) pdl_trigger();
#pragma unroll
    for (int j = 0; j < L::CHUNKS; ++j) {
      const int c = c0 + j * lanes + sub;
      if (c0 + j * lanes >= words) break;
      const uint32_t w = L::exchange(vc[j], c % L::LANES);
      if (tile == nullptr || c >= words) continue;
      *reinterpret_cast<uint4*>(kr + c * 8) = q4_values8(kc[j], kp[j]);
      *reinterpret_cast<uint4*>(vr + c * 8) = q4_values8(w, vp[j]);
    }
  }
}

// The checks that the two calls share, and their arguments.
static int q4_rows(const char* name, const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride, int64_t N,
                   int Hkv, int D, int group, const int32_t* slot_map, const void* pages, int64_t num_pages,
                   int page_size, int64_t page_stride, int32_t* status_dev, Q4Rows* a) {
  DM_ARG_CHECK(q4_shape_ok(D, group), "%s: D 64 with groups of 32 or 64, or D 128 with groups of 32, 64 or 128", name);
  DM_ARG_CHECK(N >= 0 && N <= INT_MAX && Hkv >= 1 && Hkv <= 1024, "%s: bad sizes", name);
  DM_ARG_CHECK(page_size >= 8 && (page_size & (page_size - 1)) == 0, "%s: page_size must be a power of two, 8 at least", name);
  DM_ARG_CHECK(num_pages >= 0 && num_pages <= INT_MAX / page_size, "%s: num_pages * page_size must be below 2^31", name);
  const int64_t page = q4_tile_bytes(D, group) * (page_size / 8) * Hkv;
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
  a->lanes = 3;  // the least power of two that covers a row, at most a warp
  while (a->lanes < 5 && (1 << a->lanes) < Hkv * (D / 8)) ++a->lanes;
  return DECOMOE_OK;
}

static Bytes q4_pool(const void* pages, int64_t num_pages, int page_size, int64_t page_stride, int Hkv, int D, int group) {
  const int64_t page = q4_tile_bytes(D, group) * (page_size / 8) * Hkv;
  return {pages, num_pages == 0 ? 0 : static_cast<size_t>((num_pages - 1) * page_stride + page)};
}

}  // namespace decomoe

using namespace decomoe;

extern "C" {

size_t decomoe_paged_q4_page_bytes(int page_size, int Hkv, int D, int group) {
  if (page_size < 8 || (page_size & (page_size - 1)) != 0 || Hkv < 1 || Hkv > 1024 || !q4_shape_ok(D, group)) return 0;
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
  const int64_t grid = ((N << a.lanes) + Q4_THREADS - 1) / Q4_THREADS;
  return q4_dispatch(D, group, [&](auto d, auto g) -> int {
    DM_CUDA_CHECK(launch_pdl_late(k_paged_append_q4<d.value, g.value>, dim3(static_cast<unsigned>(grid)), dim3(Q4_THREADS), 0,
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
  const int64_t grid = ((N << a.lanes) + Q4_THREADS - 1) / Q4_THREADS;
  return q4_dispatch(D, group, [&](auto d, auto g) -> int {
    DM_CUDA_CHECK(launch_pdl_late(k_paged_read_q4<d.value, g.value>, dim3(static_cast<unsigned>(grid)), dim3(Q4_THREADS), 0,
                                  reinterpret_cast<cudaStream_t>(stream), a, static_cast<__nv_bfloat16*>(k_out),
                                  static_cast<__nv_bfloat16*>(v_out)));
    return DECOMOE_OK;
  });
}

}  // extern "C"
