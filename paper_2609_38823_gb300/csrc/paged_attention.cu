// Attention of one new token per request over a paged key-value cache (decoding
// on the text-only cache, DecoMoE Section 3.2 and Algorithm 2, last step, for a
// batch of requests), the visual block of a request left out where it has exited.
#include <cfloat>

#include "decomoe_internal.cuh"

namespace decomoe {

struct PagedArgs {
  const __nv_bfloat16* q;
  const __nv_bfloat16 *k, *v;
  const int32_t *table, *len, *hide_begin, *hide_count;
  __nv_bfloat16* out;
  int32_t* status;
  int64_t q_stride, page_stride, num_pages, max_pages;
  int B, hq, hkv, shift;
  float sl2;  // scale * log2(e)
};

// One block per (request, query head), a warp every eighth visible key.
template <int D>
__global__ void __launch_bounds__(256) k_paged_attention(PagedArgs a) {
  constexpr int PER = D / 32;
  __shared__ float sm[8], sl[8], so[8][D];
  pdl_enter();
  const int b = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t cap = a.max_pages << a.shift;
  int64_t n = a.len[b];
  if (threadIdx.x == 0 && (n < 0 || n > cap)) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
  n = min(max(n, int64_t{0}), cap);
  int64_t h0 = n, hc = 0;
  if (a.hide_begin != nullptr) {
    h0 = min(max(static_cast<int64_t>(a.hide_begin[b]), int64_t{0}), n);
    hc = min(max(static_cast<int64_t>(a.hide_count[b]), int64_t{0}), n - h0);
  }
  const int64_t seen = n - hc;
  const int g = h / (a.hq / a.hkv);
  float q[PER], o[PER] = {};
  for (int i = 0; i < PER; ++i) q[i] = __bfloat162float(a.q[b * a.q_stride + h * D + lane * PER + i]);
  float m = -INFINITY, l = 0.f;
  for (int64_t j = warp; j < seen; j += 8) {
    const int64_t p = j < h0 ? j : j + hc;
    const int64_t page = a.table[b * a.max_pages + (p >> a.shift)];
    if (page < 0 || page >= a.num_pages) {
      if (lane == 0) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
      continue;
    }
    const int64_t at = page * a.page_stride +
                       ((p & ((int64_t{1} << a.shift) - 1)) * a.hkv + g) * D + lane * PER;
    float s = 0.f;
    for (int i = 0; i < PER; ++i) s = fmaf(q[i], __bfloat162float(a.k[at + i]), s);
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    s *= a.sl2;
    const float mn = fmaxf(m, s), ref = mn == -INFINITY ? 0.f : mn;
    const float f = exp2f(m - ref), w = exp2f(s - ref);
    l = l * f + w;
    for (int i = 0; i < PER; ++i) o[i] = o[i] * f + w * __bfloat162float(a.v[at + i]);
    m = mn;
  }
  if (lane == 0) {
    sm[warp] = m;
    sl[warp] = l;
  }
  for (int i = 0; i < PER; ++i) so[warp][lane * PER + i] = o[i];
  __syncthreads();
  for (int c = threadIdx.x; c < D; c += blockDim.x) {
    float mm = -INFINITY;
    for (int w = 0; w < 8; ++w) mm = fmaxf(mm, sm[w]);
    const float ref = mm == -INFINITY ? 0.f : mm;
    float ll = 0.f, oo = 0.f;
    for (int w = 0; w < 8; ++w) {
      const float f = exp2f(sm[w] - ref);
      ll += sl[w] * f;
      oo += so[w][c] * f;
    }
    a.out[(static_cast<int64_t>(b) * a.hq + h) * D + c] = __float2bfloat16_rn(ll != 0.f ? oo / ll : 0.f);
  }
}

}  // namespace decomoe

using namespace decomoe;

extern "C" {

size_t decomoe_paged_attention_workspace_bytes(int64_t B, int Hq, int Hkv, int D) {
  if (B <= 0 || Hkv <= 0 || Hq < Hkv || D <= 0) return 0;
  return 256;
}

int decomoe_paged_attention(const void* q, int64_t q_stride, int64_t B, const void* k_pages, const void* v_pages,
                            int64_t num_pages, int page_size, int64_t page_stride, const int32_t* block_table,
                            int64_t max_pages, const int32_t* seq_len, const int32_t* hide_begin,
                            const int32_t* hide_count, int Hq, int Hkv, int D, float scale, void* out, void* ws,
                            size_t ws_bytes, int32_t* status_dev, decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(B >= 0 && B <= DECOMOE_MAX_REQUESTS, "paged_attention: B must lie in [0, %d]", DECOMOE_MAX_REQUESTS);
  DM_ARG_CHECK(D == 64 || D == 128, "paged_attention: D must be 64 or 128");
  DM_ARG_CHECK(Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0, "paged_attention: Hq must be a multiple of Hkv");
  DM_ARG_CHECK(Hq <= 1024, "paged_attention: more than 1024 query heads");
  DM_ARG_CHECK(page_size >= 1 && (page_size & (page_size - 1)) == 0,
               "paged_attention: page_size must be a power of two");
  DM_ARG_CHECK(num_pages >= 0 && num_pages <= INT_MAX / page_size,
               "paged_attention: num_pages * page_size must be below 2^31");
  DM_ARG_CHECK(max_pages >= 0 && max_pages <= INT_MAX / page_size,
               "paged_attention: max_pages * page_size must be below 2^31");
  DM_ARG_CHECK(page_stride >= static_cast<int64_t>(page_size) * Hkv * D && page_stride % 8 == 0,
               "paged_attention: page_stride must be at least page_size * Hkv * D and a multiple of 8");
  DM_ARG_CHECK(q_stride >= static_cast<int64_t>(Hq) * D && q_stride % 8 == 0,
               "paged_attention: q_stride must be at least Hq * D and a multiple of 8");
  DM_ARG_CHECK((hide_begin == nullptr) == (hide_count == nullptr),
               "paged_attention: hide_begin and hide_count go together");
  if (B == 0) return DECOMOE_OK;
  DM_ARG_CHECK(q && seq_len && out && (max_pages == 0 || block_table) && (num_pages == 0 || (k_pages && v_pages)),
               "paged_attention: null pointer");
  DM_ARG_CHECK(aligned16(q) && aligned16(k_pages) && aligned16(v_pages) && aligned16(out),
               "paged_attention: pointers must be 16-byte aligned");
  if (ws == nullptr || ws_bytes < decomoe_paged_attention_workspace_bytes(B, Hq, Hkv, D)) {
    set_error("paged_attention: workspace of %zu bytes needed",
              decomoe_paged_attention_workspace_bytes(B, Hq, Hkv, D));
    return DECOMOE_ERR_WORKSPACE;
  }
  DM_ARG_CHECK(aligned16(ws), "paged_attention: workspace must be 16-byte aligned");
  PagedArgs a = {};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k = static_cast<const __nv_bfloat16*>(k_pages);
  a.v = static_cast<const __nv_bfloat16*>(v_pages);
  a.table = block_table;
  a.len = seq_len;
  a.hide_begin = hide_begin;
  a.hide_count = hide_count;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.status = status_dev;
  a.q_stride = q_stride;
  a.page_stride = page_stride;
  a.num_pages = num_pages;
  a.max_pages = max_pages;
  a.B = static_cast<int>(B);
  a.hq = Hq;
  a.hkv = Hkv;
  a.shift = __builtin_ctz(static_cast<unsigned>(page_size));
  a.sl2 = (scale > 0.f ? scale : 1.f / sqrtf(static_cast<float>(D))) * 1.4426950408889634f;
  DM_CUDA_CHECK(launch_pdl(D == 128 ? k_paged_attention<128> : k_paged_attention<64>,
                           dim3(static_cast<unsigned>(B), static_cast<unsigned>(Hq)), dim3(256), 0,
                           reinterpret_cast<cudaStream_t>(stream), a));
  return DECOMOE_OK;
}

}  // extern "C"
