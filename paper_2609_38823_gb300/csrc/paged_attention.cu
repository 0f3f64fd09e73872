// Attention of one new token per request over a paged key-value cache (decoding
// on the text-only cache, DecoMoE Section 3.2 and Algorithm 2, last step, for a
// batch of requests), the visual block of a request left out where it has exited.
#include "paged_share.cuh"

namespace decomoe {

// The visible keys of every (request, KV head) pair are cut into tiles (16 keys
// of 128 features, 32 of 64), the tiles of all pairs are numbered in order, and
// every warp of the launch takes the same number of consecutive tiles, one block
// of eight warps per SM, whatever the lengths are. A warp streams its tiles
// through a ring of its own (16-byte asynchronous copies, row by row through the
// block table, three tiles of 8 KB) and meets no other warp until it has read its
// last tile. Where a pair's tiles end inside a warp's share the result goes
// straight out; what a warp holds of a pair that goes on in another warp is joined
// in key order, first among the warps of the block, then, by a second small
// launch, among the blocks. No counters, and the result does not depend on timing.
//
// Both products run transposed on the tensor cores (mma.m16n8k16, bf16 in, fp32
// accumulate): S^T = K Q^T with 16 keys by 8 queries, O^T += V^T P^T with 16
// features by 8 queries, so that the 8 query heads of a KV head fill a tile (16
// rows by 8 keys would leave half of each product empty). The accumulator of the
// first becomes the operand of the second by two 8x8 transposes (movmatrix), and
// a query's maximum, sum and outputs all lie in the same lanes. Scores, maxima, sums and
// outputs are fp32; the weights are rounded to bf16 as operands of the second product
// (the values are bf16, and the two must be of one type): 2^-9 of a weight at most,
// relative errors of 0.0022 after the output's own rounding, which alone gives 0.0017.
//
// Bound: the stream of keys and values. 96 requests of 2000 to 16385 rows (545 MB) 95 us:
// 6.2 TB/s but for the 3 us before the first tile and the 4 us of the joins. One request of
// 2049 rows 8.6 us, all of it latency: of the scan and the search in front, and of the second
// launch behind (the contiguous kernel of attention.cu, which has neither, takes 5.0).
constexpr int PGA_WARPS = 8;
constexpr int PGA_THREADS = 32 * PGA_WARPS;
constexpr int PGA_STAGES = 3;
constexpr int PGA_BLOCKS = 160;  // of a launch, at most
constexpr int PGA_STAGE = 8192;  // bytes of one tile: keys, then values
constexpr int PGA_EXTRA = 3;     // what a (request, KV head) pair costs beside its tiles, in tiles

template <int D>
struct PgaTile {
  static constexpr int KEYS = PGA_STAGE / (4 * D);  // 16 or 32
  static constexpr int VECS = D / 8;                // 16-byte pieces of a row
  static constexpr int ROW = pga_row(D);
  static __device__ __forceinline__ int count(const PgaReq& r) { return (r.seen + KEYS - 1) / KEYS; }
};

struct PagedArgs : PagedCommon {
  const __nv_bfloat16 *k, *v;
};

__device__ __forceinline__ void pga_ldsm(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void pga_ldsm_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
// 16 bytes into shared memory, zeros where !ok (src is then not read).
__device__ __forceinline__ void pga_copy(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}

template <int D, int NT>
__global__ void __launch_bounds__(PGA_THREADS, 1) k_paged_attention(PagedArgs a) {
  using T = PgaTile<D>;
  constexpr int KS = D / 16;     // 16-feature steps of the scores, and 16-feature tiles of the outputs
  constexpr int SUB = T::KEYS / 16;
  constexpr int ROWS = 8 * NT;
  extern __shared__ __align__(1024) uint8_t pga_smem[];
  __shared__ uint32_t seen_mask[PGA_WARPS][PGA_STAGES];
  __shared__ int3 meta[PGA_WARPS];  // last piece goes on (1: begun in the share, 2: before it), its request and head tile
  int* pre = reinterpret_cast<int*>(pga_smem + PGA_WARPS * PGA_STAGES * PGA_STAGE);
  int* nz = pre + a.B + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_enter();
  const PgaPlan plan = pga_begin<T, D, PGA_WARPS>(a, pre, nz);
  const int me = blockIdx.x * PGA_WARPS + warp;
  // lane 0 seeks the start of this warp's share, lane 1 that of the next one's
  PgaWalk<T> look;
  const int from = plan.place(me + (lane & 1));
  const int first = from < plan.total ? look.seek(plan, from) : pre[a.B] * a.hv;
  const int r0 = __shfl_sync(0xffffffffu, first, 0), r1 = __shfl_sync(0xffffffffu, first, 1);
  const int gs = a.hq / a.hkv;

  uint8_t* ring = pga_smem + warp * PGA_STAGES * PGA_STAGE;
  const uint32_t ring_s = smem_u32(ring);
  float* mine = reinterpret_cast<float*>(ring);  // the last piece, once the ring is drained
  if (lane == 0) meta[warp] = make_int3(0, 0, 0);
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * ROWS * T::ROW;

  if (r0 < r1) {
    // ---- lookup, copy and use, each at its own tile
    look.b = __shfl_sync(0xffffffffu, look.b, 0);
    look.h = __shfl_sync(0xffffffffu, look.h, 0);
    look.t = __shfl_sync(0xffffffffu, look.t, 0);
    look.enter(a);
    PgaWalk<T> use = look;
    const int64_t row_elems = static_cast<int64_t>(a.hkv) * D;
    const int in_page = (1 << a.shift) - 1;
    int page = -1, off = 0, head = 0;
    bool want = false;
    auto lookup = [&]() {  // the page of this lane's key
      const int j = look.t * T::KEYS + lane;
      want = lane < T::KEYS && j < look.r.seen;
      const int p = j < look.r.h0 ? j : j + look.r.hc;
      off = p & in_page;
      head = look.h / a.qt;
      if (want) page = a.table[look.b * a.max_pages + (p >> a.shift)];
    };
    // places in a tile, the 16-byte pieces of row r exchanged by r's low three bits: of what
    // this lane copies, and of its row of the operands of the two products
    const uint32_t copy_at = (lane >> 2) * (2 * D) + (((lane & 3) ^ (lane >> 2)) << 4);
    const uint32_t k_at = (lane & 15) * (2 * D) + (((lane >> 4) ^ (lane & 7)) << 4);
    const uint32_t v_at = (((lane >> 4) << 3) + (lane & 7)) * (2 * D) + ((((lane >> 3) & 1) ^ (lane & 7)) << 4);
    auto issue = [&](int slot) {
      const bool there = want && page >= 0 && page < a.num_pages;
      if (want && !there) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
      const uint32_t mask = __ballot_sync(0xffffffffu, there);
      if (lane == 0) seen_mask[warp][slot] = mask;
      // four lanes to a row, 64 bytes of eight rows at a time
      constexpr int SETS = T::KEYS / 8, GROUPS = T::VECS / 4;
      const int64_t base = there ? page * a.page_stride + off * row_elems + static_cast<int64_t>(head) * D : -1;
      const uint32_t stage = ring_s + slot * PGA_STAGE;
#pragma unroll
      for (int i = 0; i < SETS; ++i) {
        const int64_t at = __shfl_sync(0xffffffffu, base, i * 8 + (lane >> 2));
        const bool ok = at >= 0;
        const int64_t e = (ok ? at : 0) + (lane & 3) * 8;
        const __nv_bfloat16 *k = a.k + e, *v = a.v + e;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
          const uint32_t dst = stage + i * (8 * 2 * D) + (copy_at ^ (g << 6));
          pga_copy(dst, k + g * 32, ok);
          pga_copy(dst + PGA_STAGE / 2, v + g * 32, ok);
        }
      }
    };
    const int n = r1 - r0;
    lookup();

    uint32_t qf[NT][KS][2];
    float o[KS][NT][4], m[NT][2], l[NT][2];
    auto begin_piece = [&]() {
      const int g = use.h / a.qt, q0 = (use.h - g * a.qt) * ROWS;
      const __nv_bfloat16* q = a.q + use.b * a.q_stride + static_cast<int64_t>(g) * gs * D;
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const int r = q0 + x * 8 + (lane >> 2);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            qf[x][s][i] = r < gs ? *reinterpret_cast<const uint32_t*>(q + static_cast<int64_t>(r) * D + s * 16 +
                                                                      i * 8 + 2 * (lane & 3))
                                 : 0u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          m[x][i] = -INFINITY;
          l[x][i] = 0.f;
        }
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[s][x][i] = 0.f;
      }
    };
    // a finished piece as partial rows
    auto keep_piece = [&](float* dst) {
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float* row = dst + (x * 8 + 2 * (lane & 3) + i) * T::ROW;
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            row[s * 16 + (lane >> 2)] = o[s][x][i];
            row[s * 16 + 8 + (lane >> 2)] = o[s][x][i + 2];
          }
          if (lane < 4) {
            row[D] = m[x][i];
            row[D + 1] = l[x][i];
          }
        }
    };
    bool began = use.t > 0;  // the piece's pair began in an earlier share
    int slot = 0, fill = 0;
    // the first steps only fill the ring (one copy of the code: a short share runs it cold)
    for (int i = 1 - PGA_STAGES; i < n; ++i) {
      if (i + PGA_STAGES - 1 < n) {
        issue(fill);
        fill = fill + 1 == PGA_STAGES ? 0 : fill + 1;
        if (i + PGA_STAGES < n) {
          look.next(a, pre);
          lookup();
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      if (i < 0) {
        if (i == -1) begin_piece();
        continue;
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(PGA_STAGES - 1) : "memory");
      __syncwarp();
      const uint32_t ks = ring_s + slot * PGA_STAGE, vs = ks + PGA_STAGE / 2;
      const uint32_t mask = seen_mask[warp][slot];
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        float sc[NT][4] = {}, odd[NT][4] = {};  // even and odd steps: two chains of products
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          uint32_t f[4];
          pga_ldsm(ks + u * (16 * 2 * D) + (k_at ^ (s << 5)), f);
#pragma unroll
          for (int x = 0; x < NT; ++x) pga_mma(s & 1 ? odd[x] : sc[x], f, qf[x][s][0], qf[x][s][1]);
        }
        const bool lo = (mask >> (u * 16 + (lane >> 2))) & 1u, hi = (mask >> (u * 16 + 8 + (lane >> 2))) & 1u;
        uint32_t p[NT][2];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          float mx[2];
#pragma unroll
          for (int i2 = 0; i2 < 2; ++i2) {
            sc[x][i2] = lo ? (sc[x][i2] + odd[x][i2]) * a.sl2 : -INFINITY;
            sc[x][i2 + 2] = hi ? (sc[x][i2 + 2] + odd[x][i2 + 2]) * a.sl2 : -INFINITY;
            mx[i2] = fmaxf(sc[x][i2], sc[x][i2 + 2]);
          }
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) {
            mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], w));
            mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], w));
          }
          if (__any_sync(0xffffffffu, mx[0] > m[x][0] || mx[1] > m[x][1])) {
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
              const float to = fmaxf(m[x][i2], mx[i2]);
              // nothing seen so far, and nothing here: any factor does
              const float f = to == -INFINITY ? 1.f : pga_ex2(m[x][i2] - to);
              m[x][i2] = to;
              l[x][i2] *= f;
#pragma unroll
              for (int s = 0; s < KS; ++s) {
                o[s][x][i2] *= f;
                o[s][x][i2 + 2] *= f;
              }
            }
          }
          float w[4];
#pragma unroll
          for (int i2 = 0; i2 < 4; ++i2) {
            const float ref = m[x][i2 & 1] == -INFINITY ? 0.f : m[x][i2 & 1];
            w[i2] = pga_ex2(sc[x][i2] - ref);
          }
          l[x][0] += w[0] + w[2];
          l[x][1] += w[1] + w[3];
          p[x][0] = pga_transpose(pack_bf16x2(w[0], w[1]));
          p[x][1] = pga_transpose(pack_bf16x2(w[2], w[3]));
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          uint32_t f[4];
          pga_ldsm_t(vs + u * (16 * 2 * D) + (v_at ^ (s << 5)), f);
#pragma unroll
          for (int x = 0; x < NT; ++x) pga_mma(o[s][x], f, p[x][0], p[x][1]);
        }
      }
      __syncwarp();
      slot = slot + 1 == PGA_STAGES ? 0 : slot + 1;
      const bool ends = use.t + 1 == use.tiles;
      if (ends || i + 1 == n) {
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
          for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) l[x][i2] += __shfl_xor_sync(0xffffffffu, l[x][i2], w);
        if (!ends) {  // goes on in the next share; the ring is empty
          keep_piece(mine);
          if (lane == 0) meta[warp] = make_int3(began ? 2 : 1, use.b, use.h);
        } else if (began) {
          // begun before the block: it is all that the block holds of its pair
          keep_piece(warp == 0 ? part : a.early + static_cast<int64_t>(me) * ROWS * T::ROW);
        } else {
          const int g = use.h / a.qt, q0 = (use.h - g * a.qt) * ROWS;
#pragma unroll
          for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
              const int r = q0 + x * 8 + 2 * (lane & 3) + i2;
              if (r < gs) {
                const float f = l[x][i2] != 0.f ? 1.f / l[x][i2] : 0.f;
                __nv_bfloat16* dst = a.out + (static_cast<int64_t>(use.b) * a.hq + g * gs + r) * D + (lane >> 2);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                  dst[s * 16] = __float2bfloat16_rn(o[s][x][i2] * f);
                  dst[s * 16 + 8] = __float2bfloat16_rn(o[s][x][i2 + 2] * f);
                }
              }
            }
        }
        if (i + 1 < n) {
          use.next(a, pre);
          began = false;
          begin_piece();
        }
      } else {
        ++use.t;
      }
    }
  }
  __syncthreads();
  pga_join_block<D, NT, PGA_WARPS>(a, plan, meta, pga_smem, PGA_STAGES * PGA_STAGE);
}

}  // namespace decomoe

using namespace decomoe;

extern "C" {

size_t decomoe_paged_attention_workspace_bytes(int64_t B, int Hq, int Hkv, int D) {
  if (B <= 0 || Hkv <= 0 || Hq < Hkv || D <= 0) return 0;
  // the pieces of every warp and of every block, one block per SM
  const size_t rows = static_cast<size_t>(pga_rows(Hq, Hkv)) * (D + 4) * sizeof(float);
  return static_cast<size_t>(sm_count()) * ((PGA_WARPS + 2) * rows + sizeof(int4));
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
  // a length rounded up to a tile of (at most) 32 keys is counted in 32 bits
  DM_ARG_CHECK(max_pages >= 0 && max_pages <= (INT_MAX - 31) / page_size,
               "paged_attention: max_pages * page_size must be at most 2^31 - 32");
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
  {
    const size_t each = static_cast<size_t>(B) * sizeof(int32_t);
    const size_t pool = num_pages == 0 ? 0 : static_cast<size_t>((num_pages - 1) * page_stride + static_cast<int64_t>(page_size) * Hkv * D) * 2;
    const Bytes in[] = {{q, static_cast<size_t>((B - 1) * q_stride + static_cast<int64_t>(Hq) * D) * 2},
                        {k_pages, pool},
                        {v_pages, pool},
                        {block_table, each * static_cast<size_t>(max_pages)},
                        {seq_len, each},
                        {hide_begin, each},
                        {hide_count, each}};
    const Bytes o = {out, static_cast<size_t>(B) * Hq * D * 2}, w = {ws, decomoe_paged_attention_workspace_bytes(B, Hq, Hkv, D)};
    bool apart = !overlaps(o, {w});
    for (const Bytes& b : in) apart &= !overlaps(o, {b}) && !overlaps(w, {b});
    DM_ARG_CHECK(apart, "paged_attention: out or the workspace overlaps an input or one another");
  }
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
  const int rows = pga_rows(Hq, Hkv);
  a.qt = (Hq / Hkv + rows - 1) / rows;
  a.hv = Hkv * a.qt;
  a.sl2 = (scale > 0.f ? scale : 1.f / sqrtf(static_cast<float>(D))) * 1.4426950408889634f;
  const int keys = D == 128 ? PgaTile<128>::KEYS : PgaTile<64>::KEYS;
  const int64_t most = B * ((max_pages * page_size + keys - 1) / keys) * a.hv;  // tiles, at most
  DM_ARG_CHECK(most + PGA_EXTRA * B * a.hv <= INT_MAX, "paged_attention: B * max_pages * page_size * heads is too large");
  const int grid = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(std::min(sm_count(), PGA_BLOCKS), (most + PGA_WARPS - 1) / PGA_WARPS)));
  const size_t piece = static_cast<size_t>(rows) * (D + 4);
  a.early = static_cast<float*>(ws);
  a.part = a.early + static_cast<size_t>(grid) * PGA_WARPS * piece;
  a.info = reinterpret_cast<int4*>(a.part + static_cast<size_t>(grid) * 2 * piece);
  a.extra = PGA_EXTRA;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  auto smem = [](int64_t requests) {
    return static_cast<size_t>(PGA_WARPS) * PGA_STAGES * PGA_STAGE + 2 * (static_cast<size_t>(requests) + 1) * sizeof(int);
  };
  auto go = [&](auto main, auto join) -> int {
    // the limit belongs to the kernel, not to the call: one for every batch, or a smaller one on another thread
    // could lower it before this launch
    DM_CUDA_CHECK(cudaFuncSetAttribute(main, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(smem(DECOMOE_MAX_REQUESTS))));
    DM_CUDA_CHECK(launch_pdl(main, dim3(grid), dim3(PGA_THREADS), smem(B), s, a));
    DM_CUDA_CHECK(launch_pdl(join, dim3(grid), dim3(32 * PGM_WARPS), 0, s, static_cast<const PagedCommon&>(a)));
    return DECOMOE_OK;
  };
  if (D == 128)
    DM_RET(rows == 8 ? go(k_paged_attention<128, 1>, k_paged_join<128, 1, PGA_BLOCKS>)
                     : go(k_paged_attention<128, 2>, k_paged_join<128, 2, PGA_BLOCKS>));
  else
    DM_RET(rows == 8 ? go(k_paged_attention<64, 1>, k_paged_join<64, 1, PGA_BLOCKS>)
                     : go(k_paged_attention<64, 2>, k_paged_join<64, 2, PGA_BLOCKS>));
  return DECOMOE_OK;
}

}  // extern "C"
