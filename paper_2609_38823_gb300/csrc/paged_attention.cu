// Attention of one new token per request over a paged key-value cache (decoding
// on the text-only cache, DecoMoE Section 3.2 and Algorithm 2, last step, for a
// batch of requests), the visual block of a request left out where it has exited.
#include <cfloat>

#include "decomoe_internal.cuh"

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
  static constexpr int ROW = D + 4;                 // floats of a partial row: outputs, m, l (bank-conflict-free stores)
};

struct PagedArgs {
  const __nv_bfloat16* q;
  const __nv_bfloat16 *k, *v;
  const int32_t *table, *len, *hide_begin, *hide_count;
  __nv_bfloat16* out;
  float* early;  // [warps][rows][ROW] pieces that end inside a warp's share
  float* part;   // [blocks][2][rows][ROW] joined pieces of a block: of a pair begun before it, of one that goes on after it
  int4* info;    // [blocks] the pair that begins in a block and ends in a later one: (valid, request, head tile, last block)
  int32_t* status;
  int64_t q_stride, page_stride, num_pages, max_pages;
  int B, hq, hkv, shift;
  int qt, hv;    // query tiles per KV head, (KV head, query tile) pairs
  int extra;     // what a pair costs beside its tiles, in tiles
  float sl2;     // scale * log2(e)
};

// What a request shows: its visible rows, and where its hidden block lies.
struct PgaReq {
  int seen, h0, hc;
};
__device__ __forceinline__ PgaReq pga_request(const PagedArgs& a, int b, bool* bad) {
  const int cap = static_cast<int>(a.max_pages << a.shift);
  int n = a.len[b];
  *bad |= n < 0 || n > cap;
  n = min(max(n, 0), cap);
  PgaReq r;
  r.h0 = n;
  r.hc = 0;
  if (a.hide_begin != nullptr) {
    r.h0 = min(max(a.hide_begin[b], 0), n);
    r.hc = min(max(a.hide_count[b], 0), n - r.h0);
  }
  r.seen = n - r.hc;
  return r;
}

// How the tiles are shared out. A pair costs `extra` more than its tiles (its
// lengths, queries and result go over latencies that its tiles' copies do not hide),
// so warps get equal shares of tiles + extra: places of a line on which every pair
// takes tiles + extra of them, the first `extra` belonging to its first tile.
struct PgaPlan {
  const int* pre;  // [B + 1] tiles per head tile before a request
  const int* nz;   // [B + 1] requests that see something before a request
  int B, hv, extra;
  int total;       // places in all
  int per, more;   // places of a warp, and how many warps take one more
  __device__ __forceinline__ int places(int b) const {  // before request b
    return (pre[b] + nz[b] * extra) * hv;
  }
  __device__ __forceinline__ void divide(int workers) {
    total = places(B);
    per = total / workers;
    more = total - per * workers;
  }
  __device__ __forceinline__ int place(int i) const { return i * per + min(i, more); }  // the first one of warp i
  __device__ __forceinline__ int holder(int p) const {  // the warp whose share holds place p
    const int full = more * (per + 1);
    return p < full ? p / (per + 1) : more + (p - full) / per;
  }
};

__device__ __forceinline__ float pga_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
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
__device__ __forceinline__ uint32_t pga_transpose(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void pga_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes into shared memory, zeros where !ok (src is then not read).
__device__ __forceinline__ void pga_copy(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}

// The C floats (2 or 4) of a partial row that a lane holds.
template <int C>
struct PgaVec {
  float v[C];
};
template <bool PAST_L1, int C>
__device__ __forceinline__ void pga_load(PgaVec<C>& d, const float* p) {
  if constexpr (C == 4) {
    const float4 u = PAST_L1 ? __ldcg(reinterpret_cast<const float4*>(p)) : *reinterpret_cast<const float4*>(p);
    d.v[0] = u.x, d.v[1] = u.y, d.v[2] = u.z, d.v[3] = u.w;
  } else {
    const float2 u = PAST_L1 ? __ldcg(reinterpret_cast<const float2*>(p)) : *reinterpret_cast<const float2*>(p);
    d.v[0] = u.x, d.v[1] = u.y;
  }
}
template <int C>
__device__ __forceinline__ void pga_store(float* p, const PgaVec<C>& d) {
  if constexpr (C == 4) *reinterpret_cast<float4*>(p) = make_float4(d.v[0], d.v[1], d.v[2], d.v[3]);
  else *reinterpret_cast<float2*>(p) = make_float2(d.v[0], d.v[1]);
}
// The result: the outputs over the sum (nothing seen: zeros), as bf16.
template <int C>
__device__ __forceinline__ void pga_result(__nv_bfloat16* dst, const PgaVec<C>& o, float l) {
  const float f = l != 0.f ? 1.f / l : 0.f;
  if constexpr (C == 4)
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o.v[0] * f, o.v[1] * f), pack_bf16x2(o.v[2] * f, o.v[3] * f));
  else
    *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(o.v[0] * f, o.v[1] * f);
}

// A position in the numbered tiles: tile t of pair (request b, head tile h).
template <int D>
struct PgaWalk {
  int b, h, t, tiles;
  PgaReq r;
  __device__ __forceinline__ void enter(const PagedArgs& a) {
    bool bad = false;  // marked by the launch's first look at the lengths
    r = pga_request(a, b, &bad);
    tiles = (r.seen + PgaTile<D>::KEYS - 1) / PgaTile<D>::KEYS;
  }
  // To the first tile at or after place p (p < total); its number over all pairs.
  __device__ __forceinline__ int seek(const PgaPlan& plan, int p) {
    int lo = 0, hi = plan.B;  // the last request with places <= p: it is not empty
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.places(mid) <= p) lo = mid;
      else hi = mid;
    }
    b = lo;
    tiles = plan.pre[b + 1] - plan.pre[b];
    const int in = p - plan.places(b), each = tiles + plan.extra;
    h = in / each;
    t = max(in - h * each - plan.extra, 0);
    return plan.pre[b] * plan.hv + h * tiles + t;
  }
  // To the next tile; in the last pair it stays past the end (nobody looks).
  __device__ __forceinline__ void next(const PagedArgs& a, const int* pre) {
    if (++t < tiles) return;
    t = 0;
    if (++h < a.hv) return;
    h = 0;
    do ++b;
    while (b < a.B && pre[b + 1] == pre[b]);
    if (b < a.B) enter(a);
  }
};

template <int D, int NT>
__global__ void __launch_bounds__(PGA_THREADS, 1) k_paged_attention(PagedArgs a) {
  using T = PgaTile<D>;
  constexpr int KS = D / 16;     // 16-feature steps of the scores, and 16-feature tiles of the outputs
  constexpr int SUB = T::KEYS / 16;
  constexpr int ROWS = 8 * NT;
  extern __shared__ __align__(1024) uint8_t pga_smem[];
  __shared__ int scan_w[2][PGA_WARPS];
  __shared__ uint32_t seen_mask[PGA_WARPS][PGA_STAGES];
  __shared__ int3 meta[PGA_WARPS];  // last piece goes on (1: begun in the share, 2: before it), its request and head tile
  int* pre = reinterpret_cast<int*>(pga_smem + PGA_WARPS * PGA_STAGES * PGA_STAGE);
  int* nz = pre + a.B + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_enter();

  // ---- tiles of every request, added up
  {
    const int per = (a.B + PGA_THREADS - 1) / PGA_THREADS;
    const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    bool bad = false;
    int sum = 0, some = 0;
    for (int b = b0; b < b1; ++b) {
      const int n = (pga_request(a, b, &bad).seen + T::KEYS - 1) / T::KEYS;
      pre[b + 1] = n;
      sum += n;
      some += n > 0;
    }
    if (bad && blockIdx.x == 0) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
    int inc = sum, inn = some;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, inc, o), v = __shfl_up_sync(0xffffffffu, inn, o);
      if (lane >= o) {
        inc += u;
        inn += v;
      }
    }
    if (lane == 31) {
      scan_w[0][warp] = inc;
      scan_w[1][warp] = inn;
    }
    __syncthreads();
    int at = inc - sum, an = inn - some;
#pragma unroll
    for (int w = 0; w < PGA_WARPS; ++w)
      if (w < warp) {
        at += scan_w[0][w];
        an += scan_w[1][w];
      }
    for (int b = b0; b < b1; ++b) {
      an += pre[b + 1] > 0;
      at += pre[b + 1];
      pre[b + 1] = at;
      nz[b + 1] = an;
    }
    if (tid == 0) pre[0] = nz[0] = 0;
    __syncthreads();
  }
  // requests that see nothing
  for (int b = blockIdx.x; b < a.B; b += gridDim.x)
    if (pre[b] == pre[b + 1]) {
      uint4* o = reinterpret_cast<uint4*>(a.out + static_cast<int64_t>(b) * a.hq * D);
      for (int i = tid; i < a.hq * D / 8; i += PGA_THREADS) o[i] = make_uint4(0, 0, 0, 0);
    }
  PgaPlan plan;
  plan.pre = pre;
  plan.nz = nz;
  plan.B = a.B;
  plan.hv = a.hv;
  plan.extra = pre[a.B] * a.hv > static_cast<int>(gridDim.x) * PGA_WARPS ? a.extra : 0;
  plan.divide(static_cast<int>(gridDim.x) * PGA_WARPS);
  const int me = blockIdx.x * PGA_WARPS + warp;
  // lane 0 seeks the start of this warp's share, lane 1 that of the next one's
  PgaWalk<D> look;
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
    PgaWalk<D> use = look;
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

  // ---- the block's pieces joined in key order, a warp per row, in one walk over the
  // warps: the last piece of a warp that goes on, the whole shares of the next ones, and
  // the first piece of the one in which the pair ends. What began before the block or goes
  // on after it leaves joined. All pieces are loaded ahead of the walk.
  constexpr int C = D / 32;
  int kind[PGA_WARPS];  // of a warp's last piece: 0 ends there, 1 begun in its share and goes on, 2 its whole share
#pragma unroll
  for (int w = 0; w < PGA_WARPS; ++w) kind[w] = meta[w].x;
#pragma unroll 1
  for (int r = warp; r < ROWS; r += PGA_WARPS) {
    PgaVec<C> last[PGA_WARPS], early[PGA_WARPS];
    float2 last_ml[PGA_WARPS], early_ml[PGA_WARPS];
#pragma unroll
    for (int w = 0; w < PGA_WARPS; ++w) {
      if (kind[w] != 0) {
        const float* p = reinterpret_cast<const float*>(pga_smem + w * PGA_STAGES * PGA_STAGE) + r * T::ROW;
        last_ml[w] = *reinterpret_cast<const float2*>(p + D);
        pga_load<false>(last[w], p + lane * C);
      }
      if (w > 0 && kind[w - 1] != 0 && kind[w] != 2) {
        const float* p = a.early + (static_cast<int64_t>(blockIdx.x * PGA_WARPS + w) * ROWS + r) * T::ROW;
        early_ml[w] = *reinterpret_cast<const float2*>(p + D);
        pga_load<false>(early[w], p + lane * C);
      }
    }
    if (tid == 0) {
      // a pair that begins here and ends in a later block
      int4 info = make_int4(0, 0, 0, 0);
      if (kind[PGA_WARPS - 1] != 0) {
        int w0 = PGA_WARPS - 1;
        while (w0 > 0 && kind[w0] == 2) --w0;
        if (meta[w0].x == 1) {
          info = make_int4(1, meta[w0].y, meta[w0].z, 0);
          const int tiles = pre[info.y + 1] - pre[info.y];
          const int end = plan.places(info.y) + (info.z + 1) * (tiles + plan.extra) - 1;
          info.w = plan.holder(end) / PGA_WARPS;
        }
      }
      a.info[blockIdx.x] = info;
    }
    float m = 0.f, l = 0.f;
    PgaVec<C> o;
    int w0 = 0;  // where the chain began
    auto add = [&](const float2& ml, const PgaVec<C>& v) {
      const float to = fmaxf(m, ml.x), ref = to == -INFINITY ? 0.f : to;
      const float f = pga_ex2(m - ref), e = pga_ex2(ml.x - ref);
      m = to;
      l = l * f + ml.y * e;
#pragma unroll
      for (int c = 0; c < C; ++c) o.v[c] = o.v[c] * f + v.v[c] * e;
    };
    auto leave = [&](bool open_begin, bool open_end) {
      if (open_begin || open_end) {
        float* dst = part + ((open_begin ? 0 : ROWS) + r) * T::ROW;
        pga_store(dst + lane * C, o);
        if (lane == 0) *reinterpret_cast<float2*>(dst + D) = make_float2(m, l);
      } else {
        const int b = meta[w0].y, h = meta[w0].z, g = a.qt == 1 ? h : h / a.qt, q = (h - g * a.qt) * ROWS + r;
        if (q < gs) pga_result(a.out + (static_cast<int64_t>(b) * a.hq + g * gs + q) * D + lane * C, o, l);
      }
    };
    bool on = false;  // a chain goes on into warp w
#pragma unroll
    for (int w = 0; w < PGA_WARPS; ++w) {
      if (on) {
        if (kind[w] == 2) {
          add(last_ml[w], last[w]);
          continue;
        }
        add(early_ml[w], early[w]);
        leave(w0 == 0 && kind[0] == 2, false);
      }
      on = kind[w] != 0;
      if (on) {
        w0 = w;
        m = last_ml[w].x;
        l = last_ml[w].y;
        o = last[w];
      }
    }
    if (on) leave(w0 == 0 && kind[0] == 2, true);
  }
}

// Pairs that end in a later block than they begin in: block k joins the pair that
// begins in block k of the launch before. A row's pieces are shared by several
// warps, each with its loads in flight together, whose sums are then added in order.
// While the launch before is still running the blocks of this one, already on their
// SMs where there is room, go through the same code once on whatever the workspace holds
// and store nothing: the second time its instructions are there (loads past L1, which
// keeps nothing of the first time). One request of 2049 rows 9.1 -> 8.6 us, 32 of them 30.0 ->
// 29.5.
constexpr int PGM_WARPS = 16;
template <int D, int NT>
__global__ void __launch_bounds__(32 * PGM_WARPS) k_paged_join(PagedArgs a) {
  using T = PgaTile<D>;
  constexpr int ROWS = 8 * NT, PER = PGM_WARPS / ROWS, C = D / 32, LOADS = 8, AHEAD = 8;
  __shared__ __align__(16) float so[PGM_WARPS][D];
  __shared__ float factor[PGM_WARPS][PGA_BLOCKS];
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r = warp / PER, s = warp % PER;
  auto piece = [&](int i) {
    return a.part + ((static_cast<int64_t>(blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + r) * T::ROW;
  };
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    if (pass == 1) pdl_wait();
    // the first maxima and sums come with the pair's description, whether they are its
    // pieces' or not (eight: with 32, as many requests as blocks took 1 us more)
    float2 ml[PGA_BLOCKS / 32];
    ml[0] = lane < (pass == 0 ? 2 : AHEAD) && blockIdx.x + lane < gridDim.x
                ? __ldcg(reinterpret_cast<const float2*>(piece(lane) + D))
                : make_float2(0.f, 0.f);
    int4 info = __ldcg(a.info + blockIdx.x);
    if (pass == 0) info = make_int4(1, 0, 0, min(blockIdx.x + 1, gridDim.x - 1));
    if (info.x == 0) return;
    const int gs = a.hq / a.hkv, g = a.qt == 1 ? info.z : info.z / a.qt, q = (info.z - g * a.qt) * ROWS + r;
    const int n = info.w - static_cast<int>(blockIdx.x) + 1;
    PgaVec<C> v[LOADS], o = {};
    auto fetch = [&](int i0) {
#pragma unroll
      for (int k = 0; k < LOADS; ++k)
        if (i0 + k * PER < n) pga_load<true>(v[k], piece(i0 + k * PER) + lane * C);
    };
    fetch(s);  // pieces s, s + PER, ..., LOADS of them in flight together
    if (n > AHEAD) {
#pragma unroll
      for (int k = 0; k < PGA_BLOCKS / 32; ++k)
        if (k * 32 + lane >= AHEAD && k * 32 + lane < n) ml[k] = __ldcg(reinterpret_cast<const float2*>(piece(k * 32 + lane) + D));
    }
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < PGA_BLOCKS / 32; ++k)
      if (k * 32 + lane < n) m = fmaxf(m, ml[k].x);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int k = 0; k < PGA_BLOCKS / 32; ++k)
      if (k * 32 + lane < n) {
        const float f = pga_ex2(ml[k].x - ref);
        factor[warp][k * 32 + lane] = f;
        l = fmaf(ml[k].y, f, l);
      }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
    __syncwarp();
#pragma unroll 1
    for (int i0 = s; i0 < n; i0 += LOADS * PER) {
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        const int i = i0 + k * PER;
        if (i >= n) break;
        const float f = factor[warp][i];
#pragma unroll
        for (int c = 0; c < C; ++c) o.v[c] = fmaf(v[k].v[c], f, o.v[c]);
      }
      fetch(i0 + LOADS * PER);
    }
    pga_store(so[warp] + lane * C, o);
    __syncthreads();
    if (s == 0 && q < gs) {
#pragma unroll
      for (int w = 1; w < PER; ++w) {
        pga_load<false>(v[0], so[warp + w] + lane * C);
#pragma unroll
        for (int c = 0; c < C; ++c) o.v[c] += v[0].v[c];
      }
      if (pass == 1) pga_result(a.out + (static_cast<int64_t>(info.y) * a.hq + g * gs + q) * D + lane * C, o, l);
    }
    __syncthreads();
  }
}

// Query rows of a warp's tile: 8 where a KV head has at most 8 query heads, else 16
// (a KV head of more than 16 is read once for every 16).
static int pga_rows(int Hq, int Hkv) { return Hq / Hkv <= 8 ? 8 : 16; }

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
  const size_t smem = static_cast<size_t>(PGA_WARPS) * PGA_STAGES * PGA_STAGE + 2 * (static_cast<size_t>(B) + 1) * sizeof(int);
  auto go = [&](auto main, auto join) -> int {
    DM_CUDA_CHECK(cudaFuncSetAttribute(main, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    DM_CUDA_CHECK(launch_pdl(main, dim3(grid), dim3(PGA_THREADS), smem, s, a));
    DM_CUDA_CHECK(launch_pdl(join, dim3(grid), dim3(32 * PGM_WARPS), 0, s, a));
    return DECOMOE_OK;
  };
  if (D == 128)
    DM_RET(rows == 8 ? go(k_paged_attention<128, 1>, k_paged_join<128, 1>)
                     : go(k_paged_attention<128, 2>, k_paged_join<128, 2>));
  else
    DM_RET(rows == 8 ? go(k_paged_attention<64, 1>, k_paged_join<64, 1>)
                     : go(k_paged_attention<64, 2>, k_paged_join<64, 2>));
  return DECOMOE_OK;
}

}  // extern "C"
