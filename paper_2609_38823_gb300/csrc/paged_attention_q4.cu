// Attention of one new token per request over a paged key-value cache in 4 bits
// (decoding on the text-only cache, DecoMoE Section 3.2 and Algorithm 2, last step, for a
// batch of requests), the visual block of a request left out where it has exited.
#include <cuda_fp16.h>

#include "paged_q4.cuh"
#include "paged_share.cuh"

namespace decomoe {

// The tiles (32 rows of a KV head) of all requests are numbered and divided evenly among the
// warps as in paged_attention.cu, whose joins of cut pairs this shares (paged_share.cuh): sixteen
// warps of 128 registers on every SM (eight where 16 query heads share a tile), each with a ring of two
// tiles of its own, filled by bulk copies, one for as many rows as lie in one page.
//
// out = sum_j p_j v_j / sum_j p_j with p_j = exp(scale q k_j - m), k = low + step code and the same
// for v, group by group of features:
//   q k_j = sum_g step_jg (sum_f q_f code_jf) + low_jg (sum_f q_f)
//   sum_j p_j v_jf = sum_j (p_j step_jg) code_jf + sum_j p_j low_jg
// so codes are never turned into values. Both inner sums run transposed on the tensor cores
// (mma.m16n8k16, fp16 in, fp32 accumulate: 16 keys, or features, by 8 queries). A code masked in
// place has the bits of the fp16 number code 2^-24 or code 2^-20, which the products take as they
// are: one operation makes two operands, and nothing is rounded or subtracted. Queries are
// scaled into fp16's range per row, where their eight digits are exact (but below 2^-27 of the row's
// largest). p step is rounded to fp16 (2^-11 of it at most; bf16, as the bf16 cache has it, would be
// 2^-8), scaled so that the largest step seen stays in range. low (sum q) is one more product, with
// the sum as three bf16 numbers; p low, sums, maxima and outputs are fp32.
//
// Bound: 96 requests of 2000 to 16385 rows (153 MB) 37 us, 4.2 TB/s: 4 us until the first copies are on their way
// (lengths, their sum, search, tables), 24 us of copies at 6.3 TB/s, 2 us of joins in the blocks and 4 for the joining
// launch. Of 590 instructions a tile 192 unpack codes on a pipe of
// half rate and 34 are products, issue slots are 60 % busy. The bf16 cache takes 95 us. With groups of 32 (170 MB)
// 43 us, of 128 (149 MB) 35: four groups cost four times the parameters' operations, and their 128 registers do not
// hold all that is live (56 bytes stored and 100 loaded again; with 16 queries a tile 16). One request of 2049 rows
// 10.0 us, all of it latency: 2.5 us to its first copies, 1 for them, 1.5 for a tile, 2 for the join in the block, 3
// for the launch that joins blocks, each a stretch of code that runs once.
// Steps: codes to bf16 numbers by shift, mask and subtraction, one copy per eight rows, 304
// blocks of eight warps 74 us; (code - 8) / 64 by one multiply-add, tiles of 32 rows, maxima raised
// rarely 55; fp16 subnormal operands, lookups eight tiles at a time 49; 152 blocks of sixteen warps, so
// that the joining launch is programmatic and joins half as many pieces 40; fewer branches 39; a search by half
// warps, tables and first queries brought into L2 ahead 37.9; warp numbers that are uniform to the compiler 36.9.
constexpr int Q4A_KEYS = 32;     // rows of a tile
constexpr int Q4A_SETS = Q4A_KEYS / 8;
constexpr int Q4A_STAGES = 2;    // tiles of a warp's ring (three: no faster)
constexpr int Q4A_BLOCKS = 160;  // of a launch, at most
constexpr int q4a_warps(int NT) { return NT == 1 ? 16 : 8; }  // of a block, one block per SM: as many as their registers allow
// Warps of a block that get tiles where there are few: one request of 2049 rows over 33 blocks
// of eight warps 10.2 us (now 10.0), over 17 of sixteen 11.0, over 130 of two (33 pieces a pair to join) 11.9.
constexpr int Q4A_FEW = 8;
// What a (request, KV head) pair costs beside its tiles, in tiles. With 1, 2, 3, 4 and 5 of them: 97 requests of 5 to 1553
// rows 20.5, 19.8, 20.0, 21.0 and 21.6 us, 200 of 5 to 600 21.1, 21.7, 22.5, 24.1 and 24.5; 96 of 2000 to 16385, 60 of up to
// 3000, 30 of 8000 and fewer ones within 1 %. 2 would be up to 3 % sooner for short requests alone; it stays 3 since
// the division decides the last bits of results.
constexpr int Q4A_EXTRA = 3;

// A tile: KEYS consecutive rows of a request from a multiple of KEYS on (so that eight rows
// always lie together in a page), those that are hidden or past the length left out of
// the sums. Tiles of hidden rows alone are not numbered.
struct Q4aTiles {
  static __device__ __forceinline__ int before(const PgaReq& r) {  // the hidden block
    return static_cast<int>(static_cast<unsigned>(r.h0 + Q4A_KEYS - 1) / Q4A_KEYS);
  }
  static __device__ __forceinline__ int after(const PgaReq& r) {
    return max(before(r), static_cast<int>(static_cast<unsigned>(r.h0 + r.hc) / Q4A_KEYS));
  }
  static __device__ __forceinline__ int count(const PgaReq& r) {
    const int n = r.seen + r.hc;
    return before(r) + (r.h0 + r.hc < n ? static_cast<int>(static_cast<unsigned>(n + Q4A_KEYS - 1) / Q4A_KEYS) - after(r) : 0);
  }
};

struct PagedQ4Args : PagedCommon {
  const uint8_t* pages;
  uint64_t limit_ns;
};

__device__ __forceinline__ void q4a_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ uint32_t q4a_lds(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
template <int N>
__device__ __forceinline__ void q4a_lds(uint32_t addr, uint32_t (&v)[N]) {
  static_assert(N == 1 || N == 2 || N == 4, "words of a load");
  if constexpr (N == 4)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr));
  else if constexpr (N == 2)
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(addr));
  else
    v[0] = q4a_lds(addr);
}
// pga_mma onto zeros.
__device__ __forceinline__ void q4a_mma0(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// The same product of fp16 numbers, onto zeros or c.
template <bool ZERO>
__device__ __forceinline__ void q4a_mma_h(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (ZERO)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t q4a_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The larger ones of two pairs of bf16 numbers, NaN being none.
__device__ __forceinline__ uint32_t q4a_max2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// The four codes of each half of w as fp16 pairs: masked in place a code's bits are those of a
// subnormal number, code 2^-24 or, the second and fourth, code 2^-20. The products take
// them as they are.
__device__ __forceinline__ void q4a_codes(uint32_t w, uint32_t (&f)[4]) {
  const uint32_t v = w >> 8;
  f[0] = w & 0x000f000fu;
  f[1] = w & 0x00f000f0u;
  f[2] = v & 0x000f000fu;
  f[3] = v & 0x00f000f0u;
}

// The first `count` (none or all where it is outside) of a tile's rows.
__device__ __forceinline__ uint32_t q4a_first(int count) {
  return count >= Q4A_KEYS ? 0xffffffffu : (1u << max(count, 0)) - 1u;
}

// Where the copies of a warp stand, BATCH tiles at a time: lane 4 k + s looks after set s
// (eight rows) of the batch's tile k and the page that it lies in, so that lengths, tables and places are worked out
// once in BATCH tiles. The pages of a batch are loaded when the one before it is begun.
constexpr int Q4A_BATCH = 8;
struct Q4aLook {
  int b, h, t, tiles;  // this lane's tile
  int left;            // tiles of the share from this lane's tile on; none: <= 0
  int at, page;        // its eight rows: the first, and their page
  uint32_t want;       // the tile's rows in that page that the request sees
  // To the tile `by` tiles on.
  __device__ __forceinline__ void advance(const PagedQ4Args& a, const int* pre, int by) {
    left -= by;
    if (left <= 0) return;
    t += by;
    while (t >= tiles) {
      t -= tiles;
      if (++h < a.hv) continue;
      h = 0;
      do ++b;
      while (pre[b + 1] == pre[b]);
      tiles = pre[b + 1] - pre[b];
    }
  }
  __device__ __forceinline__ void load(const PagedQ4Args& a, int set, uint32_t in_page) {
    want = 0;
    if (left <= 0) return;
    bool bad = false;  // marked by the launch's first look at the lengths
    const PgaReq r = pga_request(a, b, &bad);
    const int before = Q4aTiles::before(r), he = r.h0 + r.hc;
    at = (t < before ? t : t - before + Q4aTiles::after(r)) * Q4A_KEYS;
    want = q4a_first(r.seen + r.hc - at) & ~(q4a_first(he - at) & ~q4a_first(r.h0 - at)) & in_page;
    at += set * 8;
    if (want != 0) page = a.table[b * a.max_pages + (at >> a.shift)];
  }
};

template <int D, int G, int NT>
__global__ void __launch_bounds__(32 * q4a_warps(NT), 1) k_paged_attention_q4(PagedQ4Args a) {
  using L = Q4Tile<D, G>;
  constexpr int WARPS = q4a_warps(NT);
  constexpr int STAGES = Q4A_STAGES;
  constexpr int STAGE = Q4A_SETS * L::BYTES;
  constexpr int SUB = Q4A_KEYS / 16;
  constexpr int BLK = D / 32;      // blocks of 32 features
  constexpr int BG = BLK / G;      // of a group
  constexpr int ROWS = 8 * NT, ROW = pga_row(D);
  constexpr int RING = STAGES * STAGE;
  static_assert(ROWS * ROW * 4 <= RING, "a piece fits the ring");
  extern __shared__ __align__(1024) uint8_t q4a_smem[];
  __shared__ __align__(8) uint64_t bars[WARPS][STAGES];
  __shared__ int4 tile_info[WARPS][2 * Q4A_BATCH];  // rows seen, request, head tile, whether the pair ends (1) and begins (2)
  __shared__ int3 meta[WARPS];
  __shared__ int abort_flag;
  int* pre = reinterpret_cast<int*>(q4a_smem + WARPS * RING);
  int* nz = pre + a.B + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) abort_flag = 0;
  if (lane < STAGES) mbar_init(smem_u32(&bars[warp][lane]), 1);
  fence_mbar_init();
  pdl_enter();
  const PgaPlan plan = pga_begin<Q4aTiles, D, WARPS, Q4A_FEW, true>(a, pre, nz);
  const int me = blockIdx.x * plan.active + min(warp, plan.active);
  // the lower half of the warp seeks the start of its share, the upper half that of the next one's
  PgaWalk<Q4aTiles> seek;
  const int from = plan.place(warp < plan.active ? me + (lane >> 4) : me);
  const int found = seek.seek_by_halves(plan, from);
  const int first = from < plan.total ? found : pre[a.B] * a.hv;
  const int r0 = __shfl_sync(0xffffffffu, first, 0), r1 = __shfl_sync(0xffffffffu, first, 16);
  const int gs = a.hq / a.hkv;

  uint8_t* ring = q4a_smem + warp * RING;
  const uint32_t ring_s = smem_u32(ring), bar_s = smem_u32(&bars[warp][0]);
  float* mine = reinterpret_cast<float*>(ring);  // the last piece, once the ring is drained
  if (lane == 0) meta[warp] = make_int3(0, 0, 0);
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * ROWS * ROW;

  if (r0 < r1) {
    // ---- lookup and copy of tiles, ahead of their use
    const int n = r1 - r0;
    int b = __shfl_sync(0xffffffffu, seek.b, 0), h = __shfl_sync(0xffffffffu, seek.h, 0);  // of the piece
    const int t0 = __shfl_sync(0xffffffffu, seek.t, 0);
    bool began = t0 > 0;  // the piece's pair began in an earlier share
    // the first queries on their way into L2 while the pages are looked up (96 requests 39.0 -> 38.5 us, 97
    // short ones 20.4 -> 20.15; with 16 queries a tile 13.3 -> 13.6, so not there)
    if constexpr (NT == 1) {
      const int g = a.qt == 1 ? h : h / a.qt, row = (h - g * a.qt) * ROWS + (lane >> 2);
      if (row < gs)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(a.q + b * a.q_stride + static_cast<int64_t>(g * gs + row) * D +
                                                      (lane & 3) * (D / 4)));
    }
    const int set = lane & (Q4A_SETS - 1), mine_of = lane / Q4A_SETS;
    Q4aLook look = {b, h, t0, pre[b + 1] - pre[b], n, 0, 0, 0};
    // sets of a tile in one page, which one copy takes: those of this lane's, and whether it is the first
    const int in_one = min(1 << a.shift, Q4A_KEYS) / 8;
    const bool leads = (set & (in_one - 1)) == 0;
    const uint32_t in_page = (in_one == Q4A_SETS ? 0xffffffffu : (1u << (8 * in_one)) - 1u) << (8 * (set & -in_one));
    look.advance(a, pre, mine_of);
    look.load(a, set, in_page);
    const uint8_t* src = nullptr;
    uint32_t bytes = 0;  // of the tile
    bool there = false;
    auto begin_batch = [&](int which) {
      there = look.want != 0 && look.page >= 0 && look.page < a.num_pages;
      if (look.want != 0 && !there) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
      uint32_t mask = there ? look.want : 0u;
      mask |= __shfl_xor_sync(0xffffffffu, mask, 1);
      mask |= __shfl_xor_sync(0xffffffffu, mask, 2);
      bytes = __popc(__ballot_sync(0xffffffffu, there) >> (lane & ~(Q4A_SETS - 1)) & ((1u << Q4A_SETS) - 1)) * L::BYTES;
      if (there)
        src = a.pages + look.page * a.page_stride +
              ((static_cast<int64_t>(a.qt == 1 ? look.h : look.h / a.qt) << a.shift >> 3) +
               ((look.at & ((1 << a.shift) - 1)) >> 3)) * L::BYTES;
      if (set == 0)
        tile_info[warp][(which & 1) * Q4A_BATCH + mine_of] =
            make_int4(static_cast<int>(mask), look.b, look.h, (look.t + 1 == look.tiles) | (look.t == 0) << 1);
      look.advance(a, pre, Q4A_BATCH);
      look.load(a, set, in_page);
      __syncwarp();
    };
    auto issue = [&](int tile, int slot) {
      if (tile % Q4A_BATCH == 0) begin_batch(tile / Q4A_BATCH);
      const bool turn = mine_of == tile % Q4A_BATCH;
      const uint32_t bar = bar_s + slot * 8, dst = ring_s + slot * STAGE + set * L::BYTES;
      if (in_one == Q4A_SETS) {
        if (turn && set == 0) {
          mbar_arrive_expect_tx(bar, bytes);
          if (there) q4a_bulk(dst, src, STAGE, bar);
        }
      } else {
        if (turn && set == 0) mbar_arrive_expect_tx(bar, bytes);
        __syncwarp();
        if (turn && there && leads) q4a_bulk(dst, src, in_one * L::BYTES, bar);
      }
      __syncwarp();
    };

    // a lane's part of the operands: row kr of eight keys, word (kr, c) of the codes; keys c and
    // c + 4 of eight values, features 32 i + 4 r .. + 3
    const int r = lane >> 2, c = lane & 3, kr = (r >> 1) + 4 * (r & 1);
    uint32_t qf[NT][BLK][4], qs[NT][G == 4 ? 3 : 2];
    float sl2[NT][2];
    float o[2 * BLK][NT][4], low[NT][2][G], m[NT][2], ref[NT][2], l[NT][2];
    float pass[NT][2];  // ref: m, 0 for none; pass: m + 8
    // steps seen so far are below room; grow, a power of two, times those is below 2^6
    float room = 0.f, grow = 1.f;
    auto begin_piece = [&]() {
      const int g = a.qt == 1 ? h : h / a.qt, q0 = (h - g * a.qt) * ROWS;
      const __nv_bfloat16* q = a.q + b * a.q_stride + static_cast<int64_t>(g) * gs * D;
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const int row = q0 + x * 8 + r;
        // the queries times a power of two that brings their largest into [2^14, 2^15)
        float v[BLK][8], most = 0.f;
#pragma unroll
        for (int i = 0; i < BLK; ++i) {
          uint4 u = make_uint4(0, 0, 0, 0);
          if (row < gs) u = *reinterpret_cast<const uint4*>(q + static_cast<int64_t>(row) * D + 32 * i + 8 * c);
          v[i][0] = bf16_lo(u.x), v[i][1] = bf16_hi(u.x), v[i][2] = bf16_lo(u.y), v[i][3] = bf16_hi(u.y);
          v[i][4] = bf16_lo(u.z), v[i][5] = bf16_hi(u.z), v[i][6] = bf16_lo(u.w), v[i][7] = bf16_hi(u.w);
#pragma unroll
          for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(v[i][j]));
        }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const uint32_t up = min(268u - (__float_as_uint(most) >> 23), 253u);  // its exponent
        const float by = most <= FLT_MAX ? __uint_as_float(up << 23) : NAN;
        float sum[G];
#pragma unroll
        for (int i = 0; i < G; ++i) sum[i] = 0.f;
#pragma unroll
        for (int i = 0; i < BLK; ++i) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            v[i][j] *= by;
            sum[i / BG] += v[i][j];
          }
          // (odd codes come as 16 code)
          qf[x][i][0] = q4a_half2(v[i][0], v[i][4]);
          qf[x][i][1] = q4a_half2(v[i][1] * 0.0625f, v[i][5] * 0.0625f);
          qf[x][i][2] = q4a_half2(v[i][2], v[i][6]);
          qf[x][i][3] = q4a_half2(v[i][3] * 0.0625f, v[i][7] * 0.0625f);
        }
        // what brings a score of these back (codes are 2^-24), and softmax's factor
        // (multiplied so that nothing on the way is larger or smaller than they and the result are; at most the largest
        // number, or scores of 0 would be NaN: one key takes all the weight there)
        const float unscale = __uint_as_float((254u - up) << 23);
        const float back = fminf(up < 128u ? 0x1p24f * (a.sl2 * unscale) : a.sl2 * (0x1p24f * unscale), FLT_MAX);
#pragma unroll
        for (int i = 0; i < 2; ++i) sl2[x][i] = __shfl_sync(0xffffffffu, back, 4 * (2 * c + i));
        // a group's sum (times 2^-24, as the codes) in three bf16 numbers, 24 bits: factors of low
        uint32_t piece[G][3];
#pragma unroll
        for (int i = 0; i < G; ++i) {
          sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
          sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
          float rest = sum[i] * 0x1p-24f;
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            const float f = __bfloat162float(__float2bfloat16_rn(rest));
            piece[i][k] = pack_bf16x2(0.f, f);
            rest -= f;
          }
        }
        if constexpr (G == 1) {
          qs[x][0] = c == 0 ? piece[0][0] : c == 1 ? piece[0][1] : c == 2 ? piece[0][2] : 0u;
          qs[x][1] = 0u;
        } else if constexpr (G == 2) {
          qs[x][0] = c == 0 ? piece[0][0] : c == 1 ? piece[1][0] : c == 2 ? piece[0][1] : piece[1][1];
          qs[x][1] = c == 0 ? piece[0][2] : c == 1 ? piece[1][2] : 0u;
        } else {
#pragma unroll
          for (int k = 0; k < 3; ++k)
            qs[x][k] = c == 0 ? piece[0][k] : c == 1 ? piece[1][k] : c == 2 ? piece[2][k] : piece[3][k];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          m[x][i] = pass[x][i] = -INFINITY;
          ref[x][i] = l[x][i] = 0.f;
#pragma unroll
          for (int g2 = 0; g2 < G; ++g2) low[x][i][g2] = 0.f;
        }
#pragma unroll
        for (int s = 0; s < 2 * BLK; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[s][x][i] = 0.f;
      }
      room = 0.f;
      grow = 1.f;
    };
    // a finished piece: its sums over the lanes, the lows added to the outputs
    auto end_piece = [&]() {
      const float back = __uint_as_float((254u << 23) - __float_as_uint(grow));  // 1 / grow
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) l[x][i] += __shfl_xor_sync(0xffffffffu, l[x][i], w);
#pragma unroll
          for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) low[x][i][g] += __shfl_xor_sync(0xffffffffu, low[x][i][g], w);
#pragma unroll
            for (int s = 2 * BG * g; s < 2 * BG * (g + 1); ++s) {
              o[s][x][i] = fmaf(o[s][x][i] * 0x1p24f, back, low[x][i][g]);
              o[s][x][i + 2] = fmaf(o[s][x][i + 2] * 0x1p20f, back, low[x][i][g]);
            }
          }
        }
    };
    auto keep_piece = [&](float* dst) {
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float* row = dst + (x * 8 + 2 * c + i) * ROW;
#pragma unroll
          for (int s = 0; s < BLK; ++s)
            *reinterpret_cast<float4*>(row + 32 * s + 4 * r) =
                make_float4(o[2 * s][x][i], o[2 * s][x][i + 2], o[2 * s + 1][x][i], o[2 * s + 1][x][i + 2]);
          if (lane < 4) {
            row[D] = m[x][i];
            row[D + 1] = l[x][i];
          }
        }
    };
    int slot = 0, fill = 0;
    uint32_t parity = 0;
    // the first steps only fill the ring (one copy of the code: a short share runs it cold)
    for (int i = 1 - STAGES; i < n; ++i) {
      if (i + STAGES - 1 < n) {
        issue(i + STAGES - 1, fill);
        fill = fill + 1 == STAGES ? 0 : fill + 1;
      }
      if (i < 0) {
        if (i == -1) begin_piece();
        continue;
      }
      if (!__all_sync(0xffffffffu, mbar_try_wait(bar_s + slot * 8, parity)) &&
          !__all_sync(0xffffffffu, mbar_wait(bar_s + slot * 8, parity, a.limit_ns, &abort_flag))) {
        if (lane == 0) report_status(a.status, DECOMOE_ERR_TIMEOUT);
        // no results; what is in flight gets the same time to land
        for (int k = 1; k < STAGES && i + k < n; ++k) {
          slot = slot + 1 == STAGES ? (parity ^= 1, 0) : slot + 1;
          mbar_wait(bar_s + slot * 8, parity, a.limit_ns, &abort_flag);
        }
        break;
      }
      const uint32_t stage = ring_s + slot * STAGE;
      const int4 info = tile_info[warp][i % (2 * Q4A_BATCH)];
      if ((info.w & 2) && i > 0) {  // a new pair
        b = info.y;
        h = info.z;
        began = false;
        begin_piece();
      }
      const uint32_t mask = static_cast<uint32_t>(info.x);
      // ---- scores: sum over the groups of step (q code) + low (sum of q); queries are exact
      // in fp16 but where a value lies below 2^-27 of the query's largest
      float sc[SUB][NT][4];
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const uint32_t at[2] = {stage + 2 * u * L::BYTES, stage + (2 * u + 1) * L::BYTES};
        uint32_t kw[2][BLK], kx[4], kp[2][G];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          q4a_lds(at[hf] + L::K + kr * L::CODES + c * (L::CODES / 4), kw[hf]);
          q4a_lds(at[hf] + L::KP + kr * L::PARAMS, kp[hf]);
          kx[hf] = kx[hf + 2] = q4a_lds(at[hf] + L::KP + kr * L::PARAMS + (c % G) * 4);
        }
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          q4a_mma0(sc[u][x], kx, qs[x][0], qs[x][1]);
          if constexpr (G == 4) pga_mma(sc[u][x], kx, qs[x][2], 0u);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float acc[NT][4];
#pragma unroll
          for (int i2 = g * BG; i2 < (g + 1) * BG; ++i2) {
            uint32_t f0[4], f1[4];
            q4a_codes(kw[0][i2], f0);
            q4a_codes(kw[1][i2], f1);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const uint32_t f[4] = {f0[2 * s], f1[2 * s], f0[2 * s + 1], f1[2 * s + 1]};
#pragma unroll
              for (int x = 0; x < NT; ++x) {
                if (i2 == g * BG && s == 0) q4a_mma_h<true>(acc[x], f, qf[x][i2][0], qf[x][i2][1]);
                else q4a_mma_h<false>(acc[x], f, qf[x][i2][2 * s], qf[x][i2][2 * s + 1]);
              }
            }
          }
#pragma unroll
          for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int i2 = 0; i2 < 4; ++i2) sc[u][x][i2] = fmaf(bf16_lo(kp[i2 >> 1][g]), acc[x][i2], sc[u][x][i2]);
        }
        // (before the mask: a factor next to nothing counts as 0, and minus infinity times that is NaN)
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
          for (int i2 = 0; i2 < 4; ++i2) sc[u][x][i2] *= sl2[x][i2 & 1];
      }
      uint32_t vp[SUB][2][G];
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) q4a_lds(stage + (2 * u + hf) * L::BYTES + L::VP + kr * L::PARAMS, vp[u][hf]);
      if (mask != 0xffffffffu) {
        __syncwarp();  // (a branch of its own: as predicates it would cost every tile)
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            if (!((mask >> (16 * u + 8 * hf + kr)) & 1u)) {
              // anything may lie where nothing is seen
#pragma unroll
              for (int x = 0; x < NT; ++x) sc[u][x][2 * hf] = sc[u][x][2 * hf + 1] = -INFINITY;
#pragma unroll
              for (int g = 0; g < G; ++g) vp[u][hf][g] = 0u;
            }
      }
      // ---- a query's maximum, raised only where a score passes it by 2^8 (weights up to 2^8 cost no
      // digits), and the scale of the steps, which keeps weights times steps, the fp16 operands
      // of the value product, below 2^14: the lanes compare theirs only where one of them has to
      // change, and rescaling the outputs is rare
      uint32_t widest = 0;  // bf16 bits of the largest step (they are not negative; NaN: its sums say so)
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int g = 0; g < G; ++g) widest = q4a_max2(widest, vp[u][hf][g]);
      bool raise = bf16_lo(widest) >= room;
      float mx[NT][2];
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int i2 = 0; i2 < 2; ++i2) {
#pragma unroll
          for (int u = 0; u < SUB; ++u) {
            const float y = fmaxf(sc[u][x][i2], sc[u][x][i2 + 2]);
            mx[x][i2] = u == 0 ? y : fmaxf(mx[x][i2], y);
          }
          raise |= mx[x][i2] > pass[x][i2];
        }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int w = 1; w < 32; w <<= 1) widest = q4a_max2(widest, __shfl_xor_sync(0xffffffffu, widest, w));
        float wider = 1.f;
        if (bf16_lo(widest) >= room) {
          const uint32_t e = max(widest >> 7 & 0xffu, 7u);  // the largest step is below 2^(e - 126)
          room = e < 254 ? __uint_as_float((e + 1) << 23) : INFINITY;
          const float to = __uint_as_float((259u - min(e, 254u)) << 23);  // 2^(132 - e)
          wider = to * __uint_as_float((254u << 23) - __float_as_uint(grow));  // its inverse: a power of two
          grow = to;
        }
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
          for (int i2 = 0; i2 < 2; ++i2) {
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) mx[x][i2] = fmaxf(mx[x][i2], __shfl_xor_sync(0xffffffffu, mx[x][i2], w));
            const float to = fmaxf(m[x][i2], mx[x][i2]);
            // nothing seen so far, and nothing here: any factor does
            const float f = to == -INFINITY ? 1.f : pga_ex2(m[x][i2] - to);
            m[x][i2] = to;
            pass[x][i2] = to + 8.f;
            ref[x][i2] = to == -INFINITY ? 0.f : to;
            l[x][i2] *= f;
#pragma unroll
            for (int g = 0; g < G; ++g) low[x][i2][g] *= f;
#pragma unroll
            for (int s = 0; s < 2 * BLK; ++s) {
              o[s][x][i2] *= f * wider;
              o[s][x][i2 + 2] *= f * wider;
            }
          }
      }
      // ---- weights and values
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const uint32_t at[2] = {stage + 2 * u * L::BYTES, stage + (2 * u + 1) * L::BYTES};
        uint32_t p[NT][G][2];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          float w[4];
#pragma unroll
          for (int i2 = 0; i2 < 4; ++i2) w[i2] = pga_ex2(sc[u][x][i2] - ref[x][i2 & 1]);
          l[x][0] += w[0] + w[2];
          l[x][1] += w[1] + w[3];
          // weights times steps are the operands of the value product; lows add up in fp32
#pragma unroll
          for (int g = 0; g < G; ++g)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const float step = bf16_lo(vp[u][hf][g]) * grow, at0 = bf16_hi(vp[u][hf][g]);
              low[x][0][g] = fmaf(w[2 * hf], at0, low[x][0][g]);
              low[x][1][g] = fmaf(w[2 * hf + 1], at0, low[x][1][g]);
              p[x][g][hf] = pga_transpose(q4a_half2(w[2 * hf] * step, w[2 * hf + 1] * step));
            }
        }
        uint32_t vw[2][2][BLK / 2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            q4a_lds(at[hf] + L::V + (c + 4 * k) * L::CODES + r * (L::CODES / 8), vw[hf][k]);
#pragma unroll
        for (int i2 = 0; i2 < BLK; ++i2) {
          uint32_t f0[4], f1[4];  // of the two keys of each half
          q4a_codes(__byte_perm(vw[0][0][i2 / 2], vw[0][1][i2 / 2], i2 & 1 ? 0x7632 : 0x5410), f0);
          q4a_codes(__byte_perm(vw[1][0][i2 / 2], vw[1][1][i2 / 2], i2 & 1 ? 0x7632 : 0x5410), f1);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const uint32_t f[4] = {f0[2 * s], f0[2 * s + 1], f1[2 * s], f1[2 * s + 1]};
#pragma unroll
            for (int x = 0; x < NT; ++x) q4a_mma_h<false>(o[2 * i2 + s][x], f, p[x][i2 / BG][0], p[x][i2 / BG][1]);
          }
        }
      }
      __syncwarp();
      slot = slot + 1 == STAGES ? (parity ^= 1, 0) : slot + 1;
      const bool ends = info.w & 1;
      if (ends || i + 1 == n) {
        end_piece();
        if (!ends) {  // goes on in the next share; the ring is empty
          keep_piece(mine);
          if (lane == 0) meta[warp] = make_int3(began ? 2 : 1, b, h);
        } else if (began) {
          // begun before the block: it is all that the block holds of its pair
          keep_piece(warp == 0 ? part : a.early + static_cast<int64_t>(blockIdx.x * WARPS + warp) * ROWS * ROW);
        } else {
          const int g = a.qt == 1 ? h : h / a.qt, q0 = (h - g * a.qt) * ROWS;
#pragma unroll
          for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
              const int row = q0 + x * 8 + 2 * c + i2;
              if (row < gs) {
                const float f = l[x][i2] != 0.f ? 1.f / l[x][i2] : 0.f;
                __nv_bfloat16* dst = a.out + (static_cast<int64_t>(b) * a.hq + g * gs + row) * D + 4 * r;
#pragma unroll
                for (int s = 0; s < BLK; ++s)
                  *reinterpret_cast<uint2*>(dst + 32 * s) =
                      make_uint2(pack_bf16x2(o[2 * s][x][i2] * f, o[2 * s][x][i2 + 2] * f),
                                 pack_bf16x2(o[2 * s + 1][x][i2] * f, o[2 * s + 1][x][i2 + 2] * f));
              }
            }
        }
      }
    }
  }
  __syncthreads();
  pga_join_block<D, NT, WARPS, true>(a, plan, meta, q4a_smem, RING);
}

}  // namespace decomoe

using namespace decomoe;

extern "C" {

size_t decomoe_paged_attention_q4_workspace_bytes(int64_t B, int Hq, int Hkv, int D) {
  if (B <= 0 || Hkv <= 0 || Hq < Hkv || D <= 0) return 0;
  // the pieces of every warp and of every block, one block per SM
  const size_t rows = static_cast<size_t>(pga_rows(Hq, Hkv)) * pga_row(D) * sizeof(float);
  return static_cast<size_t>(std::min(sm_count(), Q4A_BLOCKS)) * ((q4a_warps(pga_rows(Hq, Hkv) / 8) + 2) * rows + sizeof(int4));
}

int decomoe_paged_attention_q4(const void* q, int64_t q_stride, int64_t B, const void* pages, int64_t num_pages,
                               int page_size, int64_t page_stride, int group, const int32_t* block_table, int64_t max_pages,
                               const int32_t* seq_len, const int32_t* hide_begin, const int32_t* hide_count, int Hq,
                               int Hkv, int D, float scale, void* out, void* ws, size_t ws_bytes, int32_t* status_dev,
                               decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(B >= 0 && B <= DECOMOE_MAX_REQUESTS, "paged_attention_q4: B must lie in [0, %d]", DECOMOE_MAX_REQUESTS);
  DM_ARG_CHECK(q4_shape_ok(D, group),
               "paged_attention_q4: D 64 with groups of 32 or 64, or D 128 with groups of 32, 64 or 128");
  DM_ARG_CHECK(Hkv >= 1 && Hq >= Hkv && Hq % Hkv == 0, "paged_attention_q4: Hq must be a multiple of Hkv");
  DM_ARG_CHECK(Hq <= 1024, "paged_attention_q4: more than 1024 query heads");
  DM_ARG_CHECK(page_size >= 8 && (page_size & (page_size - 1)) == 0,
               "paged_attention_q4: page_size must be a power of two, 8 at least");
  DM_ARG_CHECK(num_pages >= 0 && num_pages <= INT_MAX / page_size,
               "paged_attention_q4: num_pages * page_size must be below 2^31");
  // a length rounded up to a tile of (at most) 32 keys is counted in 32 bits
  DM_ARG_CHECK(max_pages >= 0 && max_pages <= (INT_MAX - 31) / page_size,
               "paged_attention_q4: max_pages * page_size must be at most 2^31 - 32");
  const int64_t page = q4_tile_bytes(D, group) * (page_size / 8) * Hkv;
  DM_ARG_CHECK(page_stride >= page && page_stride % 16 == 0,
               "paged_attention_q4: page_stride below a page's bytes, or no multiple of 16");
  DM_ARG_CHECK(q_stride >= static_cast<int64_t>(Hq) * D && q_stride % 8 == 0,
               "paged_attention_q4: q_stride must be at least Hq * D and a multiple of 8");
  DM_ARG_CHECK((hide_begin == nullptr) == (hide_count == nullptr),
               "paged_attention_q4: hide_begin and hide_count go together");
  if (B == 0) return DECOMOE_OK;
  DM_ARG_CHECK(q && seq_len && out && (max_pages == 0 || block_table) && (num_pages == 0 || pages),
               "paged_attention_q4: null pointer");
  DM_ARG_CHECK(aligned16(q) && aligned16(pages) && aligned16(out), "paged_attention_q4: pointers must be 16-byte aligned");
  const size_t need = decomoe_paged_attention_q4_workspace_bytes(B, Hq, Hkv, D);
  if (ws == nullptr || ws_bytes < need) {
    set_error("paged_attention_q4: workspace of %zu bytes needed", need);
    return DECOMOE_ERR_WORKSPACE;
  }
  DM_ARG_CHECK(aligned16(ws), "paged_attention_q4: workspace must be 16-byte aligned");
  {
    const size_t each = static_cast<size_t>(B) * sizeof(int32_t);
    const Bytes in[] = {{q, static_cast<size_t>((B - 1) * q_stride + static_cast<int64_t>(Hq) * D) * 2},
                        {pages, num_pages == 0 ? 0 : static_cast<size_t>((num_pages - 1) * page_stride + page)},
                        {block_table, each * static_cast<size_t>(max_pages)},
                        {seq_len, each},
                        {hide_begin, each},
                        {hide_count, each}};
    const Bytes o = {out, static_cast<size_t>(B) * Hq * D * 2}, w = {ws, need};
    bool apart = !overlaps(o, {w});
    for (const Bytes& b : in) apart &= !overlaps(o, {b}) && !overlaps(w, {b});
    DM_ARG_CHECK(apart, "paged_attention_q4: out or the workspace overlaps an input or one another");
  }
  PagedQ4Args a = {};
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.pages = static_cast<const uint8_t*>(pages);
  a.limit_ns = static_cast<uint64_t>(wait_limit_ns());
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
  a.extra = Q4A_EXTRA;
  const int64_t most = B * ((max_pages * page_size + Q4A_KEYS - 1) / Q4A_KEYS + 1) * a.hv;  // tiles, at most
  DM_ARG_CHECK(most + Q4A_EXTRA * B * a.hv <= INT_MAX, "paged_attention_q4: B * max_pages * page_size * heads is too large");
  const int warps = q4a_warps(rows / 8);
  const int grid = static_cast<int>(
      std::max<int64_t>(1, std::min<int64_t>(std::min(sm_count(), Q4A_BLOCKS), (most + Q4A_FEW - 1) / Q4A_FEW)));
  const size_t piece = static_cast<size_t>(rows) * pga_row(D);
  a.early = static_cast<float*>(ws);
  a.part = a.early + static_cast<size_t>(grid) * warps * piece;
  a.info = reinterpret_cast<int4*>(a.part + static_cast<size_t>(grid) * 2 * piece);
  auto smem = [&](int64_t requests) {
    return static_cast<size_t>(warps) * Q4A_STAGES * Q4A_SETS * q4_tile_bytes(D, group) +
           2 * (static_cast<size_t>(requests) + 1) * sizeof(int);
  };
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto main, auto join) -> int {
    // the limit belongs to the kernel, not to the call: one for every batch, or a smaller one on another thread
    // could lower it before this launch
    DM_CUDA_CHECK(cudaFuncSetAttribute(main, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(smem(DECOMOE_MAX_REQUESTS))));
    DM_CUDA_CHECK(launch_pdl(main, dim3(grid), dim3(32 * warps), smem(B), s, a));
    DM_CUDA_CHECK(launch_pdl(join, dim3(grid), dim3(32 * PGM_WARPS), 0, s, static_cast<const PagedCommon&>(a)));
    return DECOMOE_OK;
  };
  return q4_dispatch(D, group, [&](auto d, auto g) -> int {
    return rows == 8 ? go(k_paged_attention_q4<d.value, g.value, 1>, k_paged_join<d.value, 1, Q4A_BLOCKS>)
                     : go(k_paged_attention_q4<d.value, g.value, 2>, k_paged_join<d.value, 2, Q4A_BLOCKS>);
  });
}

}  // extern "C"
