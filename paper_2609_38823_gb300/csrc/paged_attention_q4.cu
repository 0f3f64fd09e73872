// Attention of one new token per request over a paged key-value cache in 4 bits
// (decoding on the text-only cache, DecoMoE Section 3.2 and Algorithm 2, last step, for a
// batch of requests), the visual block of a request left out where it has exited.
#include "paged_q4.cuh"
#include "paged_share.cuh"

namespace decomoe {

constexpr int Q4A_KEYS = 32;     // rows of a tile
constexpr int Q4A_SETS = Q4A_KEYS / 8;
constexpr int Q4A_BLOCKS = 320;  // of a launch, at most
constexpr int Q4A_EXTRA = 3;     // what a (request, KV head) pair costs beside its tiles, in tiles
constexpr int q4a_stages(int D) { return D == 128 ? 3 : 4; }

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
// The four codes of each half of w as bf16 pairs of (code - 8) / 64, exact: masked in
// place a code is a subnormal number, code 2^-133 or (four bits up) code 2^-129, which one multiply-add
// brings there.
__device__ __forceinline__ uint32_t q4a_fma(uint32_t u, uint32_t by) {
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(u), "r"(by), "r"(0xbe00be00u));  // - 1/8
  return r;
}
__device__ __forceinline__ void q4a_codes(uint32_t w, uint32_t (&f)[4]) {
  const uint32_t v = w >> 8;
  f[0] = q4a_fma(w & 0x000f000fu, 0x7f007f00u);  // 2^127
  f[1] = q4a_fma(w & 0x00f000f0u, 0x7d007d00u);  // 2^123
  f[2] = q4a_fma(v & 0x000f000fu, 0x7f007f00u);
  f[3] = q4a_fma(v & 0x00f000f0u, 0x7d007d00u);
}

// Where the copies of a warp stand in the numbered tiles: a tile of a pair, and the pair's
// rows, table and place in a page.
struct Q4aLook {
  int b, h, t, tiles, before, skip, n, h0, he;
  const int32_t* table;
  const uint8_t* head;
  __device__ __forceinline__ void pair(const PagedQ4Args& a, int tile_bytes) {
    head = a.pages + (static_cast<int64_t>(a.qt == 1 ? h : h / a.qt) << a.shift >> 3) * tile_bytes;
  }
  __device__ __forceinline__ void enter(const PagedQ4Args& a, int tile_bytes) {
    bool bad = false;  // marked by the launch's first look at the lengths
    const PgaReq r = pga_request(a, b, &bad);
    tiles = Q4aTiles::count(r);
    before = Q4aTiles::before(r);
    skip = Q4aTiles::after(r) - before;
    n = r.seen + r.hc;
    h0 = r.h0;
    he = r.h0 + r.hc;
    table = a.table + b * a.max_pages;
    pair(a, tile_bytes);
  }
  // To the next tile; in the last pair it stays past the end (nobody looks).
  __device__ __forceinline__ void next(const PagedQ4Args& a, const int* pre, int tile_bytes) {
    if (++t < tiles) return;
    t = 0;
    if (++h < a.hv) return pair(a, tile_bytes);
    h = 0;
    do ++b;
    while (b < a.B && pre[b + 1] == pre[b]);
    if (b < a.B) enter(a, tile_bytes);
  }
};

template <int D, int G, int NT>
__global__ void __launch_bounds__(PGA_THREADS, NT == 1 ? 2 : 1) k_paged_attention_q4(PagedQ4Args a) {
  using L = Q4Tile<D, G>;
  constexpr int STAGES = q4a_stages(D);
  constexpr int STAGE = Q4A_SETS * L::BYTES;
  constexpr int SUB = Q4A_KEYS / 16;
  constexpr int BLK = D / 32;      // blocks of 32 features
  constexpr int BG = BLK / G;      // of a group
  constexpr int ROWS = 8 * NT, ROW = pga_row(D);
  constexpr int RING = STAGES * STAGE;
  static_assert(ROWS * ROW * 4 <= RING, "a piece fits the ring");
  extern __shared__ __align__(1024) uint8_t q4a_smem[];
  __shared__ __align__(8) uint64_t bars[PGA_WARPS][STAGES];
  __shared__ int4 tile_info[PGA_WARPS][STAGES];  // rows seen, request, head tile, whether the pair ends
  __shared__ int3 meta[PGA_WARPS];
  __shared__ int abort_flag;
  int* pre = reinterpret_cast<int*>(q4a_smem + PGA_WARPS * RING);
  int* nz = pre + a.B + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) abort_flag = 0;
  if (lane < STAGES) mbar_init(smem_u32(&bars[warp][lane]), 1);
  fence_mbar_init();
  pdl_enter();
  const PgaPlan plan = pga_begin<Q4aTiles, D>(a, pre, nz);
  const int me = blockIdx.x * PGA_WARPS + warp;
  // lane 0 seeks the start of this warp's share, lane 1 that of the next one's
  PgaWalk<Q4aTiles> seek;
  const int from = plan.place(me + (lane & 1));
  const int first = from < plan.total ? seek.seek(plan, from) : pre[a.B] * a.hv;
  const int r0 = __shfl_sync(0xffffffffu, first, 0), r1 = __shfl_sync(0xffffffffu, first, 1);
  const int gs = a.hq / a.hkv;

  uint8_t* ring = q4a_smem + warp * RING;
  const uint32_t ring_s = smem_u32(ring), bar_s = smem_u32(&bars[warp][0]);
  float* mine = reinterpret_cast<float*>(ring);  // the last piece, once the ring is drained
  if (lane == 0) meta[warp] = make_int3(0, 0, 0);
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * ROWS * ROW;

  if (r0 < r1) {
    // ---- lookup and copy of tiles, ahead of their use
    Q4aLook look;
    look.b = __shfl_sync(0xffffffffu, seek.b, 0);
    look.h = __shfl_sync(0xffffffffu, seek.h, 0);
    look.t = __shfl_sync(0xffffffffu, seek.t, 0);
    look.enter(a, L::BYTES);
    bool began = look.t > 0;  // the piece's pair began in an earlier share
    const int in_page = (1 << a.shift) - 1;
    int page = -1, off = 0;
    uint32_t want = 0;  // the tile's rows that the request sees
    auto lookup = [&]() {  // the page of this lane's eight rows
      const int at = (look.t < look.before ? look.t : look.t + look.skip) * Q4A_KEYS;
      const int j = at + lane;
      want = __ballot_sync(0xffffffffu, j < look.n && (j < look.h0 || j >= look.he));
      const int p = at + lane * 8;
      page = -1;
      off = ((p & in_page) >> 3) * L::BYTES;
      if (lane < Q4A_SETS && ((want >> (lane * 8)) & 0xffu)) page = look.table[p >> a.shift];
    };
    auto issue = [&](int slot) {
      const bool some = lane < Q4A_SETS && ((want >> (lane * 8)) & 0xffu);
      const bool there = some && page >= 0 && page < a.num_pages;
      if (some && !there) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
      const uint32_t sets = __ballot_sync(0xffffffffu, there), bar = bar_s + slot * 8;
      if (lane == 0) {
        uint32_t mask = want;
        if (sets != (1u << Q4A_SETS) - 1)
#pragma unroll
          for (int i = 0; i < Q4A_SETS; ++i)
            if (!((sets >> i) & 1u)) mask &= ~(0xffu << (8 * i));
        tile_info[warp][slot] = make_int4(static_cast<int>(mask), look.b, look.h, look.t + 1 == look.tiles);
        mbar_arrive_expect_tx(bar, __popc(sets) * L::BYTES);
      }
      __syncwarp();
      if (there) q4a_bulk(ring_s + slot * STAGE + lane * L::BYTES, look.head + page * a.page_stride + off, L::BYTES, bar);
    };
    const int n = r1 - r0;
    lookup();

    // a lane's part of the operands: row kr of eight keys, word (kr, c) of the codes; keys c and
    // c + 4 of eight values, features 32 i + 4 r .. + 3
    const int r = lane >> 2, c = lane & 3, kr = (r >> 1) + 4 * (r & 1);
    uint32_t qf[NT][BLK][4], qs[NT][G == 4 ? 3 : 2];
    float o[2 * BLK][NT][4], low[NT][2][G], m[NT][2], l[NT][2];
    int b = look.b, h = look.h;  // of the piece
    auto begin_piece = [&]() {
      const int g = a.qt == 1 ? h : h / a.qt, q0 = (h - g * a.qt) * ROWS;
      const __nv_bfloat16* q = a.q + b * a.q_stride + static_cast<int64_t>(g) * gs * D;
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const int row = q0 + x * 8 + r;
        float sum[G];
#pragma unroll
        for (int i = 0; i < G; ++i) sum[i] = 0.f;
#pragma unroll
        for (int i = 0; i < BLK; ++i) {
          uint4 u = make_uint4(0, 0, 0, 0);
          if (row < gs) u = *reinterpret_cast<const uint4*>(q + static_cast<int64_t>(row) * D + 32 * i + 8 * c);
          sum[i / BG] += ((bf16_lo(u.x) + bf16_hi(u.x)) + (bf16_lo(u.y) + bf16_hi(u.y))) +
                         ((bf16_lo(u.z) + bf16_hi(u.z)) + (bf16_lo(u.w) + bf16_hi(u.w)));
          qf[x][i][0] = __byte_perm(u.x, u.z, 0x5410);
          qf[x][i][1] = __byte_perm(u.x, u.z, 0x7632);
          qf[x][i][2] = __byte_perm(u.y, u.w, 0x5410);
          qf[x][i][3] = __byte_perm(u.y, u.w, 0x7632);
        }
        // a 64th of a group's sum (as the codes are 64ths) in three bf16 numbers, 24 bits, each
        // with its eightfold in front
        uint32_t piece[G][3];
#pragma unroll
        for (int i = 0; i < G; ++i) {
          sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
          sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
          float rest = sum[i] * 0.015625f;
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            const float f = __bfloat162float(__float2bfloat16_rn(rest));
            piece[i][k] = pack_bf16x2(8.f * f, f);
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
          m[x][i] = -INFINITY;
          l[x][i] = 0.f;
#pragma unroll
          for (int g2 = 0; g2 < G; ++g2) low[x][i][g2] = 0.f;
        }
#pragma unroll
        for (int s = 0; s < 2 * BLK; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[s][x][i] = 0.f;
      }
    };
    // a finished piece: its sums over the lanes, the lows added to the outputs
    auto end_piece = [&]() {
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
              o[s][x][i] = fmaf(o[s][x][i], 64.f, low[x][i][g]);
              o[s][x][i + 2] = fmaf(o[s][x][i + 2], 64.f, low[x][i][g]);
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
    const float sl2 = 64.f * a.sl2;  // of scores in 64ths
    // the first steps only fill the ring (one copy of the code: a short share runs it cold)
    for (int i = 1 - STAGES; i < n; ++i) {
      if (i + STAGES - 1 < n) {
        issue(fill);
        fill = fill + 1 == STAGES ? 0 : fill + 1;
        if (i + STAGES < n) {
          look.next(a, pre, L::BYTES);
          lookup();
        }
      }
      if (i < 0) {
        if (i == -1) begin_piece();
        continue;
      }
      if (!__all_sync(0xffffffffu, mbar_wait(bar_s + slot * 8, parity, a.limit_ns, &abort_flag))) {
        if (lane == 0) report_status(a.status, DECOMOE_ERR_TIMEOUT);
        // no results; what is in flight gets the same time to land
        for (int k = 1; k < STAGES && i + k < n; ++k) {
          slot = slot + 1 == STAGES ? (parity ^= 1, 0) : slot + 1;
          mbar_wait(bar_s + slot * 8, parity, a.limit_ns, &abort_flag);
        }
        break;
      }
      const uint32_t stage = ring_s + slot * STAGE;
      const int4 info = tile_info[warp][slot];
      if (info.y != b || info.z != h) {  // a new pair
        b = info.y;
        h = info.z;
        began = false;
        begin_piece();
      }
      const uint32_t mask = static_cast<uint32_t>(info.x);
      // ---- scores: sum over the groups of step (q (code - 8)) + (low + 8 step) (sum of q)
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
#pragma unroll
          for (int i2 = 0; i2 < 4; ++i2) sc[u][x][i2] = 0.f;
          pga_mma(sc[u][x], kx, qs[x][0], qs[x][1]);
          if constexpr (G == 4) pga_mma(sc[u][x], kx, qs[x][2], 0u);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float acc[NT][4] = {};
#pragma unroll
          for (int i2 = g * BG; i2 < (g + 1) * BG; ++i2) {
            uint32_t f0[4], f1[4];
            q4a_codes(kw[0][i2], f0);
            q4a_codes(kw[1][i2], f1);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const uint32_t f[4] = {f0[2 * s], f1[2 * s], f0[2 * s + 1], f1[2 * s + 1]};
#pragma unroll
              for (int x = 0; x < NT; ++x) pga_mma(acc[x], f, qf[x][i2][2 * s], qf[x][i2][2 * s + 1]);
            }
          }
#pragma unroll
          for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int i2 = 0; i2 < 4; ++i2) sc[u][x][i2] = fmaf(bf16_lo(kp[i2 >> 1][g]), acc[x][i2], sc[u][x][i2]);
        }
      }
      if (mask != 0xffffffffu) {
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            if (!((mask >> (16 * u + 8 * hf + kr)) & 1u)) {
              // anything may lie where nothing is seen
#pragma unroll
              for (int x = 0; x < NT; ++x) sc[u][x][2 * hf] = sc[u][x][2 * hf + 1] = -INFINITY;
            }
      }
      // ---- the maxima so far, raised only where one is passed by 2^8: weights up to 2^8 cost no
      // digits, and rescaling the outputs is rare
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        float mx[2];
#pragma unroll
        for (int i2 = 0; i2 < 2; ++i2) {
          mx[i2] = fmaxf(sc[0][x][i2], sc[0][x][i2 + 2]);
#pragma unroll
          for (int u = 1; u < SUB; ++u) mx[i2] = fmaxf(mx[i2], fmaxf(sc[u][x][i2], sc[u][x][i2 + 2]));
        }
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) {
          mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], w));
          mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], w));
        }
        mx[0] *= sl2;
        mx[1] *= sl2;
        if (__any_sync(0xffffffffu, mx[0] > m[x][0] + 8.f || mx[1] > m[x][1] + 8.f)) {
#pragma unroll
          for (int i2 = 0; i2 < 2; ++i2) {
            const float to = fmaxf(m[x][i2], mx[i2]);
            // nothing seen so far, and nothing here: any factor does
            const float f = to == -INFINITY ? 1.f : pga_ex2(m[x][i2] - to);
            m[x][i2] = to;
            l[x][i2] *= f;
#pragma unroll
            for (int g = 0; g < G; ++g) low[x][i2][g] *= f;
#pragma unroll
            for (int s = 0; s < 2 * BLK; ++s) {
              o[s][x][i2] *= f;
              o[s][x][i2 + 2] *= f;
            }
          }
        }
      }
      // ---- weights and values
      float ref[NT][2];
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int i2 = 0; i2 < 2; ++i2) ref[x][i2] = m[x][i2] == -INFINITY ? 0.f : m[x][i2];
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const uint32_t at[2] = {stage + 2 * u * L::BYTES, stage + (2 * u + 1) * L::BYTES};
        uint32_t vp[2][G];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) q4a_lds(at[hf] + L::VP + kr * L::PARAMS, vp[hf]);
        if (mask != 0xffffffffu) {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            if (!((mask >> (16 * u + 8 * hf + kr)) & 1u))
#pragma unroll
              for (int g = 0; g < G; ++g) vp[hf][g] = 0u;
        }
        uint32_t p[NT][G][2];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          float w[4];
#pragma unroll
          for (int i2 = 0; i2 < 4; ++i2) w[i2] = pga_ex2(fmaf(sc[u][x][i2], sl2, -ref[x][i2 & 1]));
          l[x][0] += w[0] + w[2];
          l[x][1] += w[1] + w[3];
          // weights times steps are the operands of the value product; lows and 8 steps add up in fp32
#pragma unroll
          for (int g = 0; g < G; ++g)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const float step = bf16_lo(vp[hf][g]), at8 = fmaf(8.f, step, bf16_hi(vp[hf][g]));
              low[x][0][g] = fmaf(w[2 * hf], at8, low[x][0][g]);
              low[x][1][g] = fmaf(w[2 * hf + 1], at8, low[x][1][g]);
              p[x][g][hf] = pga_transpose(pack_bf16x2(w[2 * hf] * step, w[2 * hf + 1] * step));
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
            for (int x = 0; x < NT; ++x) pga_mma(o[2 * i2 + s][x], f, p[x][i2 / BG][0], p[x][i2 / BG][1]);
          }
        }
      }
      __syncwarp();
      slot = slot + 1 == STAGES ? (parity ^= 1, 0) : slot + 1;
      if (info.w || i + 1 == n) {
        end_piece();
        if (!info.w) {  // goes on in the next share; the ring is empty
          keep_piece(mine);
          if (lane == 0) meta[warp] = make_int3(began ? 2 : 1, b, h);
        } else if (began) {
          // begun before the block: it is all that the block holds of its pair
          keep_piece(warp == 0 ? part : a.early + static_cast<int64_t>(me) * ROWS * ROW);
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
  pga_join_block<D, NT>(a, plan, meta, q4a_smem, RING);
}

}  // namespace decomoe

using namespace decomoe;

extern "C" {

size_t decomoe_paged_attention_q4_workspace_bytes(int64_t B, int Hq, int Hkv, int D) {
  if (B <= 0 || Hkv <= 0 || Hq < Hkv || D <= 0) return 0;
  // the pieces of every warp and of every block, two blocks per SM
  const size_t rows = static_cast<size_t>(pga_rows(Hq, Hkv)) * pga_row(D) * sizeof(float);
  return static_cast<size_t>(std::min(2 * sm_count(), Q4A_BLOCKS)) * ((PGA_WARPS + 2) * rows + sizeof(int4));
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
  const int64_t page = Hkv * (page_size / 8) * q4_tile_bytes(D, group);
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
  const int per_sm = rows == 8 ? 2 : 1;
  const int grid = static_cast<int>(
      std::max<int64_t>(1, std::min<int64_t>(std::min(per_sm * sm_count(), Q4A_BLOCKS), (most + PGA_WARPS - 1) / PGA_WARPS)));
  const size_t piece = static_cast<size_t>(rows) * pga_row(D);
  a.early = static_cast<float*>(ws);
  a.part = a.early + static_cast<size_t>(grid) * PGA_WARPS * piece;
  a.info = reinterpret_cast<int4*>(a.part + static_cast<size_t>(grid) * 2 * piece);
  const size_t smem = static_cast<size_t>(PGA_WARPS) * q4a_stages(D) * Q4A_SETS * q4_tile_bytes(D, group) +
                      2 * (static_cast<size_t>(B) + 1) * sizeof(int);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto main, auto join) -> int {
    DM_CUDA_CHECK(cudaFuncSetAttribute(main, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    DM_CUDA_CHECK(launch_pdl(main, dim3(grid), dim3(PGA_THREADS), smem, s, a));
    DM_CUDA_CHECK(launch_pdl(join, dim3(grid), dim3(32 * PGM_WARPS), 0, s, static_cast<const PagedCommon&>(a)));
    return DECOMOE_OK;
  };
  return q4_dispatch(D, group, [&](auto d, auto g) -> int {
    return rows == 8 ? go(k_paged_attention_q4<d.value, g.value, 1>, k_paged_join<d.value, 1, Q4A_BLOCKS>)
                     : go(k_paged_attention_q4<d.value, g.value, 2>, k_paged_join<d.value, 2, Q4A_BLOCKS>);
  });
}

}  // extern "C"
