// Attention of one new token per request over a paged key-value cache in 4 bits
// (decoding on the text-only cache, DecoMoE Section 3.2 and Algorithm 2, last step, for a
// batch of requests), the visual block of a request left out where it has exited.
#include "paged_q4.cuh"
#include "paged_share.cuh"

namespace decomoe {

constexpr int Q4A_STAGES = 4;
constexpr int Q4A_BLOCKS = 320;  // of a launch, at most
constexpr int Q4A_EXTRA = 3;     // what a (request, KV head) pair costs beside its tiles, in tiles

// A tile: KEYS consecutive rows of a request from a multiple of KEYS on (so that eight rows
// always lie together in a page), those that are hidden or past the length left out of
// the sums. Tiles of hidden rows alone are not numbered.
template <int D, int G>
struct Q4aTile {
  using L = Q4Tile<D, G>;
  static constexpr int KEYS = 2048 / D;  // 16 or 32
  static constexpr int SETS = KEYS / 8;  // pieces of eight rows
  static constexpr int STAGE = SETS * L::BYTES;
  static constexpr int ROW = pga_row(D);
  static __device__ __forceinline__ int before(const PgaReq& r) { return (r.h0 + KEYS - 1) / KEYS; }  // the hidden block
  static __device__ __forceinline__ int after(const PgaReq& r) { return max(before(r), (r.h0 + r.hc) / KEYS); }
  static __device__ __forceinline__ int count(const PgaReq& r) {
    const int n = r.seen + r.hc;
    return before(r) + (r.h0 + r.hc < n ? (n + KEYS - 1) / KEYS - after(r) : 0);
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
// The codes at bits 4 s of the two halves of w, as bf16 numbers q - 8: 128 + q is exact
// in bf16, and so is its difference from 136.
__device__ __forceinline__ uint32_t q4a_codes(uint32_t w, int s) {
  const uint32_t u = ((w >> (4 * s)) & 0x000f000fu) | 0x43004300u;
  const __nv_bfloat162 c = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), c);
  return *reinterpret_cast<const uint32_t*>(&r);
}

template <int D, int G, int NT>
__global__ void __launch_bounds__(PGA_THREADS, NT == 1 ? 2 : 1) k_paged_attention_q4(PagedQ4Args a) {
  using T = Q4aTile<D, G>;
  using L = Q4Tile<D, G>;
  constexpr int BLK = D / 32;      // blocks of 32 features
  constexpr int BG = BLK / G;      // of a group
  constexpr int ROWS = 8 * NT;
  constexpr int RING = Q4A_STAGES * T::STAGE;
  static_assert(ROWS * T::ROW * 4 <= RING, "a piece fits the ring");
  extern __shared__ __align__(1024) uint8_t q4a_smem[];
  __shared__ __align__(8) uint64_t bars[PGA_WARPS][Q4A_STAGES];
  __shared__ uint32_t seen_mask[PGA_WARPS][Q4A_STAGES];
  __shared__ int3 meta[PGA_WARPS];
  __shared__ int abort_flag;
  int* pre = reinterpret_cast<int*>(q4a_smem + PGA_WARPS * RING);
  int* nz = pre + a.B + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) abort_flag = 0;
  if (lane < Q4A_STAGES) mbar_init(smem_u32(&bars[warp][lane]), 1);
  fence_mbar_init();
  pdl_enter();
  const PgaPlan plan = pga_begin<T, D>(a, pre, nz);
  const int me = blockIdx.x * PGA_WARPS + warp;
  // lane 0 seeks the start of this warp's share, lane 1 that of the next one's
  PgaWalk<T> look;
  const int from = plan.place(me + (lane & 1));
  const int first = from < plan.total ? look.seek(plan, from) : pre[a.B] * a.hv;
  const int r0 = __shfl_sync(0xffffffffu, first, 0), r1 = __shfl_sync(0xffffffffu, first, 1);
  const int gs = a.hq / a.hkv;

  uint8_t* ring = q4a_smem + warp * RING;
  const uint32_t ring_s = smem_u32(ring), bar_s = smem_u32(&bars[warp][0]);
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
    const int in_page = (1 << a.shift) - 1;
    int page = -1;
    uint32_t want = 0;  // the tile's rows that the request sees
    const uint8_t* src = nullptr;
    auto lookup = [&]() {  // the page of this lane's eight rows
      const int at = (look.t < T::before(look.r) ? look.t : look.t - T::before(look.r) + T::after(look.r)) * T::KEYS;
      const int j = at + lane, n = look.r.seen + look.r.hc;
      want = __ballot_sync(0xffffffffu, lane < T::KEYS && j < n && (j < look.r.h0 || j >= look.r.h0 + look.r.hc));
      const int p = at + lane * 8;
      page = -1;
      if (lane < T::SETS && ((want >> (lane * 8)) & 0xffu)) page = a.table[look.b * a.max_pages + (p >> a.shift)];
      src = a.pages + ((static_cast<int64_t>(look.h / a.qt) << a.shift >> 3) + ((p & in_page) >> 3)) * L::BYTES;
    };
    auto issue = [&](int slot) {
      const bool some = lane < T::SETS && ((want >> (lane * 8)) & 0xffu);
      const bool there = some && page >= 0 && page < a.num_pages;
      if (some && !there) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
      const uint32_t sets = __ballot_sync(0xffffffffu, there), bar = bar_s + slot * 8;
      if (lane == 0) {
        uint32_t mask = want;
#pragma unroll
        for (int i = 0; i < T::SETS; ++i)
          if (!((sets >> i) & 1u)) mask &= ~(0xffu << (8 * i));
        seen_mask[warp][slot] = mask;
        mbar_arrive_expect_tx(bar, __popc(sets) * L::BYTES);
      }
      __syncwarp();
      if (there) q4a_bulk(ring_s + slot * T::STAGE + lane * L::BYTES, src + page * a.page_stride, L::BYTES, bar);
    };
    const int n = r1 - r0;
    lookup();

    // a lane's part of the operands: row kr of eight keys, word (kr, c) of the codes; keys c and
    // c + 4 of eight values, features 32 i + 4 r .. + 3
    const int r = lane >> 2, c = lane & 3, kr = (r >> 1) + 4 * (r & 1);
    uint32_t qf[NT][BLK][4], qs[NT][G == 4 ? 3 : 2];
    float o[2 * BLK][NT][4], off[NT][2][G], m[NT][2], l[NT][2];
    auto begin_piece = [&]() {
      const int g = use.h / a.qt, q0 = (use.h - g * a.qt) * ROWS;
      const __nv_bfloat16* q = a.q + use.b * a.q_stride + static_cast<int64_t>(g) * gs * D;
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
        // a group's sum as three bf16 numbers (24 bits), each with its eightfold in front
        uint32_t piece[G][3];
#pragma unroll
        for (int i = 0; i < G; ++i) {
          sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
          sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
          float rest = sum[i];
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
          for (int g2 = 0; g2 < G; ++g2) off[x][i][g2] = 0.f;
        }
#pragma unroll
        for (int s = 0; s < 2 * BLK; ++s)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[s][x][i] = 0.f;
      }
    };
    // a finished piece: its sums over the lanes, the offsets added to the outputs
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
            for (int w = 4; w < 32; w <<= 1) off[x][i][g] += __shfl_xor_sync(0xffffffffu, off[x][i][g], w);
#pragma unroll
            for (int s = 2 * BG * g; s < 2 * BG * (g + 1); ++s) {
              o[s][x][i] += off[x][i][g];
              o[s][x][i + 2] += off[x][i][g];
            }
          }
        }
    };
    auto keep_piece = [&](float* dst) {
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float* row = dst + (x * 8 + 2 * c + i) * T::ROW;
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
    bool began = use.t > 0;  // the piece's pair began in an earlier share
    int slot = 0, fill = 0;
    uint32_t parity = 0;
    // the first steps only fill the ring (one copy of the code: a short share runs it cold)
    for (int i = 1 - Q4A_STAGES; i < n; ++i) {
      if (i + Q4A_STAGES - 1 < n) {
        issue(fill);
        fill = fill + 1 == Q4A_STAGES ? 0 : fill + 1;
        if (i + Q4A_STAGES < n) {
          look.next(a, pre);
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
        for (int k = 1; k < Q4A_STAGES && i + k < n; ++k) {
          slot = slot + 1 == Q4A_STAGES ? (parity ^= 1, 0) : slot + 1;
          mbar_wait(bar_s + slot * 8, parity, a.limit_ns, &abort_flag);
        }
        break;
      }
      const uint32_t stage = ring_s + slot * T::STAGE;
      const uint32_t mask = seen_mask[warp][slot];
#pragma unroll
      for (int u = 0; u < T::SETS / 2; ++u) {
        const uint32_t at[2] = {stage + 2 * u * L::BYTES, stage + (2 * u + 1) * L::BYTES};
        // ---- scores: sum over the groups of step (q (code - 8)) + (low + 8 step) (sum of q)
        uint32_t kp[2][G];
        float sc[NT][4] = {};
        {
          uint32_t kw[2][BLK], kx[4];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            q4a_lds(at[h] + L::K + kr * L::CODES + c * (L::CODES / 4), kw[h]);
            q4a_lds(at[h] + L::KP + kr * L::PARAMS, kp[h]);
            kx[h] = kx[h + 2] = q4a_lds(at[h] + L::KP + kr * L::PARAMS + (c % G) * 4);
          }
#pragma unroll
          for (int x = 0; x < NT; ++x) {
            pga_mma(sc[x], kx, qs[x][0], qs[x][1]);
            if constexpr (G == 4) pga_mma(sc[x], kx, qs[x][2], 0u);
          }
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float acc[NT][4] = {};
#pragma unroll
            for (int i2 = g * BG; i2 < (g + 1) * BG; ++i2)
#pragma unroll
              for (int s = 0; s < 2; ++s) {
                const uint32_t f[4] = {q4a_codes(kw[0][i2], 2 * s), q4a_codes(kw[1][i2], 2 * s),
                                       q4a_codes(kw[0][i2], 2 * s + 1), q4a_codes(kw[1][i2], 2 * s + 1)};
#pragma unroll
                for (int x = 0; x < NT; ++x) pga_mma(acc[x], f, qf[x][i2][2 * s], qf[x][i2][2 * s + 1]);
              }
#pragma unroll
            for (int x = 0; x < NT; ++x)
#pragma unroll
              for (int i2 = 0; i2 < 4; ++i2) sc[x][i2] = fmaf(bf16_lo(kp[i2 >> 1][g]), acc[x][i2], sc[x][i2]);
          }
        }
        // ---- weights
        const uint32_t sees = mask >> (16 * u);
        const bool lo = (sees >> kr) & 1u, hi = (sees >> (8 + kr)) & 1u;
        uint32_t vp[2][G];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          q4a_lds(at[h] + L::VP + kr * L::PARAMS, vp[h]);
#pragma unroll
          for (int g = 0; g < G; ++g) vp[h][g] = (h ? hi : lo) ? vp[h][g] : 0u;  // anything may lie there
        }
        uint32_t p[NT][G][2];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          float mx[2];
#pragma unroll
          for (int i2 = 0; i2 < 2; ++i2) {
            sc[x][i2] = lo ? sc[x][i2] * a.sl2 : -INFINITY;
            sc[x][i2 + 2] = hi ? sc[x][i2 + 2] * a.sl2 : -INFINITY;
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
              for (int g = 0; g < G; ++g) off[x][i2][g] *= f;
#pragma unroll
              for (int s = 0; s < 2 * BLK; ++s) {
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
          // weights times steps are the operands of the value product; lows and 8 steps add up in fp32
#pragma unroll
          for (int g = 0; g < G; ++g)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float step = bf16_lo(vp[h][g]), at8 = fmaf(8.f, step, bf16_hi(vp[h][g]));
              off[x][0][g] = fmaf(w[2 * h], at8, off[x][0][g]);
              off[x][1][g] = fmaf(w[2 * h + 1], at8, off[x][1][g]);
              p[x][g][h] = pga_transpose(pack_bf16x2(w[2 * h] * step, w[2 * h + 1] * step));
            }
        }
        // ---- values
        uint32_t vw[2][2][BLK / 2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            q4a_lds(at[h] + L::V + (c + 4 * k) * L::CODES + r * (L::CODES / 8), vw[h][k]);
#pragma unroll
        for (int i2 = 0; i2 < BLK; ++i2) {
          uint32_t t[2];  // of the two keys of each half
#pragma unroll
          for (int h = 0; h < 2; ++h) t[h] = __byte_perm(vw[h][0][i2 / 2], vw[h][1][i2 / 2], i2 & 1 ? 0x7632 : 0x5410);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const uint32_t f[4] = {q4a_codes(t[0], 2 * s), q4a_codes(t[0], 2 * s + 1), q4a_codes(t[1], 2 * s),
                                   q4a_codes(t[1], 2 * s + 1)};
#pragma unroll
            for (int x = 0; x < NT; ++x) pga_mma(o[2 * i2 + s][x], f, p[x][i2 / BG][0], p[x][i2 / BG][1]);
          }
        }
      }
      __syncwarp();
      slot = slot + 1 == Q4A_STAGES ? (parity ^= 1, 0) : slot + 1;
      const bool ends = use.t + 1 == use.tiles;
      if (ends || i + 1 == n) {
        end_piece();
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
              const int row = q0 + x * 8 + 2 * c + i2;
              if (row < gs) {
                const float f = l[x][i2] != 0.f ? 1.f / l[x][i2] : 0.f;
                __nv_bfloat16* dst = a.out + (static_cast<int64_t>(use.b) * a.hq + g * gs + row) * D + 4 * r;
#pragma unroll
                for (int s = 0; s < BLK; ++s)
                  *reinterpret_cast<uint2*>(dst + 32 * s) =
                      make_uint2(pack_bf16x2(o[2 * s][x][i2] * f, o[2 * s][x][i2 + 2] * f),
                                 pack_bf16x2(o[2 * s + 1][x][i2] * f, o[2 * s + 1][x][i2 + 2] * f));
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
  const int keys = 2048 / D;
  const int64_t most = B * ((max_pages * page_size + keys - 1) / keys + 1) * a.hv;  // tiles, at most
  DM_ARG_CHECK(most + Q4A_EXTRA * B * a.hv <= INT_MAX, "paged_attention_q4: B * max_pages * page_size * heads is too large");
  const int per_sm = rows == 8 ? 2 : 1;
  const int grid = static_cast<int>(
      std::max<int64_t>(1, std::min<int64_t>(std::min(per_sm * sm_count(), Q4A_BLOCKS), (most + PGA_WARPS - 1) / PGA_WARPS)));
  const size_t piece = static_cast<size_t>(rows) * pga_row(D);
  a.early = static_cast<float*>(ws);
  a.part = a.early + static_cast<size_t>(grid) * PGA_WARPS * piece;
  a.info = reinterpret_cast<int4*>(a.part + static_cast<size_t>(grid) * 2 * piece);
  const size_t smem = static_cast<size_t>(PGA_WARPS) * Q4A_STAGES * (keys / 8) * q4_tile_bytes(D, group) +
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
