// What the attentions over paged caches share (bf16 pages: paged_attention.cu, 4-bit
// pages: paged_attention_q4.cu): how the tiles of all requests are numbered and divided
// among the warps of a launch, and how the pieces of a (request, KV head) pair that the
// division cuts are joined. A kernel of W warps keeps for each warp a ring in shared memory,
// in which the warp's last piece waits once the ring is drained.
#pragma once

#include <cfloat>

#include "decomoe_internal.cuh"

namespace decomoe {

// Floats of a partial row: outputs, m, l (bank-conflict-free stores).
constexpr int pga_row(int D) { return D + 4; }

struct PagedCommon {
  const __nv_bfloat16* q;
  const int32_t *table, *len, *hide_begin, *hide_count;
  __nv_bfloat16* out;
  float* early;  // [warps][rows][row] pieces that end inside a warp's share
  float* part;   // [blocks][2][rows][row] joined pieces of a block: of a pair begun before it, of one that goes on after it
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
__device__ __forceinline__ PgaReq pga_request(const PagedCommon& a, int b, bool* bad) {
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
  int active;      // warps of a block that have a share
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

// The C floats (1, 2 or 4) of a partial row that a lane holds.
template <int C>
struct PgaVec {
  float v[C];
};
template <bool PAST_L1, int C>
__device__ __forceinline__ void pga_load(PgaVec<C>& d, const float* p) {
  if constexpr (C == 4) {
    const float4 u = PAST_L1 ? __ldcg(reinterpret_cast<const float4*>(p)) : *reinterpret_cast<const float4*>(p);
    d.v[0] = u.x, d.v[1] = u.y, d.v[2] = u.z, d.v[3] = u.w;
  } else if constexpr (C == 1) {
    d.v[0] = PAST_L1 ? __ldcg(p) : *p;
  } else {
    const float2 u = PAST_L1 ? __ldcg(reinterpret_cast<const float2*>(p)) : *reinterpret_cast<const float2*>(p);
    d.v[0] = u.x, d.v[1] = u.y;
  }
}
template <int C>
__device__ __forceinline__ void pga_store(float* p, const PgaVec<C>& d) {
  if constexpr (C == 4) *reinterpret_cast<float4*>(p) = make_float4(d.v[0], d.v[1], d.v[2], d.v[3]);
  else if constexpr (C == 1) *p = d.v[0];
  else *reinterpret_cast<float2*>(p) = make_float2(d.v[0], d.v[1]);
}
// The result: the outputs over the sum (nothing seen: zeros), as bf16.
template <int C>
__device__ __forceinline__ void pga_result(__nv_bfloat16* dst, const PgaVec<C>& o, float l) {
  const float f = l != 0.f ? 1.f / l : 0.f;
  if constexpr (C == 4)
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o.v[0] * f, o.v[1] * f), pack_bf16x2(o.v[2] * f, o.v[3] * f));
  else if constexpr (C == 1)
    *dst = __float2bfloat16_rn(o.v[0] * f);
  else
    *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(o.v[0] * f, o.v[1] * f);
}

// A position in the numbered tiles: tile t of pair (request b, head tile h).
// Tiles::count(r): the tiles of a request.
template <class Tiles>
struct PgaWalk {
  int b, h, t, tiles;
  PgaReq r;
  __device__ __forceinline__ void enter(const PagedCommon& a) {
    bool bad = false;  // marked by the launch's first look at the lengths
    r = pga_request(a, b, &bad);
    tiles = Tiles::count(r);
  }
  // To the first tile at or after place p (p < total); its number over all pairs.
  __device__ __forceinline__ int seek(const PgaPlan& plan, int p) {
    int lo = 0, hi = plan.B;  // the last request with places <= p: it is not empty
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (plan.places(mid) <= p) lo = mid;
      else hi = mid;
    }
    return at(plan, lo, p);
  }
  // The same by all lanes of a warp, a place for each half of it (p <= total, where it is meaningless).
  __device__ __forceinline__ int seek_by_halves(const PgaPlan& plan, int p) {
    const int lane = threadIdx.x & 15;
    int lo = 0;
    for (int n = plan.B; n > 1;) {
      n = (n + 15) >> 4;
      const int b = lo + lane * n;
      const uint32_t le = __ballot_sync(0xffffffffu, b < plan.B && plan.places(b) <= p);
      lo += (__popc(le & 0xffffu << (threadIdx.x & 16)) - 1) * n;
    }
    return at(plan, lo, p);
  }
  __device__ __forceinline__ int at(const PgaPlan& plan, int request, int p) {
    b = request;
    tiles = plan.pre[b + 1] - plan.pre[b];
    const int in = p - plan.places(b), each = max(tiles + plan.extra, 1);  // (p = total may lie behind an empty request)
    h = in / each;
    t = max(in - h * each - plan.extra, 0);
    return plan.pre[b] * plan.hv + h * tiles + t;
  }
  // To the next tile; in the last pair it stays past the end (nobody looks).
  __device__ __forceinline__ void next(const PagedCommon& a, const int* pre) {
    if (++t < tiles) return;
    t = 0;
    if (++h < a.hv) return;
    h = 0;
    do ++b;
    while (b < a.B && pre[b + 1] == pre[b]);
    if (b < a.B) enter(a);
  }
};

// The start of a launch, by every thread of a block: the tiles of every request added up
// in pre and nz (shared memory, [B + 1] each), zeros for the requests that see nothing, and
// the division of the tiles among the launch's warps: W of every block, or where FEW is not 0 and there are
// fewer tiles than that, the first FEW or more of every block. TABLE: the blocks bring the tables' lines into L2
// together, ahead of the lookups.
template <class Tiles, int D, int W, int FEW = 0, bool TABLE = false>
__device__ __forceinline__ PgaPlan pga_begin(const PagedCommon& a, int* pre, int* nz) {
  constexpr int THREADS = 32 * W;
  __shared__ int scan_w[2][W];
  // (warp numbers that the compiler sees to be the same in all lanes spare branches and joins of lanes)
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  // ---- tiles of every request, added up
  {
    const int per = (a.B + THREADS - 1) / THREADS;
    const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    bool bad = false;
    int sum = 0, some = 0;
    for (int b = b0; b < b1; ++b) {
      const PgaReq r = pga_request(a, b, &bad);
      const int n = Tiles::count(r);
      pre[b + 1] = n;
      sum += n;
      if (TABLE) {
        const int32_t* row = a.table + b * a.max_pages;
        const int used = static_cast<int>((static_cast<int64_t>(r.seen) + r.hc + (1 << a.shift) - 1) >> a.shift);
        for (int i = blockIdx.x * 32; i < used; i += gridDim.x * 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + i));
      }
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
    for (int w = 0; w < W; ++w)
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
      for (int i = tid; i < a.hq * D / 8; i += THREADS) o[i] = make_uint4(0, 0, 0, 0);
    }
  PgaPlan plan;
  plan.pre = pre;
  plan.nz = nz;
  plan.B = a.B;
  plan.hv = a.hv;
  const int blocks = static_cast<int>(gridDim.x), all = pre[a.B] * a.hv;
  plan.extra = all > blocks * W ? a.extra : 0;
  plan.active = FEW == 0 ? W : min(W, max(FEW, (all + blocks - 1) / blocks));
  plan.divide(blocks * plan.active);
  return plan;
}

// The block's pieces joined in key order, a warp per row, in one walk over the warps: the
// last piece of a warp that goes on, the whole shares of the next ones, and the first piece of
// the one in which the pair ends. What began before the block or goes on after it leaves
// joined. All pieces are loaded ahead of the walk. meta: of each warp, whether its last piece
// goes on (1: begun in its share, 2: before it), its request and head tile.
template <int D, int NT, int W, bool FEW = false>
__device__ __forceinline__ void pga_join_block(const PagedCommon& a, const PgaPlan& plan, const int3* meta,
                                               const uint8_t* rings, int ring_bytes) {
  constexpr int ROWS = 8 * NT, ROW = pga_row(D);
  constexpr int SHARERS = W > ROWS ? W / ROWS : 1;  // warps that share a row's features
  constexpr bool AHEAD = W <= 8;  // with more warps only what comes from outside the block is loaded ahead
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int gs = a.hq / a.hkv;
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * 2 * ROWS * ROW;
  constexpr int C = D / 32 / SHARERS;
  const int at = warp / ROWS * (D / SHARERS) + lane * C;
  int kind[W];  // of a warp's last piece: 0 ends there, 1 begun in its share and goes on, 2 its whole share
#pragma unroll
  for (int w = 0; w < W; ++w) kind[w] = meta[w].x;
  const int active = FEW ? plan.active : W;  // the others have nothing
#pragma unroll 1
  for (int r = SHARERS > 1 ? warp % ROWS : warp; r < ROWS; r += W) {
    PgaVec<C> last[W], early[W];
    float2 last_ml[W], early_ml[W];
    auto load_last = [&](int w) {
      const float* p = reinterpret_cast<const float*>(rings + w * ring_bytes) + r * ROW;
      last_ml[w] = *reinterpret_cast<const float2*>(p + D);
      pga_load<false>(last[w], p + at);
    };
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (AHEAD && kind[w] != 0) load_last(w);
      if (w > 0 && w < active && kind[w - 1] != 0 && kind[w] != 2) {
        const float* p = a.early + (static_cast<int64_t>(blockIdx.x * W + w) * ROWS + r) * ROW;
        early_ml[w] = *reinterpret_cast<const float2*>(p + D);
        pga_load<false>(early[w], p + at);
      }
    }
    if (tid == 0) {
      // a pair that begins here and ends in a later block
      int4 info = make_int4(0, 0, 0, 0);
      if (meta[active - 1].x != 0) {
        int w0 = active - 1;
        while (w0 > 0 && meta[w0].x == 2) --w0;
        if (meta[w0].x == 1) {
          info = make_int4(1, meta[w0].y, meta[w0].z, 0);
          const int tiles = plan.pre[info.y + 1] - plan.pre[info.y];
          const int end = plan.places(info.y) + (info.z + 1) * (tiles + plan.extra) - 1;
          info.w = plan.holder(end) / active;
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
        float* dst = part + ((open_begin ? 0 : ROWS) + r) * ROW;
        pga_store(dst + at, o);
        if (at == 0) *reinterpret_cast<float2*>(dst + D) = make_float2(m, l);
      } else {
        const int b = meta[w0].y, h = meta[w0].z, g = a.qt == 1 ? h : h / a.qt, q = (h - g * a.qt) * ROWS + r;
        if (q < gs) pga_result(a.out + (static_cast<int64_t>(b) * a.hq + g * gs + q) * D + at, o, l);
      }
    };
    bool on = false;  // a chain goes on into warp w
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if (w >= active) continue;
      if (!AHEAD && kind[w] != 0) load_last(w);
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
template <int D, int NT, int BLOCKS>
__global__ void __launch_bounds__(32 * PGM_WARPS) k_paged_join(PagedCommon a) {
  constexpr int ROWS = 8 * NT, PER = PGM_WARPS / ROWS, C = D / 32, LOADS = 8, AHEAD = 8;
  __shared__ __align__(16) float so[PGM_WARPS][D];
  __shared__ float factor[PGM_WARPS][BLOCKS];
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  const int r = warp / PER, s = warp % PER;
  auto piece = [&](int i) {
    return a.part + ((static_cast<int64_t>(blockIdx.x + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + r) * pga_row(D);
  };
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    if (pass == 1) pdl_wait();
    // the first maxima and sums come with the pair's description, whether they are its
    // pieces' or not (eight: with 32, as many requests as blocks took 1 us more)
    float2 ml[BLOCKS / 32];
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
      for (int k = 0; k < BLOCKS / 32; ++k)
        if (k * 32 + lane >= AHEAD && k * 32 + lane < n) ml[k] = __ldcg(reinterpret_cast<const float2*>(piece(k * 32 + lane) + D));
    }
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < BLOCKS / 32; ++k)
      if (k * 32 + lane < n) m = fmaxf(m, ml[k].x);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int k = 0; k < BLOCKS / 32; ++k)
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
inline int pga_rows(int Hq, int Hkv) { return Hq / Hkv <= 8 ? 8 : 16; }

}  // namespace decomoe
