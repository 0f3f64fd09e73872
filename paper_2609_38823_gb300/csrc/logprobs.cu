// Log probabilities of given tokens from a model's logits, with each row's entropy and its
// most probable alternatives: what a server returns beside the tokens it answers with
// (the base model's last step, which the method leaves unchanged).
#include <algorithm>
#include <cfloat>

#include "decomoe_internal.cuh"

namespace decomoe {

// With c = scale log2(e) and m the maximum of the elements x seen so far, a thread keeps the
// sums z of 2^d and w of 2^d d over d = (x - m) c, rescaled where m grows (pairs of elements in
// packed fp32 operations); threads, warps and blocks are added up in a fixed order against the
// largest m. Then ln p(x) = (x - m) scale - ln z and the entropy is ln z - ln 2 w / z. Elements
// count as -2^100 at least, so that masked ones (-inf, or a type's lowest value) need no case of
// their own: their 2^d is 0 and their product with d finite. A row whose maximum is not below 2^97
// in size (all masked, infinite, enormous) is computed again with every case, by one warp.
//
// The n <= 32 best: the threads fall into 64 groups, and the n-th largest of the groups'
// maxima bounds the n-th largest element from below, since groups have no element in common; about
// n to 1.5 n elements reach it. The vectors of the few runs of a thread's vectors whose maxima
// reach it are read again, elements that do are collected as 64-bit keys of value and index, all
// different, and ranked by counting; ties go to the lowest index, and no order of execution
// shows. Where more are collected than there is room for (rows of equal values), a warp reads the
// row again and keeps the n best sorted in its lanes.
//
// Bound: memory for many long rows, else latency and instructions of the best. 16384 rows of 64 KB 152 us
// without alternatives (all of the measured copy rate), 180 with five: while a row's best are found (a third of its
// time) its block loads nothing. One row of 64 KB 3.3 and 5.9 us over a cluster of eight blocks. 5238 rows of 4 KB,
// a warp each, 7.6 us without and 21 with 32. Steps of 16384 rows with five: a pass for the sums and one for the
// best 444 us; both in one, blocks per row 203; runs of vectors instead of all vectors read again 191; warp
// numbers that are uniform to the compiler 186; the groups' n-th largest bit by bit, shifts for divisions 180.
constexpr int LP_THREADS = 256;
constexpr int LP_WARPS = LP_THREADS / 32;
constexpr int LP_BEST = 32;
constexpr int LP_ROOM = 512;  // collected elements of a block, or of a row
constexpr int LP_CLUSTER = 8;  // blocks of a row, at most
constexpr int LP_RESIDENT(int W) { return W == 4 ? 48 : 40; }  // warps of an SM, for blocks of W
constexpr float LP_LN2 = 0.6931471805599453f, LP_LOG2E = 1.4426950408889634f;
constexpr float LP_LEAST = -0x1p100f;  // what elements count as at least
constexpr float LP_PLAIN = 0x1p97f;    // rows with a maximum below this in size are in the plain range

struct LpArgs {
  const void* x;
  const int32_t* tokens;
  float *logprob, *entropy, *top_logprob;
  int32_t *top_id, *status;
  int64_t T, ld;
  int V, n;
  float c;         // scale * log2(e)
  float half, per; // (x - m) scale is (half x - half m) per: half is 1/2 where x - m may not fit fp32 but the product does
};

// ---------------------------------------------------------------- arithmetic

__device__ __forceinline__ float lp_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t lp_pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 lp_split(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t lp_fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t lp_mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t lp_add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float lp_max_nan(float a, float b) {  // NaN where one is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// What a vector of 16 bytes holds: its elements, raised to LP_LEAST, as pairs; their largest;
// and the elements as they are.
template <typename E>
struct LpVec;
template <>
struct LpVec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ uint32_t word(const uint4& u, int i) {
    return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w;
  }
  static __device__ __forceinline__ uint4 raise(const uint4& u) {
    uint4 r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r.x) : "r"(u.x), "r"(0xf180f180u));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r.y) : "r"(u.y), "r"(0xf180f180u));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r.z) : "r"(u.z), "r"(0xf180f180u));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r.w) : "r"(u.w), "r"(0xf180f180u));
    return r;
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ float largest(const uint4& u) {
    const uint32_t m = max2(max2(u.x, u.y), max2(u.z, u.w));
    return fmaxf(bf16_lo(m), bf16_hi(m));
  }
  static __device__ __forceinline__ uint64_t pair(const uint4& u, int i) {
    return lp_pair(bf16_lo(word(u, i)), bf16_hi(word(u, i)));
  }
  static __device__ __forceinline__ float element(const uint4& u, int j) {
    return j & 1 ? bf16_hi(word(u, j / 2)) : bf16_lo(word(u, j / 2));
  }
  static __device__ __forceinline__ uint4 masked() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};
template <>
struct LpVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float element(const uint4& u, int j) {
    return __uint_as_float(j == 0 ? u.x : j == 1 ? u.y : j == 2 ? u.z : u.w);
  }
  static __device__ __forceinline__ uint4 raise(const uint4& u) {
    auto up = [](uint32_t v) { return __float_as_uint(lp_max_nan(__uint_as_float(v), LP_LEAST)); };
    return make_uint4(up(u.x), up(u.y), up(u.z), up(u.w));
  }
  static __device__ __forceinline__ float largest(const uint4& u) {
    return fmaxf(fmaxf(element(u, 0), element(u, 1)), fmaxf(element(u, 2), element(u, 3)));
  }
  static __device__ __forceinline__ uint64_t pair(const uint4& u, int i) {
    return i == 0 ? lp_pair(element(u, 0), element(u, 1)) : lp_pair(element(u, 2), element(u, 3));
  }
  static __device__ __forceinline__ uint4 masked() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
};

// A thread's sums; m starts at LP_LEAST.
struct LpAcc {
  float m;
  uint64_t z, w;  // pairs of partial sums
  __device__ __forceinline__ void clear() {
    m = LP_LEAST;
    z = w = 0;
  }
  __device__ __forceinline__ void grow(float to, float c) {
    const float d = fmaxf((m - to) * c, -1000.f), f = lp_ex2(d);
    const uint64_t ff = lp_pair(f, f);
    w = lp_mul2(lp_fma2(z, lp_pair(d, d), w), ff);
    z = lp_mul2(z, ff);
    m = to;
  }
  // U vectors; their largest element.
  template <typename E, int U>
  __device__ __forceinline__ float take(const uint4 (&u)[U], float c) {
    using Vec = LpVec<E>;
    uint4 x[U];
    float most = LP_LEAST;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      x[i] = Vec::raise(u[i]);
      most = fmaxf(most, Vec::largest(x[i]));
    }
    if (most > m) grow(most, c);
    const uint64_t cc = lp_pair(c, c), mm = lp_pair(-m, -m);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < Vec::N / 2; ++j) {
        const uint64_t d = lp_mul2(lp_add2(Vec::pair(x[i], j), mm), cc);
        const float2 s = lp_split(d);
        const uint64_t e = lp_pair(lp_ex2(s.x), lp_ex2(s.y));
        z = lp_add2(z, e);
        w = lp_fma2(e, d, w);
      }
    return most;
  }
  __device__ __forceinline__ void one(float v, float c) {
    v = lp_max_nan(v, LP_LEAST);
    if (v > m) grow(v, c);
    const float d = (v - m) * c, e = lp_ex2(d);
    z = lp_add2(z, lp_pair(e, 0.f));
    w = lp_fma2(lp_pair(e, 0.f), lp_pair(d, 0.f), w);
  }
};

struct LpSums {
  float m, z, w;
};
// The sums of the L lanes of each L (a power of two), in every one of them.
template <int L>
__device__ __forceinline__ LpSums lp_reduce(LpSums s, float c) {
  float m = s.m;
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float d = fmaxf((s.m - m) * c, -1000.f), f = lp_ex2(d);
  s.w = (s.w + s.z * d) * f;
  s.z *= f;
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) {
    s.z += __shfl_xor_sync(0xffffffffu, s.z, o);
    s.w += __shfl_xor_sync(0xffffffffu, s.w, o);
  }
  s.m = m;
  return s;
}
__device__ __forceinline__ LpSums lp_sums(const LpAcc& a) {
  const float2 z = lp_split(a.z), w = lp_split(a.w);
  return {a.m, z.x + z.y, w.x + w.y};
}

// ---------------------------------------------------------------- the best

// Larger values first, then lower indexes: a key of every element, 0 for none. NaN ranks as
// minus infinity, -0 as 0.
__device__ __forceinline__ uint64_t lp_key(float x, uint32_t i) {
  const uint32_t u = __float_as_uint(x != x ? -INFINITY : x + 0.f);
  const uint32_t o = u & 0x80000000u ? ~u : u | 0x80000000u;
  return static_cast<uint64_t>(o) << 32 | (0xffffffffu - i);
}
__device__ __forceinline__ float lp_key_value(uint64_t k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint32_t lp_key_index(uint64_t k) { return 0xffffffffu - static_cast<uint32_t>(k); }

// A row, or a slice of it: vectors [v0, v0 + vecs) of its whole 16-byte vectors, and (the first
// slice) up to 2 N - 2 elements around those.
template <typename E>
struct LpRow {
  const E* x;
  const uint4* xv;
  int head, vecs, v0, edges, rest_at;
  __device__ __forceinline__ LpRow(const LpArgs& a, int64_t row, int rank, int S) {
    constexpr int N = LpVec<E>::N;
    x = static_cast<const E*>(a.x) + row * a.ld;
    head = min(a.V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / static_cast<int>(sizeof(E)));
    const int all = (a.V - head) / N, rest = a.V - head - all * N;
    v0 = static_cast<int>(static_cast<int64_t>(all) * rank / S);
    vecs = static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / S) - v0;
    xv = reinterpret_cast<const uint4*>(x + head) + v0;
    edges = rank == 0 ? head + rest : 0;
    rest_at = a.V - rest;
  }
  __device__ __forceinline__ int edge_at(int i) const { return i < head ? i : rest_at + (i - head); }
  __device__ __forceinline__ int index(int v) const { return head + (v0 + v) * LpVec<E>::N; }  // of a vector's first element
};

// A row's vectors are taken in batches of LP_U a thread, thread t's vectors being t, t + threads, ...;
// up to SLOTS runs of batches leave their maxima, so that few vectors are read again.
constexpr int LP_U = 4;
constexpr int LP_SLOTS = 8;
struct LpRuns {
  int per, shift, slots;  // batches of a run (1 << shift), and runs
  __device__ __forceinline__ LpRuns(int vecs, int threads) {
    const int batches = (vecs + threads * LP_U - 1) / (threads * LP_U);
    shift = 32 - __clz((batches - 1) / LP_SLOTS);
    per = 1 << shift;
    slots = (batches + per - 1) >> shift;
  }
};

// Thread t of `threads` takes its vectors; with KEEP the maxima of its runs go to slots[run * threads],
// and those of its even and odd vectors to halves, if given.
template <typename E, bool KEEP>
__device__ __forceinline__ void lp_pass(const LpRow<E>& row, LpAcc& acc, float c, int t, int threads, LpRuns runs, float* slots,
                                        float (*halves)[2] = nullptr) {
  int v = t, left = runs.per;
  float most = LP_LEAST;
  auto ran = [&](float x) {
    if (!KEEP) return;
    most = fmaxf(most, x);
    if (--left > 0) return;
    *slots = most;
    slots += threads;
    --runs.slots;
    most = LP_LEAST;
    left = runs.per;
  };
  for (; v + (LP_U - 1) * threads < row.vecs; v += LP_U * threads) {
    uint4 u[LP_U];
#pragma unroll
    for (int i = 0; i < LP_U; ++i) u[i] = __ldg(row.xv + v + i * threads);
    ran(acc.template take<E, LP_U>(u, c));
    if (KEEP && halves != nullptr) {
#pragma unroll
      for (int i = 0; i < LP_U; ++i) (*halves)[i & 1] = fmaxf((*halves)[i & 1], LpVec<E>::largest(u[i]));
    }
  }
  if (v < row.vecs) {  // what is left, its loads in flight together
    uint4 u[LP_U - 1];
#pragma unroll
    for (int i = 0; i < LP_U - 1; ++i)
      if (v + i * threads < row.vecs) u[i] = __ldg(row.xv + v + i * threads);
    float x = LP_LEAST;
#pragma unroll
    for (int i = 0; i < LP_U - 1; ++i)
      if (v + i * threads < row.vecs) {
        const uint4 w[1] = {u[i]};
        const float y = acc.template take<E, 1>(w, c);
        x = fmaxf(x, y);
        if (KEEP && halves != nullptr) (*halves)[i & 1] = fmaxf((*halves)[i & 1], y);
      }
    ran(x);
  }
  if (KEEP)
    for (; runs.slots > 0; --runs.slots, slots += threads, most = LP_LEAST) *slots = most;
}

// The keys (count[0] of them) of the elements of `from` or more, by a warp for its threads first + lane: the
// vectors of the runs whose maxima are as large are spread over its lanes, so that one latency
// covers most rows. who: 64 ints of the warp's own.
template <typename E>
__device__ __forceinline__ void lp_collect(const LpRow<E>& row, float from, const LpRuns& runs, const float* slots, int first,
                                           int threads, uint64_t* keys, int* count, int* who) {
  const int lane = threadIdx.x & 31;
  auto push = [&](float y, int i) {
    const int at = atomicAdd(count, 1);
    if (at < LP_ROOM) keys[at] = lp_key(y, i);
  };
  static_assert(LP_U == 4, "a run is 4 << shift vectors");
  const unsigned each = LP_U << runs.shift;
  int have = 0;
  for (int s = 0; s <= runs.slots; ++s) {
    if (s == runs.slots || have > 32) {
      __syncwarp();
      for (unsigned i = lane; i < have * each; i += 32) {
        const unsigned q = i >> (runs.shift + 2);
        const int v = (who[q] & 0xffff) + threads * static_cast<int>((who[q] >> 16) * each + (i & (each - 1)));
        if (v >= row.vecs) continue;
        const uint4 u = __ldg(row.xv + v);
        if (LpVec<E>::largest(u) >= from) {
#pragma unroll
          for (int j = 0; j < LpVec<E>::N; ++j) {
            const float y = LpVec<E>::element(u, j);
            if (y >= from) push(y, row.index(v) + j);
          }
        }
      }
      __syncwarp();
      have = 0;
    }
    if (s < runs.slots) {
      const bool some = slots[s * threads + first + lane] >= from;
      const uint32_t all = __ballot_sync(0xffffffffu, some);
      if (some) who[have + __popc(all & ((1u << lane) - 1u))] = (first + lane) | s << 16;
      have += __popc(all);
    }
  }
  if (first + lane < row.edges) {
    const float y = LpVec<E>::one(row.x + row.edge_at(first + lane));
    if (y >= from) push(y, row.edge_at(first + lane));
  }
  __syncwarp();
}

// The n best of a row read once more by a warp, sorted, key i in lane i (0: none): exact
// whatever the row holds.
template <typename E>
__device__ __noinline__ uint64_t lp_sorted(LpRow<E> row, int n) {
  const int lane = threadIdx.x & 31;
  uint64_t list = 0, least = 0;  // least: the n-th
  auto offer = [&](uint64_t k) {
    uint32_t todo = __ballot_sync(0xffffffffu, k > least);
    while (todo != 0) {
      const uint64_t key = __shfl_sync(0xffffffffu, k, __ffs(todo) - 1);
      const int at = __popc(__ballot_sync(0xffffffffu, list > key));
      const uint64_t up = __shfl_up_sync(0xffffffffu, list, 1);
      list = lane < at ? list : lane == at ? key : up;
      least = __shfl_sync(0xffffffffu, list, n - 1);
      todo &= todo - 1;
      todo &= __ballot_sync(0xffffffffu, k > least);
    }
  };
  offer(lane < row.edges ? lp_key(LpVec<E>::one(row.x + row.edge_at(lane)), row.edge_at(lane)) : 0);
  for (int v = 0; v < row.vecs; v += 32) {
    const bool have = v + lane < row.vecs;
    const uint4 u = have ? __ldg(row.xv + v + lane) : make_uint4(0, 0, 0, 0);
    for (int j = 0; j < LpVec<E>::N; ++j) {
      float y = 0.f;
#pragma unroll
      for (int i = 0; i < LpVec<E>::N; ++i) y = i == j ? LpVec<E>::element(u, i) : y;
      offer(have ? lp_key(y, row.index(v + lane) + j) : 0);
    }
  }
  return list;
}

// The n best of `count` collected keys (zeros are none), key i in lane i, by a warp. Those behind the last
// are the row's first elements of minus infinity or NaN, which are not collected.
__device__ __forceinline__ uint64_t lp_rank(const uint64_t* keys, int count, int n, uint64_t* best) {
  const int lane = threadIdx.x & 31;
  if (lane < n) best[lane] = 0;
  __syncwarp();
  for (int i = lane; i < count; i += 32) {
    const uint64_t k = keys[i];
    int above = 0;
#pragma unroll 4
    for (int j = 0; j < count; ++j) above += keys[j] > k;
    if (above < n && k != 0) best[above] = k;
  }
  __syncwarp();
  return lane < n ? best[lane] : 0;
}
template <typename E>
__device__ __noinline__ uint64_t lp_fill(const E* x, int V, int n, uint64_t list) {
  const int lane = threadIdx.x & 31;
  int have = __popc(__ballot_sync(0xffffffffu, lane < n && list != 0));
  for (int i = 0; i < V && have < n; i += 32) {
    const uint32_t gone = __ballot_sync(0xffffffffu, i + lane < V && !(LpVec<E>::one(x + min(i + lane, V - 1)) >= -FLT_MAX));
    for (uint32_t todo = gone; todo != 0 && have < n; todo &= todo - 1, ++have)
      if (lane == have) list = lp_key(-INFINITY, i + __ffs(todo) - 1);
  }
  return list;
}

// Ordered as the floats are, none of them NaN; 0 is below all.
__device__ __forceinline__ uint32_t lp_order(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// A bound of the n-th largest of 64 values from below, two a lane: its upper 16 bits, found bit by bit
// between those of the least and of the largest value (seven steps or so).
__device__ __forceinline__ uint32_t lp_nth(float a, float b, int n) {
  const uint32_t x = lp_order(a) >> 16, y = lp_order(b) >> 16;
  uint32_t at = __reduce_min_sync(0xffffffffu, min(x, y));
  const uint32_t range = __reduce_max_sync(0xffffffffu, max(x, y)) - at;
  for (uint32_t step = range == 0 ? 0 : 1u << (31 - __clz(range)); step != 0; step >>= 1) {
    const uint32_t to = at + step;
    if (__popc(__ballot_sync(0xffffffffu, x >= to)) + __popc(__ballot_sync(0xffffffffu, y >= to)) >= n) at = to;
  }
  return at << 16;
}
// The least value to collect: the bound, or everything finite where some groups hold nothing plain.
__device__ __forceinline__ float lp_from(uint32_t nth) {
  const float t = __uint_as_float(nth & 0x80000000u ? nth & 0x7fffffffu : ~nth);
  return nth != 0 && t > LP_LEAST ? t : -FLT_MAX;
}
// The same bound from the maxima of a block's threads, found by one warp in what lp_pass left: for rows whose plain elements
// lie next to each other, of which few of the 64 groups see any.
template <int W>
__device__ __noinline__ float lp_from_threads(const float* slots, int runs, int n) {
  const int lane = threadIdx.x & 31;
  uint32_t x[W], least = 0xffffffffu, most = 0;
#pragma unroll
  for (int j = 0; j < W; ++j) {
    float m = LP_LEAST;
    for (int r = 0; r < runs; ++r) m = fmaxf(m, slots[(r * W + j) * 32 + lane]);
    x[j] = lp_order(m) >> 16;
    least = min(least, x[j]);
    most = max(most, x[j]);
  }
  uint32_t at = __reduce_min_sync(0xffffffffu, least);
  const uint32_t range = __reduce_max_sync(0xffffffffu, most) - at;
  for (uint32_t step = range == 0 ? 0 : 1u << (31 - __clz(range)); step != 0; step >>= 1) {
    int count = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) count += __popc(__ballot_sync(0xffffffffu, x[j] >= at + step));
    if (count >= n) at += step;
  }
  return lp_from(at << 16);
}

// ---------------------------------------------------------------- results

// A row in every case, by one warp: infinities, NaN, nothing but masks, maxima and scales of any size. Where the
// maximum is not finite it says all: minus infinity for nothing but masks, NaN or infinity for no probabilities.
// A lane has four partial sums, and three loads on their way at a time (a fourth costs the kernels that call this their
// registers: 16384 rows 182 -> 188 us). 24 rows of 151001 fp32, one of them empty, 65 us (element by element with one sum: 150).
template <typename E>
__device__ __noinline__ LpSums lp_any_case(const E* x, int V, float half, float per) {
  using Vec = LpVec<E>;
  const int lane = threadIdx.x & 31;
  LpArgs whole;
  whole.x = x;
  whole.V = V;
  whole.ld = 0;
  const LpRow<E> row(whole, 0, 0, 1);
  const float edge = lane < row.edges ? Vec::one(x + row.edge_at(lane)) : -INFINITY;
  auto walk = [&](auto take) {
    for (int v = lane; v < row.vecs; v += 3 * 32) {
      uint4 u[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) u[i] = v + 32 * i < row.vecs ? __ldg(row.xv + v + 32 * i) : Vec::masked();
#pragma unroll
      for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int j = 0; j < Vec::N; ++j) take(j & 3, Vec::element(u[i], j));
    }
  };
  float m = edge;
  walk([&](int, float y) { m = lp_max_nan(m, y); });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = lp_max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (!(fabsf(m) <= FLT_MAX)) return {m, m == -INFINITY ? 0.f : NAN, 0.f};
  float z[4] = {0.f, 0.f, 0.f, 0.f}, w[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](int j, float y) {
    // (c would be infinite for the largest scales)
    const float d = (half * y - half * m) * per * LP_LOG2E, e = lp_ex2(d);
    z[j] += e;
    w[j] = fmaf(e, fmaxf(d, -1000.f), w[j]);
  };
  add(0, edge);
  walk(add);
  z[0] = (z[0] + z[1]) + (z[2] + z[3]);
  w[0] = (w[0] + w[1]) + (w[2] + w[3]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    z[0] += __shfl_xor_sync(0xffffffffu, z[0], o);
    w[0] += __shfl_xor_sync(0xffffffffu, w[0], o);
  }
  return {m, z[0], w[0]};
}

// A row's results, by a warp: s in every lane, the keys of the best in `list`.
template <typename E>
__device__ __forceinline__ void lp_results(const LpArgs& a, int64_t row, const E* x, float logit, LpSums s,
                                           uint64_t list) {
  const int lane = threadIdx.x & 31;
  const bool plain = fabsf(s.m) < LP_PLAIN && a.c < 0x1p20f && a.c > 0x1p-80f;
  if (!plain) s = lp_any_case<E>(x, a.V, a.half, a.per);
  const float lnz = logf(s.z);
  auto logprob = [&](float y) {
    // no probability anywhere (all logits minus infinity): -inf, and an entropy of 0
    return s.z == 0.f ? -INFINITY : fmaf(a.half * y - a.half * s.m, a.per, -lnz);
  };
  if (lane == 0) {
    if (a.logprob != nullptr) a.logprob[row] = logprob(logit);
    if (a.entropy != nullptr) a.entropy[row] = s.z == 0.f ? 0.f : lnz - LP_LN2 * (s.w / s.z);
  }
  if (a.n > 0) {
    if (__any_sync(0xffffffffu, lane < a.n && list == 0)) list = lp_fill<E>(x, a.V, a.n, list);
    if (lane < a.n) {
      if (a.top_id != nullptr) a.top_id[row * a.n + lane] = static_cast<int32_t>(lp_key_index(list));
      if (a.top_logprob != nullptr) a.top_logprob[row * a.n + lane] = logprob(lp_key_value(list));
    }
  }
}

__device__ __forceinline__ bool lp_wanted(const LpArgs& a, int token) { return token >= 0 && token < a.V; }

// ---------------------------------------------------------------- short rows: a warp each

template <typename E>
__global__ void __launch_bounds__(LP_THREADS) k_logprobs_warp(LpArgs a) {
  __shared__ uint64_t keys[LP_WARPS][LP_ROOM];
  __shared__ uint64_t best[LP_WARPS][LP_BEST];
  __shared__ int count[LP_WARPS], who[LP_WARPS][64];
  __shared__ float slots[LP_WARPS][LP_SLOTS * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_enter();
  const int64_t r = static_cast<int64_t>(blockIdx.x) * LP_WARPS + warp;
  if (r >= a.T) return;
  const int token = a.tokens != nullptr ? a.tokens[r] : 0;
  if (!lp_wanted(a, token)) {
    if (token >= a.V && lane == 0) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
    return;
  }
  const LpRow<E> row(a, r, 0, 1);
  const float logit = LpVec<E>::one(row.x + token);
  const float edge = lane < row.edges ? LpVec<E>::one(row.x + row.edge_at(lane)) : 0.f;
  LpAcc acc;
  acc.clear();
  const LpRuns runs(row.vecs, 32);
  float halves[2] = {LP_LEAST, LP_LEAST};
  if (a.n > 0) lp_pass<E, true>(row, acc, a.c, lane, 32, runs, slots[warp] + lane, &halves);
  else lp_pass<E, false>(row, acc, a.c, lane, 32, runs, nullptr);
  if (lane < row.edges) acc.one(edge, a.c);
  uint64_t list = 0;
  if (a.n > 0) {
    // two groups a lane: its even vectors, and the others and the edge
    if (lane < row.edges) halves[1] = fmaxf(halves[1], edge);
    if (lane == 0) count[warp] = 0;
    __syncwarp();
    const uint32_t t = lp_nth(halves[0], halves[1], a.n);
    lp_collect<E>(row, lp_from(t), runs, slots[warp], 0, 32, keys[warp], &count[warp], who[warp]);
    list = count[warp] <= LP_ROOM ? lp_rank(keys[warp], count[warp], a.n, best[warp]) : lp_sorted<E>(row, a.n);
  }
  lp_results<E>(a, r, row.x, logit, lp_reduce<32>(lp_sums(acc), a.c), list);
}

// ---------------------------------------------------------------- few long rows: a cluster each

__device__ __forceinline__ uint32_t lp_cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t lp_at_leader(uint32_t addr) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void lp_store_at(uint32_t addr, int rank, float v) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.f32 [a], %2;\n\t}" ::"r"(addr), "r"(rank),
               "f"(v)
               : "memory");
}
__device__ __forceinline__ void lp_store_leader(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void lp_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void lp_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <typename E, int W>
__global__ void __launch_bounds__(32 * W, LP_RESIDENT(W) / W) k_logprobs_cluster(LpArgs a, int S) {
  constexpr int THREADS = 32 * W;
  __shared__ uint64_t keys[LP_ROOM];
  __shared__ uint64_t from_ranks[LP_CLUSTER * LP_BEST];
  __shared__ uint64_t best[LP_BEST];
  __shared__ LpSums warp_sums[W];
  __shared__ __align__(16) float mine_max[64], maxima[64];  // of the block's groups, and of all
  __shared__ uint64_t rank_m[LP_CLUSTER], rank_zw[LP_CLUSTER];
  __shared__ float rank_from[LP_CLUSTER];
  __shared__ int collected, who[W][64];
  __shared__ float slots[LP_SLOTS * THREADS];
  // (the warp's number as the compiler can see to be one for all lanes: 16384 rows 162 -> 155.5 us without alternatives)
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int rank = S > 1 ? static_cast<int>(lp_cluster_rank()) : 0;
  pdl_enter();
  if (S > 1) lp_cluster_arrive();  // waited for before another block's shared memory is written
  const int64_t r = blockIdx.x / S;
  const int token = a.tokens != nullptr ? a.tokens[r] : 0;
  if (!lp_wanted(a, token)) {  // every block of the cluster leaves
    if (token >= a.V && rank == 0 && tid == 0) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
    __syncwarp();
    if (S > 1) lp_cluster_wait();
    return;
  }
  const LpRow<E> row(a, r, rank, S);
  const float edge = tid < row.edges ? LpVec<E>::one(row.x + row.edge_at(tid)) : 0.f;
  const float logit = rank == 0 && warp == 0 ? LpVec<E>::one(row.x + token) : 0.f;
  LpAcc acc;
  acc.clear();
  const LpRuns runs(row.vecs, THREADS);
  if (a.n > 0) lp_pass<E, true>(row, acc, a.c, tid, THREADS, runs, slots + tid);
  else lp_pass<E, false>(row, acc, a.c, tid, THREADS, runs, nullptr);
  if (tid < row.edges) acc.one(edge, a.c);
  LpSums s = lp_reduce<32>(lp_sums(acc), a.c);
  if (lane == 0) warp_sums[warp] = s;
  // 64 groups of THREADS S / 64 lanes (a warp at most: S <= 8), `groups` of them in the block
  static_assert(THREADS / 64 * LP_CLUSTER <= 32, "groups lie in warps");
  const int lanes = THREADS / 64 * S, groups = 64 / S;
  if (a.n > 0) {
    float most = acc.m;
    for (int o = 1; o < lanes; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (lane % lanes == 0) (S > 1 ? mine_max : maxima)[tid / lanes] = most;
    if (tid == 0) collected = 0;
  }
  __syncthreads();
  if (S > 1) lp_cluster_wait();  // every block of the cluster is running
  uint64_t list = 0;
  if (a.n > 0) {
    if (S > 1) {
      if (tid < 64) lp_store_at(smem_u32(&maxima[rank * groups + tid % groups]), tid / groups, mine_max[tid % groups]);
      __syncwarp();
      lp_cluster_arrive();
      lp_cluster_wait();
    }
    float from = lp_from(lp_nth(maxima[lane], maxima[lane + 32], a.n));
    if (from == -FLT_MAX) {
      // fewer than n groups see a plain element: the largest of the blocks' own bounds (24 rows of 151001 with 600 to 5000
      // neighbours left, measured with events and a cold L2, 88 -> 20 us; with none masked 16: without a bound all of them
      // were collected, and the slice that has them read once more by one warp)
      from = lp_from_threads<W>(slots, runs.slots, a.n);
      if (S > 1) {  // (all blocks of the cluster come here, with the same maxima)
        if (tid < S) lp_store_at(smem_u32(&rank_from[rank]), tid, from);
        __syncwarp();
        lp_cluster_arrive();
        lp_cluster_wait();
        for (int i = 0; i < S; ++i) from = fmaxf(from, rank_from[i]);
      }
    }
    lp_collect<E>(row, from, runs, slots, warp * 32, THREADS, keys, &collected, who[warp]);
    __syncthreads();
    if (warp == 0) {
      if (S > 1 && collected <= a.n) list = lane < collected ? keys[lane] : 0;  // the cluster's first block ranks them all
      else list = collected <= LP_ROOM ? lp_rank(keys, collected, a.n, best) : lp_sorted<E>(row, a.n);
    }
  }
  if (warp == 0) s = lp_reduce<W>(warp_sums[lane & (W - 1)], a.c);
  if (S > 1) {
    if (warp == 0) {
      auto two = [](float hi, float lo) { return static_cast<uint64_t>(__float_as_uint(hi)) << 32 | __float_as_uint(lo); };
      if (lane == 0) {
        lp_store_leader(lp_at_leader(smem_u32(&rank_m[rank])), two(0.f, s.m));
        lp_store_leader(lp_at_leader(smem_u32(&rank_zw[rank])), two(s.z, s.w));
      }
      if (lane < a.n) lp_store_leader(lp_at_leader(smem_u32(&from_ranks[rank * a.n + lane])), list);
      __syncwarp();
    }
    lp_cluster_arrive();
    lp_cluster_wait();
    if (rank != 0 || warp != 0) return;
    if (a.n > 0) {
      int count = 0;
      for (int i = 0; i < S * a.n; i += 32) {
        const uint64_t k = i + lane < S * a.n ? from_ranks[i + lane] : 0;
        const uint32_t some = __ballot_sync(0xffffffffu, k != 0);
        if (k != 0) keys[count + __popc(some & ((1u << lane) - 1u))] = k;
        count += __popc(some);
      }
      __syncwarp();
      list = lp_rank(keys, count, a.n, best);
    }
    auto hi = [](uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); };
    auto lo = [](uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v)); };
    s = lane < S ? LpSums{lo(rank_m[lane]), hi(rank_zw[lane]), lo(rank_zw[lane])} : LpSums{LP_LEAST, 0.f, 0.f};
    s = lp_reduce<32>(s, a.c);
  }
  if (warp == 0) lp_results<E>(a, r, row.x, logit, s, list);
}

}  // namespace decomoe

using namespace decomoe;

extern "C" int decomoe_token_logprobs(const void* logits, int64_t T, int64_t V, int64_t row_stride, int dtype,
                                      const int32_t* tokens, float scale, int n, float* logprob, float* entropy,
                                      int32_t* top_id, float* top_logprob, int32_t* status_dev, decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(dtype == DECOMOE_BF16 || dtype == DECOMOE_F32, "token_logprobs: logits must be bf16 or f32");
  DM_ARG_CHECK(T >= 0 && T <= INT_MAX / 16, "token_logprobs: bad number of rows");
  DM_ARG_CHECK(V >= 1 && V <= (1 << 24), "token_logprobs: a vocabulary of 1 to 2^24 expected");
  DM_ARG_CHECK(row_stride >= V, "token_logprobs: row stride below the vocabulary's size");
  DM_ARG_CHECK(scale > 0.f && scale <= FLT_MAX, "token_logprobs: scale must be positive and finite");
  if (top_id == nullptr && top_logprob == nullptr) n = 0;
  else DM_ARG_CHECK(n >= 1 && n <= LP_BEST && n <= V, "token_logprobs: 1 to %d alternatives, at most the vocabulary's size", LP_BEST);
  DM_ARG_CHECK(logprob == nullptr || tokens != nullptr, "token_logprobs: log probabilities need tokens");
  if (T == 0) return DECOMOE_OK;
  const size_t e = dtype_bytes(dtype), rows = static_cast<size_t>(T);
  DM_ARG_CHECK(logits != nullptr, "token_logprobs: null pointer");
  DM_ARG_CHECK(reinterpret_cast<uintptr_t>(logits) % e == 0, "token_logprobs: logits are not aligned to their type");
  const Bytes in[] = {{logits, ((rows - 1) * row_stride + V) * e}, {tokens, rows * 4}};
  const Bytes out[] = {{logprob, rows * 4}, {entropy, rows * 4}, {top_id, rows * n * 4}, {top_logprob, rows * n * 4}};
  for (int i = 0; i < 4; ++i) {
    bool apart = !overlaps(out[i], {in[0], in[1]});
    for (int j = 0; j < i; ++j) apart &= !overlaps(out[i], {out[j]});
    DM_ARG_CHECK(apart, "token_logprobs: an output overlaps an input or another output");
  }
  LpArgs a = {};
  a.x = logits;
  a.tokens = tokens;
  a.logprob = logprob;
  a.entropy = entropy;
  a.top_id = top_id;
  a.top_logprob = top_logprob;
  a.status = status_dev;
  a.T = T;
  a.ld = row_stride;
  a.V = static_cast<int>(V);
  a.n = n;
  a.c = scale * LP_LOG2E;
  a.half = scale < 1.f ? 0.5f : 1.f;
  a.per = scale / a.half;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int64_t row_bytes = V * static_cast<int64_t>(e), sms = sm_count();
  auto go = [&](auto warp_rows, auto cluster, auto many) -> int {
    if (row_bytes <= 1024 || (row_bytes <= 8192 && T >= 2 * sms)) {
      DM_CUDA_CHECK(launch_pdl(warp_rows, dim3(static_cast<unsigned>((T + LP_WARPS - 1) / LP_WARPS)), dim3(LP_THREADS), 0, s, a));
      return DECOMOE_OK;
    }
    // A block per row, of four warps (twelve rows at a time on an SM) or of eight (five): whichever is sooner
    // done by this estimate, in us. Full turns and the rest go at the copy rate, the rest at least as long as a
    // block takes alone (a warp has 2 KB on their way in a us); a turn costs 4 us beside its bytes, and 4 for every
    // time that a warp reads runs again (1.25 runs an alternative). Measured with four and with eight: 700 rows of
    // 64 KB 16 and 14, 803 of 20 KB 8.2 and 10.6, 803 of 150 KB 28.6 and 33.8, 1552 of 64 KB 20 and 23, 2000 of 302
    // KB 119 and 106, 4413 of 86 KB 88 and 96, 3419 of 307 KB with 32 alternatives 243 and 196.
    auto estimate = [&](int warps) {
      const int64_t at_once = sms * (LP_RESIDENT(warps) / warps), rest = T % at_once;
      const double row = static_cast<double>(row_bytes), rate = 6.7e6, alone = 2048. * warps;
      const double run = std::max<double>(LP_U, row / (16 * 32 * warps) / LP_SLOTS);  // vectors
      const double last = rest > 0 ? std::max(static_cast<double>(rest) * row / rate, row / alone) : 0.;
      const double turns = static_cast<double>((T + at_once - 1) / at_once);
      return static_cast<double>(T - rest) * row / rate + last + (4. + 5. * a.n * run / (32 * warps)) * turns;
    };
    if (T >= 2 * sms && estimate(4) < estimate(8)) {
      DM_CUDA_CHECK(launch_pdl(many, dim3(static_cast<unsigned>(T)), dim3(128), 0, s, a, 1));
      return DECOMOE_OK;
    }
    // blocks for every SM, and a slice of at least a vector per thread
    int S = 1;
    while (S < LP_CLUSTER && T * S < 2 * sms && row_bytes > 16 * LP_THREADS * S) S *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(T * S));
    cfg.blockDim = dim3(LP_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled(T * S) ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(S);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = S > 1 ? 2 : 1;
    DM_CUDA_CHECK(cudaLaunchKernelEx(&cfg, cluster, a, S));
    return DECOMOE_OK;
  };
  return dtype == DECOMOE_BF16
             ? go(k_logprobs_warp<__nv_bfloat16>, k_logprobs_cluster<__nv_bfloat16, 8>, k_logprobs_cluster<__nv_bfloat16, 4>)
             : go(k_logprobs_warp<float>, k_logprobs_cluster<float, 8>, k_logprobs_cluster<float, 4>);
}
