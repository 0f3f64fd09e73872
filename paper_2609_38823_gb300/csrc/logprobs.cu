// Log probabilities of given tokens from a model's logits, with each row's entropy and its
// most probable alternatives: what a server returns beside the tokens it answers with
// (the base model's last step, which the method leaves unchanged).
#include <cfloat>

#include "decomoe_internal.cuh"

namespace decomoe {

// A row's vocabulary is read once, in vectors of 16 bytes, by a cluster of S blocks (S = 1
// for many rows). A thread keeps, of its elements x, their maximum m and, with
// d = (x - m) scale log2(e), the sums of 2^d and of 2^d d, both rescaled where the maximum
// grows; the block's and then the cluster's follow in a fixed order. With the row's M, Z and
// W = sum 2^d d: log p(x) = (x - M) scale - ln Z, entropy = ln Z - ln 2 W / Z.
//
// The n <= 32 best: of the threads' maxima (disjoint elements) the n-th largest is at most
// the n-th largest element, so only elements from it on can be among the n; the few threads
// that have one read their elements again and collect them, and the collected are ranked by
// counting. Elements are compared as 64-bit keys of value and index, all different, so ties
// go to the lowest index and no order of execution shows. Where more are collected than
// there is room for (a row of equal values in an unlucky order), n rounds over the slice
// take one each.
constexpr int LP_THREADS = 256;
constexpr int LP_WARPS = LP_THREADS / 32;
constexpr int LP_BEST = 32;
constexpr int LP_ROOM = 1024;  // collected elements of a block
constexpr int LP_CLUSTER = 16;
constexpr float LP_LN2 = 0.6931471805599453f;

struct LpArgs {
  const void* x;
  const int32_t* tokens;
  float *logprob, *entropy, *top_logprob;
  int32_t *top_id, *status;
  int64_t T, ld;
  int V, n;
  float scale, c;  // scale, scale * log2(e)
};

struct LpSums {
  float m, z, w;
};

__device__ __forceinline__ float lp_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The sums of a against the maximum to >= a.m; nothing (m = -inf) has none.
__device__ __forceinline__ void lp_raise(LpSums& a, float to, float c) {
  const float delta = a.m == to ? 0.f : fmaxf((a.m - to) * c, -1000.f);
  const float f = lp_ex2(delta);
  a.w = (a.w + a.z * delta) * f;
  a.z *= f;
  a.m = to;
}
__device__ __forceinline__ void lp_join(LpSums& a, LpSums b, float c) {
  const float to = fmaxf(a.m, b.m);
  lp_raise(a, to, c);
  lp_raise(b, to, c);
  a.z += b.z;
  a.w += b.w;
}
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

template <typename E>
struct LpVec;
template <>
struct LpVec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void split(const uint4& u, float (&x)[8]) {
    x[0] = bf16_lo(u.x), x[1] = bf16_hi(u.x), x[2] = bf16_lo(u.y), x[3] = bf16_hi(u.y);
    x[4] = bf16_lo(u.z), x[5] = bf16_hi(u.z), x[6] = bf16_lo(u.w), x[7] = bf16_hi(u.w);
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
};
template <>
struct LpVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void split(const uint4& u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
};

__device__ __forceinline__ uint32_t lp_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t lp_at_leader(uint32_t addr) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
__device__ __forceinline__ void lp_store_leader(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void lp_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void lp_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// The n best of count keys (all different but for zeros, which are none), best first,
// zeros after the last: by every thread of the block.
__device__ __forceinline__ void lp_best(const uint64_t* keys, int count, int n, uint64_t* best) {
  if (threadIdx.x < n) best[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += LP_THREADS) {
    const uint64_t k = keys[i];
    if (k == 0) continue;
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += keys[j] > k;
    if (rank < n) best[rank] = k;
  }
  __syncthreads();
}

template <typename E>
__global__ void __launch_bounds__(LP_THREADS) k_token_logprobs(LpArgs a, int S) {
  using Vec = LpVec<E>;
  constexpr int N = Vec::N, AHEAD = 4;
  __shared__ uint64_t keys[LP_ROOM];
  __shared__ uint64_t lists[LP_WARPS][LP_BEST];
  __shared__ uint64_t from_ranks[LP_CLUSTER * LP_BEST];
  __shared__ uint64_t best[LP_BEST];
  __shared__ LpSums warp_sums[LP_WARPS];
  __shared__ uint64_t rank_mz[LP_CLUSTER], rank_w[LP_CLUSTER];
  __shared__ uint64_t from_key;
  __shared__ int collected;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = S > 1 ? static_cast<int>(lp_rank()) : 0;
  pdl_enter();
  if (S > 1) lp_cluster_arrive();  // waited for before another block's shared memory is written
  const int64_t row = blockIdx.x / S;
  const int token = a.tokens != nullptr ? a.tokens[row] : 0;
  if (token < 0 || token >= a.V) {  // padding: every block of the cluster leaves
    if (token >= a.V && rank == 0 && tid == 0) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
    if (S > 1) lp_cluster_wait();
    return;
  }
  const E* x = static_cast<const E*>(a.x) + row * a.ld;
  // whole vectors from the first 16-byte boundary on; what lies around them is read by the first
  // threads of the first block
  const int head = min(a.V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / static_cast<int>(sizeof(E)));
  const int vecs = (a.V - head) / N, rest = a.V - head - vecs * N;
  const int v0 = static_cast<int>(static_cast<int64_t>(vecs) * rank / S);
  const int v1 = static_cast<int>(static_cast<int64_t>(vecs) * (rank + 1) / S);
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
  const bool edge = rank == 0 && tid < head + rest;
  const int edge_at = tid < head ? tid : a.V - rest + (tid - head);

  // ---- one pass
  LpSums s = {-INFINITY, 0.f, 0.f};
  int best_v = -1;  // the first vector that holds this thread's maximum; -1: the edge element
  if (edge) {
    const float e = Vec::one(x + edge_at);
    s.m = fmaxf(e, -INFINITY);  // (NaN: its sums will say so)
    const float d = (e - (s.m == -INFINITY ? 0.f : s.m)) * a.c;
    s.z = lp_ex2(d);
    s.w = s.z * fmaxf(d, -1000.f);
  }
  auto take = [&](const uint4& u, int v) {
    float y[N];
    Vec::split(u, y);
    float most = y[0];
#pragma unroll
    for (int j = 1; j < N; ++j) most = fmaxf(most, y[j]);
    if (most > s.m) {
      lp_raise(s, most, a.c);
      best_v = v;
    }
    const float ref = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float d = (y[j] - ref) * a.c, e = lp_ex2(d);
      s.z += e;
      s.w = fmaf(e, fmaxf(d, -1000.f), s.w);
    }
  };
  int v = v0 + tid;
  for (; v + (AHEAD - 1) * LP_THREADS < v1; v += AHEAD * LP_THREADS) {
    uint4 u[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) u[i] = __ldg(xv + v + i * LP_THREADS);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) take(u[i], v + i * LP_THREADS);
  }
  for (; v < v1; v += LP_THREADS) take(__ldg(xv + v), v);
  const bool any = edge || v0 + tid < v1;
  const float mine = s.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    LpSums b = {__shfl_down_sync(0xffffffffu, s.m, o), __shfl_down_sync(0xffffffffu, s.z, o),
                __shfl_down_sync(0xffffffffu, s.w, o)};
    lp_join(s, b, a.c);
  }
  if (lane == 0) warp_sums[warp] = s;

  // ---- the best
  if (a.n > 0) {
    // an element of this thread that holds its maximum
    uint64_t k = 0;
    auto scan = [&](auto f) {  // f(value, index) over this thread's elements
      if (edge) f(Vec::one(x + edge_at), edge_at);
      for (int i = v0 + tid; i < v1; i += LP_THREADS) {
        float y[N];
        Vec::split(__ldg(xv + i), y);
#pragma unroll
        for (int j = 0; j < N; ++j) f(y[j], head + i * N + j);
      }
    };
    // no element of this thread has a larger key than the value's with index 0
    const uint64_t reach = any ? lp_key(mine, 0) : 0;
    if (any) {
      if (best_v >= 0) {
        float y[N];
        Vec::split(__ldg(xv + best_v), y);
#pragma unroll
        for (int j = N - 1; j >= 0; --j)
          if (y[j] == mine) k = lp_key(y[j], head + best_v * N + j);
      } else if (edge) {
        k = lp_key(mine, edge_at);
      } else {
        k = lp_key(-INFINITY, head + (v0 + tid) * N);
      }
    }
    // the warp's 32 in order, best first
    uint64_t t = k;
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
      for (int o = size >> 1; o > 0; o >>= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, t, o);
        const bool down = (lane & size) == 0 || size == 32, first = (lane & o) == 0;
        t = (down == first) == (t > other) ? t : other;
      }
    lists[warp][lane] = t;
    if (tid == 0) {
      from_key = 1;  // fewer than n elements: all of them
      collected = 0;
    }
    __syncthreads();
    if (lane < a.n && t != 0) {
      int above = lane;
#pragma unroll
      for (int w = 0; w < LP_WARPS; ++w) {
        if (w == warp) continue;
        int lo = 0;  // how many of that list are larger
#pragma unroll
        for (int b = 16; b > 0; b >>= 1) lo += lists[w][lo + b - 1] > t ? b : 0;
        above += lo + (lists[w][lo] > t);
      }
      if (above == a.n - 1) from_key = t;
    }
    __syncthreads();
    const uint64_t from = from_key;
    if (reach >= from)
      scan([&](float y, int i) {
        const uint64_t e = lp_key(y, i);
        if (e >= from) {
          const int at = atomicAdd(&collected, 1);
          if (at < LP_ROOM) keys[at] = e;
        }
      });
    __syncthreads();
    if (collected <= LP_ROOM) {
      lp_best(keys, collected, a.n, best);
    } else {
      if (tid == 0) from_key = ~0ull;
      __syncthreads();
      for (int i = 0; i < a.n; ++i) {
        const uint64_t under = from_key;
        uint64_t e = 0;
        if (reach >= from)
          scan([&](float y, int j) {
            const uint64_t q = lp_key(y, j);
            if (q < under && q > e) e = q;
          });
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const uint64_t other = __shfl_down_sync(0xffffffffu, e, o);
          e = other > e ? other : e;
        }
        __syncthreads();  // from_key has been read
        if (lane == 0) lists[0][warp] = e;
        __syncthreads();
        if (tid == 0) {
          for (int w = 1; w < LP_WARPS; ++w) e = lists[0][w] > e ? lists[0][w] : e;
          best[i] = from_key = e;
        }
        __syncthreads();
      }
    }
  }
  __syncthreads();

  // ---- the block's sums, and the cluster's
  if (warp == 0) {
    s = lane < LP_WARPS ? warp_sums[lane] : LpSums{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int o = LP_WARPS / 2; o > 0; o >>= 1) {
      LpSums b = {__shfl_down_sync(0xffffffffu, s.m, o), __shfl_down_sync(0xffffffffu, s.z, o),
                  __shfl_down_sync(0xffffffffu, s.w, o)};
      lp_join(s, b, a.c);
    }
  }
  if (S > 1) {
    lp_cluster_wait();  // every block of the cluster is running
    if (tid == 0) {
      lp_store_leader(lp_at_leader(smem_u32(&rank_mz[rank])),
                      static_cast<uint64_t>(__float_as_uint(s.m)) << 32 | __float_as_uint(s.z));
      lp_store_leader(lp_at_leader(smem_u32(&rank_w[rank])), __float_as_uint(s.w));
    }
    if (tid < a.n) lp_store_leader(lp_at_leader(smem_u32(&from_ranks[rank * a.n + tid])), best[tid]);
    __syncwarp();
    lp_cluster_arrive();
    if (rank != 0) {
      lp_cluster_wait();
      return;
    }
    lp_cluster_wait();
    if (a.n > 0) lp_best(from_ranks, S * a.n, a.n, best);
    if (warp == 0) {
      s = LpSums{-INFINITY, 0.f, 0.f};
      if (lane < S) {
        const uint64_t mz = rank_mz[lane];
        s = LpSums{__uint_as_float(static_cast<uint32_t>(mz >> 32)), __uint_as_float(static_cast<uint32_t>(mz)),
                   __uint_as_float(static_cast<uint32_t>(rank_w[lane]))};
      }
#pragma unroll
      for (int o = LP_CLUSTER / 2; o > 0; o >>= 1) {
        LpSums b = {__shfl_down_sync(0xffffffffu, s.m, o), __shfl_down_sync(0xffffffffu, s.z, o),
                    __shfl_down_sync(0xffffffffu, s.w, o)};
        lp_join(s, b, a.c);
      }
    }
  }
  if (warp == 0) {
    s.m = __shfl_sync(0xffffffffu, s.m, 0);
    s.z = __shfl_sync(0xffffffffu, s.z, 0);
    s.w = __shfl_sync(0xffffffffu, s.w, 0);
    const float lnz = logf(s.z);
    // no probability anywhere (all logits minus infinity): -inf, and an entropy of 0
    auto logprob = [&](float y) { return s.z == 0.f ? -INFINITY : (y - s.m) * a.scale - lnz; };
    if (lane == 0) {
      if (a.logprob != nullptr) a.logprob[row] = logprob(Vec::one(x + token));
      if (a.entropy != nullptr) a.entropy[row] = s.z == 0.f ? 0.f : lnz - LP_LN2 * (s.w / s.z);
    }
    if (lane < a.n) {
      const uint64_t k = best[lane];
      if (a.top_id != nullptr) a.top_id[row * a.n + lane] = static_cast<int32_t>(lp_key_index(k));
      if (a.top_logprob != nullptr) a.top_logprob[row * a.n + lane] = logprob(lp_key_value(k));
    }
  }
}

}  // namespace decomoe

using namespace decomoe;

extern "C" int decomoe_token_logprobs(const void* logits, int64_t T, int64_t V, int64_t row_stride, int dtype,
                                      const int32_t* tokens, float scale, int n, float* logprob, float* entropy,
                                      int32_t* top_id, float* top_logprob, int32_t* status_dev, decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(dtype == DECOMOE_BF16 || dtype == DECOMOE_F32, "token_logprobs: logits must be bf16 or f32");
  DM_ARG_CHECK(T >= 0 && T <= INT_MAX / LP_CLUSTER, "token_logprobs: bad number of rows");
  DM_ARG_CHECK(V >= 1 && V <= (1 << 24), "token_logprobs: a vocabulary of 1 to 2^24 expected");
  DM_ARG_CHECK(row_stride >= V, "token_logprobs: row stride below the vocabulary's size");
  DM_ARG_CHECK(scale > 0.f && scale <= FLT_MAX, "token_logprobs: scale must be positive and finite");
  DM_ARG_CHECK(n >= 0 && n <= LP_BEST && n <= V, "token_logprobs: 0 to %d alternatives, at most the vocabulary's size", LP_BEST);
  DM_ARG_CHECK(n > 0 || (top_id == nullptr && top_logprob == nullptr), "token_logprobs: alternatives without a number of them");
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
  a.n = top_id != nullptr || top_logprob != nullptr ? n : 0;
  a.scale = scale;
  a.c = scale * 1.4426950408889634f;
  // blocks for every SM, and a slice of at least a vector per thread
  int S = 1;
  while (S < LP_CLUSTER && T * S < 2 * sm_count() && V * static_cast<int64_t>(e) > 16 * LP_THREADS * S) S *= 2;
  auto go = [&](auto kern) -> int {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(T * S));
    cfg.blockDim = dim3(LP_THREADS);
    cfg.stream = reinterpret_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = pdl_enabled(T * S) ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(S);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = S > 1 ? 2 : 1;
    if (S > 8) DM_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    DM_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kern, a, S));
    return DECOMOE_OK;
  };
  return dtype == DECOMOE_BF16 ? go(k_token_logprobs<__nv_bfloat16>) : go(k_token_logprobs<float>);
}
