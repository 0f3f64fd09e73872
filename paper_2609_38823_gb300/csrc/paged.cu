// A paged key-value cache (decoding on the text-only cache, DecoMoE Section
// 3.2 and Algorithm 2, last step, for a batch of requests): the block tables,
// slots and positions of a step's rows from the requests' lengths, and the
// store of the rows into their slots.
#include "decomoe_internal.cuh"

namespace decomoe {

// ------------------------------------------------------------------ plan
// Two running sums over the requests decide everything: rows (sum of fresh) and
// pages (sum of need - have). Every block adds up both for all B requests in
// its shared memory (a few loads per thread, whatever the grid), then takes its
// share of the rows and of the new pages, finding an item's request by binary
// search in the sums. No block waits for another: a row on a new page reads the
// page from the free list, not from the table entry that another block writes.
constexpr int PLAN_THREADS = 256;

struct PlanArgs {
  const int32_t *cached, *fresh, *free_pages, *free_head;
  int32_t *free_head_out, *table, *seq_len, *row_start, *slot_map, *positions, *status;
  int64_t n_free, max_pages, N;
  int B, shift;  // page size 1 << shift
  bool by_request;  // one row at most of each request, and row b is request b's
};

// Exclusive sums of the block's values in thread order, and their totals.
__device__ __forceinline__ void block_scan2(int64_t& a, int64_t& b, int64_t& ta, int64_t& tb) {
  __shared__ int64_t wa[PLAN_THREADS / 32], wb[PLAN_THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t ia = a, ib = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t ua = __shfl_up_sync(0xffffffffu, ia, o), ub = __shfl_up_sync(0xffffffffu, ib, o);
    if (lane >= o) {
      ia += ua;
      ib += ub;
    }
  }
  if (lane == 31) {
    wa[warp] = ia;
    wb[warp] = ib;
  }
  __syncthreads();
  int64_t ba = 0, bb = 0;
  ta = tb = 0;
#pragma unroll
  for (int w = 0; w < PLAN_THREADS / 32; ++w) {
    if (w < warp) {
      ba += wa[w];
      bb += wb[w];
    }
    ta += wa[w];
    tb += wb[w];
  }
  a = ba + ia - a;
  b = bb + ib - b;
}

// The last request whose start is at most v (starts ascend, starts[0] = 0): the
// one that holds item v, since the empty ones before it start where it does.
__device__ __forceinline__ int find_request(const int32_t* starts, int B, int32_t v) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(PLAN_THREADS) k_paged_plan(PlanArgs a) {
  extern __shared__ int32_t plan_smem[];
  int32_t* rows = plan_smem;           // [B + 1] first row of a request
  int32_t* pages = rows + a.B + 1;     // [B + 1] first of its new pages
  int32_t* held = pages + a.B + 1;     // [B] rows it has in the cache
  pdl_enter();
  const int t = threadIdx.x;
  const int64_t cap = a.max_pages << a.shift;
  const int64_t ps1 = (int64_t{1} << a.shift) - 1;
  const int64_t head = a.free_head != nullptr ? static_cast<int64_t>(*a.free_head) : 0;
  const int per = (a.B + PLAN_THREADS - 1) / PLAN_THREADS;
  const int b0 = min(a.B, t * per), b1 = min(a.B, b0 + per);
  const bool lead = blockIdx.x == 0;
  bool bad = false;
  int64_t nr = 0, np = 0;
  for (int b = b0; b < b1; ++b) {
    const int64_t c = a.cached[b], given = a.fresh[b], f = a.by_request ? min(given, int64_t{1}) : given;
    const int64_t cc = min(max(c, int64_t{0}), cap), end = min(cc + max(f, int64_t{0}), cap);
    bad |= c < 0 || f < 0 || f < given || c > cap || cc + f > cap;
    if (lead) a.seq_len[b] = static_cast<int32_t>(end);
    held[b] = static_cast<int32_t>(cc);
    // the rows of a request that the table is too narrow for are rows all the same
    rows[b] = static_cast<int32_t>(min(max(f, int64_t{0}), int64_t{INT_MAX}));
    pages[b] = static_cast<int32_t>(((end + ps1) >> a.shift) - ((cc + ps1) >> a.shift));
    nr += rows[b];
    np += pages[b];
  }
  int64_t tr, tp;
  block_scan2(nr, np, tr, tp);
  for (int b = b0; b < b1; ++b) {
    const int32_t r = rows[b], p = pages[b];
    rows[b] = static_cast<int32_t>(min(nr, int64_t{INT_MAX}));
    pages[b] = static_cast<int32_t>(min(np, int64_t{INT_MAX}));
    if (lead && !a.by_request) a.row_start[b] = rows[b];
    nr += r;
    np += p;
  }
  const int64_t all_rows = min(tr, int64_t{INT_MAX}), all_pages = min(tp, int64_t{INT_MAX});
  if (t == 0) {
    rows[a.B] = static_cast<int32_t>(all_rows);
    pages[a.B] = static_cast<int32_t>(all_pages);
    if (lead) {
      if (!a.by_request) a.row_start[a.B] = rows[a.B];
      if (a.free_head_out != nullptr)
        *a.free_head_out = static_cast<int32_t>(min(head + all_pages, max(a.n_free, head)));
      bad |= tr > a.N || head < 0 || head + tp > a.n_free;
    }
  }
  __syncthreads();
  // the page that entry i of request b's new pages gets; -1: the list has run out
  auto page_of = [&](int64_t i) -> int32_t {
    const int64_t at = head + i;
    return head >= 0 && at < a.n_free ? a.free_pages[at] : -1;
  };
  const int64_t first = static_cast<int64_t>(blockIdx.x) * PLAN_THREADS + t;
  const int64_t step = static_cast<int64_t>(gridDim.x) * PLAN_THREADS;
  for (int64_t i = first; i < all_pages; i += step) {
    const int b = find_request(pages, a.B, static_cast<int32_t>(i));
    const int64_t have = (held[b] + ps1) >> a.shift;
    a.table[b * a.max_pages + have + (i - pages[b])] = page_of(i);
  }
  for (int64_t r = first; r < a.N; r += step) {
    int32_t slot = -1, pos = -1;
    if (a.by_request ? rows[r] < rows[r + 1] : r < all_rows) {
      const int b = a.by_request ? static_cast<int>(r) : find_request(rows, a.B, static_cast<int32_t>(r));
      const int64_t p = held[b] + (a.by_request ? 0 : r - rows[b]);
      if (p < cap) {
        const int64_t have = (held[b] + ps1) >> a.shift, e = p >> a.shift;
        const int32_t page = e < have ? a.table[b * a.max_pages + e] : page_of(pages[b] + (e - have));
        const int64_t s = (static_cast<int64_t>(page) << a.shift) + (p & ps1);
        pos = static_cast<int32_t>(p);
        if (page >= 0 && s <= INT_MAX) slot = static_cast<int32_t>(s);
      }
      bad |= slot < 0;
    }
    a.slot_map[r] = slot;
    if (a.positions != nullptr) a.positions[r] = pos;
  }
  if (bad) report_status(a.status, DECOMOE_ERR_BAD_INPUT);
}

// ------------------------------------------------------------------ advance
// A request's rows after the step: a warp per request looks through the pages that the
// step asked for, 32 entries at a time, for the first one that it did not get.
__global__ void __launch_bounds__(256)
    k_paged_advance(int32_t* cached, const int32_t* seq_len, const int32_t* table, int B, int64_t max_pages, int shift,
                    int32_t* free_head, const int32_t* free_head_out) {
  pdl_enter();
  const int b = (blockIdx.x * blockDim.x + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0 && threadIdx.x == 0 && free_head != nullptr) *free_head = *free_head_out;
  if (b >= B) return;
  const int64_t ps1 = (int64_t{1} << shift) - 1;
  const int64_t n = min(max(static_cast<int64_t>(seq_len[b]), int64_t{0}), max_pages << shift);
  const int64_t have = (max(static_cast<int64_t>(cached[b]), int64_t{0}) + ps1) >> shift, need = (n + ps1) >> shift;
  int64_t end = n;
  for (int64_t e = have; e < need; e += 32) {
    const unsigned gone = __ballot_sync(0xffffffffu, e + lane < need && table[b * max_pages + e + lane] < 0);
    if (gone != 0) {
      end = min(end, (e + __ffs(gone) - 1) << shift);
      break;
    }
  }
  __syncwarp();
  if (lane == 0) cached[b] = static_cast<int32_t>(end);
}

// ------------------------------------------------------------------ append
// A plain scatter, bound by bandwidth where there are many rows and by one round trip
// where there are few. 1 << LANES threads take a row of keys and the same of values,
// with up to eight 16-byte loads of each thread in flight. 16384 rows of 1 KB twice: 12.0
// us, 5.6 TB/s read and written; a thread per 16 bytes that divides to find its row 14.2.
constexpr int APPEND_VECS = 4;  // of a thread and pool in flight
__global__ void __launch_bounds__(256)
    k_paged_append(const uint4* __restrict__ kn, int64_t ks, const uint4* __restrict__ vn, int64_t vs, int64_t N,
                   int vec, int lanes, const int32_t* __restrict__ slot_map, uint4* __restrict__ kp,
                   uint4* __restrict__ vp, int64_t slots, int shift, int64_t page_vecs, int32_t* status) {
  pdl_wait();
  const int64_t r = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) >> lanes;
  const int c0 = threadIdx.x & ((1 << lanes) - 1), step = 1 << lanes;
  if (r < N) {
    const int64_t s = slot_map[r];
    if (s >= 0 && s < slots) {
      const uint4 *k = kn + r * ks, *v = vn + r * vs;
      const int64_t at = (s >> shift) * page_vecs + (s & ((int64_t{1} << shift) - 1)) * vec;
      for (int c = c0; c < vec; c += APPEND_VECS * step) {
        uint4 a[APPEND_VECS], b[APPEND_VECS];
#pragma unroll
        for (int i = 0; i < APPEND_VECS; ++i)
          if (c + i * step < vec) {
            a[i] = k[c + i * step];
            b[i] = v[c + i * step];
          }
#pragma unroll
        for (int i = 0; i < APPEND_VECS; ++i)
          if (c + i * step < vec) {
            kp[at + c + i * step] = a[i];
            vp[at + c + i * step] = b[i];
          }
      }
    } else if (s != -1 && c0 == 0) {
      report_status(status, DECOMOE_ERR_BAD_INPUT);
    }
  }
  pdl_trigger();
}

static int plan_call(const char* name, bool by_request, const int32_t* cached, const int32_t* fresh, int64_t B,
                     int page_size, const int32_t* free_pages, int64_t n_free, const int32_t* free_head,
                     int32_t* free_head_out, int32_t* block_table, int64_t max_pages, int32_t* seq_len,
                     int32_t* row_start, int32_t* slot_map, int32_t* positions, int64_t N, int32_t* status_dev,
                     decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(B >= 0 && B <= DECOMOE_MAX_REQUESTS, "%s: B must lie in [0, %d]", name, DECOMOE_MAX_REQUESTS);
  DM_ARG_CHECK(page_size >= 1 && (page_size & (page_size - 1)) == 0, "%s: page_size must be a power of two", name);
  DM_ARG_CHECK(N >= 0 && N <= INT_MAX && n_free >= 0 && n_free <= INT_MAX, "%s: bad N or n_free", name);
  DM_ARG_CHECK(max_pages >= 0 && max_pages <= INT_MAX / page_size, "%s: max_pages * page_size must be in [0, 2^31)", name);
  DM_ARG_CHECK((by_request || row_start != nullptr) && (N == 0 || slot_map != nullptr) && (n_free == 0 || free_pages != nullptr),
               "%s: null pointer", name);
  DM_ARG_CHECK(B == 0 || (cached && fresh && seq_len && (block_table || max_pages == 0)), "%s: null pointer", name);
  const size_t one = sizeof(int32_t), each = static_cast<size_t>(B) * one;
  const Bytes in[] = {{cached, each}, {fresh, each}, {free_pages, static_cast<size_t>(n_free) * one}, {free_head, one}};
  const Bytes out[] = {{block_table, each * static_cast<size_t>(max_pages)}, {seq_len, each}, {row_start, each + one},
                       {slot_map, static_cast<size_t>(N) * one}, {positions, static_cast<size_t>(N) * one},
                       {free_head_out, one}};
  for (size_t i = 0; i < sizeof(out) / sizeof(out[0]); ++i) {
    bool apart = !overlaps(out[i], {in[0], in[1], in[2], in[3]});
    for (size_t j = 0; j < i; ++j) apart &= !overlaps(out[i], {out[j]});
    DM_ARG_CHECK(apart, "%s: an output overlaps an input or another output", name);
  }
  PlanArgs a = {};
  a.cached = cached;
  a.fresh = fresh;
  a.free_pages = free_pages;
  a.free_head = free_head;
  a.free_head_out = free_head_out;
  a.table = block_table;
  a.seq_len = seq_len;
  a.row_start = row_start;
  a.slot_map = slot_map;
  a.positions = positions;
  a.status = status_dev;
  a.n_free = n_free;
  a.max_pages = max_pages;
  a.N = N;
  a.B = static_cast<int>(B);
  a.shift = __builtin_ctz(static_cast<unsigned>(page_size));
  a.by_request = by_request;
  const int64_t items = std::max<int64_t>(N, 1);
  const int grid = static_cast<int>(std::min<int64_t>(sm_count(), (items + PLAN_THREADS - 1) / PLAN_THREADS));
  const size_t smem = (3 * static_cast<size_t>(B) + 2) * sizeof(int32_t);
  if (smem > 48 * 1024)
    DM_CUDA_CHECK(cudaFuncSetAttribute(k_paged_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
  DM_CUDA_CHECK(launch_pdl(k_paged_plan, dim3(grid), dim3(PLAN_THREADS), smem, reinterpret_cast<cudaStream_t>(stream), a));
  return DECOMOE_OK;
}

}  // namespace decomoe

using namespace decomoe;

extern "C" {

int decomoe_paged_plan(const int32_t* cached, const int32_t* fresh, int64_t B, int page_size,
                       const int32_t* free_pages, int64_t n_free, const int32_t* free_head, int32_t* free_head_out,
                       int32_t* block_table, int64_t max_pages, int32_t* seq_len, int32_t* row_start,
                       int32_t* slot_map, int32_t* positions, int64_t N, int32_t* status_dev,
                       decomoe_stream_t stream) {
  return plan_call("paged_plan", false, cached, fresh, B, page_size, free_pages, n_free, free_head, free_head_out,
                   block_table, max_pages, seq_len, row_start, slot_map, positions, N, status_dev, stream);
}

int decomoe_paged_plan_step(const int32_t* cached, const int32_t* fresh, int64_t B, int page_size,
                            const int32_t* free_pages, int64_t n_free, const int32_t* free_head,
                            int32_t* free_head_out, int32_t* block_table, int64_t max_pages, int32_t* seq_len,
                            int32_t* slot_map, int32_t* positions, int32_t* status_dev, decomoe_stream_t stream) {
  return plan_call("paged_plan_step", true, cached, fresh, B, page_size, free_pages, n_free, free_head, free_head_out,
                   block_table, max_pages, seq_len, nullptr, slot_map, positions, B, status_dev, stream);
}

int decomoe_paged_advance(int32_t* cached, const int32_t* seq_len, const int32_t* block_table, int64_t B,
                          int64_t max_pages, int page_size, int32_t* free_head, const int32_t* free_head_out,
                          decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(B >= 0 && B <= DECOMOE_MAX_REQUESTS, "paged_advance: B must lie in [0, %d]", DECOMOE_MAX_REQUESTS);
  DM_ARG_CHECK(page_size >= 1 && (page_size & (page_size - 1)) == 0, "paged_advance: page_size must be a power of two");
  DM_ARG_CHECK(max_pages >= 0 && max_pages <= INT_MAX / page_size,
               "paged_advance: max_pages * page_size must be in [0, 2^31)");
  DM_ARG_CHECK(B == 0 || (cached && seq_len && (block_table || max_pages == 0)), "paged_advance: null pointer");
  DM_ARG_CHECK((free_head == nullptr) == (free_head_out == nullptr), "paged_advance: free_head and free_head_out go together");
  const size_t each = static_cast<size_t>(B) * sizeof(int32_t);
  const Bytes lens = {seq_len, each}, table = {block_table, each * static_cast<size_t>(max_pages)};
  DM_ARG_CHECK(!overlaps({cached, each}, {lens, table}) &&
                   !overlaps({free_head, sizeof(int32_t)}, {{cached, each}, lens, table}),
               "paged_advance: cached or free_head overlaps another array");
  const int grid = static_cast<int>(std::max<int64_t>(1, (B * 32 + 255) / 256));
  DM_CUDA_CHECK(launch_pdl(k_paged_advance, dim3(grid), dim3(256), 0, reinterpret_cast<cudaStream_t>(stream), cached,
                           seq_len, block_table, static_cast<int>(B), max_pages,
                           __builtin_ctz(static_cast<unsigned>(page_size)), free_head, free_head_out));
  return DECOMOE_OK;
}

int decomoe_paged_append(const void* k_new, int64_t k_row_stride, const void* v_new, int64_t v_row_stride, int64_t N,
                         int width, int dtype, const int32_t* slot_map, void* k_pages, void* v_pages,
                         int64_t num_pages, int page_size, int64_t page_stride, int32_t* status_dev,
                         decomoe_stream_t stream) {
  clear_error();
  DM_ARG_CHECK(dtype == DECOMOE_BF16 || dtype == DECOMOE_F32, "paged_append: bad dtype");
  DM_ARG_CHECK(N >= 0 && N <= INT_MAX && width > 0, "paged_append: bad sizes");
  DM_ARG_CHECK(page_size >= 1 && (page_size & (page_size - 1)) == 0, "paged_append: page_size must be a power of two");
  DM_ARG_CHECK(num_pages >= 0 && num_pages <= INT_MAX / page_size, "paged_append: num_pages * page_size must be below 2^31");
  DM_ARG_CHECK(page_stride >= static_cast<int64_t>(page_size) * width, "paged_append: page_stride below page_size * width");
  if (N == 0) return DECOMOE_OK;
  DM_ARG_CHECK(k_new && v_new && slot_map && k_pages && v_pages, "paged_append: null pointer");
  const int64_t e = static_cast<int64_t>(dtype_bytes(dtype));
  DM_ARG_CHECK(k_row_stride >= width && v_row_stride >= width, "paged_append: row stride below width");
  DM_ARG_CHECK(width * e % 16 == 0 && k_row_stride * e % 16 == 0 && v_row_stride * e % 16 == 0 &&
                   page_stride * e % 16 == 0 && aligned16(k_new) && aligned16(v_new) && aligned16(k_pages) &&
                   aligned16(v_pages),
               "paged_append: rows and strides must be 16-byte multiples, pointers 16-byte aligned");
  const int vec = static_cast<int>(width * e / 16);
  int lanes = 0;  // the least power of two that covers a row, at most a warp
  while (lanes < 5 && (1 << lanes) < vec) ++lanes;
  const int64_t grid = ((N << lanes) + 255) / 256;
  DM_CUDA_CHECK(launch_pdl_late(k_paged_append, dim3(static_cast<unsigned>(grid)), dim3(256), 0,
                                reinterpret_cast<cudaStream_t>(stream), static_cast<const uint4*>(k_new),
                                k_row_stride * e / 16, static_cast<const uint4*>(v_new), v_row_stride * e / 16, N, vec,
                                lanes, slot_map, static_cast<uint4*>(k_pages), static_cast<uint4*>(v_pages),
                                num_pages * page_size, __builtin_ctz(static_cast<unsigned>(page_size)),
                                page_stride * e / 16, status_dev));
  return DECOMOE_OK;
}

}  // extern "C"
