// tables.cu -- pifa_page_tables: block tables, slot map and positions of one step, from the requests' lengths.
//
//   have_b = ceil(cached_b / P), want_b = ceil((cached_b + new_b) / P), off_b = sum_{a < b} (want_a - have_a)
//   table[b][have_b + i] = free[first + off_b + i]
//   token t of request b: pos = cached_b + t - q_start[b], slot = table[b][pos / P] P + pos mod P
//
// The work is two prefix sums over the requests and one short record per token and per new page: some
// kilobytes, so that latencies are all there is to it. One launch: a cluster of 1 to 8 CTAs; each scans all
// lengths into its own shared memory (a second launch, or a scan split over CTAs, would cost more than the
// repeated reads, which hit L2), then takes its share of tokens and new pages, finding their requests by
// bisection. A token on a new page takes the page from the free list itself, so no token waits for the table.
// Measured: 64 requests in decode 4.5 us; 520 requests with 8087 new tokens 8.7 us, where two CTAs' threads take four
// tokens one after another, each a bisection, divisions by the page size (64-bit ones in part) and dependent loads.
// The cluster's barrier between the scan and the writes lets a serving loop update lengths and the free
// list's head in place.
#include "pifa.h"
#include "pifa_internal.h"
#include "ptx.cuh"

namespace {

using namespace pifa;

constexpr int THREADS = 1024;
constexpr int64_t MAX_B = 4096;
constexpr int MAX_CTAS = 8;

struct TableArgs {
  const int32_t *cached, *fresh, *free_pages, *free_first;
  int32_t *table, *q_start, *kv_len, *positions, *free_next;
  int64_t* slots;
  int64_t ldt;
  int B, P, n_free, cols, T;
  int* status;
};

// Inclusive sums of a and b over the CTA's threads; `part` holds one pair per warp.
__device__ __forceinline__ void block_scan(int64_t& a, int64_t& b, int64_t (*part)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) {
      a += x;
      b += y;
    }
  }
  if (lane == 31) {
    part[warp][0] = a;
    part[warp][1] = b;
  }
  __syncthreads();
  if (warp == 0) {
    int64_t x = part[lane][0], y = part[lane][1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) {
        x += u;
        y += v;
      }
    }
    part[lane][0] = x;
    part[lane][1] = y;
  }
  __syncthreads();
  if (warp > 0) {
    a += part[warp - 1][0];
    b += part[warp - 1][1];
  }
}

// The last index i in [0, n) with first[i] <= v (first is ascending, first[0] = 0 <= v).
__device__ __forceinline__ int find(const int32_t* first, int n, int v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(THREADS, 1) page_tables(const TableArgs g) {
  extern __shared__ int32_t smem[];
  __shared__ int64_t part[32][2];
  __shared__ int64_t carry[2];
  int32_t* q_off = smem;               // B + 1: first new token of each request, at most T
  int32_t* p_off = smem + g.B + 1;     // B + 1: first new page of each request
  int32_t* cached = smem + 2 * g.B + 2;
  const int tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait_primary();
  const int first = *g.free_first;
  const int lim = 0x7fffffff;
  bool negative = first < 0, over = false;
  // Where the new tokens are more than T, those past it are no part of the step: a second round counts the pages of
  // the ones before.
  for (bool cut = false;; cut = true) {
    if (tid == 0) carry[0] = carry[1] = 0;
    for (int b0 = 0; b0 < g.B; b0 += THREADS) {
      const int b = b0 + tid;
      int c = 0, n = 0;
      if (b < g.B) {
        c = g.cached[b];
        n = g.fresh[b];
        negative |= c < 0 || n < 0;
        c = max(c, 0);
        n = max(n, 0);
        if (n > lim - c) {
          n = lim - c;
          over = true;
        }
        if (cut) n = q_off[b + 1] - q_off[b];
        cached[b] = c;
      }
      const int pages = (int)(((int64_t)c + n + g.P - 1) / g.P - ((int64_t)c + g.P - 1) / g.P);
      int64_t a = n, p = pages;
      __syncthreads();  // the last round's carry and partial sums have been read
      block_scan(a, p, part);
      const int64_t ca = carry[0], cp = carry[1];
      if (b < g.B) {
        q_off[b] = (int)min(ca + a - n, (int64_t)g.T);
        p_off[b] = (int)min(cp + p - pages, (int64_t)lim);
      }
      __syncthreads();
      if (tid == THREADS - 1) {
        carry[0] = ca + a;
        carry[1] = cp + p;
      }
    }
    __syncthreads();
    const bool fits = carry[0] <= g.T;
    if (tid == 0) {
      q_off[g.B] = (int)min(carry[0], (int64_t)g.T);
      p_off[g.B] = (int)min(carry[1], (int64_t)lim);
    }
    over |= carry[1] > (int64_t)g.n_free - max(first, 0);
    if (fits) break;
    over = true;
    __syncthreads();
  }
  cluster_sync_all();  // every CTA has read the lengths and the free list's head

  const int me = (int)blockIdx.x * THREADS + tid, step = (int)gridDim.x * THREADS;
  const int head = max(first, 0);
  for (int t = me; t < g.T; t += step) {
    int pos = 0;
    int64_t slot = -1;
    if (t < q_off[g.B]) {
      const int b = find(q_off, g.B, t);
      const int c = cached[b], have = (int)(((int64_t)c + g.P - 1) / g.P);
      pos = c + (t - q_off[b]);
      const int p = pos / g.P;
      int page = -1;
      if (p >= g.cols) {
        over = true;
      } else if (p < have) {
        page = g.table[b * g.ldt + p];
      } else {
        const int64_t e = (int64_t)head + p_off[b] + (p - have);
        if (e < g.n_free) page = g.free_pages[e];
      }
      if (page >= 0) slot = (int64_t)page * g.P + (pos - p * g.P);
    }
    g.positions[t] = pos;
    g.slots[t] = slot;
  }
  const int n_new = (int)min((int64_t)p_off[g.B], max((int64_t)g.n_free - head, (int64_t)0));
  for (int e = me; e < n_new; e += step) {
    const int b = find(p_off, g.B, e);
    const int64_t p = ((int64_t)cached[b] + g.P - 1) / g.P + (e - p_off[b]);
    if (p < g.cols) g.table[b * g.ldt + p] = g.free_pages[(int64_t)head + e];
    else over = true;
  }
  for (int b = me; b <= g.B; b += step) {
    g.q_start[b] = q_off[b];
    if (b < g.B) g.kv_len[b] = cached[b] + (q_off[b + 1] - q_off[b]);
  }
  if (me == 0) *g.free_next = (int)min((int64_t)head + p_off[g.B], (int64_t)max(g.n_free, head));
  if (negative) latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
  if (over) latch_status(g.status, PIFA_ERR_CAPACITY);
}

}  // namespace

extern "C" int pifa_page_tables(const int32_t* cached_len, const int32_t* new_len, int64_t B, int64_t page_size,
                                const int32_t* free_pages, int64_t n_free, const int32_t* free_first, int32_t* table,
                                int64_t cols, int64_t ldt, int32_t* q_start, int32_t* kv_len, int32_t* positions,
                                int64_t* slots, int64_t T, int32_t* free_next, void* cuda_stream) {
  pifa_clear_error();
  const int64_t lim = (int64_t)1 << 30;
  if (B < 0 || T < 0 || B >= lim || T >= lim) return pifa_fail(PIFA_ERR_INVALID_ARG, "B and T must be in [0, 2^30)");
  if (B > MAX_B) return pifa_fail(PIFA_ERR_UNSUPPORTED, "page tables take at most 4096 requests");
  if (page_size < 1 || page_size > 65536) return pifa_fail(PIFA_ERR_INVALID_ARG, "page_size must be in [1, 65536]");
  if (cols < 0 || cols >= lim || ldt < cols || n_free < 0 || n_free >= lim)
    return pifa_fail(PIFA_ERR_INVALID_ARG, "cols, ldt or n_free out of range");
  if (B == 0) return PIFA_OK;
  if (!cached_len || !new_len || !free_first || !q_start || !kv_len || !free_next || (n_free && !free_pages) ||
      (cols && !table) || (T && (!positions || !slots)))
    return pifa_fail(PIFA_ERR_INVALID_ARG, "null argument");
  const PifaSpan out[] = {pifa_span(table, B, cols, ldt, 4), pifa_span(q_start, 1, B + 1, B + 1, 4),
                          pifa_span(kv_len, 1, B, B, 4), pifa_span(positions, 1, T, T, 4),
                          pifa_span(slots, 1, T, T, 8), pifa_span(free_next, 1, 1, 1, 4)};
  const PifaSpan in[] = {pifa_span(cached_len, 1, B, B, 4), pifa_span(new_len, 1, B, B, 4),
                         pifa_span(free_pages, 1, n_free, n_free, 4), pifa_span(free_first, 1, 1, 1, 4)};
  for (int i = 0; i < 6; ++i) {
    for (int j = 0; j < i; ++j)
      if (pifa_spans_overlap(out[i], out[j])) return pifa_fail(PIFA_ERR_INVALID_ARG, "two outputs overlap");
    for (int j = 0; j < 4; ++j) {
      if ((i == 2 && j == 0 && kv_len == cached_len) || (i == 5 && j == 3 && free_next == free_first)) continue;
      if (pifa_spans_overlap(out[i], in[j])) return pifa_fail(PIFA_ERR_INVALID_ARG, "an output overlaps an input");
    }
  }
  cudaError_t e = cudaSuccess;
  int* status = pifa_status_word(&e);
  if (!status) return pifa_fail_cuda("device status word", e);
  const TableArgs g = {cached_len, new_len, free_pages, free_first, table, q_start, kv_len, positions, free_next, slots,
                       ldt, (int)B, (int)page_size, (int)n_free, (int)cols, (int)T, status};
  const size_t bytes = (size_t)(3 * B + 2) * 4;
  if ((e = pifa_allow_smem<page_tables>((int)((3 * MAX_B + 2) * 4))) != cudaSuccess)
    return pifa_fail_cuda("cudaFuncSetAttribute(page_tables)", e);
  unsigned ctas = 1;  // four tokens a thread before another CTA joins
  while (ctas < MAX_CTAS && (int64_t)ctas * THREADS * 4 < T) ctas *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = pifa_launch_ex(&cfg, page_tables, g);
  if (e != cudaSuccess) return pifa_fail_cuda("page_tables launch", e);
  return PIFA_OK;
}
