// attention_rows.cuh -- what the kernels for requests with few rows share (attention.cu, attention_q8.cu): their arguments, the
// dealing of steps to warps or CTAs, their launch.
#ifndef PIFA_ATTENTION_ROWS_CUH_
#define PIFA_ATTENTION_ROWS_CUH_

#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pifa.h"
#include "pifa_internal.h"
#include "ptx.cuh"
#include "steps.h"

namespace {

using namespace pifa;

constexpr int WARPS = 8;
constexpr int THREADS = 32 * WARPS;
constexpr int STEP = 16;             // keys
constexpr int MIN_STEPS = 4;         // of a warp: fewer cost more in partial sums than they save
constexpr int MAX_ROWS = 16;
constexpr int MAX_CTAS = 160;        // of the streaming kernel (one for each SM), which the workspace is sized for

struct RowArgs {
  const uint16_t *q, *k, *v;
  uint16_t* o;
  const int32_t *table, *q_start, *kv_len;
  int* sums;          // (of a cache in 16 bits) B + 1: first step of each request (times heads), then the steps of one worker (0: nothing is done)
  float* partial;     // for each worker, a warp or (8 bits) a CTA, two pieces of max_rows: O, m, l
  int64_t ldq, ldo, ldt, page_stride, token_stride, head_stride, pages;
  int T, heads, group, page_size, page_shift, cols, B, max_q, max_rows;
  float c;            // |scale| log2(e), with scale's sign in `flip`
  uint32_t flip;
  int* status;
};

struct Lengths {
  int q0, n, L;   // first row of Q, new tokens that are computed, keys
  int ahead;      // token i sees ahead + i keys
};
// Lengths of request b, kept within the buffers whatever the arrays hold.
__device__ __forceinline__ Lengths lengths_of(const RowArgs& g, int b) {
  Lengths x;
  x.q0 = min(max(g.q_start[b], 0), g.T);
  x.n = min(min(max(g.q_start[b + 1], x.q0), g.T) - x.q0, g.max_q);
  x.L = min(max(g.kv_len[b], 0), g.cols << g.page_shift);
  x.ahead = x.L - (max(g.q_start[b + 1], x.q0) - x.q0) + 1;
  return x;
}
// Steps of a request: those of its keys; a request with rows but no keys has one, to write zeros.
__device__ __forceinline__ int steps_of(const Lengths& x) { return x.n == 0 ? 0 : max((x.L + STEP - 1) / STEP, 1); }

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool F16>
__device__ __forceinline__ uint32_t pack(float a, float b) {
  if constexpr (F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}
template <bool F16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (F16) mma_m16n8k16_f16(d, a0, a1, a2, a3, b0, b1);
  else mma_m16n8k16_bf16(d, a0, a1, a2, a3, b0, b1);
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The last index i in [0, n) with first[i] <= v (ascending, first[0] = 0 <= v).
__device__ __forceinline__ int find(const int* first, int n, int v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The requests' first steps, into first[0, B], how many there are, and the share of each worker, at least `least` (all threads of
// the CTA); what `keep(b, lengths)` leaves in shared memory is there as well.
struct Run {
  int total, run;
};
template <class Keep>
__device__ __forceinline__ Run deal_steps(const RowArgs& g, int* first, int* part, int workers, int least, Keep keep) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int total = 0;
  bool over = false, falls = false;
  for (int b0 = 0; b0 < g.B; b0 += THREADS) {
    const int b = b0 + tid;
    int v = 0;
    if (b < g.B) {
      const Lengths x = lengths_of(g, b);
      over |= g.kv_len[b] > (g.cols << g.page_shift) || (int64_t)g.q_start[b + 1] - g.q_start[b] > x.n;
      falls |= g.q_start[b + 1] < g.q_start[b];
      v = steps_of(x) * g.heads;
      keep(b, x);
    }
    int a = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, a, o);
      if (lane >= o) a += x;
    }
    __syncthreads();
    if (lane == 31) part[warp] = a;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      before += w < warp ? part[w] : 0;
      all += part[w];
    }
    if (b < g.B) first[b] = total + before + a - v;
    total += all;
  }
  if (tid == 0) first[g.B] = total;
  // requests that overlap: which of them a row belongs to is not said, so nothing is done
  const bool overlap = __syncthreads_or(falls);
  if (overlap) total = 0;
  const int run = max((total - 1) / workers + 1, least);  // (total may be close to 2^31)
  if (blockIdx.x == 0) {
    if (tid == 0 && overlap) latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
    if (over) latch_status(g.status, PIFA_ERR_CAPACITY);
  }
  return {total, run};
}

// CTAs of the streaming kernel.
inline int rows_grid() {
  const int sms = pifa_sm_count();
  return sms < MAX_CTAS ? sms : MAX_CTAS;
}

// The launch of a kernel that begins before the one before it in the stream has ended.
template <auto Kernel, typename... A>
cudaError_t launch_rows(int64_t grid, size_t smem, cudaStream_t stream, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (smem > 0) {
    const cudaError_t e = pifa_allow_smem<Kernel>(223 * 1024);  // (the rest is static)
    if (e != cudaSuccess) return e;
  }
  return pifa_launch_ex(&cfg, Kernel, args...);
}
inline size_t first_bytes(const RowArgs& g) { return (size_t)(g.B + 1) * 4; }

inline int64_t sums_bytes(int64_t B) { return ((B + 2) * 4 + 255) / 256 * 256; }

// The arguments that both kinds of cache have.
inline RowArgs row_args(const PifaAttention& a, int* status) {
  RowArgs g = {};
  g.q = static_cast<const uint16_t*>(a.q);
  g.o = static_cast<uint16_t*>(a.o);
  g.table = a.table;
  g.q_start = a.q_start;
  g.kv_len = a.kv_len;
  g.sums = reinterpret_cast<int*>(a.ws);
  g.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(a.ws) + sums_bytes(a.B));
  g.ldq = a.ldq;
  g.ldo = a.ldo;
  g.ldt = a.ldt;
  g.page_stride = a.cache.page_stride;
  g.token_stride = a.cache.token_stride;
  g.head_stride = a.cache.head_stride;
  g.pages = a.cache.pages;
  g.T = (int)a.T;
  g.heads = (int)a.cache.heads;
  g.group = (int)(a.q_heads / a.cache.heads);
  g.page_size = (int)a.cache.page_size;
  while ((1 << g.page_shift) < g.page_size) ++g.page_shift;
  g.cols = (int)a.cols;
  g.B = (int)a.B;
  g.max_q = (int)a.max_q;
  g.max_rows = g.max_q * g.group;
  g.flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
  // equal weights for a scale of zero: the masked scores, -inf, still have to vanish
  g.c = a.scale_log2 == 0.0f ? 1e-30f : std::fabs(a.scale_log2);
  g.status = status;
  return g;
}

}  // namespace

#endif  // PIFA_ATTENTION_ROWS_CUH_
