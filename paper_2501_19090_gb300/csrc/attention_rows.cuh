// attention_rows.cuh -- what the kernels for requests with few rows share (attention.cu, attention_q8.cu): their arguments, the
// dealing of steps to warps, the join of heads that several warps worked on.
#ifndef PIFA_ATTENTION_ROWS_CUH_
#define PIFA_ATTENTION_ROWS_CUH_

#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pifa.h"
#include "pifa_internal.h"
#include "ptx.cuh"

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
  int* sums;          // B + 1: first step of each request (times heads), then the steps of one worker (0: nothing is done)
  float* partial;     // for each worker, a warp or a CTA, two of max_rows x (D + 2): O, m, l
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
// the CTA; CTA 0 writes them down for the join).
struct Run {
  int total, run;
};
__device__ __forceinline__ Run deal_steps(const RowArgs& g, int* first, int* part, int workers, int least) {
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
  const int run = max((total + workers - 1) / workers, least);
  if (blockIdx.x == 0) {
    for (int b = tid; b <= g.B; b += THREADS) g.sums[b] = first[b];
    if (tid == 0) {
      g.sums[g.B + 1] = overlap ? 0 : run;
      if (overlap) latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
    }
    if (over) latch_status(g.status, PIFA_ERR_CAPACITY);
  }
  return {total, run};
}

// Adds up the pieces of a request's head whose steps fell to several workers, in the order of the keys: `split` CTAs
// for each, a share of the columns apiece, a thread for four columns of a row, up to 16 threads with every
// so many-th piece where a CTA has fewer of those. Pieces and their weights are loaded together, four at a time: with few
// pieces the kernel is two latencies long, and one long sequence (144 pieces of each head) spreads over the SMs (64
// heads, 8 key / value heads, 16000 keys, both kernels: 63 us with one CTA a head, 34 with up to 8 shares and 8 threads,
// 29 with 16 and 16, 30.5 with 32 and 32; eight pieces at a time cost 64 requests 3 %).
template <bool F16, int D>
__global__ void __launch_bounds__(THREADS) attention_join(const RowArgs g, int split) {
  __shared__ float2 sh_ml[THREADS];
  __shared__ float4 sh_o[THREADS];
  pdl_launch_dependents();
  const int item = (int)blockIdx.x / split, b = item / g.heads, head = item - b * g.heads;
  const int quads = D / 4 / split, col0 = ((int)blockIdx.x - item * split) * quads * 4;  // of this CTA: fours of columns, first one
  const int slots = g.max_rows * quads, groups = min(max(THREADS / slots, 1), 16);
  const Lengths x = lengths_of(g, b);  // (before the wait: the kernel before lets this one begin when it has waited itself)
  pdl_wait_primary();
  const int run = g.sums[g.B + 1], steps = steps_of(x), from = g.sums[b] + head * steps;
  if (steps == 0 || run == 0) return;
  const int w0 = from / run, w1 = (from + steps - 1) / run;
  if (w0 == w1) return;  // the worker has finished it
  const int place = g.max_rows * (D + 2);  // a worker has two: the head that began before its run, and the last one
  for (int slot = (int)threadIdx.x % (slots * groups); slot < slots * groups; slot += THREADS) {
    const int group = slot / slots, row = (slot - group * slots) / quads, col = col0 + (slot - group * slots) % quads * 4;
    const bool here = row < x.n * g.group && (int)threadIdx.x < slots * groups;
    float top = -INFINITY, all = 0.0f;
    float4 acc = make_float4(0, 0, 0, 0);
    if (here) {
      const float* base = g.partial + row * (D + 2);
      for (int w = w0 + group; w <= w1; w += 4 * groups) {
        float2 ml[4], lo[4], hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int v = min(w + i * groups, w1);
          const float* p = base + ((int64_t)v * 2 + (v == w0 ? 1 : 0)) * place;
          ml[i] = __ldcg(reinterpret_cast<const float2*>(p + D));
          lo[i] = __ldcg(reinterpret_cast<const float2*>(p + col));
          hi[i] = __ldcg(reinterpret_cast<const float2*>(p + col + 2));
        }
        float most = top;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (w + i * groups > w1) ml[i].y = 0.0f;  // a piece that is not there
          if (ml[i].y != 0.0f) most = fmaxf(most, ml[i].x);
        }
        const float f = top > -INFINITY ? fast_exp2(top - most) : 0.0f;
        all *= f;
        acc.x *= f;
        acc.y *= f;
        acc.z *= f;
        acc.w *= f;
        top = most;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = ml[i].y != 0.0f ? fast_exp2(ml[i].x - top) : 0.0f;
          all += ml[i].y * e;
          acc.x += lo[i].x * e;
          acc.y += lo[i].y * e;
          acc.z += hi[i].x * e;
          acc.w += hi[i].y * e;
        }
      }
    }
    if (groups > 1) {  // (then every thread has one slot at most)
      sh_ml[threadIdx.x] = make_float2(top, all);
      sh_o[threadIdx.x] = acc;
      __syncthreads();
      if (group > 0) return;
      float most = top;
      for (int k = 1; k < groups; ++k) most = fmaxf(most, sh_ml[slot + k * slots].x);
      const float f = top > -INFINITY ? fast_exp2(top - most) : 0.0f;
      all *= f;
      acc.x *= f;
      acc.y *= f;
      acc.z *= f;
      acc.w *= f;
      for (int k = 1; k < groups; ++k) {
        const float2 ml = sh_ml[slot + k * slots];
        const float4 o = sh_o[slot + k * slots];
        const float e = ml.y != 0.0f ? fast_exp2(ml.x - most) : 0.0f;
        all += ml.y * e;
        acc.x += o.x * e;
        acc.y += o.y * e;
        acc.z += o.z * e;
        acc.w += o.w * e;
      }
    }
    if (here) {
      const float inv = all == 0.0f ? 0.0f : 1.0f / all;
      const int token = row / g.group;
      uint16_t* out = g.o + (int64_t)(x.q0 + token) * g.ldo + (int64_t)(head * g.group + row - token * g.group) * D + col;
      *reinterpret_cast<uint2*>(out) = make_uint2(pack<F16>(acc.x * inv, acc.y * inv), pack<F16>(acc.z * inv, acc.w * inv));
    }
  }
}

// CTAs of the streaming kernel.
inline int rows_grid() {
  const int sms = pifa_sm_count();
  return sms < MAX_CTAS ? sms : MAX_CTAS;
}

// The launch of `kernel` with `smem` bytes beside the requests' first steps, and of the join if it leaves heads to it.
template <bool F16, int D, auto Kernel, typename... A>
cudaError_t launch_rows_and_join(const RowArgs& g, size_t smem, bool joins, cudaStream_t stream, const A&... more) {
  const int sms = pifa_sm_count(), grid = rows_grid();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = smem + (size_t)(g.B + 1) * 4;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cudaError_t e = pifa_allow_smem<Kernel>(223 * 1024);  // (the rest is static)
  if (e == cudaSuccess) e = pifa_launch_ex(&cfg, Kernel, g, more...);
  if (e != cudaSuccess || !joins) return e;
  cfg.dynamicSmemBytes = 0;
  const int64_t items = (int64_t)g.B * g.heads;
  int split = 1;
  while (split < 16 && items * split * 2 <= 8 * sms && g.max_rows * (D / 4) / (split * 2) >= THREADS / 16) split *= 2;
  cfg.gridDim = dim3((unsigned)(items * split));
  return pifa_launch_ex(&cfg, attention_join<F16, D>, g, split);
}

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
