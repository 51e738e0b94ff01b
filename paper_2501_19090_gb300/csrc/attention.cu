// attention.cu -- pifa_paged_attention: argument checks and a kernel of one warp per (token, query head).
//
//   o = sum_j softmax_j(scale q . k_j) v_j over the keys j < L - n + i + 1 of new token i (L keys, n new tokens).
//
// One pass over the keys with a running maximum m and sum l in fp32: a key's weight is exp2(s - m) with
// s = scale log2(e) q . k, and sums and outputs are rescaled when m grows.
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pifa.h"
#include "pifa_internal.h"
#include "ptx.cuh"

namespace {

using namespace pifa;

struct AttnArgs {
  const uint16_t *q, *k, *v;
  uint16_t* o;
  const int32_t *table, *q_start, *kv_len;
  int64_t ldq, ldo, ldt, page_stride, token_stride, head_stride, pages;
  int T, hq, group, page_size, cols, B, max_q;
  float scale_log2;
  int* status;
};

template <bool F16>
__device__ __forceinline__ float2 unpack(uint32_t w) {
  if constexpr (F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

template <bool F16, int D>
__global__ void __launch_bounds__(128) attention_rows(const AttnArgs g) {
  constexpr int W = D / 64;  // words of two elements a lane holds
  pdl_launch_dependents();
  pdl_wait_primary();
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int t = (int)(unit / g.hq), h = (int)(unit % g.hq);
  if (t >= g.T || t >= g.q_start[g.B]) return;
  int lo = 0, hi = g.B;  // the last request with q_start <= t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (g.q_start[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int i = t - g.q_start[lo], n = g.q_start[lo + 1] - g.q_start[lo];
  int L = g.kv_len[lo];
  if (i >= g.max_q) {
    latch_status(g.status, PIFA_ERR_CAPACITY);
    return;
  }
  if ((int64_t)L > (int64_t)g.cols * g.page_size) {
    latch_status(g.status, PIFA_ERR_CAPACITY);
    L = g.cols * g.page_size;
  }
  const int seen = L - n + i + 1;
  float q[2 * W], o[2 * W] = {};
  const uint32_t* qw = reinterpret_cast<const uint32_t*>(g.q + t * g.ldq + (int64_t)h * D) + lane * W;
  for (int w = 0; w < W; ++w) {
    const float2 x = unpack<F16>(qw[w]);
    q[2 * w] = x.x * g.scale_log2;
    q[2 * w + 1] = x.y * g.scale_log2;
  }
  float m = -INFINITY, l = 0.0f;
  for (int j = 0; j < seen; ++j) {
    const int page = g.table[lo * g.ldt + j / g.page_size];
    float kf[2 * W] = {}, vf[2 * W] = {};
    if (page >= 0 && page < g.pages) {
      const int64_t at = page * g.page_stride + (j % g.page_size) * g.token_stride + (h / g.group) * g.head_stride;
      for (int w = 0; w < W; ++w) {
        const float2 x = unpack<F16>(reinterpret_cast<const uint32_t*>(g.k + at)[lane * W + w]);
        const float2 y = unpack<F16>(reinterpret_cast<const uint32_t*>(g.v + at)[lane * W + w]);
        kf[2 * w] = x.x;
        kf[2 * w + 1] = x.y;
        vf[2 * w] = y.x;
        vf[2 * w + 1] = y.y;
      }
    } else {
      latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
    }
    float s = 0.0f;
    for (int w = 0; w < 2 * W; ++w) s += q[w] * kf[w];
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    const float nm = fmaxf(m, s), up = nm == -INFINITY ? 0.0f : nm;
    const float c = exp2f(m - up), p = exp2f(s - up);
    l = l * c + p;
    for (int w = 0; w < 2 * W; ++w) o[w] = o[w] * c + p * vf[w];
    m = nm;
  }
  const float inv = l > 0.0f ? 1.0f / l : (l == l ? 0.0f : l);
  uint32_t* ow = reinterpret_cast<uint32_t*>(g.o + t * g.ldo + (int64_t)h * D) + lane * W;
  for (int w = 0; w < W; ++w) {
    if constexpr (F16) {
      const __half2 x = __floats2half2_rn(o[2 * w] * inv, o[2 * w + 1] * inv);
      ow[w] = *reinterpret_cast<const uint32_t*>(&x);
    } else {
      const __nv_bfloat162 x = __floats2bfloat162_rn(o[2 * w] * inv, o[2 * w + 1] * inv);
      ow[w] = *reinterpret_cast<const uint32_t*>(&x);
    }
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_sizes(int64_t T, int64_t hq, int64_t hk, int64_t dim, int64_t B, int64_t max_q) {
  const int64_t lim = (int64_t)1 << 30;
  if (T < 0 || T >= lim || B < 0 || B >= lim) return pifa_fail(PIFA_ERR_INVALID_ARG, "T and B must be in [0, 2^30)");
  if (hk < 1 || hk > 65536 || hq < 1 || hq % hk) return pifa_fail(PIFA_ERR_INVALID_ARG, "q_heads must be a multiple of kv_heads");
  if (max_q < 1) return pifa_fail(PIFA_ERR_INVALID_ARG, "max_q must be >= 1");
  if (hq / hk > 64) return pifa_fail(PIFA_ERR_UNSUPPORTED, "attention takes at most 64 query heads to a key / value head");
  if (dim != 64 && dim != 128) return pifa_fail(PIFA_ERR_UNSUPPORTED, "attention takes head_dim 64 or 128");
  if (B > 4096) return pifa_fail(PIFA_ERR_UNSUPPORTED, "attention takes at most 4096 requests");
  if (T * hq >= ((int64_t)1 << 32)) return pifa_fail(PIFA_ERR_UNSUPPORTED, "attention takes at most 2^32 rows of heads");
  return PIFA_OK;
}

// Whether a request's rows for one key / value head may be more than one 16-row product.
bool takes_tc(int64_t group, int64_t max_q) { return max_q > 16 || group * max_q > 16; }

}  // namespace

extern "C" {

int64_t pifa_paged_attention_workspace_size(int64_t T, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t B,
                                            int64_t max_q) {
  pifa_clear_error();
  const int st = check_sizes(T, q_heads, kv_heads, head_dim, B, max_q);
  if (st != PIFA_OK) return st;
  if (T == 0 || B == 0) return 0;
  return kWorkspaceReserve + (takes_tc(q_heads / kv_heads, max_q) ? attention_tc_workspace_bytes(T, q_heads, kv_heads, head_dim, B) : 0);
}

int pifa_paged_attention(const void* Q, int64_t ldq, int64_t T, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                         int dtype, const void* k_cache, const void* v_cache, int64_t pages, int64_t page_size,
                         int64_t page_stride, int64_t token_stride, int64_t head_stride, const int32_t* table,
                         int64_t cols, int64_t ldt, const int32_t* q_start, const int32_t* kv_len, int64_t B,
                         int64_t max_q, float scale, void* O, int64_t ldo, void* workspace, int64_t workspace_bytes,
                         void* cuda_stream) {
  pifa_clear_error();
  const int64_t need = pifa_paged_attention_workspace_size(T, q_heads, kv_heads, head_dim, B, max_q);
  if (need < 0) return (int)need;
  if (dtype != PIFA_DTYPE_BF16 && dtype != PIFA_DTYPE_FP16) return pifa_fail(PIFA_ERR_INVALID_ARG, "unknown dtype");
  const PifaCacheShape c = {pages, page_size, kv_heads, head_dim, page_stride, token_stride, head_stride};
  int st = pifa_check_cache(c, 16, 256);
  if (st != PIFA_OK) return st;
  if (page_size & (page_size - 1)) return pifa_fail(PIFA_ERR_UNSUPPORTED, "attention takes a page_size that is a power of two");
  const int64_t lim = (int64_t)1 << 31;
  if (cols < 0 || cols * page_size >= lim || ldt < cols || !std::isfinite(scale))
    return pifa_fail(PIFA_ERR_INVALID_ARG, "cols, ldt or scale out of range");
  if (T == 0 || B == 0) return PIFA_OK;
  if (!Q || !k_cache || !v_cache || !O || !q_start || !kv_len || (cols && !table))
    return pifa_fail(PIFA_ERR_INVALID_ARG, "null argument");
  const int64_t row = q_heads * head_dim;
  if (ldq < row || ldo < row) return pifa_fail(PIFA_ERR_INVALID_ARG, "leading dimension smaller than the row length");
  if (!aligned16(Q) || !aligned16(O) || !aligned16(k_cache) || !aligned16(v_cache) || ((ldq | ldo) & 7))
    return pifa_fail(PIFA_ERR_ALIGNMENT, "bases must be 16-byte aligned and leading dimensions multiples of 8");
  if (!workspace || workspace_bytes < need)
    return pifa_fail(PIFA_ERR_WORKSPACE, "workspace missing or smaller than pifa_paged_attention_workspace_size()");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u)
    return pifa_fail(PIFA_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
  const PifaSpan o = pifa_span(O, T, row, ldo, 2), ws = pifa_span(workspace, 1, need, need, 1);
  const PifaSpan in[] = {pifa_span(Q, T, row, ldq, 2), pifa_cache_span(k_cache, c), pifa_cache_span(v_cache, c),
                         pifa_span(table, B, cols, ldt, 4), pifa_span(q_start, 1, B + 1, B + 1, 4),
                         pifa_span(kv_len, 1, B, B, 4)};
  bool bad = pifa_spans_overlap(o, ws);
  for (const PifaSpan& x : in) bad = bad || pifa_spans_overlap(o, x) || pifa_spans_overlap(ws, x);
  if (bad) return pifa_fail(PIFA_ERR_INVALID_ARG, "O or workspace overlaps another buffer");
  cudaError_t e = cudaSuccess;
  int* status = pifa_status_word(&e);
  if (!status) return pifa_fail_cuda("device status word", e);
  if (takes_tc(q_heads / kv_heads, max_q)) {
    PifaAttention a = {Q, k_cache, v_cache, O, table, q_start, kv_len, T, ldq, ldo, ldt, cols, B, max_q, q_heads, c, dtype,
                       scale * 1.4426950408889634f, static_cast<uint8_t*>(workspace) + kWorkspaceReserve};
    return launch_attention_tc(a, status, pifa_wait_timeout_ns(), reinterpret_cast<cudaStream_t>(cuda_stream));
  }
  AttnArgs g = {};
  g.q = static_cast<const uint16_t*>(Q);
  g.k = static_cast<const uint16_t*>(k_cache);
  g.v = static_cast<const uint16_t*>(v_cache);
  g.o = static_cast<uint16_t*>(O);
  g.table = table;
  g.q_start = q_start;
  g.kv_len = kv_len;
  g.ldq = ldq;
  g.ldo = ldo;
  g.ldt = ldt;
  g.page_stride = page_stride;
  g.token_stride = token_stride;
  g.head_stride = head_stride;
  g.pages = pages;
  g.T = (int)T;
  g.hq = (int)q_heads;
  g.group = (int)(q_heads / kv_heads);
  g.page_size = (int)page_size;
  g.cols = (int)cols;
  g.B = (int)B;
  g.max_q = (int)(max_q < lim ? max_q : lim - 1);
  g.scale_log2 = scale * 1.4426950408889634f;
  g.status = status;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((T * q_heads + 3) / 4));
  cfg.blockDim = dim3(128);
  cfg.stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const bool f16 = dtype == PIFA_DTYPE_FP16;
  if (head_dim == 64) e = f16 ? pifa_launch_ex(&cfg, attention_rows<true, 64>, g) : pifa_launch_ex(&cfg, attention_rows<false, 64>, g);
  else e = f16 ? pifa_launch_ex(&cfg, attention_rows<true, 128>, g) : pifa_launch_ex(&cfg, attention_rows<false, 128>, g);
  if (e != cudaSuccess) return pifa_fail_cuda("attention launch", e);
  return PIFA_OK;
}

}  // extern "C"
