// attention_q8.cu -- pifa_paged_attention_q8: attention over a paged cache in 8 bits.
//
//   o = sum_j softmax_j(scale q . (s_b k_j)) t_b v_j over the keys j < L - n + i + 1 of new token i (L keys, n new tokens),
//   s_b and t_b the scales of the keys' and the values' block b = j / 16.
//
// A warp takes one row of one query head and walks its keys: the simplest form, right for every shape.
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pifa.h"
#include "pifa_internal.h"
#include "ptx.cuh"

namespace {

using namespace pifa;

constexpr int THREADS = 128;

struct Q8Args {
  const uint16_t* q;
  uint16_t* o;
  const uint8_t *k, *v, *ks, *vs;
  const int32_t *table, *q_start, *kv_len;
  int64_t ldq, ldo, ldt, page_stride, token_stride, head_stride, scale_page, scale_block, scale_head, pages;
  int T, heads, group, page_size, cols, B, max_q;
  float c;  // scale log2(e)
  int* status;
};

__device__ __forceinline__ float from_e4m3(uint32_t e) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)e));
  return __half22float2(*reinterpret_cast<const __half2*>(&h)).x;
}
__device__ __forceinline__ float scale_of(int byte) {
  return byte == 0 ? __uint_as_float(0x00400000u) : byte == 255 ? __uint_as_float(0x7fffffffu) : __uint_as_float((uint32_t)byte << 23);
}

template <bool F16, int D>
__global__ void __launch_bounds__(THREADS) attention_q8(const Q8Args g) {
  const int tid = threadIdx.x, lane = tid & 31, t = (int)blockIdx.x;
  bool over = false, falls = false;
  for (int b = tid; b < g.B; b += THREADS) {
    const int64_t n = (int64_t)g.q_start[b + 1] - g.q_start[b];
    falls |= n < 0;
    over |= n > 0 && (n > g.max_q || g.q_start[b + 1] > g.T);
    over |= g.kv_len[b] > g.cols * g.page_size;
  }
  if (over) latch_status(g.status, PIFA_ERR_CAPACITY);
  if (__syncthreads_or(falls)) {
    if (tid == 0) latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
    return;
  }
  int b = 0;  // the request of row t: the last that does not start after it
  for (int i = 1; i < g.B; ++i)
    if (g.q_start[i] <= t) b = i;
  const int q0 = g.q_start[b], token = t - q0;
  if (token < 0 || t >= g.q_start[b + 1] || token >= g.max_q) return;
  const int L = min(max(g.kv_len[b], 0), g.cols * g.page_size);
  const int seen = min(L, L - (g.q_start[b + 1] - q0) + 1 + token);
  constexpr int E = D / 32;
  for (int h = (int)blockIdx.y * (THREADS / 32) + (tid >> 5); h < g.heads * g.group; h += (int)gridDim.y * (THREADS / 32)) {
    const int head = h / g.group;
    float q[E], o[E] = {}, m = -INFINITY, l = 0.0f;
    for (int e = 0; e < E; ++e) {
      const uint16_t w = g.q[(int64_t)t * g.ldq + (int64_t)h * D + e * 32 + lane];
      q[e] = F16 ? __half2float(__ushort_as_half(w)) : __uint_as_float((uint32_t)w << 16);
    }
    for (int j = 0; j < seen; ++j) {
      const int id = g.table[b * g.ldt + j / g.page_size], at = j % g.page_size;
      const bool bad = id < 0 || id >= g.pages;
      if (bad) latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
      const int64_t from = bad ? 0 : id * g.page_stride + at * g.token_stride + head * g.head_stride;
      const int64_t sc = bad ? 0 : id * g.scale_page + at / PIFA_Q8_BLOCK * g.scale_block + head * g.scale_head;
      float s = 0.0f;
      if (!bad)
        for (int e = 0; e < E; ++e) s += q[e] * from_e4m3(g.k[from + e * 32 + lane]);
      for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      s *= bad ? 0.0f : g.c * scale_of(g.ks[sc]);
      const float up = fmaxf(m, s), f = m > -INFINITY ? exp2f(m - up) : 0.0f, p = exp2f(s - up);
      m = up;
      l = l * f + p;
      const float pv = bad ? 0.0f : p * scale_of(g.vs[sc]);
      for (int e = 0; e < E; ++e) o[e] = o[e] * f + (bad ? 0.0f : pv * from_e4m3(g.v[from + e * 32 + lane]));
    }
    for (int e = 0; e < E; ++e) {
      const float x = l == 0.0f ? 0.0f : o[e] / l;
      const uint16_t w = F16 ? __half_as_ushort(__float2half_rn(x)) : __bfloat16_as_ushort(__float2bfloat16_rn(x));
      g.o[(int64_t)t * g.ldo + (int64_t)h * D + e * 32 + lane] = w;
    }
  }
}

}  // namespace

int launch_attention_q8(const PifaAttention& a, int* status, cudaStream_t stream) {
  Q8Args g = {};
  g.q = static_cast<const uint16_t*>(a.q);
  g.o = static_cast<uint16_t*>(a.o);
  g.k = static_cast<const uint8_t*>(a.k);
  g.v = static_cast<const uint8_t*>(a.v);
  g.ks = a.q8->k;
  g.vs = a.q8->v;
  g.table = a.table;
  g.q_start = a.q_start;
  g.kv_len = a.kv_len;
  g.ldq = a.ldq;
  g.ldo = a.ldo;
  g.ldt = a.ldt;
  g.page_stride = a.cache.page_stride;
  g.token_stride = a.cache.token_stride;
  g.head_stride = a.cache.head_stride;
  g.scale_page = a.q8->shape.page_stride;
  g.scale_block = a.q8->shape.block_stride;
  g.scale_head = a.q8->shape.head_stride;
  g.pages = a.cache.pages;
  g.T = (int)a.T;
  g.heads = (int)a.cache.heads;
  g.group = (int)(a.q_heads / a.cache.heads);
  g.page_size = (int)a.cache.page_size;
  g.cols = (int)a.cols;
  g.B = (int)a.B;
  g.max_q = (int)(a.max_q < a.T ? a.max_q : a.T);
  g.c = a.scale_log2;
  g.status = status;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.T, (unsigned)((a.q_heads + 3) / 4 < 65535 ? (a.q_heads + 3) / 4 : 65535));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = stream;
  const bool f16 = a.dtype == PIFA_DTYPE_FP16;
  cudaError_t e;
  if (a.cache.dim == 64) e = f16 ? pifa_launch_ex(&cfg, attention_q8<true, 64>, g) : pifa_launch_ex(&cfg, attention_q8<false, 64>, g);
  else e = f16 ? pifa_launch_ex(&cfg, attention_q8<true, 128>, g) : pifa_launch_ex(&cfg, attention_q8<false, 128>, g);
  if (e != cudaSuccess) return pifa_fail_cuda("attention_q8 launch", e);
  return PIFA_OK;
}
