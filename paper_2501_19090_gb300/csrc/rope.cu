// rope.cu -- rotary positions (pifa_rope, forward and gradient), the same with the write of keys and values
// into a paged cache (pifa_rope_cache), and the host's frequencies.
//
//   (x, y) -> scale (x cos a - y sin a, y cos a + x sin a),  a = 2 pi frac(position freq_i / 2^64)
//
// freq_i is a whole number of 2^-64 turns, so position * freq_i modulo 2^64 (64-bit integers) is the phase
// without an error that grows with the position; its upper 32 bits, as a signed fraction of a turn, go to
// sincospif. (An fp32 product of position and radians is off by 4e-3 at position 100000.)
//
// Bound by memory: every element is read and written once, 4 bytes an element, with about 3 flops for each.
// A CTA takes whole tokens: it computes their cosines and sines once, into shared memory, for all heads (a
// thread's own would cost more issue slots than the loads and stores), and its threads deal the heads' units
// of 16 elements: two 16-byte vectors, pairs across the vectors (half) or within them (interleaved).
// Measured, head_dim 128, bf16: 8192 tokens of 64 + 8 + 8 heads into the cache (336 MB) 54 us, 6.2 TB/s (the measured copy rate
// is 6.8); 2048 tokens of 32 heads, forward and gradient (two launches, 67 MB) 15.1 us.
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pifa.h"
#include "pifa_internal.h"
#include "ptx.cuh"

namespace {

using namespace pifa;

constexpr int THREADS = 256;
constexpr int MAX_TOKENS = 4;     // tokens of one CTA
constexpr int MAX_DIM = 512;

struct RopeArgs {
  const uint16_t *q, *k, *v;
  uint16_t *qr, *kc, *vc;
  const int32_t* positions;
  const int64_t* slots;
  const int64_t* freq;
  int64_t ldq, ldk, ldv, ldqr;
  int64_t page_stride, token_stride, head_stride, n_slots;
  int page_size;
  int T, hq, hk, dim, rot;
  int tokens;                     // of one CTA
  int heads;                      // of one CTA (blockIdx.y)
  float scale;
  int inverse;
  int* status;
};

template <bool F16>
__device__ __forceinline__ float2 unpack(uint32_t w) {
  if constexpr (F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
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

template <bool F16, bool HALF>
__global__ void __launch_bounds__(THREADS) rope_kernel(const RopeArgs g) {
  __shared__ __align__(16) float2 turn[MAX_TOKENS][MAX_DIM / 2];
  __shared__ int64_t place[MAX_TOKENS];  // the token's offset in the cache, -1: not stored
  pdl_launch_dependents();
  pdl_wait_primary();
  const int t0 = (int)blockIdx.x * g.tokens, nt = min(g.tokens, g.T - t0);
  const int pairs = g.rot / 2;
  const int units = g.dim / 16, turned = g.rot / 16;
  const int h0 = (int)blockIdx.y * g.heads, nh = min(g.heads, g.hq + 2 * g.hk - h0), n = nt * nh * units;
  // a unit's two vectors: halves of the turned part, or neighbours; those of a thread's next unit are in flight
  // while it works on one, the first ones while the CTA computes its cosines and sines
  struct Unit {
    int tt, h, u, a0, a1;
    uint4 va, vb;
  } next;
  auto fetch = [&](int i) {
    const int hh = i / units;
    next.u = i - hh * units;
    next.tt = hh / nh;
    next.h = h0 + hh - next.tt * nh;
    const int64_t t = t0 + next.tt;
    const uint16_t* src = next.h < g.hq           ? g.q + t * g.ldq + (int64_t)next.h * g.dim
                          : next.h < g.hq + g.hk ? g.k + t * g.ldk + (int64_t)(next.h - g.hq) * g.dim
                                                  : g.v + t * g.ldv + (int64_t)(next.h - g.hq - g.hk) * g.dim;
    const bool apart = HALF && next.u < turned;
    next.a0 = apart ? next.u * 8 : next.u * 16;
    next.a1 = apart ? next.u * 8 + pairs : next.u * 16 + 8;
    next.va = *reinterpret_cast<const uint4*>(src + next.a0);
    next.vb = *reinterpret_cast<const uint4*>(src + next.a1);
  };
  if ((int)threadIdx.x < n) fetch(threadIdx.x);
  for (int i = threadIdx.x; i < nt * pairs; i += THREADS) {
    const int tt = i / pairs, p = i - tt * pairs;
    const uint64_t phase = (uint64_t)(int64_t)g.positions[t0 + tt] * (uint64_t)g.freq[p];
    float s, c;
    sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &s, &c);
    // two pairs make a float4; those that a unit's lanes read together lie together
    turn[tt][2 * ((p & 7) / 2 * turned + p / 8) + (p & 1)] = make_float2(c * g.scale, (g.inverse ? -s : s) * g.scale);
  }
  if (g.hk && threadIdx.x < nt) {
    const int64_t slot = g.slots[t0 + threadIdx.x];
    int64_t at = -1;
    if (slot >= 0 && slot < g.n_slots) {
      const int64_t page = slot / g.page_size;
      at = page * g.page_stride + (slot - page * g.page_size) * g.token_stride;
    } else if (slot != -1) {
      latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
    }
    place[threadIdx.x] = at;
  }
  __syncthreads();

  for (int i = threadIdx.x; i < n; i += THREADS) {
    Unit x = next;
    if (i + THREADS < n) fetch(i + THREADS);
    uint16_t* dst;
    if (x.h < g.hq) {
      dst = g.qr + (int64_t)(t0 + x.tt) * g.ldqr + (int64_t)x.h * g.dim;
    } else {
      const bool is_v = x.h >= g.hq + g.hk;
      const int64_t at = place[x.tt];
      if (at < 0) continue;
      dst = (is_v ? g.vc : g.kc) + at + (x.h - g.hq - (is_v ? g.hk : 0)) * g.head_stride;
    }
    const bool turns = x.u < turned && x.h < g.hq + g.hk;
    if (turns) {
      uint32_t* wa = reinterpret_cast<uint32_t*>(&x.va);
      uint32_t* wb = reinterpret_cast<uint32_t*>(&x.vb);
      const float4* cs = reinterpret_cast<const float4*>(turn[x.tt]) + x.u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 r = cs[j * turned];
        if constexpr (HALF) {
          const float2 v = unpack<F16>(wa[j]), y = unpack<F16>(wb[j]);
          wa[j] = pack<F16>(v.x * r.x - y.x * r.y, v.y * r.z - y.y * r.w);
          wb[j] = pack<F16>(y.x * r.x + v.x * r.y, y.y * r.z + v.y * r.w);
        } else {
          uint32_t* w = (j < 2 ? wa : wb) + 2 * (j & 1);
          const float2 p = unpack<F16>(w[0]), q = unpack<F16>(w[1]);
          w[0] = pack<F16>(p.x * r.x - p.y * r.y, p.y * r.x + p.x * r.y);
          w[1] = pack<F16>(q.x * r.z - q.y * r.w, q.y * r.z + q.x * r.w);
        }
      }
    }
    *reinterpret_cast<uint4*>(dst + x.a0) = x.va;
    *reinterpret_cast<uint4*>(dst + x.a1) = x.vb;
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Whether T rows of `na` elements and T rows of `nb` have an element in common: columns of one matrix may interleave.
bool rows_overlap(const void* a, int64_t na, int64_t lda, const void* b, int64_t nb, int64_t ldb, int64_t T) {
  if (!pifa_spans_overlap(pifa_span(a, T, na, lda, 2), pifa_span(b, T, nb, ldb, 2))) return false;
  // a's element 0 is column 0; b's is element `from`
  const int64_t from = (int64_t)(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(a)) / 2;
  if (lda == ldb) {
    const int64_t at = (from % lda + lda) % lda;
    return at < na || at + nb > lda;
  }
  for (int64_t i = 0; i < T; ++i) {  // the first row of b that ends behind the start of a's row i
    const int64_t behind = i * lda - from - nb;
    const int64_t j = behind < 0 ? 0 : behind / ldb + 1;
    if (j < T && from + j * ldb < i * lda + na) return true;
  }
  return false;
}

int check_heads(int64_t T, int64_t heads, int64_t dim, int dtype, int64_t rot, int layout, float scale) {
  const int64_t lim = (int64_t)1 << 30;
  if (T < 0 || T >= lim) return pifa_fail(PIFA_ERR_INVALID_ARG, "T must be in [0, 2^30)");
  if (heads < 1 || heads > 65536) return pifa_fail(PIFA_ERR_INVALID_ARG, "heads must be in [1, 65536]");
  if (dtype != PIFA_DTYPE_BF16 && dtype != PIFA_DTYPE_FP16) return pifa_fail(PIFA_ERR_INVALID_ARG, "unknown dtype");
  if (layout != PIFA_ROPE_HALF && layout != PIFA_ROPE_INTERLEAVED) return pifa_fail(PIFA_ERR_INVALID_ARG, "unknown layout");
  if (!std::isfinite(scale)) return pifa_fail(PIFA_ERR_INVALID_ARG, "scale must be finite");
  if (dim < 1 || rot < 2 || rot > dim) return pifa_fail(PIFA_ERR_INVALID_ARG, "need 2 <= rot_dim <= head_dim");
  if (dim % 16 || dim > MAX_DIM || rot % 16)
    return pifa_fail(PIFA_ERR_UNSUPPORTED, "head_dim and rot_dim must be multiples of 16, head_dim at most 512");
  return PIFA_OK;
}

int launch(RopeArgs g, int dtype, int layout, void* cuda_stream) {
  cudaError_t e = cudaSuccess;
  g.status = pifa_status_word(&e);
  if (!g.status) return pifa_fail_cuda("device status word", e);
  // Whole tokens, as many to a CTA as make one round of the five CTAs that an SM holds, up to MAX_TOKENS (2048 tokens
  // of 32 heads, forward and gradient: 16.1 us when this was chosen; one to a CTA 19.3). Few tokens: the heads of one are dealt to CTAs until
  // those make two for every SM, one unit for a thread at the finest.
  const int nh = g.hq + 2 * g.hk, sms = pifa_sm_count(), round = 5 * sms;
  g.tokens = g.T > round * MAX_TOKENS ? MAX_TOKENS : (g.T + round - 1) / round;
  const int finest = (nh * (g.dim / 16) + THREADS - 1) / THREADS, wanted = (2 * sms + g.T - 1) / g.T;
  const int parts = finest < wanted ? finest : wanted;
  g.heads = (nh + parts - 1) / parts;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((g.T + g.tokens - 1) / g.tokens), (unsigned)((nh + g.heads - 1) / g.heads));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const bool f16 = dtype == PIFA_DTYPE_FP16, half = layout == PIFA_ROPE_HALF;
  e = f16 ? (half ? pifa_launch_ex(&cfg, rope_kernel<true, true>, g) : pifa_launch_ex(&cfg, rope_kernel<true, false>, g))
          : (half ? pifa_launch_ex(&cfg, rope_kernel<false, true>, g) : pifa_launch_ex(&cfg, rope_kernel<false, false>, g));
  if (e != cudaSuccess) return pifa_fail_cuda("rope launch", e);
  return PIFA_OK;
}

}  // namespace

extern "C" {

int pifa_rope_frequencies(int64_t rot_dim, double base, int scaling, double factor, double original, double low,
                          double high, int64_t* freq) {
  pifa_clear_error();
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > MAX_DIM) return pifa_fail(PIFA_ERR_INVALID_ARG, "rot_dim must be even, in [2, 512]");
  if (!(base > 1.0) || !std::isfinite(base) || !freq) return pifa_fail(PIFA_ERR_INVALID_ARG, "need a finite base > 1 and freq");
  if (scaling < PIFA_ROPE_SCALE_NONE || scaling > PIFA_ROPE_SCALE_BANDS) return pifa_fail(PIFA_ERR_INVALID_ARG, "unknown scaling");
  if (scaling != PIFA_ROPE_SCALE_NONE && (!(factor >= 1.0) || !std::isfinite(factor)))
    return pifa_fail(PIFA_ERR_INVALID_ARG, "need a finite factor >= 1");
  if (scaling == PIFA_ROPE_SCALE_BASE && rot_dim < 4) return pifa_fail(PIFA_ERR_INVALID_ARG, "scaling the base needs rot_dim >= 4");
  if (scaling == PIFA_ROPE_SCALE_BANDS &&
      (!(original > 0.0) || !std::isfinite(original) || !(low >= 0.0) || !(high > low) || !std::isfinite(high)))
    return pifa_fail(PIFA_ERR_INVALID_ARG, "bands need original > 0 and 0 <= low < high");
  if (scaling == PIFA_ROPE_SCALE_BASE) base *= std::pow(factor, (double)rot_dim / (double)(rot_dim - 2));
  const double two_pi = 6.283185307179586476925286766559;
  for (int64_t i = 0; i < rot_dim / 2; ++i) {
    double turns = std::pow(base, -2.0 * (double)i / (double)rot_dim) / two_pi;  // < 0.16
    if (scaling == PIFA_ROPE_SCALE_LINEAR) turns /= factor;
    if (scaling == PIFA_ROPE_SCALE_BANDS) {
      double keep = (original * turns - low) / (high - low);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      turns *= keep + (1.0 - keep) / factor;
    }
    freq[i] = (int64_t)std::rint(std::ldexp(turns, 64));
  }
  return PIFA_OK;
}

int pifa_rope(const void* X, int64_t T, int64_t heads, int64_t ldx, int64_t head_dim, int dtype,
              const int32_t* positions, const int64_t* freq, int64_t rot_dim, int layout, float scale, int inverse,
              void* Y, int64_t ldy, void* cuda_stream) {
  pifa_clear_error();
  int st = check_heads(T, heads, head_dim, dtype, rot_dim, layout, scale);
  if (st != PIFA_OK) return st;
  if (T == 0) return PIFA_OK;
  if (!X || !Y || !positions || !freq) return pifa_fail(PIFA_ERR_INVALID_ARG, "null X, Y, positions or freq");
  const int64_t row = heads * head_dim;
  if (ldx < row || ldy < row) return pifa_fail(PIFA_ERR_INVALID_ARG, "leading dimension smaller than the row length");
  if (!aligned16(X) || !aligned16(Y) || ((ldx | ldy) & 7))
    return pifa_fail(PIFA_ERR_ALIGNMENT, "X and Y must be 16-byte aligned, ldx and ldy multiples of 8");
  if (!(X == Y && ldx == ldy) && pifa_spans_overlap(pifa_span(X, T, row, ldx, 2), pifa_span(Y, T, row, ldy, 2)))
    return pifa_fail(PIFA_ERR_INVALID_ARG, "Y overlaps X without being X");
  RopeArgs g = {};
  g.q = static_cast<const uint16_t*>(X);
  g.qr = static_cast<uint16_t*>(Y);
  g.positions = positions;
  g.freq = freq;
  g.ldq = ldx;
  g.ldqr = ldy;
  g.T = (int)T;
  g.hq = (int)heads;
  g.dim = (int)head_dim;
  g.rot = (int)rot_dim;
  g.scale = scale;
  g.inverse = inverse != 0;
  return launch(g, dtype, layout, cuda_stream);
}

int pifa_rope_cache(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t T,
                    int64_t q_heads, int64_t kv_heads, int64_t head_dim, int dtype, const int32_t* positions,
                    const int64_t* slots, const int64_t* freq, int64_t rot_dim, int layout, float scale, void* Qr,
                    int64_t ldqr, void* k_cache, void* v_cache, int64_t pages, int64_t page_size, int64_t page_stride,
                    int64_t token_stride, int64_t head_stride, void* cuda_stream) {
  pifa_clear_error();
  int st = check_heads(T, q_heads, head_dim, dtype, rot_dim, layout, scale);
  if (st != PIFA_OK) return st;
  const PifaCacheShape c = {pages, page_size, kv_heads, head_dim, page_stride, token_stride, head_stride};
  if ((st = pifa_check_cache(c, 1, 65536)) != PIFA_OK) return st;
  if (T == 0) return PIFA_OK;
  if (!Q || !K || !V || !Qr || !positions || !slots || !freq || !k_cache || !v_cache)
    return pifa_fail(PIFA_ERR_INVALID_ARG, "null argument");
  const int64_t qrow = q_heads * head_dim, krow = kv_heads * head_dim;
  if (ldq < qrow || ldqr < qrow || ldk < krow || ldv < krow)
    return pifa_fail(PIFA_ERR_INVALID_ARG, "leading dimension smaller than the row length");
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(Qr) || !aligned16(k_cache) || !aligned16(v_cache) ||
      ((ldq | ldk | ldv | ldqr) & 7))
    return pifa_fail(PIFA_ERR_ALIGNMENT, "bases must be 16-byte aligned and leading dimensions multiples of 8");
  const PifaSpan q = pifa_span(Q, T, qrow, ldq, 2), in[] = {pifa_span(K, T, krow, ldk, 2), pifa_span(V, T, krow, ldv, 2)};
  const PifaSpan qr = pifa_span(Qr, T, qrow, ldqr, 2), kc = pifa_cache_span(k_cache, c), vc = pifa_cache_span(v_cache, c);
  // the two caches may interleave (pages of keys and values in turn), so their spans may overlap; a row of Q that
  // interleaves with K and V (columns of one projection) may too, but Qr then has to be Q itself or apart
  const bool in_place = Qr == Q && ldqr == ldq;
  bool bad = in_place ? rows_overlap(Q, qrow, ldq, K, krow, ldk, T) || rows_overlap(Q, qrow, ldq, V, krow, ldv, T)
                      : pifa_spans_overlap(qr, q) || pifa_spans_overlap(qr, in[0]) || pifa_spans_overlap(qr, in[1]);
  for (const PifaSpan& cache : {kc, vc})
    bad = bad || pifa_spans_overlap(cache, q) || pifa_spans_overlap(cache, in[0]) || pifa_spans_overlap(cache, in[1]) ||
          pifa_spans_overlap(cache, qr);
  if (bad || k_cache == v_cache) return pifa_fail(PIFA_ERR_INVALID_ARG, "an output overlaps another buffer");
  RopeArgs g = {};
  g.q = static_cast<const uint16_t*>(Q);
  g.k = static_cast<const uint16_t*>(K);
  g.v = static_cast<const uint16_t*>(V);
  g.qr = static_cast<uint16_t*>(Qr);
  g.kc = static_cast<uint16_t*>(k_cache);
  g.vc = static_cast<uint16_t*>(v_cache);
  g.positions = positions;
  g.slots = slots;
  g.freq = freq;
  g.ldq = ldq;
  g.ldk = ldk;
  g.ldv = ldv;
  g.ldqr = ldqr;
  g.page_stride = page_stride;
  g.token_stride = token_stride;
  g.head_stride = head_stride;
  g.n_slots = pages * page_size;
  g.page_size = (int)page_size;
  g.T = (int)T;
  g.hq = (int)q_heads;
  g.hk = (int)kv_heads;
  g.dim = (int)head_dim;
  g.rot = (int)rot_dim;
  g.scale = scale;
  return launch(g, dtype, layout, cuda_stream);
}

}  // extern "C"
