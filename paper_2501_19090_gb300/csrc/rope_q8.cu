// rope_q8.cu -- a paged cache in 8 bits: written with the rotation (pifa_rope_cache_q8), and read back (pifa_cache_read_q8).
//
//   s = 2^e, e the least with max |x| <= 448 2^e over a block's tokens (16 slots of a page, one head);  q = rne(x / s) as e4m3
//
// A block grows: the tokens that it held keep their elements while its scale stays, and are rounded anew, rne(q s_old / s),
// when a new token raises it. With powers of two that loses nothing but in the subnormal range (a rounding there per rise), the
// scale of a block does not depend on how its tokens were dealt to calls, and a float's relative precision does not depend on it.
//
// Bound by memory. The write: a stretch, the neighbouring rows of one block, and one head go to one or some warps, which hold all its
// elements in registers from the rotation over the maximum to the rounding: every element is read and written once. CTAs of their own
// turn queries in the same launch. Few tokens (decode): a chain of latencies, slots and cosines, rows, scale, and rounds of CTAs.
// Measured, head_dim 128, bf16: 8192 tokens of 64 + 8 + 8 heads (318 MB) 59 us, 5.4 TB/s (the queries alone 47); 200 sequences in decode
// 5.0, 8 sequences, 32 + 32 + 32 heads, 3.5; reading back 50001 tokens of 8 heads (307 MB) 50.5 us, 6.1 TB/s.
#include <cmath>

#include "q8.cuh"
#include "rope.cuh"

namespace {

constexpr int THREADS = ROPE_THREADS;
constexpr int BLOCK = PIFA_Q8_BLOCK;
constexpr int MAX_WINDOW = 16;             // rows of a CTA that stores keys and values
constexpr int READ_WINDOW = 8;             // most rows of a CTA that reads (50001 tokens, 8 heads: 50 us, with 16 rows 52)
constexpr int TURN_BYTES = 38 * 1024;      // of cosines and sines: with the rest, what a CTA has without asking for more

struct StoreArgs {
  RopeArgs q;                              // the queries: rows of heads, no cache
  const uint16_t *k, *v;
  uint8_t *kc, *vc, *ks, *vs;
  const int64_t* slots;
  int64_t ldk, ldv, n_slots;
  int64_t page_stride, token_stride, head_stride;
  int64_t scale_page, scale_block, scale_head;
  int page_size, hk;
  int window, kv_heads, kv_parts, kv_ctas;  // rows and heads (of 2 hk) of a CTA that stores; CTAs of a window; all of them
  int q_parts, stride;  // every stride-th CTA stores, as long as there are such
};

struct ReadArgs {
  const uint8_t *kc, *vc, *ks, *vs;
  const int64_t* slots;
  uint16_t *k, *v;
  int64_t ldk, ldv, n_slots;
  int64_t page_stride, token_stride, head_stride;
  int64_t scale_page, scale_block, scale_head;
  int T, page_size, hk, dim, tokens;
  int* status;
};

// Neighbouring rows whose slots lie in one block.
struct Stretch {
  int row, n;          // first row (from the window's), rows
  unsigned written;    // bit o: offset o of the block is among them
  int64_t at, scale;   // offsets of the block's first token and of its scale, for head 0
};

// Two e4m3 numbers, the first in the low byte, rounded to nearest even; a NaN stays one.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t two) {
  const uint32_t h = halves_of(two);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// 2^(127 - byte); 0 for a scale that is not a number
__device__ __forceinline__ float inverse_scale_of(int byte) {
  return byte < 254 ? __uint_as_float((uint32_t)(254 - byte) << 23) : byte == 254 ? __uint_as_float(0x00400000u) : 0.0f;
}

// Keys and values of the stretches that begin in a window of rows. GW warps take a stretch of one head: up to 16 rows, EACH
// units of 16 elements a lane (a unit: two vectors of 8, as in rope_tokens).
template <bool F16, bool HALF, int EACH, int GW>
__device__ __forceinline__ void store_blocks(const StoreArgs& g, int wx, int part) {
  extern __shared__ __align__(16) float2 turns[];  // of a row: as rope_tokens lays them out
  __shared__ int64_t slot_of[MAX_WINDOW + BLOCK];  // from the row before the window on
  __shared__ Stretch list[MAX_WINDOW];
  __shared__ int count, last;
  __shared__ uint32_t most_of[THREADS / 32];
  const int tid = threadIdx.x, lane = tid & 31, T = g.q.T, dim = g.q.dim;
  const int t0 = wx * g.window, rows = min(g.window + BLOCK - 1, T - t0), inside = min(g.window, T - t0);
  const int pairs = g.q.rot / 2, units = dim / 16, turned = g.q.rot / 16;
  const int h0 = part * g.kv_heads, nh = min(g.kv_heads, 2 * g.hk - h0);
  // cosines and sines of rows [from, to)
  auto turn_rows = [&](int from, int to) {
    for (int i = from * pairs + tid; i < to * pairs; i += THREADS) {
      const int tt = i / pairs, p = i - tt * pairs;
      const uint64_t phase = (uint64_t)(int64_t)g.q.positions[t0 + tt] * (uint64_t)g.q.freq[p];
      float s, c;
      sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &s, &c);
      turns[tt * pairs + 2 * ((p & 7) / 2 * turned + p / 8) + (p & 1)] = make_float2(c * g.q.scale, s * g.q.scale);
    }
  };
  for (int i = tid; i <= rows; i += THREADS) slot_of[i] = t0 + i > 0 ? g.slots[t0 + i - 1] : -1;
  if (h0 < g.hk) turn_rows(0, inside);  // a stretch that goes on behind the window: later, when that is known
  __syncthreads();
  if (tid < 32) {
    auto good = [&](int64_t s) { return s >= 0 && s < g.n_slots; };
    const int64_t s = lane < inside ? slot_of[lane + 1] : -1, before = lane < inside ? slot_of[lane] : -1;
    if (s != -1 && !good(s)) latch_status(g.q.status, PIFA_ERR_DEVICE_INDEX);
    const bool begins = good(s) && !(good(before) && before / BLOCK == s / BLOCK);
    const unsigned all = __ballot_sync(0xffffffffu, begins);
    int end = 0;
    if (begins) {
      Stretch x = {lane, 0, 0u, 0, 0};
      const int64_t block = s / BLOCK;
      bool twice = false;
      for (; lane + x.n < rows; ++x.n) {
        const int64_t o = slot_of[lane + 1 + x.n] - block * BLOCK;
        if (o < 0 || o >= BLOCK) break;
        if (x.n == BLOCK) {
          twice = true;
          break;
        }
        twice |= (x.written >> o & 1u) != 0;
        x.written |= 1u << o;
      }
      if (twice) latch_status(g.q.status, PIFA_ERR_DEVICE_INDEX);
      const int64_t page = s / g.page_size, token = block * BLOCK - page * g.page_size;
      x.at = page * g.page_stride + token * g.token_stride;
      x.scale = page * g.scale_page + token / BLOCK * g.scale_block;
      list[__popc(all & ((1u << lane) - 1u))] = x;
      end = x.row + x.n;
    }
    end = __reduce_max_sync(0xffffffffu, end);
    if (lane == 0) {
      count = __popc(all);
      last = end;
    }
  }
  __syncthreads();
  if (h0 < g.hk && last > inside) {
    turn_rows(inside, last);
    __syncthreads();
  }

  const int group = (tid >> 5) / GW, l = tid - group * GW * 32;
  const int tasks = count * nh;
  for (int task = group; task < tasks; task += THREADS / 32 / GW) {
    const int which = task / nh, h = h0 + task - which * nh;
    const bool is_k = h < g.hk;
    const int head = is_k ? h : h - g.hk;
    const Stretch x = list[which];
    const uint16_t* src = (is_k ? g.k : g.v) + (int64_t)head * dim;
    const int64_t ld = is_k ? g.ldk : g.ldv;
    uint8_t* data = (is_k ? g.kc : g.vc) + x.at + (int64_t)head * g.head_stride;
    uint8_t* scale = (is_k ? g.ks : g.vs) + x.scale + (int64_t)head * g.scale_head;
    const bool held = !(x.written & 1u);  // tokens before these: a block begins anew with its first one
    const int was = held ? *scale : 0;
    float e[EACH][16];
    float most = 0.0f;
    const int n = x.n * units;
    auto places = [&](int u, int& a0, int& a1) {
      const bool apart = HALF && is_k && u < turned;
      a0 = apart ? u * 8 : u * 16;
      a1 = apart ? u * 8 + pairs : u * 16 + 8;
    };
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = l + k * GW * 32, r = i / units, u = i - r * units;
      if (i >= n) continue;
      int a0, a1;
      places(u, a0, a1);
      const uint16_t* row = src + (int64_t)(t0 + x.row + r) * ld;
      const uint4 va = *reinterpret_cast<const uint4*>(row + a0), vb = *reinterpret_cast<const uint4*>(row + a1);
      const uint32_t w[8] = {va.x, va.y, va.z, va.w, vb.x, vb.y, vb.z, vb.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 p = unpack<F16>(w[j]);
        e[k][2 * j] = p.x;
        e[k][2 * j + 1] = p.y;
      }
      if (is_k && u < turned) {
        const float4* cs = reinterpret_cast<const float4*>(turns + (x.row + r) * pairs) + u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float4 c = cs[j * turned];
          auto turn = [](float& a, float& b, float co, float si) {
            const float y = a * co - b * si;
            b = b * co + a * si;
            a = y;
          };
          if constexpr (HALF) {
            turn(e[k][2 * j], e[k][2 * j + 8], c.x, c.y);
            turn(e[k][2 * j + 1], e[k][2 * j + 9], c.z, c.w);
          } else {
            turn(e[k][4 * j], e[k][4 * j + 1], c.x, c.y);
            turn(e[k][4 * j + 2], e[k][4 * j + 3], c.z, c.w);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) most = max_nan(most, fabsf(e[k][j]));
    }
    auto over_group = [&](float v) {  // magnitudes, infinity and NaN among them, order as their bits do
      uint32_t b = __reduce_max_sync(0xffffffffu, __float_as_uint(v));
      if constexpr (GW > 1) {
        named_barrier_sync(1 + group, GW * 32);
        if (lane == 0) most_of[tid >> 5] = b;
        named_barrier_sync(1 + group, GW * 32);
#pragma unroll
        for (int w = 0; w < GW; ++w) b = max(b, most_of[group * GW + w]);
      }
      return b;
    };
    uint32_t top = over_group(most);
    if (top >= 0x7f800000u) {  // what is not finite is stored as NaN and leaves the scale to the others
      most = 0.0f;
#pragma unroll
      for (int k = 0; k < EACH; ++k)
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (l + k * GW * 32 < n) {
            if (fabsf(e[k][j]) < __uint_as_float(0x7f800000u)) most = fmaxf(most, fabsf(e[k][j]));
            else e[k][j] = __uint_as_float(0x7fffffffu);
          }
      top = over_group(most);
    }
    // max |x| = 2^(E - 127) (1 + f) <= 448 2^e = 1.75 2^(8 + e)
    const int fresh = max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u), 1);
    const int byte = max(fresh, was);
    const float inv = inverse_scale_of(byte);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = l + k * GW * 32, r = i / units, u = i - r * units;
      if (i >= n) continue;
      int a0, a1;
      places(u, a0, a1);
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = to_e4m3x2(e[k][4 * j] * inv, e[k][4 * j + 1] * inv) | to_e4m3x2(e[k][4 * j + 2] * inv, e[k][4 * j + 3] * inv) << 16;
      uint8_t* row = data + (slot_of[x.row + r + 1] & (BLOCK - 1)) * g.token_stride;
      *reinterpret_cast<uint2*>(row + a0) = make_uint2(w[0], w[1]);
      *reinterpret_cast<uint2*>(row + a1) = make_uint2(w[2], w[3]);
    }
    if (held && byte > was) {
      const float f = byte - was > 30 ? 0.0f : __uint_as_float((uint32_t)(127 + was - byte) << 23);
      for (int i = l; i < BLOCK * units; i += GW * 32) {
        const int r = i / units;
        if (x.written >> r & 1u) continue;
        uint4* at = reinterpret_cast<uint4*>(data + r * g.token_stride + (i - r * units) * 16);
        uint4 v = *at;
        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 a = from_e4m3x2(w[j] & 0xffffu), b = from_e4m3x2(w[j] >> 16);
          w[j] = to_e4m3x2(a.x * f, a.y * f) | to_e4m3x2(b.x * f, b.y * f) << 16;
        }
        *at = v;
      }
    }
    if (GW > 1) named_barrier_sync(1 + group, GW * 32);  // all have read the scale
    else __syncwarp();
    if (l == 0) *scale = (uint8_t)byte;
  }
}

template <bool F16, bool HALF, int EACH, int GW>
__global__ void __launch_bounds__(THREADS, EACH == 2 ? 4 : 2) rope_cache_q8(const StoreArgs g) {
  pdl_launch_dependents();
  pdl_wait_primary();
  // CTAs that store keys and values take longer and come first, of many tokens in turn with those that turn queries
  const int b = (int)blockIdx.x, at = b / g.stride;
  if (b == at * g.stride && at < g.kv_ctas) {
    store_blocks<F16, HALF, EACH, GW>(g, at / g.kv_parts, at % g.kv_parts);
  } else {
    const int q = b - min((b + g.stride - 1) / g.stride, g.kv_ctas);
    rope_tokens<F16, HALF>(g.q, q / g.q_parts, q % g.q_parts);
  }
}

// A thread takes 16 elements at a time: 16 bytes in, 32 out.
template <bool F16>
__global__ void __launch_bounds__(THREADS) cache_read_q8(const ReadArgs g) {
  __shared__ int64_t at[READ_WINDOW], scale_at[READ_WINDOW];  // -1: the row is not written
  pdl_launch_dependents();
  pdl_wait_primary();
  const int t0 = (int)blockIdx.x * g.tokens, nt = min(g.tokens, g.T - t0);
  if ((int)threadIdx.x < nt) {
    const int64_t slot = g.slots[t0 + threadIdx.x];
    int64_t a = -1;
    if (slot >= 0 && slot < g.n_slots) {
      const int64_t page = slot / g.page_size, token = slot - page * g.page_size;
      a = page * g.page_stride + token * g.token_stride;
      scale_at[threadIdx.x] = page * g.scale_page + token / BLOCK * g.scale_block;
    } else if (slot != -1) {
      latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
    }
    at[threadIdx.x] = a;
  }
  __syncthreads();
  const int units = g.dim / 16, n = nt * 2 * g.hk * units;
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const int hh = i / units, u = i - hh * units, tt = hh / (2 * g.hk), h = hh - tt * 2 * g.hk;
    if (at[tt] < 0) continue;
    const bool is_k = h < g.hk;
    const int head = is_k ? h : h - g.hk;
    const uint4 v = *reinterpret_cast<const uint4*>((is_k ? g.kc : g.vc) + at[tt] + head * g.head_stride + u * 16);
    const float s = scale_of((is_k ? g.ks : g.vs)[scale_at[tt] + head * g.scale_head]);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = scaled_from_e4m3x2<F16>(w[j / 2] >> (16 * (j & 1)) & 0xffffu, s);
    uint16_t* dst = (is_k ? g.k + (t0 + tt) * g.ldk : g.v + (t0 + tt) * g.ldv) + (int64_t)head * g.dim + u * 16;
    *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
    *reinterpret_cast<uint4*>(dst + 8) = make_uint4(o[4], o[5], o[6], o[7]);
  }
}

// Few tokens make short stretches: a warp for each (four units a lane) spares the exchange between two. Many make whole blocks: two
// units a lane leave the registers, and with them the loads in flight, to twice the CTAs. (8192 tokens, 64 + 8 + 8 heads: 83 us with
// four units, 61 with two; 200 sequences in decode: 5.8 and 7.0.)
constexpr int FEW_TOKENS = 1024;
template <bool F16, bool HALF, int EACH>
cudaError_t launch_store(const cudaLaunchConfig_t* cfg, const StoreArgs& g) {
  if (g.q.dim <= 32 * EACH) return pifa_launch_ex(cfg, rope_cache_q8<F16, HALF, EACH, 1>, g);
  if (g.q.dim <= 64 * EACH) return pifa_launch_ex(cfg, rope_cache_q8<F16, HALF, EACH, 2>, g);
  if (EACH == 4 || g.q.dim <= 128 * EACH) return pifa_launch_ex(cfg, rope_cache_q8<F16, HALF, EACH, 4>, g);
  return pifa_launch_ex(cfg, rope_cache_q8<F16, HALF, EACH, EACH == 4 ? 4 : 8>, g);
}
template <bool F16, bool HALF>
cudaError_t launch_store(const cudaLaunchConfig_t* cfg, const StoreArgs& g) {
  return g.q.T < FEW_TOKENS ? launch_store<F16, HALF, 4>(cfg, g) : launch_store<F16, HALF, 2>(cfg, g);
}

void overlap_launches(cudaLaunchConfig_t& cfg, cudaLaunchAttribute& attr, void* cuda_stream) {
  cfg.blockDim = dim3(THREADS);
  cfg.stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
}

}  // namespace

extern "C" {

int pifa_rope_cache_q8(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv, int64_t T,
                       int64_t q_heads, int64_t kv_heads, int64_t head_dim, int dtype, const int32_t* positions,
                       const int64_t* slots, const int64_t* freq, int64_t rot_dim, int layout, float scale, void* Qr,
                       int64_t ldqr, void* k_cache, void* v_cache, void* k_scale, void* v_scale, int64_t pages,
                       int64_t page_size, int64_t page_stride, int64_t token_stride, int64_t head_stride,
                       int64_t scale_page_stride, int64_t scale_block_stride, int64_t scale_head_stride, void* cuda_stream) {
  pifa_clear_error();
  int st = pifa_check_heads(T, q_heads, head_dim, dtype, rot_dim, layout, scale);
  if (st != PIFA_OK) return st;
  const PifaCacheShape c = {pages, page_size, kv_heads, head_dim, page_stride, token_stride, head_stride};
  const PifaScaleShape sc = {scale_page_stride, scale_block_stride, scale_head_stride};
  if ((st = pifa_check_cache_q8(c, sc, 65536)) != PIFA_OK) return st;
  if (T == 0) return PIFA_OK;
  if (!Q || !K || !V || !Qr || !positions || !slots || !freq || !k_cache || !v_cache || !k_scale || !v_scale)
    return pifa_fail(PIFA_ERR_INVALID_ARG, "null argument");
  const int64_t qrow = q_heads * head_dim, krow = kv_heads * head_dim;
  if (ldq < qrow || ldqr < qrow || ldk < krow || ldv < krow)
    return pifa_fail(PIFA_ERR_INVALID_ARG, "leading dimension smaller than the row length");
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(Qr) || !aligned16(k_cache) || !aligned16(v_cache) ||
      ((ldq | ldk | ldv | ldqr) & 7))
    return pifa_fail(PIFA_ERR_ALIGNMENT, "bases must be 16-byte aligned and leading dimensions multiples of 8");
  const PifaSpan in[] = {pifa_span(Q, T, qrow, ldq, 2), pifa_span(K, T, krow, ldk, 2), pifa_span(V, T, krow, ldv, 2)};
  const PifaSpan qr = pifa_span(Qr, T, qrow, ldqr, 2);
  const PifaSpan out[] = {pifa_cache_span(k_cache, c, 1), pifa_cache_span(v_cache, c, 1), pifa_scale_span(k_scale, c, sc),
                          pifa_scale_span(v_scale, c, sc)};
  // as in pifa_rope_cache: the caches, and the scales, may interleave, as may a row of Q that is turned in place with K and V
  bool bad = Qr == Q && ldqr == ldq ? pifa_rows_overlap(Q, qrow, ldq, K, krow, ldk, T) || pifa_rows_overlap(Q, qrow, ldq, V, krow, ldv, T)
                                    : pifa_spans_overlap(qr, in[0]) || pifa_spans_overlap(qr, in[1]) || pifa_spans_overlap(qr, in[2]);
  const PifaSpan index[] = {pifa_span(positions, 1, T, T, 4), pifa_span(slots, 1, T, T, 8), pifa_span(freq, 1, rot_dim / 2, rot_dim / 2, 8)};
  for (const PifaSpan& o : out) {
    bad = bad || pifa_spans_overlap(o, qr);
    for (const PifaSpan& i : in) bad = bad || pifa_spans_overlap(o, i);
    for (const PifaSpan& i : index) bad = bad || pifa_spans_overlap(o, i);
  }
  for (const PifaSpan& i : index) bad = bad || pifa_spans_overlap(qr, i);
  if (bad || k_cache == v_cache || k_scale == v_scale) return pifa_fail(PIFA_ERR_INVALID_ARG, "an output overlaps another buffer");
  cudaError_t e = cudaSuccess;
  StoreArgs g = {};
  g.q.status = pifa_status_word(&e);
  if (!g.q.status) return pifa_fail_cuda("device status word", e);
  g.q.q = static_cast<const uint16_t*>(Q);
  g.q.qr = static_cast<uint16_t*>(Qr);
  g.q.positions = positions;
  g.q.freq = freq;
  g.q.ldq = ldq;
  g.q.ldqr = ldqr;
  g.q.T = (int)T;
  g.q.hq = (int)q_heads;
  g.q.dim = (int)head_dim;
  g.q.rot = (int)rot_dim;
  g.q.scale = scale;
  g.k = static_cast<const uint16_t*>(K);
  g.v = static_cast<const uint16_t*>(V);
  g.kc = static_cast<uint8_t*>(k_cache);
  g.vc = static_cast<uint8_t*>(v_cache);
  g.ks = static_cast<uint8_t*>(k_scale);
  g.vs = static_cast<uint8_t*>(v_scale);
  g.slots = slots;
  g.ldk = ldk;
  g.ldv = ldv;
  g.n_slots = pages * page_size;
  g.page_stride = page_stride;
  g.token_stride = token_stride;
  g.head_stride = head_stride;
  g.scale_page = scale_page_stride;
  g.scale_block = scale_block_stride;
  g.scale_head = scale_head_stride;
  g.page_size = (int)page_size;
  g.hk = (int)kv_heads;
  // Queries: whole tokens, as pifa_rope deals them. Keys and values: windows of up to 16 rows.
  const int sms = pifa_sm_count(), round = 5 * sms, t = (int)T;
  g.q.tokens = t > round * MAX_TOKENS ? MAX_TOKENS : (t + round - 1) / round;
  const int finest = ((int)q_heads * ((int)head_dim / 16) + THREADS - 1) / THREADS, wanted = (2 * sms + t - 1) / t;
  g.q.heads = ((int)q_heads + (finest < wanted ? finest : wanted) - 1) / (finest < wanted ? finest : wanted);
  g.q_parts = ((int)q_heads + g.q.heads - 1) / g.q.heads;
  const int fits = TURN_BYTES / ((int)rot_dim * 4) - (BLOCK - 1);  // rows whose cosines and sines have room
  g.window = (t + sms - 1) / sms;
  if (g.window > fits) g.window = fits;
  if (g.window > MAX_WINDOW) g.window = MAX_WINDOW;
  const int windows = (t + g.window - 1) / g.window, heads = 2 * (int)kv_heads;
  int parts = (2 * sms + windows - 1) / windows;
  if (parts > (heads + 7) / 8) parts = (heads + 7) / 8;
  if (t < FEW_TOKENS) {
    // A second round of CTAs costs 2 us. So: no more that store than make a difference to their turns of eight warps, and where those of
    // the queries do not begin in the first round beside them, two CTAs an SM, they take more tokens each if then they do. (200 sequences in
    // decode, 64 + 8 + 8 heads: 5.9 us and 5.0; 64 of 32 + 32 + 32: 7.3 and 5.3.)
    const int turns = ((heads + parts - 1) / parts + 7) / 8;
    parts = (heads + 8 * turns - 1) / (8 * turns);
    const int left = 2 * sms - windows * parts, q_ctas = (t + g.q.tokens - 1) / g.q.tokens * g.q_parts;
    if (q_ctas > left && left >= (t + MAX_TOKENS - 1) / MAX_TOKENS) {
      g.q.tokens = (t + left - 1) / left;
      g.q.heads = (int)q_heads;
      g.q_parts = 1;
    }
  }
  g.kv_heads = (heads + parts - 1) / parts;
  g.kv_parts = (heads + g.kv_heads - 1) / g.kv_heads;
  g.kv_ctas = windows * g.kv_parts;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr;
  overlap_launches(cfg, attr, cuda_stream);
  const int64_t ctas = (int64_t)windows * g.kv_parts + (int64_t)((t + g.q.tokens - 1) / g.q.tokens) * g.q_parts;
  if (ctas > 0x7fffffff) return pifa_fail(PIFA_ERR_UNSUPPORTED, "too many tokens times heads");
  g.stride = t >= FEW_TOKENS && ctas >= 2 * (int64_t)g.kv_ctas ? 2 : 1;
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.dynamicSmemBytes = (size_t)(g.window + BLOCK - 1) * (size_t)rot_dim * 4;
  const bool f16 = dtype == PIFA_DTYPE_FP16, half = layout == PIFA_ROPE_HALF;
  e = f16 ? (half ? launch_store<true, true>(&cfg, g) : launch_store<true, false>(&cfg, g))
          : (half ? launch_store<false, true>(&cfg, g) : launch_store<false, false>(&cfg, g));
  if (e != cudaSuccess) return pifa_fail_cuda("rope_cache_q8 launch", e);
  return PIFA_OK;
}

int pifa_cache_read_q8(const void* k_cache, const void* v_cache, const void* k_scale, const void* v_scale, int64_t pages,
                       int64_t page_size, int64_t kv_heads, int64_t head_dim, int64_t page_stride, int64_t token_stride,
                       int64_t head_stride, int64_t scale_page_stride, int64_t scale_block_stride, int64_t scale_head_stride,
                       const int64_t* slots, int64_t T, int dtype, void* K, int64_t ldk, void* V, int64_t ldv, void* cuda_stream) {
  pifa_clear_error();
  if (T < 0 || T >= ((int64_t)1 << 30)) return pifa_fail(PIFA_ERR_INVALID_ARG, "T must be in [0, 2^30)");
  if (dtype != PIFA_DTYPE_BF16 && dtype != PIFA_DTYPE_FP16) return pifa_fail(PIFA_ERR_INVALID_ARG, "unknown dtype");
  const PifaCacheShape c = {pages, page_size, kv_heads, head_dim, page_stride, token_stride, head_stride};
  const PifaScaleShape sc = {scale_page_stride, scale_block_stride, scale_head_stride};
  const int st = pifa_check_cache_q8(c, sc, 65536);
  if (st != PIFA_OK) return st;
  if (head_dim % 16 || head_dim > MAX_DIM) return pifa_fail(PIFA_ERR_UNSUPPORTED, "head_dim must be a multiple of 16, at most 512");
  if (T == 0) return PIFA_OK;
  if (!k_cache || !v_cache || !k_scale || !v_scale || !slots || !K || !V) return pifa_fail(PIFA_ERR_INVALID_ARG, "null argument");
  const int64_t row = kv_heads * head_dim;
  if (ldk < row || ldv < row) return pifa_fail(PIFA_ERR_INVALID_ARG, "leading dimension smaller than the row length");
  if (!aligned16(K) || !aligned16(V) || !aligned16(k_cache) || !aligned16(v_cache) || ((ldk | ldv) & 7))
    return pifa_fail(PIFA_ERR_ALIGNMENT, "bases must be 16-byte aligned and leading dimensions multiples of 8");
  const PifaSpan out[] = {pifa_span(K, T, row, ldk, 2), pifa_span(V, T, row, ldv, 2)};
  const PifaSpan in[] = {pifa_cache_span(k_cache, c, 1), pifa_cache_span(v_cache, c, 1), pifa_scale_span(k_scale, c, sc),
                         pifa_scale_span(v_scale, c, sc), pifa_span(slots, 1, T, T, 8)};
  bool bad = pifa_rows_overlap(K, row, ldk, V, row, ldv, T);
  for (const PifaSpan& o : out)
    for (const PifaSpan& i : in) bad = bad || pifa_spans_overlap(o, i);
  if (bad) return pifa_fail(PIFA_ERR_INVALID_ARG, "an output overlaps another buffer");
  cudaError_t e = cudaSuccess;
  ReadArgs g = {};
  g.status = pifa_status_word(&e);
  if (!g.status) return pifa_fail_cuda("device status word", e);
  g.kc = static_cast<const uint8_t*>(k_cache);
  g.vc = static_cast<const uint8_t*>(v_cache);
  g.ks = static_cast<const uint8_t*>(k_scale);
  g.vs = static_cast<const uint8_t*>(v_scale);
  g.slots = slots;
  g.k = static_cast<uint16_t*>(K);
  g.v = static_cast<uint16_t*>(V);
  g.ldk = ldk;
  g.ldv = ldv;
  g.n_slots = pages * page_size;
  g.page_stride = page_stride;
  g.token_stride = token_stride;
  g.head_stride = head_stride;
  g.scale_page = scale_page_stride;
  g.scale_block = scale_block_stride;
  g.scale_head = scale_head_stride;
  g.T = (int)T;
  g.page_size = (int)page_size;
  g.hk = (int)kv_heads;
  g.dim = (int)head_dim;
  const int round = 8 * pifa_sm_count();
  g.tokens = (int)T >= round * READ_WINDOW ? READ_WINDOW : ((int)T + round - 1) / round;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr;
  overlap_launches(cfg, attr, cuda_stream);
  cfg.gridDim = dim3((unsigned)((g.T + g.tokens - 1) / g.tokens));
  e = dtype == PIFA_DTYPE_FP16 ? pifa_launch_ex(&cfg, cache_read_q8<true>, g) : pifa_launch_ex(&cfg, cache_read_q8<false>, g);
  if (e != cudaSuccess) return pifa_fail_cuda("cache_read_q8 launch", e);
  return PIFA_OK;
}

}  // extern "C"
