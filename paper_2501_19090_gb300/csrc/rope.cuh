// rope.cuh -- what the rotary kernels share (rope.cu, rope_q8.cu): their arguments and the rotation of whole tokens.
#ifndef PIFA_ROPE_CUH_
#define PIFA_ROPE_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pifa.h"
#include "pifa_internal.h"
#include "ptx.cuh"

namespace {

using namespace pifa;

constexpr int ROPE_THREADS = 256;
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

// Rotates the tokens and heads of CTA (bx, by) and stores them: queries as rows, keys and values in a cache of 16 bits.
template <bool F16, bool HALF>
__device__ __forceinline__ void rope_tokens(const RopeArgs& g, int bx, int by) {
  __shared__ __align__(16) float2 turn[MAX_TOKENS][MAX_DIM / 2];
  __shared__ int64_t place[MAX_TOKENS];  // the token's offset in the cache, -1: not stored
  const int t0 = bx * g.tokens, nt = min(g.tokens, g.T - t0);
  const int pairs = g.rot / 2;
  const int units = g.dim / 16, turned = g.rot / 16;
  const int h0 = by * g.heads, nh = min(g.heads, g.hq + 2 * g.hk - h0), n = nt * nh * units;
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
  for (int i = threadIdx.x; i < nt * pairs; i += ROPE_THREADS) {
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

  for (int i = threadIdx.x; i < n; i += ROPE_THREADS) {
    Unit x = next;
    if (i + ROPE_THREADS < n) fetch(i + ROPE_THREADS);
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

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

#endif  // PIFA_ROPE_CUH_
