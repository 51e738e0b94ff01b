// attention.cu -- pifa_paged_attention: argument checks, and the kernels for requests with few rows.
//
//   o = sum_j softmax_j(scale q . k_j) v_j over the keys j < L - n + i + 1 of new token i (L keys, n new tokens).
//
// Rows: the query heads of a key / value head share its keys, so the n new tokens of a request and the G heads
// of a group make n G rows, token-major. Up to 16 rows (decode and its neighbours) are one operand of
// mma.sync, which is enough here: the work is bound by the cache's bytes, of which each feeds at most
// 16 rows. More rows go to attention_tc.cu.
//
// Work is cut into steps of 16 keys of one request and one key / value head; all steps, in the order (request,
// head, step), are dealt to warps in equal runs, whatever the requests' lengths: no CTA waits for the
// longest. Each warp streams its steps on its own, without barriers between warps: it copies the 16 keys' rows of K and of V
// (cp.async, whole rows of 128 or 256 bytes, swizzled) into its own three stages of 8 KB: eight warps an SM, up to 128 KB in
// flight. The d elements of q . k may be added in any order and the columns of V assigned to any column of the
// product, which lets every shared-memory read be a 16-byte vector: a lane's pieces of K hold both halves of two
// steps of the contraction, and pairs of V's rows are interleaved in registers.
// One pass with a running maximum m: p = exp2(c s - c m); m is raised, and O and l rescaled, only when a
// score passes it by 8 in the exponent (weights reach 2^8 at most), so most steps exchange nothing between lanes.
// The weights are rounded to the cache's type, which the second product takes them in; l adds them up as they were.
// Outputs are off by 0.0022 of their size in bf16 (fp16 0.00026), by 0.0017 (0.00021) with weights in 32 bits: the rounding
// of the outputs alone. A product of the weights' lower parts as well, half as many MMAs again, was not taken.
// A head whose steps fall to one warp is finished by it; else the warps write (m, l, O) and a second kernel
// adds them up in the order of the keys.
//
// Measured, head_dim 128, bf16: 64 sequences of 400 to 16000 keys, 64 heads on 8 key / value heads (653 MB): 112 to 116 us, 5.6
// to 5.8 TB/s (the measured copy rate is 6.8); the streaming kernel 104 to 110 of it, its SMs between 165 and
// 208 thousand cycles with equal runs, since some are nearer to memory than others. Eight sequences of 1000 to 2600 keys, 32
// heads (169 MB): 36 us, 31 of it streaming. One of 300 keys, 32 heads: 10 us, latency. Copies of 16 bytes from
// eight rows at a time, which need no exchange between lanes, took 140 and 41 us: 28 bytes a request to L2, not 120.
#include <cmath>

#include "attention_rows.cuh"

namespace {

template <int D>
constexpr int kStages = 384 / D;     // of 16 keys: 8 KB (D = 128) or 4 KB

// Where a 16-byte piece of a key's row lies in shared memory: its index xor this, so that the eight lanes of a
// quarter warp, which read two keys' four neighbouring pieces of K, or two pieces of every other key of V, meet
// eight different bank groups.
__device__ __forceinline__ int k_swizzle(int key) { return (key & 1) << 2; }
__device__ __forceinline__ int v_swizzle(int key) { return key & 6; }

template <bool F16, int D>
__global__ void __launch_bounds__(THREADS, 1) attention_rows(const RowArgs g) {
  constexpr int KC = D / 32, VC = D / 64;            // 16-byte pieces of a lane: of one key, of one key of V
  constexpr int ROW = 2 * D, KEYS = 32 / (ROW / 16);   // bytes of a key's row; keys that a warp copies at once
  constexpr int STAGE_BYTES = 2 * STEP * ROW;        // K and V of a step
  constexpr int STAGES = kStages<D>;
  extern __shared__ __align__(16) uint8_t smem[];
  int* first = reinterpret_cast<int*>(smem + WARPS * STAGES * STAGE_BYTES);  // B + 1
  __shared__ int part[32];
  pdl_wait_primary();
  pdl_launch_dependents();  // (after the wait: the join reads the lengths before its own)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Run steps_here = deal_steps(g, first, part, (int)gridDim.x * WARPS, MIN_STEPS, [](int, const Lengths&) {});
  const int total = steps_here.total, run = steps_here.run;
  if (blockIdx.x == 0) {  // written down for the join
    for (int b = (int)threadIdx.x; b <= g.B; b += THREADS) g.sums[b] = first[b];
    if (threadIdx.x == 0) g.sums[g.B + 1] = total == 0 ? 0 : run;
  }

  // ---- this warp's run of steps: segments of one request and head each ----
  const int worker = warp * (int)gridDim.x + (int)blockIdx.x;  // neighbours on different SMs
  const int64_t at64 = (int64_t)worker * run;
  int at = (int)min(at64, (int64_t)total);
  const int stop = (int)min(at64 + run, (int64_t)total);
  const int gr = lane >> 2, c4 = lane & 3;
  const uint8_t* ring = smem + warp * STAGES * STAGE_BYTES;
  const uint32_t ring_at = smem_u32(ring);
  const int piece = lane % (ROW / 16), key0 = lane / (ROW / 16);
  while (at < stop) {
    const int b = find(first, g.B, at);
    const Lengths x = lengths_of(g, b);
    const int steps = steps_of(x), head = (at - first[b]) / steps, s0 = at - first[b] - head * steps;
    const int s1 = segment_end(steps, s0, at, stop);
    const int rows = x.n * g.group;
    // the rows of Q: this lane's are gr and gr + 8
    uint4 q[2][KC];
    int seen[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int row = gr + 8 * r, token = row / g.group;
      seen[r] = row < rows ? max(x.ahead + token, 0) : 0;
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        q[r][i] = make_uint4(0, 0, 0, 0);
        if (row < rows) {
          q[r][i] = *reinterpret_cast<const uint4*>(g.q + (int64_t)(x.q0 + token) * g.ldq +
                                                    (int64_t)(head * g.group + row - token * g.group) * D + c4 * 8 + 32 * i);
          q[r][i].x ^= g.flip;
          q[r][i].y ^= g.flip;
          q[r][i].z ^= g.flip;
          q[r][i].w ^= g.flip;
        }
      }
    }
    const int32_t* pages = g.table + b * g.ldt;
    const int n_pages = (x.L + g.page_size - 1) >> g.page_shift;
    int known = -1, ids = 0;  // ids: lane i holds the page of step known + i
    auto load = [&](int s, int stage) {  // K, then V, as two groups; nothing past s1
      if (s < s1) {
        if (known < 0 || s >= known + 32) {
          known = s;
          const int p = ((s + lane) * STEP) >> g.page_shift;
          ids = s + lane < s1 && p < n_pages ? pages[p] : 0;
        }
        const int id = __shfl_sync(0xffffffffu, ids, s - known);
        const bool bad = id < 0 || id >= g.pages;
        if (bad && x.L > 0) latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
        // this lane's piece of every KEYS-th key: a warp's copy is whole rows
        const int64_t at = (bad ? 0 : (int64_t)id) * g.page_stride + head * g.head_stride +
                           (((s * STEP) & (g.page_size - 1)) + key0) * g.token_stride + piece * 8;
        const int left = bad ? 0 : x.L - s * STEP - key0;  // keys from this lane's first on
        const uint32_t dst = ring_at + stage * STAGE_BYTES + key0 * ROW;
#pragma unroll
        for (int i = 0; i < STEP / KEYS; ++i) {
          const bool in = i * KEYS < left;
          cp_async16(dst + i * KEYS * ROW + ((piece ^ k_swizzle(key0 + i * KEYS)) << 4),
                     g.k + at + (in ? i * KEYS * g.token_stride : 0) - (left > 0 ? 0 : key0 * g.token_stride), in ? 16 : 0);
        }
        cp_commit();
#pragma unroll
        for (int i = 0; i < STEP / KEYS; ++i) {
          const bool in = i * KEYS < left;
          cp_async16(dst + STEP * ROW + i * KEYS * ROW + ((piece ^ v_swizzle(key0 + i * KEYS)) << 4),
                     g.v + at + (in ? i * KEYS * g.token_stride : 0) - (left > 0 ? 0 : key0 * g.token_stride), in ? 16 : 0);
        }
      } else {
        cp_commit();
      }
      cp_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) load(s0 + i, i);
    float o[VC * 8][4] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {};
    int stage = 0;
    for (int s = s0; s < s1; ++s) {
      __syncwarp();  // all lanes have read the stage that is filled next
      load(s + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
      const uint8_t* buf = ring + stage * STAGE_BYTES;
      cp_wait<2 * STAGES - 1>();
      __syncwarp();
      float sc[2][4] = {};
#pragma unroll
      for (int i = 0; i < KC; ++i)
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) {
          const uint4 k = *reinterpret_cast<const uint4*>(buf + (gr + 8 * nb) * ROW + (((c4 + 4 * i) ^ k_swizzle(gr)) << 4));
          mma<F16>(sc[nb], q[0][i].x, q[1][i].x, q[0][i].y, q[1][i].y, k.x, k.y);
          mma<F16>(sc[nb], q[0][i].z, q[1][i].z, q[0][i].w, q[1][i].w, k.z, k.w);
        }
      // keys that a row does not see; scores relative to m
      float v[2][4];
      bool grows = false;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int key = s * STEP + 8 * (k >> 1) + c4 * 2 + (k & 1);
          v[r][k] = key < seen[r] ? sc[k >> 1][2 * r + (k & 1)] * g.c : -INFINITY;
          grows |= v[r][k] > m[r] + 8.0f;
        }
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float top = fmaxf(fmaxf(v[r][0], v[r][1]), fmaxf(v[r][2], v[r][3]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          top = fmaxf(top, m[r]);
          const float f = top > m[r] ? fast_exp2(m[r] - top) : 1.0f;  // 0 where nothing was seen before
          m[r] = top;
          l[r] *= f;
#pragma unroll
          for (int i = 0; i < VC * 8; ++i) {
            o[i][2 * r] *= f;
            o[i][2 * r + 1] *= f;
          }
        }
      }
      uint32_t p[2][2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float base = m[r] > -INFINITY ? m[r] : 0.0f;
        float e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = fast_exp2(v[r][k] - base);
        l[r] += (e[0] + e[1]) + (e[2] + e[3]);
        p[r][0] = pack<F16>(e[0], e[1]);
        p[r][1] = pack<F16>(e[2], e[3]);
      }
      cp_wait<2 * STAGES - 2>();
      __syncwarp();
#pragma unroll
      for (int h = 0; h < VC; ++h) {
        uint4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int key = c4 * 2 + (k & 1) + 8 * (k >> 1);
          w[k] = *reinterpret_cast<const uint4*>(buf + (STEP + key) * ROW + (((8 * h + gr) ^ v_swizzle(key)) << 4));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // columns 2 i and 2 i + 1 of the lane's eight
          const uint32_t a = (&w[0].x)[i], bb = (&w[1].x)[i], cc = (&w[2].x)[i], dd = (&w[3].x)[i];
          mma<F16>(o[h * 8 + 2 * i], p[0][0], p[1][0], p[0][1], p[1][1], __byte_perm(a, bb, 0x5410), __byte_perm(cc, dd, 0x5410));
          mma<F16>(o[h * 8 + 2 * i + 1], p[0][0], p[1][0], p[0][1], p[1][1], __byte_perm(a, bb, 0x7632), __byte_perm(cc, dd, 0x7632));
        }
      }
      stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    cp_wait<0>();
    // o[h 8 + i][2 r + e]: row gr + 8 r, column 64 h + 16 c4 + 8 e + i
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      const int row = gr + 8 * r, token = row / g.group;
      if (row >= rows) continue;
      if (s0 == 0 && s1 == steps) {
        const float inv = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
        uint16_t* out = g.o + (int64_t)(x.q0 + token) * g.ldo + (int64_t)(head * g.group + row - token * g.group) * D + c4 * 16;
#pragma unroll
        for (int h = 0; h < VC; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack<F16>(o[h * 8 + 2 * i][2 * r + e] * inv, o[h * 8 + 2 * i + 1][2 * r + e] * inv);
            *reinterpret_cast<uint4*>(out + 64 * h + 8 * e) = make_uint4(w[0], w[1], w[2], w[3]);
          }
      } else {  // a head that began before this run: the first of the warp's two places, else the second
        float* to = g.partial + (((int64_t)worker * 2 + (s0 > 0 ? 0 : 1)) * g.max_rows + row) * (D + 2);
        float2* ml = reinterpret_cast<float2*>(to + D);
        if (c4 == 0) *ml = make_float2(m[r], l[r]);
#pragma unroll
        for (int h = 0; h < VC; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<float2*>(to + 64 * h + 16 * c4 + 8 * e + 2 * i) =
                  make_float2(o[h * 8 + 2 * i][2 * r + e], o[h * 8 + 2 * i + 1][2 * r + e]);
      }
    }
    at += s1 - s0;
  }
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

template <bool F16, int D>
cudaError_t launch_rows_and_join(const RowArgs& g, cudaStream_t stream) {
  const cudaError_t e =
      launch_rows<attention_rows<F16, D>>(rows_grid(), (size_t)WARPS * kStages<D> * 2 * STEP * 2 * D + first_bytes(g), stream, g);
  if (e != cudaSuccess) return e;
  const int64_t items = (int64_t)g.B * g.heads;
  int split = 1;
  while (split < 16 && items * split * 2 <= 8 * pifa_sm_count() && g.max_rows * (D / 4) / (split * 2) >= THREADS / 16) split *= 2;
  return launch_rows<attention_join<F16, D>>(items * split, 0, stream, g, split);
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

// Whether a cache in 8 bits is brought to 16 before a call on the tensor cores, given the room: where a head's rows may make several
// items, and the room, for the most keys that the tables can hold, is at most a gigabyte.
constexpr int64_t WIDE_ROWS_FROM = 768, WIDE_BYTES = (int64_t)1 << 30;
bool widens(int64_t group, int64_t kv_heads, int64_t dim, int64_t B, int64_t max_q, int64_t keys) {
  return keys > 0 && group * max_q > WIDE_ROWS_FROM && attention_wide_bytes(kv_heads, dim, B, keys) <= WIDE_BYTES;
}

// Whether a request's rows for one key / value head may be more than one 16-row product.
bool takes_tc(int64_t group, int64_t max_q) { return max_q > MAX_ROWS || group * max_q > MAX_ROWS; }

int64_t rows_workspace_bytes(int64_t max_rows, int64_t dim, int64_t B) {
  return sums_bytes(B) + (int64_t)MAX_CTAS * WARPS * 2 * max_rows * (dim + 2) * 4;
}

// Both forms of the cache; q8: the scales of one in 8 bits, else null.
int attend(const void* Q, int64_t ldq, int64_t T, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int dtype,
           const void* k_cache, const void* v_cache, const PifaScales* q8, int64_t pages, int64_t page_size, int64_t page_stride,
           int64_t token_stride, int64_t head_stride, const int32_t* table, int64_t cols, int64_t ldt, const int32_t* q_start,
           const int32_t* kv_len, int64_t B, int64_t max_q, float scale, void* O, int64_t ldo, void* workspace,
           int64_t workspace_bytes, void* cuda_stream) {
  pifa_clear_error();
  const int64_t need = pifa_paged_attention_workspace_size(T, q_heads, kv_heads, head_dim, B, max_q);
  if (need < 0) return (int)need;
  if (dtype != PIFA_DTYPE_BF16 && dtype != PIFA_DTYPE_FP16) return pifa_fail(PIFA_ERR_INVALID_ARG, "unknown dtype");
  const PifaCacheShape c = {pages, page_size, kv_heads, head_dim, page_stride, token_stride, head_stride};
  int st = q8 ? pifa_check_cache_q8(c, q8->shape, 256) : pifa_check_cache(c, 16, 256);
  if (st != PIFA_OK) return st;
  if (page_size & (page_size - 1)) return pifa_fail(PIFA_ERR_UNSUPPORTED, "attention takes a page_size that is a power of two");
  const int64_t lim = (int64_t)1 << 30;
  if (cols < 0 || cols >= lim || cols * page_size > lim || ldt < cols || !(std::fabs(scale) <= 1e30f))
    return pifa_fail(PIFA_ERR_INVALID_ARG, "cols, ldt or scale out of range");
  if (B * kv_heads * (cols * page_size / STEP + 1) >= 2 * lim)
    return pifa_fail(PIFA_ERR_UNSUPPORTED, "attention takes at most 2^35 keys, over all requests and heads, in the tables");
  if (T == 0 || B == 0) return PIFA_OK;
  if (!Q || !k_cache || !v_cache || !O || !q_start || !kv_len || (cols && !table) || (q8 && (!q8->k || !q8->v)))
    return pifa_fail(PIFA_ERR_INVALID_ARG, "null argument");
  const int64_t row = q_heads * head_dim;
  if (ldq < row || ldo < row) return pifa_fail(PIFA_ERR_INVALID_ARG, "leading dimension smaller than the row length");
  if (!aligned16(Q) || !aligned16(O) || !aligned16(k_cache) || !aligned16(v_cache) || ((ldq | ldo) & 7))
    return pifa_fail(PIFA_ERR_ALIGNMENT, "bases must be 16-byte aligned and leading dimensions multiples of 8");
  if (!workspace || workspace_bytes < need)
    return pifa_fail(PIFA_ERR_WORKSPACE, "workspace missing or smaller than pifa_paged_attention_workspace_size()");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u)
    return pifa_fail(PIFA_ERR_ALIGNMENT, "workspace must be 256-byte aligned");
  const bool tc = takes_tc(q_heads / kv_heads, max_q);
  const int64_t room = q8 && tc && widens(q_heads / kv_heads, kv_heads, head_dim, B, max_q, cols * page_size)
                           ? need + attention_wide_bytes(kv_heads, head_dim, B, cols * page_size) : need;
  const bool wide = room > need && workspace_bytes >= room;
  const int64_t used = wide ? room : need;
  const PifaSpan o = pifa_span(O, T, row, ldo, 2), ws = pifa_span(workspace, 1, used, used, 1);
  const int64_t elem = q8 ? 1 : 2;
  const PifaSpan none = {0, 0};
  const PifaSpan in[] = {pifa_span(Q, T, row, ldq, 2), pifa_cache_span(k_cache, c, elem), pifa_cache_span(v_cache, c, elem),
                         pifa_span(table, B, cols, ldt, 4), pifa_span(q_start, 1, B + 1, B + 1, 4),
                         pifa_span(kv_len, 1, B, B, 4), q8 ? pifa_scale_span(q8->k, c, q8->shape) : none,
                         q8 ? pifa_scale_span(q8->v, c, q8->shape) : none};
  bool bad = pifa_spans_overlap(o, ws);
  for (const PifaSpan& x : in) bad = bad || pifa_spans_overlap(o, x) || pifa_spans_overlap(ws, x);
  if (bad) return pifa_fail(PIFA_ERR_INVALID_ARG, "O or workspace overlaps another buffer");
  cudaError_t e = cudaSuccess;
  int* status = pifa_status_word(&e);
  if (!status) return pifa_fail_cuda("device status word", e);
  const PifaAttention a = {Q, k_cache, v_cache, O, table, q_start, kv_len, T, ldq, ldo, ldt, cols, B, max_q, q_heads, c, dtype,
                           scale * 1.4426950408889634f, static_cast<uint8_t*>(workspace) + kWorkspaceReserve, q8};
  if (tc) return launch_attention_tc(a, wide, status, pifa_wait_timeout_ns(), reinterpret_cast<cudaStream_t>(cuda_stream));
  if (q8) return launch_attention_rows_q8(a, status, reinterpret_cast<cudaStream_t>(cuda_stream));
  RowArgs g = row_args(a, status);
  g.k = static_cast<const uint16_t*>(k_cache);
  g.v = static_cast<const uint16_t*>(v_cache);
  const bool f16 = dtype == PIFA_DTYPE_FP16;
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (head_dim == 64) e = f16 ? launch_rows_and_join<true, 64>(g, stream) : launch_rows_and_join<false, 64>(g, stream);
  else e = f16 ? launch_rows_and_join<true, 128>(g, stream) : launch_rows_and_join<false, 128>(g, stream);
  if (e != cudaSuccess) return pifa_fail_cuda("attention launch", e);
  return PIFA_OK;
}

}  // namespace

extern "C" {

int64_t pifa_paged_attention_workspace_size(int64_t T, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t B,
                                            int64_t max_q) {
  pifa_clear_error();
  const int st = check_sizes(T, q_heads, kv_heads, head_dim, B, max_q);
  if (st != PIFA_OK) return st;
  if (T == 0 || B == 0) return 0;
  const int64_t group = q_heads / kv_heads;
  return kWorkspaceReserve + (takes_tc(group, max_q) ? attention_tc_workspace_bytes(T, q_heads, kv_heads, head_dim, B)
                                                     : rows_workspace_bytes(group * max_q, head_dim, B));
}

int64_t pifa_paged_attention_q8_workspace_size(int64_t T, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t B,
                                               int64_t max_q, int64_t cols, int64_t page_size) {
  const int64_t need = pifa_paged_attention_workspace_size(T, q_heads, kv_heads, head_dim, B, max_q);
  if (need <= 0) return need;
  const int64_t lim = (int64_t)1 << 30;
  if (cols < 0 || cols >= lim || page_size < 1 || page_size > 256 || cols * page_size > lim)
    return pifa_fail(PIFA_ERR_INVALID_ARG, "cols or page_size out of range");
  const int64_t group = q_heads / kv_heads, keys = cols * page_size;
  return need + (takes_tc(group, max_q) && widens(group, kv_heads, head_dim, B, max_q, keys)
                     ? attention_wide_bytes(kv_heads, head_dim, B, keys) : 0);
}

int pifa_paged_attention(const void* Q, int64_t ldq, int64_t T, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                         int dtype, const void* k_cache, const void* v_cache, int64_t pages, int64_t page_size,
                         int64_t page_stride, int64_t token_stride, int64_t head_stride, const int32_t* table,
                         int64_t cols, int64_t ldt, const int32_t* q_start, const int32_t* kv_len, int64_t B,
                         int64_t max_q, float scale, void* O, int64_t ldo, void* workspace, int64_t workspace_bytes,
                         void* cuda_stream) {
  return attend(Q, ldq, T, q_heads, kv_heads, head_dim, dtype, k_cache, v_cache, nullptr, pages, page_size, page_stride, token_stride,
                head_stride, table, cols, ldt, q_start, kv_len, B, max_q, scale, O, ldo, workspace, workspace_bytes, cuda_stream);
}

int pifa_paged_attention_q8(const void* Q, int64_t ldq, int64_t T, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                            int dtype, const void* k_cache, const void* v_cache, const void* k_scale, const void* v_scale,
                            int64_t pages, int64_t page_size, int64_t page_stride, int64_t token_stride, int64_t head_stride,
                            int64_t scale_page_stride, int64_t scale_block_stride, int64_t scale_head_stride,
                            const int32_t* table, int64_t cols, int64_t ldt, const int32_t* q_start, const int32_t* kv_len,
                            int64_t B, int64_t max_q, float scale, void* O, int64_t ldo, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream) {
  const PifaScales q8 = {static_cast<const uint8_t*>(k_scale), static_cast<const uint8_t*>(v_scale),
                         {scale_page_stride, scale_block_stride, scale_head_stride}};
  return attend(Q, ldq, T, q_heads, kv_heads, head_dim, dtype, k_cache, v_cache, &q8, pages, page_size, page_stride, token_stride,
                head_stride, table, cols, ldt, q_start, kv_len, B, max_q, scale, O, ldo, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
