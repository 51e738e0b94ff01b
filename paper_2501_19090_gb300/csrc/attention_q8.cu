// attention_q8.cu -- pifa_paged_attention_q8: attention over a paged cache in 8 bits.
//
//   o = sum_j softmax_j(scale q . (s_b k_j)) t_b v_j over the keys j < L - n + i + 1 of new token i (L keys, n new tokens),
//   s_b and t_b the scales of the keys' and the values' block b = j / 16.
//
// Few rows (decode and its neighbours, up to 16 a key / value head) are here; more are attention_tc.cu's. Bound by the cache's bytes, of
// which there are half as many as in 16 bits, so that the instructions a byte count twice: a step of 16 keys, one block of scales,
// costs a warp 8 copies of 16 bytes a lane, 64 conversions of two e4m3 numbers to fp16 (at two cycles each, as all but plain fp32), 16
// permutations that pair V's rows, 32 mma.sync, and as little as possible beside them: pages and scales are looked up for 32 steps
// at once, a lane for each; keys are compared with what a row sees only in steps where some row does not see all; copies have bounds only in
// a request's last step. The scales' part in softmax is in q8.cuh.
// All steps, in the order (request, head, step), are dealt to CTAs in equal runs, a run to the CTA's eight warps; each streams its steps by
// itself. Pieces of heads that fell to several warps are added up in shared memory at the end, those of heads that fell to
// several CTAs by the join.
//
// Measured, head_dim 128, bf16, 64 heads on 8 key / value heads: 64 sequences of 500 to 20000 keys (273 MB) 65 us, 4.2 TB/s; one of 100000
// (205 MB) 47 us, 4.3 TB/s; one of 800000 (1.64 GB) 279 us, 5.9 TB/s. A kernel that only reads takes 43 to 47, 34 to 36 and 229 to
// 256 us for as many bytes. About 5 us are the join, 5 to 7 the start (lengths, table, first copies), the rest SMs that get
// less from memory than others (equal shares of a plain read end between 19 and 30 us). One sequence of 351 keys, 32 heads: 8.3 us.
// Steps: a warp for each row 20.5 and 130 ms (first two cases); pieces of warps, joined by the second kernel 73 and 62 us; pieces added up in
// the CTA 73 and 52; by TMA, scales of 32 steps at a time 69 and 51; copies by the warps' lanes again 65 and 47.
// Not taken: the next step's scores beside this step's weights (71 and 53: a stage less in flight), copies that run over the ends of
// segments (73 and 53: their bookkeeping is in every step).
#include <cmath>

#include "attention_rows.cuh"
#include "q8.cuh"

namespace {

struct RowsQ8 {
  const uint8_t *k, *v, *ks, *vs;
  int64_t scale_page, scale_block, scale_head;
  int whole;  // heads of a CTA; 0: an equal run of steps, wherever heads end
};

template <int D>
constexpr int kStages = 512 / D;  // of 16 keys: 4 KB (D = 128) or 2 KB
constexpr int LEAST = WARPS;      // steps of a CTA (one sequence of 351 keys, 32 heads: 11.7 us, with twice as many 12.4)
// Where a CTA's share of the heads has at most so many keys, going by what the tables have room for, heads are not cut and nothing is
// left to the join. (Measured, cut and whole: 1 sequence of 351 keys, 32 heads 11.7 and 8.3 us; 16 of 1000 to 2000, 8 heads 24.5 and 20.3;
// 64 of 256 to 500, 8 heads 25.5 and 24.7; 64 of 480 to 940, 8 heads, 3840 keys a CTA, 31.3 and 34.6.)
constexpr int WHOLE_KEYS = 2048;

// What a warp has summed up of a head that it did not finish alone: in shared memory, for the CTA to add up.
struct Piece {
  int item, b, from, steps;  // (first step of the head) -1: none
};

// The 16-byte pieces of a key's row lie swizzled (its index xor the row's, in the 128 bytes that eight, or with D = 64 two rows of 64,
// lie in). Which of a product's 16 keys is which of the step's, and which of its columns are a lane's, is free: chosen so that the
// eight lanes that read together meet eight bank groups.
template <int D>
__device__ __forceinline__ int key_of(int n) {  // of a product's key: the step's; D = 128: 0, 4, 1, 5, ... of each eight
  return D == 128 ? (n & 8) | (n >> 1 & 3) | (n & 1) << 2 : n;
}
template <int D>
__device__ __forceinline__ int place(int key, int piece) {
  return D == 128 ? key * 128 + ((piece ^ (key & 7)) << 4) : key * 64 + ((piece ^ (key >> 1 & 3)) << 4);
}

template <bool F16, int D>
__global__ void __launch_bounds__(THREADS, 1)
    attention_rows_q8(const RowArgs g, const RowsQ8 c8) {
  constexpr int KC = D / 64, VC = D / 8;               // of a lane: 16-byte pieces of a key of K; columns of a key of V
  constexpr int PIECES = D / 16, KEYS = 32 / PIECES;   // of a key's row; keys that a warp copies at once
  constexpr int STAGE_BYTES = 2 * STEP * D;            // K and V of a step
  constexpr int STAGES = kStages<D>;
  extern __shared__ __align__(128) uint8_t smem[];
  // of each warp its first head's piece; its last one's takes the place of its stages when those are done
  float* sums = reinterpret_cast<float*>(smem + WARPS * STAGES * STAGE_BYTES);
  int* first = reinterpret_cast<int*>(sums + WARPS * g.max_rows * D);  // B + 1
  static_assert(STAGES * STAGE_BYTES >= MAX_ROWS * D * 4, "a piece fits into a warp's stages");
  __shared__ int part[32];
  __shared__ Piece pieces[2 * WARPS];
  __shared__ float2 ml[2 * WARPS][MAX_ROWS];
  const int lane = threadIdx.x & 31, warp = uniform((int)threadIdx.x >> 5);
  pdl_wait_primary();
  pdl_launch_dependents();  // (after the wait: the join reads the lengths before its own)
  const Run dealt = deal_steps(g, first, part, (int)gridDim.x, LEAST);

  // ---- this CTA's run of steps, this warp's share of it: segments of one request and head each ----
  auto begin_of = [&](int i) {  // this CTA's first step (i = 0), the next one's (1)
    const int64_t k = (int64_t)(blockIdx.x + i) * (c8.whole ? c8.whole : dealt.run);
    if (c8.whole == 0 || dealt.total == 0 || k >= g.B * g.heads) return (int)(c8.whole ? dealt.total : min(k, (int64_t)dealt.total));
    const int b = (int)k / g.heads;
    return first[b] + ((int)k - b * g.heads) * steps_of(lengths_of(g, b));
  };
  const int c0 = begin_of(0), c1 = begin_of(1);
  if (c0 == c1) return;
  const int share = (c1 - c0 + WARPS - 1) / WARPS;
  int at = min(c0 + warp * share, c1);
  const int stop = min(at + share, c1);
  if (lane < 2) pieces[2 * warp + lane].item = -1;
  __syncwarp();
  const int gr = lane >> 2, c4 = lane & 3;
  const uint8_t* ring = smem + warp * STAGES * STAGE_BYTES;
  const uint32_t ring_at = smem_u32(ring);
  const int piece = lane % PIECES, key0 = lane / PIECES;
  while (at < stop) {
    const int b = find(first, g.B, at);
    const Lengths x = lengths_of(g, b);
    const int steps = steps_of(x), head = (at - first[b]) / steps, s0 = at - first[b] - head * steps;
    const int s1 = min(steps, s0 + stop - at);
    const int rows = x.n * g.group;
    const int32_t* pages = g.table + b * g.ldt;
    const int n_pages = (x.L + g.page_size - 1) >> g.page_shift;
    // Lane i holds the place of step i of 32, and what its scales come to: of those that are being loaded and the next, of those
    // that are being computed and the next. A page comes 32 steps, its scales some steps, before what needs them.
    auto page_of = [&](int s) {
      const int p = (s * STEP) >> g.page_shift;
      return s < s1 && p < n_pages ? pages[p] : -1;
    };
    auto scales_of = [&](int s, int id) {
      if (s >= s1 || id < 0 || id >= g.pages) return NO_SCALE << 8 | 127;
      const int64_t from = id * c8.scale_page + ((s * STEP & (g.page_size - 1)) / PIFA_Q8_BLOCK) * c8.scale_block + head * c8.scale_head;
      return (int)c8.ks[from] | (int)c8.vs[from] << 8;
    };
    // where a step's first key of this head lies; -1: in no page
    auto base_of = [&](int s, int id) {
      return id < 0 || id >= g.pages ? (int64_t)-1
                                     : id * g.page_stride + ((s * STEP) & (g.page_size - 1)) * g.token_stride + head * g.head_stride;
    };
    int known = s0, ids_next = page_of(s0 + 32 + lane), scales_next;
    int64_t bases;
    {
      const int id = page_of(s0 + lane);
      bases = base_of(s0 + lane, id);
      scales_next = scales_of(s0 + lane, id);
    }
    // this lane's piece of every KEYS-th key: a warp's copy is whole rows
    const int64_t mine = key0 * g.token_stride + piece * 16;
    auto load = [&](int s, int stage) {
      if (s == known + 32) {
        known = s;
        bases = base_of(s + lane, ids_next);
        scales_next = scales_of(s + lane, ids_next);
        ids_next = page_of(s + 32 + lane);
      }
      const int64_t from = __shfl_sync(0xffffffffu, bases, s - known);
      const uint32_t dst = ring_at + stage * STAGE_BYTES;
      if (from >= 0 && (s + 1) * STEP <= x.L) {
        const uint8_t *k = c8.k + from + mine, *v = c8.v + from + mine;
#pragma unroll
        for (int i = 0; i < STEP / KEYS; ++i) {
          const int at = place<D>(key0 + i * KEYS, piece);
          cp_async16_all(dst + at, k);
          cp_async16_all(dst + STEP * D + at, v);
          k += KEYS * g.token_stride;
          v += KEYS * g.token_stride;
        }
      } else {  // keys past the last one, or of no page: zeros, that nothing is read for
        if (from < 0 && x.L > 0) latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
        const int left = from < 0 ? 0 : x.L - s * STEP;
#pragma unroll
        for (int i = 0; i < STEP / KEYS; ++i) {
          const int key = key0 + i * KEYS;
          const bool in = key < left;
          const int64_t there = in ? from + mine + i * KEYS * g.token_stride : 0;
          cp_async16(dst + place<D>(key, piece), c8.k + there, in ? 16 : 0);
          cp_async16(dst + STEP * D + place<D>(key, piece), c8.v + there, in ? 16 : 0);
        }
      }
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) {
      if (s0 + i < s1) load(s0 + i, i);
      cp_commit();
    }
    // the rows of Q: this lane's are gr and gr + 8; as fp16, times a power of two that brings bf16's into its range
    uint32_t q[2][KC][8];
    int seen[2];
    float c[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int row = gr + 8 * r, token = row / g.group;
      seen[r] = row < rows ? max(x.ahead + token, 0) : 0x7fffffff;
      c[r] = g.c;
#pragma unroll
      for (int i = 0; i < KC; ++i) {
        uint4 w[2] = {};
        if (row < rows) {
          const uint4* from = reinterpret_cast<const uint4*>(g.q + (int64_t)(x.q0 + token) * g.ldq +
                                                             (int64_t)(head * g.group + row - token * g.group) * D + (c4 + 4 * i) * 16);
          w[0] = from[0];
          w[1] = from[1];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) q[r][i][k] = (&w[k / 4].x)[k % 4] ^ g.flip;
      }
      if constexpr (!F16) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < KC; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            most = max3(most, fabsf(__uint_as_float(q[r][i][k] << 16)), fabsf(__uint_as_float(q[r][i][k] & 0xffff0000u)));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int e = row_exponent(most);
        const float up = exponent_of_2(e);
        c[r] *= exponent_of_2(-e);
#pragma unroll
        for (int i = 0; i < KC; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            q[r][i][k] = pack<true>(__uint_as_float(q[r][i][k] << 16) * up, __uint_as_float(q[r][i][k] & 0xffff0000u) * up);
      }
    }
    const int all_see = __reduce_min_sync(0xffffffffu, min(seen[0], seen[1]));  // keys before this are seen by every row
    float o[VC][4] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {};
    float base = NO_BASE;  // exponent that the values' scales are held against
    float key_scales = 0.0f, exponents = 0.0f, inverses = 0.0f;  // of step i of 32
    int scaled = s0 - 32, stage = 0;
    for (int s = s0; s < s1; ++s) {
      __syncwarp();  // all lanes have read the stage that is filled next
      if (s == scaled + 32) {
        scaled = s;
        const int now = scales_next >> 8;
        const float up = raise_base(__reduce_max_sync(0xffffffffu, now < 255 ? now - 127 : -1000), base);
        const ValueScale v = value_scale(now, base);
        key_scales = scale_of(scales_next & 0xff);
        exponents = v.exponent;
        inverses = v.inverse;
        if (up > 0.0f) {  // the sums so far, in units of the larger exponent
          const float f = exponent_of_2(-(int)fminf(up, 126.0f));
#pragma unroll
          for (int i = 0; i < VC; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[i][k] *= f;
        }
      }
      if (s + STAGES - 1 < s1) load(s + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
      cp_commit();
      const float key_scale = __shfl_sync(0xffffffffu, key_scales, s - scaled);
      const float exponent = __shfl_sync(0xffffffffu, exponents, s - scaled);
      const float inverse = __shfl_sync(0xffffffffu, inverses, s - scaled);
      const uint8_t* buf = ring + stage * STAGE_BYTES;
      cp_wait<STAGES - 1>();
      __syncwarp();
      // four sums of products in turn: an MMA's result is some thirty cycles away, and eight in a row would wait for each other
      uint4 kk[KC][2];
#pragma unroll
      for (int i = 0; i < KC; ++i)
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) kk[i][nb] = *reinterpret_cast<const uint4*>(buf + place<D>(key_of<D>(gr + 8 * nb), c4 + 4 * i));
      float part_sc[KC][2][4] = {};
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < KC; ++i)
#pragma unroll
          for (int nb = 0; nb < 2; ++nb) {
            const uint32_t w = (&kk[i][nb].x)[j];
            mma_m16n8k16_f16(part_sc[i][nb], q[0][i][2 * j], q[1][i][2 * j], q[0][i][2 * j + 1], q[1][i][2 * j + 1], halves_of(w & 0xffffu),
                             halves_of(w >> 16));
          }
      // this lane's columns of four keys
      const int group = D == 128 ? (gr >> 1) | (gr & 1) << 2 : gr;
      uint32_t w[4][VC / 4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int key = key_of<D>(c4 * 2 + (k & 1) + 8 * (k >> 1));
        if constexpr (D == 128) {
          const uint4 u = *reinterpret_cast<const uint4*>(buf + STEP * D + place<D>(key, group));
          w[k][0] = u.x, w[k][1] = u.y, w[k][2] = u.z, w[k][3] = u.w;
        } else {
          const uint2 u = *reinterpret_cast<const uint2*>(buf + STEP * D + place<D>(key, group >> 1) + 8 * (group & 1));
          w[k][0] = u.x, w[k][1] = u.y;
        }
      }
      float sc[2][4];
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int k = 0; k < 4; ++k) sc[nb][k] = KC == 2 ? part_sc[0][nb][k] + part_sc[KC - 1][nb][k] : part_sc[0][nb][k];
      // exponents of the weights times their value's scale, relative to m; keys that a row does not see
      float v[2][4];
      bool grows = false;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float cr = c[r] * key_scale;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[r][k] = fmaf(sc[k >> 1][2 * r + (k & 1)], cr, exponent);
      }
      if ((s + 1) * STEP > all_see) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (s * STEP + key_of<D>(8 * (k >> 1) + c4 * 2 + (k & 1)) >= seen[r]) v[r][k] = -INFINITY;
      }
      float top[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        top[r] = max3(v[r][0], v[r][1], fmaxf(v[r][2], v[r][3]));
        grows |= top[r] > m[r] + 8.0f;
      }
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
          top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
          top[r] = fmaxf(top[r], m[r]);
          const float f = top[r] > m[r] ? fast_exp2(m[r] - top[r]) : 1.0f;  // 0 where nothing was seen before
          m[r] = top[r];
          l[r] *= f;
#pragma unroll
          for (int i = 0; i < VC; ++i) {
            o[i][2 * r] *= f;
            o[i][2 * r + 1] *= f;
          }
        }
      }
      uint32_t p[2][2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float from = m[r] > -INFINITY ? m[r] : 0.0f;
        float e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = fast_exp2(v[r][k] - from);
        l[r] = fmaf((e[0] + e[1]) + (e[2] + e[3]), inverse, l[r]);
        p[r][0] = pack<true>(e[0], e[1]);
        p[r][1] = pack<true>(e[2], e[3]);
      }
#pragma unroll
      for (int i = 0; i < VC / 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // columns 4 i + 2 h and the next
          const uint32_t lo = __byte_perm(w[0][i], w[1][i], h ? 0x7362 : 0x5140), hi = __byte_perm(w[2][i], w[3][i], h ? 0x7362 : 0x5140);
          mma_m16n8k16_f16(o[4 * i + 2 * h], p[0][0], p[1][0], p[0][1], p[1][1], halves_of(lo & 0xffffu), halves_of(hi & 0xffffu));
          mma_m16n8k16_f16(o[4 * i + 2 * h + 1], p[0][0], p[1][0], p[0][1], p[1][1], halves_of(lo >> 16), halves_of(hi >> 16));
        }
      stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    cp_wait<0>();
    // o[i][2 r + e]: row gr + 8 r, column VC group(2 c4 + e) + i, in units of 2^base
    const float unit = base > NO_BASE ? exponent_of_2((int)base) : 1.0f;
    const bool alone = s0 == 0 && s1 == steps;
    const int which = 2 * warp + (at + s1 - s0 == stop ? 1 : 0);  // a piece's place: the warp's first, or what it ends with
    float* sum = which & 1 ? reinterpret_cast<float*>(smem + warp * STAGES * STAGE_BYTES) : sums + warp * g.max_rows * D;
    if (!alone) {
      __syncwarp();  // the stages have been read
      if (lane == 0) pieces[which] = {b * g.heads + head, b, first[b] + head * steps, steps};
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      const int row = gr + 8 * r, token = row / g.group;
      if (row >= rows) continue;
      const float inv = !alone ? 1.0f : l[r] == 0.0f ? 0.0f : 1.0f / l[r];
      auto value = [&](int i, int e) { return o[i][2 * r + e] * inv * unit; };
      if (!alone && c4 == 0) ml[which][row] = make_float2(m[r], l[r]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int n = 2 * c4 + e, col = VC * (D == 128 ? (n >> 1) | (n & 1) << 2 : n);
        if (alone) {
          uint16_t* out = g.o + (int64_t)(x.q0 + token) * g.ldo + (int64_t)(head * g.group + row - token * g.group) * D + col;
#pragma unroll
          for (int i = 0; i < VC / 8; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = pack<F16>(value(8 * i + 2 * k, e), value(8 * i + 2 * k + 1, e));
            *reinterpret_cast<uint4*>(out + 8 * i) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < VC / 4; ++i)
            *reinterpret_cast<float4*>(sum + row * D + col + 4 * i) =
                make_float4(value(4 * i, e), value(4 * i + 1, e), value(4 * i + 2, e), value(4 * i + 3, e));
        }
      }
    }
    at += s1 - s0;
  }
  // ---- the CTA's pieces, those of one head added up in the order of the keys; heads of several CTAs are left to the join ----
  __syncthreads();
  for (int k0 = 0; k0 < 2 * WARPS;) {
    const Piece x = pieces[k0];
    int k1 = k0 + 1;
    while (k1 < 2 * WARPS && (pieces[k1].item == x.item || pieces[k1].item < 0)) ++k1;
    if (x.item < 0) {
      ++k0;
      continue;
    }
    const int head = x.item - x.b * g.heads;
    const Lengths len = lengths_of(g, x.b);
    const bool whole = x.from >= c0 && x.from + x.steps <= c1;
    const int rows = len.n * g.group;
    for (int slot = threadIdx.x; slot < rows * (D / 4); slot += THREADS) {
      const int row = slot / (D / 4), col = slot % (D / 4) * 4;
      float top = -INFINITY;
      for (int k = k0; k < k1; ++k)
        if (pieces[k].item >= 0 && ml[k][row].y != 0.0f) top = fmaxf(top, ml[k][row].x);
      float all = 0.0f;
      float4 acc = make_float4(0, 0, 0, 0);
      for (int k = k0; k < k1; ++k) {
        if (pieces[k].item < 0) continue;
        const float2 v = ml[k][row];
        const float e = v.y != 0.0f ? fast_exp2(v.x - top) : 0.0f;
        const float* from = k & 1 ? reinterpret_cast<const float*>(smem + (k >> 1) * STAGES * STAGE_BYTES) : sums + (k >> 1) * g.max_rows * D;
        const float4 o = *reinterpret_cast<const float4*>(from + row * D + col);
        all += v.y * e;
        acc.x += o.x * e;
        acc.y += o.y * e;
        acc.z += o.z * e;
        acc.w += o.w * e;
      }
      if (whole) {
        const float inv = all == 0.0f ? 0.0f : 1.0f / all;
        const int token = row / g.group;
        uint16_t* out = g.o + (int64_t)(len.q0 + token) * g.ldo + (int64_t)(head * g.group + row - token * g.group) * D + col;
        *reinterpret_cast<uint2*>(out) = make_uint2(pack<F16>(acc.x * inv, acc.y * inv), pack<F16>(acc.z * inv, acc.w * inv));
      } else {  // a head that began before this CTA's run: the first of its two places, else the second
        float* to = g.partial + (((int64_t)blockIdx.x * 2 + (x.from < c0 ? 0 : 1)) * g.max_rows + row) * (D + 2);
        if (col == 0) *reinterpret_cast<float2*>(to + D) = make_float2(top, all);
        *reinterpret_cast<float2*>(to + col) = make_float2(acc.x, acc.y);
        *reinterpret_cast<float2*>(to + col + 2) = make_float2(acc.z, acc.w);
      }
    }
    k0 = k1;
  }
}

template <bool F16, int D>
cudaError_t launch_rows_q8(const RowArgs& g, const RowsQ8& c8, cudaStream_t stream) {
  return launch_rows_and_join<F16, D, attention_rows_q8<F16, D>>(g, (size_t)WARPS * (kStages<D> * 2 * STEP * D + g.max_rows * D * 4),
                                                                 c8.whole == 0, stream, c8);
}

}  // namespace

int launch_attention_rows_q8(const PifaAttention& a, int* status, cudaStream_t stream) {
  const RowArgs g = row_args(a, status);
  const int64_t heads = a.B * a.cache.heads, ctas = rows_grid();
  const int64_t share = (heads + ctas - 1) / ctas, whole = share * a.cols * a.cache.page_size <= WHOLE_KEYS ? share : 0;
  const RowsQ8 c8 = {static_cast<const uint8_t*>(a.k), static_cast<const uint8_t*>(a.v), a.q8->k, a.q8->v, a.q8->shape.page_stride,
                     a.q8->shape.block_stride, a.q8->shape.head_stride, (int)whole};
  const bool f16 = a.dtype == PIFA_DTYPE_FP16;
  cudaError_t e;
  if (a.cache.dim == 64) e = f16 ? launch_rows_q8<true, 64>(g, c8, stream) : launch_rows_q8<false, 64>(g, c8, stream);
  else e = f16 ? launch_rows_q8<true, 128>(g, c8, stream) : launch_rows_q8<false, 128>(g, c8, stream);
  return e == cudaSuccess ? PIFA_OK : pifa_fail_cuda("attention_rows_q8 launch", e);
}
