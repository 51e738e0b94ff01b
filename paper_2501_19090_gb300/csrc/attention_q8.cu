// attention_q8.cu -- pifa_paged_attention_q8: attention over a paged cache in 8 bits.
//
//   o = sum_j softmax_j(scale q . (s_b k_j)) t_b v_j over the keys j < L - n + i + 1 of new token i (L keys, n new tokens),
//   s_b and t_b the scales of the keys' and the values' block b = j / 16.
//
// Few rows (decode and its neighbours, up to 16 a key / value head) are here; more are attention_tc.cu's. Bound by the cache's bytes, of
// which there are half as many as in 16 bits, so that the instructions a byte count twice: a step of 16 keys, one block of scales,
// costs a warp 8 copies of 16 bytes a lane, 64 conversions of two e4m3 numbers to fp16 (at two cycles each, as all but plain fp32), 16
// permutations that pair V's rows, 16 mma.sync (up to 8 rows, SLIM: they are the second operand's 8 columns, K's keys and V's columns
// the first operand's 16 rows; with 9 to 16 rows, the first operand's, 32), and as little as possible beside them: pages and scales are looked
// up for 32 steps at once, a lane for each; keys are compared with what a row sees only in steps where some row does not see all; copies
// have bounds only in a request's last step. The scales' part in softmax is in q8.cuh.
// All steps, in the order (request, head, step), are dealt to CTAs in equal runs, a run to the CTA's eight warps; each streams its steps by
// itself. Pieces of heads that fell to several warps are added up in shared memory at the end, those of heads that fell to
// several CTAs by the join.
//
// Measured, head_dim 128, bf16, 64 heads on 8 key / value heads: 64 sequences of 500 to 20000 keys (273 MB) 58 to 62 us, 4.4 to 4.7
// TB/s; one of 100000 (205 MB) 40 us, 5.1 TB/s; one of 800000 (1.64 GB) 254 us, 6.5 TB/s. A kernel that only reads takes 43 to 47, 34 to
// 36 and 229 to 256 us for as many bytes. One sequence of 351 keys, 32 heads: 6.4 us; in a table with room for 32768, its heads cut, 7.1.
// 9 to 16 rows: 64 heads on 4, 100000 keys (102 MB), 28.5 us, where 8 rows take 26.3; 2 new tokens of 64 sequences (1.15 GB) 205, where one takes 192;
// head_dim 64, 64 heads on 4, 100000 keys 22.5 and 19.7. Between the first data and the last, memory is the bound (100000
// keys: 7.4 TB/s); before it are 9 to 10 thousand cycles of lengths, dealing, table, first copies, mostly their latencies and first fetches of
// code, behind it 4 to 5 thousand of adding up, and the join, 2.5 us.
// Steps (first two cases): a warp for each row 20.5 and 130 ms; pieces of warps, joined by the second kernel 73 and 62 us; pieces added up in
// the CTA 73 and 52; by TMA, scales of 32 steps at a time 69 and 51; copies by the warps' lanes again 65 and 47; four sums of products in turn
// and places of 32 steps 65 and 45; SLIM 63.8 and 44.0; a join of cut heads only 61.9 and 42.3; pieces added up by all warps without lengths,
// Q asked for before the copies 61.4 and 40.5.
// Not taken: the next step's scores beside this step's weights (71 and 53: a stage less in flight), copies that run over the ends of
// segments (73 and 53: their bookkeeping is in every step), 12 warps of three stages or 10 of four (67.4 and 45.5, 69.6 and 49.0), five stages (66.1
// and 45.6), a CTA's warps on neighbouring heads of the same tokens (46.2 for the second: DRAM's pages are not the bound).
#include <algorithm>
#include <cmath>

#include "attention_rows.cuh"
#include "q8.cuh"

namespace {

struct RowsQ8 {
  const uint8_t *k, *v, *ks, *vs;
  int64_t scale_page, scale_block, scale_head;
  int whole;  // heads of a CTA; 0: an equal run of steps, wherever heads end
  int4* cuts; // for each CTA, of the head that its run ends within: first row of Q, rows, its first and last CTA in 16 bits each, 1 + head
};
// Of partial sums a CTA has two places, for the head that began before its run and for the one that goes on behind it: of each row D
// numbers, then of each row m and l, each place a multiple of 16 bytes. (The workspace has them for eight times as many.)
template <int D>
__host__ __device__ constexpr int64_t place_floats(int64_t max_rows) { return max_rows * (D + 4); }

// One more piece of a row's sums: (m, l, four of O); l = 0: of no keys.
__device__ __forceinline__ void add_piece(float& top, float& all, float4& acc, float2 ml, float4 o) {
  const float most = ml.y != 0.0f ? fmaxf(top, ml.x) : top;
  const float f = top > -INFINITY ? fast_exp2(top - most) : 0.0f, e = ml.y != 0.0f ? fast_exp2(ml.x - most) : 0.0f;
  top = most;
  all = fmaf(all, f, ml.y * e);
  acc.x = fmaf(acc.x, f, o.x * e);
  acc.y = fmaf(acc.y, f, o.y * e);
  acc.z = fmaf(acc.z, f, o.z * e);
  acc.w = fmaf(acc.w, f, o.w * e);
}

template <int D>
constexpr int kStages = 512 / D;  // of 16 keys: 4 KB (D = 128) or 2 KB
constexpr int LEAST = WARPS;      // steps of a CTA (one sequence of 351 keys, 32 heads: 11.7 us, with twice as many 12.4)
// Heads are not cut, and nothing is left to the join, where that gives no CTA much more than its equal share, going by what the tables
// have room for: at most so many keys more, and no more in all than where requests shorter than the room, whose CTAs then wait
// for the others', cost more than the join. (Measured, cut and whole: 1 sequence of 300 keys, 32 heads, 9.6 and 8.3 us; of 700 10.0 and 10.3;
// of 2000 13.0 and 15.7; 18 sequences, 8 heads, of 700 15.4 and 11.3; of 500 to 2000 16.1 and 14.8; of 1000 to 4000 21.5 and 22.2. More heads than
// CTAs: 40 sequences, 8 heads, of 300 16.0 and 15.2, of 175 to 700 17.3 and 18.7.)
constexpr int WHOLE_MORE = 768, WHOLE_KEYS_ONE = 2048, WHOLE_KEYS = 1024;

// Lengths of so many requests are kept in shared memory (a look at them in memory takes 730 cycles each time).
constexpr int KEPT = 512;

// What a warp has summed up of a head that it did not finish alone: in shared memory, for the CTA to add up.
struct Piece {
  int from, steps, q0, rows, head;  // the head's first step and its steps; its first row of Q and its rows (0: no piece)
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

template <bool F16, int D, bool SLIM>
__global__ void __launch_bounds__(THREADS, 1) attention_rows_q8(const RowArgs g, const RowsQ8 c8) {
  constexpr int ROWS = SLIM ? 8 : MAX_ROWS;
  constexpr int KC = D / 64, VC = D / 8;               // of a lane: 16-byte pieces of a key of K; columns of a key of V
  constexpr int PIECES = D / 16, KEYS = 32 / PIECES;   // of a key's row; keys that a warp copies at once
  constexpr int STAGE_BYTES = 2 * STEP * D;            // K and V of a step
  constexpr int STAGES = kStages<D>;
  extern __shared__ __align__(128) uint8_t smem[];
  // of each warp its first head's piece; its last one's takes the place of its stages when those are done
  float* sums = reinterpret_cast<float*>(smem + WARPS * STAGES * STAGE_BYTES);
  static_assert(STAGES * STAGE_BYTES >= ROWS * D * 4, "a piece fits into a warp's stages");
  Lengths* kept = reinterpret_cast<Lengths*>(sums + WARPS * g.max_rows * D);
  int* first = reinterpret_cast<int*>(kept + min(g.B, KEPT));  // B + 1
  __shared__ int part[32];
  __shared__ Piece pieces[2 * WARPS];
  __shared__ float2 ml[2 * WARPS][ROWS];
  const int lane = threadIdx.x & 31, warp = uniform((int)threadIdx.x >> 5);
  pdl_wait_primary();
  pdl_launch_dependents();  // (the join's CTAs begin beside these, and wait for their end)
  const Run dealt = deal_steps(g, first, part, (int)gridDim.x, LEAST, [&](int b, const Lengths& x) {
    if (b < KEPT) kept[b] = x;
  });
  auto lengths = [&](int b) { return b < KEPT ? kept[b] : lengths_of(g, b); };

  // ---- this CTA's run of steps, this warp's share of it: segments of one request and head each ----
  auto begin_of = [&](uint32_t cta) {  // a CTA's first step
    if (c8.whole == 0) return (int)min(cta * (uint32_t)dealt.run, (uint32_t)dealt.total);
    const uint32_t k = cta * (uint32_t)c8.whole, b = k / (uint32_t)g.heads;
    return b >= (uint32_t)g.B || dealt.total == 0 ? dealt.total : first[b] + (int)(k - b * g.heads) * steps_of(lengths(b));
  };
  const int c0 = begin_of(blockIdx.x), c1 = begin_of(blockIdx.x + 1);
  if (threadIdx.x == 0 && c8.whole == 0) c8.cuts[blockIdx.x] = make_int4(0, 0, 0, 0);
  if (c0 == c1) return;
  const uint32_t share = (uint32_t)(c1 - c0 + WARPS - 1) / WARPS;  // (c1 may be close to 2^31)
  int at = (int)min((uint32_t)c0 + warp * share, (uint32_t)c1);
  const int stop = (int)min((uint32_t)at + share, (uint32_t)c1);
  if (lane < 2) pieces[2 * warp + lane].rows = 0;
  __syncwarp();
  const int gr = lane >> 2, c4 = lane & 3;
  const uint8_t* ring = smem + warp * STAGES * STAGE_BYTES;
  const uint32_t ring_at = smem_u32(ring);
  const int piece = lane % PIECES, key0 = lane / PIECES;
  while (at < stop) {
    const int b = find(first, g.B, at);
    const Lengths x = lengths(b);
    const int steps = steps_of(x), head = (int)((uint32_t)(at - first[b]) / (uint32_t)steps), s0 = at - first[b] - head * steps;
    const int s1 = segment_end(steps, s0, at, stop);
    const int rows = x.n * g.group;
    // The rows of Q: this lane's are gr (and gr + 8; SLIM: of the products' results, 2 c4 and 2 c4 + 1). Asked for before the copies, whose
    // queue is some thousand cycles long when all SMs begin.
    constexpr int QR = SLIM ? 1 : 2;
    uint32_t q[QR][KC][8];
#pragma unroll
    for (int r = 0; r < QR; ++r) {
      const int row = gr + 8 * r, token = row / g.group;
      const uint4* from = reinterpret_cast<const uint4*>(g.q + (int64_t)(x.q0 + token) * g.ldq +
                                                         (int64_t)(head * g.group + row - token * g.group) * D + c4 * 16);
#pragma unroll
      for (int i = 0; i < KC; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint4 w = row < rows ? from[8 * i + k] : make_uint4(0, 0, 0, 0);
          q[r][i][4 * k] = w.x;
          q[r][i][4 * k + 1] = w.y;
          q[r][i][4 * k + 2] = w.z;
          q[r][i][4 * k + 3] = w.w;
        }
    }
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
    // Q as fp16, times a power of two that brings bf16's rows into its range
    int seen[2];
    float c[2] = {g.c, g.c};
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int row = SLIM ? 2 * c4 + r : gr + 8 * r;
      seen[r] = row < rows ? max(x.ahead + row / g.group, 0) : 0x7fffffff;
    }
#pragma unroll
    for (int r = 0; r < QR; ++r) {
#pragma unroll
      for (int i = 0; i < KC; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) q[r][i][k] ^= g.flip;
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
        const float up = exponent_of_2(e), down = exponent_of_2(-e);
        if (SLIM) {
          c[0] *= __shfl_sync(0xffffffffu, down, 8 * c4);
          c[1] *= __shfl_sync(0xffffffffu, down, 8 * c4 + 4);
        } else {
          c[r] *= down;
        }
#pragma unroll
        for (int i = 0; i < KC; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            q[r][i][k] = pack<true>(__uint_as_float(q[r][i][k] << 16) * up, __uint_as_float(q[r][i][k] & 0xffff0000u) * up);
      }
    }
    const int all_see = __reduce_min_sync(0xffffffffu, min(seen[0], seen[1]));  // keys before this are seen by every row
    constexpr int OUT = SLIM ? VC / 2 : VC;
    float o[OUT][4] = {};
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
          for (int i = 0; i < OUT; ++i)
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
      float sums_qk[2][2][4] = {};
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < KC; ++i) {
          const uint32_t w0 = (&kk[i][0].x)[j], w1 = (&kk[i][1].x)[j];
          const uint32_t a = halves_of(w0 & 0xffffu), b2 = halves_of(w0 >> 16), a8 = halves_of(w1 & 0xffffu), b8 = halves_of(w1 >> 16);
          if constexpr (SLIM) {  // keys gr and gr + 8 by rows 2 c4 and 2 c4 + 1
            mma_m16n8k16_f16(sums_qk[KC == 2 ? i : j & 1][KC == 2 ? j & 1 : 0], a, a8, b2, b8, q[0][i][2 * j], q[0][i][2 * j + 1]);
          } else {               // rows gr and gr + 8 by keys 2 c4 and 2 c4 + 1 (and 8 more)
            mma_m16n8k16_f16(sums_qk[i][0], q[0][i][2 * j], q[QR - 1][i][2 * j], q[0][i][2 * j + 1], q[QR - 1][i][2 * j + 1], a, b2);
            mma_m16n8k16_f16(sums_qk[i][1], q[0][i][2 * j], q[QR - 1][i][2 * j], q[0][i][2 * j + 1], q[QR - 1][i][2 * j + 1], a8, b8);
          }
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
      // exponents of the weights times their value's scale, relative to m (the maximum less LIFT); keys that a row does not see: v[r][k] is row r's of the lane
      constexpr int EACH = SLIM ? 2 : 4;  // keys of a lane's row
      auto key_at = [&](int k) { return s * STEP + key_of<D>(SLIM ? gr + 8 * k : 8 * (k >> 1) + c4 * 2 + (k & 1)); };
      float v[2][EACH];
      bool grows = false;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float cr = c[r] * key_scale;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
          float sum;
          if constexpr (SLIM) {
            const int at = 2 * k + r;
            sum = KC == 2 ? (sums_qk[0][0][at] + sums_qk[0][1][at]) + (sums_qk[1][0][at] + sums_qk[1][1][at]) : sums_qk[0][0][at] + sums_qk[1][0][at];
          } else {
            const int at = 2 * r + (k & 1);
            sum = KC == 2 ? sums_qk[0][k >> 1][at] + sums_qk[1][k >> 1][at] : sums_qk[0][k >> 1][at];
          }
          v[r][k] = fmaf(sum, cr, exponent);
        }
      }
      if ((s + 1) * STEP > all_see) {
        if (exponent != exponent) {  // the weights are NaN, where they are not zero: 0 times NaN must not be
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < VC / 4; ++i) w[k][i] = 0;
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int k = 0; k < EACH; ++k)
            if (key_at(k) >= seen[r]) v[r][k] = -INFINITY;
      }
      float top[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        top[r] = fmaxf(v[r][0], v[r][1]);
        if constexpr (!SLIM) top[r] = max3(top[r], v[r][2], v[r][3]);
        grows |= top[r] > m[r] + RISE;
      }
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if constexpr (SLIM) {
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 4));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 8));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 16));
          } else {
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
          }
          top[r] = fmaxf(top[r] - LIFT, m[r]);
          const float f = top[r] > m[r] ? fast_exp2(m[r] - top[r]) : 1.0f;  // 0 where nothing was seen before
          m[r] = top[r];
          l[r] *= f;
#pragma unroll
          for (int i = 0; i < OUT; ++i) {
            o[i][SLIM ? r : 2 * r] *= f;
            o[i][SLIM ? r + 2 : 2 * r + 1] *= f;
          }
        }
      }
      uint32_t p[2][2];
      float e[2][EACH];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float from = m[r] > -INFINITY ? m[r] : 0.0f;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
          e[r][k] = fast_exp2(v[r][k] - from);
          sum += e[r][k];
        }
        l[r] = fmaf(sum, inverse, l[r]);
      }
      if constexpr (SLIM) {  // from keys by rows to rows by keys: the second operand's order
        p[0][0] = transposed(pack<true>(e[0][0], e[1][0]));
        p[0][1] = transposed(pack<true>(e[0][1], e[1][1]));
      } else {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          p[r][0] = pack<true>(e[r][0], e[r][1]);
          p[r][1] = pack<true>(e[r][EACH - 2], e[r][EACH - 1]);
        }
      }
#pragma unroll
      for (int i = 0; i < VC / 4; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // columns 4 i + 2 h and the next
          const uint32_t lo = __byte_perm(w[0][i], w[1][i], h ? 0x7362 : 0x5140), hi = __byte_perm(w[2][i], w[3][i], h ? 0x7362 : 0x5140);
          const uint32_t a = halves_of(lo & 0xffffu), a8 = halves_of(hi & 0xffffu), b2 = halves_of(lo >> 16), b8 = halves_of(hi >> 16);
          if constexpr (SLIM) {
            mma_m16n8k16_f16(o[2 * i + h], a, b2, a8, b8, p[0][0], p[0][1]);
          } else {
            mma_m16n8k16_f16(o[(4 * i + 2 * h) % OUT], p[0][0], p[1][0], p[0][1], p[1][1], a, a8);
            mma_m16n8k16_f16(o[(4 * i + 2 * h + 1) % OUT], p[0][0], p[1][0], p[0][1], p[1][1], b2, b8);
          }
        }
      stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    cp_wait<0>();
    // o[i][2 r + e]: row gr + 8 r, column i of the VC of lane group 2 c4 + e; SLIM: o[i][2 e + r]: row 2 c4 + r, column 2 i + e of gr's.
    // In units of 2^base, and of UNLIFT.
    const float unit = base > NO_BASE ? exponent_of_2((int)base) : 1.0f;
    const bool alone = s0 == 0 && s1 == steps;
    const int which = 2 * warp + (at + s1 - s0 == stop ? 1 : 0);  // a piece's place: the warp's first, or what it ends with
    float* sum = which & 1 ? reinterpret_cast<float*>(smem + warp * STAGES * STAGE_BYTES) : sums + warp * g.max_rows * D;
    if (!alone) {
      __syncwarp();  // the stages have been read
      if (lane == 0) pieces[which] = {first[b] + head * steps, steps, x.q0, rows, head};
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], SLIM ? 4 : 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], SLIM ? 8 : 2);
      if (SLIM) l[r] += __shfl_xor_sync(0xffffffffu, l[r], 16);
      const int row = SLIM ? 2 * c4 + r : gr + 8 * r, token = row / g.group;
      if (row >= rows) continue;
      const float inv = !alone ? UNLIFT : l[r] == 0.0f ? 0.0f : 1.0f / l[r];
      if (!alone && (SLIM ? gr : c4) == 0) ml[which][row] = make_float2(m[r], l[r] * UNLIFT);
#pragma unroll
      for (int e = 0; e < (SLIM ? 1 : 2); ++e) {
        const int n = SLIM ? gr : 2 * c4 + e, col = VC * (D == 128 ? (n >> 1) | (n & 1) << 2 : n);
        auto value = [&](int i) { return (SLIM ? o[i / 2][2 * (i & 1) + r] : o[i % OUT][2 * r + e]) * inv * unit; };
        if (alone) {
          uint16_t* out = g.o + (int64_t)(x.q0 + token) * g.ldo + (int64_t)(head * g.group + row - token * g.group) * D + col;
#pragma unroll
          for (int i = 0; i < VC / 8; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = pack<F16>(value(8 * i + 2 * k), value(8 * i + 2 * k + 1));
            *reinterpret_cast<uint4*>(out + 8 * i) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < VC / 4; ++i)
            *reinterpret_cast<float4*>(sum + row * D + col + 4 * i) = make_float4(value(4 * i), value(4 * i + 1), value(4 * i + 2), value(4 * i + 3));
        }
      }
    }
    at += s1 - s0;
  }
  // ---- the CTA's pieces, those of one head added up in the order of the keys; heads of several CTAs are left to the join. A warp for 128
  // columns of a row ----
  __syncthreads();
  Piece mine = {};  // lane i's: piece i
  if (lane < 2 * WARPS) mine = pieces[lane];
  const uint32_t valid = __ballot_sync(0xffffffffu, mine.rows > 0);
  const int before = __shfl_sync(0xffffffffu, mine.from, 31 - __clz(valid & ((1u << lane) - 1) | 1u));
  uint32_t starts = __ballot_sync(0xffffffffu, mine.rows > 0 && ((valid & ((1u << lane) - 1)) == 0 || mine.from != before));
  int turn = warp;
  while (starts) {
    const int k0 = __ffs(starts) - 1;
    starts &= starts - 1;
    const uint32_t these = valid & ~((1u << k0) - 1) & (starts ? (starts & -starts) - 1 : 0xffffffffu);
    const Piece x = pieces[k0];
    const bool whole = x.from >= c0 && x.from + x.steps <= c1;
    const int slots = x.rows * (D / 4);
    for (; turn * 32 < slots; turn += WARPS) {
      const int slot = turn * 32 + lane, row = slot / (D / 4), col = slot % (D / 4) * 4;
      if (slot >= slots) continue;
      float top = -INFINITY, all = 0.0f;
      float4 acc = make_float4(0, 0, 0, 0);
      for (uint32_t rest = these; rest;) {
        float2 v[4];
        float4 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = rest ? __ffs(rest) - 1 : k0;
          v[i] = ml[k][row];
          o[i] = *reinterpret_cast<const float4*>(
              (k & 1 ? reinterpret_cast<const float*>(smem + (k >> 1) * STAGES * STAGE_BYTES) : sums + (k >> 1) * g.max_rows * D) + row * D + col);
          if (rest == 0) {  // no piece
            v[i].y = 0.0f;
            o[i] = make_float4(0, 0, 0, 0);
          }
          rest &= rest - 1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) add_piece(top, all, acc, v[i], o[i]);
      }
      if (whole) {
        const float inv = all == 0.0f ? 0.0f : 1.0f / all;
        const int token = row / g.group;
        uint16_t* out = g.o + (int64_t)(x.q0 + token) * g.ldo + (int64_t)(x.head * g.group + row - token * g.group) * D + col;
        *reinterpret_cast<uint2*>(out) = make_uint2(pack<F16>(acc.x * inv, acc.y * inv), pack<F16>(acc.z * inv, acc.w * inv));
      } else {
        float* to = g.partial + (2 * blockIdx.x + (x.from < c0 ? 0 : 1)) * place_floats<D>(g.max_rows);
        if (col == 0) reinterpret_cast<float2*>(to + g.max_rows * D)[row] = make_float2(top, all);
        *reinterpret_cast<float4*>(to + row * D + col) = acc;
      }
    }
    turn -= (slots + 31) / 32;  // the next head's go on with the warps that had none of this one's
    if (c8.whole == 0 && threadIdx.x == 0 && x.from + x.steps > c1)
      c8.cuts[blockIdx.x] = make_int4(x.q0, x.rows, x.from / dealt.run << 16 | (x.from + x.steps - 1) / dealt.run, 1 + x.head);
  }
}

// Adds up the pieces of a head that several CTAs worked on, in the order of the keys. Two latencies and a launch, 2.5 us: a head of n + 1
// pieces has n CTAs here, those whose run ends within it, and each takes its share of the columns, so that a hundred heads of two pieces and eight
// of twenty spread alike, a load or two to a thread, over CTAs that have all begun before the pieces are there. (With CTAs for every
// head and share of columns, cut or not, most of which begin after the others: 5 us; 16 sequences of 4000 keys, 8 heads, 39.0 and here 34.0 us.)
template <bool F16, int D>
__global__ void __launch_bounds__(THREADS) attention_join_q8(const RowArgs g, const RowsQ8 c8) {
  __shared__ float2 sh_ml[THREADS];
  __shared__ float4 sh_o[THREADS];
  pdl_launch_dependents();
  pdl_wait_primary();
  const int w = (int)blockIdx.x;
  const int4 x = __ldcg(c8.cuts + w);
  if (x.w == 0) return;
  const int w0 = x.z >> 16, w1 = x.z & 0xffff, n = w1 - w0, rows = x.y, head = x.w - 1;
  const int slots = rows * (D / 4), share = (slots + n - 1) / n, end = min((w - w0 + 1) * share, slots);
  const int64_t place = place_floats<D>(g.max_rows);
  for (int from = (w - w0) * share; from < end; from += THREADS) {
    const int here = min(end - from, THREADS), groups = min(THREADS / here, n + 1);
    const int group = (int)threadIdx.x / here, slot = from + (int)threadIdx.x - group * here;
    const int row = slot / (D / 4), col = slot % (D / 4) * 4;
    float top = -INFINITY, all = 0.0f;
    float4 acc = make_float4(0, 0, 0, 0);
    if (group < groups) {
      for (int v = w0 + group; v <= w1; v += groups) {
        const float* p = g.partial + (2 * v + (v == w0 ? 1 : 0)) * place;
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(p + g.max_rows * D) + row);
        const float4 o = __ldcg(reinterpret_cast<const float4*>(p + row * D + col));
        add_piece(top, all, acc, ml, o);
      }
      sh_ml[threadIdx.x] = make_float2(top, all);
      sh_o[threadIdx.x] = acc;
    }
    __syncthreads();
    if (group == 0) {
      for (int k = 1; k < groups; ++k) add_piece(top, all, acc, sh_ml[threadIdx.x + k * here], sh_o[threadIdx.x + k * here]);
      const float inv = all == 0.0f ? 0.0f : 1.0f / all;
      const int token = row / g.group;
      uint16_t* out = g.o + (int64_t)(x.x + token) * g.ldo + (int64_t)(head * g.group + row - token * g.group) * D + col;
      *reinterpret_cast<uint2*>(out) = make_uint2(pack<F16>(acc.x * inv, acc.y * inv), pack<F16>(acc.z * inv, acc.w * inv));
    }
    __syncthreads();
  }
}

template <bool F16, int D, bool SLIM>
cudaError_t launch_rows_q8(const RowArgs& g, const RowsQ8& c8, cudaStream_t stream) {
  const int64_t ctas = rows_grid();
  const size_t smem = (size_t)WARPS * (kStages<D> * 2 * STEP * D + g.max_rows * D * 4) + (size_t)std::min(g.B, KEPT) * sizeof(Lengths) + first_bytes(g);
  const cudaError_t e = launch_rows<attention_rows_q8<F16, D, SLIM>>(ctas, smem, stream, g, c8);
  if (e != cudaSuccess || c8.whole || ctas == 1) return e;
  return launch_rows<attention_join_q8<F16, D>>(ctas - 1, 0, stream, g, c8);
}
template <bool F16, int D>
cudaError_t launch_rows_q8(const RowArgs& g, const RowsQ8& c8, cudaStream_t stream) {
  return g.max_rows <= 8 ? launch_rows_q8<F16, D, true>(g, c8, stream) : launch_rows_q8<F16, D, false>(g, c8, stream);
}

}  // namespace

int launch_attention_rows_q8(const PifaAttention& a, int* status, cudaStream_t stream) {
  const RowArgs g = row_args(a, status);
  const int64_t heads = a.B * a.cache.heads, ctas = rows_grid();
  const int64_t share = (heads + ctas - 1) / ctas, room = a.cols * a.cache.page_size;
  const bool uncut = share * room <= (share == 1 ? WHOLE_KEYS_ONE : WHOLE_KEYS) && (share * ctas - heads) * room <= WHOLE_MORE * ctas;
  const int64_t places = 2 * MAX_CTAS * (a.cache.dim == 64 ? place_floats<64>(g.max_rows) : place_floats<128>(g.max_rows));
  const RowsQ8 c8 = {static_cast<const uint8_t*>(a.k), static_cast<const uint8_t*>(a.v), a.q8->k, a.q8->v, a.q8->shape.page_stride,
                     a.q8->shape.block_stride, a.q8->shape.head_stride, uncut ? (int)share : 0,
                     reinterpret_cast<int4*>(g.partial + places)};
  const bool f16 = a.dtype == PIFA_DTYPE_FP16;
  cudaError_t e;
  if (a.cache.dim == 64) e = f16 ? launch_rows_q8<true, 64>(g, c8, stream) : launch_rows_q8<false, 64>(g, c8, stream);
  else e = f16 ? launch_rows_q8<true, 128>(g, c8, stream) : launch_rows_q8<false, 128>(g, c8, stream);
  return e == cudaSuccess ? PIFA_OK : pifa_fail_cuda("attention_rows_q8 launch", e);
}
