// attention_tc.cu -- attention of chunks of new tokens over a paged cache, on the 5th-generation tensor cores.
//
//   o = sum_j softmax_j(scale q . k_j) v_j over the keys j < L - n + i + 1 of new token i (L keys, n new tokens).
//
// Rows: the query heads of a key / value head share its keys, so the n new tokens of a request and the G heads
// of a group make n G rows, token-major. A tile is the rows of floor(128 / G) tokens, 128 of them at most, a work
// item two tiles of one request and one key / value head; it walks the keys in tiles of 128 and reads K and V
// once for both tiles.
// One pass with a running maximum: S = Q K^T (128 x 128, fp32, tensor memory); a thread owns a row, so maximum
// and sum need no exchange; p = exp2(c s - c m) goes back to tensor memory as bf16 or fp16 over S's columns
// and is the first operand of O += P V. m is only raised, and O and l rescaled, when the row's maximum
// has grown by more than 8 in the exponent (then O's columns are read and written by the row's warp);
// until then weights reach 2^8 at most, which costs neither format precision. The rounding of the weights, which l
// adds up as they were, takes the outputs' error from 0.0017 of their size to 0.0022 in bf16, from 0.00021 to 0.00026 in fp16; a
// product of their lower parts as well, half as many MMAs again, was not taken.
//
// CTA of 384 threads, one per SM, persistent:
//   warps 0-3, 4-7   softmax and epilogue of tile 0 and 1 (tensor memory quarter = warp % 4)
//   warp 8           takes work items from a queue and loads K's tiles by TMA into a ring of slots that K and V take in
//                    turn, a page (or a 128-token part of one) and 64 columns a copy, a lane for each
//   warps 9, 10      issue the MMAs of tile 0 and 1: PV, in two halves of the keys as P arrives, and the next S; one
//                    tile's softmax runs under the other tile's MMAs. (One warp for both was the bound.)
//   warp 11          loads the next item's rows of Q, as soon as the last S of a tile has been computed, and V
// P lies over S, and S of the next keys is written over both: the MMAs of one warp run in issue
// order, PV(j) before S(j + 1), and S(j)'s values were read before P was announced.
// Keys past L: their scores are masked, and their rows of V, which may hold anything, are set to zero in shared
// memory, since 0 times NaN is NaN.
//
// Work: a first kernel (one CTA) reads the lengths, lists the items (later rows of a request first: they have
// more keys) and cuts the last ones along the keys where whole items would leave SMs idle in the
// last round: a piece writes its unnormalised sums, and when all have, all warps add them up, in the order of the
// keys. Every wait is bounded; on timeout PIFA_ERR_TIMEOUT is latched and the CTA drains.
//
// Measured, head_dim 128, bf16: 2048 tokens over 30000 cached, 64 heads on 8 key / value heads, pages of 64: 1.20 to 1.27 ms,
// 1640 to 1740 TFLOP/s of the visible pairs (the measured bf16 rate is 1910 in a burst, 1702 for seconds: the power cap is what
// bounds it; 82% of the cycles have a tensor instruction). A prompt of 2048, 32 heads: 38 us, 16 tiles at most for a CTA: 3.3 us
// of plan, 2.7 until the first S, about 1.6 a tile (S to softmax to PV to S is a chain of 2450 to 3000 cycles, of
// which the MMAs of both tiles take 2048), 2 for the last outputs.
// What made it so, on the first case: 3.6 ms with spilled rows of S and one issuing warp; registers moved to the softmax
// warps 1.72; operands of the MMAs in uniform registers (one elected thread in a converged warp: 50 cycles an
// instruction, not 80), a warp for each tile's MMAs, the tiles in turn and the weights of half a tile handed over first 1.30;
// Q by TMA 1.22. Cut items cost six tiles' time: 200 tokens over 8000 took 67 us with
// a cut that left a second round, 45 with one round, 39 since all warps add up the pieces.
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pifa.h"
#include "pifa_internal.h"
#include "ptx.cuh"

namespace {

using namespace pifa;

constexpr int BM = 128;             // rows of a tile
constexpr int ROWS = 2 * BM;        // rows of an item (with those that a group's size leaves unused)
constexpr int BN = 128;             // keys of a tile
constexpr int THREADS = 384;
constexpr int PLAN_THREADS = 256;
constexpr int MAX_REST = 512;       // items that may be cut: fewer than a round's, and one more for each head
constexpr int MAX_PARTS = 456;      // pieces (times heads) that may leave partial sums: three for each SM
constexpr int EARLY = 2;            // of four times 32 keys: those whose weights are handed to the MMAs first
constexpr uint32_t HALF = BN * 128;  // 128 rows of 64 columns: 16 KB

template <int D>
struct Cfg {
  static constexpr uint32_t TILE = D / 64 * HALF;
  static constexpr int SLOTS = D == 128 ? 5 : 8;
  static constexpr uint32_t SMEM = 1024 + (2 + SLOTS) * TILE + 1024;
  static constexpr int64_t PART_FLOATS = ROWS * D + 2 * ROWS;  // O, then (m, l) of each row
};

// A work item: 16 words. The plan lists those of head 0 with everything that a CTA has to know; a CTA takes one
// for a head by filling in the last four.
struct Item {
  int b, tok0, n;          // request, first token, tokens of the request
  int L, q0, ahead;        // as Lengths
  int j0, j1, e0, e1;      // key tiles; the end of those that the rows of tile 0 and 1 see
  int part, parts;         // which piece of how many
  int slot, pad;           // place of its partial sums (in the list: of head 0, over heads)
  int head, end;           // end: no item
};

struct Plan {
  int next;          // items taken; beyond the grid's first ones if no item is cut
  int entries;
  int cuts, pieces;  // items that are cut (over heads), and their pieces
  int done;          // warps that have written a piece's sums
  int pad[3];
};

struct TcArgs {
  uint16_t* o;
  const int32_t *table, *q_start, *kv_len;
  Plan* plan;
  int* splits;        // the first entry of each item that is cut
  Item* list;
  float* partial;
  int64_t ldo, ldt, pages;
  int T, heads, group, tpt, B, max_q,   // tpt: tokens of a tile
       cols, page_size, page_shift;
  int token_at, head_at;             // their places among the tensor maps' coordinates 1 to 3; the page has the third
  float c;                           // |scale| log2(e)
  int negate;                        // scale < 0
  int wide;                          // rows of O start on 32-byte sectors
  int* status;
  uint64_t timeout_ns;
};

struct Lengths {
  int q0, n, L;   // first row of Q, new tokens that are computed, keys
  int ahead;      // token i sees ahead + i keys
};

// Lengths of request b, kept within the buffers whatever the arrays hold. Ascending starts make the tokens of all requests T at most.
__device__ __forceinline__ Lengths lengths_of(const TcArgs& g, int b) {
  Lengths x;
  x.q0 = min(max(g.q_start[b], 0), g.T);
  x.n = min(min(max(g.q_start[b + 1], x.q0), g.T) - x.q0, g.max_q);
  x.L = min(max(g.kv_len[b], 0), g.cols << g.page_shift);
  x.ahead = x.L - (max(g.q_start[b + 1], x.q0) - x.q0) + 1;
  return x;
}

// Key tiles that the tile of tokens from `tok` on sees: up to its last token's last key.
__device__ __forceinline__ int tile_end(const Lengths& x, int tpt, int tok) {
  if (tok >= x.n) return 0;
  return (max(x.ahead + min(tok + tpt, x.n) - 1, 0) + BN - 1) / BN;
}

// ---- plan ---------------------------------------------------------------------------------------
// Exclusive sum over the block's threads, and the total; `part` holds a value for each warp.
__device__ __forceinline__ unsigned long long block_scan(unsigned long long v, unsigned long long* part,
                                                         unsigned long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long a = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long x = __shfl_up_sync(0xffffffffu, a, o);
    if (lane >= o) a += x;
  }
  __syncthreads();  // part is free
  if (lane == 31) part[warp] = a;
  __syncthreads();
  unsigned long long before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < PLAN_THREADS / 32; ++w) {
    before += w < warp ? part[w] : 0;
    total += part[w];
  }
  return a - v + before;
}

__global__ void __launch_bounds__(PLAN_THREADS, 1) attention_plan(const TcArgs g, int grid) {
  extern __shared__ __align__(16) uint8_t plan_smem[];
  Lengths* len = reinterpret_cast<Lengths*>(plan_smem);          // B
  int* first = reinterpret_cast<int*>(plan_smem + (size_t)g.B * sizeof(Lengths));  // B + 1: first item of each request
  __shared__ unsigned long long part[PLAN_THREADS / 32];
  __shared__ int rest_cost[MAX_REST], whole_most;
  __shared__ unsigned long long whole_sum;
  __shared__ int cut;             // key tiles of a piece
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31;
  if (tid == 0) {
    whole_most = 0;
    whole_sum = 0;
  }
  pdl_wait_primary();
  bool over = false;
  int items = 0;
  unsigned falls = 0;  // starts that are less than the one before: counted with the items, from bit 40 on
  for (int b0 = 0; b0 < g.B; b0 += PLAN_THREADS) {
    const int b = b0 + tid;
    unsigned long long n = 0;
    if (b < g.B) {
      const Lengths x = lengths_of(g, b);
      over |= g.kv_len[b] > (g.cols << g.page_shift) || (int64_t)g.q_start[b + 1] - g.q_start[b] > x.n;
      n = (unsigned)((x.n + 2 * g.tpt - 1) / (2 * g.tpt)) | (unsigned long long)(g.q_start[b + 1] < g.q_start[b]) << 40;
      len[b] = x;
    }
    unsigned long long total;
    const int at = (int)block_scan(n, part, total);
    if (b < g.B) first[b] = items + at;
    items += (int)total;
    falls += (unsigned)(total >> 40);
  }
  if (tid == 0) first[g.B] = items;
  if (over) latch_status(g.status, PIFA_ERR_CAPACITY);
  // Requests that overlap could have more rows than T, and more items than the list has room for: nothing is done then.
  if (falls > 0) {
    items = 0;
    if (tid == 0) latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
  }
  __syncthreads();

  // the item at place k of the list, later rows of a request first, and its cost in key tiles
  auto item_at = [&](int k, Item& x) {
    int lo = 0, hi = g.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= k) lo = mid;
      else hi = mid;
    }
    const Lengths v = len[lo];
    x.b = lo;
    x.tok0 = (first[lo + 1] - 1 - k) * 2 * g.tpt;
    x.n = v.n;
    x.L = v.L;
    x.q0 = v.q0;
    x.ahead = v.ahead;
    x.e0 = tile_end(v, g.tpt, x.tok0);
    x.e1 = tile_end(v, g.tpt, x.tok0 + g.tpt);
    return max(x.e0, x.e1);
  };
  // Whole rounds of the grid stay whole; the items of the last, unfilled round may be cut.
  const int whole = (int)((int64_t)items * g.heads / grid * grid / g.heads), rest = items - whole;
  Item x;
  int cost = 0;
  for (int k0 = 0; k0 < items; k0 += PLAN_THREADS) {
    const int k = k0 + tid;
    const bool here = k < items;
    if (!__any_sync(0xffffffffu, here)) break;
    if (here) cost = item_at(k, x);
    if (here && k >= whole && k - whole < MAX_REST) rest_cost[k - whole] = cost;
    const int whole_cost = here && k < whole ? cost : 0;
    const int most = __reduce_max_sync(0xffffffffu, whole_cost), sum = __reduce_add_sync(0xffffffffu, whole_cost);
    if (lane == 0) {
      atomicMax(&whole_most, most);
      atomicAdd(&whole_sum, (unsigned long long)sum);
    }
  }
  __syncthreads();
  if (tid < 32) {
    // The time, in key tiles, if the longest of those items is cut into `want` pieces and the others into pieces
    // no longer: one round if there is a CTA for each piece; else an even share for every CTA, and the wait for
    // the last pieces: of alike ones, what is left of their last round, of unlike ones about half a piece. An item
    // costs about two tiles on top (rows of Q, first and last products), a piece with its sums four, and adding them up
    // at the end four more.
    int longest = 0;
    for (int i = 0; i < min(rest, MAX_REST); ++i) longest = max(longest, rest_cost[i]);
    const int want = tid < 16 ? tid + 1 : (int)(16.0f * exp2f(0.21f * (float)(tid - 15)));
    const int size = max((longest + want - 1) / want, 1);
    int pieces = 0, most = 0;
    float work = 0.0f;
    for (int i = 0; i < min(rest, MAX_REST); ++i) {
      const int c = rest_cost[i], n = max((c + size - 1) / size, 1);
      const float extra = n > 1 ? 4.0f : 2.0f;
      pieces += n;
      most = max(most, (c + n - 1) / n + (int)extra);
      work += (float)c + extra * (float)n;
    }
    const float jobs = (float)pieces * (float)g.heads, rounds = jobs / (float)grid;
    const float alike = pieces ? work / ((float)pieces * (float)most) : 0.0f;
    const float share = (work + (float)whole_sum + 2.0f * (float)whole) * (float)g.heads / (float)grid;
    float t = whole == 0 && rounds <= 1.0f ? (float)most
                                            : share + (float)most * (alike * (ceilf(rounds) - rounds) + (1.0f - alike) * 0.5f);
    t = fmaxf(t, fmaxf((float)most, (float)(whole_most + 2)));
    if (pieces > rest) t += 4.0f;
    // more than there is room for
    if (tid > 0 && ((int64_t)pieces * g.heads > MAX_PARTS || rest > MAX_REST || want > longest)) t = 3e38f;
    int who = tid;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float ot = __shfl_xor_sync(0xffffffffu, t, o);
      const int ow = __shfl_xor_sync(0xffffffffu, who, o);
      if (ot < t || (ot == t && ow < who)) {
        t = ot;
        who = ow;
      }
    }
    if (tid == who) cut = who == 0 ? 0x3fffffff : size;
  }
  __syncthreads();
  const int size = cut;
  unsigned long long done = 0;  // entries, from bit 32 on; partial-sum places, from bit 16 on; cut items
  for (int k0 = 0; k0 < items; k0 += PLAN_THREADS) {
    const int k = k0 + tid;
    int pieces = 0;
    if (k < items) {
      if (items > PLAN_THREADS) cost = item_at(k, x);
      pieces = k < whole ? 1 : max((cost + size - 1) / size, 1);
    }
    unsigned long long total;
    const unsigned long long at = done + block_scan(((unsigned long long)pieces << 32) |
                                                        (pieces > 1 ? ((unsigned)pieces << 16) | 1u : 0u), part, total);
    for (int p = 0; p < pieces; ++p) {  // even pieces
      Item e = x;
      e.j0 = (int)((int64_t)cost * p / pieces);
      e.j1 = (int)((int64_t)cost * (p + 1) / pieces);
      e.e0 = min(x.e0, e.j1);
      e.e1 = min(x.e1, e.j1);
      e.part = p;
      e.parts = pieces;
      e.slot = (int)(at >> 16 & 0xffffu) + p;
      e.pad = e.head = e.end = 0;
      int4* to = reinterpret_cast<int4*>(g.list + (at >> 32) + p);
      const int4* from = reinterpret_cast<const int4*>(&e);
#pragma unroll
      for (int i = 0; i < 4; ++i) to[i] = from[i];
    }
    if (pieces > 1) g.splits[at & 0xffffu] = (int)(at >> 32);
    done += total;
  }
  if (tid == 0) {
    const Plan p = {0, (int)(done >> 32), (int)(done & 0xffffu), (int)(done >> 16 & 0xffffu), 0, {0, 0, 0}};
    *g.plan = p;
  }
}

// ---- attention -------------------------------------------------------------------------------------
// Descriptor of V's tile as the MN-major second operand: rows of 64 columns (128 bytes, swizzled), one for each
// key, 8-key groups 1024 bytes apart, 64-column blocks HALF bytes apart.
__device__ __forceinline__ uint64_t sw128_mn_desc(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((HALF >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

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

// 32 columns of a row that the thread owns: whole 32-byte sectors where all rows start on one.
template <bool F16>
__device__ __forceinline__ void store_row(uint16_t* out, const float* x, bool wide) {
  uint32_t w[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) w[k] = pack<F16>(x[2 * k], x[2 * k + 1]);
  if (wide) {
    stg256(out, w);
    stg256(out + 16, w + 8);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(out + 8 * k) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
  }
}

template <bool F16, int D>
__global__ void __launch_bounds__(THREADS, 1)
    attention_tc(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                 const __grid_constant__ CUtensorMap vmap, const TcArgs g) {
  using C = Cfg<D>;
  constexpr int SLOTS = C::SLOTS;
  constexpr uint32_t TILE = C::TILE;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem + 2 * TILE;
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + SLOTS * TILE);
  uint64_t* empty = full + SLOTS;
  uint64_t* s_full = empty + SLOTS;   // S of a tile is in tensor memory
  uint64_t* p_full = s_full + 2;      // half of its P is, and its O may be added to: two for each tile
  uint64_t* o_full = p_full + 4;      // the item's last PV is done
  uint64_t* q_full = o_full + 2;
  uint64_t* q_free = q_full + 2;
  uint64_t* item_full = q_free + 2;
  uint64_t* item_free = item_full + 2;
  uint64_t* v_clean = item_free + 2;  // of a slot: rows of V past the last key are zero
  uint64_t* turn = v_clean + SLOTS;   // the tiles' MMAs alternate
  uint64_t* drain = turn + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 2);
  Item* items = reinterpret_cast<Item*>(tmem_slot + 2);

  pdl_launch_dependents();
  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < SLOTS; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 2);
      mbar_init(&v_clean[s], 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&s_full[t], 1);
      mbar_init(&p_full[2 * t], 4);
      mbar_init(&p_full[2 * t + 1], 4);
      mbar_init(&turn[t], 1);
      mbar_init(&drain[t], 1);
      mbar_init(&o_full[t], 1);
      mbar_init(&q_full[t], 1);
      mbar_init(&q_free[t], 1);
      mbar_init(&item_full[t], 1);
      mbar_init(&item_free[t], 11);
    }
    fence_mbar_init();
    prefetch_tmap(&qmap);
    prefetch_tmap(&kmap);
    prefetch_tmap(&vmap);
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
  pdl_wait_primary();
  bool dead = false;
  // all lanes of the warp wait; false (and the status latched) if the wait ran out
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    const bool ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, g.timeout_ns));
    if (!ok) {
      latch_status(g.status, PIFA_ERR_TIMEOUT);
      dead = true;
    }
    return ok;
  };

  // Registers: a softmax thread holds a row of S. 2 x 128 x 208 + 128 x 88 = 384 x 168, as launched.
  if (warp >= 8) {
  regs_lower<88>();
  // K (kv = 0) or V of an item's key tiles, fill after fill of the ring: K and V take its slots in turn. A lane
  // copies 64 columns of a page's rows (or of 128 of them). One warp issuing both was the bound for pages of 16.
  auto stream = [&](int kv, int& tiles, int b, int L, int head, int j0, int j1, auto&& every) {
    const int per_tile = g.page_size >= BN ? 1 : BN / g.page_size, box_rows = min(g.page_size, BN);
    const int mine = lane / (D / 64), half = lane % (D / 64);
    const int n_pages = (L + g.page_size - 1) >> g.page_shift;
    const int32_t* row = g.table + b * g.ldt;
    auto page_of = [&](int j) {
      const int p = ((j * BN) >> g.page_shift) + mine;
      return mine < per_tile && j < j1 && p < n_pages ? row[p] : -2;  // -2: no page
    };
    int id = page_of(j0);
    for (int j = j0; j < j1 && !dead; ++j) {
      const int next = page_of(j + 1);
      every(j);
      const bool has = id != -2 || (mine < per_tile && ((j * BN) >> g.page_shift) + mine < n_pages);
      if (has && (id < 0 || id >= g.pages)) {
        latch_status(g.status, PIFA_ERR_DEVICE_INDEX);
        id = (int)g.pages;  // outside the tensor map: zeros
      }
      const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, has)) * (uint32_t)box_rows * 128u;
      const int token = (j * BN) & (g.page_size - 1);
      const int y = g.token_at == 0 ? token : g.head_at == 0 ? head : id;
      const int z = g.token_at == 1 ? token : g.head_at == 1 ? head : id;
      const int w = g.token_at == 2 ? token : g.head_at == 2 ? head : id;
      const int fill = 2 * tiles + kv, s = fill % SLOTS;
      if (!wait(&empty[s], ((uint32_t)(fill / SLOTS) & 1u) ^ 1u)) break;
      if (lane == 0) mbar_arrive_expect_tx(&full[s], bytes);
      __syncwarp();
      if (has)
        tma_load_4d(smem_u32(ring) + (uint32_t)s * TILE + (uint32_t)half * HALF + (uint32_t)(mine * box_rows) * 128u,
                    kv ? &vmap : &kmap, half * 64, y, z, w, &full[s]);
      ++tiles;
      id = next;
    }
  };
  // nothing may land in shared memory after the CTA has left
  auto landed = [&](int kv, int tiles) {
    for (int i = max(2 * tiles - 2 * SLOTS, 0) + kv; i < 2 * tiles; i += 2)
      if (i + SLOTS >= 2 * tiles && !mbar_wait(&full[i % SLOTS], (uint32_t)(i / SLOTS) & 1u, 100000000ull))
        latch_status(g.status, PIFA_ERR_TIMEOUT);
  };
  if (warp == 8) {
    // ---------------- queue and K ----------------
    int tiles = 0;
    // An entry's words, a lane each. The list has room for MAX_PARTS entries and more, so that the first can be read
    // before it is known to be one.
    auto fetch = [&](int k) { return lane < 16 ? __ldcg(reinterpret_cast<const int*>(g.list + k / g.heads) + lane) : 0; };
    int k = (int)blockIdx.x, word = fetch(k);
    const int total = __ldcg(&g.plan->entries) * g.heads;
    // With cut items the first one comes from the queue too: a CTA that does not run yet must hold no piece, since
    // the others wait for all pieces at the end.
    const int ahead = __ldcg(&g.plan->cuts) > 0 ? 0 : (int)gridDim.x;
    if (ahead == 0) {
      if (lane == 0) k = atomicAdd(&g.plan->next, 1);
      k = __shfl_sync(0xffffffffu, k, 0);
      word = k < total ? fetch(k) : 0;
    }
    // Item n for all: false after the last, or if the wait for its place ran out.
    auto publish = [&](int n) {
      if (!wait(&item_free[n & 1], (((uint32_t)n >> 1) & 1u) ^ 1u)) return false;
      const int head = k % g.heads;
      if (lane == 12) word = word * g.heads + head;
      if (lane == 14) word = head;
      if (lane == 15) word = k >= total;
      if (lane < 16) reinterpret_cast<int*>(&items[n & 1])[lane] = word;
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_full[n & 1]);
      return k < total;
    };
    bool more = publish(0);
    for (int n = 0; more; ++n) {
      const int b = __shfl_sync(0xffffffffu, word, 0), L = __shfl_sync(0xffffffffu, word, 3);
      const int j0 = __shfl_sync(0xffffffffu, word, 6), j1 = __shfl_sync(0xffffffffu, word, 7);
      // The next item is taken towards the end of this one, each step a tile ahead of what needs it: late, so
      // that the CTA that is done first takes it, and in time for its loads to follow on.
      int step = 0, taken = 0;
      auto take = [&] {
        if (step == 0) {
          if (lane == 0) taken = ahead + atomicAdd(&g.plan->next, 1);
        } else if (step == 1) {
          k = __shfl_sync(0xffffffffu, taken, 0);
          word = k < total ? fetch(k) : 0;
        } else {
          more = publish(n + 1);
        }
        ++step;
      };
      stream(0, tiles, b, L, k % g.heads, j0, j1, [&](int j) {
        if (j >= j1 - 4 && step < 3) take();
      });
      while (!dead && step < 3) take();
      if (dead) break;
    }
    landed(0, tiles);
  } else if (warp < 11) {
    // ---------------- MMAs of a tile ----------------
    const int t = warp - 9;
    const uint32_t kind = F16 ? idesc_f16_f32(BM, BN) : idesc_bf16_f32(BM, BN);
    const uint32_t qk_desc = kind | (g.negate ? 1u << 13 : 0u);
    const uint32_t pv_desc = (F16 ? idesc_f16_f32(BM, D) : idesc_bf16_f32(BM, D)) | (1u << 16);
    // descriptors: the low word holds the address, which alone changes
    const uint32_t q_desc = (uint32_t)sw128_desc(smem_u32(smem) + (uint32_t)t * TILE);
    const uint32_t k_desc = (uint32_t)sw128_desc(smem_u32(ring)), v_desc = (uint32_t)sw128_mn_desc(smem_u32(ring));
    constexpr uint32_t hi = (1024 >> 4) | (1u << 14) | (2u << 29);
    const uint32_t s_at = tmem + t * BN, o_at = tmem + 2 * BN + t * D;
    int s = 0;
    uint32_t ph = 0, q_ph = 0, p_ph = 0, tail_ph = 0, turn_ph = t ? 0u : 1u;  // tile 0 begins
    auto advance = [&] {
      if (++s == SLOTS) {
        s = 0;
        ph ^= 1u;
      }
    };
    // S = Q K^T; then K's slot is given back, and Q after the item's last S
    auto score = [&](int slot, bool last, bool pass) {
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t at = (uint32_t)(kk / 4) * (HALF / 16) + (uint32_t)(kk % 4) * 2;
          mma_ss_words(s_at, q_desc + at, k_desc + slot * (TILE / 16) + at, hi, qk_desc, kk > 0);
        }
        mma_commit(&s_full[t]);
        if (pass) mbar_arrive(&turn[1 - t]);  // after S: the other tile's products between PV and S would delay this softmax
        mma_commit(&empty[slot]);
        if (last) mma_commit(&q_free[t]);
      }
    };
    auto skip = [&](int slot) {  // a slot that this tile does not read
      if (lane == 0) mbar_arrive(&empty[slot]);
    };
    for (int n = 0; !dead; ++n) {
      if (!wait(&item_full[n & 1], ((uint32_t)n >> 1) & 1u)) break;
      const int end = uniform(items[n & 1].end), j0 = uniform(items[n & 1].j0), j1 = uniform(items[n & 1].j1);
      const int L = uniform(items[n & 1].L), e = uniform(t ? items[n & 1].e1 : items[n & 1].e0);
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_free[n & 1]);
      if (end) break;
      if (j0 >= j1) continue;
      if (!wait(&full[s], ph)) break;
      if (j0 < e) {
        if (!wait(&q_full[t], q_ph)) break;
        q_ph ^= 1u;
        tc_fence_after();
        score(s, j0 + 1 >= e, false);
      } else {
        skip(s);
      }
      advance();
      for (int j = j0; j < j1; ++j) {
        const int vs = s;
        if (!wait(&full[vs], ph)) break;
        advance();
        const int ks = s;
        if (j + 1 < j1) {
          if (!wait(&full[ks], ph)) break;
          advance();
        }
        const int tail = L - j * BN;  // keys of this tile
        if (tail < BN) {
          if (t == 0) {
            uint8_t* v = ring + vs * TILE;
            for (int i = max(tail, 0) * 8 + lane; i < BN * 8; i += 32)
#pragma unroll
              for (int h = 0; h < D / 64; ++h) *reinterpret_cast<uint4*>(v + h * HALF + i * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&v_clean[vs]);
          } else {
            if (!wait(&v_clean[vs], (tail_ph >> vs) & 1u)) break;
            tail_ph ^= 1u << vs;
          }
        }
        if (j < e) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!wait(&p_full[2 * t + h], p_ph)) break;
            if (h == 0 && !wait(&turn[t], turn_ph)) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int k = h ? 2 * EARLY : 0; k < (h ? BN / 16 : 2 * EARLY); ++k) {
                mma_ts_words(o_at, s_at + k * 8, v_desc + vs * (TILE / 16) + k * 128, hi, pv_desc, j > j0 || k > 0);
              }
              if (h == 1) {
                if (j + 1 >= e) mma_commit(&o_full[t]);
                mma_commit(&empty[vs]);
              }
            }
          }
          if (dead) break;
          p_ph ^= 1u;
        } else {
          if (!wait(&turn[t], turn_ph)) break;
          skip(vs);
        }
        turn_ph ^= 1u;
        if (j + 1 < e) {
          score(ks, j + 2 >= e, true);
        } else {
          if (lane == 0) mbar_arrive(&turn[1 - t]);
          if (j + 1 < j1) skip(ks);
        }
      }
    }
    __syncwarp();
    if (elect_one()) {
      mma_commit(&drain[t]);  // every MMA has completed before the tensor memory is freed
      if (!mbar_wait(&drain[t], 0, 100000000ull)) latch_status(g.status, PIFA_ERR_TIMEOUT);
    }
  } else {
    // ---------------- rows of Q, and V ----------------
    int loads[2] = {0, 0}, tiles = 0;
    for (int n = 0; !dead; ++n) {
      if (!wait(&item_full[n & 1], ((uint32_t)n >> 1) & 1u)) break;
      const Item it = items[n & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_free[n & 1]);
      if (it.end) break;
      // Q waits for the last item's last S; the first V has room before
      const int jv = n > 0 ? min(it.j0 + 1, it.j1) : it.j0;
      stream(1, tiles, it.b, it.L, it.head, it.j0, jv, [](int) {});
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (dead || it.j0 >= (t ? it.e1 : it.e0)) continue;
        if (!wait(&q_free[t], (uint32_t)(loads[t] & 1) ^ 1u)) continue;
        ++loads[t];
        if (lane == 0) {  // tokens of the next request or past T may come along: rows that nobody stores
          mbar_arrive_expect_tx(&q_full[t], (uint32_t)(g.group * g.tpt) * D * 2);
          for (int h = 0; h < D / 64; ++h)
            tma_load_3d(smem_u32(smem) + (uint32_t)t * TILE + h * HALF, &qmap, h * 64, it.head * g.group, it.q0 + it.tok0 + t * g.tpt,
                        &q_full[t]);
        }
        __syncwarp();
      }
      stream(1, tiles, it.b, it.L, it.head, jv, it.j1, [](int) {});
    }
    landed(1, tiles);
    for (int t = 0; t < 2; ++t)
      if (loads[t] && !mbar_wait(&q_full[t], (uint32_t)(loads[t] - 1) & 1u, 100000000ull)) latch_status(g.status, PIFA_ERR_TIMEOUT);
  }
  } else {
    regs_raise<208>();
    // ---------------- softmax and epilogue: a row per thread ----------------
    const int t = warp >> 2, quarter = warp & 3;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t s_at = tmem + lanes + t * BN, o_at = tmem + lanes + 2 * BN + t * D;
    const float c = g.c;
    uint32_t s_ph = 0, o_ph = 0;
    const int my_tok = (quarter * 32 + lane) / g.group, h = quarter * 32 + lane - my_tok * g.group;
    for (int n = 0; !dead; ++n) {
      if (!wait(&item_full[n & 1], ((uint32_t)n >> 1) & 1u)) break;
      const Item it = items[n & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(&item_free[n & 1]);
      if (it.end) break;
      const int end = t ? it.e1 : it.e0;
      const int token = it.tok0 + t * g.tpt + my_tok;
      const bool real = my_tok < g.tpt && token < it.n;
      const int seen = real ? max(it.ahead + token, 0) : 0;
      const bool idle = !__any_sync(0xffffffffu, real);
      float m = -INFINITY, l = 0.0f;
      for (int j = it.j0; j < end; ++j) {
        if (!wait(&s_full[t], s_ph)) break;
        s_ph ^= 1u;
        if (!idle) {
          tc_fence_after();
          uint32_t v[4][32];
          // The weights of the first 64 keys with the maximum as it was, beside the search for the new one; they
          // are computed again, from S, if that has grown too far, as it does for the first keys and seldom later.
          uint64_t sum[2];
          uint32_t w[4][16];
          const uint64_t c2 = f32x2(c, c);
          auto weights = [&](int i) {  // keys 32 i to 32 i + 31
            const float mc = m > -INFINITY ? -m * c : 0.0f;
            const uint64_t mc2 = f32x2(mc, mc);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const float2 x = f32x2_parts(fma_f32x2(f32x2(__uint_as_float(v[i][2 * k]), __uint_as_float(v[i][2 * k + 1])), c2, mc2));
              const float p0 = fast_exp2(x.x), p1 = fast_exp2(x.y);
              sum[k & 1] = add_f32x2(sum[k & 1], f32x2(p0, p1));
              w[i][k] = pack<F16>(p0, p1);
            }
          };
          auto hand_over = [&](int i) {
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[2 * t + i]);
          };
          bool fresh = j == it.j0;  // no maximum yet
#pragma unroll 1
          while (true) {
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_ld_32x32b_x32(s_at + i * 32, v[i]);
            tmem_ld_wait();
            const int lim = seen - j * BN;  // keys of this tile that the row sees
            if (__any_sync(0xffffffffu, lim < BN)) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < 32; ++k) v[i][k] = i * 32 + k < lim ? v[i][k] : 0xff800000u;
            }
            float mx[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              mx[i] = fmaxf(__uint_as_float(v[i][0]), __uint_as_float(v[i][1]));
#pragma unroll
              for (int k = 2; k < 32; k += 2) mx[i] = max3(mx[i], __uint_as_float(v[i][k]), __uint_as_float(v[i][k + 1]));
            }
            const float top = max3(mx[0], mx[1], fmaxf(mx[2], mx[3]));
            if (!fresh) {
              sum[0] = sum[1] = 0;
#pragma unroll
              for (int i = 0; i < EARLY; ++i) weights(i);
              if (!__any_sync(0xffffffffu, (top - m) * c > 8.0f)) break;
            }
            fresh = false;
            const float up = fmaxf(m, top);
            const float f = m > -INFINITY ? fast_exp2((m - up) * c) : 1.0f;  // (nothing was seen before: zeros)
            m = up;
            l *= f;
            if (j > it.j0) {  // S(j) is in: so is PV(j - 1), issued before it, and O may be touched
#pragma unroll 1
              for (int i = 0; i < D / 16; ++i) {
                uint32_t o[16];
                tmem_ld_32x32b_x16(o_at + i * 16, o);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                tmem_st_32x32b_x16(o_at + i * 16, o);
              }
            }
          }
#pragma unroll
          for (int i = 0; i < EARLY; ++i) tmem_st_32x32b_x16(s_at + i * 16, w[i]);
          hand_over(0);
#pragma unroll
          for (int i = EARLY; i < 4; ++i) {
            weights(i);
            tmem_st_32x32b_x16(s_at + i * 16, w[i]);
          }
          hand_over(1);
          const float2 both = f32x2_parts(add_f32x2(sum[0], sum[1]));
          l += both.x + both.y;
        } else if (lane == 0) {
          mbar_arrive(&p_full[2 * t]);
          mbar_arrive(&p_full[2 * t + 1]);
        }
      }
      if (dead) break;
      const bool any = it.j0 < end;
      if (any) {
        if (!wait(&o_full[t], o_ph)) break;
        o_ph ^= 1u;
        tc_fence_after();
      }
      if (idle && it.parts == 1) continue;
      uint16_t* out = g.o + (int64_t)(it.q0 + token) * g.ldo + (int64_t)(it.head * g.group + h) * D;
      auto store = [&](int i, const float* x) { store_row<F16>(out + i * 32, x, g.wide); };
      if (it.parts == 1) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          uint32_t o[32];
          if (any) {
            tmem_ld_32x32b_x32(o_at + i * 32, o);
            tmem_ld_wait();
          }
          float x[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) x[k] = any && seen > 0 ? __uint_as_float(o[k]) * inv : 0.0f;
          if (real) store(i, x);
        }
      } else {
        // This piece's sums: for each 32 rows, four columns of them at a time, so that a warp's accesses are whole.
        const int w8 = t * 4 + quarter;
        float* mine = g.partial + (int64_t)it.slot * C::PART_FLOATS;
        if (!idle) {
#pragma unroll
          for (int i = 0; i < D / 32; ++i) {
            uint32_t o[32] = {};
            if (any) {
              tmem_ld_32x32b_x32(o_at + i * 32, o);
              tmem_ld_wait();
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
              __stcg(reinterpret_cast<uint4*>(mine) + (w8 * (D / 4) + i * 8 + k) * 32 + lane,
                     make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]));
          }
          __stcg(reinterpret_cast<float2*>(mine + ROWS * D) + w8 * 32 + lane, make_float2(m * c, l));
          __threadfence();
          __syncwarp();
        }
        if (lane == 0) atomicAdd(&g.plan->done, 1);
      }
    }
    // ---------------- the pieces' sums ----------------
    // Every piece has been taken by a CTA that runs, so this ends; then all warps share 32 rows x 32 columns at a time.
    // (The last warp of an item doing it alone was bound by what one SM can read.)
    const int cuts = dead ? 0 : __ldcg(&g.plan->cuts);
    if (cuts > 0) {
      const int all_done = __ldcg(&g.plan->pieces) * g.heads * 8;
      const uint64_t t0 = globaltimer_ns();
      int seen = 0;
      while (true) {
        asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(&g.plan->done) : "memory");
        if (seen >= all_done) break;
        if (globaltimer_ns() - t0 > g.timeout_ns) {
          latch_status(g.status, PIFA_ERR_TIMEOUT);
          break;
        }
        __nanosleep(40);
      }
      const bool ready = __all_sync(0xffffffffu, seen >= all_done);
      const int tasks = ready ? cuts * g.heads * 8 * (D / 32) : 0;
      for (int k = warp * (int)gridDim.x + (int)blockIdx.x; k < tasks; k += 8 * (int)gridDim.x) {
        const int i = k % (D / 32), w8 = k / (D / 32) % 8, which = k / (D / 32 * 8), head = which % g.heads;
        const Item* at = g.list + g.splits[which / g.heads];
        const int tok0 = __ldcg(&at->tok0), n_tok = __ldcg(&at->n), q0 = __ldcg(&at->q0), parts = __ldcg(&at->parts);
        const int row = w8 % 4 * 32 + lane, tok = row / g.group, h = row - tok * g.group;
        const int token = tok0 + w8 / 4 * g.tpt + tok;
        const bool real = tok < g.tpt && token < n_tok;
        if (!__any_sync(0xffffffffu, real)) continue;
        const float* from = g.partial + ((int64_t)__ldcg(&at->slot) * g.heads + head) * C::PART_FLOATS;
        const int64_t pitch = (int64_t)g.heads * C::PART_FLOATS;
        constexpr int FLIGHT = 4;  // pieces and their weights in flight
        float x[32] = {}, top = -INFINITY, all = 0.0f;
#pragma unroll 1
        for (int p0 = 0; p0 < parts; p0 += FLIGHT) {
          float2 ml[FLIGHT];
          float4 o[FLIGHT][8];
#pragma unroll
          for (int p = 0; p < FLIGHT; ++p) {
            const float* piece = from + min(p0 + p, parts - 1) * pitch;
            ml[p] = __ldcg(reinterpret_cast<const float2*>(piece + ROWS * D) + w8 * 32 + lane);
#pragma unroll
            for (int q = 0; q < 8; ++q)
              o[p][q] = __ldcg(reinterpret_cast<const float4*>(piece) + (w8 * (D / 4) + i * 8 + q) * 32 + lane);
          }
          float most = top;
#pragma unroll
          for (int p = 0; p < FLIGHT; ++p) {
            if (p0 + p >= parts) ml[p].y = 0.0f;  // a piece that is not there; nothing seen: O is zero
            if (ml[p].y != 0.0f) most = fmaxf(most, ml[p].x);
          }
          const float old = top > -INFINITY ? fast_exp2(top - most) : 0.0f;
          top = most;
          all *= old;
#pragma unroll
          for (int q = 0; q < 32; ++q) x[q] *= old;
#pragma unroll
          for (int p = 0; p < FLIGHT; ++p) {
            const float f = ml[p].y != 0.0f ? fast_exp2(ml[p].x - top) : 0.0f;
            all += ml[p].y * f;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              x[4 * q] += f * o[p][q].x;
              x[4 * q + 1] += f * o[p][q].y;
              x[4 * q + 2] += f * o[p][q].z;
              x[4 * q + 3] += f * o[p][q].w;
            }
          }
        }
        const float inv = all == 0.0f ? 0.0f : 1.0f / all;
        uint16_t* out = g.o + (int64_t)(q0 + token) * g.ldo + (int64_t)(head * g.group + h) * D + i * 32;
#pragma unroll
        for (int q = 0; q < 32; ++q) x[q] *= inv;
        if (real) store_row<F16>(out, x, g.wide);
      }
    }
  }

  // Every wait above is bounded, so every thread gets here: the tensor memory is freed after its last use.
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <bool F16, int D>
cudaError_t launch_tc(cudaLaunchConfig_t& cfg, const CUtensorMap& qmap, const CUtensorMap& kmap, const CUtensorMap& vmap, const TcArgs& g) {
  cfg.dynamicSmemBytes = Cfg<D>::SMEM;
  const cudaError_t e = pifa_allow_smem<attention_tc<F16, D>>((int)Cfg<D>::SMEM);
  return e != cudaSuccess ? e : pifa_launch_ex(&cfg, attention_tc<F16, D>, qmap, kmap, vmap, g);
}

int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }

int64_t list_bytes(int64_t T, int64_t group, int64_t B) {
  return round256((T / (2 * (BM / group)) + 1 + B + MAX_PARTS) * (int64_t)sizeof(Item));
}
constexpr int64_t kPlanBytes = MAX_PARTS / 2 * 4 + 256;  // struct Plan, then the cut items

}  // namespace

int64_t attention_tc_workspace_bytes(int64_t T, int64_t q_heads, int64_t kv_heads, int64_t dim, int64_t B) {
  const int64_t part = (dim == 64 ? Cfg<64>::PART_FLOATS : Cfg<128>::PART_FLOATS) * 4;
  return round256(kPlanBytes) + list_bytes(T, q_heads / kv_heads, B) + MAX_PARTS * part;
}

int launch_attention_tc(const PifaAttention& a, int* status, uint64_t timeout_ns, cudaStream_t stream) {
  TcArgs g = {};
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  const int64_t group = a.q_heads / a.cache.heads;
  g.o = static_cast<uint16_t*>(a.o);
  g.table = a.table;
  g.q_start = a.q_start;
  g.kv_len = a.kv_len;
  g.plan = reinterpret_cast<Plan*>(ws);
  g.splits = reinterpret_cast<int*>(ws + 256);
  g.list = reinterpret_cast<Item*>(ws + round256(kPlanBytes));
  g.partial = reinterpret_cast<float*>(ws + round256(kPlanBytes) + list_bytes(a.T, group, a.B));
  g.ldo = a.ldo;
  g.ldt = a.ldt;
  g.pages = a.cache.pages;
  g.T = (int)a.T;
  g.heads = (int)a.cache.heads;
  g.group = (int)group;
  g.tpt = BM / g.group;
  g.B = (int)a.B;
  g.max_q = (int)(a.max_q < a.T ? a.max_q : a.T);
  g.cols = (int)a.cols;
  g.page_size = (int)a.cache.page_size;
  while ((1 << g.page_shift) < g.page_size) ++g.page_shift;
  g.negate = a.scale_log2 < 0.0f;
  g.wide = ((reinterpret_cast<uintptr_t>(a.o) | (uintptr_t)(a.ldo * 2)) & 31u) == 0;
  // equal weights for a scale of zero: the masked scores, -inf, still have to vanish
  g.c = a.scale_log2 == 0.0f ? 1e-30f : std::fabs(a.scale_log2);
  g.status = status;
  g.timeout_ns = timeout_ns;
  CUtensorMap qmap, kmap, vmap;
  int order[3], st;
  const uint32_t rows = (uint32_t)(a.cache.page_size < BN ? a.cache.page_size : BN);
  if ((st = make_tmap_heads(&qmap, a.dtype, a.q, a.T, a.q_heads, a.cache.dim, a.ldq, (uint32_t)group, (uint32_t)g.tpt)) != PIFA_OK)
    return st;
  if ((st = make_tmap_cache(&kmap, a.dtype, a.k, a.cache, rows, order)) != PIFA_OK) return st;
  if ((st = make_tmap_cache(&vmap, a.dtype, a.v, a.cache, rows, order)) != PIFA_OK) return st;
  g.token_at = order[0];
  g.head_at = order[1];
  const int grid = pifa_sm_count();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1);
  cfg.blockDim = dim3(PLAN_THREADS);
  cfg.dynamicSmemBytes = (size_t)a.B * sizeof(Lengths) + (size_t)(a.B + 1) * 4;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  cudaError_t e = pifa_allow_smem<attention_plan>((int)(4096 * sizeof(Lengths) + 4097 * 4));
  if (e != cudaSuccess) return pifa_fail_cuda("cudaFuncSetAttribute(attention_plan)", e);
  e = pifa_launch_ex(&cfg, attention_plan, g, grid);
  if (e != cudaSuccess) return pifa_fail_cuda("attention_plan launch", e);
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(THREADS);
  const bool f16 = a.dtype == PIFA_DTYPE_FP16;
  if (a.cache.dim == 64) e = f16 ? launch_tc<true, 64>(cfg, qmap, kmap, vmap, g) : launch_tc<false, 64>(cfg, qmap, kmap, vmap, g);
  else e = f16 ? launch_tc<true, 128>(cfg, qmap, kmap, vmap, g) : launch_tc<false, 128>(cfg, qmap, kmap, vmap, g);
  if (e != cudaSuccess) return pifa_fail_cuda("attention_tc launch", e);
  return PIFA_OK;
}
