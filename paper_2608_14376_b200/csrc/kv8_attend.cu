// Attention over the 8-bit cache (include/corun_kv8.h): out = softmax(scale q K^T) V, and the weights that the cached tokens
// received, on tcgen05 / TMEM / TMA (sm_100a) straight from the 8-bit pages.
//
// The cached tokens are the M side of both products and the query columns (query tokens x query heads of a key head, at most
// 32) the N side, so that the cache's bytes are MMA operands as they lie in memory: no value of K or V passes
// through a register.  With C columns:
//   scores   S^T [128 tokens x 2 or 3 C] = K [128 x hd] * Q^T   K K-major, 32 values of a row per MMA
//   output   O^T [hd x 3 C]              = V^T [hd x 128] * P^T V read as the MN-major A operand
// kind::f8f6f4 wants 8-bit operands on both sides.  A query or a weight is the sum of e4m3 values, x = h0 + h1 / 16 + h2 / 256, each
// the rounding of what the ones before left (4 bits each), and takes a column for each: a bf16 query two (8 bits, exact), an fp16 query three
// (11 bits, exact), a weight three, which leave 2^-12 of it at most and 2^-16 rms.  With few columns an MMA costs the same whatever N is, so they
// are free.  Queries are brought to [128, 256) by a power of two per column, weights to at most 256: what lies below 2^-26 of the largest
// one of its column and tile is lost.  (Rounding the weights to fp16 first, whose pairs take fewer instructions: 73.7 us instead of 74.0 below, and
// 16 times as many outputs that are not the nearest ones.)
// The scales 2^e of a token's keys multiply its scores.  Those of its values go into its weight: the product takes
// w = 2^(s + e_v - M), M the largest s + e_v of the column in the tile, so that what is rounded is rounded relative to its
// share in the result; the sum of weights takes w 2^-e_v back.  (Exponents lie in [-32, 31]: neither leaves the range of 32 bits.)
// A tile's output stays in its own frame M; it is added to the running output, held in registers, in 32 bits.
//
// An item is (row, key head, split).  Rows with n G <= 32 columns are split into parts (at_splits); rows with more columns are
// kv8_chunk.cu's.  The split depends on the row's own ctx, n and window alone, sums have one fixed order, and which CTA computes an item
// has no influence on any value: a row's result does not depend on the other rows.  Every CTA (one per SM) takes a stretch of the
// item list, cut by cost.
//   warps 0, 3    producers of the even / odd tiles: block-table lookups, TMA loads, exponents
//   warp 1        issues the MMAs: whichever product can go on, an output product first
//   warp 2        query tiles, up to two ahead
//   warps 4-7, 8-11   softmax of even / odd tiles, a thread per cached token
//   warps 12-15   output: a thread per value dim
// A second kernel combines a row's splits in ascending order, a third one adds up the weights from the scores that the
// first wrote (4 bytes per token and column, where mass is wanted).  Every wait is bounded.
//
// Bound by the cache's bytes.  64 rows of 512 to 4096 tokens (32 query, 8 key heads of 128, pages of 16): 74 us, of which this kernel 67
// (50 at the copy rate) and the combine 6.6.  In the middle of a launch a tile of 32 KiB takes an SM 1430 to 1450 cycles, which is the
// copy rate; the rest is launch, the first tiles (all SMs ask for six at once: the first arrives after 5000 to 13000 cycles), and the
// last tile's chain of some 4000.  Two rows of 90 K tokens, 4 key heads, pages of 64: 47 us (29 at the copy rate).
// What brought it there, same case of 64 rows: 121 us with one producer warp and a box each for keys and values; 108 with page numbers and
// exponents in batches ahead of their use; 90 without integer divisions on the way to the next item (400 to 800 cycles a role); 76 with
// keys and values of a page in one box (a TMA instruction takes some 70 cycles to issue); 74 with two producers, six tiles in flight and the
// scores two tiles ahead.
#include <stddef.h>

#include <atomic>
#include <type_traits>

#include <math_constants.h>

#include "kv8_attend.cuh"

namespace corun {
namespace {

constexpr int AT_THREADS = 512;
static_assert(AT_MAXB <= AT_THREADS, "a thread plans a row");
constexpr int AT_SPLITS = 128;      // splits of a row at most
constexpr int AT_MIN_TILES = 2;     // tiles of a split at least
// Tiles (keys and values) in shared memory: as many as fit beside the columns' operands.
__host__ __device__ constexpr int at_ring(int C) { return C > 16 ? 4 : C > 8 ? 5 : 6; }

// What a row asks for: its new tokens (0 = left out), the tiles [t_lo, t_hi) it reads, its splits (0 = not this kernel's).
struct RowPlan {
  int c, n, first, t_lo, t_hi, ns;
};
__device__ __forceinline__ int at_lo(int c, int n, int window) { return window ? max(0, c - n - window + 1) / AT_T : 0; }
// Splits of a row that reads `tiles` tiles: two tiles each or more, and where one row's splits alone fill the SMs, a whole number
// of rounds of them (two rows of 100003 tokens and 4 key heads: 3 rounds of 37 * 4 splits of 7 or 8 tiles each).  The s-th split
// begins floor(tiles * s / ns) tiles behind t_lo.
__host__ __device__ inline int at_splits(int tiles, int n_kv, int sms) {
  int ns = tiles / AT_MIN_TILES;
  ns = ns < 1 ? 1 : ns > AT_SPLITS ? AT_SPLITS : ns;
  const int rounds = (int)((long long)ns * n_kv / sms);
  return rounds > 0 ? (rounds * sms / n_kv > 0 ? rounds * sms / n_kv : 1) : ns;
}
__device__ __forceinline__ RowPlan row_plan(int c, int first, int end, const AttendArgs &a, int G) {
  RowPlan r;
  r.c = c;
  r.first = first;
  r.n = end - first;
  if (!at_row_ok(c, first, end, a)) { r.n = 0; r.ns = 0; r.t_lo = r.t_hi = 0; return r; }
  r.t_lo = at_lo(c, r.n, a.window);
  r.t_hi = (c + AT_T - 1) / AT_T;
  r.ns = (long long)r.n * G <= AT_MAXC ? at_splits(r.t_hi - r.t_lo, a.n_kv, a.sms) : 0;
  return r;
}

// Sums over the lanes of N values each, the columns shared out on the way: lane i ends up with the sum of column i >> (5 - log2 N).
template <int N>
__device__ __forceinline__ float lane_sums(float (&v)[N], int lane) {
  int off = 16;
#pragma unroll
  for (int n = N; n > 1; n >>= 1, off >>= 1) {
    const bool up = lane & off;
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
      const float give = up ? v[i] : v[i + n / 2], keep = up ? v[i + n / 2] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, off);
    }
  }
  float s = v[0];
  for (; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
  return s;
}
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Descriptor of a tile whose rows of W bytes (128 or 64, swizzled by that width) come in groups of eight, `group` bytes
// apart.  It serves K-major operands (rows = M or N) and, with W values of the M index in a row, MN-major ones (rows = K) alike: the
// stride byte offset is the distance of the groups in both.
template <int W>
__device__ __forceinline__ uint64_t desc_rows(uint32_t smem_addr, uint32_t group) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr >> 4) & 0x3FFFu);
  d |= (uint64_t)1u << 16;
  d |= (uint64_t)(group >> 4) << 32;
  d |= (uint64_t)1u << 46;
  d |= (uint64_t)(W == 128 ? 2u : 4u) << 61;
  return d;
}
// Byte b of row r of a swizzled tile with rows of W bytes (128: chunk ^ row mod 8, 64: chunk ^ row / 2 mod 4).
template <int W>
__device__ __forceinline__ uint32_t swz(int r, int b) {
  return W == 128 ? (uint32_t)(r * 128 + ((((b >> 4) ^ (r & 7)) << 4) | (b & 15))) : (uint32_t)(r * 64 + ((((b >> 4) ^ ((r >> 1) & 3)) << 4) | (b & 15)));
}

template <int C>
struct Smem {
  static constexpr int RING = at_ring(C), EXPS = 2 * RING;         // EXPS: tiles whose exponents are held
  uint64_t full[RING], empty[RING], e_full[EXPS];
  uint64_t q_ready[2], q_free[2], s_full[2], s_free[2], p_ready[2], o_full[2], o_free[2], x_bar[2], l_ready[2], l_free[2];
  uint32_t tmem;
  int abort_flag;
  struct { int lo, hi, row, g, split, t0, acc; } mine;   // this CTA's items, where the first one is
  float q_mul[4][C];                 // 2^e of a query column times scale log2(e), by query tile
  alignas(16) float x_max[2][2][C][4];   // (read as float4) [group][use parity][column][warp]: maxima of 32 tokens
  float frame[2][C];                 // [tile parity]: the tile's frames
  float4 ab[12][C];                  // [warp - 4]: factors of old and new of every column, the tile's frame
  float lpart[2][8][C];              // [item parity][group * 4 + warp]: sums of weights
  float lframe[2][2][C];             // [item parity][group]: their frames
  int flags[EXPS];                   // [tile] 1: a new query tile, 2: the stretch's last tile
  int8_t exps[EXPS][2][8];           // [tile][kind][page of the tile]
  int row_item[AT_MAXB + 1];         // first item of every row
  int row_c[AT_MAXB], row_first[AT_MAXB], row_n[AT_MAXB];
  int warp_items[AT_THREADS / 32];
  long long warp_cost[AT_THREADS / 32];
};

// Columns of a product with `pieces` columns per query column: an M = 128 MMA takes N in steps of 16.
__host__ __device__ constexpr int at_n(int pieces, int C) { return (pieces * C + 15) / 16 * 16; }
// A bf16 query is two e4m3 values exactly (8 bits), an fp16 query three (11 bits).
template <typename T> __host__ __device__ constexpr int q_pieces() { return std::is_same<T, __nv_bfloat16>::value ? 2 : 3; }
template <typename T, int HD, int C>
__host__ __device__ constexpr int q_bytes() { return (at_n(q_pieces<T>(), C) * HD + 1023) / 1024 * 1024; }
template <typename T, int HD, int C>
constexpr int smem_bytes() { return 2 * at_ring(C) * AT_T * HD + 2 * q_bytes<T, HD, C>() + 2 * at_n(3, C) * AT_T + (int)sizeof(Smem<C>) + 1024; }

template <typename T, int HD, int C>
__global__ void __launch_bounds__(AT_THREADS, 1) attend_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ AttendArgs a) {
  constexpr int QP = q_pieces<T>(), NQ = at_n(QP, C), N = at_n(3, C);   // columns of the scores and of the output
  constexpr int RING = at_ring(C), EXPS = 2 * RING, GROUP = 8 * HD, TILE = 2 * AT_T * HD, Q_TILE = q_bytes<T, HD, C>();
  constexpr int COLS = 2 * NQ + 2 * N;
  constexpr uint32_t TMEM_COLS = COLS <= 64 ? 64 : COLS <= 128 ? 128 : COLS <= 256 ? 256 : 512;
  static_assert(offsetof(Smem<C>, x_max) % 16 == 0 && offsetof(Smem<C>, ab) % 16 == 0 && alignof(Smem<C>) >= 16, "read 16 bytes at a time");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *base_ptr = smem_raw + (base - smem_u32(smem_raw));
  // [ring of tiles][two query tiles][two weight tiles][the rest], tiles on 1 KiB.  A tile of 128 tokens: eight rows of keys, eight
  // rows of values, the next eight of keys, ...: a page's keys and values come with one box, and the groups of either are at
  // one distance throughout (the TMA instruction takes some 70 cycles to issue: the fewer boxes the better)
  const uint32_t ring = base, q_tile = base + RING * TILE, p_tile = q_tile + 2 * Q_TILE;
  uint8_t *q_ptr = base_ptr + (q_tile - base), *p_ptr = base_ptr + (p_tile - base);
  Smem<C> &sm = *reinterpret_cast<Smem<C> *>(p_ptr + 2 * N * AT_T);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = a.n_q / a.n_kv, shift = a.block == 16 ? 4 : a.block == 32 ? 5 : 6;

  if (tid == 0) {
    sm.abort_flag = 0;
    for (int s = 0; s < RING; ++s) { mbar_init(smem_u32(&sm.full[s]), 1); mbar_init(smem_u32(&sm.empty[s]), 1); }
    for (int s = 0; s < EXPS; ++s) mbar_init(smem_u32(&sm.e_full[s]), 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&sm.s_full[s]), 1); mbar_init(smem_u32(&sm.s_free[s]), 4);
      mbar_init(smem_u32(&sm.p_ready[s]), 4);
      mbar_init(smem_u32(&sm.o_full[s]), 1); mbar_init(smem_u32(&sm.o_free[s]), 4);
      mbar_init(smem_u32(&sm.q_ready[s]), 1); mbar_init(smem_u32(&sm.q_free[s]), 1);
      mbar_init(smem_u32(&sm.x_bar[s]), 4);
      mbar_init(smem_u32(&sm.l_ready[s]), 8); mbar_init(smem_u32(&sm.l_free[s]), 4);
    }
    fence_mbar_init();
    fence_proxy_async();
    prefetch_tensormap(&tm);
  }
  if (warp == 0) {
    tmem_alloc(smem_u32(&sm.tmem), TMEM_COLS);
    tmem_relinquish();
  } else if (warp >= 4) {
    // operand rows that no column writes stay zero
    uint4 *z = reinterpret_cast<uint4 *>(q_ptr);
    for (int i = tid - 128; i < (int)(p_tile - q_tile + 2 * N * AT_T) / 16; i += AT_THREADS - 128) z[i] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async();
  }
  // (programmatic launch) everything above reads nothing that another kernel writes
  griddep_wait();
  // the item list: a thread plans a row; items and their cost before every row by a sum over the threads
  {
    int items = 0, ic = 1, ns = 0, lo = 0, tiles = 0;
    if (tid < a.B) {
      const int first = a.cu ? __ldcg(a.cu + tid) : tid, end = a.cu ? __ldcg(a.cu + tid + 1) : tid + 1, ctx = __ldcg(a.ctx + tid);
      const RowPlan p = row_plan(ctx, first, end, a, G);
      sm.row_c[tid] = ctx; sm.row_first[tid] = first; sm.row_n[tid] = p.n;
      ns = p.ns;
      lo = p.t_lo;
      tiles = p.t_hi - p.t_lo;
      items = ns * a.n_kv;                            // 0 for a row that is left out
      ic = ns ? 1 + (2 * tiles + ns - 1) / ns : 1;    // a tile's cost is 2, an item's beyond its tiles 1
    }
    const long long cost = (long long)items * ic;
    int inc = items;
    long long cinc = cost;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, inc, o);
      const long long cv = __shfl_up_sync(0xffffffffu, cinc, o);
      if (lane >= o) { inc += v; cinc += cv; }
    }
    if (lane == 31) { sm.warp_items[warp] = inc; sm.warp_cost[warp] = cinc; }
    __syncthreads();
    int all = 0;
    long long call = 0;
    inc -= items;
    cinc -= cost;
    for (int w = 0; w < AT_THREADS / 32; ++w) {
      if (w < warp) { inc += sm.warp_items[w]; cinc += sm.warp_cost[w]; }
      all += sm.warp_items[w];
      call += sm.warp_cost[w];
    }
    if (tid < a.B) sm.row_item[tid] = inc;
    if (tid == 0) sm.row_item[a.B] = all;
    // a CTA's stretch: from the first item that starts at or behind blockIdx / gridDim of all cost, to the next CTA's
    const long long from = (call * blockIdx.x + gridDim.x - 1) / gridDim.x, to = (call * (blockIdx.x + 1) + gridDim.x - 1) / gridDim.x;
    if (tid == 0 && from == 0) sm.mine.lo = 0;
    if (tid == 0 && to == 0) sm.mine.hi = 0;
    if (cinc < from && from <= cinc + cost) sm.mine.lo = inc + (int)((from - cinc + ic - 1) / ic);
    if (cinc < to && to <= cinc + cost) sm.mine.hi = inc + (int)((to - cinc + ic - 1) / ic);
    __syncthreads();
    const int i = sm.mine.lo - inc;
    if (i >= 0 && i < items) {                        // where the first item is
      const int split = i % ns, size = tiles / ns, rest = tiles - size * ns;
      sm.mine.row = tid;
      sm.mine.g = i / ns;
      sm.mine.split = split;
      sm.mine.t0 = lo + size * split + (rest * split) / ns;
      sm.mine.acc = (rest * split) % ns;
    }
  }
  // the next kernel's blocks may come up beside this one's and wait for its end (all CTAs of this grid run at once)
  griddep_launch_dependents();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t s_tmem = sm.tmem, o_tmem = s_tmem + 2 * NQ;
  const int item_lo = sm.mine.lo, item_hi = sm.mine.hi;
  bool failed = false;
  // Where a role is in the CTA's stretch: the item (row b, key head g, split) and its tiles [t0, t1).  Going on to the next item takes
  // additions only (a division here would cost every role some hundred cycles an item).
  struct Cursor { int it, b, g, split, ns, size, rest, acc, c, n, first, t_lo, t_hi, t0, t1; bool new_query; } x = {};
  // tiles of a split: size, and one more where the remainders add up
  auto row_at = [&]() {
    x.c = sm.row_c[x.b]; x.n = sm.row_n[x.b]; x.first = sm.row_first[x.b];
    x.ns = (sm.row_item[x.b + 1] - sm.row_item[x.b]) / a.n_kv;
    x.t_lo = at_lo(x.c, x.n, a.window);
    x.t_hi = (x.c + AT_T - 1) / AT_T;
    x.size = (x.t_hi - x.t_lo) / x.ns;
    x.rest = (x.t_hi - x.t_lo) - x.size * x.ns;
  };
  auto tiles_at = [&]() {
    x.acc += x.rest;
    const bool one_more = x.acc >= x.ns;
    if (one_more) x.acc -= x.ns;
    x.t1 = x.t0 + x.size + (one_more ? 1 : 0);
  };
  x.it = item_lo;
  x.new_query = true;
  if (item_lo < item_hi) {
    x.b = sm.mine.row;
    row_at();
    x.g = sm.mine.g;
    x.split = sm.mine.split;
    x.t0 = sm.mine.t0;
    x.acc = sm.mine.acc;
    tiles_at();
  }
  auto next_item = [&]() {
    ++x.it;
    if (x.t1 < x.t_hi) {                              // the next split
      ++x.split;
      x.new_query = false;
      x.t0 = x.t1;
    } else {
      x.split = x.acc = 0;
      x.new_query = true;
      if (++x.g == a.n_kv) {
        x.g = 0;
        if (x.it < item_hi) {
          do ++x.b; while (sm.row_item[x.b + 1] == x.it);
          row_at();
        }
      }
      x.t0 = x.t_lo;
    }
    tiles_at();
  };
  auto wait_all = [&](uint64_t &bar, uint32_t parity) {   // by a whole warp
    const bool ok = mbar_wait(smem_u32(&bar), parity & 1u, &sm.abort_flag);
    if (!__all_sync(0xffffffffu, ok)) failed = true;
    return !failed;
  };

  if (warp == 0 || warp == 3) {
    // ---------------- producers ----------------
    // Each warp walks over all tiles and takes every other one, in batches of four, eight lanes a tile and a page a lane: while a
    // batch is loaded, the exponents of the next one and the page numbers of the one after are on their way.
    const uint64_t pol = l2_policy_evict_normal();
    const int per = AT_T >> shift;                    // pages of a tile
    struct Batch { int cnt, np, g, flags, page, ek, ev; };   // tiles; of the lane's tile: pages, key head, flags; of its page: number, exponents
    int t = x.t0, n = 0;
    auto step = [&]() {
      ++n;
      if (++t >= x.t1) { next_item(); t = x.t0; }
    };
    if (warp == 3 && x.it < item_hi) step();
    auto pages = [&](Batch &q) {
      q.cnt = q.np = q.g = q.flags = q.ek = q.ev = 0;
      const int *src = nullptr;
      for (; q.cnt < 4 && x.it < item_hi; ++q.cnt) {
        const bool fresh = x.new_query && t == x.t0, last = x.it + 1 == item_hi && t + 1 == x.t1;
        if ((lane >> 3) == q.cnt) {
          q.np = min(per, (x.c - t * AT_T + a.block - 1) >> shift);
          q.g = x.g;
          q.flags = (fresh ? 1 : 0) | (last ? 2 : 0);
          if ((lane & 7) < q.np) src = a.block_table + (size_t)x.b * a.max_blocks + (size_t)t * per + (lane & 7);
        }
        step();
        if (x.it < item_hi) step();
      }
      q.page = -1;
      if (src) q.page = load_now(src);
    };
    auto exponents = [&](Batch &q) {
      if (q.page >= 0 && (long long)q.page < a.pages) {
        const long long at = ((long long)q.page * 2) * a.n_kv + q.g;
        q.ek = load_now(a.exps + at);
        q.ev = load_now(a.exps + at + a.n_kv);
      }
    };
    auto load = [&](const Batch &q, int i, int tile) {   // the keys and values of the batch's i-th tile
      const int s = tile % RING;
      if (tile >= RING && !wait_all(sm.empty[s], (uint32_t)(tile / RING - 1))) return;
      const bool mine = (lane >> 3) == i;
      if (mine && (lane & 7) == 0) {
        sm.flags[tile % EXPS] = q.flags;
        mbar_arrive_expect_tx(smem_u32(&sm.full[s]), (uint32_t)(q.np * a.block * 2 * HD));
      }
      __syncwarp();
      const bool page_ok = q.page >= 0 && (long long)q.page < a.pages;
      const int page = page_ok ? q.page : (int)a.pages;                // behind the pool: a page outside of it reads as zeros
      if (mine && (lane & 7) < q.np)
        tma_load_5d(ring + (uint32_t)(s * TILE + (lane & 7) * a.block * 2 * HD), &tm, 0, 0, 0, q.g * (a.block >> 3), page,
                    smem_u32(&sm.full[s]), pol);
    };
    Batch b0, b1, b2;
    pages(b0);
    int m = warp == 3 ? 1 : 0, ahead = 0;             // the tile that is next; tiles of b0 that are on their way already
    exponents(b0);
    for (; ahead < b0.cnt && m + 2 * ahead < RING; ++ahead) load(b0, ahead, m + 2 * ahead);   // into free slots: before anything else is looked up
    pages(b1);
    while (b0.cnt > 0 && !failed) {
      exponents(b1);
      pages(b2);
      for (int i = 0; i < b0.cnt && !failed; ++i, m += 2) {
        if (i >= ahead) load(b0, i, m);
        if (failed) break;
        // (the tile RING before this one has been through its output product, so the exponents twice as far back have been read)
        const int e = m % EXPS;
        if ((lane >> 3) == i) { sm.exps[e][0][lane & 7] = (int8_t)b0.ek; sm.exps[e][1][lane & 7] = (int8_t)b0.ev; }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.e_full[e]));
      }
      ahead = 0;
      b0 = b1;
      b1 = b2;
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer ----------------
    if (elect_one()) {
      // D fp32, A and B e4m3 (format 0); scores: M = 128; output: M = hd, A MN-major
      const uint32_t idesc_s = (1u << 4) | ((uint32_t)(NQ >> 3) << 17) | ((uint32_t)(AT_T >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (1u << 15) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(HD >> 4) << 24);
      auto is_done = [&](uint64_t &bar, int phase) { return mbar_test(smem_u32(&bar), (uint32_t)phase & 1u); };
      // Whichever product can go on goes on: an output product as soon as its weights are there (it frees a slot of the ring), else
      // the scores of the next tile.  The order has no influence on any value.
      int nq = 0, no = 0, n_query = 0;                // tiles whose scores / outputs have been issued, query tiles
      bool more = item_lo < item_hi;
      uint32_t idle = 0;
      uint64_t idle_from = 0;
      while (more || no < nq) {
        bool did = false;
        if (no < nq && is_done(sm.p_ready[no & 1], no / 2) && (no < 2 || is_done(sm.o_free[no & 1], no / 2 - 1))) {
          const int s = no % RING, h = no & 1;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < AT_T / 32; ++k) {
            const uint64_t da = desc_rows<HD>(ring + (uint32_t)(s * TILE + GROUP + k * 8 * GROUP), 2 * GROUP);
            const uint64_t db = umma_desc_sw128(p_tile + (uint32_t)(h * N * AT_T)) + (uint64_t)(k * 2);
            umma_f8(o_tmem + (uint32_t)(h * N), da, db, idesc_o, k > 0 ? 1u : 0u);
          }
          umma_commit(smem_u32(&sm.o_full[h]));
          umma_commit(smem_u32(&sm.empty[s]));
          ++no;
          did = true;
        }
        if (more && (nq < 2 || is_done(sm.s_free[nq & 1], nq / 2 - 1)) && is_done(sm.full[nq % RING], nq / RING)) {
          const int s = nq % RING, h = nq & 1, flags = sm.flags[nq % EXPS];
          if (!(flags & 1) || is_done(sm.q_ready[n_query & 1], n_query / 2)) {
            if (flags & 1) {
              if (n_query > 0) umma_commit(smem_u32(&sm.q_free[(n_query - 1) & 1]));   // the scores with the query tile before have been issued
              ++n_query;
            }
            more = !(flags & 2);
            const uint32_t q_at = q_tile + (uint32_t)((n_query - 1) & 1) * Q_TILE;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < HD / 32; ++k)
              umma_f8(s_tmem + (uint32_t)(h * NQ), desc_rows<HD>(ring + (uint32_t)(s * TILE), 2 * GROUP) + (uint64_t)(k * 2),
                      desc_rows<HD>(q_at, GROUP) + (uint64_t)(k * 2), idesc_s, k > 0 ? 1u : 0u);
            umma_commit(smem_u32(&sm.s_full[h]));
            ++nq;
            did = true;
          }
        }
        if (did) {
          idle = 0;
        } else if ((++idle & 255u) == 0u) {            // bounded, as every wait
          const uint64_t now = globaltimer_ns();
          if (idle == 256u) idle_from = now;
          if (*(volatile int *)&sm.abort_flag) { failed = true; break; }
          if (now - idle_from > 2000000000ull) { *(volatile int *)&sm.abort_flag = 1; failed = true; break; }
        }
      }
    }
  } else if (warp == 2) {
    // ---------------- query tile ----------------
    // row piece * C + column, hd bytes, swizzled as the keys are; a warp per column, hd / 32 values a lane
    constexpr int EPL = HD / 32;
    int n_q = 0;
    for (; x.it < item_hi && !failed; next_item()) {
      if (!x.new_query) continue;
      if (n_q > 1 && !wait_all(sm.q_free[n_q & 1], (uint32_t)(n_q / 2 - 1))) break;
      uint8_t *q_at = q_ptr + (n_q & 1) * Q_TILE;
      const int cols = x.n * G;
      for (int c = 0; c < cols; ++c) {
        const T *src = (const T *)a.q + (long long)(x.first + c / G) * a.q_t + (long long)(x.g * G + c % G) * a.q_h + lane * EPL;
        float v[EPL];
        if (EPL == 4) {
          const uint2 u = __ldcg(reinterpret_cast<const uint2 *>(src));
          const T *e = reinterpret_cast<const T *>(&u);
#pragma unroll
          for (int i = 0; i < EPL; ++i) v[i] = to_f32(e[i]);
        } else {
          const uint32_t u = __ldcg(reinterpret_cast<const uint32_t *>(src));
          const T *e = reinterpret_cast<const T *>(&u);
#pragma unroll
          for (int i = 0; i < EPL; ++i) v[i] = to_f32(e[i]);
        }
        float mx = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          if (!(fabsf(v[i]) <= 3.4e38f)) v[i] = CUDART_NAN_F;        // an infinite query makes its scores NaN
          mx = fmaxf(mx, fabsf(v[i]));
        }
        mx = warp_max(mx);
        // to [128, 256): e from the exponent bits (a subnormal maximum counts as 2^-126)
        const int e = max((__float_as_int(mx) >> 23) - 127, -110) - 7;
        const float down = pow2f(-e > 126 ? 126 : -e);
        uint32_t w[QP] = {};
#pragma unroll
        for (int i = 0; i < EPL; i += 2) {
          float r0 = v[i] * down, r1 = v[i + 1] * down;
#pragma unroll
          for (int p = 0; p < QP; ++p) {
            const uint32_t h = e4m3x2_of(r0, r1);
            const float2 f = e4m3x2_to(h);
            r0 = (r0 - f.x) * 16.f;
            r1 = (r1 - f.y) * 16.f;
            w[p] |= h << (8 * i);
          }
        }
#pragma unroll
        for (int p = 0; p < QP; ++p) {
          uint8_t *dst = q_at + swz<HD>(p * C + c, lane * EPL);
          if (EPL == 4) *reinterpret_cast<uint32_t *>(dst) = w[p]; else *reinterpret_cast<uint16_t *>(dst) = (uint16_t)w[p];
        }
        if (lane == 0) sm.q_mul[n_q & 3][c] = (mx > 0.f ? pow2f(e) : 1.f) * a.scale_log2e;
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.q_ready[n_q & 1]));
      ++n_q;
    }
  } else if (warp < 12) {
    // ---------------- softmax: group 0 takes the even tiles, group 1 the odd ones ----------------
    const int grp = warp >= 8 ? 1 : 0, wq = warp & 3, tok = wq * 32 + lane, pg = tok >> shift;
    const uint32_t s_lane = s_tmem + ((uint32_t)(32 * wq) << 16) + (uint32_t)(grp * NQ);
    float4 *ab = sm.ab[warp - 4];
    float l[C];
    float m_run = AT_LOW;                             // lane c: the running frame of column c
    int n = 0, n_q = -1, k = 0;                       // k: tiles this group has done
    for (; x.it < item_hi && !failed; next_item()) {
      if (x.new_query) ++n_q;
      const int cols = x.n * G;
#pragma unroll
      for (int c = 0; c < C; ++c) l[c] = 0.f;
      m_run = AT_LOW;
      const int lim0 = x.c - x.n, lim1 = x.c - 1;          // last index that the first and the last new token see
      for (int t = x.t0; t < x.t1 && !failed; ++t, ++n) {
        if ((n & 1) != grp) continue;
        const int j = t * AT_T + tok;
        if (!wait_all(sm.e_full[n % EXPS], (uint32_t)(n / EXPS))) break;
        const float ek = pow2f(sm.exps[n % EXPS][0][pg]);
        const int ev_i = sm.exps[n % EXPS][1][pg];
        const float ev = (float)ev_i;
        if (!wait_all(sm.s_full[grp], (uint32_t)k)) break;
        tc_fence_after();
        const bool masked = (t + 1) * AT_T > lim0 + 1 || (a.window && t * AT_T <= lim1 - a.window);
        const float *qm = sm.q_mul[n_q & 3];
        float y[C];
        float *sc = a.mass ? a.scores + (((long long)x.b * a.n_kv + x.g) * a.score_tokens + j) * a.cols : nullptr;
        bool unseen = true;                           // no column sees the token
#pragma unroll
        for (int c0 = 0; c0 < C; c0 += 16) {
          constexpr int W = C < 16 ? C : 16, LD = C == 4 ? 16 : QP * W;
          uint32_t v[LD];
          if (C == 4) {
            tmem_ld8(s_lane, *reinterpret_cast<uint32_t(*)[8]>(&v[0]));
            if (QP == 3) tmem_ld8(s_lane + 8, *reinterpret_cast<uint32_t(*)[8]>(&v[8]));
          } else if (C == 8) {
#pragma unroll
            for (int p = 0; p < QP; ++p) tmem_ld8(s_lane + (uint32_t)(p * C), *reinterpret_cast<uint32_t(*)[8]>(&v[p * W]));
          } else {
#pragma unroll
            for (int p = 0; p < QP; ++p) tmem_ld16(s_lane + (uint32_t)(p * C + c0), *reinterpret_cast<uint32_t(*)[16]>(&v[(p * W) % LD]));
          }
          tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < W; ++c) {
            float s = __uint_as_float(v[(QP - 1) * W + c]);
#pragma unroll
            for (int p = QP - 2; p >= 0; --p) s = fmaf(s, 1.f / 16.f, __uint_as_float(v[p * W + c]));
            y[c0 + c] = s * (ek * qm[c0 + c]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.s_free[grp]));
        if (masked) {
          int h = 0, lim = lim0;
#pragma unroll
          for (int c = 0; c < C; ++c) {
            const bool see = j <= lim && !(a.window && j <= lim - a.window);
            if (c < cols && see) unseen = false;
            if (!see) y[c] = -CUDART_INF_F;
            if (++h == G) { h = 0; ++lim; }
          }
        } else {
          unseen = false;
        }
        if (sc) {
#pragma unroll
          for (int c = 0; c < C; c += 4) {
            if ((a.cols & 3) == 0) {
              if (c < cols) *reinterpret_cast<float4 *>(sc + c) = make_float4(y[c], y[c + 1], y[c + 2], y[c + 3]);   // (a column behind the row's own is not read)
            } else {
#pragma unroll
              for (int e = c; e < c + 4; ++e)
                if (e < cols) sc[e] = y[e];
            }
          }
        }
        // the tile's frame: the largest s + e_v of every column
        float (*xm)[4] = sm.x_max[grp][k & 1];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          y[c] += ev;
          const float mx = warp_max(y[c]);
          if (lane == 0) xm[c][wq] = mx;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.x_bar[grp]));
        if (!wait_all(sm.x_bar[grp], (uint32_t)k)) break;
        // lane c: the column's frame and what the running sum and this tile's are multiplied by
        float m_tile = AT_LOW;
        if (lane < C) {
          const float4 f = *reinterpret_cast<const float4 *>(xm[lane]);
          m_tile = fmaxf(fmaxf(fmaxf(f.x, f.y), fmaxf(f.z, f.w)), AT_LOW);
          const float m_new = fmaxf(m_run, m_tile);
          // (beyond 2^27 in magnitude the subtraction may take 16 away, and 2^16 would be beyond fp16: weights up to 1 then)
          const float low = m_tile - 8.f;
          ab[lane] = make_float4(ex2(m_run - m_new), ex2(m_tile - m_new), m_tile - low > 9.f ? m_tile : low, 0.f);
          m_run = m_new;
        }
        // the frames of the group's tile before must have been read; its output product, and so its weights, then too
        if (k > 0 && !wait_all(sm.o_free[grp], (uint32_t)(k - 1))) break;
        if (wq == 0 && lane < C) sm.frame[grp][lane] = m_tile;
        __syncwarp();
        uint8_t *p_row = p_ptr + grp * N * AT_T;
        const float back = pow2f(-ev_i);
#pragma unroll
        for (int c = 0; c < C; c += 2) {
          const float4 f0 = ab[c], f1 = ab[c + 1];
          const float w0 = ex2(y[c] - f0.z), w1 = ex2(y[c + 1] - f1.z);              // at most 256
          l[c] = fmaf(w0 * back, f0.y, l[c] * f0.x);
          l[c + 1] = fmaf(w1 * back, f1.y, l[c + 1] * f1.x);
          // as three e4m3 values: what is left is at most 2^-12 of the weight, 2^-16 on average
          float r0 = w0, r1 = w1;
#pragma unroll
          for (int p = 0; p < 3; ++p) {
            const uint32_t h = e4m3x2_of(r0, r1);
            p_row[swz<AT_T>(p * C + c, tok)] = (uint8_t)h;
            p_row[swz<AT_T>(p * C + c + 1, tok)] = (uint8_t)(h >> 8);
            if (p < 2) {
              const float2 f = e4m3x2_to(h);
              r0 = (r0 - f.x) * 16.f;
              r1 = (r1 - f.y) * 16.f;
            }
          }
        }
        // the values of a token that no column sees may be anything (its page may not even have been read): zeros
        if (masked) {
          const int s = n % RING;
          if (!wait_all(sm.full[s], (uint32_t)(n / RING))) break;
          if (unseen) {
            uint4 *z = reinterpret_cast<uint4 *>(base_ptr + s * TILE + (tok >> 3) * 2 * GROUP + GROUP + (tok & 7) * HD);
#pragma unroll
            for (int i = 0; i < HD / 16; ++i) z[i] = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.p_ready[grp]));
        ++k;
      }
      if (failed) break;
      // the item's sums: over the lanes, then over the warps
      const int ii = x.it - item_lo, h = ii & 1;
      if (ii >= 2 && !wait_all(sm.l_free[h], (uint32_t)(ii / 2 - 1))) break;
      const float sum = lane_sums<C>(l, lane);
      if ((lane & (32 / C - 1)) == 0) sm.lpart[h][grp * 4 + wq][lane / (32 / C)] = sum;
      if (wq == 0 && lane < C) sm.lframe[h][grp][lane] = m_run;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.l_ready[h]));
    }
  } else {
    // ---------------- output: thread = value dim, the running output of every column in registers ----------------
    const int wq = warp & 3;
    const bool has_dim = HD == 128 || lane < 16;
    const int d = HD == 128 ? wq * 32 + lane : wq * 16 + lane;     // an M = 64 accumulator has 16 rows in each lane quarter
    const uint32_t o_lane = o_tmem + ((uint32_t)(32 * wq) << 16);
    float4 *ab = sm.ab[warp - 4];
    float o[C];
    int n = 0;
    for (; x.it < item_hi && !failed; next_item()) {
      const int cols = x.n * G;
      float m_run = AT_LOW;                           // lane c: the running frame of column c
#pragma unroll
      for (int c = 0; c < C; ++c) o[c] = 0.f;
      for (int t = x.t0; t < x.t1 && !failed; ++t, ++n) {
        const int h = n & 1;
        if (!wait_all(sm.o_full[h], (uint32_t)(n / 2))) break;
        tc_fence_after();
        if (lane < C) {
          const float m_tile = sm.frame[h][lane], m_new = fmaxf(m_run, m_tile);
          ab[lane] = make_float4(ex2(m_run - m_new), ex2(m_tile - m_new), 0.f, 0.f);
          m_run = m_new;
        }
        __syncwarp();
#pragma unroll
        for (int c0 = 0; c0 < C; c0 += 8) {
          constexpr int W = C < 8 ? C : 8;
          uint32_t v[24];
          if (C == 4) {
            tmem_ld8(o_lane + (uint32_t)(h * N), *reinterpret_cast<uint32_t(*)[8]>(&v[0]));
            tmem_ld8(o_lane + (uint32_t)(h * N + 8), *reinterpret_cast<uint32_t(*)[8]>(&v[8]));
          } else {
#pragma unroll
            for (int p = 0; p < 3; ++p) tmem_ld8(o_lane + (uint32_t)(h * N + p * C + c0), *reinterpret_cast<uint32_t(*)[8]>(&v[p * 8]));
          }
          tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < W; ++c) {
            const float f = fmaf(fmaf(__uint_as_float(v[2 * W + c]), 1.f / 16.f, __uint_as_float(v[W + c])), 1.f / 16.f, __uint_as_float(v[c]));
            const float4 s = ab[c0 + c];
            o[c0 + c] = fmaf(f, s.y, o[c0 + c] * s.x);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.o_free[h]));
      }
      if (failed) break;
      const int ii = x.it - item_lo, h = ii & 1;
      if (!wait_all(sm.l_ready[h], (uint32_t)(ii / 2))) break;
      float L = 0.f;                                  // lane c: the sum of column c in the frame m_run
      if (lane < C) {
#pragma unroll
        for (int gr = 0; gr < 2; ++gr) {
          float v = 0.f;
#pragma unroll
          for (int w = 0; w < 4; ++w) v += sm.lpart[h][gr * 4 + w][lane];
          L = fmaf(v, ex2(sm.lframe[h][gr][lane] - m_run), L);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.l_free[h]));
      const long long bg = (long long)x.b * a.n_kv + x.g;
      if (x.ns == 1) {
        const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float f = __shfl_sync(0xffffffffu, inv, c);
          if (c < cols && has_dim)
            ((T *)a.out)[(long long)(x.first + c / G) * a.o_t + (long long)(x.g * G + c % G) * a.o_h + d] = from_f32<T>(o[c] * f);
        }
        if (a.mass && wq == 0 && lane < cols) a.ml[bg * a.cols + lane] = make_float2(m_run - 8.f, inv);
      } else {
        int step;
        const long long at = part_at(a, x.b, x.first, x.n, x.g, x.split, G, step);
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (c < cols && has_dim) a.part_o[(at + c) * HD + d] = o[c];
        if (wq == 0 && lane < cols) a.part_ml[at + lane] = make_float2(m_run, L);
      }
    }
  }
  if (failed || sm.abort_flag) {
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // let copies in flight land before the CTA retires
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (tid == 0)
    for (int i = blockIdx.x; i < AT_STATUS; i += gridDim.x) a.status[i] = sm.abort_flag ? DEV_TIMEOUT_EPILOGUE : DEV_OK;
  if (warp == 0) tmem_dealloc(s_tmem, TMEM_COLS);
}

// One block per (row, key head, column): each of four warps (eight for rows with more than AT_MANY splits) takes a part of the row's splits,
// ascending, hd / 32 dims a lane; the parts are added in their order.
constexpr int AT_PARTS = 8, AT_MANY = 32;
template <int W> struct alignas(4 * W) Floats { float v[W]; };
template <typename T, int HD>
__global__ void __launch_bounds__(32 * AT_PARTS) attend_combine_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int W = HD / 32, AHEAD = 8;
  typedef Floats<W> F;
  griddep_launch_dependents();
  __shared__ float2 sml[AT_SPLITS];
  __shared__ F so[AT_PARTS][32];
  __shared__ float sl[AT_PARTS];
  const int b = blockIdx.x / a.n_kv, g = blockIdx.x - b * a.n_kv, col = blockIdx.y, q = threadIdx.x >> 5, lane = threadIdx.x & 31, G = a.n_q / a.n_kv;
  const int first = a.cu ? a.cu[b] : b, end = a.cu ? a.cu[b + 1] : b + 1;
  const RowPlan r = row_plan(a.ctx[b], first, end, a, G);
  griddep_wait();
  if (r.ns <= 1 || col >= r.n * G) return;
  int cols;
  const long long at = part_at(a, b, r.first, r.n, g, 0, G, cols) + col;
  const int parts = r.ns > AT_MANY ? AT_PARTS : AT_PARTS / 2;
  const int per = (r.ns + parts - 1) / parts, lo = q * per, hi = min(r.ns, lo + per);
  const float *po = a.part_o + at * HD + lane * W;
  const long long step = (long long)cols * HD;
  auto load = [&](int s) {
    F f;
    if (W == 4) {
      const float4 v = __ldcg(reinterpret_cast<const float4 *>(po + s * step));
      f.v[0] = v.x; f.v[1] = v.y; f.v[2 % W] = v.z; f.v[3 % W] = v.w;
    } else {
      const float2 v = __ldcg(reinterpret_cast<const float2 *>(po + s * step));
      f.v[0] = v.x; f.v[1] = v.y;
    }
    return f;
  };
  F x[AHEAD];
#pragma unroll
  for (int e = 0; e < AHEAD; ++e)
    if (lo + e < hi) x[e] = load(lo + e);
  for (int s = threadIdx.x; s < r.ns; s += blockDim.x) sml[s] = __ldcg(a.part_ml + at + (long long)s * cols);
  __syncthreads();
  float M = AT_LOW;
  for (int s = lane; s < r.ns; s += 32) M = fmaxf(M, sml[s].x);
  M = warp_max(M);
  float L = 0.f;
  F o;
#pragma unroll
  for (int w = 0; w < W; ++w) o.v[w] = 0.f;
  for (int s0 = lo; s0 < hi; s0 += AHEAD) {
#pragma unroll
    for (int e = 0; e < AHEAD; ++e)
      if (s0 + e < hi) {
        const float f = ex2(sml[s0 + e].x - M);
        L = fmaf(f, sml[s0 + e].y, L);
#pragma unroll
        for (int w = 0; w < W; ++w) o.v[w] = fmaf(f, x[e].v[w], o.v[w]);
        if (s0 + e + AHEAD < hi) x[e] = load(s0 + e + AHEAD);
      }
  }
  so[q][lane] = o;
  if (lane == 0) sl[q] = L;
  __syncthreads();
  // thread = dim
  const int d = threadIdx.x;
  if (d >= HD) return;
  float sum = 0.f;
  L = 0.f;
  for (int e = 0; e < parts; ++e) { L += sl[e]; sum += so[e][d / W].v[d % W]; }
  const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
  ((T *)a.out)[(long long)(first + col / G) * a.o_t + (long long)(g * G + col % G) * a.o_h + d] = from_f32<T>(sum * inv);
  if (a.mass && d == 0) a.ml[(long long)blockIdx.x * a.cols + col] = make_float2(M - 8.f, inv);
}

// One thread per cached token of a (row, key head): mass += the sum of its weights over the columns, ascending.
__global__ void __launch_bounds__(256) attend_mass_kernel(const __grid_constant__ AttendArgs a) {
  __shared__ float2 ml[AT_MAXC];
  const int b = blockIdx.x / a.n_kv, G = a.n_q / a.n_kv;
  const int first = a.cu ? a.cu[b] : b, end = a.cu ? a.cu[b + 1] : b + 1;
  const RowPlan r = row_plan(a.ctx[b], first, end, a, G);
  griddep_wait();
  if (r.ns == 0) return;
  const int cols = r.n * G;
  if ((int)threadIdx.x < cols) ml[threadIdx.x] = __ldcg(a.ml + (long long)blockIdx.x * a.cols + threadIdx.x);
  __syncthreads();
  const float *sc = a.scores + (long long)blockIdx.x * a.score_tokens * a.cols;
  float *mass = a.mass + (long long)blockIdx.x * a.max_blocks * a.block;
  for (int j = r.t_lo * AT_T + blockIdx.y * 256 + threadIdx.x; j < r.c; j += gridDim.y * 256) {
    const float before = mass[j];
    const float *sj = sc + (long long)j * a.cols;
    float sum = 0.f;
    if ((a.cols & 3) == 0) {
      for (int c = 0; c < cols; c += 4) {
        const float4 s = __ldcg(reinterpret_cast<const float4 *>(sj + c));
        const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < cols) {
            const float2 f = ml[c + e];
            sum = fmaf(ex2(v[e] - f.x), f.y, sum);
          }
      }
    } else {
      for (int c = 0; c < cols; ++c) {
        const float2 f = ml[c];
        sum = fmaf(ex2(__ldcg(sj + c) - f.x), f.y, sum);
      }
    }
    mass[j] = before + sum;
  }
}

constexpr int at_columns(int wanted) { return wanted <= 4 ? 4 : wanted <= 8 ? 8 : wanted <= 16 ? 16 : 32; }

// Sizes of the workspace's parts, each on 256 bytes.
struct AttendSpace {
  int cols, max_splits;
  bool by_token;
  int64_t part_ml, part_o, ml, scores, score_tokens, bytes;
};
AttendSpace attend_space(int64_t B, int64_t T, int max_new, int n_q, int n_kv, int hd, int block, int max_blocks, bool mass) {
  auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
  const int64_t G = n_q / n_kv, all = G * max_new;
  const int64_t reach_tiles = ((int64_t)max_blocks * block + AT_T - 1) / AT_T;
  AttendSpace s;
  s.cols = (int)(all < AT_MAXC ? all : AT_MAXC);
  s.max_splits = (int)(reach_tiles / AT_MIN_TILES);       // at_splits gives no more
  s.max_splits = s.max_splits < 1 ? 1 : s.max_splits > AT_SPLITS ? AT_SPLITS : s.max_splits;
  s.score_tokens = reach_tiles * AT_T;
  s.by_token = T * G <= B * s.cols;
  const int64_t parts = (s.by_token ? T * G : B * s.cols) * n_kv * s.max_splits;
  s.part_ml = AT_STATUS * 4;
  s.part_o = s.part_ml + up(parts * 8);
  s.ml = s.part_o + up(s.max_splits > 1 ? parts * hd * 4 : 0);
  s.scores = s.ml + up(mass ? B * n_kv * s.cols * 8 : 0);
  s.bytes = s.scores + up(mass ? B * n_kv * s.score_tokens * s.cols * 4 : 0);
  return s;
}

template <typename T, int HD, int C>
cudaError_t launch_attend_c(const CUtensorMap &tm, const AttendArgs &a, int dev, int sms, cudaStream_t st) {
  // the shared-memory size is opted into once per device
  static std::atomic<uint64_t> done{0};
  constexpr int smem = smem_bytes<T, HD, C>();
  static_assert(smem <= 232448, "shared memory of a CTA");
  cudaError_t ce = cudaSuccess;
  if (dev >= 64 || !(done.load() >> dev & 1)) {
    ce = cudaFuncSetAttribute(attend_kernel<T, HD, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (ce != cudaSuccess) return ce;
    if (dev < 64) done.fetch_or(1ull << dev);
  }
  ce = launch_k(attend_kernel<T, HD, C>, dim3(sms), dim3(AT_THREADS), smem, st, true, tm, a);
  if (ce == cudaSuccess && a.max_splits > 1) {
    ce = launch_k(attend_combine_kernel<T, HD>, dim3(a.B * a.n_kv, a.cols), dim3(32 * (a.max_splits > AT_MANY ? AT_PARTS : AT_PARTS / 2)), 0, st, true, a);
  }
  if (ce == cudaSuccess && a.mass) {
    int gy = (16 * sms + a.B * a.n_kv - 1) / (a.B * a.n_kv);
    const long long most = (a.score_tokens + 255) / 256;
    if (gy > most) gy = (int)most;
    ce = launch_k(attend_mass_kernel, dim3(a.B * a.n_kv, gy), dim3(256), 0, st, true, a);
  }
  return ce;
}
template <typename T, int HD>
cudaError_t launch_attend(const CUtensorMap &tm, const AttendArgs &a, int dev, int sms, cudaStream_t st) {
  const long long all = (long long)(a.n_q / a.n_kv) * a.max_new;
  switch (at_columns(all > AT_MAXC ? AT_MAXC : (int)all)) {
    case 4: return launch_attend_c<T, HD, 4>(tm, a, dev, sms, st);
    case 8: return launch_attend_c<T, HD, 8>(tm, a, dev, sms, st);
    case 16: return launch_attend_c<T, HD, 16>(tm, a, dev, sms, st);
    default: return launch_attend_c<T, HD, 32>(tm, a, dev, sms, st);
  }
}

}  // namespace
}  // namespace corun

using namespace corun;

extern "C" {

int64_t corun_kv8_attend_bytes(int32_t B, int32_t T, int32_t max_new, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t block,
                               int32_t max_blocks, int32_t with_mass) {
  if (B < 1 || T < 1 || max_new < 1 || n_q < 1 || n_kv < 1 || n_q < n_kv || head_dim < 1 || block < 1 || max_blocks < 1) return 0;
  return attend_space(B, T, max_new, n_q, n_kv, head_dim, block, max_blocks, with_mass != 0).bytes;
}

int corun_kv8_attend(const corun_kv8_cache *cache, const corun_kv8_rows *rows, int32_t max_new, const corun_heads *q,
                     const corun_heads *out, int32_t dtype, int32_t n_q, float scale, int32_t window, float *mass, void *ws,
                     int64_t ws_bytes, void *cuda_stream) {
  if (!kv8_cache_ok(cache) || !kv8_rows_ok(rows, cache) || !q || !out || (dtype != CORUN_BF16 && dtype != CORUN_F16) ||
      rows->B > AT_MAXB || max_new < 1 || (!rows->cu && max_new != 1) || n_q < 1 || n_q % cache->n_kv || n_q / cache->n_kv > AT_MAXC || !(scale > 0.f) || isinf(scale) ||
      window < 0 || (mass && (int64_t)max_new * (n_q / cache->n_kv) > AT_MAXC) || kv8_chunk_tiles(rows->T, rows->B, n_q / cache->n_kv) > 65535)
    return CORUN_EINVAL;
  if (rows->T == 0) {                               // (tensors of no tokens may have no address)
    if (!ws || ws_bytes < AT_STATUS * (int)sizeof(int)) return CORUN_OK;
    const cudaError_t ce = cudaMemsetAsync(ws, 0, AT_STATUS * sizeof(int), (cudaStream_t)cuda_stream);
    if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
    return CORUN_OK;
  }
  if (!q->p || !out->p || !heads_on_16(*q, dtype) || !heads_on_16(*out, dtype) || !ws || !aligned_to(ws, 256)) return CORUN_EINVAL;
  const AttendSpace s = attend_space(rows->B, rows->T, max_new, n_q, cache->n_kv, cache->head_dim, cache->block, rows->max_blocks, mass != nullptr);
  if (ws_bytes < s.bytes) return CORUN_EINVAL;
  int dev = 0, sms = 0;
  cudaError_t ce = device_sms(&dev, &sms);
  if (ce != cudaSuccess || sms < 1) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  CUtensorMap tm;
  int rc = tma_encode_kv8(&tm, cache->pool, (unsigned long long)cache->pages, cache->n_kv, cache->block, cache->head_dim, 2);
  if (rc != CORUN_OK) return rc;
  char *w = (char *)ws;
  const AttendArgs a{cache->exps, cache->pages, cache->block, cache->n_kv, n_q, rows->B, rows->T, rows->max_blocks, max_new, window < (1 << 30) ? window : 0, s.cols, s.max_splits, sms, s.by_token,
                     rows->block_table, rows->ctx, rows->cu, q->p, out->p, q->token_stride, q->head_stride, out->token_stride, out->head_stride,
                     scale * 1.4426950408889634f, mass, (int *)w, (float2 *)(w + s.part_ml), (float *)(w + s.part_o), (float2 *)(w + s.ml),
                     (float *)(w + s.scores), s.score_tokens};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == CORUN_BF16) ce = cache->head_dim == 128 ? launch_attend<__nv_bfloat16, 128>(tm, a, dev, sms, st) : launch_attend<__nv_bfloat16, 64>(tm, a, dev, sms, st);
  else ce = cache->head_dim == 128 ? launch_attend<__half, 128>(tm, a, dev, sms, st) : launch_attend<__half, 64>(tm, a, dev, sms, st);
  if (ce == cudaSuccess && (int64_t)max_new * (n_q / cache->n_kv) > AT_MAXC) {
    rc = tma_encode_kv8(&tm, cache->pool, (unsigned long long)cache->pages, cache->n_kv, cache->block, cache->head_dim, 1);
    if (rc != CORUN_OK) return rc;
    ce = launch_kv8_chunk(tm, a, cache->head_dim, dtype, dev, st);
  }
  if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  return CORUN_OK;
}

int corun_kv8_sync(const void *ws, void *cuda_stream) {
  if (!ws) return CORUN_EINVAL;
  int hs[AT_STATUS] = {0};
  cudaError_t ce = cudaMemcpyAsync(hs, ws, sizeof(hs), cudaMemcpyDeviceToHost, (cudaStream_t)cuda_stream);
  if (ce == cudaSuccess) ce = cudaStreamSynchronize((cudaStream_t)cuda_stream);
  if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  for (int i = 0; i < AT_STATUS; ++i)
    if (hs[i]) return CORUN_ETIMEOUT;
  return CORUN_OK;
}

}  // extern "C"
