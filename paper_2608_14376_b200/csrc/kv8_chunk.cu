// Attention over the 8-bit cache for rows with many new tokens (include/corun_kv8.h): the chunks of prompts.
//
// One CTA per (tile of 128 / G consecutive new tokens of a row, key head), G = query heads per key head; the tile's 128 rows are its
// (token, head) pairs, row m = token m / G, head m % G.  It walks the blocks of 128 cached tokens that any of its rows sees once:
//   S[128 rows x 128 tokens] = Q * K^T      (M = 128, N = 128, fp16) into one of two TMEM buffers;
//   softmax warps, a thread per row: P = 2^(s + e_v - M), M the largest s + e_v of the row in the block, as fp16 into one of two
//     TMEM buffers (e_v: the exponents of the values' pages), M and the sum of P 2^-e_v;
//   O'[128 x hd] = P * V, P from tensor memory;
//   output warps, a thread per row and half of the dims: O and O' to the larger of the two frames and added, in registers.
// With 128 rows to a tile the products are many times the cache's bytes: here the 8-bit values are turned into fp16 once per tile and
// block (exactly; the scales stay apart), and a weight or a query is one fp16 value, where the kernel for few columns
// takes three e4m3 ones.  The output warps do that turning: they would else wait for the MMAs most of the time.
//   the output of block j - 1, the keys of block j + 2, the values of block j + 1
// in turn, beside the products.
// A query row is brought to [256, 512) by a power of two before it is rounded to fp16: exact for bf16, and for fp16, but for values
// some 2^-22 of the row's largest.  One fp16 value of a weight is off by 2^-11 at most (or 2^-25 of the block's largest), an eighth of a bf16 output's
// own rounding and as much as an fp16 output's; with a second value for the rest outputs are 6.6e-5 instead of 2.0e-4 from those in 32 bits, but
// their errors against 64 bits the same in bf16, and the case below takes 270 us: the second products are two thirds of that.
//
// Measured on 3 rows of 200 to 700 new tokens behind up to 8192 cached ones (32 query, 8 key heads of 128, bf16): 249 us, 474 TFLOP/s; the
// kernel for few columns took 1484.  A block takes 3300 to 3700 cycles, of which the products need 1024: the softmax (some 900 instructions a
// warp and block, and a third of all issue slots), the output and the turning share the schedulers (62 % of issue slots, ALU pipe 42 %,
// tensor pipe 27 %).  Turning with one fp16 tile of values and two of keys: 315 us; whichever product can go on first: 256.
//
// The cached tokens are not split: a row of few tiles behind a very long cache keeps few SMs busy (5 tokens x 8 heads, 4 key heads, 100003
// cached tokens: 2080 us on 4 SMs, where kv8_attend.cu takes 78 for 4 tokens).
//
// Every reduction has one fixed order that depends on the row's own lengths only.  All waits are bounded.
#include <math_constants.h>

#include <atomic>
#include <type_traits>

#include "kv8_attend.cuh"

namespace corun {
namespace {

constexpr int CH_THREADS = 608;     // warps 0-7 softmax, 8-15 output and conversion, 16 / 17 TMA of keys / values, 18 MMAs
constexpr int CH_KR = 2, CH_VR = 3; // 8-bit tiles of keys / values in flight
constexpr int CH_EXPS = 8;          // blocks whose exponents are held

template <int HD>
struct ChunkLayout {
  static constexpr int T8 = AT_T * HD;             // an 8-bit tile
  static constexpr int T16 = 2 * T8;               // the same in fp16: [64 dims][128 tokens x 128 bytes]
  static constexpr int Q = 0, K16 = T16, V16 = K16 + T16, K8 = V16 + 2 * T16, V8 = K8 + CH_KR * T8;
  static constexpr int SMEM = V8 + CH_VR * T8 + 1024;
  static constexpr uint32_t P_COL = 256, O_COL = 384;
};

// Two e4m3 values as two fp16 values, exactly.
__device__ __forceinline__ uint32_t widen2(uint16_t v) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(v));
  return r;
}
__device__ __forceinline__ uint2 widen4(uint32_t v) { return make_uint2(widen2((uint16_t)v), widen2((uint16_t)(v >> 16))); }

template <typename T, int HD>
__global__ void __launch_bounds__(CH_THREADS, 1) chunk_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ AttendArgs a) {
  using L = ChunkLayout<HD>;
  constexpr int KSTEPS = HD / 16;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t k8_full[CH_KR], k8_empty[CH_KR], v8_full[CH_VR], v8_empty[CH_VR], e_full[CH_EXPS], k_ready, v_ready[2], s_full[2],
      p_ready[2], p_free[2], o_full, o_free;
  __shared__ float max_s[4][128], sum_s[4][128];    // a block's frame and sum per row, four blocks in turn
  __shared__ float q_mul[128];                      // 2^e of a query row times scale log2(e)
  __shared__ int8_t exps[CH_EXPS][2][8];
  __shared__ float k_top[CH_EXPS];                  // the largest of the keys' scales
  __shared__ int row_c[AT_MAXB], row_tiles[AT_MAXB], s_row, s_qt, s_c, s_first, s_n;
  __shared__ uint32_t tmem_base_s;
  __shared__ int abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = a.n_q / a.n_kv, TQ = 128 / G, shift = a.block == 16 ? 4 : a.block == 32 ? 5 : 6;
  const int g = blockIdx.x, tile = blockIdx.y;      // heads fastest
  if (tid == 0) {
    abort_flag = 0;
    s_row = -1;
    for (int i = 0; i < CH_KR; ++i) { mbar_init(smem_u32(&k8_full[i]), 1); mbar_init(smem_u32(&k8_empty[i]), 8); }
    for (int i = 0; i < CH_VR; ++i) { mbar_init(smem_u32(&v8_full[i]), 1); mbar_init(smem_u32(&v8_empty[i]), 8); }
    for (int i = 0; i < CH_EXPS; ++i) mbar_init(smem_u32(&e_full[i]), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&v_ready[i]), 8);          // values in fp16
      mbar_init(smem_u32(&s_full[i]), 1);           // scores in TMEM
      mbar_init(smem_u32(&p_ready[i]), 128);        // every row thread has read them and written its weights, frame and sum
      mbar_init(smem_u32(&p_free[i]), 1);           // the output product has read the weights
    }
    mbar_init(smem_u32(&k_ready), 8);               // keys in fp16
    mbar_init(smem_u32(&o_full), 1);
    mbar_init(smem_u32(&o_free), 256);
    fence_mbar_init();
    fence_proxy_async();
    prefetch_tensormap(&tm);
  }
  griddep_wait();
  // the tile's row: the rows with the longest caches first, the last tile (the most blocks) of a row first
  {
    int c = 0, first = 0, n = 0, tiles = 0;
    if (tid < a.B) {
      first = a.cu ? __ldcg(a.cu + tid) : tid;
      const int end = a.cu ? __ldcg(a.cu + tid + 1) : tid + 1;
      c = __ldcg(a.ctx + tid);
      n = end - first;
      if (at_row_ok(c, first, end, a) && (long long)n * G > AT_MAXC) tiles = (n + TQ - 1) / TQ;
      row_c[tid] = c;
      row_tiles[tid] = tiles;
    }
    __syncthreads();
    int before = 0;
    if (tiles > 0)
      for (int r = 0; r < a.B; ++r)
        if (row_c[r] > c || (row_c[r] == c && r < tid)) before += row_tiles[r];
    if (tile >= before && tile < before + tiles) { s_row = tid; s_qt = tiles - 1 - (tile - before); s_c = c; s_first = first; s_n = n; }
  }
  __syncthreads();
  griddep_launch_dependents();
  if (s_row < 0) return;                            // (the grid is an upper bound)
  const int i0 = s_qt * TQ, n_tok = min(TQ, s_n - i0), t_first = s_first + i0, pos0 = s_c - s_n + i0;   // place of the tile's first token in the cache
  const int vis_end = max(pos0 + n_tok, 0);         // tokens that some row sees: [vis_lo, vis_end)
  const int vis_lo = a.window ? max(0, pos0 - a.window + 1) : 0;
  const int b0 = vis_lo / AT_T, n_blocks = max(1, (vis_end + AT_T - 1) / AT_T - b0);
  auto pages_of = [&](int j) { return min(AT_T >> shift, max(1, (vis_end - (b0 + j) * AT_T + a.block - 1) >> shift)); };

  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *base_ptr = smem_raw + (base - smem_u32(smem_raw));
  bool failed = false;
  auto wait_all = [&](uint64_t &bar, uint32_t parity) {   // by a whole warp
    const bool ok = mbar_wait(smem_u32(&bar), parity & 1u, &abort_flag);
    if (!__all_sync(0xffffffffu, ok)) failed = true;
    return !failed;
  };
  // producers: lane l fetches page l of a block; its page number is read two blocks ahead of its use, its exponents one
  const bool keys = warp == 16;
  const int *table = a.block_table + (size_t)s_row * a.max_blocks;
  int page0 = -1, page1 = -1, ek = KV8_E_MIN, ev = 0;
  auto page_at = [&](int j) { return j < n_blocks && lane < pages_of(j) ? load_now(table + ((b0 + j) * (AT_T >> shift) + lane)) : -1; };
  auto exps_at = [&](int page) {
    ek = KV8_E_MIN;                                 // (of a page that is not there: its keys are zeros, or nobody sees them)
    ev = 0;
    if (keys && page >= 0 && (long long)page < a.pages) {
      const long long at = (long long)page * 2 * a.n_kv + g;
      ek = load_now(a.exps + at);
      ev = load_now(a.exps + at + a.n_kv);
    }
  };
  auto fetch = [&](int j) {
    const int ring = keys ? CH_KR : CH_VR, buf = j % ring, np = pages_of(j), page = page0, ek_now = ek, ev_now = ev;
    page0 = page1;
    page1 = page_at(j + 2);
    if (j >= ring && !wait_all(keys ? k8_empty[buf] : v8_empty[buf], (uint32_t)(j / ring - 1))) return;
    const uint32_t fb = smem_u32(keys ? &k8_full[buf] : &v8_full[buf]);
    if (lane == 0) mbar_arrive_expect_tx(fb, (uint32_t)(np * a.block * HD));
    __syncwarp();
    if (lane < np)
      tma_load_5d(base + (uint32_t)((keys ? L::K8 : L::V8) + buf * L::T8 + lane * a.block * HD), &tm, 0, 0, keys ? 0 : 1, g * (a.block >> 3),
                  page >= 0 && (long long)page < a.pages ? page : (int)a.pages, fb, l2_policy_evict_last());   // other tiles of the row read the same pages
    if (keys) {
      // (the keys of block j - CH_KR, whose slot this is, were turned behind the output of block j - 5: what read the exponents of block
      // j - CH_EXPS has ended)
      if (lane < 8) { exps[j % CH_EXPS][0][lane] = (int8_t)ek_now; exps[j % CH_EXPS][1][lane] = (int8_t)ev_now; }
      const int top = __reduce_max_sync(0xffffffffu, ek_now);
      if (lane == 0) k_top[j % CH_EXPS] = pow2f(top);
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&e_full[j % CH_EXPS]));
      exps_at(page0);
    }
  };
  if (warp == 18) {
    tmem_alloc(smem_u32(&tmem_base_s), 512);
    tmem_relinquish();
  } else if (warp >= 16) {
    page0 = page_at(0);
    page1 = page_at(1);
    exps_at(page0);
    for (int j = 0; j < n_blocks && j < (keys ? CH_KR : CH_VR) && !failed; ++j) fetch(j);   // beside the query tile
  } else {
    // ---- the query tile; a row is HD / 4 lanes
    constexpr int LPR = HD / 4, RPW = 32 / LPR;
    const int d = 4 * (lane % LPR);
    uint2 v[8 / RPW];
#pragma unroll
    for (int k = 0; k < 8 / RPW; ++k) {
      const int m = RPW * (warp + 16 * k) + lane / LPR, t = m / G;
      v[k] = make_uint2(0u, 0u);
      if (t < n_tok) v[k] = __ldcg(reinterpret_cast<const uint2 *>((const T *)a.q + (long long)(t_first + t) * a.q_t + (long long)(g * G + m % G) * a.q_h + d));
    }
#pragma unroll
    for (int k = 0; k < 8 / RPW; ++k) {
      const int m = RPW * (warp + 16 * k) + lane / LPR;
      const T *e = reinterpret_cast<const T *>(&v[k]);
      float x[4], mx = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = to_f32(e[i]);
        if (!(fabsf(x[i]) <= 3.4e38f)) x[i] = CUDART_NAN_F;        // an infinite query makes its scores NaN
        mx = fmaxf(mx, fabsf(x[i]));
      }
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const int ex = max((__float_as_int(mx) >> 23) - 127, -110) - 8;          // to [256, 512)
      const float down = pow2f(-ex);
      const __half2 h0 = __floats2half2_rn(x[0] * down, x[1] * down), h1 = __floats2half2_rn(x[2] * down, x[3] * down);
      const uint2 w = make_uint2(*reinterpret_cast<const uint32_t *>(&h0), *reinterpret_cast<const uint32_t *>(&h1));
      *reinterpret_cast<uint2 *>(base_ptr + L::Q + (d >> 6) * (128 * 128) + m * 128 + ((((d & 63) >> 3) ^ (m & 7)) << 4) + (d & 4) * 2) = w;
      if (lane % LPR == 0) q_mul[m] = (mx > 0.f ? pow2f(ex) : 1.f) * a.scale_log2e;
    }
    fence_proxy_async();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  // warps 0-15: this thread's row
  const int quad = warp & 3, tl = quad * 32 + lane;
  const uint32_t t_lane = tmem + ((uint32_t)(quad * 32) << 16);
  const bool real = tl / G < n_tok;

  if (warp == 16 || warp == 17) {
    // ---------------- producers
    for (int j = keys ? CH_KR : CH_VR; j < n_blocks && !failed; ++j) fetch(j);
  } else if (warp == 18) {
    // ---------------- MMA issuer: the scores of block j + 2, then the values of block j
    if (elect_one()) {
      const uint32_t idesc_s = (1u << 4) | ((uint32_t)(AT_T >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
      auto wait = [&](uint64_t &bar, int phase) {
        if (!mbar_wait(smem_u32(&bar), (uint32_t)phase & 1u, &abort_flag)) failed = true;
        return !failed;
      };
      auto scores = [&](int j) {
        const int b = j & 1;
        if (!wait(k_ready, j)) return;
        tc_fence_after();
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks)
          umma_bf16(tmem + (uint32_t)b * 128, umma_desc_sw128(base + (uint32_t)(L::Q + (ks >> 2) * (128 * 128))) + (uint64_t)((ks & 3) * 2),
                    umma_desc_sw128(base + (uint32_t)(L::K16 + (ks >> 2) * (128 * 128))) + (uint64_t)((ks & 3) * 2), idesc_s, ks > 0 ? 1u : 0u);
        umma_commit(smem_u32(&s_full[b]));
      };
      scores(0);
      if (n_blocks > 1 && !failed) scores(1);
      for (int j = 0; j < n_blocks && !failed; ++j) {
        const int b = j & 1;
        if (!wait(p_ready[b], j >> 1)) break;       // with its weights a block's scores have been read, too
        if (j + 2 < n_blocks) scores(j + 2);
        if (failed || !wait(v_ready[b], j >> 1) || (j > 0 && !wait(o_free, j - 1))) break;
        tc_fence_after();
        const uint32_t p = tmem + L::P_COL + (uint32_t)b * 64;
#pragma unroll
        for (int i = 0; i < AT_T / 16; ++i)         // 16 tokens of weights are 8 columns
          umma_f16_ts(tmem + L::O_COL, p + (uint32_t)(8 * i), umma_desc_sw128_mn(base + (uint32_t)(L::V16 + b * L::T16 + i * 2048), 128 * 128, 1024u), idesc_o, i > 0 ? 1u : 0u);
        umma_commit(smem_u32(&o_full));
        umma_commit(smem_u32(&p_free[b]));
      }
    }
  } else if (warp < 8) {
    // ---------------- softmax: one thread per row; warps 0-3 the even blocks, warps 4-7 the odd ones
    const int pos = real ? pos0 + tl / G : -1;      // tokens up to pos are visible to this row
    const float qm = q_mul[tl];
    // x f + (e_v - M) is rounded once where M was rounded before: they differ by up to |M| 2^-24, which is nothing while |M| stays below 2^20, but
    // takes weights beyond fp16 from 2^28 on.  |x| is below 2^25: with keys' scales from here on, which a score might pass 2^20 with, the
    // exponents are formed as M was.
    const float far_from = real ? 0.03125f / qm : CUDART_INF_F;
    const int sb = warp >> 2;
    const uint32_t st = t_lane + (uint32_t)(sb * 128), pt = t_lane + L::P_COL + (uint32_t)(sb * 64);
    for (int j = sb; j < n_blocks; j += 2) {
      if (!wait_all(e_full[j % CH_EXPS], (uint32_t)(j / CH_EXPS))) break;
      const int8_t *ex = exps[j % CH_EXPS][0];
      const bool far = k_top[j % CH_EXPS] > far_from;
      if (!wait_all(s_full[sb], (uint32_t)(j >> 1))) break;
      tc_fence_after();
      const int lim = pos - (b0 + j) * AT_T, low = a.window ? lim - a.window : -1;   // tokens low + 1 .. lim of the block are visible
      float bm = -CUDART_INF_F, l = 0.f;
      auto block = [&](auto masked, auto may_be_far) {
        constexpr bool M = decltype(masked)::value, FAR = decltype(may_be_far)::value;
        uint32_t v[2][16];
        tmem_ld16(st, v[0]);
        auto largest = [&](const uint32_t (&x)[16], int c) {        // chunk c: tokens 16 c .. 16 c + 15, all of one page
          float m4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int t = 16 * c + i;
            m4[i & 3] = fmaxf(m4[i & 3], M && (t > lim || t <= low) ? -CUDART_INF_F : __uint_as_float(x[i]));
          }
          const int p = (16 * c) >> shift;
          bm = fmaxf(bm, fmaf(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), pow2f(ex[p]) * qm, (float)ex[8 + p]));
        };
#pragma unroll 1
        for (int c = 0; c < 8; c += 2) {
          tmem_ld_wait();
          tmem_ld16(st + (uint32_t)(16 * c + 16), v[1]);
          largest(v[0], c);
          tmem_ld_wait();
          tmem_ld16(st + (uint32_t)((16 * c + 32) & 127), v[0]);    // (the last one begins the second pass)
          largest(v[1], c + 1);
        }
        const float ref = bm == -CUDART_INF_F ? 0.f : bm;           // (nothing visible in this block: all its weights are 0)
        if (j > 1 && !wait_all(p_free[sb], (uint32_t)((j >> 1) - 1))) return;
        auto weights = [&](const uint32_t (&x)[16], int c) {
          const int p = (16 * c) >> shift, ev = ex[8 + p];
          const float f = pow2f(ex[p]) * qm, off = FAR ? (float)ev : (float)ev - ref;
          auto weight = [&](uint32_t s) {
            const float y = fmaf(__uint_as_float(s), f, off);
            return ex2(FAR ? y - ref : y);
          };
          uint32_t w[8];
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const int t = 16 * c + i;
            float p0 = weight(x[i]), p1 = weight(x[i + 1]);
            if (M && (t > lim || t <= low)) p0 = 0.f;
            if (M && (t + 1 > lim || t + 1 <= low)) p1 = 0.f;
            acc[i & 3] += p0;
            acc[(i + 1) & 3] += p1;
            const __half2 h2 = __floats2half2_rn(p0, p1);
            w[i >> 1] = *reinterpret_cast<const uint32_t *>(&h2);
          }
          l = fmaf((acc[0] + acc[1]) + (acc[2] + acc[3]), pow2f(-ev), l);
          tmem_st8(pt + (uint32_t)(8 * c), w);
        };
#pragma unroll 1
        for (int c = 0; c < 8; c += 2) {
          tmem_ld_wait();
          tmem_ld16(st + (uint32_t)(16 * c + 16), v[1]);
          weights(v[0], c);
          tmem_ld_wait();
          tmem_ld16(st + (uint32_t)(c < 6 ? 16 * c + 32 : 112), v[0]);   // (the last one is not used)
          weights(v[1], c + 1);
        }
        tmem_ld_wait();
      };
      if (!__any_sync(0xffffffffu, far || lim < AT_T - 1 || low >= 0)) block(std::false_type{}, std::false_type{});
      else if (!__any_sync(0xffffffffu, far)) block(std::true_type{}, std::false_type{});
      else block(std::true_type{}, std::true_type{});
      if (failed) break;
      // (block j - 4's have been read: the product of block j - 2, which p_free has told of, waited for the output of block j - 3)
      max_s[j & 3][tl] = bm;
      sum_s[j & 3][tl] = l;
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(smem_u32(&p_ready[sb]));
    }
  } else {
    // ---------------- output: one thread per row and half of the dims, in registers; and fp16 tiles of keys and values
    constexpr int HH = HD / 2, CPR = HD / 16;       // 16-byte pieces of an 8-bit row
    const int dh = (warp - 8) >> 2, ot = tid - 256;
    float o[HH], mx = -CUDART_INF_F, l = 0.f;
#pragma unroll
    for (int i = 0; i < HH; ++i) o[i] = 0.f;
    // 256 threads turn a tile.  Eight neighbouring lanes take four pieces of two neighbouring tokens: the two stores of a lane then go to
    // even positions of one row and odd ones of the next, all banks (with 128 dims the load meets twice in a bank).
    constexpr int TOKENS = 256 / CPR;               // tokens at a time
    const int tc = (ot & 3) + (HD == 128 ? (ot >> 5 & 1) * 4 : 0), tt = (ot >> 2 & 7) + (HD == 128 ? (ot >> 6) * 8 : (ot >> 5) * 8);
    const int t_from = tt * HD + (HD == 128 ? ((tc ^ (tt & 7)) << 4) : ((tc ^ ((tt >> 1) & 3)) << 4));
    const int t_to = (tc >> 2) * (128 * 128) + tt * 128, t_at0 = t_to + ((((tc & 3) * 2) ^ (tt & 7)) << 4), t_at1 = t_to + ((((tc & 3) * 2 + 1) ^ (tt & 7)) << 4);
    auto turn = [&](int from, int to, int t_lo, int t_hi) {         // tokens outside of [t_lo, t_hi) become zeros
      uint4 x[AT_T / TOKENS];
#pragma unroll
      for (int k = 0; k < AT_T / TOKENS; ++k) x[k] = *reinterpret_cast<const uint4 *>(base_ptr + from + t_from + k * TOKENS * HD);
      if (t_lo > 0 || t_hi < AT_T) {
#pragma unroll
        for (int k = 0; k < AT_T / TOKENS; ++k)
          if (tt + k * TOKENS < t_lo || tt + k * TOKENS >= t_hi) x[k] = make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int k = 0; k < AT_T / TOKENS; ++k) {
        const uint2 w0 = widen4(x[k].x), w1 = widen4(x[k].y), w2 = widen4(x[k].z), w3 = widen4(x[k].w);
        *reinterpret_cast<uint4 *>(base_ptr + to + t_at0 + k * TOKENS * 128) = make_uint4(w0.x, w0.y, w1.x, w1.y);
        *reinterpret_cast<uint4 *>(base_ptr + to + t_at1 + k * TOKENS * 128) = make_uint4(w2.x, w2.y, w3.x, w3.y);
      }
      fence_proxy_async();
      __syncwarp();
    };
    auto turn_keys = [&](int j) {
      const int buf = j % CH_KR;
      if (!wait_all(k8_full[buf], (uint32_t)(j / CH_KR))) return;
      if (j > 0 && !wait_all(s_full[(j - 1) & 1], (uint32_t)((j - 1) >> 1))) return;   // the scores of block j - 1 have read their keys
      turn(L::K8 + buf * L::T8, L::K16, 0, AT_T);
      if (lane == 0) { mbar_arrive(smem_u32(&k8_empty[buf])); mbar_arrive(smem_u32(&k_ready)); }
    };
    auto turn_values = [&](int j) {                 // (the product of block j - 2 has read its values: its output has been)
      const int buf = j % CH_VR;
      if (!wait_all(v8_full[buf], (uint32_t)(j / CH_VR))) return;
      // (a token that no row sees may hold anything, its page may not even have been read)
      turn(L::V8 + buf * L::T8, L::V16 + (j & 1) * L::T16, vis_lo - (b0 + j) * AT_T, vis_end - (b0 + j) * AT_T);
      if (lane == 0) { mbar_arrive(smem_u32(&v8_empty[buf])); mbar_arrive(smem_u32(&v_ready[j & 1])); }
    };
    auto output = [&](int j) {
      if (!wait_all(o_full, (uint32_t)j)) return;
      tc_fence_after();
      // the larger frame is the scale from here on: a factor for the sums so far, or for this block
      const float bm = max_s[j & 3][tl], sum = sum_s[j & 3][tl], ref = bm == -CUDART_INF_F ? 0.f : bm;
      const bool up = bm >= mx;
      const float factor = ex2(up ? mx - ref : bm - mx);
      mx = fmaxf(mx, bm);
      l = up ? fmaf(l, factor, sum) : fmaf(sum, factor, l);
      const float f_old = up ? factor : 1.f, f_new = up ? 1.f : factor;
#pragma unroll
      for (int c = 0; c < HH / 16; ++c) {
        uint32_t v[16];
        tmem_ld16(t_lane + L::O_COL + (uint32_t)(dh * HH + 16 * c), v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) o[16 * c + i] = fmaf(o[16 * c + i], f_old, __uint_as_float(v[i]) * f_new);
      }
      tc_fence_before();
      mbar_arrive(smem_u32(&o_free));
    };
    turn_keys(0);
    if (!failed) turn_values(0);
    if (n_blocks > 1 && !failed) turn_keys(1);
    for (int j = 0; j < n_blocks && !failed; ++j) {
      if (j > 0) output(j - 1);
      if (j + 2 < n_blocks && !failed) turn_keys(j + 2);            // beside the products: scores of j + 1, values of j
      if (j + 1 < n_blocks && !failed) turn_values(j + 1);
    }
    if (!failed) output(n_blocks - 1);
    // through the query tile's shared memory (all MMAs have read it), then whole rows
    constexpr int CH = HD / 8;                      // 16-byte pieces of a row
    auto at = [&](int row, int c) { return (uint32_t)(L::Q + row * HD * 2 + ((c ^ (row & 7)) << 4)); };
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int c = 0; c < CH / 2; ++c) {
      T y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = from_f32<T>(o[8 * c + i] * inv);
      *reinterpret_cast<uint4 *>(base_ptr + at(tl, dh * (CH / 2) + c)) = *reinterpret_cast<const uint4 *>(y);
    }
    asm volatile("bar.sync 1, 256;" ::: "memory");  // warps 8-15 (whatever failed)
    if (!failed) {
#pragma unroll
      for (int k = 0; k < 128 * CH / 256; ++k) {
        const int u = k * 256 + ot, row = u / CH, c = u % CH, t = row / G;
        if (t < n_tok)
          *reinterpret_cast<uint4 *>((T *)a.out + (long long)(t_first + t) * a.o_t + (long long)(g * G + row % G) * a.o_h + 8 * c) =
              *reinterpret_cast<const uint4 *>(base_ptr + at(row, c));
      }
    }
  }
  __syncwarp();
  if (failed || abort_flag) {
    if (lane == 0) a.status[(blockIdx.x + blockIdx.y * gridDim.x) % AT_STATUS] = DEV_TIMEOUT_EPILOGUE;
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);   // let copies in flight land before the CTA retires
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 18) tmem_dealloc(tmem, 512);
}

template <typename T, int HD>
cudaError_t launch_chunk(const CUtensorMap &tm, const AttendArgs &a, int dev, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};             // the shared-memory size is opted into once per device
  constexpr int smem = ChunkLayout<HD>::SMEM;
  if (dev >= 64 || !(done.load() >> dev & 1)) {
    const cudaError_t ce = cudaFuncSetAttribute(chunk_kernel<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (ce != cudaSuccess) return ce;
    if (dev < 64) done.fetch_or(1ull << dev);
  }
  const long long tiles = kv8_chunk_tiles(a.T, a.B, a.n_q / a.n_kv);
  return launch_k(chunk_kernel<T, HD>, dim3(a.n_kv, (unsigned)(tiles < 1 ? 1 : tiles)), dim3(CH_THREADS), smem, st, true, tm, a);
}

}  // namespace

cudaError_t launch_kv8_chunk(const CUtensorMap &tm, const AttendArgs &a, int head_dim, int dtype, int dev, cudaStream_t st) {
  if (dtype == CORUN_BF16) return head_dim == 128 ? launch_chunk<__nv_bfloat16, 128>(tm, a, dev, st) : launch_chunk<__nv_bfloat16, 64>(tm, a, dev, st);
  return head_dim == 128 ? launch_chunk<__half, 128>(tm, a, dev, st) : launch_chunk<__half, 64>(tm, a, dev, st);
}

}  // namespace corun
