// Eviction from the 8-bit cache by accumulated attention weight (include/corun_kv8.h).
//
// Two kernels.  The first, a CTA per (row, key head), finds the weight of the last token that stays by a radix select over
// the weights' bits (three digits of 11, 11 and 10 bits, counted with integer atomics: the order of the counts
// does not matter), then lists the tokens that stay in their order, moves their weights to the front and settles the blocks'
// exponents.  The second moves the tokens.
//
// Moving in place: the j-th token that stays was at j or behind it.  A CTA takes one stretch of dims of a (row, head, kind)
// and goes through its tokens in order; what it writes in a round lies in front of everything that later rounds read, so
// loads of the rounds to come are in flight while a round is stored, and stretches of dims do not meet.  No second copy of
// the cache is needed.  Bound by bytes: the weights once (the digits' passes hit L2), the tokens that stay once in, once out.
#include "kv8.cuh"

namespace corun {
namespace {

constexpr int EV_THREADS = 512, EV_WARPS = EV_THREADS / 32;
constexpr int EV_BINS = 2048;
constexpr int MV_THREADS = 256, MV_AHEAD = 4;

struct EvictArgs {
  uint8_t *pool;
  int8_t *exps;
  long long pages;
  int block, n_kv, hd, B, max_blocks, max_keep, sinks, recent;
  const int *block_table, *ctx, *keep;
  int *new_ctx, *kept, *n_keep;   // n_keep [B * n_kv]: tokens that stay, 0 = the row stays as it is
  float *mass;
  int8_t *delta;                  // [B * n_kv][max_keep][2]: how far a token's exponents move (<= 0)
};

// Weights in the order of unsigned integers: larger weight, larger key; both zeros alike, NaN smallest.
__device__ __forceinline__ uint32_t mass_key(float m) {
  if (m != m) return 0u;
  const uint32_t b = __float_as_uint(m + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ int8_t old_e[];               // [2][blocks of the row]
  __shared__ int hist[EV_BINS];
  __shared__ int s_w[2][EV_WARPS], s_bin, s_above, s_bad;
  const int b = blockIdx.x / a.n_kv, h = blockIdx.x - b * a.n_kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long reach = (long long)a.max_blocks * a.block;
  const int n = a.ctx[b];
  int keep = a.keep[b];
  if (keep > 0) keep = min(max(keep, a.sinks + a.recent), a.max_keep);
  int *kept = a.kept + ((long long)b * a.n_kv + h) * a.max_keep;
  int8_t *delta = a.delta + ((long long)b * a.n_kv + h) * a.max_keep * 2;
  float *mass = a.mass + ((long long)b * a.n_kv + h) * reach;
  const int *table = a.block_table + (long long)b * a.max_blocks;
  const bool cut = keep > 0 && keep < n && n <= reach;
  const int nb = cut ? (n + a.block - 1) / a.block : 0;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  for (int i = tid; i < nb; i += EV_THREADS) {
    const long long page = table[i];
    if (page < 0 || page >= a.pages) { s_bad = 1; continue; }
    old_e[i] = a.exps[(page * 2) * a.n_kv + h];
    old_e[a.max_blocks + i] = a.exps[(page * 2 + 1) * a.n_kv + h];
  }
  __syncthreads();
  const bool go = cut && !s_bad;
  if (tid == 0) a.n_keep[blockIdx.x] = go ? keep : 0;
  for (int i = tid + (go ? keep : 0); i < a.max_keep; i += EV_THREADS) kept[i] = -1;
  if (!go) return;
  // the weight of the last token that stays among those between the sinks and the recent ones
  const int lo = a.sinks, hi = n - a.recent, want = keep - a.sinks - a.recent;
  uint32_t found = 0u, mask = 0u;
  int left = want;                                // how many stay among the tokens that agree with `found` under `mask`
  if (want > 0) {
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
      const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
      for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[i] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += EV_THREADS) {
        const uint32_t k = mass_key(mass[i]);
        if (((k ^ found) & mask) == 0u) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1u)], 1);
      }
      __syncthreads();
      // the bin from the top in which the wanted token lies: thread t sums 4 bins, bins descending over the threads
      int c[4], mine = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) { c[e] = hist[EV_BINS - 1 - (4 * tid + e)]; mine += c[e]; }
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
      }
      if (lane == 31) s_w[0][warp] = inc;
      __syncthreads();
      int above = inc - mine;
      for (int w = 0; w < warp; ++w) above += s_w[0][w];
      if (above < left && left <= above + mine) {
        int e = 0;
        while (above + c[e] < left) { above += c[e]; ++e; }
        s_bin = EV_BINS - 1 - (4 * tid + e);
        s_above = above;
      }
      __syncthreads();
      found |= (uint32_t)s_bin << shift;
      mask |= ((1u << bits) - 1u) << shift;
      left -= s_above;
      __syncthreads();
    }
  }
  // tokens that stay, in order: `left` of those whose weight is the last one's, from the front
  int n_out = 0, n_eq = 0;
  for (int i0 = 0; i0 < n; i0 += EV_THREADS) {
    const int i = i0 + tid;
    float m = 0.f;
    bool always = false, eq = false, more = false;
    if (i < n) {
      m = mass[i];
      always = i < lo || i >= hi;
      const uint32_t k = mass_key(m);
      more = !always && want > 0 && k > found;
      eq = !always && want > 0 && k == found;
    }
    const uint32_t be = __ballot_sync(0xffffffffu, eq), lt = (1u << lane) - 1u;
    if (lane == 0) s_w[0][warp] = __popc(be);
    __syncthreads();
    int eq_before = n_eq, eq_all = 0;
    for (int w = 0; w < EV_WARPS; ++w) { if (w < warp) eq_before += s_w[0][w]; eq_all += s_w[0][w]; }
    const bool stays = always || more || (eq && eq_before + __popc(be & lt) < left);
    const uint32_t bs = __ballot_sync(0xffffffffu, stays);
    if (lane == 0) s_w[1][warp] = __popc(bs);
    __syncthreads();                              // (all weights of this round have been read)
    int at = n_out, all = 0;
    for (int w = 0; w < EV_WARPS; ++w) { if (w < warp) at += s_w[1][w]; all += s_w[1][w]; }
    if (stays) {
      const int j = at + __popc(bs & lt);
      kept[j] = i;
      mass[j] = m;                                // j <= i: in front of what later rounds read
    }
    n_out += all;
    n_eq += eq_all;
    __syncthreads();
  }
  // exponents of the blocks as they will be, and how far every token's move
  const int nb_new = (keep + a.block - 1) / a.block;
  for (int jb = tid; jb < nb_new * 2; jb += EV_THREADS) {
    const int blk = jb >> 1, kind = jb & 1, j0 = blk * a.block, j1 = min(keep, j0 + a.block);
    const int8_t *old = old_e + kind * a.max_blocks;
    int e = -128;
    for (int j = j0; j < j1; ++j) e = max(e, (int)old[kept[j] / a.block]);
    for (int j = j0; j < j1; ++j) delta[j * 2 + kind] = (int8_t)max(-128, (int)old[kept[j] / a.block] - e);
    a.exps[((long long)table[blk] * 2 + kind) * a.n_kv + h] = (int8_t)e;
  }
}

// blockIdx.x: (row, key head), y: kind, z: stretch of `slice` bytes of a token.
__global__ void __launch_bounds__(MV_THREADS) evict_move_kernel(const __grid_constant__ EvictArgs a, int slice) {
  const int bh = blockIdx.x, b = bh / a.n_kv, h = bh - b * a.n_kv, kind = blockIdx.y;
  const int keep = a.n_keep[bh];
  if (h == 0 && kind == 0 && blockIdx.z == 0 && threadIdx.x == 0) a.new_ctx[b] = keep > 0 ? keep : a.ctx[b];
  if (keep == 0) return;
  const int lanes = slice >> 4, per = MV_THREADS / lanes;             // threads per token, tokens per round
  const int tok = threadIdx.x / lanes, off = blockIdx.z * slice + (threadIdx.x % lanes) * 16;
  const int *kept = a.kept + (long long)bh * a.max_keep;
  const int8_t *delta = a.delta + (long long)bh * a.max_keep * 2 + kind;
  const int *table = a.block_table + (long long)b * a.max_blocks;
  auto where = [&](int i) {
    const long long page = table[i / a.block];
    return a.pool + (((page * 2 + kind) * a.n_kv + h) * a.block + i % a.block) * a.hd + off;
  };
  uint4 v[MV_AHEAD];
  int d[MV_AHEAD];                                                    // exponent shift, 1 = the token is where it was
  auto fetch = [&](int r, uint4 &x, int &s) {
    const int j = r * per + tok;
    s = 1;
    if (j < keep) {
      const int src = kept[j], dl = delta[j * 2];
      if (src != j || dl != 0) {
        s = dl;
        x = *reinterpret_cast<const uint4 *>(where(src));
      }
    }
  };
  const int rounds = (keep + per - 1) / per;
#pragma unroll
  for (int e = 0; e < MV_AHEAD; ++e) { v[e] = make_uint4(0u, 0u, 0u, 0u); fetch(e, v[e], d[e]); }
  for (int r0 = 0; r0 < rounds; r0 += MV_AHEAD) {
#pragma unroll
    for (int e = 0; e < MV_AHEAD; ++e) {
      const int r = r0 + e;
      __syncthreads();                                                // this round's loads come before its stores
      if (r < rounds && d[e] <= 0) {
        uint4 x = v[e];
        if (d[e] < 0) {
          const float f = pow2f(max(d[e], -100));
          x.x = e4m3x4_shift(x.x, f); x.y = e4m3x4_shift(x.y, f); x.z = e4m3x4_shift(x.z, f); x.w = e4m3x4_shift(x.w, f);
        }
        *reinterpret_cast<uint4 *>(where(r * per + tok)) = x;
      }
      fetch(r + MV_AHEAD, v[e], d[e]);
    }
  }
}

}  // namespace
}  // namespace corun

using namespace corun;

extern "C" {

int64_t corun_kv8_evict_bytes(int32_t B, int32_t n_kv, int32_t max_keep) {
  if (B < 1 || n_kv < 1 || max_keep < 1) return 0;
  const int64_t bh = (int64_t)B * n_kv;
  return (bh * 4 + 255) / 256 * 256 + bh * max_keep * 2;
}

int corun_kv8_evict(const corun_kv8_cache *cache, const int32_t *block_table, int32_t max_blocks, int32_t B, const int32_t *ctx,
                    int32_t *new_ctx, float *mass, const int32_t *keep, int32_t max_keep, int32_t sinks, int32_t recent,
                    int32_t *kept, void *ws, int64_t ws_bytes, void *cuda_stream) {
  if (!kv8_cache_ok(cache) || !block_table || !ctx || !new_ctx || !mass || !keep || !kept || !ws || B < 1 || B > 65535 || max_blocks < 1 ||
      max_blocks > 65536 || (int64_t)B * cache->n_kv >= (1ll << 31) || sinks < 0 || recent < 0 || max_keep < 1 ||
      (int64_t)sinks + recent > max_keep || max_keep > (int64_t)max_blocks * cache->block || !aligned_to(ws, 256) ||
      ws_bytes < corun_kv8_evict_bytes(B, cache->n_kv, max_keep))
    return CORUN_EINVAL;
  int dev = 0, sms = 0;
  cudaError_t ce = cudaGetDevice(&dev);
  if (ce == cudaSuccess) ce = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (ce != cudaSuccess || sms < 1) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const int bh = B * cache->n_kv;
  EvictArgs a{(uint8_t *)cache->pool, cache->exps, cache->pages, cache->block, cache->n_kv, cache->head_dim, B, max_blocks, max_keep, sinks,
              recent, block_table, ctx, keep, new_ctx, kept, (int *)ws, mass, (int8_t *)ws + ((int64_t)bh * 4 + 255) / 256 * 256};
  const size_t smem = 2 * (size_t)max_blocks;     // at most 128 KiB
  if (smem > 32768) ce = cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * 65536);
  if (ce == cudaSuccess) ce = launch_k(evict_select_kernel, dim3(bh), dim3(EV_THREADS), smem, st, false, a);
  // whole tokens where there are CTAs enough for the card, else stretches of 32 bytes
  const int slice = 2 * bh >= 2 * sms ? cache->head_dim : 32;
  if (ce == cudaSuccess)
    ce = launch_k(evict_move_kernel, dim3(bh, 2, cache->head_dim / slice), dim3(MV_THREADS), 0, st, false, a, slice);
  if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  return CORUN_OK;
}

}  // extern "C"
