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
// the cache is needed.  Bound by bytes: the weights once (the digits' passes read shared memory), the tokens that stay once in, once out.
// 16 rows of 6000 to 8192 tokens cut to 2048 (8 key heads of 128): listing 25 us and moving 36 us from a cold cache (under the
// profiler; 52 us in all without, 22 at the copy rate), and 33 us in all where the tokens that stay lie in order already, as behind an earlier
// eviction: they are not moved again.  The listing is a chain of passes with a CTA per (row, head) on 128 of 148 SMs; counting equal digits
// of a warp together took it to 34 us, 1024 threads changed nothing.  The move needs its loads spread over many warps: two rounds ahead
// 36 us, four 36, eight 54; sources looked up page by page instead of listed 57; stretches of 32 bytes read 112 MB instead of 68 from DRAM.
#include <atomic>

#include "kv8.cuh"

namespace corun {
namespace {

constexpr int EV_THREADS = 512, EV_WARPS = EV_THREADS / 32;
constexpr int EV_BINS = 2048;
constexpr int EV_SMEM = 180 * 1024; // dynamic shared memory at most (the exponents alone take 128 KiB at most)
constexpr int EV_PER = 4;           // tokens of a thread in a round of the listing
constexpr int MV_THREADS = 256, MV_AHEAD = 4;
constexpr int MV_LIST = 2048;       // tokens whose sources are held in shared memory

struct EvictArgs {
  uint8_t *pool;
  int8_t *exps;
  long long pages;
  int block, n_kv, hd, B, max_blocks, max_keep, sinks, recent, keys_in_smem;
  const int *block_table, *ctx, *keep;
  int *new_ctx, *kept, *n_keep;   // n_keep [B * n_kv]: tokens that stay, 0 = the row stays as it is
  float *mass;
  int *src;                       // [B * n_kv][max_keep]: a token's former row of keys in the pool
  int8_t *delta;                  // [B * n_kv][max_keep][2]: how far a token's exponents move (<= 0); 1 = the token is where it was
};

// Weights in the order of unsigned integers: larger weight, larger key; both zeros alike, NaN smallest.
__device__ __forceinline__ uint32_t mass_key(float m) {
  if (m != m) return 0u;
  const uint32_t b = __float_as_uint(m + 0.f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  // [weights' keys, where they fit][exponents of the row's blocks: keys, values]
  extern __shared__ __align__(16) uint8_t ev_smem[];
  __shared__ int hist[EV_BINS];
  __shared__ int s_w[2][EV_WARPS], s_bin, s_above, s_bad;
  const int b = blockIdx.x / a.n_kv, h = blockIdx.x - b * a.n_kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long reach = (long long)a.max_blocks * a.block;
  uint32_t *keys = reinterpret_cast<uint32_t *>(ev_smem);
  int8_t *old_e = reinterpret_cast<int8_t *>(ev_smem + (a.keys_in_smem ? reach * 4 : 0));
  griddep_wait();
  const int n = a.ctx[b];
  int keep = a.keep[b];
  if (keep > 0) keep = min(max(keep, a.sinks + a.recent), a.max_keep);
  const long long list = (long long)blockIdx.x * a.max_keep;
  int *kept = a.kept + list;
  float *mass = a.mass + (long long)blockIdx.x * reach;
  const int *table = a.block_table + (long long)b * a.max_blocks;
  const bool cut = keep > 0 && keep < n && n <= reach;
  const int nb = cut ? (n + a.block - 1) / a.block : 0;
  const int shift = a.block == 16 ? 4 : a.block == 32 ? 5 : 6;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  for (int i = tid; i < nb; i += EV_THREADS) {
    const long long page = table[i];
    if (page < 0 || page >= a.pages) { s_bad = 1; continue; }
    old_e[i] = a.exps[(page * 2) * a.n_kv + h];
    old_e[a.max_blocks + i] = a.exps[(page * 2 + 1) * a.n_kv + h];
  }
  if (cut && a.keys_in_smem)
    for (int i = tid; i < n; i += EV_THREADS) keys[i] = mass_key(mass[i]);
  __syncthreads();
  const bool go = cut && !s_bad;
  if (tid == 0) a.n_keep[blockIdx.x] = go ? keep : 0;
  for (int i = tid + (go ? keep : 0); i < a.max_keep; i += EV_THREADS) kept[i] = -1;
  if (!go) return;
  auto key_at = [&](int i) { return a.keys_in_smem ? keys[i] : mass_key(mass[i]); };
  // the weight of the last token that stays among those between the sinks and the recent ones
  const int lo = a.sinks, hi = n - a.recent, want = keep - a.sinks - a.recent;
  uint32_t found = 0u, mask = 0u;
  int left = want;                                // how many stay among the tokens that agree with `found` under `mask`
  if (want > 0) {
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
      const int shift_d = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
      for (int i = tid; i < EV_BINS; i += EV_THREADS) hist[i] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += EV_THREADS) {
        const uint32_t k = key_at(i);
        if (((k ^ found) & mask) == 0u) atomicAdd(&hist[(k >> shift_d) & ((1u << bits) - 1u)], 1);
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
      found |= (uint32_t)s_bin << shift_d;
      mask |= ((1u << bits) - 1u) << shift_d;
      left -= s_above;
      __syncthreads();
    }
  }
  // tokens that stay, in order: `left` of those whose weight is the last one's, from the front.  A thread takes EV_PER neighbours.
  int n_out = 0, n_eq = 0;
  for (int i0 = 0; i0 < n; i0 += EV_THREADS * EV_PER) {
    const int i1 = i0 + tid * EV_PER;
    float m[EV_PER];
    uint32_t sure = 0u, eq = 0u;                  // bit e: token i1 + e stays whatever comes / has the last weight
#pragma unroll
    for (int e = 0; e < EV_PER; ++e) {
      const int i = i1 + e;
      m[e] = 0.f;
      if (i < n) {
        m[e] = mass[i];
        const uint32_t k = key_at(i);
        const bool always = i < lo || i >= hi;
        if (always || (want > 0 && k > found)) sure |= 1u << e;
        else if (want > 0 && k == found) eq |= 1u << e;
      }
    }
    auto before = [&](int mine, int *s, int &all) { // of the threads before this one, and of all
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
      }
      if (lane == 31) s[warp] = inc;
      __syncthreads();
      int at = inc - mine;
      all = 0;
#pragma unroll
      for (int w = 0; w < EV_WARPS; ++w) { const int v = s[w]; if (w < warp) at += v; all += v; }
      return at;
    };
    int all_eq, all;
    int e_at = n_eq + before(__popc(eq), s_w[0], all_eq);
    uint32_t stays = sure;
#pragma unroll
    for (int e = 0; e < EV_PER; ++e)
      if (eq >> e & 1u) { if (e_at < left) stays |= 1u << e; ++e_at; }
    int j = n_out + before(__popc(stays), s_w[1], all);              // (all weights of this pass have been read)
#pragma unroll
    for (int e = 0; e < EV_PER; ++e)
      if (stays >> e & 1u) {
        kept[j] = i1 + e;
        mass[j] = m[e];                           // j <= i1 + e: in front of what later rounds read
        ++j;
      }
    n_out += all;
    n_eq += all_eq;
    __syncthreads();
  }
  // exponents of the blocks as they will be, how far every token's move, and where its values are.  A warp takes 64 tokens: four, two
  // blocks or one.
  for (int j0 = warp * 64; j0 < keep; j0 += EV_WARPS * 64) {
    int i[2], ek[2], ev[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = j0 + 32 * e + lane;
      i[e] = j < keep ? kept[j] : -1;
      ek[e] = ev[e] = -128;
      if (i[e] >= 0) { ek[e] = old_e[i[e] >> shift]; ev[e] = old_e[a.max_blocks + (i[e] >> shift)]; }
    }
    int mk[2] = {ek[0], ek[1]}, mv[2] = {ev[0], ev[1]};
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int o = 1; o < 32; o <<= 1)
        if (o < a.block) {
          mk[e] = max(mk[e], __shfl_xor_sync(0xffffffffu, mk[e], o));
          mv[e] = max(mv[e], __shfl_xor_sync(0xffffffffu, mv[e], o));
        }
    if (a.block == 64) { mk[0] = mk[1] = max(mk[0], mk[1]); mv[0] = mv[1] = max(mv[0], mv[1]); }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = j0 + 32 * e + lane;
      if (j >= keep) continue;
      const bool still = i[e] == j;
      a.delta[(list + j) * 2] = (int8_t)(still && ek[e] == mk[e] ? 1 : max(ek[e] - mk[e], -127));
      a.delta[(list + j) * 2 + 1] = (int8_t)(still && ev[e] == mv[e] ? 1 : max(ev[e] - mv[e], -127));
      a.src[list + j] = (int)(((long long)table[i[e] >> shift] * 2 * a.n_kv + h) * a.block + (i[e] & (a.block - 1)));
      if ((j & (a.block - 1)) == 0) {
        const long long page = table[j >> shift];
        a.exps[(page * 2) * a.n_kv + h] = (int8_t)mk[e];
        a.exps[(page * 2 + 1) * a.n_kv + h] = (int8_t)mv[e];
      }
    }
  }
}

// blockIdx.x: (row, key head), y: kind, z: stretch of `slice` bytes of a token.
__global__ void __launch_bounds__(MV_THREADS) evict_move_kernel(const __grid_constant__ EvictArgs a, int slice) {
  __shared__ int s_src[MV_LIST];
  __shared__ int8_t s_delta[MV_LIST];
  __shared__ int s_page[MV_LIST / 16];
  griddep_wait();
  const int bh = blockIdx.x, b = bh / a.n_kv, h = bh - b * a.n_kv, kind = blockIdx.y;
  const int keep = a.n_keep[bh];
  if (h == 0 && kind == 0 && blockIdx.z == 0 && threadIdx.x == 0) a.new_ctx[b] = keep > 0 ? keep : a.ctx[b];
  if (keep == 0) return;
  const int lanes = slice >> 4, per = MV_THREADS / lanes;             // threads per token, tokens per round
  const int tok = threadIdx.x / lanes, shift = a.block == 16 ? 4 : a.block == 32 ? 5 : 6;
  const long long list = (long long)bh * a.max_keep, kind_rows = (long long)a.n_kv * a.block;   // rows between a token's keys and values
  uint8_t *pool = a.pool + (long long)kind * kind_rows * a.hd + blockIdx.z * slice + (threadIdx.x % lanes) * 16;
  const int *table = a.block_table + (long long)b * a.max_blocks;
  for (int l0 = 0; l0 < keep; l0 += MV_LIST) {
    const int nl = min(MV_LIST, keep - l0), rounds = (nl + per - 1) / per;
    __syncthreads();
    for (int i = threadIdx.x; i < nl; i += MV_THREADS) {
      s_src[i] = __ldcg(a.src + list + l0 + i);
      s_delta[i] = a.delta[(list + l0 + i) * 2 + kind];
    }
    for (int i = threadIdx.x; i < (nl + a.block - 1) >> shift; i += MV_THREADS) s_page[i] = table[(l0 >> shift) + i];
    __syncthreads();
    uint4 v[MV_AHEAD];
    int d[MV_AHEAD];
    auto fetch = [&](int r, uint4 &x, int &s) {
      const int j = r * per + tok;
      s = 1;
      if (r < rounds && j < nl) {
        s = s_delta[j];
        if (s <= 0) x = *reinterpret_cast<const uint4 *>(pool + (long long)s_src[j] * a.hd);
      }
    };
#pragma unroll
    for (int e = 0; e < MV_AHEAD; ++e) { v[e] = make_uint4(0u, 0u, 0u, 0u); fetch(e, v[e], d[e]); }
    for (int r0 = 0; r0 < rounds; r0 += MV_AHEAD) {
#pragma unroll
      for (int e = 0; e < MV_AHEAD; ++e) {
        const int r = r0 + e;
        __syncthreads();                                              // this round's loads come before its stores
        if (r < rounds && d[e] <= 0) {
          uint4 x = v[e];
          if (d[e] < 0) {
            const float f = pow2f(max(d[e], -100));
            x.x = e4m3x4_shift(x.x, f); x.y = e4m3x4_shift(x.y, f); x.z = e4m3x4_shift(x.z, f); x.w = e4m3x4_shift(x.w, f);
          }
          const int j = r * per + tok;
          const long long row = ((long long)s_page[j >> shift] * 2 * a.n_kv + h) * a.block + (j & (a.block - 1));
          *reinterpret_cast<uint4 *>(pool + row * a.hd) = x;
        }
        fetch(r + MV_AHEAD, v[e], d[e]);
      }
    }
  }
}

}  // namespace
}  // namespace corun

using namespace corun;

extern "C" {

int64_t corun_kv8_evict_bytes(int32_t B, int32_t n_kv, int32_t max_keep) {
  if (B < 1 || n_kv < 1 || max_keep < 1) return 0;
  const int64_t bh = (int64_t)B * n_kv, up = (bh * 4 + 255) / 256 * 256;
  return up + bh * max_keep * 6;
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
  cudaError_t ce = device_sms(&dev, &sms);
  if (ce != cudaSuccess || sms < 1) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const int bh = B * cache->n_kv;
  // the weights' keys stay in shared memory where they fit (40 K tokens; beyond that every pass reads the weights from L2)
  const int64_t reach = (int64_t)max_blocks * cache->block;
  const bool keys_in_smem = reach * 4 + 2 * max_blocks <= EV_SMEM;
  char *w = (char *)ws;
  int *src = (int *)(w + ((int64_t)bh * 4 + 255) / 256 * 256);
  const EvictArgs a{(uint8_t *)cache->pool, cache->exps, cache->pages, cache->block, cache->n_kv, cache->head_dim, B, max_blocks, max_keep, sinks,
                    recent, keys_in_smem ? 1 : 0, block_table, ctx, keep, new_ctx, kept, (int *)w, mass, src, (int8_t *)(src + (int64_t)bh * max_keep)};
  const size_t smem = 2 * (size_t)max_blocks + (keys_in_smem ? (size_t)reach * 4 : 0);
  if (smem > 32768) {
    static std::atomic<uint64_t> done{0};         // opted into once per device
    if (dev >= 64 || !(done.load() >> dev & 1)) {
      ce = cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_SMEM);
      if (ce == cudaSuccess && dev < 64) done.fetch_or(1ull << dev);
    }
  }
  if (ce == cudaSuccess) ce = launch_k(evict_select_kernel, dim3(bh), dim3(EV_THREADS), smem, st, true, a);
  // stretches of 64 bytes (what DRAM hands out) where they make CTAs enough for the card, else of 32
  const int slice = cache->head_dim / 64 * 2 * bh >= sms ? 64 : 32;
  if (ce == cudaSuccess)
    ce = launch_k(evict_move_kernel, dim3(bh, 2, cache->head_dim / slice), dim3(MV_THREADS), 0, st, true, a, slice);
  if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  return CORUN_OK;
}

}  // extern "C"
