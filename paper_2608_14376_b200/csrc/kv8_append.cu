// New keys and values into the 8-bit cache (include/corun_kv8.h), with the rotation of keys and queries on the way.
//
// A unit is one page that a row's new tokens touch.  Its scale is set by all tokens of the page together, so one warp takes
// a (page, key head, kind): it reads its tokens, finds the largest magnitude, settles the page's exponent, moves what the
// page held before to it where it grew, and reads its tokens once more (from L1 by then) to store them.  The op is bound by
// bytes (16-bit inputs in, a byte a value out, queries in and out); cos and sin are computed once per CTA and used for all of
// its heads.  Units are found from ctx and cu on the device: the launch's shape depends on T and B alone, so it can be captured
// and replayed with other lengths.
// One token for each of 64 rows (32 query, 8 key heads of 128, bf16): 6 us, a chain of latencies (lengths, positions, keys, stores).  1252
// tokens of 3 rows: 14.6 us (4.4 at the copy rate; some 80 pages, 128 registers a thread).
#include "kv8.cuh"

namespace corun {
namespace {

constexpr int AP_THREADS = 256, AP_WARPS = AP_THREADS / 32;

struct AppendArgs {
  uint8_t *pool;
  int8_t *exps;
  long long pages;
  int block, n_kv, n_q, B, T, max_blocks;
  const int *block_table, *ctx, *cu, *positions;
  const void *k, *v, *q;
  void *q_out;
  long long k_t, k_h, v_t, v_h, q_t, q_h, o_t, o_h;
  float *mass;
};

// New tokens of row b and the first of them, or 0 where the row is left out.
__device__ __forceinline__ int row_tokens(const int *ctx, const int *cu, int b, int T, long long reach, int &first, int &c) {
  c = __ldcg(ctx + b);
  int n = 1;
  first = b;
  if (cu) {
    first = __ldcg(cu + b);
    const int end = __ldcg(cu + b + 1);
    n = end - first;
    if (first < 0 || end < first || end > T) return 0;
  }
  return c > 0 && n > 0 && n <= c && (long long)c <= reach ? n : 0;
}

// EPL neighbouring values of a head per lane: d0 = lane * EPL.
template <typename T, int EPL>
struct LanePack { T v[EPL]; };

template <typename T, int EPL>
__device__ __forceinline__ LanePack<T, EPL> lane_load(const T *x) {
  const int d0 = (threadIdx.x & 31) * EPL;
  LanePack<T, EPL> p;
#pragma unroll
  for (int e = 0; e < EPL; ++e) p.v[e] = x[d0 + e];
  return p;
}

// The lane's values of one head of one token, rotated with the token's cos and sin (x: the head in memory).
template <typename T, int EPL>
__device__ __forceinline__ void lane_values(const LanePack<T, EPL> &p, const T *x, const float2 *cs, int rot, bool interleaved, float (&o)[EPL]) {
  const int d0 = (threadIdx.x & 31) * EPL;
#pragma unroll
  for (int e = 0; e < EPL; ++e) o[e] = to_f32(p.v[e]);
  if (rot == 0) return;
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < EPL; e += 2) {
      if (d0 + e < rot) {
        const float2 f = cs[(d0 + e) >> 1];
        const float x1 = o[e], x2 = o[e + 1];
        o[e] = turn1(x1, x2, f);
        o[e + 1] = turn2(x1, x2, f);
      }
    }
    return;
  }
  const int half = rot >> 1;
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    const int d = d0 + e;
    float other;
    if (half % EPL == 0) {                        // the partner is the same value of another lane
      const int src = (d0 < half ? d0 + half : d0 - half) / EPL;
      other = __shfl_sync(0xffffffffu, o[e], src & 31);
    } else {
      other = d < rot ? to_f32(x[d < half ? d + half : d - half]) : 0.f;
    }
    // (with shuffles o[e] is replaced below only after every lane has read it: one e at a time, and e is its own value)
    if (d < half) o[e] = turn1(o[e], other, cs[d]);
    else if (d < rot) o[e] = turn2(other, o[e], cs[d - half]);
  }
}

template <int EPL>
__device__ __forceinline__ void store8(uint8_t *dst, const float (&x)[EPL], float f) {
  if (EPL == 4) {
    *reinterpret_cast<uint32_t *>(dst) = e4m3x2_of(x[0] * f, x[1] * f) | (e4m3x2_of(x[2 % EPL] * f, x[3 % EPL] * f) << 16);
  } else {
    *reinterpret_cast<uint16_t *>(dst) = (uint16_t)e4m3x2_of(x[0] * f, x[1] * f);
  }
}

// The unit of this CTA (blockIdx.x): a row and one of the pages that its new tokens touch; units are numbered row by row.
struct Unit { int row, page, first, c, n; };   // row -1: none (the grid is an upper bound)
__device__ __forceinline__ Unit find_unit(const AppendArgs &a, int *s_warp, Unit *s_unit) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long reach = (long long)a.max_blocks * a.block;
  if (tid == 0) s_unit->row = -1;
  griddep_wait();
  griddep_launch_dependents();
  int before = 0;
  for (int b0 = 0; b0 < a.B; b0 += AP_THREADS) {
    const int b = b0 + tid;
    int units = 0, first = 0, c = 0, n = 0;
    if (b < a.B) {
      n = row_tokens(a.ctx, a.cu, b, a.T, reach, first, c);
      if (n > 0) units = (c - 1) / a.block - (c - n) / a.block + 1;
    }
    int inc = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    int ahead = before, all = 0;
    for (int w = 0; w < AP_WARPS; ++w) { if (w < warp) ahead += s_warp[w]; all += s_warp[w]; }
    const int lo = ahead + inc - units;
    if ((int)blockIdx.x >= lo && (int)blockIdx.x < lo + units) *s_unit = Unit{b, (c - n) / a.block + (int)blockIdx.x - lo, first, c, n};
    before += all;
    __syncthreads();
    if (s_unit->row >= 0) break;
  }
  return *s_unit;
}

// The exponent of a page that new tokens of largest magnitude mx come to, and what it held before moved to it (by a warp).
template <int HD>
__device__ __forceinline__ int settle(const AppendArgs &a, long long at, int z0, float mx) {
  const int lane = threadIdx.x & 31;
  int e = kv8_exp_of(mx);
  if (z0 > 0) {
    const int e_old = a.exps[at];
    if (e > e_old) {
      const float f = pow2f(max(e_old - e, -100));
      uint4 *old = reinterpret_cast<uint4 *>(a.pool + at * a.block * HD);
#pragma unroll 2
      for (int i = lane; i < z0 * HD / 16; i += 32) {
        uint4 x = old[i];
        x.x = e4m3x4_shift(x.x, f); x.y = e4m3x4_shift(x.y, f); x.z = e4m3x4_shift(x.z, f); x.w = e4m3x4_shift(x.w, f);
        old[i] = x;
      }
    } else {
      e = e_old;
    }
  }
  __syncwarp();
  if (lane == 0) a.exps[at] = (int8_t)e;
  return e;
}

// Value by value, for layouts whose heads do not start on 16 bytes or whose rotated part is not made of whole pieces.
template <typename T, int HD>
__global__ void __launch_bounds__(AP_THREADS) append_odd_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ RopeTable tab) {
  constexpr int EPL = HD / 32, AHEAD = 4;
  typedef LanePack<T, EPL> P;
  extern __shared__ __align__(16) float2 cs[];                 // [tokens of the unit][rot / 2]
  __shared__ int s_warp[AP_WARPS];
  __shared__ Unit s_unit;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const Unit u = find_unit(a, s_warp, &s_unit);
  if (u.row < 0) return;
  const int row = u.row, jb = u.page, start = u.c - u.n;
  const int z0 = max(0, start - jb * a.block), z1 = min(a.block, u.c - jb * a.block);   // the page's new tokens
  const int t0 = u.first + jb * a.block + z0 - start, nt = z1 - z0;
  const long long reach = (long long)a.max_blocks * a.block;
  const int pairs = tab.rot >> 1;
  for (int i = tid; i < nt * pairs; i += AP_THREADS) {
    const int t = i / pairs, p = i - t * pairs;
    cs[i] = rope_cs(tab, p, __ldcg(a.positions + t0 + t));
  }
  __syncthreads();
  const long long page = __ldcg(a.block_table + (long long)row * a.max_blocks + jb);
  const bool page_ok = page >= 0 && page < a.pages;
  const int n_task = 2 * a.n_kv + a.n_q;
  for (int task = blockIdx.y * AP_WARPS + warp; task < n_task; task += gridDim.y * AP_WARPS) {
    if (task < 2 * a.n_kv) {
      const int kind = task & 1, h = task >> 1;
      if (kind == 0 && a.mass)
        for (int i = lane; i < nt; i += 32) a.mass[((long long)row * a.n_kv + h) * reach + (long long)jb * a.block + z0 + i] = 0.f;
      if (!page_ok) continue;
      const T *x = (const T *)(kind ? a.v : a.k) + (long long)t0 * (kind ? a.v_t : a.k_t) + (long long)h * (kind ? a.v_h : a.k_h);
      const long long step = kind ? a.v_t : a.k_t;
      const int rot = kind ? 0 : tab.rot;
      const long long at = (page * 2 + kind) * a.n_kv + h;
      uint8_t *dst = a.pool + at * a.block * HD + lane * EPL;
      float mx = 0.f;
      P raw[AHEAD];
      auto request = [&](int t1) {
#pragma unroll
        for (int t = 0; t < AHEAD; ++t)
          if (t1 + t < nt) raw[t] = lane_load<T, EPL>(x + (t1 + t) * step);
      };
      for (int t1 = 0; t1 < nt; t1 += AHEAD) {
        request(t1);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t)
          if (t1 + t < nt) {
            float o[EPL];
            lane_values<T, EPL>(raw[t], x + (t1 + t) * step, cs + (t1 + t) * pairs, rot, tab.interleaved, o);
#pragma unroll
            for (int e = 0; e < EPL; ++e) mx = fmaxf(mx, fabsf(o[e]));
          }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const int e_new = settle<HD>(a, at, z0, mx);
      const float f = pow2f(-e_new);
      for (int t1 = 0; t1 < nt; t1 += AHEAD) {
        if (nt > AHEAD) request(t1);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t)
          if (t1 + t < nt) {
            float o[EPL];
            lane_values<T, EPL>(raw[t], x + (t1 + t) * step, cs + (t1 + t) * pairs, rot, tab.interleaved, o);
            store8<EPL>(dst + (z0 + t1 + t) * HD, o, f);
          }
      }
    } else {
      const int h = task - 2 * a.n_kv;
      const T *x = (const T *)a.q + (long long)t0 * a.q_t + (long long)h * a.q_h;
      T *y = (T *)a.q_out + (long long)t0 * a.o_t + (long long)h * a.o_h;
      for (int t1 = 0; t1 < nt; t1 += AHEAD) {
        P raw[AHEAD];
#pragma unroll
        for (int t = 0; t < AHEAD; ++t)
          if (t1 + t < nt) raw[t] = lane_load<T, EPL>(x + (t1 + t) * a.q_t);
#pragma unroll
        for (int t = 0; t < AHEAD; ++t)
          if (t1 + t < nt) {
            float o[EPL];
            lane_values<T, EPL>(raw[t], x + (t1 + t) * a.q_t, cs + (t1 + t) * pairs, tab.rot, tab.interleaved, o);
            __syncwarp();                           // (in place: every partner has been read)
            T *to = y + (t1 + t) * a.o_t + lane * EPL;
#pragma unroll
            for (int e = 0; e < EPL; ++e) to[e] = from_f32<T>(o[e]);
          }
      }
    }
  }
}

// Sixteen bytes at a time: a thread holds a piece of a head (two groups of VEC values that are rotated together).  Keys and values: a
// warp per (kind, head), NP lanes a token, so 4 (fp32: 2; heads of 64: twice that) tokens at a time, twice over the page's new tokens.
// Queries: a thread per (token, piece) goes through heads with its pairs' cos and sin in registers.
template <typename T, int HD>
__global__ void __launch_bounds__(AP_THREADS) append_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ RopeTable tab) {
  constexpr int VEC = Piece<T>::VEC, NP = HD / (2 * VEC), SLOTS = AP_THREADS / NP, STEP = 32 / NP, AHEAD = 4;
  extern __shared__ __align__(16) float2 cs_s[];              // [tokens of the unit][rot / 2]
  __shared__ int s_warp[AP_WARPS];
  __shared__ Unit s_unit;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const Unit u = find_unit(a, s_warp, &s_unit);
  if (u.row < 0) return;
  const int jb = u.page, start = u.c - u.n;
  const int z0 = max(0, start - jb * a.block), z1 = min(a.block, u.c - jb * a.block);   // the page's new tokens
  const int t0 = u.first + jb * a.block + z0 - start, nt = z1 - z0;
  const int pairs = tab.rot >> 1;
  for (int i = tid; i < nt * pairs; i += AP_THREADS) {
    const int t = i / pairs, p = i - t * pairs;
    cs_s[i] = rope_cs(tab, p, __ldcg(a.positions + t0 + t));
  }
  __syncthreads();
  const int piece = tid % NP;
  const PieceAt at = piece_at<VEC>(tab, piece);
  auto angles = [&](int t, float2 (&cs)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
      const float4 f = *reinterpret_cast<const float4 *>(cs_s + t * pairs + piece * VEC + i);
      cs[i] = make_float2(f.x, f.y);
      cs[i + 1] = make_float2(f.z, f.w);
    }
  };
  const long long page = __ldcg(a.block_table + (long long)u.row * a.max_blocks + jb);
  const bool page_ok = page >= 0 && page < a.pages;
  for (int task = blockIdx.y * AP_WARPS + warp; task < 2 * a.n_kv; task += gridDim.y * AP_WARPS) {
    const int kind = task & 1, h = task >> 1;
    if (kind == 0 && a.mass) {
      const long long reach = (long long)a.max_blocks * a.block;
      for (int i = lane; i < nt; i += 32) a.mass[((long long)u.row * a.n_kv + h) * reach + (long long)jb * a.block + z0 + i] = 0.f;
    }
    if (!page_ok) continue;
    const long long step = kind ? a.v_t : a.k_t;
    const T *x = (const T *)(kind ? a.v : a.k) + (long long)t0 * step + (long long)h * (kind ? a.v_h : a.k_h);
    const bool turned = kind == 0 && at.turned;
    const long long block_at = (page * 2 + kind) * a.n_kv + h;
    uint8_t *dst = a.pool + (block_at * a.block + z0) * HD;
    float mx = 0.f;
    // AHEAD tokens of a lane are requested together; with no more than that they are kept for the second time
    Piece<T> v[AHEAD];
    auto request = [&](int tb) {
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        if (tb + e * STEP < nt) piece_load(v[e], x + (tb + e * STEP) * step, at);
    };
    for (int tb = lane / NP; tb < nt; tb += AHEAD * STEP) {
      request(tb);
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        if (tb + e * STEP < nt) {
          float2 cs[VEC];
          float p[VEC], q[VEC];
          if (turned) angles(tb + e * STEP, cs);
          piece_turn(v[e], cs, turned, tab.interleaved, p, q);
#pragma unroll
          for (int i = 0; i < VEC; ++i) mx = fmaxf(mx, fmaxf(fabsf(p[i]), fabsf(q[i])));
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float f = pow2f(-settle<HD>(a, block_at, z0, mx));
    for (int tb = lane / NP; tb < nt; tb += AHEAD * STEP) {
      if (nt > AHEAD * STEP) request(tb);
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        if (tb + e * STEP < nt) {
          const int t = tb + e * STEP;
          float2 cs[VEC];
          float p[VEC], q[VEC];
          if (turned) angles(t, cs);
          piece_turn(v[e], cs, turned, tab.interleaved, p, q);
          uint32_t w[2][VEC / 4];
#pragma unroll
          for (int i = 0; i < VEC; i += 4) {
            w[0][i / 4] = e4m3x2_of(p[i] * f, p[i + 1] * f) | (e4m3x2_of(p[i + 2] * f, p[i + 3] * f) << 16);
            w[1][i / 4] = e4m3x2_of(q[i] * f, q[i + 1] * f) | (e4m3x2_of(q[i + 2] * f, q[i + 3] * f) << 16);
          }
          if (VEC == 8) {
            *reinterpret_cast<uint2 *>(dst + t * HD + at.a) = make_uint2(w[0][0], w[0][VEC / 4 - 1]);
            *reinterpret_cast<uint2 *>(dst + t * HD + at.b) = make_uint2(w[1][0], w[1][VEC / 4 - 1]);
          } else {
            *reinterpret_cast<uint32_t *>(dst + t * HD + at.a) = w[0][0];
            *reinterpret_cast<uint32_t *>(dst + t * HD + at.b) = w[1][0];
          }
        }
    }
  }
  // queries: the slots are shared out among tokens (a power of two of them) and heads
  if (a.n_q == 0) return;
  int ts = 0;
  while ((1 << ts) < nt && (1 << ts) < SLOTS) ++ts;
  const int slot = tid / NP, heads_at_once = SLOTS >> ts;
  const int per = (a.n_q + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * per, h1 = min(a.n_q, h0 + per);
  for (int t = slot & ((1 << ts) - 1); t < nt; t += 1 << ts) {
    float2 cs[VEC];
    if (at.turned) angles(t, cs);
    const T *x = (const T *)a.q + (long long)(t0 + t) * a.q_t;
    T *y = (T *)a.q_out + (long long)(t0 + t) * a.o_t;
    for (int hb = h0 + (slot >> ts); hb < h1; hb += AHEAD * heads_at_once) {
      Piece<T> v[AHEAD];
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        if (hb + e * heads_at_once < h1) piece_load(v[e], x + (long long)(hb + e * heads_at_once) * a.q_h, at);
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        if (hb + e * heads_at_once < h1) {
          float p[VEC], q[VEC];
          piece_turn(v[e], cs, at.turned, tab.interleaved, p, q);
#pragma unroll
          for (int i = 0; i < VEC; ++i) { v[e].a[i] = from_f32<T>(p[i]); v[e].b[i] = from_f32<T>(q[i]); }
          T *to = y + (long long)(hb + e * heads_at_once) * a.o_h;
          *reinterpret_cast<uint4 *>(to + at.a) = *reinterpret_cast<const uint4 *>(v[e].a);
          *reinterpret_cast<uint4 *>(to + at.b) = *reinterpret_cast<const uint4 *>(v[e].b);
        }
    }
  }
}

template <typename T>
cudaError_t launch_append(const AppendArgs &a, const RopeTable &tab, int head_dim, bool wide, int sms, cudaStream_t st) {
  // a row's n tokens touch at most (n - 1) / block + 2 pages, and no more than n
  long long gx = (long long)a.T / a.block + 2ll * a.B;
  if (gx > a.T) gx = a.T;
  const int tasks = 2 * a.n_kv + a.n_q;
  int gy = (int)((4ll * sms + gx - 1) / gx);
  if (gy > (tasks + AP_WARPS - 1) / AP_WARPS) gy = (tasks + AP_WARPS - 1) / AP_WARPS;
  const size_t smem = (size_t)a.block * (tab.rot / 2) * sizeof(float2);   // at most 32 KiB
  const dim3 grid((unsigned)gx, (unsigned)gy);
  void (*kernel)(const AppendArgs, const RopeTable) =
      wide ? (head_dim == 128 ? append_kernel<T, 128> : append_kernel<T, 64>) : (head_dim == 128 ? append_odd_kernel<T, 128> : append_odd_kernel<T, 64>);
  return launch_k(kernel, grid, dim3(AP_THREADS), smem, st, true, a, tab);
}

}  // namespace
}  // namespace corun

using namespace corun;

extern "C" int corun_kv8_append(const corun_kv8_cache *cache, const corun_kv8_rows *rows, const corun_heads *k, const corun_heads *v,
                                int32_t dtype, const corun_rope *rope, const int32_t *positions, const corun_heads *q,
                                const corun_heads *q_out, int32_t n_q, float *mass, void *cuda_stream) {
  if (!kv8_cache_ok(cache) || !kv8_rows_ok(rows, cache) || !k || !v || dtype < CORUN_F32 || dtype > CORUN_F16) return CORUN_EINVAL;
  if (q && (!q_out || n_q < 1 || n_q > 65535)) return CORUN_EINVAL;
  if (rope && rope->t.rot > cache->head_dim) return CORUN_EINVAL;
  if (rows->T == 0) return CORUN_OK;               // (tensors of no tokens may have no address)
  const uintptr_t sz = (uintptr_t)dtype_size(dtype);
  if (!k->p || !v->p || !aligned_to(k->p, sz) || !aligned_to(v->p, sz) || (rope && !positions)) return CORUN_EINVAL;
  if (q && (!q->p || !q_out->p || !aligned_to(q->p, sz) || !aligned_to(q_out->p, sz))) return CORUN_EINVAL;
  if (q && q->p == q_out->p && (q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride)) return CORUN_EINVAL;
  int dev = 0, sms = 0;
  cudaError_t ce = device_sms(&dev, &sms);
  if (ce != cudaSuccess || sms < 1) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  const corun_heads none{nullptr, 0, 0}, &qi = q ? *q : none, &qo = q ? *q_out : none;
  const AppendArgs a{(uint8_t *)cache->pool, cache->exps, cache->pages, cache->block, cache->n_kv, q ? n_q : 0, rows->B, rows->T, rows->max_blocks,
                     rows->block_table, rows->ctx, rows->cu, positions, k->p, v->p, qi.p, qo.p, k->token_stride, k->head_stride,
                     v->token_stride, v->head_stride, qi.token_stride, qi.head_stride, qo.token_stride, qo.head_stride, mass};
  static const RopeTable still = {};               // rot 0: nothing is rotated
  const RopeTable &tab = rope ? rope->t : still;
  const bool wide = heads_on_16(*k, dtype) && heads_on_16(*v, dtype) && (!q || (heads_on_16(qi, dtype) && heads_on_16(qo, dtype))) &&
                    tab.rot / 2 % (16 / (int)sz) == 0;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == CORUN_F32) ce = launch_append<float>(a, tab, cache->head_dim, wide, sms, st);
  else if (dtype == CORUN_BF16) ce = launch_append<__nv_bfloat16>(a, tab, cache->head_dim, wide, sms, st);
  else ce = launch_append<__half>(a, tab, cache->head_dim, wide, sms, st);
  if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  return CORUN_OK;
}
