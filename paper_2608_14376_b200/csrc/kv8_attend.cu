// Attention over the 8-bit cache (include/corun_kv8.h): out = softmax(scale q K^T) V, and the weights that the cached tokens received.
//
// One warp per (token, query head): a lane holds head_dim / 32 dims, the cached tokens are taken one after the other with a
// running maximum and sum.  A second kernel, one thread per cached token, forms the scores again and adds up the weights.
#include <math_constants.h>

#include "kv8.cuh"

namespace corun {
namespace {

constexpr int AT_MAXB = 1024;

struct AttendArgs {
  const uint8_t *pool;
  const int8_t *exps;
  long long pages;
  int block, n_kv, n_q, B, T, max_blocks, max_new, window;
  const int *block_table, *ctx, *cu;
  const void *q;
  void *out;
  long long q_t, q_h, o_t, o_h;
  float scale;
  float *mass;
  float2 *ml;   // [T][n_q]
};

__device__ __forceinline__ int row_of(const AttendArgs &a, int t, int &first, int &n) {
  if (!a.cu) { first = t; n = 1; return t < a.B ? t : -1; }
  for (int b = 0; b < a.B; ++b) {
    first = a.cu[b];
    n = a.cu[b + 1] - first;
    if (first >= 0 && t >= first && t < first + n && first + n <= a.T) return b;
  }
  return -1;
}

template <typename T, int HD>
__global__ void __launch_bounds__(128) attend_simple_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int EPL = HD / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = blockIdx.x, hq = blockIdx.y * 4 + warp;
  if (hq >= a.n_q) return;
  int first, n;
  const int b = row_of(a, t, first, n);
  if (b < 0) return;
  const long long reach = (long long)a.max_blocks * a.block;
  const int c = a.ctx[b];
  if (c <= 0 || c > reach || n > a.max_new) return;
  const int g = hq / (a.n_q / a.n_kv), self = c - n + (t - first);
  float q[EPL], o[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) { q[e] = to_f32(((const T *)a.q)[t * a.q_t + hq * a.q_h + lane * EPL + e]) * a.scale; o[e] = 0.f; }
  float m = -CUDART_INF_F, l = 0.f;
  for (int j = a.window ? max(0, self - a.window + 1) : 0; j <= self; ++j) {
    const long long page = a.block_table[(long long)b * a.max_blocks + j / a.block];
    float k[EPL], v[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) k[e] = v[e] = 0.f;
    if (page >= 0 && page < a.pages) {
      const long long ak = (page * 2) * a.n_kv + g, av = ak + a.n_kv;
      const uint8_t *pk = a.pool + (ak * a.block + j % a.block) * HD + lane * EPL, *pv = a.pool + (av * a.block + j % a.block) * HD + lane * EPL;
      const float fk = pow2f(a.exps[ak]), fv = pow2f(a.exps[av]);
#pragma unroll
      for (int e = 0; e < EPL; e += 2) {
        const float2 x = e4m3x2_to(*(const uint16_t *)(pk + e)), y = e4m3x2_to(*(const uint16_t *)(pv + e));
        k[e] = x.x * fk; k[e + 1] = x.y * fk; v[e] = y.x * fv; v[e + 1] = y.y * fv;
      }
    }
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) s = fmaf(q[e], k[e], s);
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) s += __shfl_xor_sync(0xffffffffu, s, i);
    const float m2 = fmaxf(m, s), f = expf(m - m2), p = expf(s - m2);
    l = l * f + p;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[e] = o[e] * f + p * v[e];
    m = m2;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < EPL; ++e) ((T *)a.out)[t * a.o_t + hq * a.o_h + lane * EPL + e] = from_f32<T>(o[e] * inv);
  if (lane == 0 && a.ml) a.ml[(long long)t * a.n_q + hq] = make_float2(m, inv);
}

template <typename T, int HD>
__global__ void __launch_bounds__(128) attend_mass_simple_kernel(const __grid_constant__ AttendArgs a) {
  const int b = blockIdx.x / a.n_kv, g = blockIdx.x - b * a.n_kv, G = a.n_q / a.n_kv;
  const long long reach = (long long)a.max_blocks * a.block;
  const int c = a.ctx[b];
  if (c > reach) return;
  const int first = a.cu ? a.cu[b] : b, n = a.cu ? a.cu[b + 1] - first : 1;
  if (n > a.max_new || first < 0 || first + n > a.T) return;
  for (int j = blockIdx.y * 128 + threadIdx.x; j < c; j += gridDim.y * 128) {
    const long long page = a.block_table[(long long)b * a.max_blocks + j / a.block];
    float sum = 0.f;
    for (int i = 0; i < n; ++i) {
      const int self = c - n + i;
      if (j > self || (a.window && j <= self - a.window)) continue;
      for (int h = 0; h < G; ++h) {
        const int hq = g * G + h;
        float s = 0.f;
        if (page >= 0 && page < a.pages) {
          const long long ak = (page * 2) * a.n_kv + g;
          const uint8_t *pk = a.pool + (ak * a.block + j % a.block) * HD;
          const float fk = pow2f(a.exps[ak]);
          const T *q = (const T *)a.q + (first + i) * a.q_t + hq * a.q_h;
          for (int d = 0; d < HD; d += 2) {
            const float2 x = e4m3x2_to(*(const uint16_t *)(pk + d));
            s = fmaf(to_f32(q[d]) * a.scale, x.x * fk, s);
            s = fmaf(to_f32(q[d + 1]) * a.scale, x.y * fk, s);
          }
        }
        const float2 ml = a.ml[(long long)(first + i) * a.n_q + hq];
        sum += expf(s - ml.x) * ml.y;
      }
    }
    a.mass[(long long)blockIdx.x * reach + j] += sum;
  }
}

template <typename T, int HD>
cudaError_t launch_attend(const AttendArgs &a, cudaStream_t st) {
  cudaError_t ce = launch_k(attend_simple_kernel<T, HD>, dim3(a.T, (a.n_q + 3) / 4), dim3(128), 0, st, false, a);
  if (ce == cudaSuccess && a.mass) ce = launch_k(attend_mass_simple_kernel<T, HD>, dim3(a.B * a.n_kv, 32), dim3(128), 0, st, false, a);
  return ce;
}

}  // namespace
}  // namespace corun

using namespace corun;

extern "C" {

int64_t corun_kv8_attend_bytes(int32_t B, int32_t T, int32_t max_new, int32_t n_q, int32_t n_kv, int32_t head_dim, int32_t block,
                               int32_t max_blocks, int32_t with_mass) {
  if (B < 1 || T < 1 || max_new < 1 || n_q < 1 || n_kv < 1 || head_dim < 1 || block < 1 || max_blocks < 1) return 0;
  return 1024 + (int64_t)T * n_q * 8;
}

int corun_kv8_attend(const corun_kv8_cache *cache, const corun_kv8_rows *rows, int32_t max_new, const corun_heads *q,
                     const corun_heads *out, int32_t dtype, int32_t n_q, float scale, int32_t window, float *mass, void *ws,
                     int64_t ws_bytes, void *cuda_stream) {
  if (!kv8_cache_ok(cache) || !kv8_rows_ok(rows, cache) || !q || !out || !q->p || !out->p || (dtype != CORUN_BF16 && dtype != CORUN_F16) ||
      rows->B > AT_MAXB || max_new < 1 || (!rows->cu && max_new != 1) || n_q < 1 || n_q % cache->n_kv || n_q / cache->n_kv > 32 || !(scale > 0.f) || isinf(scale) ||
      window < 0 || (mass && (int64_t)max_new * (n_q / cache->n_kv) > 32) || !heads_on_16(*q, dtype) || !heads_on_16(*out, dtype) || !ws ||
      !aligned_to(ws, 256))
    return CORUN_EINVAL;
  if (rows->T == 0) return CORUN_OK;
  if (ws_bytes < corun_kv8_attend_bytes(rows->B, rows->T, max_new, n_q, cache->n_kv, cache->head_dim, cache->block, rows->max_blocks, mass != nullptr))
    return CORUN_EINVAL;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const AttendArgs a{(const uint8_t *)cache->pool, cache->exps, cache->pages, cache->block, cache->n_kv, n_q, rows->B, rows->T, rows->max_blocks, max_new,
                     window, rows->block_table, rows->ctx, rows->cu, q->p, out->p, q->token_stride, q->head_stride, out->token_stride,
                     out->head_stride, scale, mass, (float2 *)((char *)ws + 1024)};
  cudaError_t ce = cudaMemsetAsync(ws, 0, 1024, st);
  if (ce == cudaSuccess) {
    if (dtype == CORUN_BF16) ce = cache->head_dim == 128 ? launch_attend<__nv_bfloat16, 128>(a, st) : launch_attend<__nv_bfloat16, 64>(a, st);
    else ce = cache->head_dim == 128 ? launch_attend<__half, 128>(a, st) : launch_attend<__half, 64>(a, st);
  }
  if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  return CORUN_OK;
}

int corun_kv8_sync(const void *ws, void *cuda_stream) {
  if (!ws) return CORUN_EINVAL;
  int hs[256] = {0};
  cudaError_t ce = cudaMemcpyAsync(hs, ws, sizeof(hs), cudaMemcpyDeviceToHost, (cudaStream_t)cuda_stream);
  if (ce == cudaSuccess) ce = cudaStreamSynchronize((cudaStream_t)cuda_stream);
  if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  for (int i = 0; i < 256; ++i)
    if (hs[i]) return CORUN_ETIMEOUT;
  return CORUN_OK;
}

}  // extern "C"
