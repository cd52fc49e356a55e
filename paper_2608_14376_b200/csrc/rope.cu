// Rotary positions of queries and keys (include/corun_rope.h): y = rotated x for [T][heads][head_dim].
//
// The products are 3 operations a value, so the op is bound by its bytes: each value read and written once.  What would
// cost more than that is the angle, some 40 instructions a pair: a CTA takes a few tokens, computes their cos and sin once into shared
// memory and uses them for all of its heads.  4096 tokens of 40 heads of 128 in bf16: 17.4 us (13.0 at the copy rate).
#include <math.h>

#include <atomic>
#include <new>

#include "kv8.cuh"

namespace corun {
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TOKENS = 4;

struct HeadsView { const void *x; void *y; long long xt, xh, yt, yh; };

// Sixteen bytes at a time: an item is VEC values of each half of VEC pairs (half layout) or VEC neighbouring values (interleaved, or not
// rotated); neighbouring threads take neighbouring items and heads.  Few registers and many warps are what this takes: a thread per (token,
// piece) that keeps its cos and sin in registers over several heads took 4096 tokens of 40 heads of 128 from 17.4 to 19.3 us, with five
// heads requested together 22.3.
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack { T v[VEC]; };

template <typename T, int VEC>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const __grid_constant__ RopeTable tab, HeadsView v, const int *__restrict__ positions,
                                                            long long n_tok, int heads, int head_dim, int heads_per_cta) {
  __shared__ float2 cs[ROPE_TOKENS * ROPE_MAX_PAIRS];
  const long long t0 = (long long)blockIdx.x * ROPE_TOKENS;
  const int nt = (int)min((long long)ROPE_TOKENS, n_tok - t0);
  const int pairs = tab.rot >> 1;
  for (int i = threadIdx.x; i < nt * pairs; i += ROPE_THREADS) {
    const int t = i / pairs, p = i - t * pairs;
    cs[t * ROPE_MAX_PAIRS + p] = rope_cs(tab, p, __ldg(positions + t0 + t));
  }
  __syncthreads();
  const int h0 = blockIdx.y * heads_per_cta, nh = min(heads_per_cta, heads - h0);
  // work of a head: half layout: pairs / VEC packs of two halves, then the rest; interleaved: head_dim / VEC packs
  const int n_pair = tab.interleaved ? tab.rot / VEC : pairs / VEC;
  const int per_head = n_pair + (v.x == v.y ? 0 : (head_dim - tab.rot) / VEC);
  const int total = nt * nh * per_head;
  typedef Pack<T, VEC> P;
  for (int i = threadIdx.x; i < total; i += ROPE_THREADS) {
    const int c = i % per_head, th = i / per_head, h = th % nh, t = th / nh;
    const T *x = (const T *)v.x + (t0 + t) * v.xt + (long long)(h0 + h) * v.xh;
    T *y = (T *)v.y + (t0 + t) * v.yt + (long long)(h0 + h) * v.yh;
    if (c >= n_pair) {
      const int d = tab.rot + (c - n_pair) * VEC;
      *reinterpret_cast<P *>(y + d) = *reinterpret_cast<const P *>(x + d);
    } else if (tab.interleaved) {
      const int d = c * VEC;
      P a = *reinterpret_cast<const P *>(x + d);
#pragma unroll
      for (int e = 0; e < VEC; e += 2) {
        const float2 f = cs[t * ROPE_MAX_PAIRS + ((d + e) >> 1)];
        const float x1 = to_f32(a.v[e]), x2 = to_f32(a.v[e + 1]);
        a.v[e] = from_f32<T>(turn1(x1, x2, f));
        a.v[e + 1] = from_f32<T>(turn2(x1, x2, f));
      }
      *reinterpret_cast<P *>(y + d) = a;
    } else {
      const int d = c * VEC;
      P a = *reinterpret_cast<const P *>(x + d), b = *reinterpret_cast<const P *>(x + pairs + d);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float2 f = cs[t * ROPE_MAX_PAIRS + d + e];
        const float x1 = to_f32(a.v[e]), x2 = to_f32(b.v[e]);
        a.v[e] = from_f32<T>(turn1(x1, x2, f));
        b.v[e] = from_f32<T>(turn2(x1, x2, f));
      }
      *reinterpret_cast<P *>(y + d) = a;
      *reinterpret_cast<P *>(y + pairs + d) = b;
    }
  }
}

// Value by value, where 16 bytes at a time do not fit the layout: one thread per pair or value beyond the rotated part.
template <typename T>
__global__ void __launch_bounds__(ROPE_THREADS) rope_scalar_kernel(const __grid_constant__ RopeTable tab, HeadsView v, const int *__restrict__ positions,
                                                                   long long n_tok, int heads, int head_dim, int heads_per_cta) {
  __shared__ float2 cs[ROPE_TOKENS * ROPE_MAX_PAIRS];
  const long long t0 = (long long)blockIdx.x * ROPE_TOKENS;
  const int nt = (int)min((long long)ROPE_TOKENS, n_tok - t0);
  const int pairs = tab.rot >> 1;
  for (int i = threadIdx.x; i < nt * pairs; i += ROPE_THREADS) {
    const int t = i / pairs, p = i - t * pairs;
    cs[t * ROPE_MAX_PAIRS + p] = rope_cs(tab, p, __ldg(positions + t0 + t));
  }
  __syncthreads();
  const int h0 = blockIdx.y * heads_per_cta, nh = min(heads_per_cta, heads - h0);
  const int per_head = pairs + (v.x == v.y ? 0 : head_dim - tab.rot);
  const int total = nt * nh * per_head;
  for (int i = threadIdx.x; i < total; i += ROPE_THREADS) {
    const int c = i % per_head, th = i / per_head, h = th % nh, t = th / nh;
    const T *x = (const T *)v.x + (t0 + t) * v.xt + (long long)(h0 + h) * v.xh;
    T *y = (T *)v.y + (t0 + t) * v.yt + (long long)(h0 + h) * v.yh;
    if (c >= pairs) {
      y[tab.rot + c - pairs] = x[tab.rot + c - pairs];
    } else {
      const int d1 = tab.interleaved ? 2 * c : c, d2 = tab.interleaved ? 2 * c + 1 : c + pairs;
      const float2 f = cs[t * ROPE_MAX_PAIRS + c];
      const float x1 = to_f32(x[d1]), x2 = to_f32(x[d2]);
      y[d1] = from_f32<T>(turn1(x1, x2, f));
      y[d2] = from_f32<T>(turn2(x1, x2, f));
    }
  }
}

template <typename T>
cudaError_t launch_rope(const RopeTable &tab, const HeadsView &v, bool wide, const int *positions, long long T_, int heads, int head_dim,
                        int sms, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  const long long gx = (T_ + ROPE_TOKENS - 1) / ROPE_TOKENS;
  // few tokens: the heads are shared out among CTAs (each computes its tokens' angles again)
  long long gy = gx >= 2 * sms ? 1 : (2 * sms + gx - 1) / gx;
  if (gy > heads) gy = heads;
  const int per = (int)((heads + gy - 1) / gy);
  gy = (heads + per - 1) / per;
  const dim3 grid((unsigned)gx, (unsigned)gy);
  if (wide) return launch_k(rope_kernel<T, VEC>, grid, dim3(ROPE_THREADS), 0, st, false, tab, v, positions, T_, heads, head_dim, per);
  return launch_k(rope_scalar_kernel<T>, grid, dim3(ROPE_THREADS), 0, st, false, tab, v, positions, T_, heads, head_dim, per);
}

}  // namespace

cudaError_t device_sms(int *dev, int *sms) {
  static std::atomic<int> known[64];
  cudaError_t ce = cudaGetDevice(dev);
  if (ce != cudaSuccess) return ce;
  if (*dev < 64 && (*sms = known[*dev].load(std::memory_order_relaxed)) > 0) return ce;
  ce = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev);
  if (ce == cudaSuccess && *dev < 64) known[*dev].store(*sms, std::memory_order_relaxed);
  return ce;
}

}  // namespace corun

using namespace corun;

extern "C" {

int corun_rope_create(const corun_rope_config *c, corun_rope **out) {
  if (!c || !out) return CORUN_EINVAL;
  *out = nullptr;
  const bool stretched = c->scaling == CORUN_ROPE_PARTS || c->scaling == CORUN_ROPE_BANDS;
  if (c->rot_dim < 2 || c->rot_dim > 2 * ROPE_MAX_PAIRS || c->rot_dim % 2 || c->scaling < CORUN_ROPE_PLAIN || c->scaling > CORUN_ROPE_BANDS ||
      !(c->theta > 0.0) || !isfinite(c->theta) || !(c->magnitude >= 0.0) || !isfinite(c->magnitude))
    return CORUN_EINVAL;
  if (c->scaling != CORUN_ROPE_PLAIN && (!(c->factor >= 1.0) || !isfinite(c->factor))) return CORUN_EINVAL;
  if (c->scaling == CORUN_ROPE_BASE && c->rot_dim < 4) return CORUN_EINVAL;
  if (stretched && (c->original_context < 1 || !(c->low > 0.0) || !(c->high > c->low) || !isfinite(c->high))) return CORUN_EINVAL;
  if (c->scaling == CORUN_ROPE_PARTS && !(c->theta > 1.0)) return CORUN_EINVAL;
  corun_rope *r = new (std::nothrow) corun_rope();
  if (!r) return CORUN_ENOMEM;
  const double pi = 3.14159265358979323846;
  const int n = c->rot_dim;
  const double base = c->scaling == CORUN_ROPE_BASE ? c->theta * pow(c->factor, n / (n - 2.0)) : c->theta;
  double m = 1.0, first = 0.0, last = 0.0;
  if (c->scaling == CORUN_ROPE_PARTS) {
    auto where = [&](double turns) { return n * log(c->original_context / (turns * 2.0 * pi)) / (2.0 * log(c->theta)); };
    first = fmax(floor(where(c->high)), 0.0);
    last = fmin(ceil(where(c->low)), n - 1.0);
    m = 0.1 * log(c->factor) + 1.0;
  }
  for (int i = 0; i < n / 2; ++i) {
    double f = pow(base, -2.0 * i / n);
    if (c->scaling == CORUN_ROPE_LINEAR) f /= c->factor;
    if (c->scaling == CORUN_ROPE_PARTS) {
      const double s = fmin(fmax((i - first) / fmax(last - first, 1e-3), 0.0), 1.0);
      f = f / c->factor * s + f * (1.0 - s);
    }
    if (c->scaling == CORUN_ROPE_BANDS) {
      const double s = fmin(fmax((c->original_context * f / (2.0 * pi) - c->low) / (c->high - c->low), 0.0), 1.0);
      f = f / c->factor * (1.0 - s) + f * s;
    }
    r->t.half_turns[i] = f / pi;
  }
  r->t.magnitude = (float)(c->magnitude > 0.0 ? c->magnitude : m);
  r->t.rot = n;
  r->t.interleaved = c->interleaved ? 1 : 0;
  *out = r;
  return CORUN_OK;
}

void corun_rope_destroy(corun_rope *r) { delete r; }

int corun_rope_apply(const corun_rope *r, const corun_heads *x, const corun_heads *y, int32_t dtype, const int32_t *positions, int64_t T,
                     int32_t heads, int32_t head_dim, void *cuda_stream) {
  if (!r || !x || !y || !x->p || !y->p || !positions || dtype < CORUN_F32 || dtype > CORUN_F16 || T < 0 || T > (1ll << 31) || heads < 1 ||
      heads > 65535 || head_dim < r->t.rot || head_dim > 1024)
    return CORUN_EINVAL;
  const uintptr_t sz = (uintptr_t)dtype_size(dtype);
  if (!aligned_to(x->p, sz) || !aligned_to(y->p, sz) || !aligned_to(positions, 4)) return CORUN_EINVAL;
  if (x->p == y->p && (x->token_stride != y->token_stride || x->head_stride != y->head_stride)) return CORUN_EINVAL;
  if (T == 0) return CORUN_OK;
  int dev = 0, sms = 0;
  cudaError_t ce = device_sms(&dev, &sms);
  if (ce != cudaSuccess || sms < 1) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  const int vec = 16 / (int)sz;
  const bool wide = heads_on_16(*x, dtype) && heads_on_16(*y, dtype) && head_dim % vec == 0 && r->t.rot % (r->t.interleaved ? vec : 2 * vec) == 0;
  const HeadsView v{x->p, y->p, x->token_stride, x->head_stride, y->token_stride, y->head_stride};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (dtype == CORUN_F32) ce = launch_rope<float>(r->t, v, wide, positions, T, heads, head_dim, sms, st);
  else if (dtype == CORUN_BF16) ce = launch_rope<__nv_bfloat16>(r->t, v, wide, positions, T, heads, head_dim, sms, st);
  else ce = launch_rope<__half>(r->t, v, wide, positions, T, heads, head_dim, sms, st);
  if (ce != cudaSuccess) { g_last_cuda_error = (int)ce; return CORUN_ECUDA; }
  return CORUN_OK;
}

}  // extern "C"
