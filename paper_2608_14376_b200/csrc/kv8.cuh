// What the kernels of the 8-bit key / value cache and of the rotary positions share: typed loads, e4m3 conversions,
// power-of-two scales, the table of rotary frequencies and the argument checks of the C ABI.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/corun_kv8.h"
#include "gemm.cuh"
#include "launch.cuh"
#include "ptx.cuh"

namespace corun {

constexpr int ROPE_MAX_PAIRS = 128;
// A rotation by value, as kernels take it: half turns per position of every pair, and the magnitude.
struct RopeTable {
  double half_turns[ROPE_MAX_PAIRS];
  float magnitude;
  int rot, interleaved;   // rot 0 = nothing is rotated
};

}  // namespace corun

struct corun_rope { corun::RopeTable t; };

namespace corun {

constexpr int KV8_E_MIN = -32, KV8_E_MAX = 31;

// The current device and its SM count (asked of the driver once per device).
cudaError_t device_sms(int *dev, int *sms);
inline bool aligned_to(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline int dtype_size(int dtype) { return dtype == CORUN_F32 ? 4 : 2; }
// Every head of the view starts on 16 bytes.
inline bool heads_on_16(const corun_heads &v, int dtype) {
  const int64_t per = 16 / dtype_size(dtype);
  return aligned_to(v.p, 16) && v.token_stride % per == 0 && v.head_stride % per == 0;
}
inline bool kv8_cache_ok(const corun_kv8_cache *c) {
  return c && c->pool && c->exps && c->pages >= 1 && (c->block == 16 || c->block == 32 || c->block == 64) && c->n_kv >= 1 &&
         c->n_kv <= 4096 && (c->head_dim == 64 || c->head_dim == 128) && c->pages < (1ll << 31) &&
         c->pages * 2 * c->n_kv * c->block < (1ll << 31) && aligned_to(c->pool, 16);
}
inline bool kv8_rows_ok(const corun_kv8_rows *r, const corun_kv8_cache *c) {
  return r && r->block_table && r->ctx && r->max_blocks >= 1 && (int64_t)r->max_blocks * c->block < (1ll << 30) && r->B >= 1 &&
         r->B <= 65535 && r->T >= 0 && (r->cu || r->T == r->B);
}

#ifdef __CUDACC__
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }

// 2^e for |e| <= 126, exact.
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }
// The smallest e in range with amax <= 448 * 2^e = 1.75 * 2^(8 + e).
__device__ __forceinline__ int kv8_exp_of(float amax) {
  const int b = __float_as_int(amax) & 0x7fffffff;
  const int e = (b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0);
  return e < KV8_E_MIN ? KV8_E_MIN : (e > KV8_E_MAX ? KV8_E_MAX : e);
}
__device__ __forceinline__ uint32_t e4m3x2_of(float lo, float hi) {   // rounds to nearest even, cuts at 448
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 e4m3x2_to(uint32_t v) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)v, __NV_E4M3);
  return __half22float2(__half2(h));
}
// Four stored values times 2^d (d <= 0 when a block's scale grows).
__device__ __forceinline__ uint32_t e4m3x4_shift(uint32_t v, float f) {
  const float2 a = e4m3x2_to(v & 0xffffu), b = e4m3x2_to(v >> 16);
  return e4m3x2_of(a.x * f, a.y * f) | (e4m3x2_of(b.x * f, b.y * f) << 16);
}

// cos and sin of a pair at a position, times the magnitude.  The angle is formed and reduced in 64 bits, in half turns, so that the
// reduction is exact; cos and sin of its first 24 bits come from 32-bit functions, and the rest r (at most 2^-25) adds its first-order
// term: within 1.5 * 2^-24 as 64 bits throughout are within 2^-25, in a fifth of the instructions (the times are the same).
__device__ __forceinline__ float2 rope_cs(const RopeTable &tab, int pair, int pos) {
  const double t = (double)pos * tab.half_turns[pair], u = t - 2.0 * rint(0.5 * t);
  const float hi = (float)u, r = (float)(u - (double)hi) * 3.14159265f;
  float s, c;
  sincospif(hi, &s, &c);
  return make_float2(fmaf(-s, r, c) * tab.magnitude, fmaf(c, r, s) * tab.magnitude);
}

// x1 c - x2 s and x2 c + x1 s, rounded the same way in every kernel.
__device__ __forceinline__ float turn1(float x1, float x2, float2 cs) { return fmaf(x1, cs.x, -__fmul_rn(x2, cs.y)); }
__device__ __forceinline__ float turn2(float x1, float x2, float2 cs) { return fmaf(x2, cs.x, __fmul_rn(x1, cs.y)); }

// A head cut into pieces of two groups of VEC values (16 bytes each): piece p of the rotated part holds VEC pairs, p VEC .. p VEC + VEC - 1; the
// pieces behind it are the values that are not rotated.  Needs rot / 2 and head_dim / 2 to be multiples of VEC.
template <typename T> struct Piece {
  static constexpr int VEC = 16 / (int)sizeof(T);
  alignas(16) T a[VEC], b[VEC];
};
struct PieceAt { int a, b; bool turned; };
template <int VEC>
__device__ __forceinline__ PieceAt piece_at(const RopeTable &tab, int p) {
  const int half = tab.rot >> 1, n = half / VEC;
  if (p >= n) { const int d = tab.rot + (p - n) * 2 * VEC; return {d, d + VEC, false}; }
  if (tab.interleaved) return {2 * p * VEC, 2 * p * VEC + VEC, true};
  return {p * VEC, half + p * VEC, true};
}
template <typename T>
__device__ __forceinline__ void piece_load(Piece<T> &v, const T *x, const PieceAt &at) {
  *reinterpret_cast<uint4 *>(v.a) = *reinterpret_cast<const uint4 *>(x + at.a);
  *reinterpret_cast<uint4 *>(v.b) = *reinterpret_cast<const uint4 *>(x + at.b);
}
// The piece's values in 32 bits, rotated where it belongs to the rotated part: cs[i] is pair p VEC + i's cos and sin.
template <typename T, int VEC>
__device__ __forceinline__ void piece_turn(const Piece<T> &v, const float2 (&cs)[VEC], bool turned, bool interleaved, float (&a)[VEC], float (&b)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) { a[i] = to_f32(v.a[i]); b[i] = to_f32(v.b[i]); }
  if (!turned) return;
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
      const float a1 = a[2 * i], a2 = a[2 * i + 1], b1 = b[2 * i], b2 = b[2 * i + 1];
      const float2 f = cs[i], g = cs[VEC / 2 + i];
      a[2 * i] = turn1(a1, a2, f);
      a[2 * i + 1] = turn2(a1, a2, f);
      b[2 * i] = turn1(b1, b2, g);
      b[2 * i + 1] = turn2(b1, b2, g);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float x1 = a[i], x2 = b[i];
      a[i] = turn1(x1, x2, cs[i]);
      b[i] = turn2(x1, x2, cs[i]);
    }
  }
}
#endif

}  // namespace corun
