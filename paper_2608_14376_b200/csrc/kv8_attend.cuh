// What the two attention kernels over the 8-bit cache share: the call's arguments and a row's plan.
// kv8_attend.cu takes the rows with at most AT_MAXC query columns (new tokens x query heads of a key head), kv8_chunk.cu the others; which
// kernel takes a row depends on that row alone.
#pragma once
#include "kv8.cuh"

namespace corun {

constexpr int AT_T = 128;           // cached tokens per tile
constexpr int AT_MAXC = 32;         // columns of a row that is split over its cached tokens
constexpr int AT_MAXB = 512;        // rows per call: a thread plans one
constexpr int AT_STATUS = 256;      // status words at the start of the workspace
constexpr float AT_LOW = -3.4028235e38f;   // a maximum over nothing: no finite score is below it

struct AttendArgs {
  const int8_t *exps;
  long long pages;
  int block, n_kv, n_q, B, T, max_blocks, max_new, window, cols, max_splits, sms;   // cols: columns per (row, key head) in the workspace
  bool by_token;      // partial results: the row's place goes by its first token, not by its number
  const int *block_table, *ctx, *cu;
  const void *q;
  void *out;
  long long q_t, q_h, o_t, o_h;
  float scale_log2e;
  float *mass;
  int *status;
  float2 *part_ml;    // a row's [n_kv][max_splits][columns] (part_at): frame, sum
  float *part_o;      // the same, hd values each
  float2 *ml;         // [B][n_kv][cols]: frame, 1 / sum (with mass)
  float *scores;      // [B][n_kv][tokens padded to tiles][cols] (with mass)
  long long score_tokens;
};

#ifdef __CUDACC__
// Whether a row of the call takes part.
__device__ __forceinline__ bool at_row_ok(int c, int first, int end, const AttendArgs &a) {
  const int n = end - first;
  return c > 0 && (long long)c <= (long long)a.max_blocks * a.block && first >= 0 && end > first && n <= a.max_new && end <= a.T;
}
// Where the partial results of a row's split begin, and how many columns lie between two splits.  A row's columns are its tokens' times
// G, so a call's rows together need no more than T * G, which is less than B times the largest row's where few rows bring many tokens.
__device__ __forceinline__ long long part_at(const AttendArgs &a, int b, int first, int n, int g, int split, int G, int &cols) {
  cols = a.by_token ? n * G : a.cols;
  return (long long)(a.by_token ? first * G : b * a.cols) * (a.n_kv * a.max_splits) + (long long)(g * a.max_splits + split) * cols;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
// Whether a barrier's phase is over, without waiting (try_wait may hold the thread for a while).
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.b32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Loads that are issued where they stand (the compiler may move an ordinary one down to its first use), from L2: this kernel may have come up
// beside the one that wrote the values, whose SM-local lines a cached load could still meet.
__device__ __forceinline__ int load_now(const int *p) {
  int v;
  asm volatile("ld.global.cg.b32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ int load_now(const int8_t *p) {
  int v;
  asm volatile("ld.global.cg.s8 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
#endif

// Tiles that the new tokens of a call's rows with more than AT_MAXC columns can make at most: a row's n tokens are n / TQ + 1 or fewer, and
// rows with AT_MAXC columns or fewer have none.
inline long long kv8_chunk_tiles(int T, int B, int G) {
  const int least = AT_MAXC / G + 1;
  const long long rows = T / least < B ? T / least : B;
  return T / (128 / G) + rows;
}
// Rows with more than AT_MAXC columns.  tm: tensor map whose boxes hold one page of one head and kind.  dtype: CORUN_BF16 or CORUN_F16.
cudaError_t launch_kv8_chunk(const CUtensorMap &tm, const AttendArgs &a, int head_dim, int dtype, int dev, cudaStream_t st);

}  // namespace corun
