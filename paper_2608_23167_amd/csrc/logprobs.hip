// Log probabilities of given tokens, entropy and the most probable tokens of
// rows of logits, in one pass over the logits.
//
// With m = max x, z = sum exp(x - m) and t = sum (x - m) exp(x - m):
//   log p(v) = (x_v - m) - ln z,   entropy = ln z - t / z.
// (m, z, t) of two parts join by moving both to the larger maximum M: for
// delta = m - M, z -> z e^delta and t -> e^delta (t + z delta).
// Logits of -inf (and the [MASK] id, which counts as one) add nothing; a row
// with a NaN or a +inf has NaN log probabilities and entropy.
#include "internal.h"
#include "row_stats.h"

namespace ssm {

struct Soft {
  float m, z, t;
};
__device__ __forceinline__ Soft soft_empty() { return {-INFINITY, 0.f, 0.f}; }
// Differences to a maximum, no lower than SOFT_LOW: its exponential is 0 in
// float32, and products with a finite number stay finite (0 * -inf is NaN).
// NaN stays NaN.
constexpr float SOFT_LOW = -200.f;
__device__ __forceinline__ float soft_diff(float x, float m) {
  const float y = x - m;
  return y < SOFT_LOW ? SOFT_LOW : y;
}
__device__ __forceinline__ void soft_move(Soft& a, float m) {     // to the maximum m >= a.m
  const float dl = soft_diff(a.m, m), e = expf(dl);
  a.t = e * (a.t + a.z * dl);
  a.z *= e;
  a.m = m;
}
__device__ __forceinline__ void soft_add(Soft& a, float x) {
  if (x == -INFINITY) return;
  if (x > a.m) soft_move(a, x);
  const float y = soft_diff(x, a.m), e = expf(y);
  a.z += e;
  a.t += e * y;
}
__device__ __forceinline__ Soft soft_join(Soft a, Soft b) {
  if (b.z == 0.f) return a;
  if (a.z == 0.f) return b;
  const float M = fmaxf(a.m, b.m);
  if (M > a.m) soft_move(a, M);
  if (M > b.m) soft_move(b, M);
  return {M, a.z + b.z, a.t + b.t};
}
__device__ __forceinline__ Soft soft_wave(Soft a) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const Soft b{__shfl_xor(a.m, o, 64), __shfl_xor(a.z, o, 64), __shfl_xor(a.t, o, 64)};
    a = (threadIdx.x & o) ? soft_join(b, a) : soft_join(a, b);   // the same order in every lane
  }
  return a;
}

// One workgroup of 256 threads per row.
template <typename T>
__global__ void __launch_bounds__(256) logprobs_kernel(const T* __restrict__ logits, int V,
                                                       int mask_id, int n_targets,
                                                       const int32_t* __restrict__ targets, int k,
                                                       float* __restrict__ lp,
                                                       float* __restrict__ entropy,
                                                       int32_t* __restrict__ top_ids,
                                                       float* __restrict__ top_lp) {
  __shared__ Soft part[4];
  __shared__ float bv[4];
  __shared__ int bi[4];
  const size_t row = blockIdx.x;
  const int tid = threadIdx.x, wave = tid >> 6;
  const T* L = logits + row * V;
  float lv[STAT_K];
  int li[STAT_K];
#pragma unroll
  for (int q = 0; q < STAT_K; ++q) { lv[q] = -INFINITY; li[q] = STAT_NONE; }
  Soft a = soft_empty();
  for (int v = tid; v < V; v += 256) {
    if (v == mask_id) continue;
    const float x = ldf(L + v);
    soft_add(a, x);
    if (x > lv[STAT_K - 1]) stat_insert(lv, li, x, v);
  }
  a = soft_wave(a);
  if ((tid & 63) == 0) part[wave] = a;
  __syncthreads();
  a = soft_join(soft_join(part[0], part[1]), soft_join(part[2], part[3]));
  const float lz = logf(a.z);
  if (tid == 0 && entropy) entropy[row] = lz - a.t / a.z;
  for (int i = tid; i < n_targets; i += 256) {
    const int id = targets[row * n_targets + i];
    float r = __uint_as_float(0x7fc00000u);
    if (id >= 0 && id < V) r = ((id == mask_id ? -INFINITY : ldf(L + id)) - a.m) - lz;
    lp[row * n_targets + i] = r;
  }
  for (int q = 0; q < k; ++q) {                     // the best of the threads' best, k times
    float v = lv[0];
    int i = li[0];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float ov = __shfl_xor(v, o, 64);
      const int oi = __shfl_xor(i, o, 64);
      if (stat_better(ov, oi, v, i)) { v = ov; i = oi; }
    }
    __syncthreads();
    if ((tid & 63) == 0) { bv[wave] = v; bi[wave] = i; }
    __syncthreads();
    for (int w = 0; w < 4; ++w)
      if (stat_better(bv[w], bi[w], v, i)) { v = bv[w]; i = bi[w]; }
    if (tid == 0) {
      top_ids[row * k + q] = i == STAT_NONE ? -1 : i;
      top_lp[row * k + q] = i == STAT_NONE ? -INFINITY : (v - a.m) - lz;
    }
    if (li[0] == i && i != STAT_NONE) {
#pragma unroll
      for (int u = 0; u + 1 < STAT_K; ++u) { lv[u] = lv[u + 1]; li[u] = li[u + 1]; }
      lv[STAT_K - 1] = -INFINITY;
      li[STAT_K - 1] = STAT_NONE;
    }
  }
}

size_t token_logprobs_ws_bytes(int rows, int V, int k) {
  (void)rows; (void)V; (void)k;
  return 0;
}

hipError_t launch_token_logprobs(int dtype, int rows, int V, const void* logits, int mask_id,
                                 int n_targets, const int32_t* targets, int k, float* lp,
                                 float* entropy, int32_t* top_ids, float* top_lp, void* ws,
                                 hipStream_t st) {
  (void)ws;
  if (rows == 0) return hipSuccess;
  auto go = [&](auto* x) {
    using T = std::remove_cv_t<std::remove_pointer_t<decltype(x)>>;
    launch(logprobs_kernel<T>, dim3(rows), dim3(256), 0, st, x, V, mask_id, n_targets, targets, k,
           lp, entropy, top_ids, top_lp);
    return hipGetLastError();
  };
  if (dtype == 0) return go((const float*)logits);
  if (dtype == 1) return go((const bf16_t*)logits);
  return go((const f16_t*)logits);
}

}  // namespace ssm
