// Products of 8-bit rows with 8-bit weights:
//   out[m, n] = a_scale[m] * w_scale[n] * sum_k a[m, k] * w[n, k]
// The sums are int32 and exact (K < 2^17), whatever the order; the two scales
// are multiplied onto the sum in float32 and the result is rounded once.
#include "internal.h"

namespace ssm {

// Where a result goes.
struct I8Out {
  void* p;
  int dtype;                 // 0 float32, 1 bfloat16, 2 float16
  const float *sa, *sw;
  int N;
  __device__ __forceinline__ void store(int m, int n, int acc) const {
    const float v = (float)acc * (sa[m] * sw[n]);
    const size_t i = (size_t)m * N + n;
    if (dtype == 0) ((float*)p)[i] = v;
    else if (dtype == 1) ((bf16_t*)p)[i] = f2bf(v);
    else ((f16_t*)p)[i] = (f16_t)v;
  }
};

// Any size and alignment: 64 x 64 tiles, 64 columns of K at a time through LDS
// byte by byte, four products an instruction.
__global__ void __launch_bounds__(256) gemm_i8_any_kernel(const int8_t* __restrict__ A,
                                                          const int8_t* __restrict__ W, int M, int N,
                                                          int K, I8Out out) {
  __shared__ int As[64][17], Ws[64][17];
  const int tid = threadIdx.x, tm = tid >> 4, tn = tid & 15;
  const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  int acc[4][4] = {};
  for (int k0 = 0; k0 < K; k0 += 64) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = (tid >> 6) + 4 * i, c = tid & 63, k = k0 + c;
      const int8_t a = (m0 + r < M && k < K) ? A[(size_t)(m0 + r) * K + k] : (int8_t)0;
      const int8_t w = (n0 + r < N && k < K) ? W[(size_t)(n0 + r) * K + k] : (int8_t)0;
      ((int8_t*)As[r])[c] = a;
      ((int8_t*)Ws[r])[c] = w;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      int a[4], w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) { a[i] = As[tm + 16 * i][c]; w[i] = Ws[tn + 16 * i][c]; }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_sdot4(a[i], w[j], acc[i][j], false);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + tm + 16 * i, n = n0 + tn + 16 * j;
      if (m < M && n < N) out.store(m, n, acc[i][j]);
    }
}

size_t gemm_i8_ws_bytes(int M, int N, int K) {
  (void)M; (void)N; (void)K;
  return 0;
}

hipError_t gemm_i8(int M, int N, int K, const int8_t* a, const float* sa, const int8_t* w,
                   const float* sw, int out_dtype, void* out, void* ws, hipStream_t st) {
  (void)ws;
  if (M == 0) return hipSuccess;
  launch(gemm_i8_any_kernel, dim3(ceil_div(N, 64), ceil_div(M, 64)), dim3(256), 0, st, a, w, M, N, K,
         I8Out{out, out_dtype, sa, sw, N});
  return hipGetLastError();
}

}  // namespace ssm
