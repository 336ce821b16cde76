// Rows to 8-bit codes with one float32 scale each: RMSNorm with the residual's
// addition, plain rows, and SwiGLU of [gate | up] rows.
//
// A row y gets scale s = max|y| / 127 and codes q = round(y / s), ties to even,
// so that q * s is within s / 2 of y.  A row whose largest magnitude is below
// I8_TINY (rows of zeros among them) gets scale 0 and codes 0: 127 / max|y|
// would leave the float32 range there.  A row with an infinity or a NaN gets
// scale NaN and codes 0, so that whatever is computed from it is NaN.
#include "internal.h"

namespace ssm {

constexpr float I8_TINY = 0x1p-100f;

// Sum, and largest |value| as bits (NaN above infinity above the finite), over
// a workgroup of 256 threads; `red` has 4 entries.
__device__ __forceinline__ float block_sum256(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}
__device__ __forceinline__ uint32_t block_max256(uint32_t v, uint32_t* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return max(max(red[0], red[1]), max(red[2], red[3]));
}
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Factor from values to codes and the row's scale, from its largest magnitude.
struct Codes {
  float inv, scale;
};
__device__ __forceinline__ Codes codes_of(uint32_t amax_bits) {
  const float amax = __uint_as_float(amax_bits);
  if (amax_bits >= 0x7f800000u) return {0.f, __uint_as_float(0x7fc00000u)};
  if (amax < I8_TINY) return {0.f, 0.f};
  return {127.f / amax, amax / 127.f};
}
// y is finite where inv is not 0; |y * inv| <= 127 (1 + 2^-23), which rounds to 127.
__device__ __forceinline__ int8_t code(float y, float inv) {
  return inv == 0.f ? (int8_t)0 : (int8_t)__float2int_rn(y * inv);
}

template <typename T> struct RowValue {           // plain rows
  const T* x;
  __device__ __forceinline__ float operator()(int c) const { return ldf(x + c); }
};
__device__ __forceinline__ float swiglu(float g, float u) { return g / (1.f + expf(-g)) * u; }
template <typename T> struct SwigluValue {        // gate in [0, d), up in [d, 2 d)
  const T* x;
  int d;
  __device__ __forceinline__ float operator()(int c) const { return swiglu(ldf(x + c), ldf(x + d + c)); }
};

// One workgroup per row, any width and alignment: the row is read twice.
template <typename T, bool SWIGLU>
__global__ void __launch_bounds__(256) quant_i8_kernel(const T* __restrict__ x, int d,
                                                       int8_t* __restrict__ q,
                                                       float* __restrict__ scale) {
  __shared__ uint32_t red[4];
  const size_t row = blockIdx.x;
  auto value = [&] {
    if constexpr (SWIGLU) return SwigluValue<T>{x + row * 2 * d, d};
    else return RowValue<T>{x + row * d};
  }();
  uint32_t a = 0;
  for (int c = threadIdx.x; c < d; c += 256) a = max(a, abs_bits(value(c)));
  const Codes k = codes_of(block_max256(a, red));
  for (int c = threadIdx.x; c < d; c += 256) q[row * d + c] = code(value(c), k.inv);
  if (threadIdx.x == 0) scale[row] = k.scale;
}

// One workgroup per row, any width and alignment.  resid may be x itself: the
// last pass reads each element before it writes it.
template <typename TD, typename TG>
__global__ void __launch_bounds__(256) norm_i8_kernel(const float* x, const TD* delta,
                                                      const TG* __restrict__ g, int d, float eps,
                                                      float* resid, int8_t* __restrict__ q,
                                                      float* __restrict__ scale) {
  __shared__ float red[4];
  __shared__ uint32_t redu[4];
  const size_t at = (size_t)blockIdx.x * d;
  auto sum = [&](int c) { return delta ? x[at + c] + ldf(delta + at + c) : x[at + c]; };
  float ss = 0.f;
  for (int c = threadIdx.x; c < d; c += 256) { const float r = sum(c); ss += r * r; }
  ss = block_sum256(ss, red);
  const float inv = 1.0f / sqrtf(ss / (float)d + eps);
  uint32_t a = 0;
  for (int c = threadIdx.x; c < d; c += 256) a = max(a, abs_bits(sum(c) * inv * ldf(g + c)));
  const Codes k = codes_of(block_max256(a, redu));
  for (int c = threadIdx.x; c < d; c += 256) {
    const float r = sum(c);
    q[at + c] = code(r * inv * ldf(g + c), k.inv);
    if (resid) resid[at + c] = r;
  }
  if (threadIdx.x == 0) scale[blockIdx.x] = k.scale;
}

template <typename T>
static hipError_t quant_t(int rows, int d, bool sw, const T* x, int8_t* q, float* scale, hipStream_t st) {
  if (sw) launch(quant_i8_kernel<T, true>, dim3(rows), dim3(256), 0, st, x, d, q, scale);
  else launch(quant_i8_kernel<T, false>, dim3(rows), dim3(256), 0, st, x, d, q, scale);
  return hipGetLastError();
}

hipError_t launch_quant_i8(int dtype, int rows, int d, bool swiglu, const void* x, int8_t* q,
                           float* scale, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  if (dtype == 0) return quant_t(rows, d, swiglu, (const float*)x, q, scale, st);
  if (dtype == 1) return quant_t(rows, d, swiglu, (const bf16_t*)x, q, scale, st);
  return quant_t(rows, d, swiglu, (const f16_t*)x, q, scale, st);
}

template <typename TD, typename TG>
static hipError_t norm_t(int rows, int d, const float* x, const TD* delta, const TG* g, float eps,
                         float* resid, int8_t* q, float* scale, hipStream_t st) {
  launch(norm_i8_kernel<TD, TG>, dim3(rows), dim3(256), 0, st, x, delta, g, d, eps, resid, q, scale);
  return hipGetLastError();
}
template <typename TG>
static hipError_t norm_g(int delta_dtype, int rows, int d, const float* x, const void* delta,
                         const TG* g, float eps, float* resid, int8_t* q, float* scale, hipStream_t st) {
  if (delta_dtype == 1) return norm_t(rows, d, x, (const bf16_t*)delta, g, eps, resid, q, scale, st);
  if (delta_dtype == 2) return norm_t(rows, d, x, (const f16_t*)delta, g, eps, resid, q, scale, st);
  return norm_t(rows, d, x, (const float*)delta, g, eps, resid, q, scale, st);
}

hipError_t launch_norm_i8(int rows, int d, const float* x, const void* delta, int delta_dtype,
                          const void* g, int gain_dtype, float eps, float* resid, int8_t* q,
                          float* scale, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  if (gain_dtype == 0)
    return norm_g(delta_dtype, rows, d, x, delta, (const float*)g, eps, resid, q, scale, st);
  return norm_g(delta_dtype, rows, d, x, delta, (const bf16_t*)g, eps, resid, q, scale, st);
}

}  // namespace ssm
