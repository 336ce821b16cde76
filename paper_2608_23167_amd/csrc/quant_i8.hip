// Rows to 8-bit codes with one float32 scale each: RMSNorm with the residual's
// addition, plain rows, and SwiGLU of [gate | up] rows.
//
// A row y gets scale s = max|y| / 127 and codes q = round(y / s), ties to even,
// so that q * s is within s / 2 of y.  A row whose largest magnitude is below
// I8_TINY (rows of zeros among them) gets scale 0 and codes 0: 127 / max|y|
// would leave the float32 range there.  A row with an infinity or a NaN gets
// scale NaN and codes 0, so that whatever is computed from it is NaN.
#include "dcheck.h"
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

__device__ __forceinline__ float swiglu(float g, float u) { return g / (1.f + expf(-g)) * u; }

// ---- rows held in registers ---------------------------------------------------
// TPR threads to a row (64: four rows to a workgroup, each a wave of its own;
// 256 or 1024: the workgroup), NV pieces of V elements to a thread, piece
// number t + TPR i of the row.  Every element is read once, the row's sum and
// largest magnitude are reduced together, and the codes leave from registers.
// Bound by memory: the norm of 14208 x 4096 with a float32 residual 137 us (757 MB at
// 5.5 TB/s; read three times by one workgroup a row 290), 5081 x 3584 float32 rows
// 16.6 us (5.5 TB/s), 12288 x 4096 bfloat16 weights 28 us (5.4 TB/s); few rows by the
// launch and two trips to memory: SwiGLU of 240 x 12288 6.2 us, the norm of one row 3.6.
// SwiGLU of many 16-bit rows by the vector ALUs (an exponential and a division an element):
// 3840 x 12288 bfloat16 52 us (4.6 TB/s), the ALUs busy 92% of the clocks; float32 83 (5.1).
template <int V, typename T> __device__ __forceinline__ void load_v(const T* p, float (&v)[V]) {
  if constexpr (V == 1) {
    v[0] = ldf(p);
  } else if constexpr (std::is_same<T, float>::value) {
    const float4 f = *(const float4*)p;
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  } else {
    using U = std::conditional_t<V == 8, u32x4_t, uint2>;
    const U u = *(const U*)p;
    const T* e = (const T*)&u;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = ldf(e + i);
  }
}
template <int V> __device__ __forceinline__ void store_codes(int8_t* q, const float (&y)[V], float inv) {
  if constexpr (V == 1) {
    *q = code(y[0], inv);
  } else {
    uint32_t w[V / 4] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) w[i >> 2] |= (uint32_t)(uint8_t)code(y[i], inv) << (8 * (i & 3));
    if constexpr (V == 8) *(uint2*)q = uint2{w[0], w[1]};
    else *(uint32_t*)q = w[0];
  }
}

// 1 / sqrt(mean + eps) for a row's sum of squares; NaN, which makes the row's scale NaN,
// where that sum has overflowed: 1 / sqrt(inf) = 0 would make a row of zeros of it.
__device__ __forceinline__ float inverse_rms(float ss, int d, float eps) {
  const float ms = ss / (float)d + eps;
  return ms < INFINITY ? 1.0f / sqrtf(ms) : __uint_as_float(0x7fc00000u);
}

// Sum and largest bits over the TPR threads of a row.
template <int TPR>
__device__ __forceinline__ void row_reduce(float& s, uint32_t& a, float* red, uint32_t* redu) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    s += __shfl_xor(s, o, 64);
    a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
  }
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = s; redu[threadIdx.x >> 6] = a; }
    __syncthreads();
    s = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) { s += red[w]; a = max(a, redu[w]); }
  }
}

template <typename T, bool SWIGLU, int V, int NV, int TPR>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR)
quant_rows_kernel(const T* __restrict__ x, int rows, int d, int8_t* __restrict__ q,
                  float* __restrict__ scale) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  __shared__ float red[16];
  __shared__ uint32_t redu[16];
  SSM_DCHECK(d <= V * NV * TPR && d % V == 0);
  const int t = threadIdx.x % TPR;
  const size_t row = (size_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (row >= (size_t)rows) return;                  // whole waves, and only where a wave is a row
  const T* xr = x + row * d * (SWIGLU ? 2 : 1);
  float y[NV][V];
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + TPR * i) * V;
    if (c < d) {
      load_v<V>(xr + c, y[i]);
      if constexpr (SWIGLU) {
        float u[V];
        load_v<V>(xr + d + c, u);
#pragma unroll
        for (int e = 0; e < V; ++e) y[i][e] = swiglu(y[i][e], u[e]);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) a = max(a, abs_bits(y[i][e]));
    }
  }
  float none = 0.f;
  row_reduce<TPR>(none, a, red, redu);
  const Codes k = codes_of(a);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + TPR * i) * V;
    if (c < d) store_codes<V>(q + row * d + c, y[i], k.inv);
  }
  if (t == 0) scale[row] = k.scale;
}

// The largest |y| is the largest |r g| times 1 / rms, so one reduction serves
// both statistics.  resid may be x or delta: a thread reads its elements first.
template <typename TD, typename TG, int V, int NV, int TPR>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR)
norm_rows_kernel(const float* x, const TD* delta, const TG* __restrict__ g, int rows, int d, float eps,
                 float* resid, int8_t* __restrict__ q, float* __restrict__ scale) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  __shared__ float red[16];
  __shared__ uint32_t redu[16];
  SSM_DCHECK(d <= V * NV * TPR && d % V == 0);
  const int t = threadIdx.x % TPR;
  const size_t row = (size_t)blockIdx.x * RPB + threadIdx.x / TPR;
  if (row >= (size_t)rows) return;
  const size_t at = row * d;
  float r[NV][V], dv[NV][V], gv[NV][V];             // all loads first: one trip to memory
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + TPR * i) * V;
    if (c < d) {
      load_v<V>(x + at + c, r[i]);
      if (delta) load_v<V>(delta + at + c, dv[i]);
      load_v<V>(g + c, gv[i]);
    }
  }
  float ss = 0.f;
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + TPR * i) * V;
    if (c < d) {
      if (delta) {
#pragma unroll
        for (int e = 0; e < V; ++e) r[i][e] += dv[i][e];
      }
      if (resid) {
        if constexpr (V == 4) *(float4*)(resid + at + c) = make_float4(r[i][0], r[i][1], r[i][2], r[i][3]);
        else resid[at + c] = r[i][0];
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        ss += r[i][e] * r[i][e];
        r[i][e] *= gv[i][e];
        a = max(a, abs_bits(r[i][e]));
      }
    }
  }
  row_reduce<TPR>(ss, a, red, redu);
  const float inv = inverse_rms(ss, d, eps);
  const Codes k = codes_of(abs_bits(__uint_as_float(a) * inv));
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + TPR * i) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) r[i][e] *= inv;
    if (c < d) store_codes<V>(q + at + c, r[i], k.inv);
  }
  if (t == 0) scale[row] = k.scale;
}

// ---- rows of any width, read again in each pass -----------------------------------
template <typename T> struct RowValue {           // plain rows
  const T* x;
  __device__ __forceinline__ float operator()(int c) const { return ldf(x + c); }
};
template <typename T> struct SwigluValue {        // gate in [0, d), up in [d, 2 d)
  const T* x;
  int d;
  __device__ __forceinline__ float operator()(int c) const { return swiglu(ldf(x + c), ldf(x + d + c)); }
};

// One workgroup per row, any width and alignment: the row is read twice.
template <typename T, bool SWIGLU>
__global__ void __launch_bounds__(256) quant_i8_kernel(const T* __restrict__ x, int rows, int d,
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
                                                      const TG* __restrict__ g, int rows, int d, float eps,
                                                      float* resid, int8_t* __restrict__ q,
                                                      float* __restrict__ scale) {
  __shared__ float red[4];
  __shared__ uint32_t redu[4];
  const size_t at = (size_t)blockIdx.x * d;
  auto sum = [&](int c) { return delta ? x[at + c] + ldf(delta + at + c) : x[at + c]; };
  float ss = 0.f;
  for (int c = threadIdx.x; c < d; c += 256) { const float r = sum(c); ss += r * r; }
  ss = block_sum256(ss, red);
  const float inv = inverse_rms(ss, d, eps);
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

static bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// The register form for a row of d elements, in pieces of 4 where the addresses
// allow it: the fewest threads that hold the row.
#define ROWS_DISPATCH(GO)                 \
  do {                                    \
    if (vec) {                            \
      if (d <= 1024) GO(4, 4, 64);        \
      if (d <= 4096) GO(4, 4, 256);       \
      if (d <= 8192) GO(4, 8, 256);       \
      if (d <= 16384) GO(4, 4, 1024);     \
      if (d <= 32768) GO(4, 8, 1024);     \
    } else {                              \
      if (d <= 1024) GO(1, 16, 64);       \
      if (d <= 4096) GO(1, 16, 256);      \
      if (d <= 8192) GO(1, 32, 256);      \
      if (d <= 32768) GO(1, 32, 1024);    \
    }                                     \
  } while (0)

template <typename T>
static hipError_t quant_t(int rows, int d, bool sw, const T* x, int8_t* q, float* scale, hipStream_t st) {
  const bool vec = d % 4 == 0 && aligned(x, 4 * sizeof(T)) && aligned(q, 4);
  const size_t width = sw ? (size_t)2 * d : d;
  const auto by_rows = [&](auto plain, auto gated, int threads, int rows_per_wg) {
    return launch_rows(rows, threads, rows_per_wg, [&](int at, int n) {
      launch(sw ? gated : plain, dim3(ceil_div(n, rows_per_wg)), dim3(threads), 0, st, x + at * width, n, d,
             q + (size_t)at * d, scale + at);
    });
  };
#define QUANT(V, NV, TPR)                                                                         \
  return by_rows(quant_rows_kernel<T, false, V, NV, TPR>, quant_rows_kernel<T, true, V, NV, TPR>, \
                 TPR < 256 ? 256 : TPR, TPR < 256 ? 256 / TPR : 1)
  if constexpr (sizeof(T) == 2) {                  // 16-byte loads of 16-bit rows
    if (d % 8 == 0 && aligned(x, 16) && aligned(q, 8)) {
      if (d <= 1024) QUANT(8, 2, 64);
      if (d <= 4096) QUANT(8, 2, 256);
      if (d <= 8192) QUANT(8, 1, 1024);
      if (d <= 16384) QUANT(8, 2, 1024);
      if (d <= 32768) QUANT(8, 4, 1024);
    }
  }
  ROWS_DISPATCH(QUANT);
#undef QUANT
  return by_rows(quant_i8_kernel<T, false>, quant_i8_kernel<T, true>, 256, 1);
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
  const bool vec = d % 4 == 0 && aligned(x, 16) && aligned(g, 4 * sizeof(TG)) && aligned(q, 4) &&
                   aligned(delta, 4 * sizeof(TD)) && aligned(resid, 16);
  const auto by_rows = [&](auto kernel, int threads, int rows_per_wg) {
    return launch_rows(rows, threads, rows_per_wg, [&](int row, int n) {
      const size_t at = (size_t)row * d;
      launch(kernel, dim3(ceil_div(n, rows_per_wg)), dim3(threads), 0, st, x + at, delta ? delta + at : delta, g,
             n, d, eps, resid ? resid + at : resid, q + at, scale + row);
    });
  };
#define NORM(V, NV, TPR) \
  return by_rows(norm_rows_kernel<TD, TG, V, NV, TPR>, TPR < 256 ? 256 : TPR, TPR < 256 ? 256 / TPR : 1)
  ROWS_DISPATCH(NORM);
#undef NORM
  return by_rows(norm_i8_kernel<TD, TG>, 256, 1);
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

// The rows of one launch, for tests.
#ifdef SSM_DEBUG
extern "C" int64_t ssm_debug_rows_a_launch(int32_t threads, int32_t rows_per_wg) {
  return ssm::rows_a_launch(threads, rows_per_wg);
}
#endif
