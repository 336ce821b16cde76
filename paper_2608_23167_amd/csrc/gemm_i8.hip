// Products of 8-bit rows with 8-bit weights:
//   out[m, n] = a_scale[m] * w_scale[n] * sum_k a[m, k] * w[n, k]
// The sums are int32 and exact (K < 2^17), whatever the order; the two scales
// are multiplied onto the sum in float32 and the result is rounded once.
//
// Rows and weights are row-major.  v_mfma_i32_16x16x64_i8 takes 16 bytes of
// one row from each lane (row lane % 16, columns 16 (lane / 16) .. + 15 of 64),
// so a 16-byte load is an operand as it stands; the weights are its first
// operand, and a lane then holds 4 consecutive outputs of one row.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "internal.h"
#include "tiles.h"

namespace ssm {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4_t mma_i8(i32x4_t w, i32x4_t a, i32x4_t c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, a, c, 0, 0, 0);
}

// Where a result goes.
struct I8Out {
  void* p;
  int dtype;                 // 0 float32, 1 bfloat16, 2 float16
  int vec;                   // 4 consecutive columns may be stored at once
  const float *sa, *sw;
  int M, N;
  __device__ __forceinline__ void put(size_t i, float v) const {
    if (dtype == 0) ((float*)p)[i] = v;
    else if (dtype == 1) ((bf16_t*)p)[i] = f2bf(v);
    else ((f16_t*)p)[i] = (f16_t)v;
  }
  __device__ __forceinline__ void store(int m, int n, int acc) const {
    put((size_t)m * N + n, (float)acc * (sa[m] * sw[n]));
  }
  // scales of columns n .. n + 3 (those past the last are not used)
  __device__ __forceinline__ void scales4(int n, float (&s)[4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = sw[min(n + r, N - 1)];
  }
  // columns n .. n + 3 of row m < M, n a multiple of 4
  __device__ __forceinline__ void store4(int m, int n, const i32x4_t& acc, const float (&s)[4]) const {
    const float sm = sa[m];
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = (float)acc[r] * (sm * s[r]);
    const size_t i = (size_t)m * N + n;
    if (vec && n < N) {
      if (dtype == 0) {
        *(float4*)((float*)p + i) = make_float4(v[0], v[1], v[2], v[3]);
      } else if (dtype == 1) {
        *(uint2*)((bf16_t*)p + i) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      } else {
        const f16x4_t h = {(f16_t)v[0], (f16_t)v[1], (f16_t)v[2], (f16_t)v[3]};
        *(f16x4_t*)((f16_t*)p + i) = h;
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (n + r < N) put(i + r, v[r]);
    }
  }
};

// ---------------------------------------------------------------------------
// Any size and alignment
// ---------------------------------------------------------------------------
// 64 x 64 tiles, 64 columns of K at a time through LDS byte by byte, four
// products an instruction.
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

// The kernels below need K a multiple of 16 and 16-byte aligned operands: every
// 16-byte chunk of a row is then whole and inside its row.

// ---------------------------------------------------------------------------
// Few rows: K split over the waves of a workgroup
// ---------------------------------------------------------------------------
// 16 weight rows and up to 16 FM rows to a workgroup of 8 waves.  Wave w takes
// an eighth of the K-steps of 64 and reads its operands straight from memory
// (no operand is read by two waves of a workgroup); the eight partial sums
// join in LDS.  Bound by the weights' bytes: each wave keeps two batches of U
// K-steps in flight.
template <int FM, int U>
__global__ void __launch_bounds__(512) gemm_i8_few_kernel(const int8_t* __restrict__ A,
                                                          const int8_t* __restrict__ W, int M, int N,
                                                          int K, I8Out out) {
  __shared__ i32x4_t red[8][FM][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * FM);
  const int steps = (K + 63) >> 6, s0 = wave * steps >> 3, s1 = (wave + 1) * steps >> 3;
  const int8_t* wp = W + (size_t)min(n0 + r16, N - 1) * K;
  const int8_t* ap[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) ap[i] = A + (size_t)min(m0 + 16 * i + r16, M - 1) * K;
  i32x4_t acc[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) acc[i] = i32x4_t{0, 0, 0, 0};
  if (s0 < s1) {
    i32x4_t w[2][U], a[2][U][FM];
    // K-steps s .. s + U - 1; past s1 or K the activations are 0
    auto load = [&](int s, i32x4_t (&lw)[U], i32x4_t (&la)[U][FM]) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (s + u) * 64 + q * 16, kc = min(k, K - 16);
        const bool in = s + u < s1 && k < K;
        lw[u] = *(const i32x4_t*)(wp + kc);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const i32x4_t v = *(const i32x4_t*)(ap[i] + kc);
          la[u][i] = in ? v : i32x4_t{0, 0, 0, 0};
        }
      }
    };
    auto mma = [&](const i32x4_t (&lw)[U], const i32x4_t (&la)[U][FM]) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[i] = mma_i8(lw[u], la[u][i], acc[i]);
    };
    load(s0, w[0], a[0]);
    for (int s = s0; s < s1; s += 2 * U) {
      load(s + U, w[1], a[1]);
      mma(w[0], a[0]);
      load(s + 2 * U, w[0], a[0]);
      mma(w[1], a[1]);
    }
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) red[wave][i][lane] = acc[i];
  __syncthreads();
  // output o of the tile: column o % 16 of row o / 16
  for (int o = threadIdx.x; o < 256 * FM; o += 512) {
    const int n = o & 15, m = o >> 4;
    if (m0 + m >= M || n0 + n >= N) continue;
    int sum = 0;
#pragma unroll
    for (int v = 0; v < 8; ++v) sum += ((const int*)&red[v][m >> 4][(n >> 2) * 16 + (m & 15)])[n & 3];
    out.store(m0 + m, n0 + n, sum);
  }
}

// ---------------------------------------------------------------------------
// Cached steps: weights straight into registers, rows through LDS
// ---------------------------------------------------------------------------
// 16 FM rows and 16 FN NW weight rows to a workgroup of NW waves; every wave
// multiplies all the rows with its own 16 FN weight rows.  K-steps of 128.  A
// weight is read by one wave only, so it goes from memory to the registers of
// that wave, D K-steps ahead; the rows are read by every wave and go through
// two LDS buffers, loaded two K-steps ahead and written one ahead, one barrier
// a K-step.  In LDS a row group's 64 columns are 1 KB in operand order (chunk
// c of row r at 16 (c % 4) + (r ^ 2 c)): the exclusive or spreads the 8 chunks
// of a row, written by neighbouring threads, over the banks.
template <int FM, int FN, int NW, int D>
__global__ void __launch_bounds__(64 * NW) gemm_i8_stream_kernel(const int8_t* __restrict__ A,
                                                                 const int8_t* __restrict__ W, int M,
                                                                 int N, int K, int mt, int n_split,
                                                                 int* __restrict__ part, int ldp,
                                                                 I8Out out) {
  constexpr int T = 64 * NW, BM = 16 * FM, BN = 16 * FN * NW, CH = BM * 8, CA = (CH + T - 1) / T;
  constexpr int BUF = BM * 128;
  static_assert(D % 2 == 0, "the two row buffers alternate");
  __shared__ __attribute__((aligned(1024))) char smem[2 * BUF];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  int t, mtile, split;
  tile_of(blockIdx.x, gridDim.x, gridDim.x / n_split, mt, split, t, mtile);
  const int m0 = mtile * BM, n0 = t * BN + wave * 16 * FN;
  const int k_steps = (K + 127) >> 7;
  const int ks0 = (int)((long long)split * k_steps / n_split), ks1 = (int)((long long)(split + 1) * k_steps / n_split);
  const int nk = ks1 - ks0, kend = min(K, ks1 * 128);

  const int8_t* wp[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) wp[j] = W + (size_t)min(n0 + 16 * j + r16, N - 1) * K;
  const int8_t* ap[CA];
  int a_dst[CA], a_col[CA];
#pragma unroll
  for (int i = 0; i < CA; ++i) {
    const int x = min(tid + T * i, CH - 1), r = x >> 3, c = x & 7;   // past the last: the last again
    ap[i] = A + (size_t)min(m0 + r, M - 1) * K;
    a_col[i] = c * 16;
    a_dst[i] = ((r >> 4) * 2 + (c >> 2)) * 1024 + ((c & 3) * 16 + ((r & 15) ^ (2 * c))) * 16;
  }
  i32x4_t wr[D][FN][2], ar[2][CA];
  auto load_w = [&](int x, i32x4_t (&v)[FN][2]) {
    const int k = (ks0 + min(x, nk - 1)) * 128 + q * 16;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) v[j][h] = *(const i32x4_t*)(wp[j] + min(k + 64 * h, K - 16));
  };
  // rows of K-step x; 0 past this split's columns, so that steps past the last add nothing
  auto load_a = [&](int x, i32x4_t (&v)[CA]) {
#pragma unroll
    for (int i = 0; i < CA; ++i) {
      const int k = (ks0 + x) * 128 + a_col[i];
      const i32x4_t u = *(const i32x4_t*)(ap[i] + min(k, K - 16));
      v[i] = k < kend ? u : i32x4_t{0, 0, 0, 0};
    }
  };
  auto write_a = [&](const i32x4_t (&v)[CA], int buf) {
#pragma unroll
    for (int i = 0; i < CA; ++i)
      if (CH % T == 0 || tid + T * i < CH) *(i32x4_t*)(smem + buf * BUF + a_dst[i]) = v[i];
  };
  i32x4_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  auto mma = [&](const i32x4_t (&w)[FN][2], int buf) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* src = smem + buf * BUF + h * 1024 + (q * 16 + (r16 ^ (2 * (4 * h + q)))) * 16;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const i32x4_t a = *(const i32x4_t*)(src + i * 2048);
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mma_i8(w[j][h], a, acc[i][j]);
      }
    }
  };

  load_a(0, ar[0]);
  load_a(1, ar[1]);
#pragma unroll
  for (int u = 0; u < D; ++u) load_w(u, wr[u]);
  write_a(ar[0], 0);
  load_a(2, ar[0]);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  for (int x0 = 0; x0 < nk; x0 += D) {
#pragma unroll
    for (int u = 0; u < D; ++u) {
      const int x = x0 + u;
      write_a(ar[(u + 1) & 1], (u + 1) & 1);        // K-step x + 1
      load_a(x + 3, ar[(u + 1) & 1]);
      mma(wr[u], u & 1);
      load_w(x + D, wr[u]);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
  }
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int n = n0 + 16 * j + 4 * q;
    float s[4];
    if (!part) out.scales4(n, s);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = m0 + 16 * i + r16;
      if (m >= M) continue;
      if (!part) out.store4(m, n, acc[i][j], s);
      else if (n < ldp) *(i32x4_t*)(part + ((size_t)split * M + m) * ldp + n) = acc[i][j];
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows: two wave groups in alternation
// ---------------------------------------------------------------------------
// A BM x BN tile to a workgroup of 8 waves in a WM x WN grid, K-steps of 128 in
// two halves of 64.  Waves w and w + 4 share a SIMD; the waves 4-7 run half a
// phase behind the waves 0-3, so that on every SIMD one wave issues MFMAs while
// the other reads its next operands from LDS and starts copies.  A phase of a
// wave is
//   memory part:  LDS reads of one half K-step's fragments, copies of later
//                 K-steps (global_load_lds), wait for the reads, barrier;
//   MFMA part:    FM x FN MFMAs on them, barrier.
// Barriers number the slots: in slot 4t (even) the first group reads half 0
// of K-step t, in 4t + 1 the second group does while the first multiplies, and
// so on.  LDS rings: two stages of rows (BM x 128, each half separate), three of
// weights (BN x 128).  What a copy overwrites and where it is read:
//   weights t + 2        stage read last in slot 4t - 1, copied in 4t / 4t + 1,
//                        read from slot 4t + 8 on;
//   rows t + 1, half 1:  read last in slot 4t - 1, copied in 4t / 4t + 1,
//                        read from slot 4t + 6 on;
//   rows t + 2, half 0:  read last in slot 4t + 1, copied in 4t + 2 / 4t + 3,
//                        read from slot 4t + 8 on.
// Each wave waits, before the barrier that opens a slot in which the first
// group reads, until only its copies of the last two phases are in flight.
// Copies past the last K-step repeat the last one (never read), which keeps
// the count uniform.
//
// A copy is 1 KB, 16 bytes a lane in order.  One of weights covers 8 rows of
// 128 bytes, chunk c of row r at place c ^ ((r / 2) % 8); one of rows covers 16
// rows of 64 bytes, chunk c of row r at place c ^ ((r / 4) % 4): in both the 16
// rows of a fragment read fall on 16 different 16-byte columns of the banks.
// What is left of K past the last whole K-step is multiplied from registers.
template <int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(512, 2) gemm_i8_pp_kernel(const int8_t* __restrict__ A,
                                                            const int8_t* __restrict__ W, int M,
                                                            int N, int K, int mt, int n_split,
                                                            int* __restrict__ part, int ldp,
                                                            I8Out out) {
  static_assert(WM * WN == 8, "8 waves");
  constexpr int RW = BM / WM, CW = BN / WN, FM = RW / 16, FN = CW / 16;
  constexpr int LA = BM / 128, LW = BN / 64;       // copies per wave: half K-step of rows, K-step of weights
  static_assert(BM % 128 == 0 && BN % 64 == 0, "whole copies per wave");
  constexpr int A_HALF = BM * 64, A_STAGE = 2 * A_HALF, W_STAGE = BN * 128;   // bytes
  constexpr int INFLIGHT = LW + 2 * LA;
  __shared__ __attribute__((aligned(1024))) char smem[2 * A_STAGE + 3 * W_STAGE];
  char* const Ws = smem + 2 * A_STAGE;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const bool late = wave >= 4;                     // the second group
  int t, mtile, split;
  tile_of(blockIdx.x, gridDim.x, gridDim.x / n_split, mt, split, t, mtile);
  const int m0 = mtile * BM, n0 = t * BN;
  const int k_steps = K >> 7;                      // whole ones
  const int ks0 = (int)((long long)split * k_steps / n_split);
  const int nk = (int)((long long)(split + 1) * k_steps / n_split) - ks0, last = nk - 1;   // nk >= 1 (host-checked)

  // copy sources: a uniform first row, and the lane's row and chunk from there
  const int8_t *a_src[LA], *w_src[LW];
  uint32_t a_off[LA], w_off[LW];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int b = min(m0 + 16 * (wave * LA + i), M - 1), r = lane >> 2;
    a_src[i] = A + (size_t)b * K + (size_t)ks0 * 128;
    a_off[i] = (uint32_t)min(r, M - 1 - b) * K + (((lane & 3) ^ (r >> 2)) << 4);
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const int p = wave * LW + i, b = min(n0 + 8 * p, N - 1), r = lane >> 3;
    w_src[i] = W + (size_t)b * K + (size_t)ks0 * 128;
    w_off[i] = (uint32_t)min(r, N - 1 - b) * K + (((lane & 7) ^ (r >> 1) ^ (4 * (p & 1))) << 4);
  }
  auto copy = [](const int8_t* src, uint32_t off, char* dst) {
    __builtin_amdgcn_global_load_lds((const void*)(src + off),
                                     (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
  };
  // half kk of K-step v (rows), into stage v % 2
  auto issue_a = [&](int v, int kk) {
    const int vs = min(v, last);
    char* dst = smem + (v & 1) * A_STAGE + kk * A_HALF + wave * LA * 1024;
#pragma unroll
    for (int i = 0; i < LA; ++i) copy(a_src[i] + (size_t)vs * 128 + kk * 64, a_off[i], dst + i * 1024);
  };
  // K-step v (weights), into ring slot `slot`
  auto issue_w = [&](int v, int slot) {
    const int vs = min(v, last);
    char* dst = Ws + slot * W_STAGE + wave * LW * 1024;
#pragma unroll
    for (int i = 0; i < LW; ++i) copy(w_src[i] + (size_t)vs * 128, w_off[i], dst + i * 1024);
  };

  i32x4_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  i32x4_t af[FM], wf[FN];

  // LDS offsets of this wave's fragments
  const int r16 = lane & 15, g4 = lane >> 4;
  const int a_frag = wm * FM * 1024 + r16 * 64 + ((g4 ^ (r16 >> 2)) << 4);
  const int w_lane = r16 * 128 + ((g4 ^ (r16 >> 1)) << 4);        // half 0; half 1: chunk ^ 4
  auto read = [&](int v, int slot, int kk) {
    const char* a = smem + (v & 1) * A_STAGE + kk * A_HALF + a_frag;
    const char* w = Ws + slot * W_STAGE + wn * CW * 128 + (w_lane ^ (kk << 6));
#pragma unroll
    for (int j = 0; j < FN; ++j) wf[j] = *(const i32x4_t*)(w + j * 2048);
#pragma unroll
    for (int i = 0; i < FM; ++i) af[i] = *(const i32x4_t*)(a + i * 1024);
  };
  auto mma = [&]() {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mma_i8(wf[j], af[i], acc[i][j]);
    __builtin_amdgcn_s_setprio(0);
  };
  // end of a memory part / of an MFMA part
  auto end_mem = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));   // lgkmcnt(0)
    if (late) wait_vmcnt<INFLIGHT>();
    pp_barrier();
  };
  auto end_mma = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    if (!late) wait_vmcnt<INFLIGHT>();
    pp_barrier();
  };

  issue_w(0, 0);
  issue_a(0, 0);
  issue_a(0, 1);
  issue_w(1, 1);
  issue_a(1, 0);
  wait_vmcnt<LW + LA>();
  pp_barrier();
  if (late) pp_barrier();
  int s0 = 0, s2 = 2;                               // ring slots of K-steps v and v + 2
  for (int v = 0; v < nk; ++v) {
    read(v, s0, 0);
    issue_w(v + 2, s2);
    issue_a(v + 1, 1);
    end_mem();
    mma();
    end_mma();
    read(v, s0, 1);
    issue_a(v + 2, 0);
    end_mem();
    mma();
    end_mma();
    s2 = s0;
    s0 = s0 == 2 ? 0 : s0 + 1;
  }
  if (!late) pp_barrier();
  wait_vmcnt<0>();                                  // no copy lands after the workgroup ends

  if ((K & 127) && split == n_split - 1) {          // the columns past the last whole K-step
    for (int k0 = k_steps * 128; k0 < K; k0 += 64) {
      const int k = k0 + 16 * g4, kc = min(k, K - 16);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        wf[j] = *(const i32x4_t*)(W + (size_t)min(n0 + wn * CW + 16 * j + r16, N - 1) * K + kc);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const i32x4_t u = *(const i32x4_t*)(A + (size_t)min(m0 + wm * RW + 16 * i + r16, M - 1) * K + kc);
        af[i] = k < K ? u : i32x4_t{0, 0, 0, 0};
      }
      mma();
    }
  }

  // acc[i][j][r] = C[m0 + RW wm + 16 i + lane % 16][n0 + CW wn + 16 j + 4 (lane / 16) + r]
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int n = n0 + wn * CW + 16 * j + 4 * g4;
    float s[4];
    if (!part) out.scales4(n, s);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = m0 + wm * RW + 16 * i + r16;
      if (m >= M) continue;
      if (!part) out.store4(m, n, acc[i][j], s);
      else if (n < ldp) *(i32x4_t*)(part + ((size_t)split * M + m) * ldp + n) = acc[i][j];
    }
  }
}

// ---------------------------------------------------------------------------
// Sum of split-K partials
// ---------------------------------------------------------------------------
// 4 columns a thread; part is [S, M, ldp] with ldp a multiple of 16.
__global__ void __launch_bounds__(256) gemm_i8_sum_kernel(const int* __restrict__ part, int S, int M,
                                                          int ldp, I8Out out) {
  const size_t x = (size_t)blockIdx.x * 256 + threadIdx.x, per = ldp >> 2;
  if (x >= (size_t)M * per) return;
  const int m = (int)(x / per), n = 4 * (int)(x % per);
  if (n >= out.N) return;
  i32x4_t sum = {0, 0, 0, 0};
  for (int v = 0; v < S; ++v) sum += *(const i32x4_t*)(part + ((size_t)v * M + m) * ldp + n);
  float s[4];
  out.scales4(n, s);
  out.store4(m, n, sum, s);
}

// ---------------------------------------------------------------------------
// Launch choice
// ---------------------------------------------------------------------------
enum { I8_FEW = 0, I8_STREAM = 1, I8_PP = 2 };
struct I8Plan {
  int kind, tile, split;
};

static int i8_ldp(int N) { return (N + 15) & ~15; }

// Tiles of the stream kernel (fm x 16 rows, fn x 16 x nw weight rows) and of
// the alternating one.
struct I8Stream { int fm, fn, nw; };
static constexpr I8Stream I8_STREAMS[] = {{2, 1, 8}, {4, 1, 8}, {8, 1, 8}, {8, 1, 4}, {8, 2, 4}, {16, 2, 4}, {16, 1, 4}, {4, 1, 4}};
struct I8Pp { int bm, bn; };
static constexpr I8Pp I8_PPS[] = {{256, 256}, {256, 128}, {128, 256}, {128, 128}};

static I8Plan i8_plan(int M, int N, int K) {
#ifdef SSM_TUNING
  if (const char* e = getenv("SSM_I8_CFG")) {     // kind:tile:split, for sweeps
    I8Plan p;
    if (sscanf(e, "%d:%d:%d", &p.kind, &p.tile, &p.split) == 3) return p;
  }
#endif
  if (M <= 32) return {I8_FEW, 0, 1};
  const int steps = (K + 127) / 128;
  if (M <= 384 || K < 512) {
    const int tile = M <= 64 ? 1 : M <= 128 ? 2 : 5;
    const I8Stream& s = I8_STREAMS[tile];
    const int tiles = ceil_div(M, 16 * s.fm) * ceil_div(N, 16 * s.fn * s.nw);
    int S = 1;
    while (S < 8 && tiles * S * 2 <= 320 && steps / (S * 2) >= 4) S *= 2;
    return {I8_STREAM, tile, S};
  }
  const int tiles = ceil_div(M, 256) * ceil_div(N, 256);
  int S = 1;
  while (S < 4 && tiles * (S + 1) <= 256 && (K / 128) / (S + 1) >= 8) ++S;
  return {I8_PP, 0, S};
}

size_t gemm_i8_ws_bytes(int M, int N, int K) {
  if (M == 0 || K % 16) return 0;
  const I8Plan p = i8_plan(M, N, K);
  return p.split > 1 ? (size_t)p.split * M * i8_ldp(N) * 4 : 0;
}

template <int FM, int FN, int NW>
static void launch_stream(const I8Plan& p, int M, int N, int K, const int8_t* a, const int8_t* w,
                          int* part, const I8Out& out, hipStream_t st) {
  const int mt = ceil_div(M, 16 * FM);
  launch((gemm_i8_stream_kernel<FM, FN, NW, 4>), dim3(mt * ceil_div(N, 16 * FN * NW) * p.split),
         dim3(64 * NW), 0, st, a, w, M, N, K, mt, p.split, part, i8_ldp(N), out);
}
template <int BM, int BN, int WM, int WN>
static void launch_pp(const I8Plan& p, int M, int N, int K, const int8_t* a, const int8_t* w,
                      int* part, const I8Out& out, hipStream_t st) {
  const int mt = ceil_div(M, BM);
  launch((gemm_i8_pp_kernel<BM, BN, WM, WN>), dim3(mt * ceil_div(N, BN) * p.split), dim3(512), 0, st,
         a, w, M, N, K, mt, p.split, part, i8_ldp(N), out);
}

hipError_t gemm_i8(int M, int N, int K, const int8_t* a, const float* sa, const int8_t* w,
                   const float* sw, int out_dtype, void* out, void* ws, hipStream_t st) {
  if (M == 0) return hipSuccess;
  const size_t es = out_dtype == 0 ? 4 : 2;
  const I8Out o{out, out_dtype, N % 4 == 0 && ((uintptr_t)out & (4 * es - 1)) == 0, sa, sw, M, N};
  if (K % 16 || ((uintptr_t)a & 15) || ((uintptr_t)w & 15)) {
    launch(gemm_i8_any_kernel, dim3(ceil_div(N, 64), ceil_div(M, 64)), dim3(256), 0, st, a, w, M, N, K, o);
    return hipGetLastError();
  }
  const I8Plan p = i8_plan(M, N, K);
  int* part = p.split > 1 ? (int*)ws : nullptr;
  if (p.kind == I8_FEW) {
    if (M <= 16)
      launch((gemm_i8_few_kernel<1, 4>), dim3(ceil_div(N, 16), 1), dim3(512), 0, st, a, w, M, N, K, o);
    else
      launch((gemm_i8_few_kernel<2, 4>), dim3(ceil_div(N, 16), ceil_div(M, 32)), dim3(512), 0, st, a, w, M, N, K, o);
    return hipGetLastError();
  }
  if (p.kind == I8_STREAM) {
    switch (p.tile) {
      case 0: launch_stream<2, 1, 8>(p, M, N, K, a, w, part, o, st); break;
      case 1: launch_stream<4, 1, 8>(p, M, N, K, a, w, part, o, st); break;
      case 2: launch_stream<8, 1, 8>(p, M, N, K, a, w, part, o, st); break;
      case 3: launch_stream<8, 1, 4>(p, M, N, K, a, w, part, o, st); break;
      case 4: launch_stream<8, 2, 4>(p, M, N, K, a, w, part, o, st); break;
      case 5: launch_stream<16, 2, 4>(p, M, N, K, a, w, part, o, st); break;
      case 6: launch_stream<16, 1, 4>(p, M, N, K, a, w, part, o, st); break;
      default: launch_stream<4, 1, 4>(p, M, N, K, a, w, part, o, st); break;
    }
  } else {
    switch (p.tile) {
      case 0: launch_pp<256, 256, 2, 4>(p, M, N, K, a, w, part, o, st); break;
      case 1: launch_pp<256, 128, 4, 2>(p, M, N, K, a, w, part, o, st); break;
      case 2: launch_pp<128, 256, 2, 4>(p, M, N, K, a, w, part, o, st); break;
      default: launch_pp<128, 128, 4, 2>(p, M, N, K, a, w, part, o, st); break;
    }
  }
  if (part) {
    const size_t n = (size_t)M * (i8_ldp(N) / 4);
    launch(gemm_i8_sum_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, part, p.split, M,
           i8_ldp(N), o);
  }
  return hipGetLastError();
}

}  // namespace ssm
