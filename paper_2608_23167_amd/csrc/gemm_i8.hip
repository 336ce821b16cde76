// Products of 8-bit rows with 8-bit weights:
//   out[m, n] = a_scale[m] * w_scale[n] * sum_k a[m, k] * w[n, k]
// The sums are int32 and exact (K < 2^17), whatever the order; the two scales
// are multiplied onto the sum in float32, the row's first, and the result is rounded once.
//
// Rows and weights are row-major.  v_mfma_i32_16x16x64_i8 takes 16 bytes of
// one row from each lane (row lane % 16, columns 16 (lane / 16) .. + 15 of 64),
// so a 16-byte load is an operand as it stands; the weights are its first
// operand, and a lane then holds 4 consecutive outputs of one row.
#include <stdio.h>
#include <stdlib.h>

#include "dcheck.h"
#include "internal.h"
#include "tiles.h"

namespace ssm {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4_t mma_i8(i32x4_t w, i32x4_t a, i32x4_t c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, a, c, 0, 0, 0);
}

__device__ __forceinline__ void put4(float* p, const float (&v)[4]) {
  *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void put4(bf16_t* p, const float (&v)[4]) {
  *(uint2*)p = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}
__device__ __forceinline__ void put4(f16_t* p, const float (&v)[4]) {
  *(f16x4_t*)p = f16x4_t{(f16_t)v[0], (f16_t)v[1], (f16_t)v[2], (f16_t)v[3]};
}

// A sum with its scales.  The product of the two scales can leave the float32 range where
// the result does not (0 times infinity, or a result of 0), so it is not formed.
__device__ __forceinline__ float scaled(int sum, float sa, float sw) { return (float)sum * sa * sw; }

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
    put((size_t)m * N + n, scaled(acc, sa[m], sw[n]));
  }
  // scales of columns n .. n + 3 (those past the last are not used)
  __device__ __forceinline__ void scales4(int n, float (&s)[4]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = sw[min(n + r, N - 1)];
  }
  // columns n .. n + 3 of row m < M, n a multiple of 4, whose scales are sm and s
  __device__ __forceinline__ void store4(int m, int n, const i32x4_t& acc, float sm, const float (&s)[4]) const {
    const size_t i = (size_t)m * N + n;
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = scaled(acc[r], sm, s[r]);
    if (vec && n < N) {
      if (dtype == 0) put4((float*)p + i, v);
      else if (dtype == 1) put4((bf16_t*)p + i, v);
      else put4((f16_t*)p + i, v);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (n + r < N) put(i + r, v[r]);
    }
  }
};

// The scales of a wave's tile of FM x FN operands, loaded when the kernel starts:
// fetched after the products they cost a trip to memory that nothing hides (2 of
// the 12 us of a launch of one 256 x 256 tile).
template <int FM, int FN> struct TileScales {
  float m[FM], n[FN][4];
  __device__ __forceinline__ void load(const I8Out& out, int row, int col) {
#pragma unroll
    for (int i = 0; i < FM; ++i) m[i] = out.sa[min(row + 16 * i, out.M - 1)];
#pragma unroll
    for (int j = 0; j < FN; ++j) out.scales4(col + 16 * j, n[j]);
  }
  // the loads stay above this point
  __device__ __forceinline__ void hold() {
#pragma unroll
    for (int i = 0; i < FM; ++i) asm volatile("" : "+v"(m[i]));
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) asm volatile("" : "+v"(n[j][r]));
  }
};

// A wave's tile: acc[i][j][r] belongs to row m + 16 i, column n + 16 j + r, where n
// is n0 plus 4 times a quarter of the lane's number.  To the partials of this
// split, [splits, M, ldp], or out.
template <int FM, int FN, typename T>
__device__ __forceinline__ void rows_out(T* p, const i32x4_t (&acc)[FM][FN], int m, int M, int N,
                                         const TileScales<FM, FN>& sc) {
#pragma unroll
  for (int i = 0; i < FM; ++i, p += (size_t)16 * N) {
    if (m + 16 * i >= M) return;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = scaled(acc[i][j][r], sc.m[i], sc.n[j][r]);
      put4(p + 16 * j, v);
    }
  }
}
// The same element by element: a tile of the last columns, or rows that are not aligned.
template <int FM, int FN, typename T>
__device__ __forceinline__ void rows_edge(T* p, bool bf, const i32x4_t (&acc)[FM][FN], int m, int M, int n, int N,
                                          const TileScales<FM, FN>& sc) {
#pragma unroll
  for (int i = 0; i < FM; ++i, p += (size_t)16 * N) {
    if (m + 16 * i >= M) return;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (n + 16 * j + r >= N) continue;
        const float v = scaled(acc[i][j][r], sc.m[i], sc.n[j][r]);
        if constexpr (std::is_same<T, float>::value) p[16 * j + r] = v;
        else p[16 * j + r] = bf ? f2bf(v) : __builtin_bit_cast(uint16_t, (f16_t)v);
      }
  }
}
template <int FM, int FN>
__device__ __forceinline__ void tile_out(const i32x4_t (&acc)[FM][FN], const TileScales<FM, FN>& sc, int m,
                                         int n0, int n, int split, int* part, int ldp, const I8Out& out) {
  const int M = out.M;
  if (part) {
    int* p = part + ((size_t)split * M + m) * ldp + n;
#pragma unroll
    for (int i = 0; i < FM; ++i, p += (size_t)16 * ldp) {
      if (m + 16 * i >= M) return;
#pragma unroll
      for (int j = 0; j < FN; ++j)
        if (n0 + 16 * j < ldp) *(i32x4_t*)(p + 16 * j) = acc[i][j];   // ldp is a multiple of 16
    }
    return;
  }
  const size_t at = (size_t)m * out.N + n;
  if (out.vec && n0 + 16 * FN <= out.N) {
    if (out.dtype == 0) rows_out<FM, FN>((float*)out.p + at, acc, m, M, out.N, sc);
    else if (out.dtype == 1) rows_out<FM, FN>((bf16_t*)out.p + at, acc, m, M, out.N, sc);
    else rows_out<FM, FN>((f16_t*)out.p + at, acc, m, M, out.N, sc);
    return;
  }
  if (out.dtype == 0) rows_edge<FM, FN>((float*)out.p + at, 0, acc, m, M, n, out.N, sc);
  else rows_edge<FM, FN>((uint16_t*)out.p + at, out.dtype == 1, acc, m, M, n, out.N, sc);
}

// ---------------------------------------------------------------------------
// Any size and alignment
// ---------------------------------------------------------------------------
// 64 x 64 tiles, 4 waves of 32 x 32 each, K-steps of 128 through two LDS buffers, the
// loads two K-steps ahead.  16-byte loads at any address; the bytes of a chunk that
// K ends in are loaded singly, so that nothing past a row is read.  In LDS a group of
// 16 rows' 64 columns are 1 KB in operand order, chunk c of row r at 16 (c % 4) +
// (r ^ 2 c): the exclusive or spreads the 8 chunks of a row, written by neighbouring
// threads, over the banks.
typedef i32x4_t i32x4_any_t __attribute__((aligned(1)));

__device__ __forceinline__ i32x4_t chunk_any(const int8_t* row, int k, int K) {
  if (k + 16 <= K) return *(const i32x4_any_t*)(row + k);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < K) w[i >> 2] |= (uint32_t)(uint8_t)row[k + i] << (8 * (i & 3));
  return i32x4_t{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

__global__ void __launch_bounds__(256) gemm_i8_any_kernel(const int8_t* __restrict__ A,
                                                          const int8_t* __restrict__ W, int K, I8Out out) {
  constexpr int BUF = 64 * 128;
  __shared__ __attribute__((aligned(1024))) char smem[2][2][BUF];   // buffer, operand
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r16 = lane & 15, q = lane >> 4;
  const int M = out.M, N = out.N, m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
  const int nk = (K + 127) >> 7;
  SSM_DCHECK(m0 < M && n0 < N);
  const int8_t* src[2][2];
  int dst[2], col[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int x = tid + 256 * i, r = x >> 3, c = x & 7;
    src[0][i] = A + (size_t)min(m0 + r, M - 1) * K;
    src[1][i] = W + (size_t)min(n0 + r, N - 1) * K;
    col[i] = c * 16;
    dst[i] = ((r >> 4) * 2 + (c >> 2)) * 1024 + ((c & 3) * 16 + ((r & 15) ^ (2 * c))) * 16;
  }
  i32x4_t v[2][2];
  auto load = [&](int x) {
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
      for (int i = 0; i < 2; ++i) v[o][i] = chunk_any(src[o][i], x * 128 + col[i], K);
  };
  auto write = [&](int buf) {
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
      for (int i = 0; i < 2; ++i) *(i32x4_t*)(smem[buf][o] + dst[i]) = v[o][i];
  };
  const int wm = (wave & 1) * 2, wn = (wave >> 1) * 2;             // first 16-row group of the wave
  i32x4_t acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  load(0);
  write(0);
  load(1);                                          // past K: zeros
  __syncthreads();
  for (int x = 0; x < nk; ++x) {
    write((x + 1) & 1);                             // read last in x - 1
    load(x + 2);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = h * 1024 + (q * 16 + (r16 ^ (2 * (4 * h + q)))) * 16;
      i32x4_t a[2], w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) a[i] = *(const i32x4_t*)(smem[x & 1][0] + (wm + i) * 2048 + at);
#pragma unroll
      for (int j = 0; j < 2; ++j) w[j] = *(const i32x4_t*)(smem[x & 1][1] + (wn + j) * 2048 + at);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = mma_i8(w[j], a[i], acc[i][j]);
    }
    lds_written_barrier();
  }
  TileScales<2, 2> sc;
  const int m = m0 + 16 * wm + r16, n = n0 + 16 * wn;
  sc.load(out, m, n + 4 * q);
  tile_out(acc, sc, m, n, n + 4 * q, 0, nullptr, 0, out);
}

// The kernels below need K a multiple of 16 and 16-byte aligned operands: every
// 16-byte chunk of a row is then whole and inside its row.

// ---------------------------------------------------------------------------
// Few rows: K split over the waves of a workgroup
// ---------------------------------------------------------------------------
// 16 weight rows and up to 16 rows to a workgroup of 8 waves.  Wave w takes an eighth
// of the K-steps of 64 and reads its operands straight from memory (no operand is
// read by two waves of a workgroup); the eight partial sums join in LDS.  Bound by
// the weights' bytes: each wave keeps two batches of U K-steps in flight.  One row of
// 4096 x 4096: 6.5 us (2.6 TB/s; launch and one trip to memory are 4 of them).
template <int U>
__global__ void __launch_bounds__(512) gemm_i8_few_kernel(const int8_t* __restrict__ A,
                                                          const int8_t* __restrict__ W, int K, I8Out out) {
  __shared__ i32x4_t red[8][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int M = out.M, N = out.N, n0 = blockIdx.x * 16;
  SSM_DCHECK(M <= 16 && n0 < N && K >= 16 && K % 16 == 0);
  const int steps = (K + 63) >> 6, s0 = wave * steps >> 3, s1 = (wave + 1) * steps >> 3;
  const int8_t* wp = W + (size_t)min(n0 + r16, N - 1) * K;
  const int8_t* ap = A + (size_t)min(r16, M - 1) * K;
  i32x4_t acc = {0, 0, 0, 0};
  if (s0 < s1) {
    i32x4_t w[2][U], a[2][U];
    // K-steps s .. s + U - 1; past s1 or K the activations are 0
    auto load = [&](int s, i32x4_t (&lw)[U], i32x4_t (&la)[U]) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (s + u) * 64 + q * 16, kc = min(k, K - 16);
        lw[u] = *(const i32x4_t*)(wp + kc);
        const i32x4_t v = *(const i32x4_t*)(ap + kc);
        la[u] = s + u < s1 && k < K ? v : i32x4_t{0, 0, 0, 0};
      }
    };
    auto mma = [&](const i32x4_t (&lw)[U], const i32x4_t (&la)[U]) {
#pragma unroll
      for (int u = 0; u < U; ++u) acc = mma_i8(lw[u], la[u], acc);
    };
    load(s0, w[0], a[0]);
    for (int s = s0; s < s1; s += 2 * U) {
      load(s + U, w[1], a[1]);
      mma(w[0], a[0]);
      load(s + 2 * U, w[0], a[0]);
      mma(w[1], a[1]);
    }
  }
  red[wave][lane] = acc;
  __syncthreads();
  // output o of the tile: column o % 16 of row o / 16
  const int o = threadIdx.x, n = o & 15, m = o >> 4;
  if (o >= 256 || m >= M || n0 + n >= N) return;
  int sum = 0;
#pragma unroll
  for (int v = 0; v < 8; ++v) sum += ((const int*)&red[v][(n >> 2) * 16 + m])[n & 3];
  out.store(m, n0 + n, sum);
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
// so on.  LDS rings: PA stages of rows (BM x 128, each half separate), PA + 1 of
// weights (BN x 128).  What a copy overwrites and where it is read:
//   weights t + PA             stage of t - 1, read last in slot 4t - 1, copied in
//                              4t / 4t + 1, read from slot 4 (t + PA) on;
//   rows t + PA - 1, half 1:   stage of t - 1, read last in slot 4t - 1, copied in
//                              4t / 4t + 1, read from slot 4 (t + PA) - 2 on;
//   rows t + PA, half 0:       stage of t, read last in slot 4t + 1, copied in
//                              4t + 2 / 4t + 3, read from slot 4 (t + PA) on.
// A wave waits, before the barrier that opens a slot in which the first group
// reads, until only its copies of the last 2 (PA - 1) phases are in flight: at
// the end of (t, half 1) the oldest of those follow rows t + 1, half 0, and at
// the end of (t, half 0) they follow rows t, half 1.  Copies past the last
// K-step repeat the last one (never read), which keeps the count uniform.
//
// A copy is 1 KB, 16 bytes a lane in order.  One of weights covers 8 rows of
// 128 bytes, chunk c of row r at place c ^ ((r / 2) % 8); one of rows covers 16
// rows of 64 bytes, chunk c of row r at place c ^ half_place(r).  A 16-byte read takes
// 16 lanes at a time: in both layouts 16 consecutive ones fall on 16 different
// 16-byte columns of the banks, and so do the lanes 0-3, 12-15, 20-23 and 24-27 (4-11,
// 16-19 and 28-31) together, which counters say is how they go: with r / 4 for
// half_place(r), even for the first grouping only, 13% of the clocks were conflicts.
// What is left of K past the last whole K-step is multiplied from registers.
// 3840 x 24576 x 4096: 350-357 us, 2190 TOP/s; the MFMAs are busy 51% of the clocks, at 1.97
// GHz (kernels that wait for memory run at 2.3 and more).  Of a round of 61 us 10 pass before the
// first product and after the last; workgroups that stay for several tiles and start
// the next one's copies before they store were tried: the loop around it all spilled.
__device__ __forceinline__ int half_place(int r) {      // 0, 2, 3, 1 for r / 4 = 0 .. 3
  return ((r >> 2) & 1) * 2 ^ ((r >> 3) & 1) * 3;
}

// tile_of with the row tiles in groups of 4, innermost in a group: the 32 tiles that an XCD
// works on at a time are then about 4 x 8 and need 12 strips of rows and weights in its
// L2, where 15 x 2 need 17, and 3840 x 24576 x 4096 fetches 629 instead of 1192 MiB.  That
// one takes as long either way (351 and 354 us in turn); 3840 x 12288 x 4096 180 -> 173, 14208 x
// 24576 x 4096 1300 -> 1215 (2350 TOP/s); groups of 8 360, 175 and 1275.
__device__ __forceinline__ void grouped_tile_of(int w, int total, int ntm, int mt, int& split, int& tn,
                                                int& tm) {
  constexpr int GROUP = 4;
  const int per = total / 8;
  const int v = w < per * 8 ? (w % 8) * per + (w / 8) : w;
  split = v / ntm;
  const int x = v % ntm, nt = ntm / mt, first = x / (GROUP * nt) * GROUP, rows = min(GROUP, mt - first);
  const int y = x - first * nt;
  tm = first + y % rows;
  tn = y / rows;
}

template <int BM, int BN, int WM, int WN, int PA>
__global__ void __launch_bounds__(512, 2) gemm_i8_pp_kernel(const int8_t* __restrict__ A,
                                                            const int8_t* __restrict__ W, int K, int mt,
                                                            int n_split, int* __restrict__ part,
                                                            int ldp, I8Out out) {
  static_assert(WM * WN == 8, "8 waves");
  constexpr int RW = BM / WM, CW = BN / WN, FM = RW / 16, FN = CW / 16;
  static_assert(RW % 16 == 0 && CW % 16 == 0, "whole fragments per wave");
  constexpr int CA = BM / 16, CB = BN / 8;         // copies: half K-step of rows, K-step of weights
  static_assert(CA % 4 == 0 && CB % 4 == 0, "the waves of a group copy the same number");
  // of those, per wave of the first and of the second group
  constexpr int LA0 = (CA + 7) / 8, LA1 = (CA + 3) / 8, LW0 = (CB + 7) / 8, LW1 = (CB + 3) / 8;
  constexpr int A_HALF = BM * 64, A_STAGE = 2 * A_HALF, W_STAGE = BN * 128;   // bytes
  constexpr int FLIGHT0 = (PA - 1) * (LW0 + 2 * LA0), FLIGHT1 = (PA - 1) * (LW1 + 2 * LA1);
  __shared__ __attribute__((aligned(1024))) char smem[PA * A_STAGE + (PA + 1) * W_STAGE];
  char* const Ws = smem + PA * A_STAGE;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const bool late = wave >= 4;                     // the second group
  int t, mtile, split;
  grouped_tile_of(blockIdx.x, gridDim.x, gridDim.x / n_split, mt, split, t, mtile);
  const int M = out.M, N = out.N, m0 = mtile * BM, n0 = t * BN;
  const int k_steps = K >> 7;                      // whole ones
  const int ks0 = (int)((long long)split * k_steps / n_split);
  const int nk = (int)((long long)(split + 1) * k_steps / n_split) - ks0, last = nk - 1;   // nk >= 1 (host-checked)
  SSM_DCHECK(nk >= 1 && m0 < M && n0 < N && (part != nullptr) == (n_split > 1) && ldp >= N);
  const int rot = t % nk;
  auto kmap = [rot, nk](int x) { const int y = x + rot; return y >= nk ? y - nk : y; };

  // copy sources: a uniform first row, and the lane's row and chunk from there
  const int8_t *a_src[LA0], *w_src[LW0];
  uint32_t a_off[LA0], w_off[LW0];
#pragma unroll
  for (int i = 0; i < LA0; ++i) {
    const int b = min(m0 + 16 * (wave + 8 * i), M - 1), r = lane >> 2;
    a_src[i] = A + (size_t)b * K + (size_t)ks0 * 128;
    a_off[i] = (uint32_t)min(r, M - 1 - b) * K + (((lane & 3) ^ half_place(r)) << 4);
  }
#pragma unroll
  for (int i = 0; i < LW0; ++i) {
    const int p = wave + 8 * i, b = min(n0 + 8 * p, N - 1), r = lane >> 3;
    w_src[i] = W + (size_t)b * K + (size_t)ks0 * 128;
    w_off[i] = (uint32_t)min(r, N - 1 - b) * K + (((lane & 7) ^ (r >> 1) ^ (4 * (p & 1))) << 4);
  }
  auto copy = [](const int8_t* src, uint32_t off, char* dst) {
    __builtin_amdgcn_global_load_lds((const void*)(src + off),
                                     (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
  };
  // half kk of K-step v (rows), into stage `slot`
  auto issue_a = [&](int v, int kk, int slot) {
    const int vs = kmap(min(v, last));
    char* dst = smem + slot * A_STAGE + kk * A_HALF + wave * 1024;
#pragma unroll
    for (int i = 0; i < LA0; ++i)
      if (i < LA1 || !late) copy(a_src[i] + (size_t)vs * 128 + kk * 64, a_off[i], dst + i * 8192);
  };
  // K-step v (weights), into stage `slot`
  auto issue_w = [&](int v, int slot) {
    const int vs = kmap(min(v, last));
    char* dst = Ws + slot * W_STAGE + wave * 1024;
#pragma unroll
    for (int i = 0; i < LW0; ++i)
      if (i < LW1 || !late) copy(w_src[i] + (size_t)vs * 128, w_off[i], dst + i * 8192);
  };

  i32x4_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  i32x4_t af[FM], wf[FN];

  // LDS offsets of this wave's fragments
  const int r16 = lane & 15, g4 = lane >> 4;
  const int a_frag = wm * FM * 1024 + r16 * 64 + ((g4 ^ half_place(r16)) << 4);
  const int w_lane = r16 * 128 + ((g4 ^ (r16 >> 1)) << 4);        // half 0; half 1: chunk ^ 4
  auto read = [&](int slot_a, int slot_w, int kk) {
    const char* a = smem + slot_a * A_STAGE + kk * A_HALF + a_frag;
    const char* w = Ws + slot_w * W_STAGE + wn * CW * 128 + (w_lane ^ (kk << 6));
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
    if (late) wait_vmcnt<FLIGHT1>();
    pp_barrier();
  };
  auto end_mma = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    if (!late) wait_vmcnt<FLIGHT0>();
    pp_barrier();
  };

  TileScales<FM, FN> sc;
  if (!part) sc.load(out, m0 + wm * RW + r16, n0 + wn * CW + 4 * g4);
#pragma unroll
  for (int j = 0; j < PA; ++j) {                    // in the order of the loop's copies
    issue_w(j, j);
    if (j > 0) issue_a(j - 1, 1, j - 1);
    issue_a(j, 0, j);
  }
  if (late) wait_vmcnt<FLIGHT1>();
  else wait_vmcnt<FLIGHT0>();
  if (!part) sc.hold();
  pp_barrier();
  if (late) pp_barrier();
  int sa = 0, sw = 0;                               // stages of K-step v
  for (int v = 0; v < nk; ++v) {
    read(sa, sw, 0);
    issue_w(v + PA, sw == 0 ? PA : sw - 1);
    issue_a(v + PA - 1, 1, sa == 0 ? PA - 1 : sa - 1);
    end_mem();
    mma();
    end_mma();
    read(sa, sw, 1);
    issue_a(v + PA, 0, sa);
    end_mem();
    mma();
    end_mma();
    sa = sa == PA - 1 ? 0 : sa + 1;
    sw = sw == PA ? 0 : sw + 1;
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
  tile_out(acc, sc, m0 + wm * RW + r16, n0 + wn * CW, n0 + wn * CW + 4 * g4, split, part, ldp, out);
}

// ---------------------------------------------------------------------------
// Cached steps: two wave groups that share K
// ---------------------------------------------------------------------------
// The alternation above for smaller tiles, where a phase's LDS reads and its
// barriers would outlast its MFMAs: the waves 0-3 take half 0 of every K-step of
// 128 and the waves 4-7 half 1, each group the whole BM x BN tile (WM x WN = 4
// waves), so a wave has a tile twice as large and reads less for each MFMA, and a
// K-step takes 1 or 2 barriers instead of 4.  The groups' sums join in LDS at the end.
// Rows and weights share a ring of R stages; all copies are whole lines (8 rows of
// 128 bytes, chunks placed as above).
//  * In alternation (AHEAD false): slot 2t, the first group reads half 0 of K-step t
//    while the second multiplies half 1 of t - 1; slot 2t + 1, the other way round.  A
//    wave's copies of K-step t + R - 1, begun in its memory part of t, overwrite the stage
//    of t - 1, read last in slot 2t - 1.  Before the barrier that opens slot 2t + 2 each
//    wave waits until only its copies of the R - 2 latest K-steps are in flight: those of
//    t + 1 have then landed.
//  * Both groups at once (AHEAD true, tiles up to 128 x 96, whose MFMAs are shorter than a
//    trip to LDS): in K-step t a wave reads its operands of t + 1 into a second set of
//    registers, begins its copies of t + R into the stage of t (read in t - 1), multiplies
//    K-step t, and waits as above, so that t + 2 has landed; one barrier.  120 x 4096 x 4096
//    on 64 x 32 tiles 12.1 -> 10.6 us, 240 x 4096 x 4096 on 64 x 64 14.1 -> 13.1, 120 x 24576 x
//    4096 on 128 x 96 26.7 -> 25.5; 128 x 192 34.7 -> 35.3, 256 x 128 spills (83 -> 90).
// Weights that one workgroup reads (a single row tile, K not split) are loaded
// nontemporal, which leaves the caches to the rows: 120 x 24576 x 4096 29.5 -> 27.7 us, 40
// rows 21.6 -> 20.1, 120 x 126464 x 4096 124.6 -> 120.4; with two row tiles or splits it
// costs (376 x 12288 x 4096 28.9 -> 31.9, 120 x 4096 x 12288 20.9 -> 23.5).
// Bound by the weight stream and the ramp at both ends: 120 x 24576 x 4096 25.0 us, 101 MB
// of weights at 4.0 TB/s (gemm_i8_pp_kernel on the same tile 30.0 us; weights straight into
// registers, rows through LDS, one barrier a K-step 31.7); 240 x 4096 x 12288 in 4 splits
// 20 us and 4.4 for their sum; 1127 x 3584 x 18944 by LDS (64 KB read and 32 written a K-step,
// 768 clocks at its rate, for 512 of MFMAs), 85 us, 1800 TOP/s.
template <int BM, int BN, int WM, int WN, int R, bool AHEAD>
__global__ void __launch_bounds__(512, 2) gemm_i8_ks_kernel(const int8_t* __restrict__ A,
                                                            const int8_t* __restrict__ W, int K, int mt,
                                                            int n_split, int* __restrict__ part,
                                                            int ldp, I8Out out) {
  static_assert(WM * WN == 4 && R >= 3, "4 waves to a group");
  constexpr int RW = BM / WM, CW = BN / WN, FM = RW / 16, FN = CW / 16;
  static_assert(RW % 32 == 0 && CW % 16 == 0, "whole fragments per wave, an even number of rows of them");
  constexpr int CA = BM / 8, CB = BN / 8;          // copies of a K-step
  static_assert(CA % 4 == 0 && CB % 4 == 0, "the waves of a group copy the same number");
  // of those, per wave of the first and of the second group
  constexpr int LA0 = (CA + 7) / 8, LA1 = (CA + 3) / 8, LW0 = (CB + 7) / 8, LW1 = (CB + 3) / 8;
  constexpr int STAGE = (BM + BN) * 128;           // bytes: rows, then weights
  constexpr int FLIGHT0 = (R - 2) * (LA0 + LW0), FLIGHT1 = (R - 2) * (LA1 + LW1);
  static_assert(R * STAGE >= 4 * (FM / 2) * FN * 2 * 1024, "the groups' sums fit the ring");
  __shared__ __attribute__((aligned(1024))) char smem[R * STAGE];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int w4 = wave & 3, wm = w4 % WM, wn = w4 / WM;
  const bool late = wave >= 4;                     // the second group
  int t, mtile, split;
  tile_of(blockIdx.x, gridDim.x, gridDim.x / n_split, mt, split, t, mtile);
  const int M = out.M, N = out.N, m0 = mtile * BM, n0 = t * BN;
  const int k_steps = K >> 7;                      // whole ones
  const int ks0 = (int)((long long)split * k_steps / n_split);
  const int nk = (int)((long long)(split + 1) * k_steps / n_split) - ks0, last = nk - 1;   // nk >= 1 (host-checked)
  SSM_DCHECK(nk >= 1 && m0 < M && n0 < N && (part != nullptr) == (n_split > 1) && ldp >= N);
  const int rot = t % nk;
  auto kmap = [rot, nk](int x) { const int y = x + rot; return y >= nk ? y - nk : y; };

  // copy sources: a uniform first row, and the lane's row and chunk from there
  const int8_t *a_src[LA0], *w_src[LW0];
  uint32_t a_off[LA0], w_off[LW0];
  const int r8 = lane >> 3;
  auto chunk = [&](int p) { return (uint32_t)(((lane & 7) ^ (r8 >> 1) ^ (4 * (p & 1))) << 4); };
#pragma unroll
  for (int i = 0; i < LA0; ++i) {
    const int p = wave + 8 * i, b = min(m0 + 8 * p, M - 1);
    a_src[i] = A + (size_t)b * K + (size_t)ks0 * 128;
    a_off[i] = (uint32_t)min(r8, M - 1 - b) * K + chunk(p);
  }
#pragma unroll
  for (int i = 0; i < LW0; ++i) {
    const int p = wave + 8 * i, b = min(n0 + 8 * p, N - 1);
    w_src[i] = W + (size_t)b * K + (size_t)ks0 * 128;
    w_off[i] = (uint32_t)min(r8, N - 1 - b) * K + chunk(p);
  }
  auto copy = [](const int8_t* src, uint32_t off, char* dst) {
    __builtin_amdgcn_global_load_lds((const void*)(src + off),
                                     (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
  };
  auto copy_once = [](const int8_t* src, uint32_t off, char* dst) {        // 2: nontemporal
    __builtin_amdgcn_global_load_lds((const void*)(src + off),
                                     (__attribute__((address_space(3))) void*)dst, 16, 0, 2);
  };
  const bool once = mt == 1 && n_split == 1;
  auto issue = [&](int v, int stage) {             // K-step v
    const size_t k = (size_t)kmap(min(v, last)) * 128;
    char* dst = smem + stage * STAGE + wave * 1024;
#pragma unroll
    for (int i = 0; i < LA0; ++i)
      if (i < LA1 || !late) copy(a_src[i] + k, a_off[i], dst + i * 8192);
#pragma unroll
    for (int i = 0; i < LW0; ++i)
      if (i < LW1 || !late) {
        if (once) copy_once(w_src[i] + k, w_off[i], dst + BM * 128 + i * 8192);
        else copy(w_src[i] + k, w_off[i], dst + BM * 128 + i * 8192);
      }
  };

  i32x4_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = i32x4_t{0, 0, 0, 0};
  i32x4_t af[AHEAD ? 2 : 1][FM], wf[AHEAD ? 2 : 1][FN];

  const int r16 = lane & 15, g4 = lane >> 4;
  const int frag = r16 * 128 + (((g4 ^ (r16 >> 1)) << 4) ^ (late ? 64 : 0));   // this group's half
  auto read = [&](int stage, i32x4_t (&ar)[FM], i32x4_t (&wr)[FN]) {
    const char* a = smem + stage * STAGE + wm * RW * 128 + frag;
    const char* w = smem + stage * STAGE + BM * 128 + wn * CW * 128 + frag;
#pragma unroll
    for (int j = 0; j < FN; ++j) wr[j] = *(const i32x4_t*)(w + j * 2048);
#pragma unroll
    for (int i = 0; i < FM; ++i) ar[i] = *(const i32x4_t*)(a + i * 2048);
  };
  auto mma = [&](const i32x4_t (&ar)[FM], const i32x4_t (&wr)[FN]) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mma_i8(wr[j], ar[i], acc[i][j]);
    __builtin_amdgcn_s_setprio(0);
  };
  auto wait_reads = [] { __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14)); };   // lgkmcnt(0)
  auto wait_copies = [&] {
    if (late) wait_vmcnt<FLIGHT1>();
    else wait_vmcnt<FLIGHT0>();
  };

  // the groups share the epilogue: the first keeps the fragments i < FM / 2, the
  // second the rest
  constexpr int H = FM / 2;
  TileScales<H, FN> sc;
  if (!part) sc.load(out, m0 + wm * RW + (late ? 16 * H : 0) + r16, n0 + wn * CW + 4 * g4);
#pragma unroll
  for (int j = 0; j < (AHEAD ? R : R - 1); ++j) issue(j, j);
  wait_copies();
  if (!part) sc.hold();
  pp_barrier();
  int st = 0;                                       // stage of K-step v
  if constexpr (AHEAD) {
    read(0, af[0], wf[0]);
    wait_reads();
    pp_barrier();
    auto step = [&](int v, int now) {
      const int next = st == R - 1 ? 0 : st + 1;
      read(next, af[now ^ 1], wf[now ^ 1]);
      issue(v + R, st);
      __builtin_amdgcn_sched_barrier(0);
      mma(af[now], wf[now]);
      __builtin_amdgcn_sched_barrier(0);
      wait_reads();
      wait_copies();
      pp_barrier();
      st = next;
    };
    for (int v = 0; v < nk; v += 2) {
      step(v, 0);
      if (v + 1 < nk) step(v + 1, 1);
    }
  } else {
    if (late) pp_barrier();
    for (int v = 0; v < nk; ++v) {
      read(st, af[0], wf[0]);
      issue(v + R - 1, st == 0 ? R - 1 : st - 1);
      __builtin_amdgcn_sched_barrier(0);
      wait_reads();
      if (late) wait_vmcnt<FLIGHT1>();
      pp_barrier();
      mma(af[0], wf[0]);
      __builtin_amdgcn_sched_barrier(0);
      if (!late) wait_vmcnt<FLIGHT0>();
      pp_barrier();
      st = st == R - 1 ? 0 : st + 1;
    }
    if (!late) pp_barrier();
  }
  wait_vmcnt<0>();                                  // no copy lands in the sums below

  if ((K & 127) && split == n_split - 1) {          // the columns past the last whole K-step
    const int k0 = k_steps * 128 + (late ? 64 : 0);
    if (k0 < K) {
      const int k = k0 + 16 * g4, kc = min(k, K - 16);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        wf[0][j] = *(const i32x4_t*)(W + (size_t)min(n0 + wn * CW + 16 * j + r16, N - 1) * K + kc);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const i32x4_t u = *(const i32x4_t*)(A + (size_t)min(m0 + wm * RW + 16 * i + r16, M - 1) * K + kc);
        af[0][i] = k < K ? u : i32x4_t{0, 0, 0, 0};
      }
      mma(af[0], wf[0]);
    }
  }

  // each group hands the other's half over
  __syncthreads();
  char* mine = smem + (wave * H * FN) * 1024 + lane * 16;
  const char* theirs = smem + ((wave ^ 4) * H * FN) * 1024 + lane * 16;
#pragma unroll
  for (int i = 0; i < H; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) *(i32x4_t*)(mine + (i * FN + j) * 1024) = late ? acc[i][j] : acc[i + H][j];
  __syncthreads();
  i32x4_t sum[H][FN];
#pragma unroll
  for (int i = 0; i < H; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      sum[i][j] = (late ? acc[i + H][j] : acc[i][j]) + *(const i32x4_t*)(theirs + (i * FN + j) * 1024);
  tile_out(sum, sc, m0 + wm * RW + (late ? 16 * H : 0) + r16, n0 + wn * CW, n0 + wn * CW + 4 * g4, split, part,
           ldp, out);
}

// ---------------------------------------------------------------------------
// Sum of split-K partials
// ---------------------------------------------------------------------------
// 4 columns a thread, a row to a workgroup (or several, a grid apart); part is [S, M,
// ldp] with ldp a multiple of 16.  The S loads of a thread are in flight together.
template <int S>
__global__ void __launch_bounds__(256) gemm_i8_sum_kernel(const int* __restrict__ part, int ldp, I8Out out) {
  const int n = 4 * (int)(blockIdx.x * 256 + threadIdx.x);
  SSM_DCHECK(ldp >= out.N);
  if (n >= out.N) return;
  float s[4];
  out.scales4(n, s);
  for (int m = blockIdx.y; m < out.M; m += gridDim.y) {
    i32x4_t v[S];
#pragma unroll
    for (int i = 0; i < S; ++i) v[i] = *(const i32x4_t*)(part + ((size_t)i * out.M + m) * ldp + n);
    const float sm = out.sa[m];
    i32x4_t sum = v[0];
#pragma unroll
    for (int i = 1; i < S; ++i) sum += v[i];
    out.store4(m, n, sum, sm, s);
  }
}

// ---------------------------------------------------------------------------
// Launch choice
// ---------------------------------------------------------------------------
// The kernel, tile and number of K splits that should take the least time; for up to
// I8_FEW_ROWS rows gemm_i8_few_kernel is one of the choices.  A round is a workgroup on
// each of the 256 CUs (one fits a CU).  In a round of w workgroups a K-step of 128
// takes step + fill * w / 256 us, the second part for what the CUs share, but the
// weights come no faster than I8_HBM bytes a us; `fixed` is what a round takes besides.
// The coefficients were fitted to 161 sizes (40-3840 rows, 700-126464 columns, K 1024-18944) times
// 12 tiles times 6 splits, the weights from memory, before grouped_tile_of: there the choice
// took 0.4% more than the best in the mean, 12% at most.  On 70 other sizes drawn over 17-4000
// rows, 500-40000 columns and K 1024-18944 it takes 2.5% more in the mean, above 5% on 14 of them
// and 24% at most (256 x 192 tiles for 2383 x 10205 x 1200, 101 us, where 128 x 256 take 81).  In
// rows of launches, with what lies between them, the kernel for few rows took 7.3 us for
// one row of 4096 x 4096 (64 x 32 tiles 10.3), 12.5 of 4096 x 12288 (15.1), but 27.7 of
// 24576 x 4096 (64 x 96 tiles 20.4), and for 16 rows 8.6, 17.4 and 38.6 (10.1, 15.5, 20.8).
static constexpr int I8_FEW_ROWS = 16;
struct I8Tile {
  int bm, bn;
  float step, fill, fixed;
};
// number, gemm_i8_pp_kernel (1) or gemm_i8_ks_kernel (0), BM, BN, WM, WN, stages; step, fill, fixed
#define I8_TILES(X)                              \
  X(0, 0, 64, 32, 2, 2, 8, 0.18f, 0.02f, 1.9f)   \
  X(1, 0, 64, 64, 2, 2, 8, 0.24f, 0.03f, 2.0f)   \
  X(2, 0, 64, 96, 2, 2, 8, 0.24f, 0.07f, 4.1f)   \
  X(3, 0, 128, 64, 2, 2, 6, 0.29f, 0.10f, 2.4f)  \
  X(4, 0, 128, 96, 2, 2, 5, 0.35f, 0.20f, 3.0f)  \
  X(5, 0, 128, 128, 2, 2, 5, 0.34f, 0.27f, 3.3f) \
  X(6, 0, 128, 160, 2, 2, 4, 0.46f, 0.23f, 3.7f) \
  X(7, 0, 128, 192, 2, 2, 4, 0.44f, 0.30f, 4.3f) \
  X(8, 0, 256, 128, 2, 2, 3, 0.54f, 0.32f, 3.4f) \
  X(9, 1, 128, 256, 2, 4, 2, 0.93f, 0.19f, 2.9f) \
  X(10, 1, 256, 192, 4, 2, 2, 0.76f, 0.60f, 1.5f) \
  X(11, 1, 256, 256, 2, 4, 2, 0.84f, 0.55f, 9.2f)
static constexpr I8Tile I8_TILE[] = {
#define X(I, PP, BM, BN, WM, WN, R, STEP, FILL, FIXED) {BM, BN, STEP, FILL, FIXED},
    I8_TILES(X)
#undef X
};
static constexpr int I8_CUS = 256;
static constexpr int I8_SPLITS[] = {1, 2, 3, 4, 6, 8};
static constexpr float I8_HBM = 6.5e6f;          // bytes a us
static constexpr float I8_SUM_BYTES = 5.0e6f;    // of partials written and read again, a us
static constexpr float I8_SUM_US = 1.8f;         // the launch that adds them

struct I8Plan {
  int tile, split;           // tile -1: gemm_i8_few_kernel
};

static int i8_ldp(int N) { return (N + 15) & ~15; }

// Of gemm_i8_few_kernel: what its workgroups and their weights take, and every row more.
static float i8_few_cost(int M, int N, int K) {
  return (2.0e-4f * N + (float)N * K / 5.2e6f) * (1.f + 0.03f * (M - 1));
}

static float i8_cost(const I8Tile& t, int M, int N, int K, int S) {
  const long wgs = (long)ceil_div(M, t.bm) * ceil_div(N, t.bn) * S, full = wgs / I8_CUS, rem = wgs % I8_CUS;
  const float steps = (float)ceil_div(K / 128, S), weights = (float)N * K / I8_HBM / wgs;
  auto round = [&](long w) {
    const float mma = steps * (t.step + t.fill * w / I8_CUS), hbm = weights * w;
    return (mma > hbm ? mma : hbm) + t.fixed;
  };
  float us = full * round(I8_CUS);
  if (rem) us += round(rem);
  return S > 1 ? us + I8_SUM_US + 8.f * S * M * N / I8_SUM_BYTES : us;
}

static I8Plan i8_plan(int M, int N, int K) {
#ifdef SSM_TUNING
  if (const char* e = getenv("SSM_I8_CFG")) {     // tile:split, for sweeps
    I8Plan p;
    if (sscanf(e, "%d:%d", &p.tile, &p.split) == 2) return p;
  }
#endif
  I8Plan best{-1, 1};
  float least = M <= I8_FEW_ROWS ? i8_few_cost(M, N, K) : 1e30f;
  if (K < 128) return best;                        // the tiles need a whole K-step
  for (int i = 0; i < (int)(sizeof(I8_TILE) / sizeof(I8_TILE[0])); ++i)
    for (int S : I8_SPLITS) {
      if (S > 1 && K / 128 / S < 4) break;
      const float us = i8_cost(I8_TILE[i], M, N, K, S);
      if (us < least) {
        best = {i, S};
        least = us;
      }
    }
  return best;
}

size_t gemm_i8_ws_bytes(int M, int N, int K) {
  if (M == 0 || K % 16) return 0;                  // see gemm_i8: no splits without whole chunks
  const I8Plan p = i8_plan(M, N, K);
  return p.split > 1 ? (size_t)p.split * M * i8_ldp(N) * 4 : 0;
}

template <int PP, int BM, int BN, int WM, int WN, int R>
static void launch_tile(int split, int M, int N, int K, const int8_t* a, const int8_t* w, int* part,
                        const I8Out& out, hipStream_t st) {
  const int mt = ceil_div(M, BM);
  const dim3 grid(mt * ceil_div(N, BN) * split), block(512);
  if constexpr (PP)
    launch((gemm_i8_pp_kernel<BM, BN, WM, WN, R>), grid, block, 0, st, a, w, K, mt, split, part, i8_ldp(N), out);
  else
    launch((gemm_i8_ks_kernel<BM, BN, WM, WN, R, (BM * BN <= 128 * 96)>), grid, block, 0, st, a, w, K, mt, split,
           part, i8_ldp(N), out);
}

hipError_t gemm_i8(int M, int N, int K, const int8_t* a, const float* sa, const int8_t* w,
                   const float* sw, int out_dtype, void* out, void* ws, hipStream_t st) {
  if (M == 0) return hipSuccess;
  const size_t es = out_dtype == 0 ? 4 : 2;
  const I8Out o{out, out_dtype, N % 4 == 0 && ((uintptr_t)out & (4 * es - 1)) == 0, sa, sw, M, N};
  if (K % 16 || (K < 128 && M > I8_FEW_ROWS) || ((uintptr_t)a & 15) || ((uintptr_t)w & 15)) {
    launch(gemm_i8_any_kernel, dim3(ceil_div(N, 64), ceil_div(M, 64)), dim3(256), 0, st, a, w, K, o);
    return hipGetLastError();
  }
  const I8Plan p = i8_plan(M, N, K);
  int* part = p.split > 1 ? (int*)ws : nullptr;
  switch (p.tile) {
#define X(I, PP, BM, BN, WM, WN, R, STEP, FILL, FIXED) \
  case I: launch_tile<PP, BM, BN, WM, WN, R>(p.split, M, N, K, a, w, part, o, st); break;
    I8_TILES(X)
#undef X
    default:
      launch(gemm_i8_few_kernel<4>, dim3(ceil_div(N, 16)), dim3(512), 0, st, a, w, K, o);
  }
  if (part) {
    const auto add = [&](auto kernel) {
      launch(kernel, dim3(ceil_div(N, 1024), M < 65535 ? M : 65535), dim3(256), 0, st, part, i8_ldp(N), o);
    };
    switch (p.split) {                             // I8_SPLITS
      case 2: add(gemm_i8_sum_kernel<2>); break;
      case 3: add(gemm_i8_sum_kernel<3>); break;
      case 4: add(gemm_i8_sum_kernel<4>); break;
      case 6: add(gemm_i8_sum_kernel<6>); break;
      default: add(gemm_i8_sum_kernel<8>); break;
    }
  }
  return hipGetLastError();
}

}  // namespace ssm

// The launch that sizes with aligned operands get, for tests of the choice: rows and
// columns of the tile (16 x 16: gemm_i8_few_kernel, 0 x 0: gemm_i8_any_kernel), K splits.
#ifdef SSM_DEBUG
extern "C" int32_t ssm_debug_gemm_i8_plan(int32_t M, int32_t N, int32_t K, int32_t* out) {
  using namespace ssm;
  if (K % 16 || (K < 128 && M > I8_FEW_ROWS)) {
    out[0] = out[1] = 0;
    out[2] = 1;
    return 0;
  }
  const I8Plan p = i8_plan(M, N, K);
  out[0] = p.tile < 0 ? 16 : I8_TILE[p.tile].bm;
  out[1] = p.tile < 0 ? 16 : I8_TILE[p.tile].bn;
  out[2] = p.split;
  return 0;
}
#endif
