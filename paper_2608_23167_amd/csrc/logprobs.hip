// Log probabilities of given tokens, entropy and the most probable tokens of
// rows of logits, in one pass over the logits.
//
// With m = max x, z = sum exp(x - m) and t = sum (x - m) exp(x - m):
//   log p(v) = (x_v - m) - ln z,   entropy = ln z - t / z.
// (m, z, t) of two parts join by moving both to the larger maximum M: for
// delta = m - M, z -> z e^delta and t -> e^delta (t + z delta).
// Logits of -inf (and the [MASK] id, which counts as one) add nothing.  A row
// with a NaN or a +inf, or with nothing above -inf, has an m that is not
// finite, and m - m makes its log probabilities and entropy NaN.
#include "dcheck.h"
#include "internal.h"
#include "row_stats.h"

namespace ssm {

constexpr float LOG2E = 1.44269504088896340736f;

// The larger of two, NaN if either is (fmaxf drops it).
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// e^y for y <= 0, as v_exp_f32 gives it (one unit in the last place; y log2(e) is
// rounded, which is |y| half units more).
__device__ __forceinline__ float exp_neg(float y) { return __builtin_amdgcn_exp2f(y * LOG2E); }

struct Soft {
  float m, z, t;
};
// A difference to a maximum, no lower than SOFT_LOW: its exponential is 0 in
// float32, and products with a finite number stay finite (0 * -inf is NaN).
// The NaN of -inf - -inf becomes SOFT_LOW too; that of a NaN logit lives on in m.
constexpr float SOFT_LOW = -200.f;
__device__ __forceinline__ float soft_diff(float x, float m) { return fmaxf(x - m, SOFT_LOW); }
__device__ __forceinline__ void soft_move(Soft& a, float m) {     // to the maximum m >= a.m
  const float dl = soft_diff(a.m, m), e = exp_neg(dl);
  a.t = e * (a.t + a.z * dl);
  a.z *= e;
  a.m = m;
}
// Reductions over a wave by data-parallel moves (about 60 clocks; six shuffles
// through LDS hardware take six times that): rows of 16 lanes, then across
// rows, the total in lane 63 and from there, uniform, to all.
template <class Op>
__device__ __forceinline__ int wave_reduce(int v, int identity, Op op) {
#define DPP(ctrl, rows) v = op(v, __builtin_amdgcn_update_dpp(identity, v, ctrl, rows, 0xf, false))
  DPP(0x111, 0xf);   // row_shr 1, 2, 4, 8
  DPP(0x112, 0xf);
  DPP(0x114, 0xf);
  DPP(0x118, 0xf);
  DPP(0x142, 0xa);   // lane 15 of rows 0 and 2 to rows 1 and 3
  DPP(0x143, 0xc);   // lane 31 to rows 2 and 3
#undef DPP
  return __builtin_amdgcn_readlane(v, 63);
}
template <class Op>
__device__ __forceinline__ float wave_reduce_f(float v, float identity, Op op) {
  return __int_as_float(wave_reduce(__float_as_int(v), __float_as_int(identity), [op](int a, int b) {
    return __float_as_int(op(__int_as_float(a), __int_as_float(b)));
  }));
}
__device__ __forceinline__ float wave_top(float v) {               // not of NaN
  return wave_reduce_f(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ int wave_low(int v) {
  return wave_reduce(v, STAT_NONE, [](int a, int b) { return min(a, b); });
}
// The lane below's value (lane 0 keeps its own).
__device__ __forceinline__ int from_below(int v) {
  return __builtin_amdgcn_update_dpp(v, v, 0x138, 0xf, 0xf, false);
}
__device__ __forceinline__ Soft soft_wave(Soft a) {
  const auto add = [](float x, float y) { return x + y; };
  soft_move(a, wave_reduce_f(a.m, -INFINITY, [](float x, float y) { return max_nan(x, y); }));
  return {a.m, wave_reduce_f(a.z, 0.f, add), wave_reduce_f(a.t, 0.f, add)};
}
__device__ __forceinline__ float lane_of(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// The k best of up to 64 lists, best first, list l in lane l: next(j) gives entry
// j < k of this lane's list (value -inf and id STAT_NONE past its end), and
// emit(q, v, i) gets the q-th best in every lane.
template <class Next, class Emit>
__device__ __forceinline__ void merge_lists(int k, Next next, Emit emit) {
  float v;
  int i, at = 0;
  next(0, v, i);
  for (int q = 0; q < k; ++q) {
    const float bv = wave_top(v);
    const int bi = wave_low(v == bv ? i : STAT_NONE);
    emit(q, bv, bi);
    if (i == bi && bi != STAT_NONE) {              // ids are different: one lane's
      if (++at < k) next(at, v, i);
      else { v = -INFINITY; i = STAT_NONE; }
    }
  }
}

// Statistics of one part of a row, as the second launch reads them.
struct Part {
  Soft s;
  float v[STAT_K];
  int id[STAT_K];
};

// Results of a row from its statistics: every lane of a wave calls it, next as in
// merge_lists.
template <typename T, class Next>
__device__ __forceinline__ void row_results(size_t row, const Soft& s, const T* L, int V, int mask_id,
                                            int n_targets, const int32_t* targets, int k, float* lp,
                                            float* entropy, int32_t* top_ids, float* top_lp, Next next) {
  const int lane = threadIdx.x & 63;
  const float spoilt = s.m - s.m;                  // 0, or NaN
  const float lz = logf(s.z);
  if (lane == 0 && entropy) entropy[row] = (lz - s.t / s.z) + spoilt;
  for (int i = lane; i < n_targets; i += 64) {
    const int id = targets[row * n_targets + i];
    float r = __uint_as_float(0x7fc00000u);
    if (id >= 0 && id < V) r = (((id == mask_id ? -INFINITY : ldf(L + id)) - s.m) - lz) + spoilt;
    lp[row * n_targets + i] = r;
  }
  merge_lists(k, next, [&](int q, float v, int i) {
    SSM_DCHECK(i == STAT_NONE || (i >= 0 && i < V && i != mask_id));
    if (lane == 0) {
      top_ids[row * k + q] = i == STAT_NONE ? -1 : i;
      top_lp[row * k + q] = i == STAT_NONE ? -INFINITY : ((v - s.m) - lz) + spoilt;
    }
  });
}

// Bound by the vector ALUs and memory alike: 12.7 VALU instructions a column keep the
// SIMDs 82% busy while 3840 rows of 126464 bfloat16 logits are read at 5.1 TB/s (190 us);
// 54 registers leave room for 7 waves a SIMD, which the loads need (at 127 registers
// and 4 waves 252 us).
// One workgroup of NW waves per part of a row: columns [p chunk, (p + 1) chunk)
// of row blockIdx.x / parts.  A wave takes tiles of 64 lanes x 16 columns,
// 16-byte loads, the next tile's in flight while one is worked on; what lies
// before the first aligned address and past the last whole tile is loaded
// singly.  Per tile a lane takes its maximum, moves (m, z, t) there and adds its
// 16 exponentials.
// The wave's k best so far sit in its lanes 0 .. k - 1; the bar is the k-th.  A
// tile is looked through only if some lane's maximum is above the bar (its ids are
// above those before it, so an equal value never displaces), which for values in
// no order happens k ln(tiles) times a wave.  Where more than k lanes are above
// it, as in the first tile or in rising rows, the k-th largest of the lanes'
// maxima is a floor for this tile's candidates.  Each candidate then goes to its
// place in the list by value and id; one that finds none takes along all that
// are no better than the k-th (3840 rows of 126464 bfloat16 logits, k = 8: random 190-195 us
// and 175 with k = 0; all equal 180, without this 867; rising 915, without 3637).
template <typename T, int NW>
__global__ void __launch_bounds__(64 * NW) logprobs_kernel(
    const T* __restrict__ logits, int V, int mask_id, int n_targets,
    const int32_t* __restrict__ targets, int k, int parts, int chunk, float* __restrict__ lp,
    float* __restrict__ entropy, int32_t* __restrict__ top_ids, float* __restrict__ top_lp,
    Part* __restrict__ out) {
  constexpr int E = 16, VE = 16 / sizeof(T), NL = E / VE, TILE = 64 * E;
  __shared__ Part sh[NW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const size_t row = blockIdx.x / parts;
  const int p = blockIdx.x % parts;
  const T* L = logits + row * V;
  const int lo = p * chunk, hi = min(V, lo + chunk);
  SSM_DCHECK(k <= STAT_K && lo < hi);
  const int skew = (int)(((uintptr_t)(L + lo) & 15) / sizeof(T));
  const int body = min(hi, lo + (skew ? VE - skew : 0));       // first aligned column
  const int tiles = (hi - body) / TILE, tail = body + tiles * TILE;

  Soft s{-INFINITY, 0.f, 0.f};
  float bv = -INFINITY;                            // lane q < k: the q-th best
  int bi = STAT_NONE;
  float bar = k > 0 ? -INFINITY : INFINITY;        // the k-th best's value

  // x[e]: column first + off(e) of this lane, rising with e; lane l's first is
  // base + l step
  auto work = [&](float (&x)[E], int base, int end, int step, auto off) {
    const int first = base + lane * step;
    if (mask_id >= base && mask_id < end) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (off(e) == mask_id - first) x[e] = -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < E; ++e) top = max_nan(top, x[e]);
    soft_move(s, max_nan(s.m, top));
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float y = soft_diff(x[e], s.m), ex = exp_neg(y);
      s.z += ex;
      s.t += ex * y;
    }
    if (__ballot(!(top <= bar)) == 0) return;      // NaN goes on
    if (__any(top != top)) {                       // NaN logits are not listed
      top = -INFINITY;
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, x[e]);
    }
    float floor = bar;
    if (__popcll(__ballot(top > bar)) > k) {
      for (int q = 0; q < k; ++q) {
        floor = wave_top(top);
        if (lane == __ffsll((unsigned long long)__ballot(top == floor)) - 1) top = -INFINITY;
      }
    }
    const float over = bar;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      unsigned long long found = __ballot(x[e] > over && x[e] >= floor);
      while (found) {
        const int l = __ffsll(found) - 1;
        found &= found - 1;
        const float v = lane_of(x[e], l);
        const int id = base + l * step + off(e);
        const int place = __popcll(__ballot(lane < k && stat_better(bv, bi, v, id)));
        if (place >= k) {                          // with it go all that are no better than the k-th
          const float kv = lane_of(bv, k - 1);
          const int ki = __builtin_amdgcn_readlane(bi, k - 1);
          found &= __ballot(stat_better(x[e], base + lane * step + off(e), kv, ki));
          continue;
        }
        const float uv = __int_as_float(from_below(__float_as_int(bv)));
        const int ui = from_below(bi);
        if (lane == place) { bv = v; bi = id; }
        else if (lane > place) { bv = uv; bi = ui; }
      }
    }
    if (k > 0) bar = lane_of(bv, k - 1);
  };
  auto single = [&](int from, int to) {            // at most TILE columns, loaded singly
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int v = from + 64 * e + lane;
      x[e] = v < to ? ldf(L + v) : -INFINITY;
    }
    work(x, from, to, 1, [](int e) { return 64 * e; });
  };
  auto load = [&](int tile, u32x4_t (&r)[NL]) {
    const T* src = L + body + tile * TILE + lane * VE;
#pragma unroll
    for (int j = 0; j < NL; ++j) r[j] = *(const u32x4_t*)(src + j * 64 * VE);
  };

  if (wave == 0 && body > lo) single(lo, body);
  if (wave < tiles) {
    u32x4_t r[NL];
    load(wave, r);
    for (int i = wave; i < tiles; i += NW) {
      float x[E];
#pragma unroll
      for (int j = 0; j < NL; ++j)
#pragma unroll
        for (int e = 0; e < VE; ++e) x[j * VE + e] = ldf((const T*)&r[j] + e);
      load(min(i + NW, tiles - 1), r);
      const int base = body + i * TILE;
      work(x, base, base + TILE, VE, [](int e) { return (e / VE) * 64 * VE + e % VE; });
    }
  }
  if (wave == tiles % NW && tail < hi) single(tail, hi);

  s = soft_wave(s);
  if (lane == 0) sh[wave].s = s;
  if (lane < STAT_K) { sh[wave].v[lane] = bv; sh[wave].id[lane] = bi; }
  __syncthreads();
  if (wave != 0) return;
  s = soft_wave(lane < NW ? sh[lane].s : Soft{-INFINITY, 0.f, 0.f});
  auto next = [&](int j, float& v, int& i) {
    v = lane < NW ? sh[lane].v[j] : -INFINITY;
    i = lane < NW ? sh[lane].id[j] : STAT_NONE;
  };
  if (parts == 1) {
    row_results(row, s, L, V, mask_id, n_targets, targets, k, lp, entropy, top_ids, top_lp, next);
  } else {
    Part* o = out + blockIdx.x;
    if (lane == 0) o->s = s;
    merge_lists(k, next, [&](int q, float v, int i) {
      if (lane == 0) { o->v[q] = v; o->id[q] = i; }
    });
  }
}

// One wave per row: joins the statistics of its parts (at most 64).
template <typename T>
__global__ void __launch_bounds__(64) logprobs_join_kernel(
    const Part* __restrict__ in, int parts, const T* __restrict__ logits, int V, int mask_id,
    int n_targets, const int32_t* __restrict__ targets, int k, float* __restrict__ lp,
    float* __restrict__ entropy, int32_t* __restrict__ top_ids, float* __restrict__ top_lp) {
  const int lane = threadIdx.x;
  const size_t row = blockIdx.x;
  SSM_DCHECK(parts <= 64);
  const Part* mine = in + row * parts + lane;
  Soft s{-INFINITY, 0.f, 0.f};
  if (lane < parts) s = mine->s;
  s = soft_wave(s);
  row_results(row, s, logits + row * V, V, mask_id, n_targets, targets, k, lp, entropy, top_ids, top_lp,
              [&](int j, float& v, int& i) {
    v = lane < parts ? mine->v[j] : -INFINITY;
    i = lane < parts ? mine->id[j] : STAT_NONE;
  });
}

// Waves of a workgroup, and parts of a row.
//  * Up to 2048 columns a wave takes a row (at most two tiles).
//  * Up to 256 rows, a workgroup of 16 waves on each CU takes a whole row where that is
//    sooner than parts: 6 us + 0.113 us a thousand columns against 9.5 us (two launches) +
//    0.68 us a million of all rows' columns.  Measured, float32: one row of 16384 8.0
//    against 10.5 us, of 65536 14.9 against 10.7; 120 rows of 32768 12.8 against 14.7;
//    240 rows of 126464 27.6 against 31.6.
//  * Else workgroups of 4 waves; whole rows once there are 385, below in as many parts as
//    768 workgroups, 3 to a CU, have rows, of at least a tile to each wave.  A part is a
//    multiple of 4096 columns, a tile to each wave, so there are fewer parts than that
//    where V / 4096 is near their number, and the last holds what is left: one row of
//    152064 columns is 18 parts of 8192 and one of 4608, 120 rows of 126464 are 5 parts
//    of 24576 and one of 3584 each.  120 rows of 126464 in 6 parts 23.9 us, in 8 23.5 (k = 5,
//    which is 10 us of it: 13.8 with k = 0); 400 rows whole 43.4, in 2 parts 46.9.
struct LogprobsPlan {
  int waves, parts, chunk;
};
static LogprobsPlan logprobs_plan(int rows, int V) {
  constexpr int LEAST = 4096, WORKGROUPS = 768, CUS = 256;
  if (V <= 2048) return {1, 1, V};
  if (V > LEAST && rows <= CUS && V * (113.0 - 0.68 * rows) < 3.5e6) return {16, 1, V};
  int parts = WORKGROUPS / rows;
  if (parts > V / LEAST) parts = V / LEAST;
  if (parts > 64) parts = 64;
  if (parts <= 1) return {4, 1, V};
  const int chunk = ceil_div(ceil_div(V, parts), LEAST) * LEAST;
  return {4, ceil_div(V, chunk), chunk};
}

size_t token_logprobs_ws_bytes(int rows, int V, int k) {
  (void)k;
  if (rows == 0) return 0;
  const LogprobsPlan p = logprobs_plan(rows, V);
  return p.parts > 1 ? (size_t)rows * p.parts * sizeof(Part) : 0;
}

hipError_t launch_token_logprobs(int dtype, int rows, int V, const void* logits, int mask_id,
                                 int n_targets, const int32_t* targets, int k, float* lp,
                                 float* entropy, int32_t* top_ids, float* top_lp, void* ws,
                                 hipStream_t st) {
  if (rows == 0) return hipSuccess;
  const LogprobsPlan p = logprobs_plan(rows, V);
  Part* part = (Part*)ws;
  auto go = [&](auto* x) {
    using T = std::remove_cv_t<std::remove_pointer_t<decltype(x)>>;
    const auto rows_by = [&](auto kernel) {
      return launch_rows(rows, 64 * p.waves * p.parts, 1, [&](int at, int n) {
        const size_t r = at;
        launch(kernel, dim3(n * p.parts), dim3(64 * p.waves), 0, st, x + r * V, V, mask_id, n_targets,
               targets ? targets + r * n_targets : targets, k, p.parts, p.chunk, lp ? lp + r * n_targets : lp,
               entropy ? entropy + r : entropy, top_ids ? top_ids + r * k : top_ids, top_lp ? top_lp + r * k : top_lp,
               part);                              // rows in parts are few: one launch
      });
    };
    hipError_t e;
    if (p.waves == 1) e = rows_by(logprobs_kernel<T, 1>);
    else if (p.waves == 16) e = rows_by(logprobs_kernel<T, 16>);
    else e = rows_by(logprobs_kernel<T, 4>);
    if (e != hipSuccess || p.parts == 1) return e;
    launch(logprobs_join_kernel<T>, dim3(rows), dim3(64), 0, st, part, p.parts, x, V, mask_id,
           n_targets, targets, k, lp, entropy, top_ids, top_lp);
    return hipGetLastError();
  };
  if (dtype == 0) return go((const float*)logits);
  if (dtype == 1) return go((const bf16_t*)logits);
  return go((const f16_t*)logits);
}

}  // namespace ssm
