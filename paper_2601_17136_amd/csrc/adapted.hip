// A projection that the rows share, with a low-rank adapter for each row:
//   y_i = w x_i + up_g t_i,  t_i = f_g down_g x_i,  g = ids_i,
// and its gradient by x and by the adapters:
//   dx_i = w^T dy_i + down_g^T u_i,  u_i = f_g up_g^T dy_i,
//   ddown_g = sum_i u_i x_i^T,  dup_g = sum_i dy_i t_i^T.
//
// The rows are sorted by adapter (a stable order, so that sums have one), and t
// and u lie in that order, in fp32.  With w and the adapters turned, dx is the
// same operator as y: the kernels know one projection.
//
//   plan       order of the rows, where each adapter's begin
//   turn       (gradient) w^T, up^T, down^T
//   shrink     t, u: 16 or 32 rows of one adapter a workgroup
//   project    w's product with the adapters' part added before the one rounding:
//              direct, from the rows as they are (at most 64 rows, or little work),
//              or in tiles of the sorted rows (head_tile.h; fp32: pair_tile.h)
//   outer      (gradient) the adapters' gradients of a piece of an adapter's rows
//   join       their sums over the pieces
//
// t and u are used in fp32 or, beside 16-bit matrices, as three parts of 16 bits, all of
// their 24 bits: their products are few beside w's.  A row by itself takes one launch, at
// most 64 rows two.
#include <algorithm>
#include <cmath>

#include "model_ops.h"
#include "pair_tile.h"
#include "wave_rows.h"

namespace kkm {

namespace {

// Where the rows of each adapter are.  Bucket `adapters` holds the rows without
// one, the next one those whose id is none of them.
struct RowPlan {
  int32_t *order, *place, *bucket;  // row at a place, place of a row, bucket of a place
  int32_t *start;                   // adapters + 3: a bucket's first place
  int32_t *tile, *piece;            // adapters + 1: its first tile of `shrink`, its first piece
};

// The rows are cut into runs of a workgroup (`run` rows), whose wavefronts count and
// then place theirs, 64 at a time.  More than one run: a launch counts them first, and
// each workgroup sums what lies before its own.  20000 rows of 8 adapters by one
// workgroup 31 us, by 20 in two launches 5 and 8, of which most is the launches.
constexpr int kPlanWaves = 16, kPlanAhead = 8;  // ids of so many 64 rows are read at a time
__device__ inline int bucket_of(int g, int adapters) { return g < 0 ? adapters : g >= adapters ? adapters + 1 : g; }
// The lanes whose b is this lane's (none of b < 0).
__device__ inline unsigned long long alike(int b, int bits) {
  unsigned long long same = __ballot(b >= 0);
  for (int k = 0; k < bits; ++k) {
    const unsigned long long set = __ballot(b >> k & 1);
    same &= b >> k & 1 ? set : ~set;
  }
  return b >= 0 ? same : 0;
}
__device__ inline bool leads(unsigned long long same) {
  return same && __ffsll((unsigned long long)same) - 1 == (int)(threadIdx.x & 63);
}

__global__ __launch_bounds__(kPlanWaves * 64) void count_kernel(const int32_t* __restrict__ ids, int64_t n, int adapters,
                                                                int64_t run, int bits, int* __restrict__ counts) {
  extern __shared__ int cnt[];  // [nb]
  const int nb = adapters + 2;
  for (int e = threadIdx.x; e < nb; e += kPlanWaves * 64) cnt[e] = 0;
  __syncthreads();
  const int64_t lo = blockIdx.x * run, hi = min(lo + run, n);
  for (int64_t i0 = lo; i0 < hi; i0 += kPlanWaves * 64) {
    const int b = i0 + threadIdx.x < hi ? bucket_of(ids[i0 + threadIdx.x], adapters) : -1;
    const unsigned long long same = alike(b, bits);
    if (leads(same)) atomicAdd(cnt + b, __popcll(same));
  }
  __syncthreads();
  for (int e = threadIdx.x; e < nb; e += kPlanWaves * 64) counts[(int64_t)blockIdx.x * nb + e] = cnt[e];
}

__global__ __launch_bounds__(kPlanWaves * 64) void plan_kernel(const int32_t* __restrict__ ids, int64_t n, int adapters,
                                                               int64_t run, const int* __restrict__ counts, int bits,
                                                               int tile, int piece, RowPlan q) {
  extern __shared__ int cnt[];  // [kPlanWaves][nb]
  __shared__ int sums[kPlanWaves][3];
  const int nb = adapters + 2, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int e = threadIdx.x; e < kPlanWaves * nb; e += kPlanWaves * 64) cnt[e] = 0;
  __syncthreads();
  const int64_t from = blockIdx.x * run, to = min(from + run, n);
  const int64_t per = (run / kPlanWaves + 63) / 64 * 64, lo = min(from + wave * per, to), hi = min(lo + per, to);
  volatile int* own = cnt + wave * nb;
  int b8[kPlanAhead];
  auto read = [&](int64_t i0) {
#pragma unroll
    for (int u = 0; u < kPlanAhead; ++u)
      b8[u] = i0 + u * 64 + lane < hi ? bucket_of(ids[i0 + u * 64 + lane], adapters) : -1;
  };
  for (int64_t i0 = lo; i0 < hi; i0 += 64 * kPlanAhead) {
    read(i0);
#pragma unroll
    for (int u = 0; u < kPlanAhead; ++u) {
      if (i0 + u * 64 >= hi) break;
      const unsigned long long same = alike(b8[u], bits);
      if (leads(same)) own[b8[u]] += __popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
  }
  __syncthreads();
  // first places: by bucket, then by run and wavefront; tiles and pieces likewise
  int first = 0, tiles = 0, pieces = 0;  // of the buckets before this round's
  for (int b0 = 0; b0 < nb; b0 += kPlanWaves * 64) {
    const int b = b0 + threadIdx.x;
    int total = 0, before = 0;
    if (b < nb) {
      if (counts)
#pragma unroll 8
        for (int r = 0; r < (int)gridDim.x; ++r) {
          const int c = counts[(int64_t)r * nb + b];
          total += c;
          if (r < (int)blockIdx.x) before += c;
        }
      else
        for (int w = 0; w < kPlanWaves; ++w) total += cnt[w * nb + b];
    }
    int v[3] = {total, b < adapters ? (total + tile - 1) / tile : 0, b < adapters ? (total + piece - 1) / piece : 0};
    int s[3] = {v[0], v[1], v[2]};
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int t = __shfl_up(s[k], o, 64);
        if (lane >= o) s[k] += t;
      }
    if (lane == 63)
      for (int k = 0; k < 3; ++k) sums[wave][k] = s[k];
    __syncthreads();
    int base[3] = {first, tiles, pieces}, all[3] = {first, tiles, pieces};
    for (int w = 0; w < kPlanWaves; ++w)
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        if (w < wave) base[k] += sums[w][k];
        all[k] += sums[w][k];
      }
    if (b < nb) {
      int at = base[0] + s[0] - v[0];
      if (blockIdx.x == 0) {
        q.start[b] = at;
        if (b <= adapters) {
          q.tile[b] = base[1] + s[1] - v[1];
          q.piece[b] = base[2] + s[2] - v[2];
        }
      }
      at += before;
      for (int w = 0; w < kPlanWaves; ++w) {
        const int c = cnt[w * nb + b];
        cnt[w * nb + b] = at;
        at += c;
      }
    }
    first = all[0], tiles = all[1], pieces = all[2];
    __syncthreads();
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) q.start[nb] = first;
  for (int64_t i0 = lo; i0 < hi; i0 += 64 * kPlanAhead) {
    read(i0);
#pragma unroll
    for (int u = 0; u < kPlanAhead; ++u) {
      const int64_t i = i0 + u * 64 + lane;
      if (i0 + u * 64 >= hi) break;
      const int b = b8[u];
      const bool here = b >= 0;
      const unsigned long long same = alike(b, bits);
      const int rank = __popcll(same & ((1ull << lane) - 1));
      int at = 0;
      if (here) at = own[b] + rank;
      __builtin_amdgcn_wave_barrier();
      if (here && rank == 0) own[b] = at + __popcll(same);
      __builtin_amdgcn_wave_barrier();
      if (here) {
        q.order[at] = (int32_t)i;
        q.place[i] = at;
        q.bucket[at] = b;
      }
    }
  }
}

// The bucket that unit `at` of a list of first units belongs to.
__device__ inline int owner(const int32_t* __restrict__ first, int count, int at) {
  int lo = 0, hi = count;  // first[lo] <= at < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first[mid] <= at)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// ------------------------------------------------------------------ turned copies

// dst[c][r] = src[r][c] of `count` matrices, 64 x 64 at a time.  4096 x 4096 and 16
// adapters of 32 ranks on both sides, bfloat16: 17 us, 5.1 TB/s read and written.
struct TurnJob {
  const void* src;
  int64_t ld, rows, cols, ldd;
  void* dst;
  int64_t blocks, bx, per;  // of the job; across the columns; of a matrix
};
struct TurnJobs {
  TurnJob j[3];
};
template <typename T>
__global__ __launch_bounds__(256) void turn_kernel(TurnJobs jobs) {
  constexpr int VEC = kVec<T>, LANES = 64 / VEC, PASS = 256 / LANES;  // lanes of a row, rows of a pass
  __shared__ T tile[64][64 + 4 / sizeof(T)];
  const int64_t total = jobs.j[0].blocks + jobs.j[1].blocks + jobs.j[2].blocks;
  for (int64_t unit = blockIdx.x; unit < total; unit += gridDim.x) {
    int64_t g = unit;
    int k = 0;
    while (k < 2 && g >= jobs.j[k].blocks) g -= jobs.j[k++].blocks;
    const TurnJob& j = jobs.j[k];
    const int64_t mat = g / j.per, b = g - mat * j.per, c0 = b % j.bx * 64, r0 = b / j.bx * 64;
    const T* src = (const T*)j.src + mat * j.rows * j.ld + c0;
    T* dst = (T*)j.dst + mat * j.cols * j.ldd;
    const int wide = (int)min((int64_t)64, j.cols - c0), col = threadIdx.x % LANES * VEC;
#pragma unroll
    for (int o = 0; o < 64; o += PASS) {
      const int r = o + threadIdx.x / LANES;
      const bool use = r0 + r < j.rows;
      const raw_vec<T> v = load_raw(src + (use ? r0 + r : 0) * j.ld, col, use ? wide : 0);
#pragma unroll
      for (int e = 0; e < VEC; ++e) tile[r][col + e] = v[e];
    }
    __syncthreads();
    const int high = (int)min((int64_t)64, j.ldd - r0);  // (rows past the last are zero)
#pragma unroll
    for (int o = 0; o < 64; o += PASS) {
      const int c = o + threadIdx.x / LANES, r = threadIdx.x % LANES * VEC;
      if (c >= wide || r >= high) continue;
      raw_vec<T> v;
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = tile[r + e][c];
      T* to = dst + (c0 + c) * j.ldd + r0 + r;
      if (r + VEC <= high)
        *(any_vec<T>*)to = v;
      else
        for (int e = 0; e < high - r; ++e) to[e] = v[e];
    }
    __syncthreads();
  }
}

// The power of two that brings a largest entry to 2^14 .. 2^15; 0 of zero, infinities and NaN.
__device__ inline int power_for(float top) {
  if (!(top > 0.f && top < INFINITY)) return 0;
  int e;
  (void)frexpf(top, &e);
  return 15 - e;
}

// ------------------------------------------------------------------ t and u

struct ShrinkJob {
  const void* x;
  int64_t ldx;
  int d;
  const void* low;  // adapters x rank x d, rows lowld apart
  int64_t lowld;
  float* t;         // n x rank padded to 16 RB, in sorted order
  int* exps;        // a row's power of two, or null
  unsigned blocks;
};
struct ShrinkJobs {
  ShrinkJob j[2];
  int adapters, rank;
  const float* factor;
  RowPlan plan;
};

// NB x 16 rows of an adapter by its rank; the wavefronts share the width and join in
// LDS.  Bound by reading the rows: 8192 bfloat16 rows of 4096, 32 ranks of 16 adapters
// 25 us, 2.6 TB/s, both sides of the gradient 41, 3.3 TB/s (45 a call on average with
// lanes of 16 rows each).
template <typename T, class S>
__global__ __launch_bounds__(S::WV * 64) void shrink_kernel(ShrinkJobs q) {
  constexpr int R = S::NA * 16, N = S::NB * 16;
  static_assert(S::WV * N * (R + 1) * 4 <= S::lds_bytes, "the sums' place");
  __shared__ __attribute__((aligned(1024))) char lds[S::lds_bytes];
  const bool second = blockIdx.x >= q.j[0].blocks;
  const ShrinkJob& j = q.j[second];
  const int at = blockIdx.x - (second ? q.j[0].blocks : 0u);
  if (at >= q.plan.tile[q.adapters]) return;
  const int g = __builtin_amdgcn_readfirstlane(owner(q.plan.tile, q.adapters, at));
  const int p0 = q.plan.start[g] + N * (at - q.plan.tile[g]), p1 = min(p0 + N, q.plan.start[g + 1]);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15,
            k4 = lane >> 4;
  floatx4 acc[S::NA][S::NB];
#pragma unroll
  for (int i = 0; i < S::NA; ++i)
#pragma unroll
    for (int n = 0; n < S::NB; ++n) acc[i][n] = floatx4{0.f, 0.f, 0.f, 0.f};
  wave_rows<T, S>([&](int r) { return (const T*)j.low + ((int64_t)g * q.rank + min(r, q.rank - 1)) * j.lowld; },
                  [&](int r) { return (const T*)j.x + (int64_t)q.plan.order[min(p0 + r, p1 - 1)] * j.ldx; }, j.d, lds, acc);
  __syncthreads();
  float (*zs)[N][R + 1] = (float (*)[N][R + 1])lds;
#pragma unroll
  for (int i = 0; i < S::NA; ++i)
#pragma unroll
    for (int n = 0; n < S::NB; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) zs[wave][n * 16 + l16][i * 16 + 4 * k4 + r] = acc[i][n][r];
  __syncthreads();
  const float f = q.factor ? q.factor[g] : 1.f;
  for (int e = threadIdx.x; e < N * R; e += S::WV * 64) {
    const int row = e / R, c = e % R;
    if (p0 + row >= p1) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < S::WV; w += 4)
      v += (zs[w][row][c] + zs[w + 1][row][c]) + (zs[w + 2][row][c] + zs[w + 3][row][c]);
    const float o = c < q.rank ? v * f : 0.f;
    j.t[(int64_t)(p0 + row) * R + c] = o;
    zs[0][row][c] = o;
  }
  if (!j.exps) return;
  __syncthreads();
  if (threadIdx.x >= N || p0 + (int)threadIdx.x >= p1) return;
  float top = 0.f;
  for (int c = 0; c < R; ++c) top = fmaxf(top, fabsf(zs[0][threadIdx.x][c]));
  j.exps[p0 + threadIdx.x] = power_for(top);
}

// Few rows, in their own order (no plan): a workgroup a row, its wavefronts the
// adapter's rows of the rank in turn.  32 rows of 4096, each its own 16 ranks: 6 us.
template <typename T>
__global__ __launch_bounds__(1024) void shrink_rows_kernel(const T* __restrict__ x, int64_t ldx, int d,
                                                           const T* __restrict__ down, int adapters, int rank, int R,
                                                           const int32_t* __restrict__ ids,
                                                           const float* __restrict__ factor, float* __restrict__ t) {
  constexpr int VEC = kVec<T>;
  const int64_t row = blockIdx.x;
  const int g = ids[row], lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (g < 0 || g >= adapters) return;
  const float f = factor ? factor[g] : 1.f;
  const T* xr = x + row * ldx;
  for (int r = wave; r < R; r += 16) {
    float s = 0.f;
    if (r < rank) {
      const T* a = down + ((int64_t)g * rank + r) * d;
#pragma unroll 4
      for (int k = lane * VEC; k < d; k += 64 * VEC) {
        float u[VEC], v[VEC];
        load_part(xr, k, d, u);
        load_part(a, k, d, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s = fmaf(u[e], v[e], s);
      }
      s = wave_sum(s);
    }
    if (lane == 0) t[row * R + r] = r < rank ? s * f : 0.f;  // (zero from rank on, at any f)
  }
}

// ------------------------------------------------------------------ the projection

struct ProjectArgs {
  const void* x;
  int64_t ldx, n;
  int d;
  const void* w;
  int64_t ldw;
  int m;
  int adapters, rank;
  const void* up;  // adapters x m x rank, rows uld apart
  int64_t uld;
  const float* t;  // n x R, in sorted order
  const int* texp; // binary16's tiles: a row's power of two
  int R;
  RowPlan plan;
  const int32_t* ids;
  void* y;
  int64_t ldy;
};

// NA x 16 columns of y by NB x 16 rows, from the rows as they are; the wavefronts share
// the width and join in LDS.  Bound by reading w, and by the rows, which every workgroup
// reads: 32 rows of 4096 by 4096, 32 adapters of 16, bfloat16: 10.5 us, 3.6 TB/s.
template <typename T, class S>
__global__ __launch_bounds__(S::WV * 64) void direct_kernel(ProjectArgs a) {
  constexpr int C = S::NA * 16, N = S::NB * 16, THREADS = S::WV * 64, EACH = (C * N + THREADS - 1) / THREADS,
                VEC = kVec<T>, AHEAD = EACH <= 2 ? 2 : 0;
  static_assert(S::WV * N * (C + 1) * 4 <= S::lds_bytes, "the sums' place");
  __shared__ __attribute__((aligned(1024))) char lds[S::lds_bytes];
  const unsigned across = (unsigned)((a.m + C - 1) / C);
  const int64_t v0 = (int64_t)(blockIdx.x % across) * C, t0 = (int64_t)(blockIdx.x / across) * N;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15,
            k4 = lane >> 4;
  // the adapters' part of this thread's entries, as far as it can be had before t
  int adapter[EACH], place[EACH];
  raw_vec<T> ahead[EACH][AHEAD + 1];
  auto up_of = [&](int o, int64_t col) { return (const T*)a.up + ((int64_t)adapter[o] * a.m + col) * a.uld; };
#pragma unroll
  for (int o = 0; o < EACH; ++o) {
    const int e = o * THREADS + threadIdx.x;
    const int64_t row = t0 + e / C, col = v0 + e % C;
    const bool here = e < C * N && row < a.n && col < a.m;
    adapter[o] = here ? a.ids[row] : -1;
    place[o] = here ? a.plan.place ? a.plan.place[row] : (int)row : 0;
    const bool has = adapter[o] >= 0 && adapter[o] < a.adapters;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) ahead[o][i] = load_raw(has ? up_of(o, col) : (const T*)a.up, i * VEC, has ? a.rank : 0);
  }
  floatx4 acc[S::NA][S::NB];
#pragma unroll
  for (int i = 0; i < S::NA; ++i)
#pragma unroll
    for (int n = 0; n < S::NB; ++n) acc[i][n] = floatx4{0.f, 0.f, 0.f, 0.f};
  wave_rows<T, S>([&](int r) { return (const T*)a.w + min(v0 + r, (int64_t)a.m - 1) * a.ldw; },
                  [&](int r) { return (const T*)a.x + min(t0 + r, a.n - 1) * a.ldx; }, a.d, lds, acc);
  __syncthreads();
  float (*zs)[N][C + 1] = (float (*)[N][C + 1])lds;
#pragma unroll
  for (int i = 0; i < S::NA; ++i)
#pragma unroll
    for (int n = 0; n < S::NB; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) zs[wave][n * 16 + l16][i * 16 + 4 * k4 + r] = acc[i][n][r];
  __syncthreads();
#pragma unroll
  for (int o = 0; o < EACH; ++o) {
    const int e = o * THREADS + threadIdx.x, c = e % C, t = e / C;
    const int64_t col = v0 + c, row = t0 + t;
    if (e >= C * N || col >= a.m || row >= a.n) continue;
    float low = 0.f;
    if (adapter[o] >= a.adapters) {
      low = __builtin_nanf("");
    } else if (adapter[o] >= 0) {
      const float* tr = a.t + (int64_t)place[o] * a.R;
      auto add = [&](const raw_vec<T>& b, int k) {  // (t is zero from rank on)
#pragma unroll
        for (int i = 0; i < VEC; ++i) low = fmaf(tr[k + i], (float)b[i], low);
      };
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (i * VEC < a.rank) add(ahead[o][i], i * VEC);
      for (int k = AHEAD * VEC; k < a.rank; k += VEC) add(load_raw(up_of(o, col), k, a.rank), k);
    }
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < S::WV; w += 4) v += (zs[w][t][c] + zs[w + 1][t][c]) + (zs[w + 2][t][c] + zs[w + 3][t][c]);
    ((T*)a.y)[row * a.ldy + col] = (T)(v + low);
  }
}

// A row by itself, of a rank of at most 16: its adapter's rows of `down` stand beside 16
// rows of w, so that t needs no launch of its own.  784 fp32 to 64, rank 8: a call 9.1 us where two
// launches took 12.8.
template <typename T>
__global__ __launch_bounds__(512) void one_row_kernel(ProjectArgs a, const T* __restrict__ down,
                                                      const float* __restrict__ factor) {
  using S = WaveRows<T, 2, 1, 8>;
  __shared__ __attribute__((aligned(1024))) char lds[S::lds_bytes];
  const int64_t v0 = (int64_t)blockIdx.x * 16;
  const int g = a.ids[0], lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool has = g >= 0 && g < a.adapters;
  const T* low = has ? down + (int64_t)g * a.rank * a.d : nullptr;
  const float f = has && factor ? factor[g] : 1.f;
  floatx4 acc[2][1] = {{floatx4{0.f, 0.f, 0.f, 0.f}}, {floatx4{0.f, 0.f, 0.f, 0.f}}};
  wave_rows<T, S>(
      [&](int r) {
        return r < 16 || !has ? (const T*)a.w + min(v0 + (r & 15), (int64_t)a.m - 1) * a.ldw
                              : low + (int64_t)min(r - 16, a.rank - 1) * a.d;
      },
      [&](int) { return (const T*)a.x; }, a.d, lds, acc);
  __syncthreads();
  float (*zs)[32] = (float (*)[32])lds;  // [wavefront][16 of w, 16 of the rank]
  if ((lane & 15) == 0)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) zs[wave][i * 16 + 4 * (lane >> 4) + r] = acc[i][0][r];
  __syncthreads();
  auto sum = [&](int c) {
    return ((zs[0][c] + zs[1][c]) + (zs[2][c] + zs[3][c])) + ((zs[4][c] + zs[5][c]) + (zs[6][c] + zs[7][c]));
  };
  const int64_t col = v0 + threadIdx.x;
  if (threadIdx.x >= 16 || col >= a.m) return;
  float v = sum(threadIdx.x);
  if (has) {
    const T* up = (const T*)a.up + ((int64_t)g * a.m + col) * a.rank;
    float low_part = 0.f;
    for (int k = 0; k < a.rank; ++k) low_part = fmaf(sum(16 + k) * f, (float)up[k], low_part);
    v += low_part;
  } else if (g >= a.adapters) {
    v = __builtin_nanf("");
  }
  ((T*)a.y)[col] = (T)v;
}

// A tile of the sorted rows; the adapters of each 32 rows one after another.  Their
// products go into sums of their own, of which a row takes its adapter's: what
// another adapter holds, were it NaN, does not reach it.  Bound by the matrix cores: 8192
// bfloat16 rows of 4096 by 4096 with 32 ranks 256 us, 1.07 PFLOP/s; fp32, 20000 of
// 784 by 1024 130 us, 247 TFLOP/s of fp32 products, 30 of it tiles' ends.
struct TileProject {
  ProjectArgs a;
  Side x, w;
  int K, nkc, mt, nt;
  PairSide px, pw;       // fp32: pairs, each row at a power of two of its own
  const int *ex, *ew;
};
template <typename T, class S, class Rows>
__global__ __launch_bounds__(S::threads, S::per_cu) void project_kernel(TileProject q) {
  constexpr int LD = S::BN + 4, ROWS = S::GM * 32;
  constexpr int kBytes = S::lds_bytes > ROWS * LD * 4 ? S::lds_bytes : ROWS * LD * 4;
  __shared__ __attribute__((aligned(1024))) char lds[kBytes];
  const ProjectArgs& a = q.a;
  int mi, ni;
  tile_of(blockIdx.x, (unsigned)(q.mt * q.nt), q.mt, q.nt, mi, ni);
  const int64_t r0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::GN, wn = wave % S::GN, l32 = lane & 31, h = lane >> 5;
  int bucket[S::WM];  // of row lane % 32 of each 32
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi) bucket[bi] = a.plan.bucket[min(r0 + (wm * S::WM + bi) * 32 + l32, a.n - 1)];
  floatx16 acc[S::WM][S::WN];
  if constexpr (sizeof(T) == 4) {
    pair_product<S>(q.px, q.pw, r0, n0, 0, q.nkc, lds, acc);
  } else {
    Rows rows;
    if constexpr (std::is_same<Rows, InOrder>::value) rows.order = a.plan.order;
    tile_product<T, S, Rows>(q.x, q.w, r0, n0, q.K, q.nkc, 1, 0, q.nkc, lds, acc, rows);
  }
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi) {
    const int b0 = (int)r0 + (wm * S::WM + bi) * 32;
    if (b0 >= a.n) continue;
    const int b1 = (int)min((int64_t)b0 + 32, a.n);
    // Runs of an adapter, in order, those without one and of none of them last.  As far as
    // registers go t stays in them, and the next run's entries of up are on their way while
    // one's are multiplied, both of the first HELD steps of 16 ranks.  A call of 2048
    // bfloat16 rows of 4096 to 4096, 1024 adapters of 16 130 us, without 149; 512 rows, 512
    // adapters of 64 150 and 181, with half as many steps held 173; 175 fp32 rows of 720 to
    // 699, 48 of 18 40 and 46; 20000 fp32 rows of 784 to 1024, 8 of 8 170 each way.
    constexpr int HELD = S::WM * S::WN <= 2 ? 4 : S::WM * S::WN <= 4 ? 2 : 0;
    const int at = min(b0 + l32, b1 - 1), steps = a.R / 16;
    const float* tr = a.t + (int64_t)at * a.R;
    const int te = std::is_same<T, half_t>::value ? a.texp[at] : 0;
    // (of fp32 the halves of a wavefront have half of the ranks each)
    auto rank0 = [&](int i) { return sizeof(T) == 4 ? h * (a.R / 2) + i * 8 : h * 8 + i * 16; };
    // fp32, or three parts: 24 bits of bfloat16, and of binary16 at the row's power of two
    constexpr int PARTS = sizeof(T) == 4 ? 1 : 3;
    auto coefs = [&](int i, float (&v)[8]) {
      const floatx4 t0 = *(const floatx4*)(tr + rank0(i)), t1 = *(const floatx4*)(tr + rank0(i) + 4);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        v[c] = c < 4 ? t0[c & 3] : t1[c & 3];
        if (std::is_same<T, half_t>::value) v[c] = ldexpf(v[c], te);
      }
    };
    auto next_part = [&](float (&v)[8]) {
      raw_n<8, T> part;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        part[c] = (T)v[c];
        v[c] -= (float)part[c];
      }
      return part;
    };
    auto fetch = [&](int g, int i, raw_n<8, T> (&up)[S::WN]) {
#pragma unroll
      for (int bj = 0; bj < S::WN; ++bj) {
        const int64_t col = min(n0 + (wn * S::WN + bj) * 32 + l32, (int64_t)a.m - 1);
        up[bj] = load_n<8>((const T*)a.up + ((int64_t)g * a.m + col) * a.uld, rank0(i), a.rank);
      }
    };
    raw_n<8, T> coef[HELD + 1][PARTS], ahead[HELD + 1][S::WN];  // (the last of ahead: of the steps past these)
    int g = __builtin_amdgcn_readlane(bucket[bi], 0);
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (i < steps && g < a.adapters) {
        float v[8];
        coefs(i, v);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) coef[i][k] = next_part(v);
        fetch(g, i, ahead[i]);
      }
    if constexpr (sizeof(T) == 4) {
      int ew[S::WN];
#pragma unroll
      for (int bj = 0; bj < S::WN; ++bj) ew[bj] = q.ew[min(n0 + (wn * S::WN + bj) * 32 + l32, (int64_t)a.m - 1)];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int ex = q.ex[min(b0 + acc_row(r, h), b1 - 1)];
#pragma unroll
        for (int bj = 0; bj < S::WN; ++bj) acc[bi][bj][r] = ldexpf(acc[bi][bj][r], -(ex + ew[bj]));
      }
    }
    for (int p = 0; p < b1 - b0;) {
      const int e = min(p + __popc((unsigned)__ballot(bucket[bi] == g)), b1 - b0);
      const int then = e < b1 - b0 ? __builtin_amdgcn_readlane(bucket[bi], e) : a.adapters;
      if (g < a.adapters) {
        floatx16 low[S::WN];
#pragma unroll
        for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
          for (int r = 0; r < 16; ++r) low[bj][r] = 0.f;
        auto products = [&](const raw_n<8, T>& part, const raw_n<8, T> (&up)[S::WN]) {
#pragma unroll
          for (int bj = 0; bj < S::WN; ++bj)
            if constexpr (sizeof(T) == 4) {
#pragma unroll
              for (int c = 0; c < 8; ++c) low[bj] = __builtin_amdgcn_mfma_f32_32x32x2f32(part[c], up[bj][c], low[bj], 0, 0, 0);
            } else {
              low[bj] = mfma16(part, up[bj], low[bj]);
            }
        };
#pragma unroll
        for (int i = 0; i < HELD; ++i)
          if (i < steps) {
#pragma unroll
            for (int k = 0; k < PARTS; ++k) products(coef[i][k], ahead[i]);
            if (then < a.adapters) fetch(then, i, ahead[i]);
          }
        for (int i = HELD; i < steps; ++i) {
          float v[8];
          coefs(i, v);
          fetch(g, i, ahead[HELD]);
#pragma unroll
          for (int k = 0; k < PARTS; ++k) products(next_part(v), ahead[HELD]);  // (a part at a time: fewer registers)
        }
        if constexpr (std::is_same<T, half_t>::value)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int e2 = a.texp[min(b0 + acc_row(r, h), b1 - 1)];
#pragma unroll
            for (int bj = 0; bj < S::WN; ++bj) low[bj][r] = ldexpf(low[bj][r], -e2);
          }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = acc_row(r, h);
          if (row >= p && row < e)
#pragma unroll
            for (int bj = 0; bj < S::WN; ++bj) acc[bi][bj][r] += low[bj][r];
        }
      } else if (g > a.adapters) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = acc_row(r, h);
          if (row >= p && row < e)
#pragma unroll
            for (int bj = 0; bj < S::WN; ++bj) acc[bi][bj][r] = __builtin_nanf("");
        }
      }
      p = e, g = then;
    }
  }
  // through LDS, 32 rows of each of GM at a time, so that rows are written 8 entries a lane
  float* sums = (float*)lds;
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi) {
    if (bi) __syncthreads();
#pragma unroll
    for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        sums[(wm * 32 + acc_row(r, h)) * LD + (wn * S::WN + bj) * 32 + l32] = acc[bi][bj][r];
    __syncthreads();
#pragma unroll
    for (int e = threadIdx.x; e < ROWS * (S::BN / 8); e += S::threads) {
      const int lr = e / (S::BN / 8), lc = e % (S::BN / 8) * 8;
      const int64_t place = r0 + (lr / 32 * S::WM + bi) * 32 + lr % 32, col = n0 + lc;
      if (place >= a.n || col >= a.m) continue;
      const float* v = sums + lr * LD + lc;
      T* y = (T*)a.y + (int64_t)a.plan.order[place] * a.ldy + col;
      raw_n<8, T> o;
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = (T)v[k];
      if (col + 8 <= a.m) {
        *(any_n<8, T>*)y = o;
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (col + k < a.m) y[k] = o[k];
      }
    }
  }
}

// Copies for the tiles, in sorted order where `order` is not null: 16-bit rows kp wide,
// zero from d on; fp32 rows as pairs, kp a whole number of blocks, each at the power of
// two that brings its largest entry to 2^14 .. 2^15 (`exps`): 22 bits of an entry down to
// 2^-28 of the row's largest, and 2^-50 of that below.  A row with an infinity or NaN is
// taken as it is.  20000 fp32 rows of 784 and 1024 of w 32 us, 4.1 TB/s.
struct CopyJob {
  const void* src;
  int64_t ld, rows;
  void* dst;
  int* exps;
  const int32_t* order;
  unsigned blocks;
};
struct CopyJobs {
  CopyJob j[2];
};
template <typename T>
__global__ __launch_bounds__(256) void copy_kernel(CopyJobs jobs, int d, int kp) {
  const bool second = blockIdx.x >= jobs.j[0].blocks;
  const CopyJob& j = jobs.j[second];
  const int64_t block = blockIdx.x - (second ? jobs.j[0].blocks : 0u);
  if constexpr (sizeof(T) == 2) {
    const int64_t per = kp / 8, step = (int64_t)j.blocks * 256;
    for (int64_t i = block * 256 + threadIdx.x; i < j.rows * per; i += step) {
      const int64_t row = i / per;
      const int c = (int)(i - row * per) * 8;
      *(raw_vec<T>*)((T*)j.dst + row * kp + c) = load_raw((const T*)j.src + (j.order ? j.order[row] : row) * j.ld, c, d);
    }
  } else {  // a wavefront a row
    const int lane = threadIdx.x & 63;
    for (int64_t row = block * 4 + (threadIdx.x >> 6); row < j.rows; row += (int64_t)j.blocks * 4) {
      const T* src = (const T*)j.src + (j.order ? j.order[row] : row) * j.ld;
      float top = 0.f;
      bool whole = true;
#pragma unroll 4
      for (int c = lane * 4; c < d; c += 256) {
        float v[4];
        load_part(src, c, d, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          top = fmaxf(top, fabsf(v[e]));
          whole &= fabsf(v[e]) < INFINITY;
        }
      }
#pragma unroll
      for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      const int e2 = __all(whole) ? power_for(top) : 0;
      if (lane == 0) j.exps[row] = e2;
      half_t* dst = (half_t*)j.dst + row * (2 * kp);
#pragma unroll 2
      for (int c = lane * 8; c < kp; c += 512) {
        const raw_n<8, T> v = load_n<8>(src, c, d);
        f16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          half_t x, y;
          split_pair(ldexpf(v[e], e2), x, y);
          hi[e] = x, lo[e] = y;
        }
        half_t* to = dst + pair_at(c);
        *(f16x8*)to = hi;
        *(f16x8*)(to + kPairBlock) = lo;
      }
    }
  }
}

// ------------------------------------------------------------------ the adapters' gradients

// out[r][c] = sum over a piece of an adapter's rows of coef[place][r] X[row][c], to
// the piece's slab: CT x 16 of the rank by 16 kVec columns a workgroup.  A step is 4
// rows: a lane loads kVec columns of row lane / 16; the four wavefronts take every
// fourth run of steps and join in LDS.  20000 fp32 rows of 784 + 1024, 8 ranks 40 us, 3.6
// TB/s.
struct OuterJob {
  const float* coef;  // n x R, in sorted order
  const void* X;
  int64_t ldx;
  int d;
  float* slabs;  // piece x rank x d
  unsigned bx;   // workgroups across the columns
};
struct OuterJobs {
  OuterJob j[2];
  int adapters, rank, R, piece;
  RowPlan plan;
};
template <typename T, int CT>
__global__ __launch_bounds__(256) void outer_kernel(OuterJobs q) {
  constexpr int VEC = kVec<T>, W = 16 * VEC, UN = CT > 2 ? 2 : 4;
  __shared__ float red[CT * 16][W + 1];
  const int at = blockIdx.y;
  if (at >= q.plan.piece[q.adapters]) return;
  const bool second = blockIdx.x >= q.j[0].bx;
  const OuterJob& j = q.j[second];
  const int c0 = (blockIdx.x - (second ? q.j[0].bx : 0u)) * W, s0 = blockIdx.z * (CT * 16);
  const int g = __builtin_amdgcn_readfirstlane(owner(q.plan.piece, q.adapters, at));
  const int p0 = q.plan.start[g] + q.piece * (at - q.plan.piece[g]), p1 = min(p0 + q.piece, q.plan.start[g + 1]);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15,
            k4 = lane >> 4;
  const int col = c0 + l16 * VEC;
  floatx4 acc[VEC][CT];
#pragma unroll
  for (int e = 0; e < VEC; ++e)
#pragma unroll
    for (int t = 0; t < CT; ++t) acc[e][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  // the next step's rows are on their way while one is multiplied, and the one's after that are being looked up
  const bool inside = c0 + W <= j.d;
  int row[UN];
  raw_vec<T> x[UN], xn[UN];
  float c[UN][CT], cn[UN][CT];
  auto find = [&](int p) {
#pragma unroll
    for (int u = 0; u < UN; ++u) row[u] = q.plan.order[min(p + u * 4 + k4, p1 - 1)];
  };
  auto fetch = [&](int p) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const T* xr = (const T*)j.X + (int64_t)row[u] * j.ldx;
      if (inside)
        xn[u] = *(const any_vec<T>*)(xr + col);
      else
        xn[u] = load_raw(xr, col, j.d);
      const float* cr = j.coef + (int64_t)min(p + u * 4 + k4, p1 - 1) * q.R + s0 + l16;
#pragma unroll
      for (int t = 0; t < CT; ++t) cn[u][t] = cr[t * 16];
    }
  };
  int p = p0 + wave * (4 * UN);
  find(p);
  fetch(p);
  find(p + 16 * UN);
  for (; p < p1; p += 16 * UN) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const bool use = p + u * 4 + k4 < p1;
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[u][e] = use ? xn[u][e] : (T)0.f;
#pragma unroll
      for (int t = 0; t < CT; ++t) c[u][t] = use ? cn[u][t] : 0.f;
    }
    fetch(p + 16 * UN);
    find(p + 32 * UN);
#pragma unroll
    for (int u = 0; u < UN; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e)
#pragma unroll
        for (int t = 0; t < CT; ++t)
          acc[e][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(c[u][t], (float)x[u][e], acc[e][t], 0, 0, 0);
  }
  for (int o = 0; o < 4; ++o) {
    if (wave == o)
#pragma unroll
      for (int e = 0; e < VEC; ++e)
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float* v = &red[t * 16 + 4 * k4 + r][l16 * VEC + e];
            *v = o ? *v + acc[e][t][r] : acc[e][t][r];
          }
    __syncthreads();
  }
  float* slab = j.slabs + (int64_t)at * q.rank * j.d;
  for (int e = threadIdx.x; e < CT * 16 * W; e += 256) {
    const int r = e / W, c = e % W;
    if (s0 + r < q.rank && c0 + c < j.d) slab[(int64_t)(s0 + r) * j.d + c0 + c] = red[r][c];
  }
}

// As outer_kernel for 16-bit rows, on the 16-bit matrix cores: 32 rows a step, 8 of
// them a lane's, whose 8 x 8 values it turns in registers so that a column's 8 rows lie
// together.  coef is three bfloat16 parts, all of its 24 bits; a binary16 row is two, which
// hold all of it, and five products (the sixth lies below the last bit kept).  8192
// bfloat16 rows of 4096 + 4096 and 32 ranks: 41 us, 3.3 TB/s, where the fp32 matrix cores
// take 78.
template <typename T, int CT>
__global__ __launch_bounds__(256) void outer16_kernel(OuterJobs q) {
  constexpr int W = 128;
  constexpr bool kHalf = std::is_same<T, half_t>::value;
  __shared__ float red[CT * 16][W + 1];
  const int at = blockIdx.y;
  if (at >= q.plan.piece[q.adapters]) return;
  const bool second = blockIdx.x >= q.j[0].bx;
  const OuterJob& j = q.j[second];
  const int c0 = (blockIdx.x - (second ? q.j[0].bx : 0u)) * W, s0 = blockIdx.z * (CT * 16);
  const int g = __builtin_amdgcn_readfirstlane(owner(q.plan.piece, q.adapters, at));
  const int p0 = q.plan.start[g] + q.piece * (at - q.plan.piece[g]), p1 = min(p0 + q.piece, q.plan.start[g + 1]);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15,
            k4 = lane >> 4;
  const int col = c0 + l16 * 8;
  const bool inside = c0 + W <= j.d;
  floatx4 acc[8][CT];
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int t = 0; t < CT; ++t) acc[e][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  int row[8];
  raw_vec<T> xn[8];
  float cn[8][CT];
  auto find = [&](int p) {
#pragma unroll
    for (int u = 0; u < 8; ++u) row[u] = q.plan.order[min(p + k4 * 8 + u, p1 - 1)];
  };
  auto fetch = [&](int p) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const T* xr = (const T*)j.X + (int64_t)row[u] * j.ldx;
      if (inside)
        xn[u] = *(const any_vec<T>*)(xr + col);
      else
        xn[u] = load_raw(xr, col, j.d);
      const float* cr = j.coef + (int64_t)min(p + k4 * 8 + u, p1 - 1) * q.R + s0 + l16;
#pragma unroll
      for (int t = 0; t < CT; ++t) cn[u][t] = cr[t * 16];
    }
  };
  int p = p0 + wave * 32;
  find(p);
  fetch(p);
  find(p + 128);
  for (; p < p1; p += 128) {
    const int left = p1 - p - k4 * 8;  // rows from this one on take no part
    unsigned w[8][4];
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        typedef T pair __attribute__((ext_vector_type(2)));
        const pair v = {xn[u][2 * e], xn[u][2 * e + 1]};
        w[u][e] = u < left ? __builtin_bit_cast(unsigned, v) : 0u;
      }
    frag<bf16_t> part[3][CT];
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        float v = u < left ? cn[u][t] : 0.f;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          part[k][t][u] = (bf16_t)v;
          v -= (float)part[k][t][u];
        }
      }
    fetch(p + 128);
    find(p + 256);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      typedef unsigned words __attribute__((ext_vector_type(4)));
      words v;
#pragma unroll
      for (int u = 0; u < 4; ++u)  // column e of rows 2 u and 2 u + 1
        v[u] = __builtin_amdgcn_perm(w[2 * u + 1][e / 2], w[2 * u][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
      const frag<T> x = __builtin_bit_cast(frag<T>, v);
      if constexpr (kHalf) {
        frag<bf16_t> xh, xl;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          xh[u] = (bf16_t)(float)x[u];
          xl[u] = (bf16_t)((float)x[u] - (float)xh[u]);
        }
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
          for (int k = 2; k >= 0; --k) {  // small ones first
            acc[e][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[k][t], k == 2 ? xh : xl, acc[e][t], 0, 0, 0);
            if (k < 2) acc[e][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[k][t], xh, acc[e][t], 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
          for (int k = 2; k >= 0; --k)
            acc[e][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(part[k][t], x, acc[e][t], 0, 0, 0);
      }
    }
  }
  for (int o = 0; o < 4; ++o) {
    if (wave == o)
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float* v = &red[t * 16 + 4 * k4 + r][l16 * 8 + e];
            *v = o ? *v + acc[e][t][r] : acc[e][t][r];
          }
    __syncthreads();
  }
  float* slab = j.slabs + (int64_t)at * q.rank * j.d;
  for (int e = threadIdx.x; e < CT * 16 * W; e += 256) {
    const int r = e / W, c = e % W;
    if (s0 + r < q.rank && c0 + c < j.d) slab[(int64_t)(s0 + r) * j.d + c0 + c] = red[r][c];
  }
}

// The pieces' sums, in order: ddown as it is, dup turned.
struct JoinArgs {
  const float *down_slabs, *up_slabs;
  int adapters, rank, d, m;
  const int32_t* piece;
  void *ddown, *dup;  // each may be null
};
// A workgroup has 64 columns of 8 rows of an adapter's rank, a wavefront two of these
// rows.  33 MB of slabs 15 us.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a) {
  __shared__ float turned[64][8 + 1];
  const int rb = (a.rank + 7) / 8, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t per_d = a.ddown ? (int64_t)rb * ((a.d + 63) / 64) : 0, per_u = a.dup ? (int64_t)rb * ((a.m + 63) / 64) : 0;
  for (int64_t unit = blockIdx.x; unit < a.adapters * (per_d + per_u); unit += gridDim.x) {
    const bool up = unit >= a.adapters * per_d;
    const int64_t i = up ? unit - a.adapters * per_d : unit, per = up ? per_u : per_d, g = i / per, b = i - g * per;
    const int r0 = (int)(b % rb) * 8 + wave * 2, width = up ? a.m : a.d;
    const int64_t c0 = b / rb * 64, c = c0 + lane;
    const int k0 = a.piece[g], k1 = a.piece[g + 1];
    const bool use = c < width && r0 < a.rank;
    const int64_t second = r0 + 1 < a.rank ? width : 0;
    const float* p = (up ? a.up_slabs : a.down_slabs) + (use ? ((int64_t)k0 * a.rank + r0) * width + c : 0);
    float s[2] = {0.f, 0.f};
    if (use)
#pragma unroll 4
      for (int k = k0; k < k1; ++k, p += (int64_t)a.rank * width) {
        s[0] += p[0];
        s[1] += p[second];
      }
    if (!up) {
#pragma unroll
      for (int r = 0; r < 2; ++r)
        if (use && r0 + r < a.rank) ((T*)a.ddown)[(g * a.rank + r0 + r) * a.d + c] = (T)s[r];
      continue;
    }
    turned[lane][wave * 2] = s[0];
    turned[lane][wave * 2 + 1] = s[1];
    __syncthreads();
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const int e = o * 256 + threadIdx.x, r = (int)(b % rb) * 8 + e % 8;
      if (r < a.rank && c0 + e / 8 < width) ((T*)a.dup)[(g * a.m + c0 + e / 8) * a.rank + r] = (T)turned[e / 8][e % 8];
    }
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(256) void zero_kernel(T* out, int64_t count) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) out[i] = (T)0.f;
}

// ------------------------------------------------------------------ host

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t up_to(int64_t v, int64_t m) { return cdiv(v, m) * m; }

// Rank blocks of 16 that the kernels know.
int rank_blocks(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8; }

// Scratch is laid out by the same code that sizes it (p null).
struct Layout {
  char* p;
  size_t used = 0;
  template <typename T>
  T* take(int64_t count) {
    T* r = p ? (T*)(p + used) : nullptr;
    used += ((size_t)count * sizeof(T) + 255) / 256 * 256;
    return r;
  }
};

// A piece of an adapter's rows in `outer`: 64 at least, and so many that the pieces of
// all fill the card with two workgroups a CU, four of fp32.  The adapters' gradients in
// microseconds with two / four / eight: bfloat16 8192 x 4096 to 4096, 16 adapters of 32
// ranks 104 / 109 / 121, 4096 x 1000 to 1000, 60 of 16 60 / 70 / 71, binary16, 32 of 64 121 /
// 156 / 157; fp32 20000 x 784 to 1024, 8 of 8 105 / 89 / 87.
int piece_of(const AdaptArgs& a) {
  const int64_t w = 16 * 16 / (int64_t)elem_bytes(a.type), across = cdiv(a.d, w) + cdiv(a.m, w);
  const int64_t pieces = std::max<int64_t>(1, (a.type == TYPE_F32 ? 1024 : 512) / across);
  return (int)std::min<int64_t>(up_to(std::max<int64_t>(64, cdiv(a.n, pieces)), 16), 1 << 20);
}
int64_t most_pieces(const AdaptArgs& a) { return cdiv(a.n, piece_of(a)) + std::min<int64_t>(a.adapters, a.n); }

constexpr int kFewRows = 64;  // so many rows run as they are, and take no plan (t in their own order)
constexpr double kFewProducts = 1 << 23;  // so many run from the rows as they are: 1000 x 54 to 7, fp32, 22 us, in tiles 24

// The tiles of a projection, and what its launch takes in them, in microseconds: `end`,
// and a chunk's time in a full round of 256 tiles and in one of few.  A call, of 16-bit
// rows n x d to m, in 256 x 256 / 256 x 128 / 128 x 128 / 128 x 64 / 64 x 64: 8192 x 4096 to
// 4096 287 / 313 / 360 / 396 / 478, 1024 x 4096 to 4096 113 / 69 / 62 / 69 / 78, 256 x 4096 to
// 4096 115 / 67 / 50 / 48 / 40, 20000 x 784 to 256 64 / 49 / 54 / 54 / 53, 3000 x 1000 to 776
// 59 / 43 / 33 / 38 / 36; fp32, 20000 x 784 to 1024 - / 179 / 180 / 177 / 195.
struct TileTime {
  int high, wide;
  double end, alone, full;    // 16 bits, 64 indices
  double alone32, full32;     // pairs, 32
};
constexpr TileTime kTiles[5] = {{256, 256, 8, 1.45, 2.05, 0, 0},
                                {256, 128, 6, 0.77, 1.15, 0.85, 1.35},
                                {128, 128, 5, 0.5, 0.68, 0.5, 0.73},
                                {128, 64, 4, 0.42, 0.39, 0.33, 0.39},
                                {64, 64, 3, 0.3, 0.225, 0.2, 0.225}};
double tile_time(const TileTime& t, bool f32, int64_t n, int d, int m) {
  const double tiles = (double)cdiv(n, t.high) * cdiv(m, t.wide) / 256, rounds = std::floor(tiles), left = tiles - rounds;
  const double alone = f32 ? t.alone32 : t.alone, full = f32 ? t.full32 : t.full;
  return t.end + cdiv(d, f32 ? kPairBlock : kChunkK) *
                     (rounds * full + (left > 0 ? alone + (full - alone) * left * left * left : 0));
}

// One projection: 0, or one more than the tiles it runs in, and what copies that takes.
struct Way {
  int tiled;
  bool gather, copy_x, copy_w;
  int kp;
};
Way way_of(int type, int64_t n, int d, int m, const void* x, int64_t ldx, const void* w, int64_t ldw, bool w_padded) {
  Way r{};
  if (n > kFewRows && (double)n * m * d > kFewProducts) {
    double best = 0;
    for (int k = type == TYPE_F32 ? 1 : 0; k < 5; ++k) {  // (a pair's two sums are too many for 256 x 256)
      const double t = tile_time(kTiles[k], type == TYPE_F32, n, d, m);
      if (!r.tiled || t < best) best = t, r.tiled = k + 1;
    }
  }
  r.kp = (int)up_to(d, type == TYPE_F32 ? kPairBlock : 8);
  auto fits = [&](const void* p, int64_t ld) {
    return type != TYPE_F32 && d % 8 == 0 && ld % 8 == 0 && ld < (1 << 21) && (uintptr_t)p % 16 == 0;
  };
  r.gather = fits(x, ldx) && n * ldx * 2 < 0x7fff0000;
  r.copy_x = !r.gather;
  r.copy_w = w_padded ? type == TYPE_F32 : !fits(w, ldw);  // (padded: whole rows of kp, zero from d on)
  return r;
}
// Rows of a tile of `shrink`: each reads its adapter's matrix once.  A call with 16 / 32:
// 8192 bfloat16 rows of 4096, 16 adapters of 32 ranks 298 / 293, 4096 binary16 of 1000, 32
// of 64 59 / 51, 2048 bfloat16 of 4096, 4 of 16 48 / 51.
int shrink_rows(const AdaptArgs& a) { return a.n >= 4096 && a.n >= 64 * (int64_t)a.adapters && a.rank <= 64 ? 32 : 16; }
int64_t most_tiles(const AdaptArgs& a) { return cdiv(a.n, shrink_rows(a)) + std::min<int64_t>(a.adapters, a.n); }
// Rows of a workgroup that plans: all of few, else 1024, or a 64th of all.
int64_t plan_run(int64_t n) { return n <= 2048 ? 2048 : std::max<int64_t>(1024, up_to(cdiv(n, 64), 1024)); }
int64_t plan_runs(int64_t n) { return cdiv(n, plan_run(n)); }

struct Scratch {
  RowPlan plan;
  int* counts;
  float *t, *u;
  int *texp, *uexp;
  void *wt, *upt, *downt;  // turned
  void *xc, *wc;           // the tiles' copies
  int *ex, *ew;
  float *down_slabs, *up_slabs;
  size_t bytes;
};
Scratch scratch_of(const AdaptArgs& a, bool grad, void* p) {
  Layout l{(char*)p};
  Scratch s{};
  const int size = (int)elem_bytes(a.type), R = rank_blocks(a.rank) * 16;
  s.plan.order = l.take<int32_t>(a.n);
  s.plan.place = l.take<int32_t>(a.n);
  s.plan.bucket = l.take<int32_t>(a.n);
  s.plan.start = l.take<int32_t>(a.adapters + 3);
  s.plan.tile = l.take<int32_t>(a.adapters + 1);
  s.plan.piece = l.take<int32_t>(a.adapters + 1);
  s.t = l.take<float>(a.n * R);
  s.counts = l.take<int>(plan_runs(a.n) * (a.adapters + 2));
  auto exps = [&](const Way& w) { return w.tiled && a.type == TYPE_F16 ? l.take<int>(a.n) : nullptr; };
  auto copies = [&](const Way& w, int64_t rows) {
    if (!w.tiled) return;
    const int64_t row = (int64_t)w.kp * size;
    if (w.copy_x) s.xc = l.take<char>(a.n * row);
    if (w.copy_w) s.wc = l.take<char>(rows * row);
    if (a.type == TYPE_F32) s.ex = l.take<int>(a.n), s.ew = l.take<int>(rows);
  };
  if (!grad) {
    const Way w = way_of(a.type, a.n, a.d, a.m, a.x, a.ldx, a.w, a.ldw, false);
    s.texp = exps(w);
    copies(w, a.m);
  } else {
    s.u = l.take<float>(a.n * R);
    if (a.dx || a.ddown) s.upt = l.take<char>((int64_t)a.adapters * a.rank * a.m * size);
    if (a.dx) {
      s.downt = l.take<char>((int64_t)a.adapters * a.rank * a.d * size);
      s.wt = l.take<char>((int64_t)a.d * up_to(a.m, 8) * size);
      const Way w = way_of(a.type, a.n, a.m, a.d, a.dy, a.lddy, nullptr, 0, true);
      s.uexp = exps(w);
      copies(w, a.d);
    }
    if (a.ddown) s.down_slabs = l.take<float>(most_pieces(a) * a.rank * a.d);
    if (a.dup) s.up_slabs = l.take<float>(most_pieces(a) * a.rank * a.m);
  }
  s.bytes = l.used;
  return s;
}

template <typename T>
TurnJob turn_job(const void* src, int64_t count, int64_t ld, int64_t rows, int64_t cols, int64_t ldd, void* dst) {
  TurnJob j{src, ld, rows, cols, ldd, dst, 0, cdiv(cols, 64), 0};
  j.per = j.bx * cdiv(std::max(rows, ldd), 64);
  j.blocks = j.per * count;
  return j;
}

template <typename T, class S>
hipError_t launch_tiles(const ProjectArgs& a, const Way& w, const Scratch& sc, hipStream_t s) {
  CopyJobs jobs{};
  auto job = [&](CopyJob& j, const void* src, int64_t ld, int64_t rows, void* dst, int* exps, const int32_t* order) {
    const int64_t units = sizeof(T) == 4 ? cdiv(rows, 4) : cdiv(rows * (w.kp / 8), 256);
    j = {src, ld, rows, dst, exps, order, (unsigned)std::min<int64_t>(units, 8192)};
  };
  if (w.copy_x) job(jobs.j[0], a.x, a.ldx, a.n, sc.xc, sc.ex, a.plan.order);
  if (w.copy_w) job(jobs.j[1], a.w, a.ldw, a.m, sc.wc, sc.ew, nullptr);
  if (const unsigned blocks = jobs.j[0].blocks + jobs.j[1].blocks) copy_kernel<T><<<blocks, 256, 0, s>>>(jobs, a.d, w.kp);
  TileProject q{};
  q.a = a;
  q.K = w.kp;
  q.nkc = (int)cdiv(w.kp, sizeof(T) == 4 ? kPairBlock : kChunkK);
  if constexpr (sizeof(T) == 4) {
    q.px = {(const half_t*)sc.xc, 2 * w.kp, a.n};
    q.pw = {(const half_t*)sc.wc, 2 * w.kp, a.m};
    q.ex = sc.ex;
    q.ew = sc.ew;
  } else {
    q.x = w.copy_x ? Side{sc.xc, w.kp, 0, a.n} : Side{a.x, a.ldx, 0, a.n};
    q.w = w.copy_w ? Side{sc.wc, w.kp, 0, a.m} : Side{a.w, a.ldw, 0, a.m};
  }
  q.mt = (int)cdiv(a.n, S::BM);
  q.nt = (int)cdiv(a.m, S::BN);
  const unsigned grid = (unsigned)(q.mt * q.nt);
  if constexpr (sizeof(T) == 2)
    if (w.gather) {
      project_kernel<T, S, InOrder><<<grid, S::threads, 0, s>>>(q);
      return hipGetLastError();
    }
  project_kernel<T, S, AsTheyAre><<<grid, S::threads, 0, s>>>(q);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_project(const ProjectArgs& a, const Way& w, const Scratch& sc, hipStream_t s) {
  switch (w.tiled) {
    case 1:
      if constexpr (sizeof(T) == 2) return launch_tiles<T, BigTile>(a, w, sc, s);
      break;
    case 2: return launch_tiles<T, TileShape<2, 2, 4, 2, 3>>(a, w, sc, s);
    case 3: return launch_tiles<T, TileShape<1, 2, 4, 2, 4>>(a, w, sc, s);
    case 4: return launch_tiles<T, TileShape<2, 1, 2, 2, 3>>(a, w, sc, s);
    case 5: return launch_tiles<T, TileShape<1, 1, 2, 2, 4>>(a, w, sc, s);
  }
  auto launch = [&](auto shape) {
    using S = decltype(shape);
    direct_kernel<T, S><<<(unsigned)(cdiv(a.m, S::NA * 16) * cdiv(a.n, S::NB * 16)), S::WV * 64, 0, s>>>(a);
  };
  if (a.n <= 16)
    launch(WaveRows<T, 1, 1, 8>{});
  else if (a.n <= 32)
    launch(WaveRows<T, 1, 2, 8>{});
  else if (a.n <= 64)
    launch(WaveRows<T, 1, 4, 8>{});
  else
    launch(WaveRows<T, 4, 2, 4>{});
  return hipGetLastError();
}

template <typename T, int RB>
void launch_shrink_rank(const AdaptArgs& a, const ShrinkJobs& q, hipStream_t s) {
  const unsigned blocks = q.j[0].blocks + q.j[1].blocks;
  auto launch = [&](auto shape) {
    using S = decltype(shape);
    shrink_kernel<T, S><<<blocks, S::WV * 64, 0, s>>>(q);
  };
  if constexpr (RB <= 4)
    if (shrink_rows(a) == 32) return launch(WaveRows<T, RB, 2, 8>{});
  launch(WaveRows<T, RB, 1, RB == 8 ? 4 : 8>{});  // (more registers a wavefront)
}
template <typename T>
void launch_shrink(const AdaptArgs& a, const ShrinkJobs& q, hipStream_t s) {
  switch (rank_blocks(a.rank)) {
    case 1: return launch_shrink_rank<T, 1>(a, q, s);
    case 2: return launch_shrink_rank<T, 2>(a, q, s);
    case 4: return launch_shrink_rank<T, 4>(a, q, s);
    default: return launch_shrink_rank<T, 8>(a, q, s);
  }
}

template <typename T>
hipError_t launch_typed(const AdaptArgs& a, bool grad, void* scratch, hipStream_t s) {
  const int RB = rank_blocks(a.rank), R = RB * 16;
  if (a.n == 0) {
    for (int k = 0; k < 2; ++k) {
      T* out = (T*)(k ? a.dup : a.ddown);
      const int64_t count = (int64_t)a.adapters * a.rank * (k ? a.m : a.d);
      if (grad && out) zero_kernel<T><<<(unsigned)std::min<int64_t>(cdiv(count, 256), 4096), 256, 0, s>>>(out, count);
    }
    return hipGetLastError();
  }
  const Scratch sc = scratch_of(a, grad, scratch);
  const bool few = !grad && a.n <= kFewRows;
  const int piece = piece_of(a);
  if (!few) {
    int bits = 1;
    while (1 << bits < a.adapters + 2) ++bits;
    const int64_t run = plan_run(a.n);
    const unsigned runs = (unsigned)plan_runs(a.n);
    const size_t lds = (a.adapters + 2) * sizeof(int);
    if (runs > 1) count_kernel<<<runs, kPlanWaves * 64, lds, s>>>(a.ids, a.n, a.adapters, run, bits, sc.counts);
    plan_kernel<<<runs, kPlanWaves * 64, kPlanWaves * lds, s>>>(a.ids, a.n, a.adapters, run, runs > 1 ? sc.counts : nullptr,
                                                                bits, shrink_rows(a), piece, sc.plan);
  }
  const unsigned tiles = (unsigned)most_tiles(a);
  ShrinkJobs sh{};
  sh.adapters = a.adapters;
  sh.rank = a.rank;
  sh.factor = a.factor;
  sh.plan = sc.plan;
  const ShrinkJob of_x = {a.x, a.ldx, a.d, a.down, a.d, sc.t, sc.texp, tiles};
  ProjectArgs p{};
  p.n = a.n;
  p.adapters = a.adapters;
  p.rank = a.rank;
  p.uld = a.rank;
  p.R = R;
  p.plan = sc.plan;
  p.ids = a.ids;
  if (!grad) {
    p.x = a.x, p.ldx = a.ldx, p.d = a.d;
    p.w = a.w, p.ldw = a.ldw, p.m = a.m;
    p.up = a.up;
    p.t = sc.t, p.texp = sc.texp;
    p.y = a.y, p.ldy = a.ldy;
    if (a.n == 1 && a.rank <= 16) {
      one_row_kernel<T><<<(unsigned)cdiv(a.m, 16), 512, 0, s>>>(p, (const T*)a.down, a.factor);
      return hipGetLastError();
    }
    if (few) {
      p.plan.place = nullptr;
      shrink_rows_kernel<T><<<(unsigned)a.n, 1024, 0, s>>>((const T*)a.x, a.ldx, a.d, (const T*)a.down, a.adapters, a.rank,
                                                           R, a.ids, a.factor, sc.t);
    } else {
      sh.j[0] = of_x;
      launch_shrink<T>(a, sh, s);
    }
    return launch_project<T>(p, way_of(a.type, a.n, a.d, a.m, a.x, a.ldx, a.w, a.ldw, false), sc, s);
  }
  TurnJobs turn{};
  const int64_t mp = up_to(a.m, 8);
  if (sc.upt) turn.j[0] = turn_job<T>(a.up, a.adapters, a.rank, a.m, a.rank, a.m, sc.upt);
  if (a.dx) {
    turn.j[1] = turn_job<T>(a.down, a.adapters, a.d, a.rank, a.d, a.rank, sc.downt);
    turn.j[2] = turn_job<T>(a.w, 1, a.ldw, a.m, a.d, mp, sc.wt);
  }
  if (const int64_t blocks = turn.j[0].blocks + turn.j[1].blocks + turn.j[2].blocks)
    turn_kernel<T><<<(unsigned)std::min<int64_t>(blocks, 1 << 20), 256, 0, s>>>(turn);
  const ShrinkJob of_dy = {a.dy, a.lddy, a.m, sc.upt, a.m, sc.u, sc.uexp, tiles};
  int count = 0;
  if (sc.upt) sh.j[count++] = of_dy;
  if (a.dup) sh.j[count++] = of_x;
  launch_shrink<T>(a, sh, s);
  if (a.dx) {
    p.x = a.dy, p.ldx = a.lddy, p.d = a.m;
    p.w = sc.wt, p.ldw = mp, p.m = a.d;
    p.up = sc.downt;
    p.t = sc.u, p.texp = sc.uexp;
    p.y = a.dx, p.ldy = a.lddx;
    const hipError_t e = launch_project<T>(p, way_of(a.type, a.n, a.m, a.d, a.dy, a.lddy, sc.wt, mp, true), sc, s);
    if (e != hipSuccess) return e;
  }
  if (!a.ddown && !a.dup) return hipGetLastError();
  constexpr int W = 16 * kVec<T>;
  OuterJobs o{};
  o.adapters = a.adapters;
  o.rank = a.rank;
  o.R = R;
  o.piece = piece;
  o.plan = sc.plan;
  count = 0;
  if (a.ddown) o.j[count++] = {sc.u, a.x, a.ldx, a.d, sc.down_slabs, (unsigned)cdiv(a.d, W)};
  if (a.dup) o.j[count++] = {sc.t, a.dy, a.lddy, a.m, sc.up_slabs, (unsigned)cdiv(a.m, W)};
  const dim3 grid(o.j[0].bx + o.j[1].bx, (unsigned)most_pieces(a), RB == 8 ? 2 : 1);
  // (binary16 of at most 16 ranks, both gradients by the fp32 matrix cores / in parts: 3001 x 1001 to 777, 5 adapters
  // of 12 35 / 36 us, 4096 x 1000 to 1000, 60 of 16 49 / 57, 20000 x 784 to 1024, 8 of 8 72 / 71, 8192 x 4096 to 4096, 16
  // of 16 81 / 77)
  auto outer = [&](auto ct) {
    if constexpr (std::is_same<T, bf16_t>::value || (sizeof(T) == 2 && ct.value > 1))
      outer16_kernel<T, ct.value><<<grid, 256, 0, s>>>(o);
    else
      outer_kernel<T, ct.value><<<grid, 256, 0, s>>>(o);
  };
  if (RB == 1)
    outer(std::integral_constant<int, 1>{});
  else if (RB == 2)
    outer(std::integral_constant<int, 2>{});
  else
    outer(std::integral_constant<int, 4>{});
  const JoinArgs j = {sc.down_slabs, sc.up_slabs, a.adapters, a.rank, a.d, a.m, sc.plan.piece, a.ddown, a.dup};
  const int64_t units = a.adapters * cdiv(a.rank, 8) * ((a.ddown ? cdiv(a.d, 64) : 0) + (a.dup ? cdiv(a.m, 64) : 0));
  join_kernel<T><<<(unsigned)std::min<int64_t>(units, 1 << 20), 256, 0, s>>>(j);
  return hipGetLastError();
}

}  // namespace

size_t adapt_scratch(const AdaptArgs& a, bool grad) { return a.n ? scratch_of(a, grad, nullptr).bytes : 0; }

hipError_t launch_adapt(const AdaptArgs& a, bool grad, void* scratch, hipStream_t s) {
  if (a.type == TYPE_F32) return launch_typed<float>(a, grad, scratch, s);
  return a.type == TYPE_F16 ? launch_typed<half_t>(a, grad, scratch, s)
                            : launch_typed<bf16_t>(a, grad, scratch, s);
}

}  // namespace kkm
