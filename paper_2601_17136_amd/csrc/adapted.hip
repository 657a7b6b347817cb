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
//   shrink     t, u: 16 rows of one adapter a workgroup
//   project    w's product with the adapters' part added before the one rounding:
//              direct, from the rows as they are (at most 64 rows or columns, or
//              little work), or in tiles of the sorted rows (head_tile.h)
//   outer      (gradient) the adapters' gradients of a piece of an adapter's rows
//   join       their sums over the pieces
//
// The adapters' products run on the fp32 matrix cores: they are few beside w's, and
// t and u keep all their bits.
#include <algorithm>

#include "few_mma.h"
#include "pair_tile.h"
#include "model_ops.h"

namespace kkm {

namespace {

// Where the rows of each adapter are.  Bucket `adapters` holds the rows without
// one, the next one those whose id is none of them.
struct RowPlan {
  int32_t *order, *place, *bucket;  // row at a place, place of a row, bucket of a place
  int32_t *start;                   // adapters + 3: a bucket's first place
  int32_t *tile, *piece;            // adapters + 1: its first tile of `shrink`, its first piece
};

// One workgroup: each wavefront counts and then places a run of rows, 64 at a time.
constexpr int kPlanWaves = 16;
__global__ __launch_bounds__(kPlanWaves * 64) void plan_kernel(const int32_t* __restrict__ ids, int64_t n, int adapters,
                                                               int bits, int tile, int piece, RowPlan q) {
  extern __shared__ int cnt[];  // [kPlanWaves][nb]
  __shared__ int sums[kPlanWaves][3];
  const int nb = adapters + 2, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int e = threadIdx.x; e < kPlanWaves * nb; e += kPlanWaves * 64) cnt[e] = 0;
  __syncthreads();
  const int64_t per = ((n + kPlanWaves - 1) / kPlanWaves + 63) / 64 * 64, lo = wave * per, hi = min(lo + per, n);
  auto bucket_of = [&](int64_t i) {
    const int g = ids[i];
    return g < 0 ? adapters : g >= adapters ? adapters + 1 : g;
  };
  volatile int* own = cnt + wave * nb;
  constexpr int U = 8;  // runs of 64 rows whose ids are read at a time
  int b8[U];
  auto read = [&](int64_t i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) b8[u] = i0 + u * 64 + lane < hi ? bucket_of(i0 + u * 64 + lane) : -1;
  };
  for (int64_t i0 = lo; i0 < hi; i0 += 64 * U) {
    read(i0);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (b8[u] >= 0) atomicAdd(cnt + wave * nb + b8[u], 1);
  }
  __syncthreads();
  // first places: by bucket, then by wavefront; tiles and pieces likewise
  int first = 0, tiles = 0, pieces = 0;  // of the buckets before this round's
  for (int b0 = 0; b0 < nb; b0 += kPlanWaves * 64) {
    const int b = b0 + threadIdx.x;
    int total = 0;
    if (b < nb)
      for (int w = 0; w < kPlanWaves; ++w) total += cnt[w * nb + b];
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
      q.start[b] = at;
      if (b <= adapters) {
        q.tile[b] = base[1] + s[1] - v[1];
        q.piece[b] = base[2] + s[2] - v[2];
      }
      for (int w = 0; w < kPlanWaves; ++w) {
        const int c = cnt[w * nb + b];
        cnt[w * nb + b] = at;
        at += c;
      }
    }
    first = all[0], tiles = all[1], pieces = all[2];
    __syncthreads();
  }
  if (threadIdx.x == 0) q.start[nb] = first;
  for (int64_t i0 = lo; i0 < hi; i0 += 64 * U) {
    read(i0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * 64 + lane;
      if (i0 + u * 64 >= hi) break;
      const int b = b8[u];
      const bool here = b >= 0;
      unsigned long long same = __ballot(here);
      for (int k = 0; k < bits; ++k) {
        const unsigned long long set = __ballot(b >> k & 1);
        same &= b >> k & 1 ? set : ~set;
      }
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

// dst[c][r] = src[r][c] of `count` matrices, 64 x 64 at a time.
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

// ------------------------------------------------------------------ t and u

struct ShrinkJob {
  const void* x;
  int64_t ldx;
  int d;
  const void* low;  // adapters x rank x d, rows lowld apart
  int64_t lowld;
  float* t;         // n x rank padded to 16 RB, in sorted order
  unsigned blocks;
};
struct ShrinkJobs {
  ShrinkJob j[2];
  int adapters, rank;
  const float* factor;
  RowPlan plan;
};

// NT x 16 rows of an adapter by its rank; the WV wavefronts take runs of steps of the
// width in turn and join in LDS.
template <typename T, int RB, int NT, int WV>
__global__ __launch_bounds__(WV * 64) void shrink_kernel(ShrinkJobs q) {
  constexpr int VEC = kVec<T>, KS = 4 * VEC, UN = RB + NT > 4 ? 1 : RB + NT > 3 ? 2 : 4, R = RB * 16;
  __shared__ float zs[WV][NT * 16][R + 1];
  const bool second = blockIdx.x >= q.j[0].blocks;
  const ShrinkJob& j = q.j[second];
  const int at = blockIdx.x - (second ? q.j[0].blocks : 0u);
  if (at >= q.plan.tile[q.adapters]) return;
  const int g = __builtin_amdgcn_readfirstlane(owner(q.plan.tile, q.adapters, at));
  const int p0 = q.plan.start[g] + NT * 16 * (at - q.plan.tile[g]), p1 = min(p0 + NT * 16, q.plan.start[g + 1]);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15,
            k4 = lane >> 4;
  const T *pb[NT], *pa[RB];
#pragma unroll
  for (int i = 0; i < NT; ++i) pb[i] = (const T*)j.x + (int64_t)q.plan.order[min(p0 + i * 16 + l16, p1 - 1)] * j.ldx;
#pragma unroll
  for (int i = 0; i < RB; ++i)
    pa[i] = (const T*)j.low + ((int64_t)g * q.rank + min(i * 16 + l16, q.rank - 1)) * j.lowld;
  floatx4 acc[RB][NT];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[i][n] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto steps = [&](int s, auto whole) {
    raw_vec<T> fa[UN][RB], fb[UN][NT];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int k = (s + u) * KS + k4 * VEC;
#pragma unroll
      for (int n = 0; n < NT; ++n) fb[u][n] = whole ? *(const any_vec<T>*)(pb[n] + k) : load_raw(pb[n], k, j.d);
#pragma unroll
      for (int i = 0; i < RB; ++i) fa[u][i] = whole ? *(const any_vec<T>*)(pa[i] + k) : load_raw(pa[i], k, j.d);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u)
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[i][n] = mfma_few(fa[u][i], fb[u][n], acc[i][n]);
  };
  const int full = j.d / KS;
  int s = wave * UN;
  for (; s + UN <= full; s += WV * UN) steps(s, std::true_type{});
  for (; s * KS < j.d; s += WV * UN) steps(s, std::false_type{});
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) zs[wave][n * 16 + l16][i * 16 + 4 * k4 + r] = acc[i][n][r];
  __syncthreads();
  const float f = q.factor ? q.factor[g] : 1.f;
  for (int e = threadIdx.x; e < NT * 16 * R; e += WV * 64) {
    const int row = e / R, c = e % R;
    if (p0 + row >= p1) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WV; w += 4)
      v += (zs[w][row][c] + zs[w + 1][row][c]) + (zs[w + 2][row][c] + zs[w + 3][row][c]);
    j.t[(int64_t)(p0 + row) * R + c] = c < q.rank ? v * f : 0.f;
  }
}

// Few rows, in their own order (no plan): a workgroup a row, its wavefronts the
// adapter's rows of the rank in turn.
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
    if (lane == 0) t[row * R + r] = s * f;
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
  int R;
  RowPlan plan;
  const int32_t* ids;
  void* y;
  int64_t ldy;
};

// CT x 16 columns of y by NT x 16 rows, from the rows as they are.
template <typename T, int CT, int NT, int WV>
__global__ __launch_bounds__(WV * 64) void direct_kernel(ProjectArgs a) {
  constexpr int VEC = kVec<T>, KS = 4 * VEC, UN = CT + NT > 4 ? 2 : 4;
  __shared__ float zs[WV][NT * 16][CT * 16 + 1];
  const unsigned across = (unsigned)((a.m + CT * 16 - 1) / (CT * 16));
  const int64_t v0 = (int64_t)(blockIdx.x % across) * (CT * 16), t0 = (int64_t)(blockIdx.x / across) * (NT * 16);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15,
            k4 = lane >> 4;
  const T *pa[CT], *pb[NT];
#pragma unroll
  for (int i = 0; i < CT; ++i) pa[i] = (const T*)a.w + min(v0 + i * 16 + l16, (int64_t)a.m - 1) * a.ldw;
#pragma unroll
  for (int i = 0; i < NT; ++i) pb[i] = (const T*)a.x + min(t0 + i * 16 + l16, a.n - 1) * a.ldx;
  floatx4 acc[CT][NT];
#pragma unroll
  for (int i = 0; i < CT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto steps = [&](int s, auto whole) {
    raw_vec<T> fa[UN][CT], fb[UN][NT];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int k = (s + u) * KS + k4 * VEC;
#pragma unroll
      for (int i = 0; i < CT; ++i) fa[u][i] = whole ? *(const any_vec<T>*)(pa[i] + k) : load_raw(pa[i], k, a.d);
#pragma unroll
      for (int i = 0; i < NT; ++i) fb[u][i] = whole ? *(const any_vec<T>*)(pb[i] + k) : load_raw(pb[i], k, a.d);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u)
#pragma unroll
      for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = mfma_few(fa[u][i], fb[u][j], acc[i][j]);
  };
  const int full = a.d / KS;
  int s = wave * UN;
  for (; s + UN <= full; s += WV * UN) steps(s, std::true_type{});
  for (; s * KS < a.d; s += WV * UN) steps(s, std::false_type{});
#pragma unroll
  for (int i = 0; i < CT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) zs[wave][j * 16 + l16][i * 16 + 4 * k4 + r] = acc[i][j][r];
  __syncthreads();
  for (int e = threadIdx.x; e < CT * NT * 256; e += WV * 64) {
    const int c = e % (CT * 16), t = e / (CT * 16);
    const int64_t col = v0 + c, row = t0 + t;
    if (col >= a.m || row >= a.n) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WV; w += 4) v += (zs[w][t][c] + zs[w + 1][t][c]) + (zs[w + 2][t][c] + zs[w + 3][t][c]);
    const int g = a.ids[row];
    if (g >= a.adapters) {
      v = __builtin_nanf("");
    } else if (g >= 0) {
      const T* up = (const T*)a.up + ((int64_t)g * a.m + col) * a.uld;
      const float* tr = a.t + (a.plan.place ? a.plan.place[row] : row) * a.R;
      float s0 = 0.f;
      for (int k = 0; k < a.rank; k += VEC) {
        float b[VEC];
        load_part(up, k, a.rank, b);
#pragma unroll
        for (int o = 0; o < VEC; ++o) s0 = fmaf(tr[k + o], b[o], s0);  // (t is zero from rank on)
      }
      v += s0;
    }
    ((T*)a.y)[row * a.ldy + col] = (T)v;
  }
}

// A tile of the sorted rows; the adapters of each 32 rows one after another.  Their
// products go into sums of their own, of which a row takes its adapter's: what
// another adapter holds, were it NaN, does not reach it.
struct TileProject {
  ProjectArgs a;
  Side x, w;
  int K, nkc, mt, nt;
  PairSide px, pw;       // fp32: pairs, each row at a power of two of its own
  const int *ex, *ew;
};
template <typename T, class S, class Rows>
__global__ __launch_bounds__(S::threads, S::per_cu) void project_kernel(TileProject q) {
  __shared__ __attribute__((aligned(1024))) char lds[S::lds_bytes];
  const ProjectArgs& a = q.a;
  int mi, ni;
  tile_of(blockIdx.x, (unsigned)(q.mt * q.nt), q.mt, q.nt, mi, ni);
  const int64_t r0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN;
  floatx16 acc[S::WM][S::WN];
  if constexpr (sizeof(T) == 4) {
    pair_product<S, 3>(q.px, q.pw, r0, n0, 0, q.nkc, lds, acc);
  } else {
    Rows rows;
    if constexpr (std::is_same<Rows, InOrder>::value) rows.order = a.plan.order;
    tile_product<T, S, Rows>(q.x, q.w, r0, n0, q.K, q.nkc, 1, 0, q.nkc, lds, acc, rows);
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::GN, wn = wave % S::GN, l32 = lane & 31, h = lane >> 5;
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi) {
    const int b0 = (int)r0 + (wm * S::WM + bi) * 32;
    if (b0 >= a.n) continue;
    const int b1 = (int)min((int64_t)b0 + 32, a.n);
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
    for (int p = b0; p < b1;) {
      const int g = __builtin_amdgcn_readfirstlane(a.plan.bucket[p]);
      const int e = min(__builtin_amdgcn_readfirstlane(a.plan.start[g + 1]), b1);
      if (g < a.adapters) {
        floatx16 low[S::WN];
#pragma unroll
        for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
          for (int r = 0; r < 16; ++r) low[bj][r] = 0.f;
        const float* tr = a.t + (int64_t)min(b0 + l32, b1 - 1) * a.R + h * (a.R / 2);
        for (int k = 0; k < a.R / 2; k += 8) {
          const floatx4 t0 = *(const floatx4*)(tr + k), t1 = *(const floatx4*)(tr + k + 4);
#pragma unroll
          for (int bj = 0; bj < S::WN; ++bj) {
            const int64_t col = min(n0 + (wn * S::WN + bj) * 32 + l32, (int64_t)a.m - 1);
            const T* up = (const T*)a.up + ((int64_t)g * a.m + col) * a.uld;
            const raw_n<8, T> u = load_n<8>(up, h * (a.R / 2) + k, a.rank);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              low[bj] = __builtin_amdgcn_mfma_f32_32x32x2f32(i < 4 ? t0[i & 3] : t1[i & 3], (float)u[i], low[bj], 0, 0, 0);
          }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int place = b0 + acc_row(r, h);
          if (place >= p && place < e)
#pragma unroll
            for (int bj = 0; bj < S::WN; ++bj) acc[bi][bj][r] += low[bj][r];
        }
      } else if (g > a.adapters) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int place = b0 + acc_row(r, h);
          if (place >= p && place < e)
#pragma unroll
            for (int bj = 0; bj < S::WN; ++bj) acc[bi][bj][r] = __builtin_nanf("");
        }
      }
      p = e;
    }
    int row[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) row[r] = a.plan.order[min(b0 + acc_row(r, h), b1 - 1)];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (b0 + acc_row(r, h) >= b1) continue;
#pragma unroll
      for (int bj = 0; bj < S::WN; ++bj) {
        const int64_t col = n0 + (wn * S::WN + bj) * 32 + l32;
        if (col < a.m) ((T*)a.y)[row[r] * a.ldy + col] = (T)acc[bi][bj][r];
      }
    }
  }
}

// Copies for the tiles, in sorted order where `order` is not null: 16-bit rows kp wide,
// zero from d on; fp32 rows as pairs, kp a whole number of blocks, each at the power of
// two that brings its largest entry to 2^14 .. 2^15 (`exps`): 22 bits of an entry down to
// 2^-17 of the row's largest, and 2^-40 of that below.  A row with an infinity or NaN is
// taken as it is.
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
      int e2 = 0;
      if (top > 0.f && __all(whole)) {
        (void)frexpf(top, &e2);
        e2 = 15 - e2;
      }
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
// fourth run of steps and join in LDS.
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
      const int place = p + u * 4 + k4;
      const bool use = place < p1;
      xn[u] = load_raw((const T*)j.X + (int64_t)row[u] * j.ldx, col, use ? j.d : 0);
#pragma unroll
      for (int t = 0; t < CT; ++t) cn[u][t] = use ? j.coef[(int64_t)place * q.R + s0 + t * 16 + l16] : 0.f;
    }
  };
  int p = p0 + wave * (4 * UN);
  find(p);
  fetch(p);
  find(p + 16 * UN);
  for (; p < p1; p += 16 * UN) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      x[u] = xn[u];
#pragma unroll
      for (int t = 0; t < CT; ++t) c[u][t] = cn[u][t];
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

// The pieces' sums, in order: ddown as it is, dup turned.
struct JoinArgs {
  const float *down_slabs, *up_slabs;
  int adapters, rank, d, m;
  const int32_t* piece;
  void *ddown, *dup;  // each may be null
};
// A workgroup has 64 columns of 8 rows of an adapter's rank, its wavefronts every fourth piece.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a) {
  __shared__ float red[4][8][64 + 1];
  const int rb = (a.rank + 7) / 8, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t per_d = a.ddown ? (int64_t)rb * ((a.d + 63) / 64) : 0, per_u = a.dup ? (int64_t)rb * ((a.m + 63) / 64) : 0;
  for (int64_t unit = blockIdx.x; unit < a.adapters * (per_d + per_u); unit += gridDim.x) {
    const bool up = unit >= a.adapters * per_d;
    const int64_t i = up ? unit - a.adapters * per_d : unit, per = up ? per_u : per_d, g = i / per, b = i - g * per;
    const int r0 = (int)(b % rb) * 8, width = up ? a.m : a.d;
    const int64_t c = b / rb * 64 + lane;
    const float* slabs = up ? a.up_slabs : a.down_slabs;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int k1 = a.piece[g + 1], rows = min(8, a.rank - r0);
    if (c < width)
#pragma unroll 2
      for (int k = a.piece[g] + wave; k < k1; k += 4) {
        const float* p = slabs + ((int64_t)k * a.rank + r0) * width + c;
#pragma unroll
        for (int r = 0; r < 8; ++r)
          if (r < rows) s[r] += p[(int64_t)r * width];
      }
#pragma unroll
    for (int r = 0; r < 8; ++r) red[wave][r][lane] = s[r];
    __syncthreads();
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      const int e = o * 256 + threadIdx.x, r = up ? e % 8 : e / 64, l = up ? e / 8 : e % 64;
      const int64_t col = b / rb * 64 + l;
      if (r >= rows || col >= width) continue;
      const float v = (red[0][r][l] + red[1][r][l]) + (red[2][r][l] + red[3][r][l]);
      if (up)
        ((T*)a.dup)[(g * a.m + col) * a.rank + r0 + r] = (T)v;
      else
        ((T*)a.ddown)[(g * a.rank + r0 + r) * a.d + col] = (T)v;
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

// A piece of an adapter's rows in `outer`: so many that the pieces fill the card
// about twice over, 64 at least.
int piece_of(const AdaptArgs& a) {
  const int64_t w = 16 * 16 / (int64_t)elem_bytes(a.type), across = cdiv(a.d, w) + cdiv(a.m, w);
  const int64_t pieces = std::max<int64_t>(1, 2048 / across);
  return (int)std::min<int64_t>(up_to(std::max<int64_t>(64, cdiv(a.n, pieces)), 16), 1 << 20);
}
int64_t most_pieces(const AdaptArgs& a) { return cdiv(a.n, piece_of(a)) + std::min<int64_t>(a.adapters, a.n); }

// One projection: whether it runs in tiles, and what copies that takes.
struct Way {
  bool tiled, big, gather, copy_x, copy_w;
  int kp;
};
Way way_of(int type, int64_t n, int d, int m, const void* x, int64_t ldx, const void* w, int64_t ldw, bool w_padded) {
  Way r{};
  r.tiled = n > 64 && m > 64 && (double)n * m * d > 2e9;
  r.kp = (int)up_to(d, type == TYPE_F32 ? kPairBlock : 8);
  auto fits = [&](const void* p, int64_t ld) {
    return type != TYPE_F32 && d % 8 == 0 && ld % 8 == 0 && ld < (1 << 21) && (uintptr_t)p % 16 == 0;
  };
  r.gather = fits(x, ldx) && n * ldx * 2 < 0x7fff0000;
  r.copy_x = !r.gather;
  r.copy_w = w_padded ? type == TYPE_F32 : !fits(w, ldw);  // (padded: whole rows of kp, zero from d on)
  r.big = cdiv(n, 256) * cdiv(m, 256) >= 128;
  return r;
}
// Rows of a tile of `shrink`: each reads its adapter's matrix once.
int shrink_rows(const AdaptArgs& a) { return a.n >= 4096 && a.n >= 64 * (int64_t)a.adapters && a.rank <= 64 ? 32 : 16; }
int64_t most_tiles(const AdaptArgs& a) { return cdiv(a.n, shrink_rows(a)) + std::min<int64_t>(a.adapters, a.n); }
constexpr int kFewRows = 64;  // so many rows take no plan: t in their own order

struct Scratch {
  RowPlan plan;
  float *t, *u;
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
  auto copies = [&](const Way& w, int64_t rows) {
    if (!w.tiled) return;
    const int64_t row = (int64_t)w.kp * size;
    if (w.copy_x) s.xc = l.take<char>(a.n * row);
    if (w.copy_w) s.wc = l.take<char>(rows * row);
    if (a.type == TYPE_F32) s.ex = l.take<int>(a.n), s.ew = l.take<int>(rows);
  };
  if (!grad) {
    copies(way_of(a.type, a.n, a.d, a.m, a.x, a.ldx, a.w, a.ldw, false), a.m);
  } else {
    s.u = l.take<float>(a.n * R);
    if (a.dx || a.ddown) s.upt = l.take<char>((int64_t)a.adapters * a.rank * a.m * size);
    if (a.dx) {
      s.downt = l.take<char>((int64_t)a.adapters * a.rank * a.d * size);
      s.wt = l.take<char>((int64_t)a.d * up_to(a.m, 8) * size);
      copies(way_of(a.type, a.n, a.m, a.d, a.dy, a.lddy, nullptr, 0, true), a.d);
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
  if (sizeof(T) == 2 && w.gather)
    project_kernel<T, S, InOrder><<<grid, S::threads, 0, s>>>(q);
  else
    project_kernel<T, S, AsTheyAre><<<grid, S::threads, 0, s>>>(q);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_project(const ProjectArgs& a, const Way& w, const Scratch& sc, hipStream_t s) {
  if (w.tiled) {
    if constexpr (sizeof(T) == 4)
      return w.big ? launch_tiles<T, PairShape<TileShape<2, 2, 4, 2>, 3>>(a, w, sc, s)
                   : launch_tiles<T, PairShape<TileShape<1, 2, 4, 2>, 4>>(a, w, sc, s);
    else
      return w.big ? launch_tiles<T, BigTile>(a, w, sc, s) : launch_tiles<T, SmallTile>(a, w, sc, s);
  }
  auto grid = [&](int ct, int nt) { return (unsigned)(cdiv(a.m, ct * 16) * cdiv(a.n, nt * 16)); };
  if (a.n <= 16)
    direct_kernel<T, 1, 1, 8><<<grid(1, 1), 512, 0, s>>>(a);
  else if (a.n <= 32)
    direct_kernel<T, 1, 2, 8><<<grid(1, 2), 512, 0, s>>>(a);
  else if (a.n <= 64)
    direct_kernel<T, 1, 4, 8><<<grid(1, 4), 512, 0, s>>>(a);
  else
    direct_kernel<T, 4, 2, 4><<<grid(4, 2), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int RB>
void launch_shrink_rank(const AdaptArgs& a, const ShrinkJobs& q, hipStream_t s) {
  const unsigned blocks = q.j[0].blocks + q.j[1].blocks;
  if constexpr (RB <= 4)
    if (shrink_rows(a) == 32) return (void)(shrink_kernel<T, RB, 2, 4><<<blocks, 256, 0, s>>>(q));
  // (by the call's sizes alone: a gradient has the same bits whether or not others are asked for)
  if (most_tiles(a) <= 256)  // few tiles: a workgroup's own time counts
    shrink_kernel<T, RB, 1, RB == 8 ? 8 : 16><<<blocks, RB == 8 ? 512 : 1024, 0, s>>>(q);
  else
    shrink_kernel<T, RB, 1, 4><<<blocks, 256, 0, s>>>(q);
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
    plan_kernel<<<1, kPlanWaves * 64, kPlanWaves * (a.adapters + 2) * sizeof(int), s>>>(
        a.ids, a.n, a.adapters, bits, shrink_rows(a), piece, sc.plan);
  }
  const unsigned tiles = (unsigned)most_tiles(a);
  ShrinkJobs sh{};
  sh.adapters = a.adapters;
  sh.rank = a.rank;
  sh.factor = a.factor;
  sh.plan = sc.plan;
  const ShrinkJob of_x = {a.x, a.ldx, a.d, a.down, a.d, sc.t, tiles};
  ProjectArgs p{};
  p.n = a.n;
  p.adapters = a.adapters;
  p.rank = a.rank;
  p.uld = a.rank;
  p.R = R;
  p.plan = sc.plan;
  p.ids = a.ids;
  if (!grad) {
    sh.j[0] = of_x;
    if (few) {
      p.plan.place = nullptr;
      shrink_rows_kernel<T><<<(unsigned)a.n, 1024, 0, s>>>((const T*)a.x, a.ldx, a.d, (const T*)a.down, a.adapters, a.rank,
                                                           R, a.ids, a.factor, sc.t);
    } else {
      launch_shrink<T>(a, sh, s);
    }
    p.x = a.x, p.ldx = a.ldx, p.d = a.d;
    p.w = a.w, p.ldw = a.ldw, p.m = a.m;
    p.up = a.up;
    p.t = sc.t;
    p.y = a.y, p.ldy = a.ldy;
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
  const ShrinkJob of_dy = {a.dy, a.lddy, a.m, sc.upt, a.m, sc.u, tiles};
  int count = 0;
  if (sc.upt) sh.j[count++] = of_dy;
  if (a.dup) sh.j[count++] = of_x;
  launch_shrink<T>(a, sh, s);
  if (a.dx) {
    p.x = a.dy, p.ldx = a.lddy, p.d = a.m;
    p.w = sc.wt, p.ldw = mp, p.m = a.d;
    p.up = sc.downt;
    p.t = sc.u;
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
  if (RB == 1)
    outer_kernel<T, 1><<<grid, 256, 0, s>>>(o);
  else if (RB == 2)
    outer_kernel<T, 2><<<grid, 256, 0, s>>>(o);
  else
    outer_kernel<T, 4><<<grid, 256, 0, s>>>(o);
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
