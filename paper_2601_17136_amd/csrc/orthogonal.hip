// An update orthogonalised by Newton-Schulz products.  With the short side as
// rows, X = u / (|u| + eps) and per step
//   A = X X^T,  X <- a X + (b A + c A^2) X,
// which brings X's singular values s to a s + b s^3 + c s^5 and keeps its singular
// vectors.  Two forms:
//
// flat (short side at most kFlat): every step is a polynomial of G = u u^T, so the
//   steps run on the S x S matrix alone, in LDS, and one product Q u ends them.  A
//   product of polynomials loses what iterated products of X keep (its small
//   singular values' accuracy is that of their squares), so G, the steps and Q u
//   are held in 64 bits, on the 64-bit matrix cores.  |u|^2 is G's trace.  What G's
//   roundings leave where a singular value is zero, of either sign, a step multiplies
//   by a^2 as well: after as many steps as multiply by 2^12 the X so far is stored, in
//   64 bits, and the next ones begin with its own G (Stages).
// tiled: X and X^T as pairs of binary16 parts (pair_tile.h), three launches a
//   step.  A and A^2 are symmetric, so only tiles on and above their diagonals are
//   multiplied.  Two parts hold 22 bits at a fixed power of two: a host-side bound
//   on the singular values after each step keeps every entry in range.  Measured
//   against 64 bits their error is 0.4 to 0.9 of that of fp32 products; of rows or
//   columns 1e-7 times the others it is 3 times, of 1e-9 times 300 times, since entries
//   end at 2^-50 of that bound.
//
// Microseconds, flat / tiled, fp32: 64 x 64 73 / 68, 64 x 784 102 / 94, 8 of 48 x 784 70 / 99,
// 64 x 4096 147 / 197, 33 x 50000 150 / 1579.
#include <algorithm>
#include <cmath>

#include "model_ops.h"
#include "pair_tile.h"
#include "vec_io.h"

namespace kkm {

namespace {

constexpr int kFlat = 64;
typedef double doublex4 __attribute__((ext_vector_type(4)));

// What is orthogonalised, entry by entry: x itself, or the momentum's step.
struct Source {
  const void* x;  // x, or the gradient
  int64_t ld, stride;
  float* v;       // null: x itself
  float momentum;
  int nesterov;
  int64_t m, n;
};
// What the flat form holds of an entry of type T.
template <typename T>
using flat_t = typename std::conditional<std::is_same<T, double>::value, double, float>::type;
// v's new value is written where `update`, else v holds it already.
template <typename T, bool UPDATE>
__device__ inline flat_t<T> entry(const Source& q, int64_t b, int64_t i, int64_t j) {
  const flat_t<T> g = (flat_t<T>)((const T*)q.x)[b * q.stride + i * q.ld + j];
  if constexpr (std::is_same<T, double>::value) return g;  // (an X between stages)
  if (!q.v) return g;
  float* p = q.v + (b * q.m + i) * q.n + j;
  float v = *p;
  if (UPDATE) {
    v = q.momentum * v + g;
    *p = v;
  }
  return q.nesterov ? g + q.momentum * v : v;
}

// Where the result goes: y, or w = keep w - rate O.
struct Target {
  void* y;
  int64_t ld, stride;
  int update;
  float rate, keep;
};
template <typename T, typename O>
__device__ inline void put(const Target& t, int64_t b, int64_t i, int64_t j, O o) {
  T* p = (T*)t.y + b * t.stride + i * t.ld + j;
  if constexpr (std::is_same<T, double>::value)
    *p = o;
  else
    *p = (T)(t.update ? t.keep * (float)*p - t.rate * (float)o : (float)o);
}
// `count` of 8 neighbouring entries of a row.
template <typename T>
__device__ inline void put(const Target& t, int64_t b, int64_t i, int64_t j, int count, const float (&o)[8]) {
  T* p = (T*)t.y + b * t.stride + i * t.ld + j;
  raw_n<8, T> v;
  if (t.update) {
    const raw_n<8, T> w = load_n<8>(p, 0, count);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (T)(t.keep * (float)w[k] - t.rate * o[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (T)o[k];
  }
  if (count == 8) {
    *(any_n<8, T>*)p = v;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < count) p[k] = v[k];
  }
}

// ------------------------------------------------------------------ flat

constexpr int kLong = 64, kLongLd = kLong + 4;  // long-side indices of a chunk; its padded rows in LDS

// The chunk [k0, k0 + 64) of the long side into u[short][long], zero elsewhere.
template <typename T, bool UPDATE, int SB, typename U>
__device__ inline void load_chunk(const Source& q, int64_t b, int64_t k0, bool tall, U (*u)[kLongLd]) {
  const int S = (int)(tall ? q.n : q.m);
  const int64_t len = tall ? q.m : q.n;
  for (int e = threadIdx.x; e < SB * 16 * kLong; e += 256) {
    const int i = tall ? e % (SB * 16) : e / kLong, k = tall ? e / (SB * 16) : e % kLong;
    U v = 0;
    if (i < S && k0 + k < len) v = tall ? entry<T, UPDATE>(q, b, k0 + k, i) : entry<T, UPDATE>(q, b, i, k0 + k);
    u[i][k] = v;
  }
}

// A slab of G: chunks [split * per, ..) of matrix blockIdx.y; the four wavefronts
// take 16 of a chunk's 64 indices each.  8 fp32 matrices of 8 x 784 4 us, most of it the
// launch, as of flat_apply.
template <typename T, int SB>
__global__ __launch_bounds__(256) void flat_gram_kernel(Source q, bool tall, int per, double* __restrict__ slabs) {
  constexpr int S16 = SB * 16;
  __shared__ union {
    flat_t<T> u[S16][kLongLd];
    double red[S16][S16];
  } lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
  const int64_t b = blockIdx.y, len = tall ? q.m : q.n;
  doublex4 acc[SB][SB];
#pragma unroll
  for (int i = 0; i < SB; ++i)
#pragma unroll
    for (int j = 0; j < SB; ++j) acc[i][j] = doublex4{0, 0, 0, 0};
  for (int c = 0; c < per; ++c) {
    const int64_t k0 = ((int64_t)blockIdx.x * per + c) * kLong;
    if (k0 >= len) break;
    __syncthreads();
    load_chunk<T, true, SB>(q, b, k0, tall, lds.u);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      double f[SB];
#pragma unroll
      for (int i = 0; i < SB; ++i) f[i] = lds.u[i * 16 + l16][wave * 16 + s * 4 + g];
#pragma unroll
      for (int i = 0; i < SB; ++i)
#pragma unroll
        for (int j = i; j < SB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f64_16x16x4f64(f[i], f[j], acc[i][j], 0, 0, 0);
    }
  }
  for (int o = 0; o < 4; ++o) {
    __syncthreads();
    if (wave == o)
#pragma unroll
      for (int i = 0; i < SB; ++i)
#pragma unroll
        for (int j = i; j < SB; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            double* p = &lds.red[i * 16 + g + 4 * r][j * 16 + l16];
            *p = o ? *p + acc[i][j][r] : acc[i][j][r];
          }
  }
  __syncthreads();
  double* out = slabs + (b * gridDim.x + blockIdx.x) * (S16 * S16);
  for (int e = threadIdx.x; e < S16 * S16; e += 256) {
    const int i = e / S16, j = e % S16;
    out[e] = i / 16 <= j / 16 ? lds.red[i][j] : lds.red[j][i];
  }
}

// C = A B of S16 x S16 matrices in LDS, of COUNT matrices A by one B, a wavefront's
// blocks at a time.  (They are symmetric but for roundings.  Products with B's rows in
// the place of its columns multiply what is not by up to 30 a step: 2e-10 off after six
// steps where these are 1e-13.)
template <int SB, int COUNT>
constexpr int kBlocks = (COUNT * SB * SB + 3) / 4;
template <int SB, int LD, int COUNT>
__device__ inline void square_products(const double* const (&A)[COUNT], const double* B,
                                       doublex4 (&acc)[kBlocks<SB, COUNT>]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < kBlocks<SB, COUNT>; ++t) {
    const int blk = t * 4 + wave, of = blk % (SB * SB);
    acc[t] = doublex4{0, 0, 0, 0};
    if (blk >= COUNT * SB * SB) continue;
    const double* pa = (COUNT > 1 && blk >= SB * SB ? A[COUNT - 1] : A[0]) + (of / SB * 16 + l16) * LD + g;
    const double* pb = B + g * LD + of % SB * 16 + l16;
#pragma unroll
    for (int k = 0; k < SB * 16; k += 4)
      acc[t] = __builtin_amdgcn_mfma_f64_16x16x4f64(pa[k], pb[k * LD], acc[t], 0, 0, 0);
  }
}
template <int SB, int LD, int COUNT, class F>
__device__ inline void each_entry(const doublex4 (&acc)[kBlocks<SB, COUNT>], F f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < kBlocks<SB, COUNT>; ++t) {
    const int blk = t * 4 + wave, of = blk % (SB * SB);
    if (blk >= COUNT * SB * SB) continue;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = of / SB * 16 + g + 4 * r, j = of % SB * 16 + l16;
      f(blk / (SB * SB), i, j, i * LD + j, acc[t][r]);
    }
  }
}

// The steps [s0, s1) on A = G alone, each by a I + R with R = b A + c A^2: q and Q with
// X_last = (q I + Q) X, X = u inv, inv returned (1 of an X between stages).  q stays
// apart because Q alone has no part where a singular value is zero.  Q's product and A's
// first are independent and run together.  Starts and ends with a barrier.
template <int SB, int LD>
__device__ inline double flat_steps(double* A, double* R, double* Q, const NewtonSteps& c, int s0, int s1, double eps,
                                    double& q) {
  constexpr int S16 = SB * 16;
  __syncthreads();
  double inv = 1;
  if (s0 == 0) {
    double tr = 0;
#pragma unroll
    for (int i = 0; i < S16; ++i) tr += A[i * LD + i];
    inv = 1.0 / fmax(sqrt(tr) + eps, 1e-100);  // (fp32's smallest is 1e-45: of a zero matrix and eps below)
    __syncthreads();
    for (int e = threadIdx.x; e < S16 * S16; e += 256) A[e / S16 * LD + e % S16] *= inv * inv;
    __syncthreads();
  }
  doublex4 one[kBlocks<SB, 1>], two[kBlocks<SB, 2>];
  q = 1;
  for (int s = s0; s < s1; ++s) {
    const bool first = s == s0, last = s + 1 == s1;
    square_products<SB, LD, 1>({A}, A, one);
    const double ca = c.coef[3 * s], cb = c.coef[3 * s + 1], cc = c.coef[3 * s + 2];
    each_entry<SB, LD, 1>(one, [&](int, int, int, int at, double v) {
      R[at] = cb * A[at] + cc * v;
      if (first) Q[at] = R[at];
    });
    __syncthreads();
    // q I + Q <- (q I + Q) (a I + R), A <- A (a I + R)^2
    auto onto_q = [&](int at, double v) { Q[at] = q * R[at] + (ca * Q[at] + v); };
    auto onto_a = [&](int at, double v) { A[at] = ca * A[at] + v; };
    if (!first && !last) {
      square_products<SB, LD, 2>({Q, A}, R, two);
      __syncthreads();
      each_entry<SB, LD, 2>(two, [&](int which, int, int, int at, double v) {
        if (which)
          onto_a(at, v);
        else
          onto_q(at, v);
      });
      __syncthreads();
    } else if (!first || !last) {
      square_products<SB, LD, 1>({first ? A : Q}, R, one);
      __syncthreads();
      each_entry<SB, LD, 1>(one, [&](int, int, int, int at, double v) {
        if (first)
          onto_a(at, v);
        else
          onto_q(at, v);
      });
      __syncthreads();
    }
    q *= ca;
    if (last) break;
    square_products<SB, LD, 1>({A}, R, one);
    __syncthreads();
    each_entry<SB, LD, 1>(one, [&](int, int, int, int at, double v) { onto_a(at, v); });
    __syncthreads();
  }
  return inv;
}

// The steps of a stage by themselves, of a G in slabs: inv Q and inv q.  Bound by the
// chain of products in one workgroup: five steps of 16 x 16 9.3 us, of 64 x 64 54.
template <int SB>
__global__ __launch_bounds__(256) void flat_steps_kernel(const double* __restrict__ slabs, int count, NewtonSteps c,
                                                         int s0, int s1, double eps, double* __restrict__ out,
                                                         double* __restrict__ out_q) {
  constexpr int S16 = SB * 16, LD = S16 + 2;
  __shared__ double A[S16 * LD], R[S16 * LD], Q[S16 * LD];
  const int64_t b = blockIdx.x;
  for (int e = threadIdx.x; e < S16 * S16; e += 256) {
    double s = 0;
#pragma unroll 8
    for (int k = 0; k < count; ++k) s += slabs[(b * count + k) * (S16 * S16) + e];
    A[e / S16 * LD + e % S16] = s;
  }
  double q;
  const double inv = flat_steps<SB, LD>(A, R, Q, c, s0, s1, eps, q);
  if (threadIdx.x == 0) out_q[b] = q * inv;
  for (int e = threadIdx.x; e < S16 * S16; e += 256) out[b * (S16 * S16) + e] = Q[e / S16 * LD + e % S16] * inv;
}

// O = q u + Q u, a chunk of the long side at a time; a wavefront has 16 of its indices.
// (O may lie on u: a workgroup reads and writes its own chunks.)
template <typename T, int SB, typename OT>
__global__ __launch_bounds__(256) void flat_apply_kernel(Source q, bool tall, const double* __restrict__ Qs,
                                                         const double* __restrict__ qs, Target out) {
  constexpr int S16 = SB * 16, LD = S16 + 2;
  using U = typename std::conditional<std::is_same<OT, double>::value, double, flat_t<T>>::type;
  __shared__ U u[S16][kLongLd];
  __shared__ double Q[S16 * LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4;
  const int64_t b = blockIdx.y, len = tall ? q.m : q.n;
  const int S = (int)(tall ? q.n : q.m);
  const double whole = qs[b];
  for (int e = threadIdx.x; e < S16 * S16; e += 256) Q[e / S16 * LD + e % S16] = Qs[b * (S16 * S16) + e];
  for (int64_t k0 = (int64_t)blockIdx.x * kLong; k0 < len; k0 += (int64_t)gridDim.x * kLong) {
    __syncthreads();
    load_chunk<T, false, SB>(q, b, k0, tall, u);
    __syncthreads();
    doublex4 acc[SB];
#pragma unroll
    for (int i = 0; i < SB; ++i) acc[i] = doublex4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < S16; j += 4) {
      const double f = u[j + g][wave * 16 + l16];
#pragma unroll
      for (int i = 0; i < SB; ++i)
        acc[i] = __builtin_amdgcn_mfma_f64_16x16x4f64(Q[(i * 16 + l16) * LD + j + g], f, acc[i], 0, 0, 0);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SB; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        U& v = u[i * 16 + g + 4 * r][wave * 16 + l16];
        v = (U)(whole * (double)v + acc[i][r]);
      }
    __syncthreads();
    for (int e = threadIdx.x; e < S16 * kLong; e += 256) {
      const int i = tall ? e % S16 : e / kLong, k = tall ? e / S16 : e % kLong;
      if (i >= S || k0 + k >= len) continue;
      if (tall)
        put<OT>(out, b, k0 + k, i, u[i][k]);
      else
        put<OT>(out, b, i, k0 + k, u[i][k]);
    }
  }
}

// ------------------------------------------------------------------ tiled

// Eight entries of u, the row's from j on (zero past its end).
template <typename T, bool UPDATE>
__device__ inline void entries(const Source& q, int64_t b, int64_t i, int64_t j, float (&u)[8]) {
  const int left = (int)min(q.n - j, (int64_t)8);
  const raw_n<8, T> g = load_n<8>((const T*)q.x + b * q.stride + i * q.ld + j, 0, left);
#pragma unroll
  for (int k = 0; k < 8; ++k) u[k] = (float)g[k];
  if (!q.v) return;
  float* p = q.v + (b * q.m + i) * q.n + j;
  raw_n<8, float> v = load_n<8>(p, 0, left);
  if (UPDATE) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = q.momentum * v[k] + u[k];
    if (left == 8) {
      *(any_n<8, float>*)p = v;
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < left) p[k] = v[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) u[k] = q.nesterov ? u[k] + q.momentum * v[k] : v[k];
}

// Sums of squares, a grid apart, in 64 bits; the momentum's new values.  4096 x 4096
// bfloat16 30 us, 5.6 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void squares_kernel(Source q, double* __restrict__ part) {
  __shared__ double red[4];
  const int64_t b = blockIdx.y, per = (q.n + 7) / 8;
  double s = 0;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < q.m * per; e += (int64_t)gridDim.x * 256) {
    float u[8];
    entries<T, true>(q, b, e / per, e % per * 8, u);
#pragma unroll
    for (int k = 0; k < 8; ++k) s += (double)u[k] * (double)u[k];
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[b * gridDim.x + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// Pairs of u / (|u| + eps), 2^exp times: `along`'s rows are u's, `across`'s its columns.
// 4096 x 4096 bfloat16 50 us, 4.7 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void pairs_kernel(Source q, const double* __restrict__ part, int count, double eps,
                                                    float up, half_t* along, int64_t ld_along, half_t* across,
                                                    int64_t ld_across) {
  __shared__ float tile[64][65];
  __shared__ double red[4];
  const int64_t b = blockIdx.z, i0 = (int64_t)blockIdx.y * 64, j0 = (int64_t)blockIdx.x * 64;
  double s = 0;
  for (int k = threadIdx.x; k < count; k += 256) s += part[b * count + k];
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  const double norm = sqrt((red[0] + red[1]) + (red[2] + red[3])) + eps;
  for (int e = threadIdx.x; e < 64 * 8; e += 256) {
    const int lr = e / 8, lc = e % 8 * 8;
    const int64_t i = i0 + lr, j = j0 + lc;
    float u[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (i < q.m && j < q.n) entries<T, false>(q, b, i, j, u);
    f16x8 hi, lo;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float v = j + k < q.n ? (float)((double)u[k] / norm) * up : 0.f;
      tile[lr][lc + k] = v;
      half_t x, y;
      split_pair(v, x, y);
      hi[k] = x, lo[k] = y;
    }
    if (i < q.m && j < ld_along / 2) {
      half_t* p = along + (b * q.m + i) * ld_along + pair_at(j);
      *(f16x8*)p = hi;
      *(f16x8*)(p + kPairBlock) = lo;
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 64 * 8; e += 256) {
    const int lc = e / 8, lr = e % 8 * 8;
    const int64_t c = j0 + lc, r = i0 + lr;
    if (c >= q.n || r >= ld_across / 2) continue;
    f16x8 hi, lo;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      half_t x, y;
      split_pair(tile[lr + k][lc], x, y);
      hi[k] = x, lo[k] = y;
    }
    half_t* p = across + (b * q.n + c) * ld_across + pair_at(r);
    *(f16x8*)p = hi;
    *(f16x8*)(p + kPairBlock) = lo;
  }
}

// A tile's entries v = ca base + cm acc, base a pair matrix of the product's own
// rows and columns (null: none).  Stored as pairs in the same order (`along`), in
// the other (`across`), or as the result.
struct TileArgs {
  PairSide a, b;
  int64_t stride_a, stride_b;  // of a matrix of the batch
  int64_t M, N;
  int nkb, mt, nt;
  bool half;                   // symmetric: tiles on and above the diagonal's blocks of BM x BM
  const half_t* base;
  int64_t ld_base, stride_base;
  float ca, cm;                // what base's and the sums' stored values are multiplied by
  half_t *along, *across;
  int64_t ld_along, ld_across, stride_along, stride_across;
  Target out;
  // The first `whole` tiles run whole; of the others' `splits` parts of the contraction
  // each, the sums go to slabs, and a second launch joins and stores them.
  int whole, splits;
  float* slabs;
};

// A symmetric product's tiles, R times as high as wide: of row tile i those from its
// block of the diagonal on.  In bands of 8 row tiles by their columns, of which the
// first are as high as the diagonal leaves them; an XCD has a contiguous run, as
// tile_of's.
constexpr int kBand = 8;
template <int R>
__host__ __device__ inline int band_tiles(int b, int mt, int nt) {  // of band b
  const int p = mt - b * kBand < kBand ? mt - b * kBand : kBand, cols = nt - R * kBand * b;
  // (row i of the band has R i columns less; the last may have none of a wider tile's)
  return p * cols - R * (p * (p - 1) / 2);
}
template <int R>
__device__ inline void half_tile_of(unsigned g, unsigned total, int mt, int nt, int& mi, int& ni) {
  const unsigned per = total >> 3, rem = total & 7, x = g & 7;
  int t = (int)(x * per + min(x, rem) + (g >> 3)), b = 0;
  for (int n = band_tiles<R>(0, mt, nt); t >= n; n = band_tiles<R>(++b, mt, nt)) t -= n;
  const int p = min(kBand, mt - b * kBand), low = R * (p * (p - 1) / 2);  // tiles of columns lower than p
  int c, r;
  if (t < low) {
    int k = 1;  // R columns of height k
    while (t >= R * k) t -= R * k++;
    c = R * (k - 1) + t / k;
    r = t % k;
  } else {
    c = R * (p - 1) + (t - low) / p;
    r = (t - low) % p;
  }
  mi = __builtin_amdgcn_readfirstlane(b * kBand + r);
  ni = __builtin_amdgcn_readfirstlane(R * kBand * b + c);
}

// Bound by the matrix cores where tiles fill the card (4096 square, three products of
// parts: a square in 186 us, matrix cores busy 78 %; X's product 345, 1.2 PFLOP/s of
// binary16 products), by a launch's own time where they do not: 1024 x 784 11.5 us a launch,
// of which its blocks take 5.
// The sums pass through LDS, 32 rows of each of the workgroup's GM at a time, so that
// base is read and every result written 16 bytes a lane, whole 128-byte blocks in both
// orders.
template <class S, bool LAST, bool JOIN, typename OT>
__global__ __launch_bounds__(S::threads, S::per_cu) void pair_kernel(TileArgs q) {
  constexpr int LD = S::BN + 4, ROWS = S::GM * 32, kRatio = S::BM / S::BN;
  static_assert(S::BM % S::BN == 0, "the diagonal's tiles");
  constexpr int kBytes = S::lds_bytes > ROWS * LD * 4 ? S::lds_bytes : ROWS * LD * 4;
  __shared__ __attribute__((aligned(1024))) char lds[kBytes];
  const int64_t bt = blockIdx.y;
  int mi, ni;
  const unsigned tiles = (unsigned)(q.half ? q.mt * q.nt - kRatio * (q.mt * (q.mt - 1) / 2) : q.mt * q.nt);
  const int past = (int)blockIdx.x + (JOIN ? q.whole : 0) - q.whole;  // parts, or tiles, beyond the whole ones
  const unsigned tile = past < 0 ? blockIdx.x : q.whole + (JOIN ? past : past / q.splits);
  if (q.half)
    half_tile_of<kRatio>(tile, tiles, q.mt, q.nt, mi, ni);
  else
    tile_of(tile, tiles, q.mt, q.nt, mi, ni);
  const int64_t r0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN;
  // (JOIN: a workgroup has one of WM times 32 GM rows of a tile)
  constexpr int BI = JOIN ? 1 : S::WM;
  const int bi0 = JOIN ? (int)blockIdx.z : 0;
  floatx16 acc[BI][S::WN];
  constexpr int64_t kTile = (int64_t)S::BM * S::BN;
  // a thread's own sums, a workgroup apart
  float* slab = q.slabs + (bt * ((int)tiles - q.whole) * q.splits + (JOIN ? past * q.splits : past)) * kTile + threadIdx.x;
  auto each = [&](auto f) {
#pragma unroll
    for (int bi = 0; bi < BI; ++bi)
#pragma unroll
      for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          acc[bi][bj][r] = f(acc[bi][bj][r], (((bi0 + bi) * S::WN + bj) * 16 + r) * S::threads);
  };
  if constexpr (JOIN) {
    each([&](float, int at) { return slab[at]; });
#pragma unroll 2
    for (int k = 1; k < q.splits; ++k)
      each([&](float v, int at) { return v + slab[k * kTile + at]; });
  } else {
    PairSide a = q.a, b = q.b;
    a.p += bt * q.stride_a;
    b.p += bt * q.stride_b;
    const int part = past < 0 ? 0 : past % q.splits, parts = past < 0 ? 1 : q.splits;
    pair_product<S>(a, b, r0, n0, q.nkb * part / parts, q.nkb * (part + 1) / parts, lds, acc);
    if (past >= 0) {
      each([&](float v, int at) { return slab[at] = v; });
      return;
    }
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::GN, wn = wave % S::GN, l32 = lane & 31, h = lane >> 5;
  const half_t* base = q.base ? q.base + bt * q.stride_base : nullptr;
  half_t* along = q.along ? q.along + bt * q.stride_along : nullptr;
  half_t* across = q.across ? q.across + bt * q.stride_across : nullptr;
  const bool turned = !q.half || ni >= (mi + 1) * kRatio;  // (the diagonal's blocks are whole as they are)
  float* sums = (float*)lds;
#pragma unroll
  for (int own = 0; own < BI; ++own) {
    const int bi = bi0 + own;
    if (own) __syncthreads();
#pragma unroll
    for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        sums[(wm * 32 + acc_row(r, h)) * LD + (wn * S::WN + bj) * 32 + l32] = acc[own][bj][r];
    __syncthreads();
#pragma unroll
    for (int e = threadIdx.x; e < ROWS * (S::BN / 8); e += S::threads) {
      const int lr = e / (S::BN / 8), lc = e % (S::BN / 8) * 8;
      const int64_t row = r0 + (lr / 32 * S::WM + bi) * 32 + lr % 32, col = n0 + lc;
      float* p = sums + lr * LD + lc;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p[k] * q.cm;
      const bool in = row < q.M && col < q.N;
      if (base && in) {
        const half_t* from = base + row * q.ld_base + pair_at(col);
        const f16x8 hi = *(const f16x8*)from, lo = *(const f16x8*)(from + kPairBlock);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += q.ca * join_pair(hi[k], lo[k]);
      }
      if constexpr (LAST) {
        if (in) put<OT>(q.out, bt, row, col, (int)min(q.N - col, (int64_t)8), v);
      } else {
        f16x8 hi, lo;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (!(row < q.M && col + k < q.N)) v[k] = 0.f;
          half_t x, y;
          split_pair(v[k], x, y);
          hi[k] = x, lo[k] = y;
          p[k] = v[k];
        }
        if (row < q.M && col < q.ld_along / 2) {
          half_t* to = along + row * q.ld_along + pair_at(col);
          *(f16x8*)to = hi;
          *(f16x8*)(to + kPairBlock) = lo;
        }
      }
    }
    if constexpr (!LAST) {
      __syncthreads();
      if (turned)
#pragma unroll
        for (int e = threadIdx.x; e < S::BN * (ROWS / 8); e += S::threads) {
          // four neighbouring lanes have 32 rows of a column
          const int lc = e / 4 % S::BN, lr = (e / 4 / S::BN * 4 + e % 4) * 8;
          const int64_t row = r0 + (lr / 32 * S::WM + bi) * 32 + lr % 32, col = n0 + lc;
          if (col >= q.N || row >= q.ld_across / 2) continue;
          f16x8 hi, lo;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            half_t x, y;
            split_pair(sums[(lr + k) * LD + lc], x, y);
            hi[k] = x, lo[k] = y;
          }
          half_t* to = across + col * q.ld_across + pair_at(row);
          *(f16x8*)to = hi;
          *(f16x8*)(to + kPairBlock) = lo;
        }
    }
  }
}

// ------------------------------------------------------------------ host

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t align(size_t v) { return (v + 255) / 256 * 256; }

int flat_splits(const OrthoArgs& a) {
  const int64_t chunks = cdiv(std::max(a.m, a.n), kLong);
  return (int)std::min<int64_t>({chunks, std::max<int64_t>(1, 512 / a.batch), 64});
}
int flat_side(const OrthoArgs& a) { return (int)cdiv(std::min(a.m, a.n), 16); }
bool is_flat(const OrthoArgs& a) { return std::min(a.m, a.n) <= kFlat; }
// Stages of steps: as many together as let no zero singular value's rest grow past 2^12
// times a rounding, and that X's own roundings, which q I and Q take from each other, past
// 2^12 of theirs.  Duplicate rows and 32 steps of 3.4445: 1e-12 off; in one stage from
// the 16th on by as much as the result.
constexpr double kStageGrowth = 4096;
int stage_end(const NewtonSteps& c, int s0) {
  double grown = 1;
  for (int s = s0; s < c.steps; ++s) {
    grown *= std::max(1.0, std::fabs(c.coef[3 * s]));
    if (s > s0 && grown > kStageGrowth) return s;
  }
  return c.steps;
}
constexpr size_t kFlatBytes = (size_t)1 << 28;  // scratch of the matrices of a launch, about
int64_t flat_bytes(const OrthoArgs& a) {
  const int64_t kept = stage_end(a.newton, 0) < a.newton.steps ? a.m * a.n : 0;
  return ((int64_t)(flat_splits(a) + 1) * flat_side(a) * flat_side(a) * 256 + 1 + kept) * (int64_t)sizeof(double);
}
int64_t flat_group(const OrthoArgs& a) {
  return std::min<int64_t>({a.batch, 65535, std::max<int64_t>(1, (int64_t)kFlatBytes / flat_bytes(a))});
}

Source source_of(const OrthoArgs& a, int64_t b0) {
  const size_t size = elem_bytes(a.type);
  return Source{(const char*)a.x + b0 * a.stride_x * size, a.ldx, a.stride_x, a.v ? a.v + b0 * a.m * a.n : nullptr,
                a.momentum, a.nesterov, a.m, a.n};
}
Target target_of(const OrthoArgs& a, int64_t b0) {
  return Target{(char*)a.y + b0 * a.stride_y * elem_bytes(a.type), a.ldy, a.stride_y, a.v != nullptr, a.rate, a.keep};
}

template <typename T, int SB>
hipError_t launch_flat(const OrthoArgs& a, void* scratch, hipStream_t s) {
  const int splits = flat_splits(a);
  const bool tall = a.m > a.n;
  const int64_t chunks = cdiv(std::max(a.m, a.n), kLong);
  const int per = (int)cdiv(chunks, splits);
  const int64_t group = flat_group(a);
  double* slabs = (double*)scratch;
  double* Q = slabs + group * splits * (SB * SB * 256);
  double* q = Q + group * (SB * SB * 256);
  double* kept = q + group;  // the X between stages
  const Source between{kept, a.n, a.m * a.n, nullptr, 0.f, 0, a.m, a.n};
  const Target keep{kept, a.n, a.m * a.n, 0, 0.f, 0.f};
  const unsigned across = (unsigned)std::min<int64_t>(chunks, std::max<int64_t>(1, 2048 / std::min<int64_t>(a.batch, 2048)));
  for (int64_t b0 = 0; b0 < a.batch; b0 += group) {
    const unsigned nb = (unsigned)std::min(group, a.batch - b0);
    for (int s0 = 0, s1; s0 < a.newton.steps; s0 = s1) {
      s1 = stage_end(a.newton, s0);
      const bool last = s1 == a.newton.steps;
      auto stage = [&](auto from, const Source& src) {
        using F = decltype(from);
        flat_gram_kernel<F, SB><<<dim3(splits, nb), 256, 0, s>>>(src, tall, per, slabs);
        flat_steps_kernel<SB><<<nb, 256, 0, s>>>(slabs, splits, a.newton, s0, s1, a.eps, Q, q);
        if (last)
          flat_apply_kernel<F, SB, T><<<dim3(across, nb), 256, 0, s>>>(src, tall, Q, q, target_of(a, b0));
        else
          flat_apply_kernel<F, SB, double><<<dim3(across, nb), 256, 0, s>>>(src, tall, Q, q, keep);
      };
      if (s0 == 0)
        stage(T{}, source_of(a, b0));
      else
        stage(double{}, between);
    }
  }
  return hipGetLastError();
}

// The largest magnitude of a s + b s^3 + c s^5 over [0, top], with some room: at the end
// or where the derivative, a + 3 b q + 5 c q^2 with q = s^2, is zero.
double largest(double a, double b, double c, double top) {
  auto at = [&](double q) { return std::fabs(std::sqrt(q) * (a + q * (b + q * c))); };
  double most = at(top * top);
  double roots[2] = {-1, -1};
  if (c != 0) {
    const double d = 9 * b * b - 20 * a * c;
    if (d >= 0)
      for (int i = 0; i < 2; ++i) roots[i] = (-3 * b + (i ? 1 : -1) * std::sqrt(d)) / (10 * c);
  } else if (b != 0) {
    roots[0] = -a / (3 * b);
  }
  for (double q : roots)
    if (q > 0 && q < top * top) most = std::max(most, at(q));
  return most * 1.01 + 1e-6;
}
// That of b q + c q^2 over [0, top^2]: of B's eigenvalues.
double largest_even(double b, double c, double top) {
  const double end = top * top, q = c != 0 ? -b / (2 * c) : -1;
  double most = std::fabs(end * (b + end * c));
  if (q > 0 && q < end) most = std::max(most, std::fabs(q * (b + q * c)));
  return most * 1.01 + 1e-6;
}
int room_for(double top) { return 15 - std::max(-30, (int)std::ceil(std::log2(top))); }

// The tiles of a launch, and what it takes with them, in microseconds: `end`, and a
// block's time in a full round of 256 tiles and in one of few.  Measured, a Gram matrix
// and X's product of 4096 / 3000 / 2048 / 1024 square: 256 x 128 288 / 98 / 66 / 35 and 345 /
// 204 / 71 / 34, 128 x 128 269 / 114 / 39 / 22 and 395 / 182 / 52 / 21, 128 x 64 254 / 106 / 44 /
// 18 and 415 / 177 / 56 / 17, 64 x 64 268 / 110 / 46 / 14 and 475 / 194 / 64 / 13.
using Pair256x128 = TileShape<2, 2, 4, 2, 3>;   // 144 KB
using Pair128 = TileShape<1, 2, 4, 2, 4>;       // 128 KB
using Pair128x64 = TileShape<2, 1, 2, 2, 3>;    // 72 KB
using Pair64 = TileShape<1, 1, 2, 2, 4>;        // 64 KB
struct PairCost {
  double end, alone, full;
};
// How a launch runs: in which tiles, how many of them whole, and the parts of the
// others (1: none), by what it takes.  The tiles past the last full round of 256 leave
// most CUs idle for a round's time; in parts they take a share of it and a second
// launch.  A Gram matrix of 4096 in 272 tiles of 256 x 128 288 us, in 256 and 16 of 8 parts
// each 182 and 12.
struct PairRun {
  int shape, whole, splits;
  int64_t slab;  // floats
};
template <class S>
void consider(int shape, const PairCost& c, const TileArgs& q, unsigned nb, double& best, PairRun& run) {
  const int64_t mt = cdiv(q.M, S::BM), nt = cdiv(q.N, S::BN);
  const int64_t tiles = q.half ? mt * nt - S::BM / S::BN * (mt * (mt - 1) / 2) : mt * nt;
  const double all = (double)nb * tiles / 256, rounds = std::floor(all), left = all - rounds;
  auto take = [&](double t, int64_t whole, int splits) {
    if (run.splits && t >= best) return;
    best = t;
    run = {shape, (int)whole, splits, splits > 1 ? (tiles - whole) * splits * nb * S::BM * S::BN : 0};
  };
  auto round = [&](double part) { return part > 0 ? c.alone + (c.full - c.alone) * part * part * part : 0; };
  take(c.end + q.nkb * (rounds * c.full + round(left)), tiles, 1);
  if (nb != 1 || rounds < 1 || left == 0) return;
  const int64_t whole = (int64_t)rounds * 256;
  for (int splits = 2; splits <= 8 && left * splits <= 1 && q.nkb / splits >= 4; ++splits)
    take(c.end + q.nkb * (rounds * c.full + round(left * splits) / splits) + 10 + splits * (S::BM * S::BN * 4e-5 / S::WM),
         whole, splits);
}
PairRun pair_run(const TileArgs& q, unsigned nb) {
  PairRun run{};
  double best = 0;
  consider<Pair256x128>(0, {7, 0.85, 1.35}, q, nb, best, run);
  consider<Pair128>(1, {6, 0.5, 0.73}, q, nb, best, run);
  consider<Pair128x64>(2, {6, 0.33, 0.39}, q, nb, best, run);
  consider<Pair64>(3, {6, 0.2, 0.225}, q, nb, best, run);
  return run;
}
template <class S, bool LAST, typename OT>
void launch_shape(TileArgs q, const PairRun& run, unsigned nb, hipStream_t s) {
  q.mt = (int)cdiv(q.M, S::BM);
  q.nt = (int)cdiv(q.N, S::BN);
  q.whole = run.whole;
  q.splits = run.splits;
  const int tiles = q.half ? q.mt * q.nt - S::BM / S::BN * (q.mt * (q.mt - 1) / 2) : q.mt * q.nt;
  const unsigned blocks = (unsigned)(run.whole + (tiles - run.whole) * run.splits);
  pair_kernel<S, LAST, false, OT><<<dim3(blocks, nb), S::threads, 0, s>>>(q);
  if (run.whole < tiles)
    pair_kernel<S, LAST, true, OT><<<dim3((unsigned)(tiles - run.whole), nb, S::WM), S::threads, 0, s>>>(q);
}
template <bool LAST, typename OT>
void launch_pair(const TileArgs& q, unsigned nb, hipStream_t s) {
  const PairRun run = pair_run(q, nb);
  switch (run.shape) {
    case 0: return launch_shape<Pair256x128, LAST, OT>(q, run, nb, s);
    case 1: return launch_shape<Pair128, LAST, OT>(q, run, nb, s);
    case 2: return launch_shape<Pair128x64, LAST, OT>(q, run, nb, s);
    default: return launch_shape<Pair64, LAST, OT>(q, run, nb, s);
  }
}

// The tiled form's layout for one group of matrices.
struct TiledPlan {
  int64_t S, len;     // short and long side
  int64_t ldx, ldxt;  // of X (S rows) and X^T (len rows)
  int64_t group;      // matrices at a time
  int parts;
  size_t x, xt, a, norm, slabs, total;  // bytes of one buffer each, and of all
};
constexpr size_t kGroupBytes = (size_t)1 << 30;
TiledPlan tiled_plan(const OrthoArgs& a) {
  TiledPlan p;
  p.S = std::min(a.m, a.n);
  p.len = std::max(a.m, a.n);
  p.ldx = pair_ld(p.len);
  p.ldxt = pair_ld(p.S);
  p.parts = (int)std::min<int64_t>(cdiv(a.m * cdiv(a.n, 8), 256), 1024);
  const size_t one = (size_t)(2 * p.S * p.ldx + 2 * p.len * p.ldxt + 2 * p.S * p.ldxt) * sizeof(half_t);
  p.group = std::max<int64_t>(1, std::min<int64_t>({a.batch, (int64_t)(kGroupBytes / one), 65535}));
  p.x = align((size_t)p.group * p.S * p.ldx * sizeof(half_t));
  p.xt = align((size_t)p.group * p.len * p.ldxt * sizeof(half_t));
  p.a = align((size_t)p.group * p.S * p.ldxt * sizeof(half_t));
  p.norm = align((size_t)p.group * p.parts * sizeof(double));
  // the largest of the launches' slabs (only of a matrix by itself)
  p.slabs = 0;
  for (int k = 0; k < 4; ++k) {
    TileArgs q{};
    q.half = k < 2;
    q.M = k == 3 ? p.len : p.S;
    q.N = k == 2 ? p.len : p.S;
    q.nkb = (int)((k == 0 ? p.ldx : p.ldxt) / (2 * kPairBlock));
    p.slabs = std::max(p.slabs, align((size_t)pair_run(q, 1).slab * sizeof(float)));
  }
  p.total = 2 * (p.x + p.xt + p.a) + p.norm + p.slabs;
  return p;
}

template <typename T>
hipError_t launch_tiled(const OrthoArgs& a, void* scratch, hipStream_t s) {
  const TiledPlan p = tiled_plan(a);
  const bool tall = a.m > a.n;
  char* at = (char*)scratch;
  auto take = [&](size_t bytes) {
    half_t* q = (half_t*)at;
    at += bytes;
    return q;
  };
  half_t *X[2], *XT[2];
  for (int i = 0; i < 2; ++i) X[i] = take(p.x), XT[i] = take(p.xt);
  half_t *A = take(p.a), *B = take(p.a);
  double* norm = (double*)take(p.norm);
  float* slabs = (float*)at;
  const int64_t sx = p.S * p.ldx, sxt = p.len * p.ldxt, sa = p.S * p.ldxt;
  for (int64_t b0 = 0; b0 < a.batch; b0 += p.group) {
    const unsigned nb = (unsigned)std::min(p.group, a.batch - b0);
    const Source src = source_of(a, b0);
    squares_kernel<T><<<dim3(p.parts, nb), 256, 0, s>>>(src, norm);
    double top = 1.01;  // of X's singular values, and so of its entries
    int ex = room_for(top);
    half_t *along = tall ? XT[0] : X[0], *across = tall ? X[0] : XT[0];
    pairs_kernel<T><<<dim3((unsigned)cdiv(a.n, 64), (unsigned)cdiv(a.m, 64), nb), 256, 0, s>>>(
        src, norm, p.parts, a.eps, std::ldexp(1.f, ex), along, tall ? p.ldxt : p.ldx, across, tall ? p.ldx : p.ldxt);
    for (int t = 0; t < a.newton.steps; ++t) {
      const half_t *x = X[t & 1], *xt = XT[t & 1];
      const double ca = a.newton.coef[3 * t], cb = a.newton.coef[3 * t + 1], cc = a.newton.coef[3 * t + 2];
      const int eb = room_for(largest_even(cb, cc, top)), ea = cc == 0 ? eb : room_for(top * top);
      TileArgs g{};
      g.slabs = slabs;
      g.a = g.b = {x, p.ldx, p.S};
      g.stride_a = g.stride_b = sx;
      g.M = g.N = p.S;
      g.nkb = (int)(p.ldx / (2 * kPairBlock));
      g.half = true;
      g.cm = (float)std::ldexp(cc == 0 ? cb : 1.0, ea - 2 * ex);
      g.along = g.across = cc == 0 ? B : A;
      g.ld_along = g.ld_across = p.ldxt;
      g.stride_along = g.stride_across = sa;
      launch_pair<false, float>(g, nb, s);
      if (cc != 0) {
        g.a = g.b = {A, p.ldxt, p.S};
        g.stride_a = g.stride_b = sa;
        g.nkb = (int)(p.ldxt / (2 * kPairBlock));
        g.base = A;
        g.ld_base = p.ldxt;
        g.stride_base = sa;
        g.ca = (float)std::ldexp(cb, eb - ea);
        g.cm = (float)std::ldexp(cc, eb - 2 * ea);
        g.along = g.across = B;
        launch_pair<false, float>(g, nb, s);
      }
      const bool last = t + 1 == a.newton.steps;
      top = largest(ca, cb, cc, top);
      const int en = last ? 0 : room_for(top);  // the result is stored as it is
      TileArgs m{};
      m.slabs = slabs;
      const PairSide sb = {B, p.ldxt, p.S}, sxs = {xt, p.ldxt, p.len};
      const bool turned = last && tall;  // the result's rows are the long side
      m.a = turned ? sxs : sb;
      m.b = turned ? sb : sxs;
      m.stride_a = turned ? sxt : sa;
      m.stride_b = turned ? sa : sxt;
      m.M = turned ? p.len : p.S;
      m.N = turned ? p.S : p.len;
      m.nkb = (int)(p.ldxt / (2 * kPairBlock));
      m.base = turned ? xt : x;
      m.ld_base = turned ? p.ldxt : p.ldx;
      m.stride_base = turned ? sxt : sx;
      m.ca = (float)std::ldexp(ca, en - ex);
      m.cm = (float)std::ldexp(1.0, en - eb - ex);
      if (last) {
        m.out = target_of(a, b0);
        launch_pair<true, T>(m, nb, s);
      } else {
        m.along = X[(t + 1) & 1];
        m.ld_along = p.ldx;
        m.stride_along = sx;
        m.across = XT[(t + 1) & 1];
        m.ld_across = p.ldxt;
        m.stride_across = sxt;
        launch_pair<false, float>(m, nb, s);
      }
      ex = en;
    }
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const OrthoArgs& a, void* scratch, hipStream_t s) {
  if (!is_flat(a)) return launch_tiled<T>(a, scratch, s);
  switch (flat_side(a)) {
    case 1: return launch_flat<T, 1>(a, scratch, s);
    case 2: return launch_flat<T, 2>(a, scratch, s);
    case 3: return launch_flat<T, 3>(a, scratch, s);
    default: return launch_flat<T, 4>(a, scratch, s);
  }
}

}  // namespace

// The bound on the singular values after every step that the tiled form's powers
// of two rest on; false where it is not finite or past 2^12.
bool newton_in_range(const NewtonSteps& c) {
  double top = 1.01;
  for (int t = 0; t < c.steps; ++t) {
    top = largest(c.coef[3 * t], c.coef[3 * t + 1], c.coef[3 * t + 2], top);
    if (!(top <= 4096)) return false;
  }
  return true;
}

size_t ortho_scratch(const OrthoArgs& a) {
  if (a.batch == 0) return 0;
  if (!is_flat(a)) return tiled_plan(a).total;
  return (size_t)(flat_group(a) * flat_bytes(a));
}

hipError_t launch_ortho(const OrthoArgs& a, void* scratch, hipStream_t s) {
  if (a.batch == 0) return hipSuccess;
  if (a.type == TYPE_F32) return launch_typed<float>(a, scratch, s);
  return a.type == TYPE_F16 ? launch_typed<half_t>(a, scratch, s) : launch_typed<bf16_t>(a, scratch, s);
}

}  // namespace kkm
