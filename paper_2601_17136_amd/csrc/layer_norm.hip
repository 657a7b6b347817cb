// Layer norm and its gradient.
//
//   mu = mean x, r = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) r, y = xh w + b
//   g = dy w,  dx = r (g - mean g - xh mean(g xh)),  dw = sum_i dy xh,  db = sum_i dy
//
// Both are bound by memory: x in and y out; x and dy in and dx out.  A row
// lives in the registers of its T threads (a wavefront up to 4 vectors a lane,
// then a workgroup of 256), so it is read once.  The mean is taken twice: what the
// first sum's rounding left of it is the mean of x - mu, summed beside the squares,
// and both it and its square are taken off.  Rows of one value so have xh = 0;
// with the first mean alone 1000 values of 30000 gave xh = -0.5.  A group goes over
// rows a grid apart and keeps its columns' w and b, and in the gradient the fp32
// sums of dw and db, in registers; a workgroup's sums go to its line of the
// scratch, and a second launch adds the lines in order, so the gradient's bits do
// not depend on timing.  Rows wider than the registers take a loop over the row
// per pass instead.
#include <algorithm>
#include <type_traits>

#include "model_ops.h"
#include "vec_io.h"

namespace kkm {

namespace {

constexpr int kThreads = 256;

// Workgroups, at most: a narrow row needs many for the bytes in flight, wider
// ones gain from w and b loaded once, and in the gradient from fewer lines of
// sums, one a workgroup.  Microseconds at 2048 / 1024 workgroups, forward: 40001
// binary16 rows of 301 19 / 23; 8231 bfloat16 rows of 744 12 / 10; 3961 fp32 rows
// of 7880 54 / 48.  At 1024 / 512, the gradient: 28 / 46, 20 / 16, 112 / 97.
int wgs_fwd(int d) { return d <= 512 ? 2048 : 1024; }
int wgs_grad(int d) { return d <= 512 ? 1024 : 512; }

// v and w summed over the T threads of a row; T = 256: through red, one of two
// halves used in turn, so that one barrier suffices.
template <int T>
__device__ inline void row_sums(float& v, float& w, float (*red)[2][4], int& turn) {
  v = wave_sum(v);
  w = wave_sum(w);
  if (T > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      red[turn][0][wave] = v;
      red[turn][1][wave] = w;
    }
    __syncthreads();
    v = (red[turn][0][0] + red[turn][0][1]) + (red[turn][0][2] + red[turn][0][3]);
    w = (red[turn][1][0] + red[turn][1][1]) + (red[turn][1][2] + red[turn][1][3]);
    turn ^= 1;
  }
}
template <int T>
__device__ inline float row_sum(float v, float (*red)[2][4], int& turn) {
  v = wave_sum(v);
  if (T > 64) {
    if ((threadIdx.x & 63) == 0) red[turn][0][threadIdx.x >> 6] = v;
    __syncthreads();
    v = (red[turn][0][0] + red[turn][0][1]) + (red[turn][0][2] + red[turn][0][3]);
    turn ^= 1;
  }
  return v;
}

// 1 / sqrt(variance + eps) of squares about a mean that is off by `left`.
__device__ inline float inverse_deviation(float squares, float left, float eps) {
  const float var = squares - left * left;
  return 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);  // (a NaN stays one)
}

// Forward, x read once: 20000 fp32 rows of 784 21 us, 6.0 TB/s of what it must read
// and write; 16384 bfloat16 rows of 4096 44 us, 6.1 TB/s; 40001 binary16 rows of
// 301 18 to 19 us, 2.6 TB/s (38 of a wavefront's 64 lanes have features there).
template <typename XT, typename WT, int T, int NV>
__global__ __launch_bounds__(kThreads) void layer_norm_kernel(const XT* __restrict__ x, int64_t ldx,
                                                              const WT* __restrict__ w, const WT* __restrict__ b,
                                                              float eps, int64_t n, int d, XT* __restrict__ y,
                                                              int64_t ldy, float* __restrict__ mean,
                                                              float* __restrict__ rstd) {
  constexpr int VEC = kVec<XT>;
  __shared__ float red[2][2][4];
  int turn = 0;
  const int t = threadIdx.x % T;
  const int64_t step = (int64_t)gridDim.x * (kThreads / T);
  int64_t row = (int64_t)blockIdx.x * (kThreads / T) + threadIdx.x / T;
  float wv[NV][VEC], bv[NV][VEC];
  raw_vec<XT> next[NV];  // the next row, on its way while this one is summed
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int j = 0; j < NV; ++j) next[j] = load_raw(x + r * ldx, (j * T + t) * VEC, d);
  };
  if (row < n) fetch(row);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    load_beside<VEC>(w, (j * T + t) * VEC, d, 1.f, wv[j]);
    load_beside<VEC>(b, (j * T + t) * VEC, d, 0.f, bv[j]);
  }
  const float inv_d = 1.f / (float)d;
  for (; row < n; row += step) {
    float v[NV][VEC], s = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      to_floats<XT>(next[j], v[j]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += v[j][e];
    }
    if (row + step < n) fetch(row + step);
    const float mu = row_sum<T>(s, red, turn) * inv_d;
    float q = 0.f, left = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        v[j][e] = (j * T + t) * VEC + e < d ? v[j][e] - mu : 0.f;
        q = fmaf(v[j][e], v[j][e], q);
        left += v[j][e];
      }
    row_sums<T>(q, left, red, turn);
    left *= inv_d;
    const float r = inverse_deviation(q * inv_d, left, eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] = fmaf((v[j][e] - left) * r, wv[j][e], bv[j][e]);
      store_part(y + row * ldy, (j * T + t) * VEC, d, o);
    }
    if (t == 0) {
      if (mean) mean[row] = mu + left;
      if (rstd) rstd[row] = r;
    }
  }
}

// Gradient, x and dy read once: the same rows in 35 us, 5.4 TB/s; 89 us, 4.5 TB/s;
// 30 us, 2.4 TB/s.  The sums over the rows cost it the lines besides: 17 MB
// written for the bfloat16 rows.
template <typename XT, typename WT, int T, int NV>
__global__ __launch_bounds__(kThreads) void layer_norm_grad_kernel(
    const XT* __restrict__ x, int64_t ldx, const WT* __restrict__ w, const float* __restrict__ mean,
    const float* __restrict__ rstd, const XT* __restrict__ dy, int64_t lddy, int64_t n, int d, XT* __restrict__ dx,
    int64_t lddx, float* __restrict__ lines, WT* __restrict__ dw, WT* __restrict__ db) {
  constexpr int VEC = kVec<XT>, G = kThreads / T;
  __shared__ float red[2][2][4];
  __shared__ float part[G > 1 ? T * NV * VEC : 1];
  int turn = 0;
  const int t = threadIdx.x % T, grp = threadIdx.x / T;
  const int64_t step = (int64_t)gridDim.x * G;
  int64_t row = (int64_t)blockIdx.x * G + grp;
  float wv[NV][VEC], sw[NV][VEC], sb[NV][VEC], mun = 0.f, rn = 0.f;
  raw_vec<XT> xn[NV], gn[NV];  // the next row, on its way while this one is summed
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      xn[j] = load_raw(x + r * ldx, (j * T + t) * VEC, d);
      gn[j] = load_raw(dy + r * lddy, (j * T + t) * VEC, d);
    }
    mun = mean[r];
    rn = rstd[r];
  };
  if (row < n) fetch(row);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    load_beside<VEC>(w, (j * T + t) * VEC, d, 1.f, wv[j]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) sw[j][e] = sb[j][e] = 0.f;
  }
  const float inv_d = 1.f / (float)d;
  for (; row < n; row += step) {
    const float mu = mun, r = rn;
    float xh[NV][VEC], g[NV][VEC], s = 0.f, q = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float dv[VEC];
      to_floats<XT>(xn[j], xh[j]);
      to_floats<XT>(gn[j], dv);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        xh[j][e] = (j * T + t) * VEC + e < d ? (xh[j][e] - mu) * r : 0.f;
        g[j][e] = dv[e] * wv[j][e];
        sw[j][e] = fmaf(dv[e], xh[j][e], sw[j][e]);
        sb[j][e] += dv[e];
        s += g[j][e];
        q = fmaf(g[j][e], xh[j][e], q);
      }
    }
    if (row + step < n) fetch(row + step);
    row_sums<T>(s, q, red, turn);
    s *= inv_d;
    q *= inv_d;
    if (dx) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float o[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = r * (g[j][e] - s - xh[j][e] * q);
        store_part(dx + row * lddx, (j * T + t) * VEC, d, o);
      }
    }
  }
  if (!lines) return;
  // the workgroup's line, dw in the first d, db in the next (or, of the only one,
  // dw and db); its groups add up in order
  float* line = lines + (int64_t)blockIdx.x * 2 * d;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    auto mine = [&](int j, int e) { return k ? sb[j][e] : sw[j][e]; };
    if (G > 1) {
      for (int o = 0; o < G; ++o) {
        __syncthreads();
        if (grp == o)
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              float* p = part + (j * VEC + e) * T + t;
              *p = o ? *p + mine(j, e) : mine(j, e);
            }
      }
      __syncthreads();
    }
    if (grp == 0)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int i = (j * T + t) * VEC + e;
          if (i >= d) continue;
          const float v = G > 1 ? part[(j * VEC + e) * T + t] : mine(j, e);
          WT* out = k ? db : dw;
          if (gridDim.x > 1) line[(int64_t)k * d + i] = v;
          else if (out) out[i] = (WT)v;
        }
  }
}

// dw and db from the lines: a workgroup takes 64 of the 2 d columns, its
// sixteen wavefronts every sixteenth line.  4 to 5 us at the sizes above, of which
// most is the launch; 41 for 40000 columns.
template <typename WT>
__global__ __launch_bounds__(1024) void norm_lines_kernel(const float* __restrict__ lines, int nlines, int d,
                                                          WT* __restrict__ dw, WT* __restrict__ db) {
  __shared__ float part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < 2 * (int64_t)d) {
    float a[8] = {};
    int l = wave;
    for (; l + 112 < nlines; l += 128)
#pragma unroll
      for (int u = 0; u < 8; ++u) a[u] += lines[(int64_t)(l + 16 * u) * 2 * d + c];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (l + 16 * u < nlines) a[u] += lines[(int64_t)(l + 16 * u) * 2 * d + c];
    s = ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
  }
  part[wave][lane] = s;
  __syncthreads();
  if (wave || c >= 2 * (int64_t)d) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += part[w][lane];
  if (c < d) {
    if (dw) dw[c] = (WT)s;
  } else if (db) {
    db[c - d] = (WT)s;
  }
}

// Rows too wide for the registers: a workgroup per row and a pass over it for
// the mean, the variance and the result (from the second on out of L2).  2000 rows
// of 40000: fp32 231 us, 2.8 TB/s of x and y; bfloat16 113 us, 2.8.
template <typename XT, typename WT>
__global__ __launch_bounds__(kThreads) void layer_norm_wide_kernel(const XT* __restrict__ x, int64_t ldx,
                                                                   const WT* __restrict__ w,
                                                                   const WT* __restrict__ b, float eps, int64_t n,
                                                                   int d, XT* __restrict__ y, int64_t ldy,
                                                                   float* __restrict__ mean,
                                                                   float* __restrict__ rstd) {
  constexpr int VEC = kVec<XT>;
  __shared__ float red[2][2][4];
  int turn = 0;
  const float inv_d = 1.f / (float)d;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const XT* xr = x + row * ldx;
    float s = 0.f, q = 0.f, left = 0.f, v[VEC];
    for (int i = threadIdx.x * VEC; i < d; i += kThreads * VEC) {
      load_part(xr, i, d, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) s += v[e];
    }
    const float mu = row_sum<256>(s, red, turn) * inv_d;
    for (int i = threadIdx.x * VEC; i < d; i += kThreads * VEC) {
      load_part(xr, i, d, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float c = i + e < d ? v[e] - mu : 0.f;
        q = fmaf(c, c, q);
        left += c;
      }
    }
    row_sums<256>(q, left, red, turn);
    left *= inv_d;
    const float r = inverse_deviation(q * inv_d, left, eps);
    for (int i = threadIdx.x * VEC; i < d; i += kThreads * VEC) {
      float wv[VEC], bv[VEC];
      load_part(xr, i, d, v);
      load_beside<VEC>(w, i, d, 1.f, wv);
      load_beside<VEC>(b, i, d, 0.f, bv);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = fmaf((v[e] - mu - left) * r, wv[e], bv[e]);
      store_part(y + row * ldy, i, d, v);
    }
    if (threadIdx.x == 0) {
      if (mean) mean[row] = mu + left;
      if (rstd) rstd[row] = r;
    }
  }
}

// dx of the wide rows, a workgroup per row as above.  2000 rows of 40000: fp32 296 us,
// 3.2 TB/s of x, dy and dx; bfloat16 132, 3.6.
template <typename XT, typename WT>
__global__ __launch_bounds__(kThreads) void layer_norm_grad_wide_kernel(
    const XT* __restrict__ x, int64_t ldx, const WT* __restrict__ w, const float* __restrict__ mean,
    const float* __restrict__ rstd, const XT* __restrict__ dy, int64_t lddy, int64_t n, int d, XT* __restrict__ dx,
    int64_t lddx) {
  constexpr int VEC = kVec<XT>;
  __shared__ float red[2][2][4];
  int turn = 0;
  const float inv_d = 1.f / (float)d;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const float mu = mean[row], r = rstd[row];
    float s = 0.f, q = 0.f, v[VEC], g[VEC], wv[VEC];
    for (int i = threadIdx.x * VEC; i < d; i += kThreads * VEC) {
      load_part(x + row * ldx, i, d, v);
      load_part(dy + row * lddy, i, d, g);
      load_beside<VEC>(w, i, d, 1.f, wv);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float a = g[e] * wv[e];
        s += a;
        q = fmaf(a, (v[e] - mu) * r, q);
      }
    }
    row_sums<256>(s, q, red, turn);
    s *= inv_d;
    q *= inv_d;
    for (int i = threadIdx.x * VEC; i < d; i += kThreads * VEC) {
      load_part(x + row * ldx, i, d, v);
      load_part(dy + row * lddy, i, d, g);
      load_beside<VEC>(w, i, d, 1.f, wv);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = r * (g[e] * wv[e] - s - (v[e] - mu) * r * q);
      store_part(dx + row * lddx, i, d, v);
    }
  }
}

// The wide rows' lines: workgroup (c, l) sums 256 columns over every gridDim.y-th
// row.  2000 rows of 40000: fp32 160 us, 4.0 TB/s; bfloat16 139 us, 2.3.
template <typename XT>
__global__ __launch_bounds__(kThreads) void norm_cols_wide_kernel(const XT* __restrict__ x, int64_t ldx,
                                                                  const float* __restrict__ mean,
                                                                  const float* __restrict__ rstd,
                                                                  const XT* __restrict__ dy, int64_t lddy, int64_t n,
                                                                  int d, float* __restrict__ lines) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= d) return;
  float sw = 0.f, sb = 0.f;
  for (int64_t row = blockIdx.y; row < n; row += gridDim.y) {
    const float g = (float)dy[row * lddy + c];
    sw = fmaf(g, ((float)x[row * ldx + c] - mean[row]) * rstd[row], sw);
    sb += g;
  }
  float* line = lines + (int64_t)blockIdx.y * 2 * d;
  line[c] = sw;
  line[d + c] = sb;
}

// f(T, NV) for the narrowest rows in registers that hold d elements, up to 32
// a thread (the gradient's sums, w and two rows take 200 registers then), or
// f(0, 0) where none does.
template <int N>
using width = std::integral_constant<int, N>;
template <int VEC, typename F>
void by_width(int d, F&& f) {
  auto with = [&](auto t, auto nv) {
    if (d > t * nv * VEC) return false;
    f(t, nv);
    return true;
  };
  if (with(width<64>{}, width<1>{}) || with(width<64>{}, width<2>{}) || with(width<64>{}, width<4>{}) ||
      with(width<256>{}, width<2>{}) || with(width<256>{}, width<4>{}))
    return;
  if constexpr (VEC <= 4)
    if (with(width<256>{}, width<8>{})) return;
  f(width<0>{}, width<0>{});
}

template <typename XT, typename WT>
hipError_t norm_typed(const NormArgs& a, hipStream_t s) {
  by_width<kVec<XT>>(a.d, [&](auto t_, auto nv_) {
    constexpr int T = decltype(t_)::value, NV = decltype(nv_)::value;
    if constexpr (T == 0) {
      hipLaunchKernelGGL((layer_norm_wide_kernel<XT, WT>), dim3((unsigned)std::min<int64_t>(a.n, wgs_fwd(a.d))),
                         dim3(kThreads), 0, s, (const XT*)a.x, a.ldx, (const WT*)a.w, (const WT*)a.b, a.eps, a.n, a.d,
                         (XT*)a.y, a.ldy, a.mean, a.rstd);
    } else {
      const int64_t wgs = (a.n + kThreads / T - 1) / (kThreads / T);
      hipLaunchKernelGGL((layer_norm_kernel<XT, WT, T, NV>), dim3((unsigned)std::min<int64_t>(wgs, wgs_fwd(a.d))),
                         dim3(kThreads), 0, s, (const XT*)a.x, a.ldx, (const WT*)a.w, (const WT*)a.b, a.eps, a.n, a.d,
                         (XT*)a.y, a.ldy, a.mean, a.rstd);
    }
  });
  return hipGetLastError();
}

template <typename XT, typename WT>
hipError_t norm_grad_typed(const NormArgs& a, float* lines, hipStream_t s) {
  const bool sums = a.dw || a.db;
  int nlines = norm_lines(a.n, a.d);
  if (a.n > 0) by_width<kVec<XT>>(a.d, [&](auto t_, auto nv_) {
    constexpr int T = decltype(t_)::value, NV = decltype(nv_)::value;
    if constexpr (T == 0) {
      // the sums first: dx may lie over dy or x
      if (sums)
        hipLaunchKernelGGL((norm_cols_wide_kernel<XT>),
                           dim3((unsigned)((a.d + kThreads - 1) / kThreads), (unsigned)nlines), dim3(kThreads), 0, s,
                           (const XT*)a.x, a.ldx, a.mean, a.rstd, (const XT*)a.dy, a.lddy, a.n, a.d, lines);
      if (a.dx)
        hipLaunchKernelGGL((layer_norm_grad_wide_kernel<XT, WT>), dim3((unsigned)std::min<int64_t>(a.n, wgs_fwd(a.d))),
                           dim3(kThreads), 0, s, (const XT*)a.x, a.ldx, (const WT*)a.w, a.mean, a.rstd,
                           (const XT*)a.dy, a.lddy, a.n, a.d, (XT*)a.dx, a.lddx);
    } else {
      const int64_t groups = kThreads / T;
      nlines = (int)std::min<int64_t>(nlines, (a.n + groups - 1) / groups);
      hipLaunchKernelGGL((layer_norm_grad_kernel<XT, WT, T, NV>), dim3((unsigned)nlines), dim3(kThreads), 0, s,
                         (const XT*)a.x, a.ldx, (const WT*)a.w, a.mean, a.rstd, (const XT*)a.dy, a.lddy, a.n, a.d,
                         (XT*)a.dx, a.lddx, sums ? lines : nullptr, (WT*)a.dw, (WT*)a.db);
      if (nlines == 1) nlines = -1;  // one workgroup needs no second launch
    }
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !sums || nlines < 0) return e;
  hipLaunchKernelGGL((norm_lines_kernel<WT>), dim3((unsigned)((2 * (int64_t)a.d + 63) / 64)), dim3(1024), 0, s,
                     lines, nlines, a.d, (WT*)a.dw, (WT*)a.db);
  return hipGetLastError();
}

template <typename F>
hipError_t by_types(const NormArgs& a, F&& f) {
  switch (a.type) {
    case TYPE_F32: return f(float{}, float{});
    case TYPE_F16: return a.wtype == TYPE_F32 ? f(half_t{}, float{}) : f(half_t{}, half_t{});
    default: return a.wtype == TYPE_F32 ? f(bf16_t{}, float{}) : f(bf16_t{}, bf16_t{});
  }
}

}  // namespace

int norm_lines(int64_t n, int d) { return (int)std::min<int64_t>(n, wgs_grad(d)); }
size_t norm_scratch(int64_t n, int d) { return (size_t)norm_lines(n, d) * 2 * (size_t)d * sizeof(float); }

hipError_t launch_layer_norm(const NormArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  return by_types(a, [&](auto x, auto w) { return norm_typed<decltype(x), decltype(w)>(a, s); });
}

// lines: norm_scratch(n, d) bytes, or null where neither dw nor db is wanted.
// n = 0: dw and db become 0.
hipError_t launch_layer_norm_grad(const NormArgs& a, float* lines, hipStream_t s) {
  return by_types(a, [&](auto x, auto w) { return norm_grad_typed<decltype(x), decltype(w)>(a, lines, s); });
}

}  // namespace kkm
