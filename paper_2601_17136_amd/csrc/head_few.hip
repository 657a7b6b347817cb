// The class head where one side of it is short (at most kFew classes, or at most
// kFew rows of h), and where there is little work.  No operand is copied or
// padded: lanes load 16 bytes of a row each, in the shape the 16 x 16 matrix
// instructions take them, and every sum and G stay in fp32.  With a short side
// the scores are a matrix of S <= kFew columns, and the work is to read h (or w)
// and write its gradient once.
//
//   few classes:  scores_few (G = softmax less targets, [n][S]), then dW = G^T H
//                 (cols_few, reads H once more) and dH = G W (rows_few)
//   few rows:     scores_few (the scores Z, [classes][S]), targets_few (lse, loss),
//                 grad_few (Z becomes G^T), then dW = G^T H (rows_few) and
//                 dH = G W (cols_few, reads W once more)
//   little work:  scores_direct (Z, [n][classes]), row_direct (lse, loss, Z becomes
//                 G), then dW (cols_few) and dH (rows_direct)
//
// Both gradients are one launch, grads_few, and their sums over slabs another.
// (Z is S scores per class beside the d values of its row of w.)
#include <algorithm>
#include <type_traits>

#include "head_pairs.h"
#include "model_ops.h"
#include "vec_io.h"

namespace kkm {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
typedef float floatx4 __attribute__((ext_vector_type(4)));

// The products of 16 bytes of each row: a lane's elements of row lane % 16 at
// k = kVec * (lane / 16) + e.  fp32: four instructions of 4 k each, one per e.
__device__ inline floatx4 mfma_few(raw_vec<float> a, raw_vec<float> b, floatx4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}
__device__ inline floatx4 mfma_few(raw_vec<half_t> a, raw_vec<half_t> b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ inline floatx4 mfma_few(raw_vec<bf16_t> a, raw_vec<bf16_t> b, floatx4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

struct FewArgs {
  const void *h, *w;
  int64_t ldh, ldw, n;
  int d, classes, m;
  float zscale, scale, tscale;  // zscale: scale log2 e
  const float* offset;
  const int32_t* ids;
  const float *tlogits, *dloss;
  float *loss, *lse, *lse2, *coef;
  float* C;       // G [n][S], or Z and G^T [classes][S]
  float2* part;   // few rows: [class tile][n]
  int32_t* fix_id;
  float* fix_val;
};

// z in base 2 of CT x NT blocks of 16 classes by 16 rows of h into zs[row][class],
// the workgroup's four wavefronts taking every fourth run of UN steps of the
// features, so that one reads 256 neighbouring bytes of a row at a time.
// -inf where a class is left out or past the last.
template <typename XT, int CT, int NT>
__device__ inline void scores_block(const FewArgs& a, int64_t v0, int64_t t0, float (*zs)[NT * 16][CT * 16 + 1]) {
  constexpr int VEC = kVec<XT>, KS = 4 * VEC, UN = CT + NT > 4 ? 2 : 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const XT *pa[CT], *pb[NT];
#pragma unroll
  for (int i = 0; i < CT; ++i)
    pa[i] = (const XT*)a.w + min(v0 + i * 16 + l16, (int64_t)a.classes - 1) * a.ldw;
#pragma unroll
  for (int i = 0; i < NT; ++i) pb[i] = (const XT*)a.h + min(t0 + i * 16 + l16, a.n - 1) * a.ldh;
  floatx4 acc[CT][NT];
#pragma unroll
  for (int i = 0; i < CT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto steps = [&](int s, auto whole) {
    raw_vec<XT> fa[UN][CT], fb[UN][NT];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int k = (s + u) * KS + g * VEC;
#pragma unroll
      for (int i = 0; i < CT; ++i)
        fa[u][i] = whole ? *(const any_vec<XT>*)(pa[i] + k) : load_raw(pa[i], k, a.d);
#pragma unroll
      for (int i = 0; i < NT; ++i)
        fb[u][i] = whole ? *(const any_vec<XT>*)(pb[i] + k) : load_raw(pb[i], k, a.d);
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
  for (; s + UN <= full; s += 4 * UN) steps(s, std::true_type{});
  for (; s * KS < a.d; s += 4 * UN) steps(s, std::false_type{});
#pragma unroll
  for (int i = 0; i < CT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) zs[wave][j * 16 + l16][i * 16 + 4 * g + r] = acc[i][j][r];
  __syncthreads();
  for (int x = threadIdx.x; x < CT * NT * 256; x += 256) {
    const int c = x % (CT * 16), t = x / (CT * 16);
    const int64_t v = v0 + c;
    const float off = v >= a.classes ? -INFINITY : a.offset ? a.offset[v] * kLog2e : 0.f;
    const float z = (zs[0][t][c] + zs[1][t][c]) + (zs[2][t][c] + zs[3][t][c]);
    zs[0][t][c] = off == -INFINITY ? -INFINITY : fmaf(z, a.zscale, off);
  }
  __syncthreads();
}

// sums and maxima over P neighbouring lanes
template <int P>
__device__ inline float near_sum(float v) {
#pragma unroll
  for (int o = P / 2; o; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
template <int P>
__device__ inline float near_max(float v) {
#pragma unroll
  for (int o = P / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ inline float safe(float m) { return m == -INFINITY ? 0.f : m; }
__device__ inline float pair_key(const FewArgs& a, int64_t at, int& id, bool& bad) {
  return kkm::pair_key(a.ids, a.tlogits, at, a.tscale, a.classes, id, bad);
}

// Few classes: 32 rows of h by all classes; eight lanes finish a row, lane p
// owning the classes c % 8 = p, so that no two add to one target.  Few
// are bound by reading h: 60000 fp32 rows of 780, 10 classes, 59 us with G, 3.2
// TB/s, the loss alone 37, 5.0 TB/s.  64 of them by the fp32 matrix instructions:
// 20000 rows of 784 36 us, 56 TFLOP/s (a pass of 38.9 us is one of 42.5 if held to
// three wavefronts a SIMD; the others may be).  dH
// in this launch as well, from G in LDS, read w again for every 32 rows and was
// slower in 45 of 47 cases: those two with gradient 158 / 148 and 121 / 111, 200 rows
// of 64 and 20 classes 22.6 / 19.0, but 20000 bfloat16 rows of 2048, 64 classes 185 /
// 196.
template <typename XT, int CT>
__global__ __launch_bounds__(256, CT == 4 && sizeof(XT) == 4 ? 1 : 3) void scores_few_classes_kernel(FewArgs a) {
  constexpr int NT = 2, S = CT * 16;
  __shared__ float zs[4][NT * 16][S + 1];
  const int64_t t0 = (int64_t)blockIdx.x * (NT * 16);
  const int row = threadIdx.x >> 3, p = threadIdx.x & 7;
  const int64_t i = t0 + row;
  // the first eight pairs and the row's factor, loaded ahead
  const bool here = i < a.n;
  const int pairs = here ? a.m : 0;
  int id0 = -1;
  bool bad = false;
  const float p0 = p < pairs ? pair_key(a, i * a.m + p, id0, bad) : -INFINITY;
  const float dl = here && a.C ? a.dloss[i] : 0.f;
  scores_block<XT, CT, NT>(a, 0, t0, zs);
  float* z = zs[0][row];
  float* q = zs[1][row];
  float m = -INFINITY, s = 0.f;
#pragma unroll
  for (int c = p; c < S; c += 8) {
    m = fmaxf(m, z[c]);
    q[c] = 0.f;
  }
  m = near_max<8>(m);
  const float m0 = safe(m);
#pragma unroll
  for (int c = p; c < S; c += 8) s += __builtin_amdgcn_exp2f(z[c] - m0);
  const float lse2 = m + log2f(near_sum<8>(s));
  // the target: its largest logit, then its sum, then each pair
  float tm = p0, ts = 0.f, loss = 0.f;
  int id;
  for (int j = p + 8; j < pairs; j += 8) tm = fmaxf(tm, pair_key(a, i * a.m + j, id, bad));
  tm = safe(near_max<8>(tm));
  ts = id0 < 0 ? 0.f : pair_weight(p0, tm, a.tscale);
  for (int j = p + 8; j < pairs; j += 8) {
    const float t = pair_key(a, i * a.m + j, id, bad);
    ts += id < 0 ? 0.f : pair_weight(t, tm, a.tscale);
  }
  ts = near_sum<8>(ts);
  bad = near_sum<8>(bad ? 1.f : 0.f) != 0.f;
  const bool some = ts != 0.f;
  const float inv = some ? 1.f / ts : 0.f;
  for (int j0 = 0; j0 < a.m; j0 += 8) {
    bool b;
    id = j0 ? -1 : id0;
    float t = p0;
    if (j0 && j0 + p < pairs) t = pair_key(a, i * a.m + j0 + p, id, b);
    const float mine = id < 0 ? 0.f : pair_weight(t, tm, a.tscale) * inv;
    for (int o = 0; o < min(8, a.m - j0); ++o) {
      const int v = __shfl(id, o, 8);
      const float qj = __shfl(mine, o, 8);
      if (v < 0 || (v & 7) != p) continue;
      if (qj != 0.f) loss += qj * (logf(qj) + (z[v] == -INFINITY ? INFINITY : lse2 - z[v]) * kLn2);
      q[v] += qj;
    }
  }
  loss = near_sum<8>(loss);
  if (here && p == 0) {
    a.loss[i] = bad ? __builtin_nanf("") : some ? loss : 0.f;
    a.lse[i] = lse2 * kLn2;
  }
  if (!a.C) return;
  float cf = dl * a.scale;
  if (!some || lse2 == -INFINITY) cf = 0.f;
  if (bad) cf = __builtin_nanf("");
  if (here && p == 0) a.coef[i] = cf;
  const float l2 = safe(lse2);
  if (!here) return;
#pragma unroll
  for (int c = p; c < S; c += 8)
    a.C[i * S + c] = cf == 0.f || z[c] == -INFINITY ? 0.f : cf * (__builtin_amdgcn_exp2f(z[c] - l2) - q[c]);
}

// Few rows: CT x 16 classes by all rows of h; the rows' (largest, sum) of the
// tile, and Z.  Bound by reading w: one row, 32768 bfloat16 classes of 2048 22 us,
// 6.1 TB/s.
template <typename XT, int CT, int NT>
__global__ __launch_bounds__(256) void scores_few_rows_kernel(FewArgs a) {
  constexpr int S = NT * 16, P = 256 / S;
  __shared__ float zs[4][S][CT * 16 + 1];
  const int64_t v0 = (int64_t)blockIdx.x * (CT * 16);
  scores_block<XT, CT, NT>(a, v0, 0, zs);
  const int row = threadIdx.x / P, p = threadIdx.x % P;
  const float* z = zs[0][row];
  float m = -INFINITY, s = 0.f;
  for (int c = p; c < CT * 16; c += P) m = fmaxf(m, z[c]);
  m = near_max<P>(m);
  for (int c = p; c < CT * 16; c += P) s += __builtin_amdgcn_exp2f(z[c] - safe(m));
  s = near_sum<P>(s);
  if (p == 0 && row < a.n) a.part[(int64_t)blockIdx.x * a.n + row] = make_float2(m, s);
  for (int x = threadIdx.x; x < CT * 16 * S; x += 256) {
    const int c = x / S, t = x % S;
    if (v0 + c < a.classes) a.C[(v0 + c) * S + t] = zs[0][t][c];
  }
}

// Few rows: a workgroup joins a row's tiles and takes its targets from Z, a
// thread per pair.  4 to 5 us, of which most is the launch.
template <int S>
__global__ __launch_bounds__(256) void targets_few_kernel(FewArgs a, int ntiles) {
  __shared__ float red[3][4];
  __shared__ int sid[kMaxTop];
  __shared__ float sq[kMaxTop];
  const int64_t i = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto all_sum = [&](float v, int slot) {
    v = wave_sum(v);
    __syncthreads();
    if (lane == 0) red[slot][wave] = v;
    __syncthreads();
    return (red[slot][0] + red[slot][1]) + (red[slot][2] + red[slot][3]);
  };
  auto all_max = [&](float v, int slot) {
    v = near_max<64>(v);
    __syncthreads();
    if (lane == 0) red[slot][wave] = v;
    __syncthreads();
    return fmaxf(fmaxf(red[slot][0], red[slot][1]), fmaxf(red[slot][2], red[slot][3]));
  };
  float m = -INFINITY, s = 0.f;
  for (int t = tid; t < ntiles; t += 256) {
    const float2 v = a.part[(int64_t)t * a.n + i];
    const float nm = fmaxf(m, v.x);
    s = s * __builtin_amdgcn_exp2f(m - safe(nm)) + v.y * __builtin_amdgcn_exp2f(v.x - safe(nm));
    m = nm;
  }
  const float top = all_max(m, 0);
  const float lse2 = top + log2f(all_sum(s * __builtin_amdgcn_exp2f(m - safe(top)), 1));
  int id = -1;
  bool bad = false;
  float t = -INFINITY;
  if (tid < a.m) t = pair_key(a, i * a.m + tid, id, bad);
  const float tm = safe(all_max(t, 2));
  const float e = id < 0 ? 0.f : pair_weight(t, tm, a.tscale);
  const float ts = all_sum(e, 0);
  bad = all_sum(bad ? 1.f : 0.f, 1) != 0.f;
  const bool some = ts != 0.f;
  const float q = some ? e / ts : 0.f, z = id < 0 ? 0.f : a.C[(int64_t)id * S + i];
  const float l = q != 0.f ? q * (logf(q) + (z == -INFINITY ? INFINITY : lse2 - z) * kLn2) : 0.f;
  const float loss = all_sum(l, 2);
  if (tid == 0) {
    a.loss[i] = bad ? __builtin_nanf("") : some ? loss : 0.f;
    a.lse[i] = lse2 * kLn2;
  }
  if (!a.coef) return;
  float cf = a.dloss[i] * a.scale;
  if (!some || lse2 == -INFINITY) cf = 0.f;
  if (bad) cf = __builtin_nanf("");
  if (tid == 0) {
    a.lse2[i] = safe(lse2);
    a.coef[i] = cf;
  }
  if (tid < a.m) {
    sid[tid] = id;
    sq[tid] = q;
  }
  __syncthreads();
  if (tid >= a.m) return;
  float qs = 0.f;  // a class named twice: once, with both
  bool first = true;
  for (int j = 0; j < a.m; ++j)
    if (sid[j] == id) {
      qs += sq[j];
      first &= j >= tid;
    }
  a.fix_id[i * a.m + tid] = first && cf != 0.f ? id : -1;
  a.fix_val[i * a.m + tid] = z == -INFINITY ? 0.f : cf * (__builtin_amdgcn_exp2f(z - safe(lse2)) - qs);
}

// Few rows: Z becomes G^T; the targets' entries come from the rows' lists.  16 rows,
// 32000 classes 4 us.
__global__ __launch_bounds__(256) void grad_few_kernel(float* __restrict__ C, int64_t count, int S, int64_t n, int m,
                                                       const float* __restrict__ lse2, const float* __restrict__ coef,
                                                       const int32_t* __restrict__ id, const float* __restrict__ val) {
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (x >= count) return;
  const int64_t v = x / S, t = x - v * S;
  const float cf = t < n ? coef[t] : 0.f;
  float g = 0.f;
  if (cf != 0.f) {
    g = cf * __builtin_amdgcn_exp2f(C[x] - lse2[t]);
    for (int j = 0; j < m; ++j)
      if (id[t * m + j] == v) g = val[t * m + j];
  }
  C[x] = g;
}

// A row that takes no part: weight[row] is `none` (0, or -inf).
__device__ inline bool takes_part(const float* weight, float none, int64_t row) {
  return !weight || weight[row] != none;
}

// out (R x d) = C (R x S) B (S x d), rows of B that take no part left out, rows
// of out that take none 0.  The matrix instructions have the features as rows:
// one of a lane's kVec features each, so that a lane ends with 16 or 32
// neighbouring features of a row of out, the four lanes of a row 64 bytes at a
// time.  A wavefront keeps its 16 kVec features of B in registers and goes over
// blocks of 16 rows a grid apart, the next one's C on its way.
struct RowsJob {
  const float* C;
  int64_t ldc;  // rows_direct only: C's width
  const void* B;
  int64_t ldb;
  int rows_b;
  const float* weight_b;  // rows of B that take no part have `none_b` here
  float none_b;
  int64_t R;
  int d;
  const float* weight_r;  // rows of out that take no part have `none_r` here
  float none_r;
  void* out;
  int64_t ldo;
  int per;       // rows_direct: classes of a slab
  float* slabs;  // rows_direct: where out is null
  unsigned gx, gy;  // the workgroups
};

template <typename XT, int S>
__device__ inline void rows_few(const RowsJob& q, unsigned bx, unsigned by) {
  const float* __restrict__ C = q.C;
  const XT* __restrict__ B = (const XT*)q.B;
  XT* __restrict__ out = (XT*)q.out;
  const float *weight_b = q.weight_b, *weight_r = q.weight_r;
  const float none_b = q.none_b;
  const int64_t ldb = q.ldb, R = q.R, ldo = q.ldo;
  const int rows_b = q.rows_b, d = q.d;
  constexpr int VEC = kVec<XT>, KB = S / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int c0 = (by * 4 + wave) * (16 * VEC);
  if (c0 >= d) return;
  const int place = (l16 >> 2) + 4 * (l16 & 3);  // matrix row 4 g + r holds the features from kVec (g + 4 r)
  raw_vec<XT> b[KB][4];
#pragma unroll
  for (int k0 = 0; k0 < KB; ++k0)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = 16 * k0 + 4 * g + e;
      const bool use = k < rows_b && takes_part(weight_b, none_b, k);
      b[k0][e] = load_raw(B + (int64_t)(use ? k : 0) * ldb, c0 + place * VEC, use ? d : 0);
    }
  floatx4 c[KB], cn[KB];
  float wn = 1.f;  // (compared where it is used: the row is on its way)
  auto fetch = [&](int64_t r0) {
    const int64_t row = min(r0 + l16, R - 1);
#pragma unroll
    for (int k0 = 0; k0 < KB; ++k0) cn[k0] = *(const floatx4*)(C + row * S + 16 * k0 + 4 * g);
    if (weight_r) wn = weight_r[row];
  };
  const int64_t step = (int64_t)q.gx * 16;
  int64_t r0 = (int64_t)bx * 16;
  fetch(r0);
  for (; r0 < R; r0 += step) {
#pragma unroll
    for (int k0 = 0; k0 < KB; ++k0) c[k0] = cn[k0];
    const bool part = wn != q.none_r;
    fetch(r0 + step);
    floatx4 acc[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k0 = 0; k0 < KB; ++k0)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32((float)b[k0][e][j], c[k0][e], acc[j], 0, 0, 0);
    const int64_t row = r0 + l16;
    if (row >= R) continue;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[j] = part ? acc[j][r] : 0.f;
      store_part(out + row * ldo, c0 + VEC * (g + 4 * r), d, v);
    }
  }
}

// out (M x d) = C^T X, rows of X (R x d) that take no part left out and rows of
// out that take none 0: S columns of C a workgroup, and where by splits the rows
// of X, their sums into that slab.  A step is 4 UN rows: a lane loads VEC features of row
// lane / 16 in each of CH blocks of 16 VEC features, and S / 16 of the row's
// entries of C.  The four wavefronts take every fourth step and join in LDS.
template <typename XT, int S>
struct ColsShape {
  static constexpr int CT = S / 16, VEC = kVec<XT> * CT > 16 ? 16 / CT : kVec<XT>;  // features of a load
  static constexpr int CH = 16 / (VEC * CT);                                        // 64 sums a lane
  // (bytes in flight: of S = 16 twice as many, where the registers allow it; 60000
  // rows of 780, 10 classes, with gradient 166 -> 157 us, of S = 32 97 -> 110)
  static constexpr int UN = S == 16 ? 8 / CH : 4 / CH;
  static constexpr int lds = S * (16 * VEC + 1);  // floats
  static constexpr int width = CH * 16 * VEC;  // 256, 128 or 64
};
struct ColsJob {
  const float* C;
  int64_t ldc;
  const void* X;
  int64_t ldx, R;
  int d;
  const float* weight;  // rows of X that take no part have `none` here
  float none;
  int64_t per;
  float* slabs;
  int M;
  const float* weight_m;  // rows of out that take no part have `none_m` here
  float none_m;
  void* out;              // null: slabs
  int64_t ldo;
  unsigned gx, gy, gz;  // the workgroups: features, splits, columns of C
};

template <typename XT, int S>
__device__ inline void cols_few(const ColsJob& q, unsigned bx, unsigned by, unsigned bz, float* lds) {
  using Sh = ColsShape<XT, S>;
  constexpr int VEC = Sh::VEC, CT = Sh::CT, CH = Sh::CH, UN = Sh::UN;
  typedef float cvec __attribute__((ext_vector_type(CT)));
  float (*red)[16 * VEC + 1] = (float (*)[16 * VEC + 1])lds;  // [S]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int c0 = bx * Sh::width, s0 = bz * S, M = q.M, d = q.d;
  const float* __restrict__ C = q.C + s0;
  const XT* __restrict__ X = (const XT*)q.X;
  XT* __restrict__ out = (XT*)q.out;
  const float *weight = q.weight, *weight_m = q.weight_m;
  const float none = q.none;
  const int64_t ldc = q.ldc, ldx = q.ldx, ldo = q.ldo;
  const int64_t lo = (int64_t)by * q.per, hi = min(lo + q.per, q.R);
  floatx4 acc[CH][VEC][CT];
#pragma unroll
  for (int h = 0; h < CH; ++h)
#pragma unroll
    for (int j = 0; j < VEC; ++j)
#pragma unroll
      for (int t = 0; t < CT; ++t) acc[h][j][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  raw_n<VEC, XT> x[UN][CH], xn[UN][CH];  // this step's, and the next one's on their way
  float c[UN][CT], cn[UN][CT];
  bool un[UN];
  const bool inside = c0 + Sh::width <= d;
  auto fetch = [&](int64_t s) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int64_t row = s + u * 4 + g;
      const bool use = row < hi && takes_part(weight, none, row);
      const XT* xr = X + (use ? row : lo) * ldx;
#pragma unroll
      for (int h = 0; h < CH; ++h) {
        const int col = c0 + (h * 16 + l16) * VEC;
        if (inside) {
          xn[u][h] = *(const any_n<VEC, XT>*)(xr + col);
        } else {
          xn[u][h] = load_n<VEC>(xr, col, d);
        }
      }
      const cvec cv = *(const cvec*)(C + (row < hi ? row : lo) * ldc + CT * l16);
#pragma unroll
      for (int t = 0; t < CT; ++t) cn[u][t] = ((const float*)&cv)[t];
      un[u] = use;
    }
  };
  constexpr int step = 16 * UN;  // rows of the four wavefronts' steps
  int64_t s = lo + wave * (4 * UN);
  if (s < hi) fetch(s);
  for (; s < hi; s += step) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
#pragma unroll
      for (int h = 0; h < CH; ++h)
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][h][e] = un[u] ? xn[u][h][e] : (XT)0.f;
#pragma unroll
      for (int t = 0; t < CT; ++t) c[u][t] = un[u] ? cn[u][t] : 0.f;
    }
    if (s + step < hi) fetch(s + step);
#pragma unroll
    for (int u = 0; u < UN; ++u)
#pragma unroll
      for (int h = 0; h < CH; ++h)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
#pragma unroll
          for (int t = 0; t < CT; ++t)
            acc[h][j][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(c[u][t], (float)x[u][h][j], acc[h][j][t], 0, 0, 0);
  }
  // entry r of block (j, t): row CT (4 g + r) + t of the slab, feature VEC l16 + j
  float* slab = q.slabs + ((int64_t)by * M + s0) * d;
#pragma unroll
  for (int h = 0; h < CH; ++h) {
    for (int o = 0; o < 4; ++o) {
      if (wave == o)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
#pragma unroll
          for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float* p = &red[CT * (4 * g + r) + t][VEC * l16 + j];
              *p = o ? *p + acc[h][j][t][r] : acc[h][j][t][r];
            }
      __syncthreads();
    }
    for (int y = threadIdx.x; y < S * 16 * VEC; y += 256) {
      const int sr = y / (16 * VEC), cc = c0 + h * 16 * VEC + y % (16 * VEC);
      if (cc >= d || s0 + sr >= M) continue;
      const float v = red[sr][y % (16 * VEC)];
      if (out)
        out[(s0 + sr) * ldo + cc] = (XT)(takes_part(weight_m, q.none_m, s0 + sr) ? v : 0.f);
      else
        slab[(int64_t)sr * d + cc] = v;
    }
    __syncthreads();
  }
}

// out (M x d) from the slabs, in order, so that the bits do not depend on timing;
// rows whose weight is `none` are 0.  4 to 5 us, of which most is the launch.
struct SlabsJob {
  const float* slabs;
  int count, M, d;
  const float* weight;
  float none;
  void* out;
  int64_t ldo;
  unsigned blocks;
};
struct SlabsJobs {
  SlabsJob j[2];
};
template <typename OT>
__global__ __launch_bounds__(256) void slabs_few_kernel(SlabsJobs jobs) {
  const bool second = blockIdx.x >= jobs.j[0].blocks;
  const SlabsJob& q = jobs.j[second];
  const int d = q.d, count = q.count;
  const int64_t x = (int64_t)(blockIdx.x - (second ? jobs.j[0].blocks : 0u)) * 64 + (threadIdx.x & 63);
  const int wave = threadIdx.x >> 6;
  const int64_t entries = (int64_t)q.M * d;
  __shared__ float red[4][64];
  float s = 0.f;
  if (x < entries)
#pragma unroll 8
    for (int k = wave; k < count; k += 4) s += q.slabs[(int64_t)k * entries + x];
  red[wave][threadIdx.x & 63] = s;
  __syncthreads();
  if (wave || x >= entries) return;
  const int lane = threadIdx.x;
  s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
  const int64_t row = x / d;
  ((OT*)q.out)[row * q.ldo + (x - row * d)] = (OT)(takes_part(q.weight, q.none, row) ? s : 0.f);
}

// ------------------------------------------------------------------ both sides longer, little work

// 32 rows of h by 64 classes: Z in base 2, [n][ldz].  2000 fp32 rows of 300, 400
// classes: 15 us, 32 TFLOP/s (row_direct 5 us, both gradients 25 us, 38 TFLOP/s).
template <typename XT>
__global__ __launch_bounds__(256) void scores_direct_kernel(FewArgs a, int64_t ldz) {
  __shared__ float zs[4][32][65];
  const int64_t v0 = (int64_t)blockIdx.x * 64, t0 = (int64_t)blockIdx.y * 32;
  scores_block<XT, 4, 2>(a, v0, t0, zs);
#pragma unroll
  for (int x = threadIdx.x; x < 32 * 64; x += 256)
    if (t0 + x / 64 < a.n) a.C[(t0 + x / 64) * ldz + v0 + x % 64] = zs[0][x / 64][x % 64];
}

// lse, the loss, and Z becomes G: a row by WR wavefronts (1, or 4 where it is
// long), which all hold its pairs, lane l the pairs l, l + 64, ...
template <int NQ, int WR>
__global__ __launch_bounds__(256) void row_direct_kernel(FewArgs a, int64_t ldz, bool grad) {
  __shared__ float red[2][4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t i = WR == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
  if (i >= a.n) return;
  float* zr = a.C + i * ldz;
  int id[NQ];
  float q[NQ], z[NQ], tm = -INFINITY, ts = 0.f;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    const int j = k * 64 + lane;
    id[k] = -1;
    q[k] = j < a.m ? pair_key(a, i * a.m + j, id[k], bad) : -INFINITY;
    z[k] = id[k] >= 0 ? zr[id[k]] : 0.f;
    tm = fmaxf(tm, q[k]);
  }
  const float dl = grad ? a.dloss[i] : 0.f;
  float m = -INFINITY, s = 0.f;
  const int64_t c0 = (WR == 1 ? lane : threadIdx.x) * 4;
#pragma unroll 4
  for (int64_t c = c0; c < ldz; c += 256 * WR) {
    const floatx4 v = *(const floatx4*)(zr + c);
    const float nm = fmaxf(fmaxf(m, fmaxf(v[0], v[1])), fmaxf(v[2], v[3])), n0 = safe(nm);
    s *= __builtin_amdgcn_exp2f(m - n0);
#pragma unroll
    for (int e = 0; e < 4; ++e) s += __builtin_amdgcn_exp2f(v[e] - n0);
    m = nm;
  }
  float top = near_max<64>(m);
  s = wave_sum(s * __builtin_amdgcn_exp2f(m - safe(top)));
  if (WR > 1) {
    if (lane == 0) {
      red[0][wave] = top;
      red[1][wave] = s;
    }
    __syncthreads();  // (also: every target's z is read before any G is written)
    top = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) s += red[1][w] * __builtin_amdgcn_exp2f(red[0][w] - safe(top));
  }
  const float lse2 = top + log2f(s);
  tm = safe(near_max<64>(tm));
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    q[k] = id[k] < 0 ? 0.f : pair_weight(q[k], tm, a.tscale);
    ts += q[k];
  }
  ts = wave_sum(ts);
  bad = __ballot(bad) != 0;
  const bool some = ts != 0.f, writer = lane == 0 && (WR == 1 || wave == 0);
  float l = 0.f;
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    q[k] = some ? q[k] / ts : 0.f;
    if (q[k] != 0.f) l += q[k] * (logf(q[k]) + (z[k] == -INFINITY ? INFINITY : lse2 - z[k]) * kLn2);
  }
  l = wave_sum(l);
  if (writer) {
    a.loss[i] = bad ? __builtin_nanf("") : some ? l : 0.f;
    a.lse[i] = lse2 * kLn2;
  }
  if (!grad) return;
  float cf = dl * a.scale;
  if (!some || lse2 == -INFINITY) cf = 0.f;
  if (bad) cf = __builtin_nanf("");
  if (writer) a.coef[i] = cf;
  const float l2 = safe(lse2);
#pragma unroll 4
  for (int64_t c = c0; c < ldz; c += 256 * WR) {
    floatx4 v = *(const floatx4*)(zr + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = cf == 0.f ? 0.f : cf * __builtin_amdgcn_exp2f(v[e] - l2);
    *(floatx4*)(zr + c) = v;
  }
  // the targets' entries, a class named twice once, after the row's own stores
  float g[NQ];
  bool first[NQ];
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    float qs = 0.f;
    first[k] = true;
    for (int jj = 0; jj < a.m; ++jj) {
      int ij = -1;
      float qj = 0.f;
#pragma unroll
      for (int kk = 0; kk < NQ; ++kk)
        if (jj / 64 == kk) {
          ij = __shfl(id[kk], jj & 63, 64);
          qj = __shfl(q[kk], jj & 63, 64);
        }
      if (ij == id[k]) {
        qs += qj;
        if (jj < k * 64 + lane) first[k] = false;
      }
    }
    g[k] = z[k] == -INFINITY ? 0.f : cf * (__builtin_amdgcn_exp2f(z[k] - l2) - qs);
  }
  if (WR > 1) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the row is written
  }
  if (cf == 0.f || (WR > 1 && wave)) return;
#pragma unroll
  for (int k = 0; k < NQ; ++k)
    if (id[k] >= 0 && first[k]) zr[id[k]] = g[k];
}

// out (R x d) = C (R x K) B (K x d) for any K (C padded with zeros to 16): as
// rows_few, 32 rows by 16 kVec features a workgroup, whose wavefronts
// take every fourth 16 of K and join in LDS.  bz splits K into slabs.
template <typename XT>
constexpr int kDirectLds = 4 * 32 * (16 * kVec<XT> + 4);  // floats
template <typename XT>
__device__ inline void rows_direct(const RowsJob& q, unsigned bx, unsigned by, unsigned bz, float* lds) {
  constexpr int VEC = kVec<XT>, W = 16 * VEC;
  float (*red)[32][W + 4] = (float (*)[32][W + 4])lds;  // [4]
  const float* __restrict__ C = q.C;
  const XT* __restrict__ B = (const XT*)q.B;
  XT* __restrict__ out = (XT*)q.out;
  const float *weight_b = q.weight_b, *weight_r = q.weight_r;
  const float none_b = q.none_b;
  const int64_t ldc = q.ldc, ldb = q.ldb, R = q.R, ldo = q.ldo;
  const int K = q.rows_b, d = q.d, per = q.per;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int c0 = bx * W, place = (l16 >> 2) + 4 * (l16 & 3);
  const int64_t r0 = (int64_t)by * 32;
  const float* cr[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) cr[t] = C + min(r0 + t * 16 + l16, R - 1) * ldc + 4 * g;
  floatx4 acc[VEC][2];
#pragma unroll
  for (int j = 0; j < VEC; ++j)
#pragma unroll
    for (int t = 0; t < 2; ++t) acc[j][t] = floatx4{0.f, 0.f, 0.f, 0.f};
  raw_vec<XT> b[4], bn[4];
  floatx4 c[2], cn[2];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) cn[t] = *(const floatx4*)(cr[t] + k0);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = k0 + 4 * g + e;
      const bool use = k < K && takes_part(weight_b, none_b, k);
      bn[e] = load_raw(B + (int64_t)(use ? k : 0) * ldb, c0 + place * VEC, use ? d : 0);
    }
  };
  const int end = min(K, ((int)bz + 1) * per);
  int k0 = bz * per + wave * 16;
  if (k0 < end) fetch(k0);
  for (; k0 < end; k0 += 64) {
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = bn[e];
#pragma unroll
    for (int t = 0; t < 2; ++t) c[t] = cn[t];
    if (k0 + 64 < end) fetch(k0 + 64);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int j = 0; j < VEC; ++j)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x4f32((float)b[e][j], c[t][e], acc[j][t], 0, 0, 0);
  }
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) red[wave][t * 16 + l16][VEC * (g + 4 * r) + j] = acc[j][t][r];
  __syncthreads();
#pragma unroll
  for (int x = threadIdx.x; x < 32 * 16; x += 256) {
    const int rr = x / 16, cc = (x % 16) * VEC;
    const int64_t row = r0 + rr;
    if (row >= R || c0 + cc >= d) continue;
    const bool part = takes_part(weight_r, q.none_r, row);
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      v[e] = part ? (red[0][rr][cc + e] + red[1][rr][cc + e]) + (red[2][rr][cc + e] + red[3][rr][cc + e]) : 0.f;
    if (out) {
      store_part(out + row * ldo, c0 + cc, d, v);
    } else {
      float* p = q.slabs + ((int64_t)bz * R + row) * d + c0 + cc;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c0 + cc + e < d) p[e] = v[e];
    }
  }
}

// Both gradients in one launch, the sums' workgroups first (what they read may
// still be in the last-level cache).  ROWS: rows_few, rows_direct or neither.
// Bound by reading the long side: both of 60000 fp32 rows of 780, 10 classes 79 us, 4.7
// TB/s of h and dH; of 16 rows, 32000 bfloat16 classes of 2000 73 us, 3.5 TB/s of w
// and dW.  64 classes by the fp32 matrix instructions: both of 20000 rows of 784 63
// to 69 us, 58 to 63 TFLOP/s.
enum { ROWS_NONE, ROWS_FEW, ROWS_DIRECT };
template <typename XT, int S, int ROWS>
__global__ __launch_bounds__(256, 2) void grads_few_kernel(ColsJob c, RowsJob r) {
  constexpr int kLds = ROWS == ROWS_DIRECT && kDirectLds<XT> > ColsShape<XT, S>::lds ? kDirectLds<XT>
                                                                                      : ColsShape<XT, S>::lds;
  __shared__ __attribute__((aligned(16))) float lds[kLds];
  unsigned b = blockIdx.x;
  const unsigned nc = c.gx * c.gy * c.gz;
  auto uniform = [](unsigned v) { return (unsigned)__builtin_amdgcn_readfirstlane((int)v); };
  if (b < nc) {
    const unsigned x = uniform(b % c.gx), yz = uniform(b / c.gx);
    cols_few<XT, S>(c, x, uniform(yz % c.gy), uniform(yz / c.gy), lds);
  } else if constexpr (ROWS != ROWS_NONE) {
    b -= nc;
    const unsigned x = uniform(b % r.gx), yz = uniform(b / r.gx), y = uniform(yz % r.gy);
    if constexpr (ROWS == ROWS_FEW) rows_few<XT, S>(r, x, y);
    else rows_direct<XT>(r, x, y, uniform(yz / r.gy), lds);
  }
}

// ------------------------------------------------------------------ plan

int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct FewPlan {
  bool classes;  // few classes, or few rows
  int S;         // the short side, padded to 16, 32 or 64
  int64_t R;     // the long side
  int ct;        // few rows: class blocks of a tile
  int ntiles;
  int splits;
  int64_t per;
  size_t C, part, lse2, coef, fix_id, fix_val, slabs, bytes;
};

FewPlan few_plan(const HeadArgs& a, bool grad) {
  FewPlan p{};
  p.classes = a.classes <= kFew;
  const int64_t s = p.classes ? a.classes : a.n;
  p.S = s <= 16 ? 16 : s <= 32 ? 32 : 64;
  p.R = p.classes ? a.n : a.classes;
  p.ct = a.classes >= 16384 ? 4 : a.classes >= 4096 ? 2 : 1;
  if (p.S == 64) p.ct = std::min(p.ct, 2);
  p.ntiles = (int)cdiv(a.classes, 16 * p.ct);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t r = at;
    at += up(bytes, 1024);
    return r;
  };
  if (grad || !p.classes) p.C = take((size_t)p.R * p.S * 4);
  if (!p.classes) p.part = take((size_t)p.ntiles * a.n * 8);
  if (grad) {
    p.lse2 = take((size_t)a.n * 4);
    p.coef = take((size_t)a.n * 4);
    if (!p.classes) {
      p.fix_id = take((size_t)a.n * a.m * 4);
      p.fix_val = take((size_t)a.n * a.m * 4);
    }
    // rows of a slab: enough workgroups for the chip, no more slabs than their sum is worth
    const int64_t chunks = cdiv(a.d, p.S == 16 ? 256 : p.S == 32 ? 128 : 64);  // ColsShape::width
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(cdiv(p.S == 64 ? 512 : 768, chunks), cdiv(p.R, 64)));
    p.per = up(cdiv(p.R, p.splits), 64);
    p.splits = (int)cdiv(p.R, p.per);
    if (p.splits > 1) p.slabs = take((size_t)p.splits * s * a.d * 4);
  }
  p.bytes = at;
  return p;
}

#define KKM_TRY(expr)                        \
  do {                                       \
    hipError_t e_ = (expr);                  \
    if (e_ != hipSuccess) return e_;         \
  } while (0)

template <int N>
using num = std::integral_constant<int, N>;
template <typename F>
void by_short(int S, F&& f) {
  if (S == 16) f(num<16>{});
  else if (S == 32) f(num<32>{});
  else f(num<64>{});
}

template <typename XT, int S>
ColsJob cols_job(const float* weight, float none, const float* C, int64_t ldc, const void* X, int64_t ldx, int64_t R,
                 int d, int splits, int64_t per, float* slabs, int M, const float* weight_m, float none_m, void* out,
                 int64_t ldo) {
  return {C, ldc, X, ldx, R, d, weight, none, per, slabs, M, weight_m, none_m, splits > 1 ? nullptr : out, ldo,
          (unsigned)cdiv(d, ColsShape<XT, S>::width), (unsigned)splits, (unsigned)cdiv(M, S)};
}
SlabsJob sum_job(const float* slabs, int count, int M, int d, const float* weight, float none, void* out, int64_t ldo) {
  return {slabs, count, M, d, weight, none, out, ldo, (unsigned)cdiv((int64_t)M * d, 64)};
}
template <typename XT, int S, int ROWS>
void launch_grads(const ColsJob& c, const RowsJob& r, unsigned blocks_r, hipStream_t s) {
  hipLaunchKernelGGL((grads_few_kernel<XT, S, ROWS>), dim3(c.gx * c.gy * c.gz + blocks_r), dim3(256), 0, s, c, r);
}
template <typename XT>
void launch_sums(const SlabsJobs& jobs, hipStream_t s) {
  if (const unsigned blocks = jobs.j[0].blocks + jobs.j[1].blocks)
    hipLaunchKernelGGL((slabs_few_kernel<XT>), dim3(blocks), dim3(256), 0, s, jobs);
}

template <typename XT>
hipError_t few_typed(const HeadArgs& a, bool grad, char* ws, hipStream_t s) {
  const FewPlan p = few_plan(a, grad);
  FewArgs f{a.h, a.w, a.ldh, a.ldw, a.n, a.d, a.classes, a.m, a.scale * kLog2e, a.scale, a.tscale, a.offset,
            a.ids, a.tlogits, a.dloss, a.loss, a.lse, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
  if (grad || !p.classes) f.C = (float*)(ws + p.C);
  if (grad) {
    f.lse2 = (float*)(ws + p.lse2);
    f.coef = (float*)(ws + p.coef);
  }
  if (p.classes) {
    by_short(p.S, [&](auto S) {
      hipLaunchKernelGGL((scores_few_classes_kernel<XT, decltype(S)::value / 16>), dim3((unsigned)cdiv(a.n, 32)),
                         dim3(256), 0, s, f);
    });
    KKM_TRY(hipGetLastError());
  } else {
    f.part = (float2*)(ws + p.part);
    f.fix_id = (int32_t*)(ws + p.fix_id);
    f.fix_val = (float*)(ws + p.fix_val);
    by_short(p.S, [&](auto S) {
      constexpr int NT = decltype(S)::value / 16;
      const dim3 grid((unsigned)p.ntiles);
      if (p.ct == 1)
        hipLaunchKernelGGL((scores_few_rows_kernel<XT, 1, NT>), grid, dim3(256), 0, s, f);
      else if (p.ct == 2)
        hipLaunchKernelGGL((scores_few_rows_kernel<XT, 2, NT>), grid, dim3(256), 0, s, f);
      else if constexpr (NT < 4)
        hipLaunchKernelGGL((scores_few_rows_kernel<XT, 4, NT>), grid, dim3(256), 0, s, f);
      hipLaunchKernelGGL((targets_few_kernel<decltype(S)::value>), dim3((unsigned)a.n), dim3(256), 0, s, f, p.ntiles);
    });
    KKM_TRY(hipGetLastError());
    if (grad) {
      const int64_t count = p.R * p.S;
      hipLaunchKernelGGL(grad_few_kernel, dim3((unsigned)cdiv(count, 256)), dim3(256), 0, s, f.C, count, p.S, a.n, a.m,
                         f.lse2, f.coef, f.fix_id, f.fix_val);
      KKM_TRY(hipGetLastError());
    }
  }
  if (!grad) return hipSuccess;
  // the long side's gradient, then the short side's
  const float none = -INFINITY;
  void* long_out = p.classes ? a.dh : a.dw;
  void* short_out = p.classes ? a.dw : a.dh;
  const int rows_b = p.classes ? a.classes : (int)a.n;
  constexpr int VEC = kVec<XT>;
  by_short(p.S, [&](auto S_) {
    constexpr int S = decltype(S_)::value;
    ColsJob c{};
    RowsJob r{};
    SlabsJobs sums{};
    float* slabs = (float*)(ws + p.slabs);
    // who takes part: of the long side and of the short one
    const float *in_long = p.classes ? f.coef : a.offset, *in_short = p.classes ? a.offset : f.coef;
    const float none_long = p.classes ? 0.f : none, none_short = p.classes ? none : 0.f;
    if (short_out) {
      c = cols_job<XT, S>(in_long, none_long, f.C, p.S, p.classes ? a.h : a.w, p.classes ? a.ldh : a.ldw, p.R, a.d,
                          p.splits, p.per, slabs, rows_b, in_short, none_short, short_out,
                          p.classes ? a.lddw : a.lddh);
      if (p.splits > 1)
        sums.j[0] = sum_job(slabs, p.splits, rows_b, a.d, in_short, none_short, short_out,
                            p.classes ? a.lddw : a.lddh);
    }
    if (long_out) {
      const unsigned cols = (unsigned)cdiv(a.d, 64 * VEC);
      r = {f.C, p.S, p.classes ? a.w : a.h, p.classes ? a.ldw : a.ldh, rows_b, in_short, none_short, p.R, a.d,
           in_long, none_long, long_out, p.classes ? a.lddh : a.lddw, 0, nullptr,
           (unsigned)std::min<int64_t>(cdiv(p.R, 16), std::max(1u, (S == 64 ? 512u : 1536u) / cols)), cols};
      launch_grads<XT, S, ROWS_FEW>(c, r, r.gx * r.gy, s);
    } else if (short_out) {
      launch_grads<XT, S, ROWS_NONE>(c, r, 0, s);
    }
    launch_sums<XT>(sums, s);
  });
  return hipGetLastError();
}

struct DirectPlan {
  int64_t ldz, per;  // per: rows of h of a slab of dW
  int splits;
  int perh, splitsh;  // classes of a slab of dH
  size_t C, coef, slabs_w, slabs_h, bytes;
};

DirectPlan direct_plan(const HeadArgs& a, bool grad) {
  DirectPlan p{};
  p.ldz = up(a.classes, 64);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t r = at;
    at += up(bytes, 1024);
    return r;
  };
  p.C = take((size_t)a.n * p.ldz * 4);
  if (grad) {
    p.coef = take((size_t)a.n * 4);
    const int64_t chunks = cdiv(a.d, 64);
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(cdiv(512, chunks * (p.ldz / 64)), cdiv(a.n, 128)));
    p.per = up(cdiv(a.n, p.splits), 64);
    p.splits = (int)cdiv(a.n, p.per);
    p.splitsh = (int)std::max<int64_t>(1, std::min<int64_t>(cdiv(256, cdiv(a.d, 256 / (int)elem_bytes(a.type)) * cdiv(a.n, 32)), p.ldz / 256));
    p.perh = (int)up(cdiv(a.classes, p.splitsh), 64);
    p.splitsh = (int)cdiv(a.classes, p.perh);
    if (p.splits > 1) p.slabs_w = take((size_t)p.splits * a.classes * a.d * 4);
    if (p.splitsh > 1) p.slabs_h = take((size_t)p.splitsh * a.n * a.d * 4);
  }
  p.bytes = at;
  return p;
}

template <typename XT>
hipError_t direct_typed(const HeadArgs& a, bool grad, char* ws, hipStream_t s) {
  const DirectPlan p = direct_plan(a, grad);
  FewArgs f{a.h, a.w, a.ldh, a.ldw, a.n, a.d, a.classes, a.m, a.scale * kLog2e, a.scale, a.tscale, a.offset,
            a.ids, a.tlogits, a.dloss, a.loss, a.lse, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
  f.C = (float*)(ws + p.C);
  f.coef = (float*)(ws + p.coef);
  hipLaunchKernelGGL((scores_direct_kernel<XT>), dim3((unsigned)(p.ldz / 64), (unsigned)cdiv(a.n, 32)), dim3(256), 0, s,
                     f, p.ldz);
  auto rows = [&](auto nq, auto wr) {
    hipLaunchKernelGGL((row_direct_kernel<decltype(nq)::value, decltype(wr)::value>),
                       dim3((unsigned)(wr == 1 ? cdiv(a.n, 4) : a.n)), dim3(256), 0, s, f, p.ldz, grad);
  };
  const bool longer = a.classes > 1024;
  if (a.m <= 64) longer ? rows(num<1>{}, num<4>{}) : rows(num<1>{}, num<1>{});
  else longer ? rows(num<4>{}, num<4>{}) : rows(num<4>{}, num<1>{});
  KKM_TRY(hipGetLastError());
  if (!grad) return hipSuccess;
  ColsJob c{};
  RowsJob r{};
  SlabsJobs sums{};
  float *sw = (float*)(ws + p.slabs_w), *sh = (float*)(ws + p.slabs_h);
  if (a.dw) {
    c = cols_job<XT, 64>(f.coef, 0.f, f.C, p.ldz, a.h, a.ldh, a.n, a.d, p.splits, p.per, sw, a.classes, a.offset,
                         -INFINITY, a.dw, a.lddw);
    if (p.splits > 1) sums.j[0] = sum_job(sw, p.splits, a.classes, a.d, a.offset, -INFINITY, a.dw, a.lddw);
  }
  if (a.dh) {
    r = {f.C, p.ldz, a.w, a.ldw, a.classes, a.offset, -INFINITY, a.n, a.d, f.coef, 0.f, p.splitsh > 1 ? nullptr : a.dh,
         a.lddh, p.perh, sh, (unsigned)cdiv(a.d, 16 * kVec<XT>), (unsigned)cdiv(a.n, 32)};
    launch_grads<XT, 64, ROWS_DIRECT>(c, r, r.gx * r.gy * p.splitsh, s);
    if (p.splitsh > 1) sums.j[1] = sum_job(sh, p.splitsh, (int)a.n, a.d, f.coef, 0.f, a.dh, a.lddh);
  } else {
    launch_grads<XT, 64, ROWS_NONE>(c, r, 0, s);
  }
  launch_sums<XT>(sums, s);
  return hipGetLastError();
}

}  // namespace

// DIRECT up to so much work (n times classes times d): it needs four launches in
// place of eight or more and no copies, but multiplies in fp32 on the way to the
// gradients, and holds n times classes scores.  Microseconds with gradient, TILED
// / DIRECT: fp32, 400 classes of 300 features 71 / 31 at n = 100, 89 / 50 at 2000, 136
// / 116 at 6600 and 133 / 127 at 8000, on either side of the limit; 700 of 300 114 /
// 118 at 4000; 400 of 100 186 / 144 at 20000; 100 of 1000 130 / 54 at 2000, 514 / 405
// at 30000; 1000 of 1000 121 / 41 at 100, 190 / 198 at 2000; 1000 of 300 203 / 250 at
// 8000.  bfloat16, 400 of 300 48 / 37 at 100, 59 / 65 at 2000; 1000 of 300 52 / 42 at
// 500, 62 / 89 at 2000; 400 of 64 61 / 70 at 8000.  At a limit the two are within 10 %.
HeadForm head_form(const HeadArgs& a) {
  if (a.classes <= kFew || a.n <= kFew) return HEAD_FEW;
  const double work = (double)a.n * a.classes * a.d;
  const double most = a.type != TYPE_F32 ? 1.5e8 : a.classes <= 128 ? 3e9 : a.d >= 600 ? 2e9 : 8e8;
  return a.n * (int64_t)a.classes <= kDirectScores && work <= most ? HEAD_DIRECT : HEAD_TILED;
}

size_t head_short_scratch(const HeadArgs& a, bool grad) {
  return head_form(a) == HEAD_FEW ? few_plan(a, grad).bytes : direct_plan(a, grad).bytes;
}

hipError_t launch_head_short(const HeadArgs& a, bool grad, void* scratch, hipStream_t s) {
  const bool few = head_form(a) == HEAD_FEW;
  auto run = [&](auto x) {
    using XT = decltype(x);
    return few ? few_typed<XT>(a, grad, (char*)scratch, s) : direct_typed<XT>(a, grad, (char*)scratch, s);
  };
  switch (a.type) {
    case TYPE_F32: return run(float{});
    case TYPE_F16: return run(half_t{});
    default: return run(bf16_t{});
  }
}

}  // namespace kkm
