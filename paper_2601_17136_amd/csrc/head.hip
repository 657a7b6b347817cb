// A class head's losses and their gradients, with at most 256 MB of the logits in
// memory.
//
//   z(i, v) = scale h_i . w_v + offset_v,   lse_i = log sum_v exp z(i, v)
//   loss_i = sum_j q_j (log q_j - z(i, id_j) + lse_i)      over the row's pairs (id_j, q_j)
//   G(i, v) = dloss_i scale (exp(z(i, v) - lse_i) - sum_{j: id_j = v} q_j)
//   dH = G W,   dW = G^T H
//
// Forward: scores_kernel multiplies 16-bit tiles on the matrix cores and keeps
// of a tile each row's largest logit and sum of exponentials; targets_kernel
// joins them to lse, takes the few logits of the row's targets as plain dot
// products, and writes the loss.  Gradient: pieces of the classes, as many as
// keep G below kPieceBytes; of a piece the scores are computed again and G is
// written in both orders, the targets' entries in place (of rows with several
// targets by fix_kernel), and two products, in one launch where their tiles are
// alike, give the piece's rows of dW and its part of dH.
//
// The first classes' logits, at most 256 MB of them, stay for G where that takes
// less (kept_tiles).  The others are multiplied again: four products where a caller
// that kept all would take three.  G in its two orders and the kept logits are at
// most 256 MB each, or 256 classes (for 8192 rows of 32768 classes all of them would
// be 2.1 GB); a gradient's scratch has the transposed copies, copies of rows that
// do not serve in place, and sums besides: 1.28 GB for those rows of 4096 bfloat16
// features.  Bound by the matrix cores, whose clock falls to 1.75 - 1.97 GHz under
// this load.
//
// Operands are 16 bits with the contraction index contiguous.  Rows of binary16
// and bfloat16 that are aligned to 16 bytes serve in place; others are copied.
// fp32 is split into three bfloat16 planes (head_tile.h).  The gradient's
// products take copies of W and H with the other index contiguous, in which
// classes left out and rows without a target are zero, so that nothing that
// stands there (an infinity, a NaN) reaches a sum.
#include <algorithm>

#include "head_pairs.h"
#include "head_tile.h"
#include "model_ops.h"

namespace kkm {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
typedef float floatx4 __attribute__((ext_vector_type(4)));
constexpr size_t kPieceBytes = (size_t)256 << 20;

// Binary16 has no room for weights (dloss) of every size, so each row has its own
// power of two: G is held for a weight of 2^13 to 2^14 whatever the row's is (a
// probability to 4e-9 keeps all its bits), and dH's rows are put right as they
// are stored.  dW sums over the rows: its copy of h takes the row's power, with
// the largest entry of all rows (weight times largest feature, the row's level)
// just below 2^15.  A row's features then keep their bits down to 2^-29 of that entry.
constexpr int kHalfG = 14, kHalfH = 15;
// Words that share the search for the highest level, each in a cache line of its
// own: an atomic a row on one line took 40000 rows of 256 with 1000 classes 150 us.
constexpr int kLevels = 64, kLevelStep = 32, kLevelBias = 1024;

typedef unsigned short shorts8 __attribute__((ext_vector_type(8)));

__device__ inline int exponent_of(float v) {  // |v| in [1/2, 1) 2^e; 0 of 0, infinities and NaN
  if (v == 0.f || !isfinite(v)) return 0;
  int e;
  (void)frexpf(v, &e);
  return e;
}
// The words' highest, for a whole wavefront; 0 where no row has one.
__device__ inline int top_level(const unsigned* __restrict__ level) {
  unsigned m = level[(threadIdx.x & (kLevels - 1)) * kLevelStep];
#pragma unroll
  for (int o = 32; o; o >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, o, 64));
  return m ? (int)m - kLevelBias : 0;
}

// ------------------------------------------------------------------ operands

// A launch's work-items are a 32-bit count: a job of more than so many workgroups
// of 256 goes over its items with what it has.
constexpr int64_t kMaxBlocks = (int64_t)1 << 22;
constexpr int64_t kMaxItems = (int64_t)1 << 31;

// A copy of h and one of w run in one launch: the first `split` workgroups are
// the first job's.
struct StageJob {
  const void* src;
  int64_t ld, rows;
  void* dst;
  int64_t plane;
  const float* weight;  // transposed copies: rows of weight `none` are zero; may be null
  float none;
  int64_t rp;           // their width
  const float* dloss;   // binary16's h: rows take their weights' powers of two; null: none
};
struct StageJobs {
  StageJob j[2];
  unsigned split;
  const unsigned* level;  // with dloss: the words of top_level
  float scale;
  float* alpha;           // takes what dW's sums are multiplied by
};

// Rows in place of src's, kp wide (zero from d on), as P planes.  A thread
// writes 8 values.  3001 + 10007 binary16 rows of 1001 11 us, 4.8 TB/s; 8000 fp32
// rows of 1000 to three planes 16 us.
template <typename XT, typename E, int P>
__global__ __launch_bounds__(256) void stage_rows_kernel(StageJobs jobs, int d, int kp) {
  const bool second = blockIdx.x >= jobs.split;
  const StageJob& j = jobs.j[second];
  const unsigned first = second ? jobs.split : 0u, blocks = second ? gridDim.x - first : min(jobs.split, gridDim.x);
  const int64_t per = kp / 8, step = (int64_t)blocks * 256;
  for (int64_t i = (int64_t)(blockIdx.x - first) * 256 + threadIdx.x; i < j.rows * per; i += step) {
    const int64_t row = i / per;
    const int c = (int)(i - row * per) * 8;
    const XT* src = (const XT*)j.src + row * j.ld;
    float v[8];
    if constexpr (sizeof(XT) == 2) {
      load_part(src, c, d, v);
    } else {
      float a[4], b[4];
      load_part(src, c, d, a);
      load_part(src, c + 4, d, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
    }
    frag<E> o[P];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      E pl[P];
      split_planes<E, P>(v[e], pl);
#pragma unroll
      for (int p = 0; p < P; ++p) o[p][e] = pl[p];
    }
#pragma unroll
    for (int p = 0; p < P; ++p) *(frag<E>*)((E*)j.dst + p * j.plane + row * kp + c) = o[p];
  }
}

// The transposed copies: dst[c][row], rp rows wide (zero from `rows` on).  A
// workgroup turns a 64 x 64 block through LDS.  8192 + 32768 bfloat16 rows of 4096
// 127 us, 5.3 TB/s read and written.
template <typename XT, typename E, int P>
__global__ __launch_bounds__(256) void stage_cols_kernel(StageJobs jobs, int d) {
  constexpr int VEC = kVec<XT>, LANES = 64 / VEC, PASS = 256 / LANES;  // lanes of a row, rows of a pass
  __shared__ XT tile[64][64 + 4 / sizeof(XT)];
  const bool second = blockIdx.x >= jobs.split;
  const StageJob& j = jobs.j[second];
  const XT* src = (const XT*)j.src;
  E* dst = (E*)j.dst;
  const int64_t r0 = (int64_t)(blockIdx.x - (second ? jobs.split : 0u)) * 64, rows = j.rows, ld = j.ld, rp = j.rp,
                plane = j.plane;
  const int c0 = blockIdx.y * 64, col = (threadIdx.x % LANES) * VEC;
  int top = 0;
  if (std::is_same<XT, half_t>::value && j.dloss) {
    top = top_level(jobs.level);
    if (blockIdx.x == 0 && c0 == 0 && threadIdx.x == 0) *jobs.alpha = ldexpf(jobs.scale, top - kHalfG - kHalfH);
  }
#pragma unroll
  for (int k = 0; k < 64 / PASS; ++k) {
    const int rr = k * PASS + threadIdx.x / LANES;
    const int64_t row = r0 + rr;
    const bool use = row < rows && !(j.weight && j.weight[row] == j.none);
    raw_vec<XT> v = load_raw(src + (use ? row : 0) * ld, c0 + col, use ? d : 0);
    if constexpr (std::is_same<XT, half_t>::value) {
      if (j.dloss && use) {
        // (a row that set no level has zeros, or is NaN in any case)
        const float f = ldexpf(1.f, min(exponent_of(j.dloss[row]) + kHalfH - top, 64));
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = (XT)((float)v[e] * f);
      }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) tile[rr][col + e] = v[e];
  }
  __syncthreads();
  const int part = (threadIdx.x & 7) * 8;
#pragma unroll
  for (int c = threadIdx.x >> 3; c < 64; c += 32) {
    if (c0 + c >= d || r0 + part >= rp) continue;
    frag<E> o[P];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      E pl[P];
      split_planes<E, P>((float)tile[part + e][c], pl);
#pragma unroll
      for (int p = 0; p < P; ++p) o[p][e] = pl[p];
    }
#pragma unroll
    for (int p = 0; p < P; ++p) *(frag<E>*)(dst + p * plane + (int64_t)(c0 + c) * rp + r0 + part) = o[p];
  }
}

// ------------------------------------------------------------------ scores

template <typename E>
__device__ inline unsigned pack2(E lo, E hi) {
  typedef E e2 __attribute__((ext_vector_type(2)));
  const e2 v = {lo, hi};
  return __builtin_bit_cast(unsigned, v);
}

// (x, y) holds entries 0 .. 3 of this lane's column, two to a word; afterwards
// entry lane % 4 of the four neighbouring lanes' columns.
__device__ inline void turn4(unsigned& x, unsigned& y) {
  const int lane = threadIdx.x;
  const unsigned xn = __builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true);  // lane ^ 1
  const unsigned yn = __builtin_amdgcn_mov_dpp((int)y, 0xb1, 0xf, 0xf, true);
  const bool odd = lane & 1;
  const unsigned a = odd ? (xn >> 16) | (x & 0xffff0000u) : (x & 0xffffu) | (xn << 16);
  const unsigned b = odd ? (yn >> 16) | (y & 0xffff0000u) : (y & 0xffffu) | (yn << 16);
  const bool upper = lane & 2;  // entries 2 and 3 are wanted there
  const unsigned send = upper ? a : b;
  const unsigned got = __builtin_amdgcn_mov_dpp((int)send, 0x4e, 0xf, 0xf, true);  // lane ^ 2
  x = upper ? got : a;
  y = upper ? b : got;
}

// lo: a of the lower half of the wavefront, b's lower half in the upper; hi: a's upper half, b's upper half.
__device__ inline void swap_halves(unsigned a, unsigned b, unsigned& lo, unsigned& hi) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  lo = r[0];
  hi = r[1];
}

template <typename E>
struct ScoreArgs {
  Side w, h;
  int64_t n;
  int classes, v0;  // v0: first class of the piece
  int K, nkc, nseg, mt, nt;
  float zscale;         // scale log2 e
  const float* offset;  // may be null
  unsigned* level;      // forward: cleared for targets_kernel; may be null
  float2* part;         // forward: (largest, sum) in base 2 of each class tile and row, [tile][n]
  floatx4* z;           // logits in base 2 of the first `kept` class tiles, in the order of the tiles' lanes,
  int kept;             // written forward, read for G
  // gradient: rows' lse in base 2 and factors, G [row][class of the piece] and its transpose
  const float *lse2, *coef;
  const int32_t* fix_id;  // one target per row: its entry of G (else fix_kernel's work), or null
  const float* fix_val;
  E *G, *Gt;
  int64_t ldg, planeg, ldt, planet;
};

// Tile of classes (the matrix rows) by rows of H (the columns): a lane holds 16
// classes a block of one row of H, so a row's largest and sum stay in a lane
// up to one exchange and the wavefronts' sums in LDS.  The epilogue holds up the
// matrix cores once a tile: 9 us of a 256 x 256 tile, 19 with G, which it stores in
// both orders at 3.4 TB/s.  bfloat16, 8192 rows of 4096: 32768 classes, of which 8192
// are kept, 1.92 ms, 1.15 PFLOP/s, matrix cores busy 62 % of the cycles (a library
// product of that shape 1.41 PFLOP/s); with G, 16384 classes 1.09 ms, 1.01 PFLOP/s, 57
// %.  fp32, 4000 rows of 1000, 4000 classes: 159 us, 1.2 PFLOP/s of plane products;
// with G 196 us, or 57 of kept logits.  G of kept logits is bound by memory and needs
// no LDS: 20011 binary16 classes of 1777 rows 77 to 82 us, 3.5 TB/s, where
// multiplying again takes 141.
enum ScoresMode { SCORES_LOSS, SCORES_G, SCORES_G_OF_Z };
template <typename E, class S, int P, int MODE>
__global__ __launch_bounds__(S::threads, MODE == SCORES_G_OF_Z ? 2 : S::per_cu) void scores_kernel(ScoreArgs<E> a) {
  constexpr bool GRAD = MODE != SCORES_LOSS;
  __shared__ __attribute__((aligned(1024))) char lds[MODE == SCORES_G_OF_Z ? 16 : S::lds_bytes];
  if (!GRAD && a.level && blockIdx.x == 0 && threadIdx.x < kLevels) a.level[threadIdx.x * kLevelStep] = 0u;
  int mi, ni;
  tile_of(blockIdx.x, gridDim.x, a.mt, a.nt, mi, ni);
  const int64_t c0 = a.v0 + (int64_t)mi * S::BM, t0 = (int64_t)ni * S::BN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::GN, wn = wave % S::GN, l32 = lane & 31, h = lane >> 5;
  floatx16 acc[S::WM][S::WN];
  floatx4* kept = a.z + (((int64_t)ni * a.kept + mi) * S::waves + wave) * (S::WM * S::WN * 4 * 64) + lane;
  if constexpr (MODE == SCORES_G_OF_Z) {
#pragma unroll
    for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
      for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const floatx4 z = kept[((bi * S::WN + bj) * 4 + q) * 64];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[bi][bj][4 * q + e] = z[e];
        }
  } else {
    tile_product<E, S>(a.w, a.h, c0, t0, a.K, a.nkc, a.nseg, 0, a.nseg * a.nkc, lds, acc);
    // z in base 2; -inf where a class is left out, whatever its product
#pragma unroll
    for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t v = c0 + (wm * S::WM + bi) * 32 + 8 * q + 4 * h + e;
          const float off = v >= a.classes ? -INFINITY : a.offset ? a.offset[v] * kLog2e : 0.f;
#pragma unroll
          for (int bj = 0; bj < S::WN; ++bj) {
            const float z = fmaf(acc[bi][bj][4 * q + e], a.zscale, off);
            acc[bi][bj][4 * q + e] = off == -INFINITY ? -INFINITY : z;
          }
        }
    if (MODE == SCORES_LOSS && mi < a.kept) {
#pragma unroll
      for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
        for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            floatx4 z;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = acc[bi][bj][4 * q + e];
            kept[((bi * S::WN + bj) * 4 + q) * 64] = z;
          }
    }
  }
  if constexpr (!GRAD) {
    float2* red = (float2*)lds;  // [wm][column of the tile]
#pragma unroll
    for (int bj = 0; bj < S::WN; ++bj) {
      float m = -INFINITY;
#pragma unroll
      for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[bi][bj][r]);
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      const float m0 = m == -INFINITY ? 0.f : m;
      float s = 0.f;
#pragma unroll
      for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
        for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f(acc[bi][bj][r] - m0);
      s += __shfl_xor(s, 32, 64);
      if (h == 0) red[wm * S::BN + (wn * S::WN + bj) * 32 + l32] = make_float2(m, s);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < S::BN; c += S::threads) {
      if (t0 + c >= a.n) break;
      float m = -INFINITY, s = 0.f;
#pragma unroll
      for (int g = 0; g < S::GM; ++g) m = fmaxf(m, red[g * S::BN + c].x);
      const float m0 = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int g = 0; g < S::GM; ++g) {
        const float2 v = red[g * S::BN + c];
        s += v.y * __builtin_amdgcn_exp2f(v.x - m0);
      }
      a.part[(c0 / S::BM) * a.n + t0 + c] = make_float2(m, s);
    }
  } else {
    const int64_t cl = c0 - a.v0;
#pragma unroll
    for (int bj = 0; bj < S::WN; ++bj) {
      const int64_t t = t0 + (wn * S::WN + bj) * 32 + l32;
      const float lse2 = t < a.n ? a.lse2[t] : 0.f, cf = t < a.n ? a.coef[t] : 0.f;
      const bool one = a.fix_id && t < a.n;
      const int at = one ? a.fix_id[t] - (int)a.v0 : -1;  // (no class is at -1 - v0)
      const float val = one ? a.fix_val[t] : 0.f;
#pragma unroll
      for (int bi = 0; bi < S::WM; ++bi) {
        const int64_t v = cl + (wm * S::WM + bi) * 32;
        unsigned o[P][4][2];  // classes 8 q + 4 h + 0 .. 3 of row t, two to a word
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          E pl[4][P];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // (a row without a target has no gradient, whatever its logits)
            const float g = cf == 0.f ? 0.f : cf * __builtin_amdgcn_exp2f(acc[bi][bj][4 * q + e] - lse2);
            split_planes<E, P>((int)v + 8 * q + 4 * h + e == at ? val : g, pl[e]);
          }
#pragma unroll
          for (int p = 0; p < P; ++p) {
            o[p][q][0] = pack2(pl[0][p], pl[1][p]);
            o[p][q][1] = pack2(pl[2][p], pl[3][p]);
          }
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
          // G^T: four neighbouring lanes turn their 4 x 4 entries, so that a lane
          // has four rows of h of one class
          E* gt = a.Gt + p * a.planet + (v + 4 * h + (l32 & 3)) * a.ldt + (t & ~(int64_t)3);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            unsigned x = o[p][q][0], y = o[p][q][1];
            turn4(x, y);
            *(uint2*)(gt + (int64_t)(8 * q) * a.ldt) = make_uint2(x, y);
          }
          // G: the halves of the wavefront exchange, so that a lane has 16
          // neighbouring classes, the lower half 0 .. 15, the upper 16 .. 31
          E* g = a.G + p * a.planeg + t * a.ldg + v + 16 * h;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint4 w;
            swap_halves(o[p][q][0], o[p][q + 2][0], w.x, w.z);
            swap_halves(o[p][q][1], o[p][q + 2][1], w.y, w.w);
            *(uint4*)(g + 8 * q) = w;
          }
        }
      }
    }
  }
}

// ------------------------------------------------------------------ targets

struct TargetArgs {
  const void *h, *w;
  int64_t ldh, ldw, n;
  int d, classes, m, ntiles;
  float scale, tscale;
  const float* offset;
  const int32_t* ids;
  const float* tlogits;
  const float2* part;
  float *loss, *lse;
  // gradient
  const float* dloss;
  unsigned* level;  // the words of top_level; null: G holds dloss as it is
  float *lse2, *coef, *alpha;  // alpha: what a row of dH's sums is multiplied by, beside level
  int32_t* fix_id;  // n x m
  float* fix_val;
};

// One wavefront per row: joins the tiles' sums, takes the targets' logits, and
// writes loss and lse; for the gradient also the row's factor and its entries
// of G at the targets.  Bound by gathering the targets' rows of w: 4096 rows of 2048
// with 32 bfloat16 targets each (537 MB) 85 us, 6.3 TB/s.  Every P lanes take four
// targets at a time.  Of up to four targets a row's 64 lanes: the loss with ids at
// P = 64 / 16, 20000 rows of 784, 1000 bfloat16 classes 74 / 87 us, 8192 of 4096, 4000
// classes 238 / 263 (short rows differ by 3 %: 43373 of 35, 137 classes, 4 pairs 63 /
// 61).  Of more, 16, or 8 for short rows: at 64 / 16, the 20000 rows with 16 pairs
// 108 / 93, 49190 of 304, 217 classes, 10 pairs 98 / 75; at 64 / 8, 43373 of 35, 137
// classes, 47 pairs 310 / 85.
template <typename XT, int NQ, int P>
__global__ __launch_bounds__(256) void targets_kernel(TargetArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (i >= a.n) return;
  float m = -INFINITY, s = 0.f;
  for (int t = lane; t < a.ntiles; t += 64) {
    const float2 v = a.part[(int64_t)t * a.n + i];
    const float nm = fmaxf(m, v.x), n0 = nm == -INFINITY ? 0.f : nm;
    s = s * __builtin_amdgcn_exp2f(m - n0) + v.y * __builtin_amdgcn_exp2f(v.x - n0);
    m = nm;
  }
  float top = m;
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float top0 = top == -INFINITY ? 0.f : top;
  s = wave_sum(s * __builtin_amdgcn_exp2f(m - top0));
  const float lse2 = top + log2f(s);  // -inf where every class is left out

  // the row's pairs, lane l holding l, l + 64, ..: id (-1: none), q
  int id[NQ];
  float q[NQ], z[NQ], tm = -INFINITY, ts = 0.f;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    const int j = k * 64 + lane;
    id[k] = -1;
    q[k] = j < a.m ? pair_key(a.ids, a.tlogits, i * a.m + j, a.tscale, a.classes, id[k], bad) : -INFINITY;
    tm = fmaxf(tm, q[k]);
    z[k] = 0.f;
  }
  bad = __ballot(bad) != 0;
#pragma unroll
  for (int o = 32; o; o >>= 1) tm = fmaxf(tm, __shfl_xor(tm, o, 64));
  if (tm == -INFINITY) tm = 0.f;
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    q[k] = id[k] < 0 ? 0.f : pair_weight(q[k], tm, a.tscale);
    ts += q[k];
  }
  ts = wave_sum(ts);
  const bool some = ts != 0.f;  // (a NaN among the teacher's logits stays one)
  const float inv = some ? 1.f / ts : 0.f;
#pragma unroll
  for (int k = 0; k < NQ; ++k) q[k] *= inv;

  // the targets' logits, four dot products at a time by each P lanes
  constexpr int VEC = kVec<XT>, W = P * VEC, STEP = 4 * (64 / P);
  const int part = lane % P, group = lane / P;
  const XT* hr = (const XT*)a.h + i * a.ldh;
  shorts8 largest = {};  // of the row's binary16 features
  for (int j0 = 0; j0 < a.m; j0 += STEP) {
    const XT* wr[4];
    int idj[4];
    bool any = false;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      idj[u] = -1;
#pragma unroll
      for (int k = 0; k < NQ; ++k)
        if (j0 / 64 == k) idj[u] = __shfl(id[k], (j0 + 4 * group + u) & 63, 64);  // (STEP divides 64: one k for all)
      any |= idj[u] >= 0;
      wr[u] = (const XT*)a.w + (int64_t)max(idj[u], 0) * a.ldw;
    }
    if (!__any(any)) continue;
    // (a pair that is none reads row 0 of w, and its sum is not used)
    float dot[4] = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](const raw_vec<XT>& hv, const raw_vec<XT> (&wv)[4]) {
      if constexpr (std::is_same<XT, half_t>::value)  // (without their signs halves are ordered as their bits)
        largest = __builtin_elementwise_max(largest, __builtin_bit_cast(shorts8, hv) & (unsigned short)0x7fff);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) dot[u] = fmaf((float)hv[e], (float)wv[u][e], dot[u]);
    };
    int c = part * VEC;
#pragma unroll 4
    for (int c0 = 0; c0 + W <= a.d; c0 += W, c += W) {
      raw_vec<XT> wv[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) wv[u] = *(const any_vec<XT>*)(wr[u] + c);
      add(*(const any_vec<XT>*)(hr + c), wv);
    }
    if (c < a.d) {
      raw_vec<XT> wv[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) wv[u] = load_raw(wr[u], c, a.d);
      add(load_raw(hr, c, a.d), wv);
    }
    const int mine = (lane - j0) & 63;  // this lane's pair among the STEP
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (!__any(idj[u] >= 0)) continue;
      float sum = dot[u];
      if constexpr (P == 64) {
        sum = wave_sum(sum);
      } else {
#pragma unroll
        for (int o = P / 2; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
      }
      const float off = a.offset && idj[u] >= 0 ? a.offset[idj[u]] * kLog2e : 0.f;
      float zz = off == -INFINITY ? -INFINITY : fmaf(sum, a.scale * kLog2e, off);
      if constexpr (P < 64) zz = __shfl(zz, (mine / 4 * P) & 63, 64);
#pragma unroll
      for (int k = 0; k < NQ; ++k)
        if (j0 / 64 == k && mine < STEP && mine % 4 == u) z[k] = zz;
    }
  }
  float l = 0.f;
#pragma unroll
  for (int k = 0; k < NQ; ++k)
    if (q[k] != 0.f) {  // lse2 - z is +inf at a target that is left out, where every class is too
      const float gap = z[k] == -INFINITY ? INFINITY : lse2 - z[k];
      l += q[k] * (logf(q[k]) + gap * kLn2);
    }
  l = wave_sum(l);
  if (lane == 0) {
    a.loss[i] = bad ? __builtin_nanf("") : some ? l : 0.f;
    a.lse[i] = lse2 * kLn2;
  }
  if (!a.coef) return;
  const float dl = a.dloss[i];
  float cf = dl * a.scale;
  if (a.level) {
    const int e = exponent_of(dl);
    if (cf != 0.f) cf = ldexpf(dl, kHalfG - e);
    int bits = __builtin_reduce_max(largest);
#pragma unroll
    for (int o = 32; o; o >>= 1) bits = max(bits, __shfl_xor(bits, o, 64));
    if (lane == 0) {
      const float most = (float)__builtin_bit_cast(half_t, (unsigned short)bits);
      a.alpha[i] = ldexpf(a.scale, e - kHalfG);
      // (a row of none of these is 0 or NaN, whatever its level)
      if (some && !bad && cf != 0.f && isfinite(cf) && isfinite(lse2) && most > 0.f && isfinite(most))
        atomicMax(&a.level[(blockIdx.x & (kLevels - 1)) * kLevelStep],
                  (unsigned)(e + exponent_of(most) + kLevelBias));
    }
  }
  if (!some || lse2 == -INFINITY) cf = 0.f;
  if (bad) cf = __builtin_nanf("");
  if (lane == 0) {
    a.lse2[i] = lse2 == -INFINITY ? 0.f : lse2;
    a.coef[i] = cf;
  }
  // the entries of G at the targets, a class named twice once
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    const int j = k * 64 + lane;
    float qs = 0.f;
    bool first = true;
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
        if (jj < j) first = false;
      }
    }
    if (j < a.m) {
      a.fix_id[i * a.m + j] = first && cf != 0.f ? id[k] : -1;
      a.fix_val[i * a.m + j] = z[k] == -INFINITY ? 0.f : cf * (__builtin_amdgcn_exp2f(z[k] - lse2) - qs);
    }
  }
}

// The entries of G at the targets, for several a row: 1777 rows of 20 pairs 5 us, of
// which most is the launch.
template <typename E, int P>
__global__ __launch_bounds__(256) void fix_kernel(const int32_t* __restrict__ id, const float* __restrict__ val,
                                                  int64_t n, int m, int v0, int v1, E* __restrict__ G, int64_t ldg,
                                                  int64_t planeg, E* __restrict__ Gt, int64_t ldt, int64_t planet) {
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (x >= n * m) return;
  const int v = id[x];
  if (v < v0 || v >= v1) return;
  const int64_t i = x / m;
  E pl[P];
  split_planes<E, P>(val[x], pl);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    G[p * planeg + i * ldg + (v - v0)] = pl[p];
    Gt[p * planet + (v - v0) * ldt + i] = pl[p];
  }
}

// ------------------------------------------------------------------ products

struct ProductArgs {
  Side a, b;
  int64_t M, N;
  int K, nkc, nseg, mt, nt;
  int per;              // chunks of a slab
  unsigned blocks;      // tiles times slabs
  float* slabs;         // fp32 sums, M x N each, or null: straight to out
  int add;              // to what the slabs hold
  void* out;
  int64_t ldo;
  const float* alpha;   // null: 1
  int each;             // alpha holds one for each row
  const float* weight;  // rows whose weight is `none` are 0, whatever stands in a and b; may be null
  float none;
};
// The two products of a piece run in one launch where their tiles are alike.
// Bound by the matrix cores: both products of 8192 rows of 4096 and 16384 classes
// 1.96 ms, 1.12 PFLOP/s, matrix cores busy 63 %; 3001 rows of 1001 and 10007 binary16
// classes 139 us, 0.87: 160 workgroups have a tile of dW, 47 chunks long, and 96 half
// of a tile of dH, 79 chunks long, which the others wait for.
struct ProductJobs {
  ProductArgs j[2];
};

template <typename E, typename OT, class S>
__global__ __launch_bounds__(S::threads, S::per_cu) void product_kernel(ProductJobs jobs) {
  __shared__ __attribute__((aligned(1024))) char lds[S::lds_bytes];
  const bool second = blockIdx.x >= jobs.j[0].blocks;
  const ProductArgs& a = jobs.j[second];
  const unsigned g = blockIdx.x - (second ? jobs.j[0].blocks : 0u), tiles = (unsigned)(a.mt * a.nt);
  const int sl = __builtin_amdgcn_readfirstlane((int)(g / tiles));
  int mi, ni;
  tile_of(g - sl * tiles, tiles, a.mt, a.nt, mi, ni);
  const int64_t r0 = (int64_t)mi * S::BM, n0 = (int64_t)ni * S::BN;
  const int c0 = sl * a.per, c1 = min(c0 + a.per, a.nseg * a.nkc);
  floatx16 acc[S::WM][S::WN];
  tile_product<E, S>(a.a, a.b, r0, n0, a.K, a.nkc, a.nseg, c0, c1, lds, acc);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::GN, wn = wave % S::GN, l32 = lane & 31, h = lane >> 5;
  const float alpha = a.alpha && !a.each ? *a.alpha : 1.f;
  float* slab = a.slabs ? a.slabs + (int64_t)sl * a.M * a.N : nullptr;
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi) {
    const int64_t b0 = r0 + (wm * S::WM + bi) * 32;
    // what the rows are multiplied by, and which of them are 0, before any store
    float f[16];
    unsigned none = 0;
#pragma unroll
    for (int r = 0; r < 16; ++r) f[r] = alpha;
    if (std::is_same<E, half_t>::value && !slab && a.each)
#pragma unroll
      for (int r = 0; r < 16; ++r) f[r] = a.alpha[min(b0 + acc_row(r, h), a.M - 1)];
    if (!slab && a.weight)
#pragma unroll
      for (int r = 0; r < 16; ++r) none |= a.weight[min(b0 + acc_row(r, h), a.M - 1)] == a.none ? 1u << r : 0u;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int64_t row = b0 + acc_row(r, h);
      if (row >= a.M) continue;
#pragma unroll
      for (int bj = 0; bj < S::WN; ++bj) {
        const int64_t col = n0 + (wn * S::WN + bj) * 32 + l32;
        if (col >= a.N) continue;
        if (slab) {
          float* p = slab + row * a.N + col;
          *p = a.add ? *p + acc[bi][bj][r] : acc[bi][bj][r];
        } else {
          ((OT*)a.out)[row * a.ldo + col] = (OT)(none >> r & 1 ? 0.f : acc[bi][bj][r] * f[r]);
        }
      }
    }
  }
}

// out from the slabs, in order, so that the bits do not depend on timing; a thread
// takes four neighbouring entries of a row.  8192 rows of 4096, dH of bfloat16: 45 us.
struct SlabJob {
  const float* slabs;
  int count;
  int64_t M, N;
  const float* alpha;  // as ProductArgs'
  int each;
  const float* weight;
  float none;
  void* out;
  int64_t ldo;
  unsigned blocks;
};
struct SlabJobs {
  SlabJob j[2];
};
template <typename OT>
__global__ __launch_bounds__(256) void slabs_kernel(SlabJobs jobs) {
  const bool second = blockIdx.x >= jobs.j[0].blocks;
  const SlabJob& j = jobs.j[second];
  const float *slabs = j.slabs, *alpha = j.alpha, *weight = j.weight;
  OT* out = (OT*)j.out;
  const int count = j.count;
  const int64_t M = j.M, N = j.N, ldo = j.ldo;
  const int64_t per = (N + 3) / 4, step = (int64_t)j.blocks * 256;
  const float f = alpha && !j.each ? *alpha : 1.f;
  typedef OT o4 __attribute__((ext_vector_type(4)));
  typedef o4 any4 __attribute__((aligned(alignof(OT))));
  const unsigned first = second ? jobs.j[0].blocks : 0u;
  for (int64_t x = (int64_t)(blockIdx.x - first) * 256 + threadIdx.x; x < M * per; x += step) {
    const int64_t row = x / per, c = (x - row * per) * 4;
    const int m = (int)min((int64_t)4, N - c);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < count; ++k) {
      const float* p = slabs + (k * M + row) * N + c;
      if (m == 4) {
        const raw_vec<float> v = *(const any_vec<float>*)p;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += v[e];
      } else {
        for (int e = 0; e < m; ++e) s[e] += p[e];
      }
    }
    const float fr = j.each ? alpha[row] : f;
    const bool none = weight && weight[row] == j.none;
    o4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (OT)(none ? 0.f : s[e] * fr);
    if (m == 4)
      *(any4*)(out + row * ldo + c) = o;
    else
      for (int e = 0; e < m; ++e) out[row * ldo + c + e] = o[e];
  }
}

template <typename OT>
__global__ __launch_bounds__(256) void zero_rows_kernel(OT* __restrict__ out, int64_t M, int64_t N, int64_t ldo) {
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < M * N; x += (int64_t)gridDim.x * 256)
    out[x / N * ldo + x % N] = (OT)0.f;
}

// ------------------------------------------------------------------ plan

int64_t up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int kPad = 256;  // G's rows and classes: whole tiles of any shape

// (a tile's rows are reached by 32-bit offsets: kMaxStride)
constexpr int64_t kMaxStride = (int64_t)1 << 21;
bool in_place(const HeadArgs& a, const void* p, int64_t ld) {
  return a.type != TYPE_F32 && a.d % 8 == 0 && ld % 8 == 0 && ld <= kMaxStride && (uintptr_t)p % 16 == 0;
}

// What a launch of tiles takes, in microseconds, by which tiles and slabs are
// chosen.  A workgroup's chunk of 64 and its epilogue, as measured on full
// launches: 256 x 256 tiles 1.7 and 6 (scores 9, with G's stores 19), one on a
// CU; 128 x 128 tiles 1.2 and 4 (4, 9), two on a CU.
struct TileCost {
  double chunk, end;
  int slots;
};
TileCost tile_cost(bool big) { return big ? TileCost{1.7, 6, 256} : TileCost{1.2, 4, 512}; }
int64_t tile_count(int64_t M, int64_t N, bool big) {
  return big ? cdiv(M, BigTile::BM) * cdiv(N, BigTile::BN) : cdiv(M, SmallTile::BM) * cdiv(N, SmallTile::BN);
}
// A launch of scores; *big: in which tiles it takes less.
double scores_time(int64_t classes, int64_t n, int64_t chunks, int planes, bool grad, bool* big) {
  double t[2];
  for (int b = 0; b < 2; ++b) {
    const TileCost c = tile_cost(b);
    const double end = planes * (grad ? (b ? 19 : 9) : (b ? 9 : 4));
    t[b] = cdiv(tile_count(classes, n, b), c.slots) * (chunks * c.chunk + (grad ? end : end / planes));
  }
  *big = t[1] < t[0];
  return t[*big];
}
bool big_scores(int64_t classes, int64_t n, int64_t chunks, int planes, bool grad) {
  bool big;
  scores_time(classes, n, chunks, planes, grad, &big);
  return big;
}

// Class tiles whose logits stay for G rather than be multiplied again: those of
// the first piece that fit a piece's bytes, where that takes less.  4 bytes of each
// are written and read, beside G's, at 4.5 TB/s.  Microseconds with gradient,
// multiplied again / kept: fp32, 4553 rows of 3268, 834 classes 988 / 731, 8000 of
// 300, 1500 classes 305 / 282; bfloat16, 8000 classes of 8000 rows of 100 250 / 346,
// of 512 427 / 476, of 2048 1081 / 950; 984 classes of 2020 rows of 752 72 / 65;
// binary16, 2000 of 30000 of 256 343 / 406, 3000 of 18979 of 1979 1205 / 1077.  A part
// of the classes: bfloat16, 32768 of 8192 rows of 4096 8262 / 7969, fp32, 9001 of 9000
// of 1500 6080 / 5518.
int kept_tiles(int64_t classes, int64_t n, int64_t chunks, int planes, bool big, int piece) {
  const int side = big ? BigTile::BM : SmallTile::BM;
  const int64_t row_tiles = cdiv(n, side), bytes = row_tiles * side * side * 4;
  int64_t fit = std::min((int64_t)piece / side, (int64_t)(kPieceBytes / bytes));
  // (the other classes' tiles, of either shape, begin at a multiple of kPad and so end in the piece)
  fit = fit * side >= classes ? cdiv(classes, side) : fit * side / kPad * kPad / side;
  if (fit <= 0) return 0;
  bool again_big;
  const int64_t first = std::min<int64_t>(piece, classes), rest = first - std::min(first, fit * side);
  const double again = scores_time(first, n, chunks, planes, true, &again_big);
  const double left = rest ? 5 + scores_time(rest, n, chunks, planes, true, &again_big) : 0;
  const double keep = 8 + (double)(fit * bytes / 4) * (8 + 4 * planes) / 4.5e6;
  return 1.15 * keep + left < again ? (int)fit : 0;
}

// When the last of n0 workgroups of d0 and then n1 of d1 ends, dealt to `slots`
// places in order as these fall free.
double makespan(int64_t n0, double d0, int64_t n1, double d1, int slots) {
  if (n0 + n1 > 6 * (int64_t)slots) return (n0 * d0 + n1 * d1) / slots + 0.5 * std::max(d0, d1);
  struct Places {
    double at;
    int64_t count;
  } q[32] = {{0, slots}};  // ordered by time
  int len = 1;
  const int64_t n[2] = {n0, n1};
  const double d[2] = {d0, d1};
  double last = 0;
  for (int j = 0; j < 2; ++j)
    for (int64_t left = n[j]; left > 0;) {
      const int64_t take = std::min(left, q[0].count);
      const double end = q[0].at + d[j];
      last = std::max(last, end);
      left -= take;
      if (!(q[0].count -= take)) {
        for (int i = 1; i < len; ++i) q[i - 1] = q[i];
        --len;
      }
      int at = len;
      while (at > 0 && q[at - 1].at > end) --at;
      if (len == 32) return (n0 * d0 + n1 * d1) / slots + 0.5 * std::max(d0, d1);
      for (int i = len; i > at; --i) q[i] = q[i - 1];
      q[at] = {end, take};
      ++len;
    }
  return last;
}

// The two products of a piece, dH (of n x d over the piece's classes) and dW:
// tiles and slabs of each.  Tiles alike run in one launch, whose workgroups share
// the CUs; slabs are written and read once.  A
// gradient has the same bits whether or not the other one is asked for.
struct ProductChoice {
  bool big[2];
  int slabs[2];
};
ProductChoice choose_products(const int64_t (&M)[2], int64_t N, const int64_t (&chunks)[2]) {
  static const int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  ProductChoice best{};
  double least = 1e300;
  struct Side1 {
    int64_t wgs;
    double one, extra;
    bool big;
    int slabs;
  };
  Side1 opt[2][20];
  int num[2] = {0, 0};
  for (int j = 0; j < 2; ++j)
    for (int big = 0; big < 2; ++big)
      for (int s : counts) {
        if (s > 1 && chunks[j] / s < 4) break;
        const TileCost c = tile_cost(big);
        const int64_t wgs = tile_count(M[j], N, big) * s;
        if (s > 1 && wgs > 4 * c.slots) break;
        const double one = cdiv(chunks[j], s) * c.chunk + c.end;
        const double extra = s > 1 ? s * (double)M[j] * N * 8 / 4.5e6 : 0;
        opt[j][num[j]++] = {wgs, one, extra, big != 0, s};
      }
  for (int i = 0; i < num[0]; ++i)
    for (int k = 0; k < num[1]; ++k) {
      const Side1 &x = opt[0][i], &y = opt[1][k];
      const int sx = tile_cost(x.big).slots, sy = tile_cost(y.big).slots;
      double t = x.big == y.big ? makespan(x.wgs, x.one, y.wgs, y.one, sx)
                                : makespan(x.wgs, x.one, 0, 0, sx) + makespan(y.wgs, y.one, 0, 0, sy) + 5;
      t += x.extra + y.extra + (x.slabs > 1 || y.slabs > 1 ? 5 : 0);
      if (t < least) {
        least = t;
        best = {{x.big, y.big}, {x.slabs, y.slabs}};
      }
    }
  return best;
}

struct HeadPlan {
  int planes, nseg, kp;
  int64_t n_pad, v_pad;
  bool big, bigg;       // scores in BigTile: the forward pass, and for G
  int kept;             // class tiles whose logits stay for G
  int ntiles;
  int piece;            // classes of a piece (a multiple of kPad)
  int sh, sw;           // slabs of dH and dW (0: none)
  bool bigh, bigw;
  // workspace offsets
  size_t h, w, part, z, ht, wt, lse2, coef, level, alpha, alpha_w, fix_id, fix_val, G, Gt, slabs_h, slabs_w, bytes;
};

HeadPlan plan_of(const HeadArgs& a, bool grad) {
  HeadPlan p{};
  p.planes = a.type == TYPE_F32 ? 3 : 1;
  p.nseg = a.type == TYPE_F32 ? kSegs : 1;
  p.kp = (int)up(a.d, kChunkK);
  p.n_pad = up(a.n, kPad);
  p.v_pad = up(a.classes, kPad);
  p.big = big_scores(a.classes, a.n, (int64_t)p.nseg * p.kp / kChunkK, p.planes, false);
  p.ntiles = (int)cdiv(a.classes, p.big ? BigTile::BM : SmallTile::BM);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t r = at;
    at += up(bytes, 1024);
    return r;
  };
  if (!in_place(a, a.h, a.ldh)) p.h = take((size_t)p.planes * a.n * p.kp * 2);
  if (!in_place(a, a.w, a.ldw)) p.w = take((size_t)p.planes * a.classes * p.kp * 2);
  p.part = take((size_t)p.ntiles * a.n * 8);
  if (grad) {
    p.piece = (int)std::min<int64_t>(p.v_pad, std::max<int64_t>(kPad, kPieceBytes / ((size_t)p.planes * p.n_pad * 2) /
                                                                          kPad * kPad));
    p.ht = take((size_t)p.planes * a.d * p.n_pad * 2);
    p.wt = take((size_t)p.planes * a.d * p.v_pad * 2);
    p.lse2 = take((size_t)a.n * 4);
    p.coef = take((size_t)a.n * 4);
    // (2 KB between the operands and G: what a launch reads at a time meets in fewer
    // channels; both products of 8192 bfloat16 rows of 2048, 16384 classes 1020 -> 981 us)
    (void)take(2048);
    p.fix_id = take((size_t)a.n * a.m * 4);
    p.fix_val = take((size_t)a.n * a.m * 4);
    p.G = take((size_t)p.planes * p.n_pad * p.piece * 2);
    p.Gt = take((size_t)p.planes * p.n_pad * p.piece * 2);
    p.kept = kept_tiles(a.classes, a.n, (int64_t)p.nseg * p.kp / kChunkK, p.planes, p.big, p.piece);
    const int64_t side = p.big ? BigTile::BM : SmallTile::BM;
    p.z = take((size_t)(p.kept * cdiv(a.n, side) * side * side * 4));
    const int64_t pieces = cdiv(a.classes, p.piece), of_piece = std::min<int64_t>(p.piece, a.classes);
    p.bigg = big_scores(of_piece, a.n, (int64_t)p.nseg * p.kp / kChunkK, p.planes, true);
    const ProductChoice c = choose_products({a.n, of_piece}, a.d, {p.nseg * cdiv(of_piece, kChunkK),
                                                                   p.nseg * cdiv(a.n, kChunkK)});
    p.bigh = c.big[0];
    p.bigw = c.big[1];
    p.sh = c.slabs[0] > 1 || pieces > 1 ? c.slabs[0] : 0;
    p.sw = c.slabs[1] > 1 ? c.slabs[1] : 0;
    p.slabs_h = take((size_t)p.sh * a.n * a.d * 4);
    p.slabs_w = take((size_t)p.sw * std::min<int64_t>(p.piece, a.classes) * a.d * 4);
    if (a.type == TYPE_F16) {
      p.level = take(kLevels * kLevelStep * 4);
      p.alpha = take((size_t)a.n * 4);
      p.alpha_w = take(4);
    }
  }
  p.bytes = at;
  return p;
}

#define KKM_TRY(expr)                        \
  do {                                       \
    hipError_t e_ = (expr);                  \
    if (e_ != hipSuccess) return e_;         \
  } while (0)

unsigned blocks_of(int64_t items) { return (unsigned)std::min(cdiv(items, 256), kMaxBlocks); }

template <typename XT, typename E, int P>
struct Head {
  const HeadArgs& a;
  const HeadPlan& p;
  char* ws;
  hipStream_t s;

  template <typename T>
  T* at(size_t off) const { return (T*)(ws + off); }

  // The operands as they are multiplied: in place, or a copy at `off`, whose job joins `jobs`.
  Side side(const void* src, int64_t ld, int64_t rows, size_t off, StageJobs& jobs, int& count) const {
    if (in_place(a, src, ld)) return {src, ld, 0, rows};
    const int64_t plane = rows * p.kp;
    jobs.j[count] = {src, ld, rows, at<E>(off), plane, nullptr, 0.f, 0, nullptr};
    const unsigned blocks = blocks_of(rows * (p.kp / 8));
    if (count++ == 0) jobs.split = blocks;
    return {at<E>(off), p.kp, plane, rows};
  }

  template <int MODE>
  hipError_t scores(ScoreArgs<E> sa, int64_t classes) const {
    const bool big = MODE == SCORES_G ? p.bigg : p.big;
    sa.nkc = p.kp / kChunkK;
    sa.mt = (int)cdiv(classes, big ? BigTile::BM : SmallTile::BM);
    sa.nt = (int)cdiv(a.n, big ? BigTile::BN : SmallTile::BN);
    const dim3 grid((unsigned)((int64_t)sa.mt * sa.nt));
    if (big)
      hipLaunchKernelGGL((scores_kernel<E, BigTile, P, MODE>), grid, dim3(BigTile::threads), 0, s, sa);
    else
      hipLaunchKernelGGL((scores_kernel<E, SmallTile, P, MODE>), grid, dim3(SmallTile::threads), 0, s, sa);
    return hipGetLastError();
  }

  // chunks of a slab, and the slabs that a product of K writes
  int share(int K, int slabs) const {
    return (int)cdiv(cdiv(K, kChunkK) * p.nseg, std::max(slabs, 1));
  }
  int written(int K, int slabs) const {
    return (int)cdiv(cdiv(K, kChunkK) * p.nseg, share(K, slabs));
  }

  // out (M x N) = A B^T over K, or its slabs where there are any (K0: the first
  // piece's K, from which the slabs' shares are)
  ProductArgs product(Side x, Side y, int64_t M, int64_t N, int K, int K0, bool big, int slabs, float* slab, int add,
                      void* out, int64_t ldo, const float* alpha, int each, const float* weight,
                      float none) const {
    ProductArgs pa{};
    pa.a = x;
    pa.b = y;
    pa.M = M;
    pa.N = N;
    pa.K = K;
    pa.nkc = (int)cdiv(K, kChunkK);
    pa.nseg = p.nseg;
    pa.mt = (int)cdiv(M, big ? BigTile::BM : SmallTile::BM);
    pa.nt = (int)cdiv(N, big ? BigTile::BN : SmallTile::BN);
    pa.per = share(K0, slabs);
    pa.blocks = (unsigned)((int64_t)pa.mt * pa.nt * cdiv(pa.nkc * pa.nseg, pa.per));
    pa.slabs = slabs ? slab : nullptr;
    pa.add = add;
    pa.out = out;
    pa.ldo = ldo;
    pa.alpha = alpha;
    pa.each = alpha && each;
    pa.weight = weight;
    pa.none = none;
    return pa;
  }
  hipError_t multiply(const ProductJobs& jobs, bool big) const {
    const dim3 grid(jobs.j[0].blocks + jobs.j[1].blocks);
    if (big)
      hipLaunchKernelGGL((product_kernel<E, XT, BigTile>), grid, dim3(BigTile::threads), 0, s, jobs);
    else
      hipLaunchKernelGGL((product_kernel<E, XT, SmallTile>), grid, dim3(SmallTile::threads), 0, s, jobs);
    return hipGetLastError();
  }
  SlabJob sum(const float* slabs, int count, int64_t M, int64_t N, const float* alpha, int each, const float* weight,
              float none, void* out, int64_t ldo) const {
    return {slabs, count, M, N, alpha, alpha && each, weight, none, out, ldo, blocks_of(M * cdiv(N, 4))};
  }

  hipError_t run(bool grad) const {
    ScoreArgs<E> sa{};
    StageJobs copies{};
    int count = 0;
    sa.h = side(a.h, a.ldh, a.n, p.h, copies, count);
    sa.w = side(a.w, a.ldw, a.classes, p.w, copies, count);
    if (count) {
      const unsigned rest = count > 1 ? blocks_of(copies.j[1].rows * (p.kp / 8)) : 0u;
      hipLaunchKernelGGL((stage_rows_kernel<XT, E, P>), dim3(copies.split + rest), dim3(256), 0, s, copies, a.d, p.kp);
      KKM_TRY(hipGetLastError());
    }
    sa.n = a.n;
    sa.classes = a.classes;
    sa.K = in_place(a, a.h, a.ldh) || in_place(a, a.w, a.ldw) ? a.d : p.kp;
    sa.nseg = p.nseg;
    sa.zscale = a.scale * kLog2e;
    sa.offset = a.offset;
    sa.part = at<float2>(p.part);
    const bool half = grad && a.type == TYPE_F16;
    if (half) sa.level = at<unsigned>(p.level);
    if (grad) {
      sa.z = at<floatx4>(p.z);
      sa.kept = p.kept;
    }
    // (the classes whose logits are kept, 256 MB of them, lie in the first launch)
    const int64_t side = p.big ? BigTile::BM : SmallTile::BM, threads = p.big ? BigTile::threads : SmallTile::threads;
    const int64_t most = std::max<int64_t>(kMaxItems / (cdiv(a.n, side) * threads), 1) * side;
    for (int64_t v0 = 0; v0 < a.classes; v0 += most) {
      ScoreArgs<E> some = sa;
      some.v0 = (int)v0;
      if (v0) some.kept = 0;
      KKM_TRY(scores<SCORES_LOSS>(some, std::min(most, a.classes - v0)));
    }

    TargetArgs ta{a.h, a.w, a.ldh, a.ldw, a.n, a.d, a.classes, a.m, p.ntiles, a.scale, a.tscale, a.offset,
                  a.ids, a.tlogits, sa.part, a.loss, a.lse, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
    if (grad) {
      ta.dloss = a.dloss;
      ta.lse2 = at<float>(p.lse2);
      ta.coef = at<float>(p.coef);
      ta.fix_id = at<int32_t>(p.fix_id);
      ta.fix_val = at<float>(p.fix_val);
      if (half) {
        ta.level = sa.level;
        ta.alpha = at<float>(p.alpha);
      }
    }
    const dim3 tg((unsigned)cdiv(a.n, 4));
    auto targets = [&](auto P_) {
      constexpr int TP = decltype(P_)::value;
      if (a.m <= 64)
        hipLaunchKernelGGL((targets_kernel<XT, 1, TP>), tg, dim3(256), 0, s, ta);
      else
        hipLaunchKernelGGL((targets_kernel<XT, 4, TP>), tg, dim3(256), 0, s, ta);
    };
    if (a.m <= 4) targets(std::integral_constant<int, 64>{});
    else if (a.d <= 8 * kVec<XT>) targets(std::integral_constant<int, 8>{});
    else targets(std::integral_constant<int, 16>{});
    KKM_TRY(hipGetLastError());
    if (!grad) return hipSuccess;

    Side ht{at<E>(p.ht), p.n_pad, (int64_t)a.d * p.n_pad, a.d}, wt{at<E>(p.wt), p.v_pad, (int64_t)a.d * p.v_pad, a.d};
    StageJobs turned{};
    const float* alpha_w = half ? at<float>(p.alpha_w) : nullptr;
    if (a.dw) {
      if (half) {
        turned.level = ta.level;
        turned.scale = a.scale;
        turned.alpha = at<float>(p.alpha_w);
      }
      turned.j[0] = {a.h, a.ldh, a.n, at<E>(p.ht), ht.plane, ta.coef, 0.f, p.n_pad, half ? a.dloss : nullptr};
      turned.split = (unsigned)cdiv(a.n, 64);
    }
    if (a.dh) turned.j[1] = {a.w, a.ldw, a.classes, at<E>(p.wt), wt.plane, a.offset, -INFINITY, p.v_pad, nullptr};
    hipLaunchKernelGGL((stage_cols_kernel<XT, E, P>),
                       dim3(turned.split + (a.dh ? (unsigned)cdiv(a.classes, 64) : 0u), (unsigned)cdiv(a.d, 64)),
                       dim3(256), 0, s, turned, a.d);
    KKM_TRY(hipGetLastError());
    sa.lse2 = ta.lse2;
    sa.coef = ta.coef;
    if (a.m == 1) {
      sa.fix_id = ta.fix_id;
      sa.fix_val = ta.fix_val;
    }
    sa.G = at<E>(p.G);
    sa.Gt = at<E>(p.Gt);
    sa.ldg = p.piece;
    sa.planeg = sa.planet = p.n_pad * p.piece;
    sa.ldt = p.n_pad;
    const int kn = (int)up(a.n, kChunkK);
    const int kv0 = (int)up(std::min(p.piece, a.classes), kChunkK);
    for (int v0 = 0; v0 < a.classes; v0 += p.piece) {
      const int cnt = std::min(p.piece, a.classes - v0), kv = (int)up(cnt, kChunkK);
      sa.v0 = v0;
      const int kept = v0 ? 0 : (int)std::min<int64_t>(cnt, (int64_t)p.kept * (p.big ? BigTile::BM : SmallTile::BM));
      if (kept) KKM_TRY(scores<SCORES_G_OF_Z>(sa, kept));
      if (kept < cnt) {
        ScoreArgs<E> rest = sa;
        rest.v0 += kept;
        rest.G += kept;
        rest.Gt += (int64_t)kept * sa.ldt;
        KKM_TRY(scores<SCORES_G>(rest, cnt - kept));
      }
      if (a.m > 1) {
        hipLaunchKernelGGL((fix_kernel<E, P>), dim3((unsigned)cdiv(a.n * a.m, 256)), dim3(256), 0, s, ta.fix_id,
                           ta.fix_val, a.n, a.m, v0, v0 + cnt, sa.G, sa.ldg, sa.planeg, sa.Gt, sa.ldt, sa.planet);
        KKM_TRY(hipGetLastError());
      }
      ProductArgs ph{}, pw{};
      SlabJobs sums{};
      int n_sums = 0;
      if (a.dh) {
        Side wv = wt;
        wv.p = at<E>(p.wt) + v0;
        ph = product({sa.G, sa.ldg, sa.planeg, p.n_pad}, wv, a.n, a.d, kv, kv0, p.bigh, p.sh, at<float>(p.slabs_h),
                     v0 > 0, a.dh, a.lddh, ta.alpha, 1, ta.coef, 0.f);
        if (p.sh && v0 + p.piece >= a.classes)
          sums.j[n_sums++] = sum(at<float>(p.slabs_h), written(kv0, p.sh), a.n, a.d, ta.alpha, 1, ta.coef,
                                 0.f, a.dh, a.lddh);
      }
      if (a.dw) {
        XT* dw = (XT*)a.dw + (int64_t)v0 * a.lddw;
        // (a NaN in G or in h is in every class's sum, but not in the gradient of one left out)
        const float* off = a.offset ? a.offset + v0 : nullptr;
        pw = product({sa.Gt, sa.ldt, sa.planet, p.piece}, ht, cnt, a.d, kn, kn, p.bigw, p.sw, at<float>(p.slabs_w), 0,
                     dw, a.lddw, alpha_w, 0, off, -INFINITY);
        if (p.sw)
          sums.j[n_sums++] = sum(at<float>(p.slabs_w), written(kn, p.sw), cnt, a.d, alpha_w, 0, off,
                                 -INFINITY, dw, a.lddw);
      }
      if (a.dh && a.dw && p.bigh == p.bigw) {
        KKM_TRY(multiply({{ph, pw}}, p.bigh));
      } else {
        if (a.dh) KKM_TRY(multiply({{ph, {}}}, p.bigh));
        if (a.dw) KKM_TRY(multiply({{pw, {}}}, p.bigw));
      }
      if (n_sums) {
        hipLaunchKernelGGL((slabs_kernel<XT>), dim3(sums.j[0].blocks + sums.j[1].blocks), dim3(256), 0, s, sums);
        KKM_TRY(hipGetLastError());
      }
    }
    return hipSuccess;
  }
};

template <typename XT, typename E, int P>
hipError_t launch_typed(const HeadArgs& a, bool grad, void* scratch, hipStream_t s) {
  if (a.n == 0) {
    if (grad && a.dw) {
      hipLaunchKernelGGL((zero_rows_kernel<XT>), dim3(blocks_of((int64_t)a.classes * a.d)), dim3(256), 0, s,
                         (XT*)a.dw, a.classes, a.d, a.lddw);
      return hipGetLastError();
    }
    return hipSuccess;
  }
  const HeadPlan p = plan_of(a, grad);
  return Head<XT, E, P>{a, p, (char*)scratch, s}.run(grad);
}

}  // namespace

size_t head_scratch(const HeadArgs& a, bool grad) {
  return a.n == 0 ? 0 : head_form(a) != HEAD_TILED ? head_short_scratch(a, grad) : plan_of(a, grad).bytes;
}

hipError_t launch_head(const HeadArgs& a, bool grad, void* scratch, hipStream_t s) {
  if (a.n > 0 && head_form(a) != HEAD_TILED) return launch_head_short(a, grad, scratch, s);
  switch (a.type) {
    case TYPE_F32: return launch_typed<float, bf16_t, 3>(a, grad, scratch, s);
    case TYPE_F16: return launch_typed<half_t, half_t, 1>(a, grad, scratch, s);
    default: return launch_typed<bf16_t, bf16_t, 1>(a, grad, scratch, s);
  }
}

}  // namespace kkm
