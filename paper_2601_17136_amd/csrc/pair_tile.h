// The matrix product of operands held as two binary16 parts, for the products of
// an orthogonalised update: one workgroup's tile of A B^T.
//
// A value v is hi + 2^-11 lo, hi = v rounded to binary16 and lo 2^11 times the rest
// rounded again, at a power of two chosen so that the largest entry stays in range:
// 22 bits, as long as hi has its 11 (down to 2^-28 of a largest of 2^14), and 2^-50 of
// the largest below.  (lo at hi's own power kept 22 bits down to 2^-17 only and 2^-39
// below: binary16's smallest step.)  A product is hi hi + 2^-11 (lo hi + hi lo), lo lo
// lying below the last bit kept, on the 16-bit matrix cores; the two sums are fp32, by
// themselves, and joined once.
#pragma once
#include "head_tile.h"

namespace kkm {

// Rows of blocks of 32 contraction indices, 32 hi then 32 lo: 128 bytes, which a
// load takes whole.  Indices past the last are zero up to a whole block.
constexpr int kPairBlock = 32;
struct PairSide {
  const half_t* p;
  int64_t ld;  // elements, 64 a block
  int64_t rows;
};
inline int64_t pair_ld(int64_t k) { return (k + kPairBlock - 1) / kPairBlock * (2 * kPairBlock); }
__device__ inline int64_t pair_at(int64_t col) { return col / kPairBlock * (2 * kPairBlock) + col % kPairBlock; }
constexpr float kLoUp = 0x1p11f, kLoDown = 0x1p-11f;
__device__ inline void split_pair(float v, half_t& hi, half_t& lo) {
  hi = (half_t)v;
  lo = (half_t)((v - (float)hi) * kLoUp);
}
__device__ inline float join_pair(half_t hi, half_t lo) { return (float)hi + (float)lo * kLoDown; }

// acc = the tile at rows row0 of a and col0 of b over blocks [c0, c1) of the
// contraction.  Rows past an operand's end read its last one.  Loads go straight to
// LDS, NST - 1 blocks ahead; a step's operands are read from LDS during the step
// before, across the block's one barrier too.
template <class S>
__device__ inline void pair_product(const PairSide& a, const PairSide& b, int64_t row0, int64_t col0, int c0, int c1,
                                    char* lds, floatx16 (&acc)[S::WM][S::WN]) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host pass knows no buffer resources)
  constexpr unsigned kBound = 0x7ffffff0u;
  constexpr int L = S::LA + S::LB, F = S::WM + S::WN, per = S::WM * S::WN, NST = S::NST;
  constexpr int M = 3 * per, R = 2 * F;  // products and reads of a step
  constexpr int kAhead = (NST - 2) * L;  // loads that may be on their way when a block has to be there
  static_assert(kAhead < 64, "what the counter holds");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::GN, wn = wave % S::GN, l32 = lane & 31, h = lane >> 5;
  const int lrow = lane / S::slots;
  auto slot = [&](int j) { return (lane % S::slots) ^ S::turn(j * S::group + lrow); };
  unsigned va[S::LA], vb[S::LB];
#pragma unroll
  for (int j = 0; j < S::LA; ++j) {
    const int64_t r = row0 + (wave * S::LA + j) * S::group + lrow;
    va[j] = (unsigned)((min(r, a.rows - 1) - row0) * a.ld * 2) + slot(j) * 16;
  }
#pragma unroll
  for (int j = 0; j < S::LB; ++j) {
    const int64_t r = col0 + (wave * S::LB + j) * S::group + lrow;
    vb[j] = (unsigned)((min(r, b.rows - 1) - col0) * b.ld * 2) + slot(j) * 16;
  }
  floatx16 low[S::WM][S::WN];  // lo hi + hi lo
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
    for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[bi][bj][r] = low[bi][bj][r] = 0.f;
  const auto ra = __builtin_amdgcn_make_buffer_rsrc((void*)(a.p + row0 * a.ld), 0, kBound, 0x00027000);
  const auto rb = __builtin_amdgcn_make_buffer_rsrc((void*)(b.p + col0 * b.ld), 0, kBound, 0x00027000);
  int fc = c0, fst = 0;  // the block being fetched (past the last it is that one again), and its stage
  auto issue = [&](int j) {
    char* st = lds + fst * S::stage_bytes;
    const int so = fc * S::row_bytes;
    if (j < S::LA)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(st + (wave * S::LA + j) * 1024), 16, va[j], so, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rb, (lds_void*)(st + S::BM * S::row_bytes + (wave * S::LB + j - S::LA) * 1024), 16, vb[j - S::LA], so, 0, 0);
  };
  auto advance = [&]() {
    fst = fst + 1 == NST ? 0 : fst + 1;
    if (fc + 1 < c1) ++fc;
  };
  f16x8 fa[2][2][S::WM], fb[2][2][S::WN];  // [set][part: hi, lo]
  auto read = [&](int set, const char* st, int k, int i) {  // b and a, hi and then lo
    const int part = i >= F, o = i - part * F;
    const int sl = ((4 * part + 2 * k + h) ^ S::turn(l32)) * 16;
    if (o < S::WN)
      fb[set][part][o] = *(const f16x8*)(st + S::BM * S::row_bytes + ((wn * S::WN + o) * 32 + l32) * S::row_bytes + sl);
    else
      fa[set][part][o - S::WN] = *(const f16x8*)(st + ((wm * S::WM + o - S::WN) * 32 + l32) * S::row_bytes + sl);
  };
  // Products of b's lo, of a's lo, of hi and hi.
  auto multiply = [&](int k, const char* st, int kn) {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const int p = m / per, bi = m % per / S::WN, bj = m % S::WN;
      floatx16& sum = p == 2 ? acc[bi][bj] : low[bi][bj];
      sum = mfma16(fa[k][p == 1][bi], fb[k][p == 0][bj], sum);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = m * R / M; j < (m + 1) * R / M; ++j) read(k ^ 1, st, kn, j);
      if (k == 0)
#pragma unroll
        for (int j = m * L / M; j < (m + 1) * L / M; ++j) issue(j);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto arrive = [&]() {  // this wavefront's part of the next block is in LDS; the barrier: everyone's
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((kAhead & 15) | (kAhead >> 4) << 14 | 7 << 4);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int st = 0; st < NST - 1; ++st) {
#pragma unroll
    for (int j = 0; j < L; ++j) issue(j);
    advance();
  }
  arrive();
#pragma unroll
  for (int i = 0; i < R; ++i) read(0, lds, 0, i);
  int cst = 0;
  for (int c = c0; c < c1; ++c) {
    // (the block fetched goes into the stage of block c - 1, which everyone has read)
    const char* st = lds + cst * S::stage_bytes;
    cst = cst + 1 == NST ? 0 : cst + 1;
    multiply(0, st, 1);
    arrive();
    multiply(1, lds + cst * S::stage_bytes, 0);
    advance();
  }
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
    for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[bi][bj][r] = fmaf(low[bi][bj][r], kLoDown, acc[bi][bj][r]);
  wait_loads();
  __syncthreads();
#endif
}

}  // namespace kkm
