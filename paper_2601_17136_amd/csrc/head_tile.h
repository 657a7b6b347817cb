// The 16-bit matrix product of the class head's kernels: one workgroup's tile
// of A B^T, both operands with their contraction index contiguous.
#pragma once
#include "tile_mma.h"
#include "vec_io.h"

#include <type_traits>

namespace kkm {

// An operand: rows of 16-bit values, K of them contiguous (a multiple of 8, at
// 16-byte aligned addresses), in 1 or 3 planes that sum to the values.
struct Side {
  const void* p;
  int64_t ld, plane;  // elements
  int64_t rows;
};
// Rows of a taken in another order, row i being row order[i] of memory; all of them lie
// within 2 GB of p.
struct InOrder {
  const int32_t* order;
};
struct AsTheyAre {};

// fp32 operands are three bfloat16 planes (hi, mid, lo: 24 bits, fp32's range),
// and their product the six plane products above 2^-24 of it, small ones first.
constexpr int kSegs = 6;
__device__ inline int seg_a(int s) { return s == 0 ? 2 : s == 2 || s == 3 ? 1 : 0; }
__device__ inline int seg_b(int s) { return s == 1 ? 2 : s == 2 || s == 4 ? 1 : 0; }

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
template <typename E>
using frag = std::conditional_t<std::is_same<E, bf16_t>::value, bf16x8, f16x8>;

__device__ inline floatx16 mfma16(f16x8 a, f16x8 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ inline floatx16 mfma16(bf16x8 a, bf16x8 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// x as P parts of type E, each the rest of those before rounded.
template <typename E, int P>
__device__ inline void split_planes(float x, E (&out)[P]) {
  out[0] = (E)x;
  if constexpr (P == 3) {
    const bool fin = isfinite((float)out[0]);
    const float r = fin ? x - (float)out[0] : 0.f;
    out[1] = (E)r;
    out[2] = (E)(r - (float)out[1]);
  }
}

constexpr int kChunkK = 64;  // contraction indices of a chunk, to which operands are padded

// A workgroup of GM x GN wavefronts, each WM x WN blocks of 32 x 32; NST chunks
// lie in LDS.
template <int WM_, int WN_, int GM_, int GN_, int NST_ = 2>
struct TileShape {
  static constexpr int WM = WM_, WN = WN_, GM = GM_, GN = GN_;
  static constexpr int NST = NST_, BM = WM * GM * 32, BN = WN * GN * 32, waves = GM * GN, threads = waves * 64;
  static constexpr int row_bytes = kChunkK * 2, slots = row_bytes / 16, group = 64 / slots;  // rows of a 1 KB load
  static constexpr int stage_bytes = (BM + BN) * row_bytes, lds_bytes = stage_bytes * NST;
  static constexpr int per_cu = lds_bytes <= 80 * 1024 ? 2 : 1;  // workgroups
  static constexpr int LA = BM / group / waves, LB = BN / group / waves;  // loads per wavefront and chunk
  static_assert(BM % (group * waves) == 0 && BN % (group * waves) == 0, "");
  static_assert(LA * group % 16 == 0 && LB * group % 16 == 0, "turn() of a wavefront's rows goes by its own");
  // 16-byte slot s of a row lies at s ^ turn(row): sixteen rows at one s meet in
  // none of LDS's 64 banks
  __device__ static int turn(int row) { return (row >> 1) & 7; }
};
using BigTile = TileShape<4, 2, 2, 4>;    // 256 x 256, 128 KB
using SmallTile = TileShape<2, 2, 2, 2>;  // 128 x 128, 64 KB

typedef __attribute__((address_space(3))) void lds_void;

__device__ inline void wait_loads() { __builtin_amdgcn_s_waitcnt(7 << 4); }  // every load and LDS read done

// acc = the tile at rows row0 of a and col0 of b, over chunks [c0, c1) of the
// nseg x nkc (segment, chunk) pairs.  Loads go straight to LDS and permute
// their source instead of their target, which is a wavefront's 1 KB in order.
// Rows past the operand's end read its last one (what they give is not stored),
// contraction indices past K read zero.  Chunk c + NST - 1 is requested
// while chunk c is multiplied; a step's operands are read from LDS while the
// step before is multiplied, across the chunk's one barrier too.
template <typename E, class S, class Rows = AsTheyAre>
__device__ inline void tile_product(const Side& a, const Side& b, int64_t row0, int64_t col0, int K, int nkc, int nseg,
                                    int c0, int c1, char* lds, floatx16 (&acc)[S::WM][S::WN], Rows rows = {}) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host pass knows no buffer resources)
  constexpr unsigned kBound = 0x7ffffff0u, kOut = 0x80000000u;
  constexpr int NS = kChunkK / 16, L = S::LA + S::LB, NST = S::NST;
  constexpr int SP = NS / 2;               // a chunk's loads go out in its first SP steps
  constexpr int kAhead = (NST - 2) * L;    // loads that may be on their way when a chunk has to be there
  static_assert(kAhead < 64, "what the counter holds");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::GN, wn = wave % S::GN, l32 = lane & 31, h = lane >> 5;
  const int lrow = lane / S::slots;
  auto slot = [&](int j) { return (lane % S::slots) ^ S::turn(j * S::group + lrow); };  // what this lane loads
  unsigned va[S::LA], vb[S::LB];
#pragma unroll
  for (int j = 0; j < S::LA; ++j) {
    const int64_t r = row0 + (wave * S::LA + j) * S::group + lrow;
    if constexpr (std::is_same<Rows, InOrder>::value)
      va[j] = (unsigned)(rows.order[min(r, a.rows - 1)] * a.ld * 2) + slot(j) * 16;
    else
      va[j] = (unsigned)((min(r, a.rows - 1) - row0) * a.ld * 2) + slot(j) * 16;
  }
#pragma unroll
  for (int j = 0; j < S::LB; ++j) {
    const int64_t r = col0 + (wave * S::LB + j) * S::group + lrow;
    vb[j] = (unsigned)((min(r, b.rows - 1) - col0) * b.ld * 2) + slot(j) * 16;
  }
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
    for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[bi][bj][r] = 0.f;

  // The chunk being fetched: its resources, place along k, and stage.  Past the
  // last chunk it is that one again, so that the count of loads stays.
  int fc = c0, fs = c0 / nkc, fk = c0 % nkc, fst = 0;
  auto base = [&](const Side& x, int plane, int64_t row) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)x.p + (plane * x.plane + row * x.ld) * 2), 0, kBound,
                                             0x00027000);
  };
  auto issue = [&](int j) {  // load j of the chunk's L
    const int left = K - fk * kChunkK;  // slots from left / 8 on lie past K
    char* st = lds + fst * S::stage_bytes;
    const int so = fk * S::row_bytes;
    if (j < S::LA) {
      auto r = base(a, nseg > 1 ? seg_a(fs) : 0, std::is_same<Rows, InOrder>::value ? 0 : row0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(st + (wave * S::LA + j) * 1024), 16,
                                               slot(j) * 8 < left ? va[j] : kOut, so, 0, 0);
    } else {
      const int i = j - S::LA;
      auto r = base(b, nseg > 1 ? seg_b(fs) : 0, col0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(st + S::BM * S::row_bytes + (wave * S::LB + i) * 1024),
                                               16, slot(i) * 8 < left ? vb[i] : kOut, so, 0, 0);
    }
  };
  auto next = [](int st) { return NST == 2 ? st ^ 1 : st + 1 == NST ? 0 : st + 1; };
  auto advance = [&]() {
    fst = next(fst);
    if (++fc < c1 && ++fk == nkc) {
      fk = 0;
      ++fs;
    }
  };
  frag<E> fa[2][S::WM], fb[2][S::WN];
  // operand i of step k (the columns' first: the products start with them)
  auto read = [&](int set, const char* st, int k, int i) {
    const int sl = ((2 * k + h) ^ S::turn(l32)) * 16;
    if (i < S::WN)
      fb[set][i] = *(const frag<E>*)(st + S::BM * S::row_bytes + ((wn * S::WN + i) * 32 + l32) * S::row_bytes + sl);
    else
      fa[set][i - S::WN] = *(const frag<E>*)(st + ((wm * S::WM + i - S::WN) * 32 + l32) * S::row_bytes + sl);
  };
  // The products of step k.  Among them, one at a time, so that the wavefronts
  // do not queue up for LDS or the loads with the matrix cores idle: the reads of
  // the next step's operands (step kn of stage st) and the step's share of the
  // next chunk's loads.
  auto multiply = [&](int k, const char* st, int kn) {
    constexpr int per = S::WM * S::WN, all = SP * per;
#pragma unroll
    for (int i = 0; i < per; ++i) {
      const int bi = i / S::WN, bj = i % S::WN;
      acc[bi][bj] = mfma16(fa[k & 1][bi], fb[k & 1][bj], acc[bi][bj]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = i * (S::WM + S::WN) / per; j < (i + 1) * (S::WM + S::WN) / per; ++j) read((k + 1) & 1, st, kn, j);
      if (k < SP)
#pragma unroll
        for (int j = ((k * per + i) * L + all - 1) / all; j < ((k * per + i + 1) * L + all - 1) / all; ++j) issue(j);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto arrive = [&]() {  // this wavefront's part of the next chunk is in LDS; the barrier: everyone's
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((kAhead & 15) | (kAhead >> 4) << 14 | 7 << 4);  // (0: every load) and every LDS read
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
  for (int i = 0; i < S::WM + S::WN; ++i) read(0, lds, 0, i);
  int cst = 0;
  for (int c = c0; c < c1; ++c) {
    // (the chunk fetched goes into the stage of chunk c - 1, which everyone has read)
    const char* st = lds + cst * S::stage_bytes;
    cst = next(cst);
#pragma unroll
    for (int k = 0; k < NS - 1; ++k) multiply(k, st, k + 1);
    arrive();
    multiply(NS - 1, lds + cst * S::stage_bytes, 0);
    advance();
  }
  wait_loads();
  __syncthreads();
#endif
}

// Entry r of a 32 x 32 block lies in row acc_row(r, lane / 32), column lane % 32.
__device__ inline int acc_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// Tile t of mt x nt as (row, column) tiles: XCD x = workgroup % 8 takes a
// contiguous run of the bands of 8 row tiles by their columns, so that what its
// workgroups read at a time meets in its L2.
__device__ inline void tile_of(unsigned g, unsigned total, int mt, int nt, int& mi, int& ni) {
  const unsigned per = total >> 3, rem = total & 7, x = g & 7;
  const unsigned t = x * per + min(x, rem) + (g >> 3);
  const unsigned band = t / (8u * nt), u = t - band * 8u * nt, p = min(8u, (unsigned)mt - band * 8u);
  mi = __builtin_amdgcn_readfirstlane((int)(band * 8u + u % p));  // (divisions run in vector registers)
  ni = __builtin_amdgcn_readfirstlane((int)(u / p));
}

}  // namespace kkm
