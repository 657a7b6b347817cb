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

// A workgroup of GM x GN wavefronts, each WM x WN blocks of 32 x 32; chunks of
// kChunkK contraction indices, STAGES of them in LDS.
constexpr int kChunkK = 64;
template <int WM_, int WN_, int GM_, int GN_, int STAGES_>
struct TileShape {
  static constexpr int WM = WM_, WN = WN_, GM = GM_, GN = GN_, STAGES = STAGES_;
  static constexpr int BM = WM * GM * 32, BN = WN * GN * 32, waves = GM * GN, threads = waves * 64;
  static constexpr int stage_bytes = (BM + BN) * kChunkK * 2, lds_bytes = stage_bytes * STAGES;
  static constexpr int loads = (BM + BN) / 8 / waves;  // 1 KB loads (8 rows) per wavefront and chunk
  static_assert((BM / 8) % waves == 0 && (BN / 8) % waves == 0, "");
};
using BigTile = TileShape<4, 2, 2, 4, 2>;    // 256 x 256, 128 KB
using SmallTile = TileShape<2, 2, 2, 2, 2>;  // 128 x 128, 64 KB

typedef __attribute__((address_space(3))) void lds_void;

// acc = the tile at rows row0 of a and col0 of b, over chunks [c0, c1) of the
// nseg x nkc (segment, chunk) pairs.  A row in LDS is 128 bytes, its 16-byte
// slots at slot ^ (row % 8), so that neither the loads nor the operand reads
// meet in a bank; the loads permute their source instead of their target, which
// is a wavefront's 1 KB in order.  Rows past the operand's end read its last
// one (what they give is not stored), contraction indices past K read zero.
template <typename E, class S>
__device__ inline void tile_product(const Side& a, const Side& b, int64_t row0, int64_t col0, int K, int nkc, int nseg,
                                    int c0, int c1, char* lds, floatx16 (&acc)[S::WM][S::WN]) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host pass knows no buffer resources)
  constexpr int LA = S::BM / 8 / S::waves, LB = S::BN / 8 / S::waves;
  constexpr unsigned kBound = 0x7ffffff0u, kOut = 0x80000000u;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::GN, wn = wave % S::GN, l32 = lane & 31, h = lane >> 5;
  const int slot = (lane & 7) ^ (lane >> 3);  // of the source row lane / 8
  unsigned va[LA], vb[LB];
#pragma unroll
  for (int j = 0; j < LA; ++j) {
    const int64_t r = row0 + (wave * LA + j) * 8 + (lane >> 3);
    va[j] = (unsigned)((min(r, a.rows - 1) - row0) * a.ld * 2) + slot * 16;
  }
#pragma unroll
  for (int j = 0; j < LB; ++j) {
    const int64_t r = col0 + (wave * LB + j) * 8 + (lane >> 3);
    vb[j] = (unsigned)((min(r, b.rows - 1) - col0) * b.ld * 2) + slot * 16;
  }
#pragma unroll
  for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
    for (int bj = 0; bj < S::WN; ++bj)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[bi][bj][r] = 0.f;

  int fs = c0 / nkc, fk = c0 % nkc;  // the next chunk to fetch
  auto fetch = [&](int c) {
    const int sa = nseg > 1 ? seg_a(fs) : 0, sb = nseg > 1 ? seg_b(fs) : 0;
    auto ra = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)a.p + (sa * a.plane + row0 * a.ld) * 2), 0,
                                                kBound, 0x00027000);
    auto rb = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)b.p + (sb * b.plane + col0 * b.ld) * 2), 0,
                                                kBound, 0x00027000);
    char* st = lds + ((c - c0) % S::STAGES) * S::stage_bytes;
    const int so = fk * (kChunkK * 2);
    const bool out = fk * kChunkK + slot * 8 >= K;
#pragma unroll
    for (int j = 0; j < LA; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(st + (wave * LA + j) * 1024), 16, out ? kOut : va[j],
                                               so, 0, 0);
#pragma unroll
    for (int j = 0; j < LB; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void*)(st + S::BM * 128 + (wave * LB + j) * 1024), 16,
                                               out ? kOut : vb[j], so, 0, 0);
    if (++fk == nkc) {
      fk = 0;
      ++fs;
    }
  };
  fetch(c0);
  for (int c = c0; c < c1; ++c) {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wavefront's part of chunk c; the barrier: everyone's
    __syncthreads();                     // and everyone has read chunk c - 1, whose buffer c + 1 takes
    if (c + 1 < c1) fetch(c + 1);
    const char* st = lds + ((c - c0) % S::STAGES) * S::stage_bytes;
#pragma unroll
    for (int k = 0; k < kChunkK / 16; ++k) {
      const int sl = ((2 * k + h) ^ (l32 & 7)) * 16;
      frag<E> fa[S::WM], fb[S::WN];
#pragma unroll
      for (int bi = 0; bi < S::WM; ++bi)
        fa[bi] = *(const frag<E>*)(st + ((wm * S::WM + bi) * 32 + l32) * 128 + sl);
#pragma unroll
      for (int bj = 0; bj < S::WN; ++bj)
        fb[bj] = *(const frag<E>*)(st + S::BM * 128 + ((wn * S::WN + bj) * 32 + l32) * 128 + sl);
#pragma unroll
      for (int bi = 0; bi < S::WM; ++bi)
#pragma unroll
        for (int bj = 0; bj < S::WN; ++bj) acc[bi][bj] = mfma16(fa[bi], fb[bj], acc[bi][bj]);
    }
  }
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
