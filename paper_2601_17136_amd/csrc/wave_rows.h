// Products of few rows with few rows over a long width, a wavefront by itself: it loads
// its share of the width in whole 128-byte lines, at any address, and turns it through
// LDS into the shape of the 16 x 16 matrix instructions.  (Lanes that load 16 bytes of 16
// rows each use half a line at a time: 32 bfloat16 rows of 4096 by 4096 took 15 us that
// way, half of them for the 32 rows, which lie in L2.)
#pragma once
#include "few_mma.h"

namespace kkm {

// NA x 16 rows of a by NB x 16 rows of b, WV wavefronts.
template <typename T, int NA_, int NB_, int WV_>
struct WaveRows {
  static constexpr int NA = NA_, NB = NB_, WV = WV_;
  static constexpr int chunk = 128 / (int)sizeof(T);  // elements of a row
  static constexpr int L = (NA + NB) * 2;             // loads of a chunk, 8 rows each
  static constexpr int lds_bytes = WV * L * 1024;
};

// acc[i][j] += a's block i by b's block j (a's rows are the instruction's rows) over this
// wavefront's chunks of [0, d), every WV-th; two are on their way in registers while one
// is multiplied.  row_a(r), row_b(r): where row r begins (rows past the last may repeat
// one).  Ends without a barrier.
template <typename T, class S, class RA, class RB>
__device__ inline void wave_rows(RA row_a, RB row_b, int d, char* lds, floatx4 (&acc)[S::NA][S::NB]) {
  constexpr int VEC = kVec<T>, L = S::L;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15,
            k4 = lane >> 4;
  // 16-byte slot s of a row lies at s ^ turn(row): sixteen rows at one s meet in none of LDS's banks
  auto turn = [](int row) { return (row >> 1) & 7; };
  const T* from[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const int r = i * 8 + lane / 8;
    from[i] = i < 2 * S::NA ? row_a(r) : row_b(r - 16 * S::NA);
  }
  char* own = lds + wave * (L * 1024);
  const int count = (d + S::chunk - 1) / S::chunk;
  raw_vec<T> reg[2][L];
  auto fetch = [&](int set, int c) {
    const int k = c * S::chunk + (lane & 7) * VEC;
    if ((c + 1) * S::chunk <= d) {
#pragma unroll
      for (int i = 0; i < L; ++i) reg[set][i] = *(const any_vec<T>*)(from[i] + k);
    } else if (c < count) {
#pragma unroll
      for (int i = 0; i < L; ++i) reg[set][i] = load_raw(from[i], k, d);
    }
  };
  auto in_order = []() {  // of the wavefront's own LDS accesses, which the hardware keeps
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  auto to_lds = [&](int set) {
    in_order();
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int r = i * 8 + lane / 8;
      *(raw_vec<T>*)(own + r * 128 + ((lane & 7) ^ turn(r)) * 16) = reg[set][i];
    }
    in_order();
  };
  auto products = [&]() {
    raw_vec<T> fa[2][S::NA], fb[2][S::NB];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int slot = ((4 * k + k4) ^ turn(l16)) * 16;
#pragma unroll
      for (int i = 0; i < S::NA; ++i) fa[k][i] = *(const raw_vec<T>*)(own + (i * 16 + l16) * 128 + slot);
#pragma unroll
      for (int j = 0; j < S::NB; ++j) fb[k][j] = *(const raw_vec<T>*)(own + ((S::NA + j) * 16 + l16) * 128 + slot);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < S::NA; ++i)
#pragma unroll
        for (int j = 0; j < S::NB; ++j) acc[i][j] = mfma_few(fa[k][i], fb[k][j], acc[i][j]);
  };
  int c = wave;
  fetch(0, c);
  fetch(1, c + S::WV);
  for (; c < count; c += 2 * S::WV) {
    to_lds(0);
    fetch(0, c + 2 * S::WV);
    products();
    if (c + S::WV >= count) break;
    to_lds(1);
    fetch(1, c + 3 * S::WV);
    products();
  }
}

}  // namespace kkm
