// A row's answer from its logits: penalties for ids already given, biases, a mask
// of the ids allowed, and of what is left the first of the largest, its log
// probability and the log sum.  One pass over the logits: lanes hold 16 of them
// each, so that the largest is known before the sum and both before the store.
// A row is 16, 64 or 256 lanes wide; one of more than 4096 classes is cut into
// slices, whose (largest, sum, id) a second launch joins.
//
// What a row's lists say of a class lies in LDS, a word per class of the slice:
// how often it was given in the low bits, one more than the last of its biases
// above.  Whole numbers, so that their order does not matter.
#include <algorithm>
#include <climits>

#include "model_ops.h"
#include "vec_io.h"

namespace kkm {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kEach = 16;         // logits of a lane
constexpr int kSlice = 256 * kEach;
constexpr int kCountBits = 22;
constexpr int64_t kMostBlocks = (int64_t)1 << 22;
static_assert(kMaxGiven < 1 << kCountBits, "a count stays below the biases' bits");
static_assert(kMaxBiases < 1 << (32 - kCountBits), "");

struct Part {
  float top, sum;
  int id, bad;
};

// (largest, lowest id of it) over L lanes of a wavefront.
template <int L>
__device__ inline void near_top(float& top, int& id) {
#pragma unroll
  for (int o = (L < 64 ? L : 64) / 2; o; o >>= 1) {
    const float t = __shfl_xor(top, o, 64);
    const int i = __shfl_xor(id, o, 64);
    if (t > top || (t == top && i < id)) top = t, id = i;
  }
}

__device__ inline void finish(const ChooseArgs& a, int64_t row, const Part& p) {
  const bool none = p.top == -INFINITY;
  const float l = logf(p.sum), nan = __builtin_nanf("");
  if (a.ids) a.ids[row] = none || p.bad ? -1 : p.id;
  if (a.logp) a.logp[row] = p.bad ? nan : none ? -INFINITY : -l;
  if (a.lse) a.lse[row] = p.bad ? nan : none ? -INFINITY : p.top + l;
}

// The sum of exponentials' term; an infinite largest counts itself alone.
__device__ inline float term(float u, float top) {
  return u == top ? 1.f : __builtin_amdgcn_exp2f((u - top) * kLog2e);
}

template <typename T, int L, bool LISTS>
__global__ __launch_bounds__(256) void choose_kernel(ChooseArgs a, int slices, int64_t units) {
#pragma clang fp contract(off)
  constexpr int VEC = kVec<T>, NV = kEach / VEC, ROWS = 256 / L, WIDE = L * kEach;
  __shared__ __attribute__((aligned(16))) unsigned word[LISTS ? kSlice : 4];
  __shared__ float red_top[4], red_sum[4];
  __shared__ int red_id[4], red_bad[4];
  const int l = threadIdx.x % L, r = threadIdx.x / L, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t row = L == 256 ? unit / slices : unit * ROWS + r;
    const int slice = L == 256 ? (int)(unit - row * slices) : 0, v0 = slice * WIDE;
    const bool here = row < a.n;
    const int left = here ? min(a.classes - v0, WIDE) : 0;  // classes of the row's slice
    raw_vec<T> raw[NV];
    const T* z = (const T*)a.z + (here ? row : 0) * a.ldz + v0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * L + l) * VEC;
      if (c < left) raw[j] = load_raw(z, c, left);
    }
    int which = -1;
    if (a.masks && here) which = a.mask_ids ? a.mask_ids[row] : (int)row;
    if (LISTS) {
#pragma unroll
      for (int j = 0; j < kEach / 4; ++j) *(uint4*)&word[(j * 256 + threadIdx.x) * 4] = uint4{0, 0, 0, 0};
      __syncthreads();
      unsigned* own = word + r * WIDE;
      if (here)
        for (int j = l; j < a.nbias; j += L) {
          const int c = a.bias_ids[row * a.nbias + j] - v0;
          if ((unsigned)c < (unsigned)left) atomicMax(own + c, (unsigned)(j + 1) << kCountBits);
        }
      __syncthreads();
      if (here)
        for (int j = l; j < a.ngiven; j += L) {
          const int c = a.given[row * a.ngiven + j] - v0;
          if ((unsigned)c < (unsigned)left) atomicAdd(own + c, 1u);
        }
      __syncthreads();
    }
    float u[NV][VEC], top = -INFINITY;
    int id = INT_MAX;
    bool bad = false;
    const bool lost = which >= a.nmasks;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * L + l) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) u[j][e] = -INFINITY;
      if (c >= left) continue;
      unsigned bits = ~0u;
      if (which >= 0 && !lost) bits = a.masks[(int64_t)which * a.words + (v0 + c) / 32] >> ((v0 + c) & 31);
      float off[VEC];
      if (a.offset) load_beside(a.offset + v0, c, left, 0.f, off);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float p = (float)raw[j][e];
        float b = 0.f;
        bool biased = false;
        if (LISTS) {
          const unsigned w = word[r * WIDE + c + e], count = w & ((1u << kCountBits) - 1), at = w >> kCountBits;
          if (count) {
            p = p > 0.f ? p / a.repeat : p * a.repeat;
            const float f = (float)count * a.frequency;
            p = p - (a.presence + f);
          }
          biased = at != 0;
          if (biased) b = a.bias[row * a.nbias + at - 1];
        }
        if (a.offset) p = p + off[e];
        if (biased) p = p + b;
        p = p * a.scale;
        if (lost) p = __builtin_nanf("");
        // (out, whatever its logit)
        if (!(bits >> e & 1) || c + e >= left || (a.offset && off[e] == -INFINITY) || b == -INFINITY) p = -INFINITY;
        u[j][e] = p;
        bad |= p != p;
        if (p > top) top = p, id = v0 + c + e;
      }
    }
    near_top<L>(top, id);
    if (L == 256) {
      if (lane == 0) red_top[wave] = top, red_id[wave] = id;
      __syncthreads();
      top = red_top[0], id = red_id[0];
#pragma unroll
      for (int w = 1; w < 4; ++w)
        if (red_top[w] > top || (red_top[w] == top && red_id[w] < id)) top = red_top[w], id = red_id[w];
    }
    float sum = 0.f;
    if (top > -INFINITY)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += term(u[j][e], top);
    if (a.out && here) {
      T* out = (T*)a.out + row * a.ldo + v0;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * L + l) * VEC;
        if (c < left) store_part(out, c, left, u[j]);
      }
    }
    int any = bad;
#pragma unroll
    for (int o = (L < 64 ? L : 64) / 2; o; o >>= 1) {
      sum += __shfl_xor(sum, o, 64);
      any |= __shfl_xor(any, o, 64);
    }
    if (L == 256) {
      if (lane == 0) red_sum[wave] = sum, red_bad[wave] = any;
      __syncthreads();
      sum = (red_sum[0] + red_sum[1]) + (red_sum[2] + red_sum[3]);
      any = red_bad[0] | red_bad[1] | red_bad[2] | red_bad[3];
    }
    const Part part = {top, sum, id, any};
    if (l == 0 && here) {
      if (slices > 1)
        ((Part*)a.parts)[unit] = part;
      else
        finish(a, row, part);
    }
    if (L == 256 || LISTS) __syncthreads();  // before the next unit's words and reductions
  }
}

// A row's slices, by a wavefront.
__global__ __launch_bounds__(256) void join_kernel(ChooseArgs a, int slices) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.n) return;
  const Part* p = (const Part*)a.parts + row * slices;
  Part all = {-INFINITY, 0.f, INT_MAX, 0};
  for (int s = lane; s < slices; s += 64) {
    const Part q = p[s];
    all.bad |= q.bad;
    if (q.top > all.top || (q.top == all.top && q.id < all.id)) all.top = q.top, all.id = q.id;
  }
  near_top<64>(all.top, all.id);
  for (int s = lane; s < slices; s += 64)
    if (p[s].sum > 0.f) all.sum += p[s].sum * term(p[s].top, all.top);
  all.sum = wave_sum(all.sum);
#pragma unroll
  for (int o = 32; o; o >>= 1) all.bad |= __shfl_xor(all.bad, o, 64);
  if (lane == 0) finish(a, row, all);
}

int slices_of(const ChooseArgs& a) { return a.classes > 64 * kEach ? (a.classes + kSlice - 1) / kSlice : 1; }

template <typename T, int L>
void launch_rows(const ChooseArgs& a, int slices, hipStream_t s) {
  const int64_t units = L == 256 ? a.n * slices : (a.n + 256 / L - 1) / (256 / L);
  const unsigned blocks = (unsigned)std::min(units, kMostBlocks);
  if (a.ngiven || a.nbias)
    choose_kernel<T, L, true><<<blocks, 256, 0, s>>>(a, slices, units);
  else
    choose_kernel<T, L, false><<<blocks, 256, 0, s>>>(a, slices, units);
}

template <typename T>
hipError_t launch_typed(const ChooseArgs& a, hipStream_t s) {
  const int slices = slices_of(a);
  if (a.classes <= 16 * kEach)
    launch_rows<T, 16>(a, 1, s);
  else if (a.classes <= 64 * kEach)
    launch_rows<T, 64>(a, 1, s);
  else
    launch_rows<T, 256>(a, slices, s);
  if (slices > 1) join_kernel<<<(unsigned)((a.n + 3) / 4), 256, 0, s>>>(a, slices);
  return hipGetLastError();
}

}  // namespace

size_t choose_scratch(const ChooseArgs& a) {
  const int slices = slices_of(a);
  return slices > 1 ? (size_t)a.n * slices * sizeof(Part) : 0;
}

hipError_t launch_choose(const ChooseArgs& a, hipStream_t s) {
  if (a.n == 0) return hipSuccess;
  if (a.type == TYPE_F32) return launch_typed<float>(a, s);
  return a.type == TYPE_F16 ? launch_typed<half_t>(a, s) : launch_typed<bf16_t>(a, s);
}

}  // namespace kkm
