// A row's answer from its logits: penalties for ids already given, biases, a mask
// of the ids allowed, and of what is left the first of the largest, its log
// probability and the log sum.  One pass over the logits: lanes hold 16 of them
// each, so that the largest is known before the sum and both before the store.
// A row is 16, 64 or 256 lanes wide; one of more than 256 lanes hold is cut into
// slices, whose (largest, sum, id) a second launch joins.
//
// What a row's lists say of a class lies in LDS, a word per class of the slice: how
// often it was given in the low bits, one more than the last of its biases above.
// Whole numbers, so that their order does not matter.  A bit per class says whether its
// word is used at all: lanes look at 4 or 8 of these at a time, and only classes that a
// list names cost more than their scale, mask, exponential and store.
//
// Bound by memory without lists (512 bfloat16 rows of 131072: 48 us, 5.6 TB/s; with masks
// 53), by the list phases' waits and the named classes with them: 64 ids given 75 us, 1024
// with 32 biases and a mask 101.  Six workgroups a CU (16 bits, two registers kept in
// memory; five of fp32) take 101 where five take 108 and what the compiler gives 124.
// Several slices a workgroup, 32 logits a lane and a part for each wavefront were slower.
#include <algorithm>
#include <climits>

#include "model_ops.h"
#include "vec_io.h"

namespace kkm {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kEach = 16;  // logits of a lane
constexpr int kAhead = 4;  // ids of a row's list that a lane reads before it needs them
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
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 5 : 6) void choose_kernel(ChooseArgs a, int slices, int64_t units) {
#pragma clang fp contract(off)
  constexpr int VEC = kVec<T>, EACH = kEach, NV = EACH / VEC, ROWS = 256 / L, WIDE = L * EACH;
  __shared__ unsigned word[LISTS ? 256 * EACH : 4];
  __shared__ unsigned used[LISTS ? 8 * EACH : 4];  // bits
  __shared__ float red_top[4], red_sum[4];
  __shared__ int red_id[4];
  const int l = threadIdx.x % L, r = threadIdx.x / L, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    // (n times slices is below 2^31; in scalar registers)
    const unsigned whole = L == 256 ? __builtin_amdgcn_readfirstlane((unsigned)unit / (unsigned)slices) : 0u;
    const int64_t row = L == 256 ? whole : unit * ROWS + r;
    const int slice = L == 256 ? __builtin_amdgcn_readfirstlane((unsigned)unit - whole * slices) : 0, v0 = slice * WIDE;
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
    const bool lost = which >= a.nmasks;
    unsigned own = r * WIDE;  // the row's words
    if (LISTS) {
      const int32_t* given = a.given + row * a.ngiven;
      const int32_t* biased = a.bias_ids + row * a.nbias;
      const int ngiven = here ? a.ngiven : 0, nbias = here ? a.nbias : 0;
      int g[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) g[k] = k * L + l < ngiven ? given[k * L + l] : -1;
      const int b0 = l < nbias ? biased[l] : -1;
      for (int e = threadIdx.x; e < 8 * EACH; e += 256) used[e] = 0;
      __syncthreads();
      // An entry of a list that lies in the slice.  First all clear their words (all of
      // them: 119 us where these few take 101, the cases' 512 rows of 131072).
      auto at = [&](int c, auto f) {
        if ((unsigned)(c - v0) < (unsigned)left) f(own + (c - v0));
      };
      auto claim = [&](unsigned w) {
        word[w] = 0;
        atomicOr(&used[w / 32], 1u << (w % 32));
      };
      at(b0, claim);
      for (int j = L + l; j < nbias; j += L) at(biased[j], claim);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) at(g[k], claim);
      for (int j = kAhead * L + l; j < ngiven; j += L) at(given[j], claim);
      __syncthreads();
      if (a.nbias) {  // (all biases before any count: a count lies below their bits)
        auto last = [&](int c, int j) { at(c, [&](unsigned w) { atomicMax(&word[w], (unsigned)(j + 1) << kCountBits); }); };
        last(b0, l);
        for (int j = L + l; j < nbias; j += L) last(biased[j], j);
        __syncthreads();
      }
      auto count = [&](unsigned w) { atomicAdd(&word[w], 1u); };
#pragma unroll
      for (int k = 0; k < kAhead; ++k) at(g[k], count);
      for (int j = kAhead * L + l; j < ngiven; j += L) at(given[j], count);
      __syncthreads();
    }
    float u[NV][VEC], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (j * L + l) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) u[j][e] = -INFINITY;
      if (c >= left) continue;
      unsigned out = 0, named = 0;  // bits of the vector's classes
      if (which >= 0 && !lost) out = ~(a.masks[(int64_t)which * a.words + (v0 + c) / 32] >> ((v0 + c) & 31));
      if (LISTS) named = used[(own + c) / 32] >> ((own + c) % 32) & ((1u << VEC) - 1);
      float p[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) p[e] = (float)raw[j][e];
      if (LISTS && named)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const unsigned count = named >> e & 1 ? word[own + c + e] & ((1u << kCountBits) - 1) : 0;
          if (!count) continue;
          const float f = (float)count * a.frequency, s = p[e] > 0.f ? p[e] / a.repeat : p[e] * a.repeat;
          p[e] = s - (a.presence + f);
        }
      if (a.offset) {
        float off[VEC];
        load_beside(a.offset + v0, c, left, 0.f, off);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (off[e] == -INFINITY) out |= 1u << e;  // whatever its logit
          p[e] = p[e] + off[e];
        }
      }
      if (LISTS && named)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const unsigned at = named >> e & 1 ? word[own + c + e] >> kCountBits : 0;
          if (!at) continue;
          const float b = a.bias[row * a.nbias + at - 1];
          if (b == -INFINITY) out |= 1u << e;
          p[e] = p[e] + b;
        }
      if (lost) out = 0;  // (NaN, what else is said of a class)
      if (c + VEC > left) out |= ~0u << (left - c);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        p[e] = p[e] * a.scale;
        if (lost) p[e] = __builtin_nanf("");
        u[j][e] = out >> e & 1 ? -INFINITY : p[e];
        top = fmaxf(top, u[j][e]);  // (a NaN comes out in the sum)
      }
    }
    const float mine = top;
#pragma unroll
    for (int o = (L < 64 ? L : 64) / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    if (L == 256) {
      if (lane == 0) red_top[wave] = top;
      __syncthreads();
      top = fmaxf(fmaxf(red_top[0], red_top[1]), fmaxf(red_top[2], red_top[3]));
    }
    int id = INT_MAX;
    if (mine == top && top > -INFINITY)
#pragma unroll
      for (int j = NV - 1; j >= 0; --j)
#pragma unroll
        for (int e = VEC - 1; e >= 0; --e)
          if (u[j][e] == top) id = v0 + (j * L + l) * VEC + e;
    float sum = 0.f;
    const float base = top == -INFINITY ? 0.f : top;
    if (base < INFINITY) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += __builtin_amdgcn_exp2f((u[j][e] - base) * kLog2e);
    } else {  // its equals alone, and a NaN
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += u[j][e] == base ? 1.f : u[j][e] != u[j][e] ? u[j][e] : 0.f;
    }
    if (a.out && here) {
      T* out = (T*)a.out + row * a.ldo + v0;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int c = (j * L + l) * VEC;
        if (c < left) store_part(out, c, left, u[j]);
      }
    }
#pragma unroll
    for (int o = (L < 64 ? L : 64) / 2; o; o >>= 1) {
      sum += __shfl_xor(sum, o, 64);
      id = min(id, __shfl_xor(id, o, 64));
    }
    if (L == 256) {
      if (lane == 0) red_sum[wave] = sum, red_id[wave] = id;
      __syncthreads();
      sum = (red_sum[0] + red_sum[1]) + (red_sum[2] + red_sum[3]);
      id = min(min(red_id[0], red_id[1]), min(red_id[2], red_id[3]));
    }
    const Part part = {top, sum, id, sum != sum};
    if (l == 0 && here) {
      if (slices > 1)
        ((Part*)a.parts)[unit] = part;
      else
        finish(a, row, part);
    }
    // before the next unit's words and reductions
    if ((L == 256 || LISTS) && unit + gridDim.x < units) __syncthreads();
  }
}

// A row's slices, by a wavefront.
__global__ __launch_bounds__(256) void join_kernel(ChooseArgs a, int parts) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.n) return;
  const Part* p = (const Part*)a.parts + row * parts;
  Part all = {-INFINITY, 0.f, INT_MAX, 0};
  for (int s = lane; s < parts; s += 64) {
    const Part q = p[s];
    all.bad |= q.bad;
    if (q.top > all.top || (q.top == all.top && q.id < all.id)) all.top = q.top, all.id = q.id;
  }
  near_top<64>(all.top, all.id);
  for (int s = lane; s < parts; s += 64)
    if (p[s].sum > 0.f) all.sum += p[s].sum * term(p[s].top, all.top);  // (of NaN or nothing: no part)
  all.sum = wave_sum(all.sum);
#pragma unroll
  for (int o = 32; o; o >>= 1) all.bad |= __shfl_xor(all.bad, o, 64);
  if (lane == 0) finish(a, row, all);
}

int slices_of(const ChooseArgs& a) {
  return a.classes > 64 * kEach ? (a.classes + 256 * kEach - 1) / (256 * kEach) : 1;
}

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
