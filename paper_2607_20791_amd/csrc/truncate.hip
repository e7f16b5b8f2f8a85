// One draw per row under temperature, top-k, top-p and min-p.
//
// With the ids in the order of their logits (equal ones by id) each limit keeps a leading part, and the kept ids are the
// shortest of these.  Weights are whole multiples of 2^-43 of the largest one's, so that sums are exact in 64-bit integers
// and no order of adding them matters.
#include <cmath>

#include "paged.hpp"
#include "weights.hpp"

namespace rgd {

namespace {

typedef unsigned long long u64;
constexpr double kOne = 8796093022208.0;  // 2^43: the largest weight; 2^20 of them stay below 2^63
constexpr int kThreads = 1024;

// The last id that a limit keeps, as (key, id): kept are larger keys, and equal ones up to that id.
struct Last {
  uint32_t key;
  int id;
  RGD_DEV bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= id); }
};

struct Row {
  const float* z;
  int V;
  float top;
  double per_z;
  RGD_DEV float at(int i) const {
    const float v = z[i] + 0.f;  // -0 is 0
    return v != v ? -INFINITY : v;
  }
  RGD_DEV u64 weight(float v) const {
    if (v == -INFINITY) return 0;
    return (u64)rint(exp2_f64(((double)v - (double)top) * per_z) * kOne);
  }
};

RGD_DEV u64 wave_sum_u64(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

struct Shared {
  u64 mass[256];
  unsigned count[256];
  u64 red[kThreads / 64];
  float fred[kThreads / 64];
  uint32_t key;
  int id;
  u64 left;
  unsigned rank;
};

RGD_DEV u64 block_total(u64 v, Shared& sh) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 t = 0;
  for (int i = 0; i < kThreads / 64; ++i) t += sh.red[i];
  return t;
}

// The sum over the threads before this one.
RGD_DEV u64 block_before(u64 v, Shared& sh) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  u64 incl = v;
  for (int o = 1; o < 64; o <<= 1) {
    const u64 t = __shfl_up(incl, o, 64);
    if (lane >= o) incl += t;
  }
  __syncthreads();
  if (lane == 63) sh.red[w] = incl;
  __syncthreads();
  u64 before = 0;
  for (int i = 0; i < w; ++i) before += sh.red[i];
  return before + incl - v;
}

// The last kept id where the ids in order reach a count (k > 0) or, of those that `in` keeps, a mass: eight bits of the
// key at a time.
RGD_DEV Last find(const Row& r, const Last& in, unsigned k, double mass, Shared& sh) {
  uint32_t prefix = 0, mask = 0;
  unsigned rank = 0;  // of the ids above the prefix
  u64 sum = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (threadIdx.x < 256) {
      sh.mass[threadIdx.x] = 0;
      sh.count[threadIdx.x] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < r.V; i += kThreads) {
      const float v = r.at(i);
      const uint32_t key = ordered_u32(v);
      if ((key & mask) == prefix && in.keeps(key, i)) {
        atomicAdd(&sh.count[key >> shift & 255], 1u);
        if (!k) atomicAdd(&sh.mass[key >> shift & 255], r.weight(v));
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int b = 255;
      unsigned n = rank;
      u64 m = sum;
      for (; b > 0; --b) {
        if (sh.count[b] && (k ? n + sh.count[b] >= k : (double)(m + sh.mass[b]) >= mass)) break;
        n += sh.count[b];
        m += sh.mass[b];
      }
      sh.key = prefix | (uint32_t)b << shift;
      sh.rank = n;
      sh.left = m;
    }
    __syncthreads();
    prefix = sh.key;
    rank = sh.rank;
    sum = sh.left;
    mask |= 255u << shift;
  }
  // the ids of this key, each of the same weight, in their order
  const float v = from_ordered_u32(prefix);
  const double w = (double)r.weight(v);
  u64 more;
  if (k) more = k - rank;
  else more = w > 0 ? (u64)fmax(ceil((mass - (double)sum) / w), 1.0) : 1;
  const int per = (r.V + kThreads - 1) / kThreads, i0 = threadIdx.x * per, i1 = min(i0 + per, r.V);
  u64 mine = 0;
  for (int i = i0; i < i1; ++i) mine += ordered_u32(r.at(i)) == prefix && in.keeps(prefix, i);
  u64 before = block_before(mine, sh);
  if (threadIdx.x == 0) sh.id = r.V - 1;
  __syncthreads();
  if (before < more && before + mine >= more)
    for (int i = i0; i < i1; ++i)
      if (ordered_u32(r.at(i)) == prefix && in.keeps(prefix, i) && ++before == more) sh.id = i;
  __syncthreads();
  return Last{prefix, sh.id};
}

__global__ __launch_bounds__(kThreads) void truncate_kernel(TruncateArgs a) {
  __shared__ Shared sh;
  const int row = blockIdx.x;
  Row r;
  r.z = a.z + (size_t)row * a.ldz;
  r.V = a.V;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < a.V; i += kThreads) top = fmaxf(top, r.at(i));
  top = block_max(top, sh.fred);
  if (!finite_top(top)) {
    if (threadIdx.x == 0) {
      a.out[row] = -1;
      if (a.logp) a.logp[row] = -INFINITY;
    }
    return;
  }
  r.top = top;
  const float T = a.T ? a.T[row] : 1.f;
  if (!(T > 0.f)) {
    int id = a.V;
    for (int i = threadIdx.x; i < a.V; i += kThreads)
      if (r.at(i) == top) id = min(id, i);
    __syncthreads();
    if (threadIdx.x == 0) sh.id = a.V;
    __syncthreads();
    atomicMin(&sh.id, id);
    __syncthreads();
    if (threadIdx.x == 0) {
      a.out[row] = sh.id;
      if (a.logp) a.logp[row] = 0.f;
    }
    return;
  }
  r.per_z = 1.4426950408889634 / (double)T;
  Last last{ordered_u32(-INFINITY), -1};  // every id that is above -inf
  const int k = a.top_k ? a.top_k[row] : 0;
  if (k > 0 && k < a.V) {
    const Last l = find(r, Last{0, a.V}, k, 0.0, sh);
    if (last.keeps(l.key, l.id)) last = l;  // else fewer than k are above -inf
  }
  const float p = a.top_p ? a.top_p[row] : 1.f;
  if (p < 1.f) {
    u64 mine = 0;
    for (int i = threadIdx.x; i < a.V; i += kThreads) {
      const float v = r.at(i);
      if (last.keeps(ordered_u32(v), i)) mine += r.weight(v);
    }
    const u64 total = block_total(mine, sh);
    last = find(r, last, 0, fmax((double)p, 0.0) * (double)total, sh);
  }
  const float mp = a.min_p ? a.min_p[row] : 0.f;
  if (mp > 0.f) {
    const float thr = threshold(top, mp < 1.f ? (double)T * log((double)mp) : 0.0);
    const uint32_t key = ordered_u32(thr);
    if (key > last.key) last = Last{key, a.V};
  }
  const int per = (a.V + kThreads - 1) / kThreads, i0 = threadIdx.x * per, i1 = min(i0 + per, a.V);
  u64 mine = 0;
  for (int i = i0; i < i1; ++i) {
    const float v = r.at(i);
    if (last.keeps(ordered_u32(v), i)) mine += r.weight(v);
  }
  u64 before = block_before(mine, sh);
  const u64 total = block_total(mine, sh);
  const double u = fmin(fmax((double)a.u[row], 0.0), 1.0 - 1.0 / 16777216.0);
  const double target = u * (double)total;
  if (mine && (double)before <= target && (double)(before + mine) > target)
    for (int i = i0; i < i1; ++i) {
      const float v = r.at(i);
      if (!last.keeps(ordered_u32(v), i)) continue;
      before += r.weight(v);
      if ((double)before > target) {
        a.out[row] = i;
        if (a.logp)
          a.logp[row] = (float)(((double)v - (double)top) / (double)T - log((double)total / kOne));
        break;
      }
    }
}

}  // namespace

size_t sample_truncated_workspace_bytes(int R, int V) { return 256; }

hipError_t sample_truncated(const TruncateArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(truncate_kernel, dim3(a.R), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace rgd
