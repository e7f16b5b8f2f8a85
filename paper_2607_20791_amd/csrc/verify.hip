// Verification of drafted tokens against the target's truncated distribution.
//
// With w_j = exp((z_j - max z) / T) for the kept ids (w_j >= min_p) and W their
// sum, p_j = w_j / W.  Draft x of the distribution q is accepted while
// u q(x) < p(x); the first refusal draws from max(p - q, 0).  Sequences sampled
// this way are distributed as if drawn from p one by one: x is emitted with
// probability min(p, q) + (1 - sum min(p, q)) max(p - q, 0) / sum max(p - q, 0) = p.
#include <algorithm>
#include <cmath>

#include "paged.hpp"

namespace rgd {

namespace {

constexpr int kThreads = 1024;

RGD_DEV double block_sum_f64(double v, double* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < kThreads / 64; ++i) t += red[i];
  return t;
}

// One row's distribution: the maximum, the lowest kept z - max, the sum of the
// weights.  alive: the maximum is finite.  T == 0: first holds the argmax.
struct RowDist {
  float top;
  double W;
  int first;
  bool alive;
};

struct Rule {
  double T, low;  // kept: z - max >= low
};

RGD_DEV double weight(const Rule& k, const RowDist& r, float z, int id) {
  if (k.T == 0.0) return id == r.first ? 1.0 : 0.0;
  const double x = (double)z - (double)r.top;
  return x >= k.low ? exp(x / k.T) : 0.0;
}

RGD_DEV RowDist row_dist(const float* z, int V, const Rule& k, double* red, float* redf, int* redi) {
  RowDist r;
  float mx = -INFINITY;
  for (int i = threadIdx.x; i < V; i += kThreads) mx = fmaxf(mx, z[i]);
  r.top = block_max(mx, redf);
  r.alive = r.top > -INFINITY && r.top < INFINITY;
  r.first = 0x7FFFFFFF;
  r.W = 1.0;
  if (!r.alive) return r;
  if (k.T == 0.0) {
    int at = 0x7FFFFFFF;
    for (int i = threadIdx.x; i < V; i += kThreads)
      if (z[i] == r.top) at = min(at, i);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) at = min(at, __shfl_xor(at, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) redi[threadIdx.x >> 6] = at;
    __syncthreads();
    for (int i = 0; i < kThreads / 64; ++i) r.first = min(r.first, redi[i]);
    return r;
  }
  double w = 0.0;
  for (int i = threadIdx.x; i < V; i += kThreads) w += weight(k, r, z[i], i);
  r.W = block_sum_f64(w, red);
  return r;
}

// One workgroup per sequence, its rows one after the other.
__global__ __launch_bounds__(kThreads) void verify_kernel(VerifyArgs a, Rule k) {
  __shared__ double red[kThreads / 64];
  __shared__ float redf[kThreads / 64];
  __shared__ int redi[kThreads / 64];
  const int s = blockIdx.x, t = threadIdx.x;
  const int nd = a.n_draft ? min(max(a.n_draft[s], 0), a.K) : a.K;
  const bool onehot = !a.draft || k.T == 0.0;
  const float* u = a.u + (size_t)s * (a.K + 1);
  int* out = a.out + (size_t)s * (a.K + 1);
  const int* x = a.tokens + (size_t)s * a.K;
  int i = 0;
  RowDist p, q;
  bool refused = false, inside = false;
  const float *zp = nullptr, *zq = nullptr;
  for (;; ++i) {
    zp = a.target + ((size_t)s * (a.K + 1) + i) * a.V;
    p = row_dist(zp, a.V, k, red, redf, redi);
    if (i >= nd) break;
    const int id = x[i];
    inside = (unsigned)id < (unsigned)a.V;
    double px = 0.0, qx = 0.0;
    if (inside && p.alive) px = weight(k, p, zp[id], id) / p.W;
    if (onehot) {
      qx = 1.0;
    } else {
      zq = a.draft + ((size_t)s * a.K + i) * a.V;
      q = row_dist(zq, a.V, k, red, redf, redi);
      if (inside && q.alive) qx = weight(k, q, zq[id], id) / q.W;
    }
    if (!((double)u[i] * qx < px)) {
      refused = true;
      break;
    }
    if (t == 0) out[i] = id;
  }
  if (t == 0) a.n_accepted[s] = i;
  for (int j = i + 1 + t; j <= a.K; j += kThreads) out[j] = -1;
  if (!p.alive) {
    if (t == 0) out[i] = -1;
    return;
  }
  // the draw: thread t owns ids [t * per, (t + 1) * per)
  const int per = (a.V + kThreads - 1) / kThreads, lo = min(a.V, t * per), hi = min(a.V, lo + per);
  const int taken = refused && inside ? x[i] : -1;
  const bool sub = refused && !onehot && q.alive;
  auto rest = [&](int id, bool plain) {
    double r = weight(k, p, zp[id], id) / p.W;
    if (plain) return r;
    if (sub) r -= weight(k, q, zq[id], id) / q.W;
    else if (onehot && id == taken) r = 0.0;
    return r > 0.0 ? r : 0.0;
  };
  bool plain = false;
  double mine = 0.0, all = 0.0;
  for (int round = 0; round < 2 && all == 0.0; ++round) {
    plain = round == 1;  // nothing left (rounding): p itself
    mine = 0.0;
    for (int id = lo; id < hi; ++id) mine += rest(id, plain);
    all = block_sum_f64(mine, red);
  }
  double incl = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double v = __shfl_up(incl, o, 64);
    if ((t & 63) >= o) incl += v;
  }
  __syncthreads();
  if ((t & 63) == 63) red[t >> 6] = incl;
  __syncthreads();
  double run = incl - mine;
  for (int w = 0; w < t >> 6; ++w) run += red[w];
  const double target = (double)u[a.K] * all;
  int found = 0x7FFFFFFF, last = -1;
  for (int id = lo; id < hi; ++id) {
    const double r = rest(id, plain);
    if (r <= 0.0) continue;
    run += r;
    last = id;
    if (run > target) {
      found = id;
      break;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    found = min(found, __shfl_xor(found, o, 64));
    last = max(last, __shfl_xor(last, o, 64));
  }
  __shared__ int sf[kThreads / 64], sl[kThreads / 64];
  if ((t & 63) == 0) {
    sf[t >> 6] = found;
    sl[t >> 6] = last;
  }
  __syncthreads();
  if (t == 0) {
    for (int w = 0; w < kThreads / 64; ++w) {
      found = min(found, sf[w]);
      last = max(last, sl[w]);
    }
    out[i] = found != 0x7FFFFFFF ? found : last;
  }
}

}  // namespace

size_t verify_workspace_bytes(int, int, int) { return 256; }

hipError_t verify_drafts(const VerifyArgs& a, hipStream_t s) {
  const Rule k{(double)a.T, a.min_p > 0.f ? (double)a.T * std::log((double)a.min_p) : -(double)INFINITY};
  hipLaunchKernelGGL(verify_kernel, dim3(a.S), dim3(kThreads), 0, s, a, k);
  return hipGetLastError();
}

}  // namespace rgd
