// What the sequences of a group share: the leading pages that all of them hold in front of their new tokens.
//
// Two short kernels, once for all layers of a turn: one finds, for each sequence, its group's first member with new tokens
// and how far their tables agree, the other the least of these over each group.  Both look through all sequences for
// each one (S^2 reads of the caches), so that nothing has to be cleared or counted by atomics and results never depend on
// an order.  288 sequences 4.8 + 4.7 us: two launches and the chains of reads in them bound it.
#include "paged.hpp"
#include "share.hpp"

namespace rgd {

namespace {

RGD_DEV int label_of(const ShareArgs& a, int s) { return a.group ? a.group[s] : 0; }
RGD_DEV int count_of(const ShareArgs& a, int s) { return a.n_new ? min(max(a.n_new[s], 0), a.n) : a.n; }

// The sums and minima of 256 threads, in all of them.
RGD_DEV int block_add(int v, int* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}
RGD_DEV int block_least(int v, int* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return min(min(red[0], red[1]), min(red[2], red[3]));
}

// One workgroup per sequence: its group's first member, the tokens of members before it, where its group's tokens
// start in the plan's list (behind n of each sequence with a lower label), and the pages that it has in common with the
// first member.
__global__ __launch_bounds__(256) void share_find_kernel(ShareArgs a, Plan p) {
  __shared__ int red[4];
  const int s = blockIdx.x, S = a.c.S, label = label_of(a, s), m = count_of(a, s);
  const bool grouped = (unsigned)label < (unsigned)S;
  int first = S, before = 0, lower = 0;
  if (grouped)
    for (int t = threadIdx.x; t < S; t += 256) {
      const int l = label_of(a, t), k = count_of(a, t);
      if (l == label && k > 0) {
        first = min(first, t);
        before += t < s ? k : 0;
      }
      lower += (unsigned)l < (unsigned)label;
    }
  first = block_least(first, red);
  before = block_add(before, red);
  lower = block_add(lower, red);
  const bool in = grouped && m > 0;
  const int most = in ? max(paged_len(a.c, s) - m, 0) / a.c.ps : 0;  // whole pages in front of the new tokens
  const int *mine = a.c.pages + (size_t)s * a.c.width, *like = a.c.pages + (size_t)(in ? first : s) * a.c.width;
  int run = most;
  for (int j0 = 0; in && first != s && j0 < run; j0 += 1024) {
    int miss = most;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = min(j0 + k * 256 + (int)threadIdx.x, most - 1);
      if (mine[j] != like[j]) miss = min(miss, j);
    }
    run = block_least(miss, red);
    if (run < most) break;
  }
  if (threadIdx.x == 0) {
    p.tokens[s] = m;
    p.leader[s] = in ? first : -1;
    p.run[s] = run;
    p.row[s] = lower * a.n + before;
    if (s == 0) *p.head = PlanHead::of(a.c, a.n, a.Hq);
  }
  if (in)
    for (int i = threadIdx.x; i < m; i += 256) p.rows[lower * a.n + before + i] = s * a.n + i;
}

// One workgroup per sequence, those of first members at work: what the group shares and its tokens.
__global__ __launch_bounds__(256) void share_groups_kernel(ShareArgs a, Plan p) {
  __shared__ int red[4];
  const int s = blockIdx.x, S = a.c.S, leader = p.leader[s];
  int least = 1 << 30, tokens = 0, members = 0;
  if (leader == s) {
    for (int t = threadIdx.x; t < S; t += 256)
      if (p.leader[t] == s) {
        least = min(least, p.run[t]);
        tokens += p.tokens[t];
        ++members;
      }
    least = block_least(least, red);
    tokens = block_add(tokens, red);
    members = block_add(members, red);
  }
  const int shared = leader == s && members > 1 ? least * a.c.ps : 0;
  if (threadIdx.x == 0) {
    p.group[s] = PlanGroup{shared, shared ? tokens : 0, p.row[s], 0};
    if (leader < 0) {
      p.shared[s] = 0;
      if (a.shared) a.shared[s] = 0;
    }
  }
  if (leader == s)
    for (int t = threadIdx.x; t < S; t += 256)
      if (p.leader[t] == s) {
        p.shared[t] = shared;
        if (a.shared) a.shared[t] = shared;
      }
}

}  // namespace

size_t paged_share_ints(const PagedView& c, int n) { return Plan::ints(c.S, n); }

hipError_t paged_share(const ShareArgs& a, hipStream_t s) {
  const Plan p(a.plan, a.c.S);
  hipLaunchKernelGGL(share_find_kernel, dim3(a.c.S), dim3(256), 0, s, a, p);
  hipLaunchKernelGGL(share_groups_kernel, dim3(a.c.S), dim3(256), 0, s, a, p);
  return hipGetLastError();
}

}  // namespace rgd
