// Causal attention of a sequence's last few tokens over its pages.
#include <algorithm>

#include "paged.hpp"

namespace rgd {

namespace {

// One workgroup per (token, query head), 256 positions at a time: scores, one
// position a thread; their running maximum and sum; the weighted values, one
// dimension a thread.
template <typename T>
__global__ __launch_bounds__(256) void paged_attn_kernel(PagedAttnArgs a) {
  __shared__ float qs[128], w[256], red[4], acc_s[256];
  const PagedView& c = a.c;
  const int s = blockIdx.x / a.n, i = blockIdx.x % a.n, h = blockIdx.y, g = h / (a.Hq / c.Hkv), t = threadIdx.x;
  const int m_new = a.n_new ? min(max(a.n_new[s], 0), a.n) : a.n;
  if (i >= m_new) return;
  const int end = paged_len(c, s) - m_new + i + 1;
  const size_t row = (size_t)s * a.n + i;
  const float scale = 1.f / sqrtf((float)c.D);
  if (t < c.D) qs[t] = load_f((const T*)a.q + row * a.ldq + (size_t)h * c.D + t) * scale;
  const T* pk = (const T*)a.pool_k;
  const T* pv = (const T*)a.pool_v;
  const int d = t % c.D, part = t / c.D, parts = 256 / c.D;
  float top = -INFINITY, sum = 0.f, acc = 0.f;
  __syncthreads();
  for (int p0 = 0; p0 < end; p0 += 256) {
    const int pos = p0 + t;
    float x = -INFINITY;
    if (pos < end) {
      const int page = c.pages[(size_t)s * c.width + pos / c.ps];
      if (page_ok(c, page)) {
        const T* kr = pk + (((size_t)page * c.Hkv + g) * c.ps + pos % c.ps) * c.D;
        x = 0.f;
        for (int e = 0; e < c.D; ++e) x += qs[e] * load_f(kr + e);
      }
    }
    const float nt = fmaxf(top, block_max(x, red));
    const float down = nt == -INFINITY ? 1.f : expf(top - nt);
    const float e = nt == -INFINITY ? 0.f : expf(x - nt);
    top = nt;
    sum = sum * down + block_sum(e, red);
    w[t] = e;
    __syncthreads();
    acc *= down;
    for (int j = part; j < 256 && p0 + j < end; j += parts) {
      const int page = c.pages[(size_t)s * c.width + (p0 + j) / c.ps];
      if (page_ok(c, page)) acc += w[j] * load_f(pv + (((size_t)page * c.Hkv + g) * c.D + d) * c.ps + (p0 + j) % c.ps);
    }
    __syncthreads();
  }
  acc_s[t] = acc;
  __syncthreads();
  if (t < c.D) {
    float o = 0.f;
    for (int k = 0; k < parts; ++k) o += acc_s[k * c.D + t];
    store_f((T*)a.out + row * a.Hq * c.D + (size_t)h * c.D + t, sum == 0.f ? 0.f : o / sum);
  }
  if (t == 0 && a.lse) a.lse[row * a.Hq + h] = sum == 0.f ? -INFINITY : top + logf(sum);
}

}  // namespace

size_t paged_attention_workspace_floats(const PagedView&, int, int) { return 64; }

hipError_t paged_attention(const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.c.S * a.n, a.Hq);
  if (a.c.esz == 2)
    hipLaunchKernelGGL(paged_attn_kernel<bf16_t>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(paged_attn_kernel<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace rgd
