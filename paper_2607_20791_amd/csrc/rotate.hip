// Head norms, rotary positions and the append of a paged cache's new tokens, in one pass over the rows of a fused
// projection.
//
// y = x / sqrt(mean(x^2) + eps) * gain for each head of q and k; the pair (a, b) of the first `dim` dimensions becomes
// scale (a cos - b sin, b cos + a sin) of the angle position * freq.  Few operations a byte: reading the rows
// once and writing them once bounds it.
//
// An angle enters as a part of a turn: position * (freq / 2 pi) and its distance from the nearest whole number in fp64
// (2^31 positions lose 2^-23 of a turn at most), the rest in fp32, where sine and cosine of a part in [-1/2, 1/2] are
// exact to a rounding.  No table of angles is read, so a position may be anything.
#include <cmath>

#include "paged.hpp"

namespace rgd {

namespace {

// One workgroup per (16 positions that lie together in a page, KV head, sequence): the KV head's k and v and the query
// heads that read it.  A row is D / E neighbouring lanes with 16 bytes each.
template <typename T>
__global__ __launch_bounds__(256) void rotate_append_kernel(RotateArgs a) {
  constexpr int E = 16 / sizeof(T);
  __shared__ T vt[128][16 + E];
  __shared__ float2 turn[16][64];  // (cos, sin) of a position and pair
  __shared__ float rows[256 * E];
  const PagedView& c = a.c;
  const int s = blockIdx.x / a.blocks, g = blockIdx.y, D = c.D, G = a.G;
  const int m = a.n_new ? min(max(a.n_new[s], 0), a.n) : a.n;
  const int len = paged_len(c, s), base = len - m;  // position of token 0
  const int p0 = ((base >> 4) + (int)blockIdx.x % a.blocks) * 16;
  if (m == 0 || p0 >= len) return;
  const int lo = max(base - p0, 0), hi = min(len - p0, 16);  // the block's positions that are new
  const long long row0 = (long long)s * a.n + (p0 - base);   // token of the block's first position (from lo on)
  int page = -1;
  if (p0 >= 0) page = c.pages[(size_t)s * c.width + p0 / c.ps];
  const bool ok = page_ok(c, page);
  const size_t head = ((size_t)(ok ? page : 0) * c.Hkv + g) * c.ps * D;
  const int slot = ok ? p0 % c.ps : 0, half = a.dim / 2, per = D / E;
  T *pk = (T*)a.pool_k + head + (size_t)slot * D, *pv = (T*)a.pool_v + head + slot;

  for (int i = threadIdx.x; i < (hi - lo) * half; i += 256) {
    const int t = lo + i / half, j = i % half;
    const int pos = a.positions ? a.positions[row0 + t] : p0 + t;
    const double x = (double)pos * a.turns[j];
    float sn, cs;
    sincospif(2.f * (float)(x - rint(x)), &sn, &cs);
    turn[t][j] = float2{cs * a.scale, sn * a.scale};
  }
  for (int i = threadIdx.x; i < (hi - lo) * per; i += 256) {
    const int t = lo + i / per, d = i % per * E;
    const u32x4 v = *(const u32x4*)((const T*)a.v + (row0 + t) * a.ldv + g * D + d);
    const T* x = (const T*)&v;
#pragma unroll
    for (int e = 0; e < E; ++e) vt[d + e][t] = x[e];
  }
  __syncthreads();

  const int d = (int)threadIdx.x % per * E;
  float* mine = rows + (int)threadIdx.x / per * D;
  for (int i = threadIdx.x; i < (hi - lo) * (G + 1) * per; i += 256) {
    const int r = i / per, t = lo + r / (G + 1), h = r % (G + 1);  // head G: k
    const long long token = row0 + t;
    const T* src = h < G ? (const T*)a.q + token * a.ldq + (size_t)(g * G + h) * D
                         : (const T*)a.k + token * a.ldk + (size_t)g * D;
    const float* gain = h < G ? a.q_norm : a.k_norm;
    u32x4 in = *(const u32x4*)(src + d);
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = load_f((const T*)&in + e);
    if (gain) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) sum = fmaf(x[e], x[e], sum);
      for (int o = per / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      const float inv = 1.f / sqrtf(sum / D + a.eps);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] * inv * gain[d + e];
    }
    if (a.interleaved) {
#pragma unroll
      for (int e = 0; e < E; e += 2)
        if (d + e < a.dim) {
          const float2 w = turn[t][(d + e) / 2];
          const float p = x[e], q = x[e + 1];
          x[e] = p * w.x - q * w.y;
          x[e + 1] = q * w.x + p * w.y;
        }
    } else if (half) {
#pragma unroll
      for (int e = 0; e < E; ++e) mine[d + e] = x[e];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // a row's lanes read what its lanes wrote
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (d + e < a.dim) {
          const bool first = d + e < half;
          const float2 w = turn[t][first ? d + e : d + e - half];
          const float other = mine[first ? d + e + half : d + e - half];
          x[e] = x[e] * w.x + (first ? -other : other) * w.y;
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // before the next row's
      __builtin_amdgcn_wave_barrier();
    }
    u32x4 res;
#pragma unroll
    for (int e = 0; e < E; ++e) store_f((T*)&res + e, x[e]);
    if (h < G) *(u32x4*)((T*)a.out + token * a.ldo + (size_t)(g * G + h) * D + d) = res;
    else if (ok) *(u32x4*)(pk + (size_t)t * D + d) = res;
  }
  if (!ok) return;
  for (int i = threadIdx.x; i < D * (16 / E); i += 256) {
    const int dd = i / (16 / E), t = i % (16 / E) * E;
    T* dst = pv + (size_t)dd * c.ps + t;
    if (t >= lo && t + E <= hi) {
      *(u32x4*)dst = *(const u32x4*)&vt[dd][t];
    } else {
      for (int e = 0; e < E; ++e)
        if (t + e >= lo && t + e < hi) dst[e] = vt[dd][t + e];
    }
  }
}

}  // namespace

hipError_t paged_append_rotated(const RotateArgs& a0, hipStream_t s) {
  RotateArgs a = a0;
  a.blocks = (a.n + 14) / 16 + 1;  // that n positions can touch
  const dim3 grid(a.blocks * a.c.S, a.c.Hkv);
  if (a.c.esz == 2) hipLaunchKernelGGL(rotate_append_kernel<bf16_t>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(rotate_append_kernel<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

void rotary_frequencies(int dim, double theta, const RotaryScaling* scaling, double* freq, float* scale) {
  constexpr double kTurn = 6.283185307179586;
  const int half = dim / 2;
  *scale = 1.f;
  if (scaling && scaling->kind == kRotaryBase) theta *= std::pow(scaling->factor, dim / (dim - 2.0));
  for (int j = 0; j < half; ++j) freq[j] = std::pow(theta, -2.0 * j / dim);
  if (!scaling || scaling->kind == kRotaryBase) return;
  const double factor = scaling->factor, context = scaling->context, low = scaling->low, high = scaling->high;
  // the index of the pair that makes so many turns over the trained context
  auto index = [&](double turns) { return dim * std::log(context / (kTurn * turns)) / (2 * std::log(theta)); };
  double first = 0, last = 0;
  if (scaling->kind == kRotaryByIndex) {
    first = std::fmax(std::floor(index(high)), 0.0);
    last = std::fmin(std::ceil(index(low)), dim - 1.0);
    *scale = (float)(1.0 + 0.1 * std::log(factor));
  }
  for (int j = 0; j < half; ++j) {
    double kept = 0.0;  // the share that stays as it is
    if (scaling->kind == kRotaryByRotations) kept = (context * freq[j] / kTurn - low) / (high - low);
    if (scaling->kind == kRotaryByIndex) kept = 1.0 - (j - first) / std::fmax(last - first, 1e-3);
    kept = std::fmin(std::fmax(kept, 0.0), 1.0);
    freq[j] = freq[j] * ((1.0 - kept) / factor + kept);
  }
}

}  // namespace rgd
