// Head norms, rotary positions and the append of a paged cache's new tokens, in one pass over the rows of a fused
// projection.
//
// y = x / sqrt(mean(x^2) + eps) * gain for each head of q and k; the pair (a, b) of the first `dim` dimensions becomes
// scale (a cos - b sin, b cos + a sin) of the angle position * freq.  Reading the rows once and writing them once bounds
// it from below, at 5.35 TB/s; the operations on a row, some 110 a lane, are the greater part of the rest.  8 x 1000 tokens
// of 32 + 8 + 8 heads of 128 in bf16, 109 MB: 26 us, 4.1 TB/s, where the last-level cache still holds the rows, and 32 to 34, 3.3 TB/s,
// where it does not.  Pairs of neighbours 26 us, of half a head 28, at odd distances 31; fp32 55 to 62.  One token: 5.9 us (7.6 a call), of
// which the launch and three loads that need one another's results are most.
//
// An angle enters as a part of a turn: position * (freq / 2 pi) and its distance from the nearest whole number in fp64
// (2^31 positions lose 2^-23 of a turn at most), the rest in fp32, where sine and cosine of a part in [-1/2, 1/2] are
// exact to a rounding.  No table of angles is read, so a position may be anything.
#include <cmath>
#include <type_traits>

#include "paged.hpp"

namespace rgd {

namespace {

constexpr int kFill = 768;  // workgroups that the chip holds, three per CU

// Where the other value of a pair is: in the same lane; eight lanes on of sixteen, one place of it; in one other lane, in the
// same place; or anywhere in the row.
enum Partner { kSame, kAcross, kLane, kAny };
template <typename T>
Partner partner_of(int D, int dim, int interleaved) {
  constexpr int E = 16 / sizeof(T);
  return interleaved || dim == 0 ? kSame : dim == D && D == 16 * E ? kAcross : dim / 2 % E == 0 ? kLane : kAny;
}

// The sum of neighbouring lanes' values, in each of them.
template <int LANES>
RGD_DEV float sum_lanes(float v) {
  auto add = [&](auto ctrl) {
    const int x = __float_as_int(v);
    v += __int_as_float(__builtin_amdgcn_update_dpp(x, x, decltype(ctrl)::value, 0xf, 0xf, false));
  };
  add(std::integral_constant<int, 0xb1>());                             // lane ^ 1
  add(std::integral_constant<int, 0x4e>());                             // lane ^ 2
  if constexpr (LANES >= 8) add(std::integral_constant<int, 0x141>());  // 7 - lane of eight
  if constexpr (LANES >= 16) add(std::integral_constant<int, 0x128>()); // eight lanes on of sixteen
  if constexpr (LANES >= 32) v += __shfl_xor(v, 16, 64);
  return v;
}

// One workgroup per (16 positions that lie together in a page, `heads` KV heads, sequence): the KV heads' k and v and the
// query heads that read them.  A row is D / E neighbouring lanes with 16 bytes each; a thread keeps to one position, so it
// reads that one's sines and cosines once, and takes every few of its rows, kAhead of which are on their way (a call of
// the case above: four 35 us, six 32, eight 33, ten 33.5).  Angles are taken once for the heads of a workgroup, so it
// takes as many as leave the chip full: one KV head per workgroup 44 us, two 41, four 33, eight 49, all with four rows.
template <typename T, int D, Partner P>
__global__ __launch_bounds__(256, 3) void rotate_append_kernel(RotateArgs a) {
  constexpr int E = 16 / sizeof(T), kLanes = D / E, kRows = 256 / kLanes, kAhead = 6, kV = (16 * kLanes + 255) / 256;
  __shared__ T vt[2][D][16 + E];
  __shared__ float2 turn[16][D / 2 + 1];  // (cos, sin) of a position and pair
  __shared__ float rows[P == kAny ? kRows : 1][D];
  const PagedView& c = a.c;
  const int s = blockIdx.x / a.blocks, heads = a.heads, g0 = blockIdx.y * heads, G = a.G;
  const int m = a.n_new ? min(max(a.n_new[s], 0), a.n) : a.n;
  const int len = paged_len(c, s), base = len - m;  // position of token 0
  const int p0 = ((base >> 4) + (int)blockIdx.x % a.blocks) * 16;
  if (m == 0 || p0 >= len) return;
  const int lo = max(base - p0, 0), count = min(len - p0, 16) - lo;  // the block's positions that are new
  const long long token0 = (long long)s * a.n + (p0 - base) + lo;
  const int lane = (int)threadIdx.x % kLanes, d = lane * E, half = a.dim / 2;
  // rows that lie side by side: positions first, then heads, of which the last are k's
  const int abreast = min(kRows, count > 1 ? 1 << (32 - __clz(count - 1)) : 1);
  const int t0 = (int)threadIdx.x / kLanes % abreast, h0 = (int)threadIdx.x / kLanes / abreast, hs = kRows / abreast;
  const int queries = heads * G, all = queries + heads;

  auto source = [&](int t, int h) {
    const long long token = token0 + t;
    return *(const u32x4*)((h < queries ? (const T*)a.q + token * a.ldq + (size_t)(g0 * G + h) * D
                                        : (const T*)a.k + token * a.ldk + (size_t)(g0 + h - queries) * D) + d);
  };
  u32x4 in[kAhead], v[kV];
  auto fetch = [&](int t) {
#pragma unroll
    for (int b = 0; b < kAhead; ++b)
      if (t < count && h0 + b * hs < all) in[b] = source(t, h0 + b * hs);
  };
  auto fetch_v = [&](int g) {
#pragma unroll
    for (int b = 0; b < kV; ++b) {
      const int t = (int)threadIdx.x / kLanes + b * kRows;
      if (t < count) v[b] = *(const u32x4*)((const T*)a.v + (token0 + t) * a.ldv + (size_t)g * D + d);
    }
  };
  fetch(t0);
  int page = -1;
  if (p0 >= 0) page = c.pages[(size_t)s * c.width + p0 / c.ps];
  const bool ok = page_ok(c, page);
  const size_t head = ((size_t)(ok ? page : 0) * c.Hkv + g0) * c.ps * D;
  const int slot = ok ? p0 % c.ps : 0;
  T *pk = (T*)a.pool_k + head + (size_t)(slot + lo) * D, *pv = (T*)a.pool_v + head + slot;
  float gain[2][E];
  if (a.q_norm) {
#pragma unroll
    for (int e = 0; e < E; ++e) gain[0][e] = a.q_norm[d + e];
  }
  if (a.k_norm) {
#pragma unroll
    for (int e = 0; e < E; ++e) gain[1][e] = a.k_norm[d + e];
  }

  for (int i = threadIdx.x; i < count * half; i += 256) {
    const int t = i / half, j = i - t * half;
    const int pos = a.positions ? a.positions[token0 + t] : p0 + lo + t;
    const double x = (double)pos * a.turns[j];
    float sn, cs;
    sincospif(2.f * (float)(x - rint(x)), &sn, &cs);
    turn[t][j] = float2{cs * a.scale, sn * a.scale};
  }
  __syncthreads();

  const int partner = ((int)threadIdx.x & 63) + (d < half ? half / E : -(half / E));
  float* mine = rows[P == kAny ? threadIdx.x / kLanes : 0];
  const int dim = P == kAcross ? D : a.dim;
  for (int t = t0; t < count; t += abreast) {
    if (t != t0) fetch(t);
    float cs[E], sn[E];  // x' = x cos + partner sin
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (d + e >= dim) continue;
      const int j = P == kSame ? (d + e) / 2 : d + e < half ? d + e : d + e - half;
      const float2 w = turn[t][j];
      cs[e] = w.x;
      sn[e] = (P == kSame ? e % 2 == 0 : d + e < half) ? -w.y : w.y;
    }
    for (int h1 = h0; h1 < all; h1 += kAhead * hs)
#pragma unroll
      for (int b = 0; b < kAhead; ++b) {
        const int h = h1 + b * hs;
        if (h >= all) break;
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = load_f((const T*)&in[b] + e);
        if (h + kAhead * hs < all) in[b] = source(t, h + kAhead * hs);
        if (h < queries ? a.q_norm : a.k_norm) {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) sum = fmaf(x[e], x[e], sum);
          const float inv = rsqrtf(sum_lanes<kLanes>(sum) / D + a.eps);
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] = x[e] * inv * (h < queries ? gain[0][e] : gain[1][e]);
        }
        float other[E];
        if constexpr (P == kSame) {
#pragma unroll
          for (int e = 0; e < E; ++e) other[e] = x[e ^ 1];
        } else if constexpr (P == kAcross) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int i = __float_as_int(x[e]);
            other[e] = __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x128, 0xf, 0xf, false));
          }
        } else if constexpr (P == kLane) {
#pragma unroll
          for (int e = 0; e < E; ++e) other[e] = __shfl(x[e], partner, 64);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) mine[d + e] = x[e];
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // a row's lanes read what its lanes wrote
          __builtin_amdgcn_wave_barrier();
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (d + e < dim) other[e] = mine[d + e < half ? d + e + half : d + e - half];
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // before the next row's
          __builtin_amdgcn_wave_barrier();
        }
        if (d + E <= dim) {
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] = x[e] * cs[e] + other[e] * sn[e];
        } else if constexpr (P == kSame || P == kAny) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (d + e < dim) x[e] = x[e] * cs[e] + other[e] * sn[e];
        }
        u32x4 res;
        if constexpr (E == 8) res = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
        else res = __builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]});
        if (h < queries) *(u32x4*)((T*)a.out + (token0 + t) * a.ldo + (size_t)(g0 * G + h) * D + d) = res;
        else if (ok) *(u32x4*)(pk + ((size_t)(h - queries) * c.ps + t) * D + d) = res;
      }
  }
  if (!ok) return;
  fetch_v(g0);
  for (int i = 0; i < heads; ++i) {
#pragma unroll
    for (int b = 0; b < kV; ++b) {
      const int t = (int)threadIdx.x / kLanes + b * kRows;
      const T* x = (const T*)&v[b];
      if (t < count) {
#pragma unroll
        for (int e = 0; e < E; ++e) vt[i & 1][d + e][lo + t] = x[e];
      }
    }
    if (i + 1 < heads) fetch_v(g0 + i + 1);
    __syncthreads();
    for (int j = threadIdx.x; j < D * (16 / E); j += 256) {
      const int dd = j / (16 / E), t = j % (16 / E) * E;
      T* dst = pv + ((size_t)i * D + dd) * c.ps + t;
      if (t >= lo && t + E <= lo + count) {
        *(u32x4*)dst = *(const u32x4*)&vt[i & 1][dd][t];
      } else {
        for (int e = 0; e < E; ++e)
          if (t + e >= lo && t + e < lo + count) dst[e] = vt[i & 1][dd][t + e];
      }
    }
  }
}

template <typename T, int D>
void rotate_append(const RotateArgs& a, hipStream_t s) {
  const dim3 grid(a.blocks * a.c.S, a.c.Hkv / a.heads);
  switch (partner_of<T>(D, a.dim, a.interleaved)) {
    case kSame: hipLaunchKernelGGL((rotate_append_kernel<T, D, kSame>), grid, dim3(256), 0, s, a); break;
    case kAcross:
      if constexpr (D * sizeof(T) == 256) hipLaunchKernelGGL((rotate_append_kernel<T, D, kAcross>), grid, dim3(256), 0, s, a);
      break;
    case kLane: hipLaunchKernelGGL((rotate_append_kernel<T, D, kLane>), grid, dim3(256), 0, s, a); break;
    case kAny: hipLaunchKernelGGL((rotate_append_kernel<T, D, kAny>), grid, dim3(256), 0, s, a);
  }
}
template <typename T>
void rotate_append(const RotateArgs& a, hipStream_t s) {
  switch (a.c.D) {
    case 32: return rotate_append<T, 32>(a, s);
    case 64: return rotate_append<T, 64>(a, s);
    default: return rotate_append<T, 128>(a, s);
  }
}

}  // namespace

hipError_t paged_append_rotated(const RotateArgs& a0, hipStream_t s) {
  RotateArgs a = a0;
  a.blocks = (a.n + 14) / 16 + 1;  // that n positions can touch
  a.heads = a.c.Hkv;
  while (a.heads > 1 && (a.c.Hkv % a.heads || (size_t)a.blocks * a.c.S * (a.c.Hkv / a.heads) < kFill)) --a.heads;
  if (a.c.esz == 2) rotate_append<bf16_t>(a, s);
  else rotate_append<float>(a, s);
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
