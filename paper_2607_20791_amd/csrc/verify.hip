// Verification of drafted tokens against the target's truncated distribution.
//
// With w_j = exp((z_j - max z) / T) for the kept ids (w_j >= min_p) and W their
// sum, p_j = w_j / W.  Draft x of the distribution q is accepted while
// u q(x) < p(x); the first refusal draws from max(p - q, 0).  Sequences sampled
// this way are distributed as if drawn from p one by one: x is emitted with
// probability min(p, q) + (1 - sum min(p, q)) max(p - q, 0) / sum max(p - q, 0) = p.
//
// One read of all logits bounds it.  Pass 1 streams them and keeps the maxima of every
// 64 ids (a quarter of a span): with a row's maximum its threshold is known, and only
// quarters whose maximum reaches it hold kept ids.  Those alone are read again for the rows'
// sums (pass 2), the spans that hold any for the rest of p over q in the one row per sequence
// that is drawn from (pass 3), and four spans for the draw (pass 4).  Weights
// and sums are fp64: the token drawn hangs on sums of up to 2^20 weights, which fp32
// would leave wrong in one draw of a few.  T == 0: pass 1, then the first
// id of each row's maximum.
//
// Measured, passes 1 to 4: 64 sequences of up to 4 drafts with logits of their own (512 rows of
// 152064 in all, 311 MB) 47 + 27 + 19 + 6 us; 32 greedy probes of up to 15 tokens (230 MB) 38 + 8 + 7 + 5; one
// sequence of 4 drafts (9 rows of 128256, 4.6 MB) 3.3 + 4.5 + 6.1 + 4.0, launches and latency.
#include <algorithm>
#include <cmath>

#include "paged.hpp"
#include "weights.hpp"

namespace rgd {

namespace {

constexpr int kSpan = 256;       // ids per span: one wave, four a lane
constexpr int kQuarter = 64;     // ids per quarter of a span: 16 lanes
constexpr int kWaveSpans = 8;    // pass 1: spans of a wave
constexpr int kChunk = kWaveSpans * kSpan;
constexpr int kMaxSpans = 4096;
constexpr int kMaxPart = 32;     // spans of a wave in pass 2, at most
constexpr int kMaxParts = 16;    // workgroups that share a row in pass 3
constexpr int kResident = 5120;  // waves of pass 2 at a time: 20 per CU

typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));  // rows need no alignment

// 2^x to 1e-14 for x <= 0: the Taylor series of 2^f, |f| <= 1/2, to f^11.
RGD_DEV double exp2_f64(double x) {
  x = fmax(x, -1100.0);  // below: 0 either way (and -inf - rint(-inf) is not a number)
  const double n = rint(x), g = (x - n) * 0.6931471805599453;
  double s = 1.0 / 39916800.0;
  s = fma(s, g, 1.0 / 3628800.0);
  s = fma(s, g, 1.0 / 362880.0);
  s = fma(s, g, 1.0 / 40320.0);
  s = fma(s, g, 1.0 / 5040.0);
  s = fma(s, g, 1.0 / 720.0);
  s = fma(s, g, 1.0 / 120.0);
  s = fma(s, g, 1.0 / 24.0);
  s = fma(s, g, 1.0 / 6.0);
  s = fma(s, g, 0.5);
  s = fma(s, g, 1.0);
  s = fma(s, g, 1.0);
  return ldexp(s, (int)n);
}

RGD_DEV double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

struct DrawInfo;

struct Job {
  VerifyArgs a;
  double per_z, low;  // log2(e) / T; kept: z - max >= low
  int spans, chunks, groups, part, parts2, parts3;
  float* quarter_max; // [rows][spans][4]
  float* chunk_max;   // [rows][chunks]
  float* top;         // [rows]
  double* sums;       // [rows][parts2]
  double2* rest;      // [S][groups]: rest of p over q, and p, of the drawn row's groups
  DrawInfo* draws;             // [S]
  unsigned short* listed;      // [S][spans]: the drawn row's spans that reach its threshold
};

// Rows: the target's S (K + 1), then the drafts' S K.
RGD_DEV long long target_row(const VerifyArgs& a, int s, int i) { return (long long)s * (a.K + 1) + i; }
RGD_DEV long long draft_row(const VerifyArgs& a, int s, int i) {
  return (long long)a.S * (a.K + 1) + (long long)s * a.K + i;
}
RGD_DEV int drafts_of(const VerifyArgs& a, int s) { return a.n_draft ? min(max(a.n_draft[s], 0), a.K) : a.K; }

// The logits of a row, or null where it is not asked for.
RGD_DEV const float* row_logits(const VerifyArgs& a, long long r) {
  const long long nt = (long long)a.S * (a.K + 1);
  if (r < nt) {
    const int s = (int)(r / (a.K + 1)), i = (int)(r - (long long)s * (a.K + 1));
    return i <= drafts_of(a, s) ? a.target + r * a.V : nullptr;
  }
  r -= nt;
  const int s = (int)(r / a.K), i = (int)(r - (long long)s * a.K);
  return i < drafts_of(a, s) ? a.draft + r * a.V : nullptr;
}

// This lane's ids of a span, 4 lane + {0..3}; behind the row -inf.
RGD_DEV f4 load_span(const float* z, int V, int span) {
  const int at = span * kSpan + (threadIdx.x & 63) * 4;
  f4 v;
  if ((span + 1) * kSpan <= V) return *(const f4*)(z + at);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = at + e < V ? z[at + e] : -INFINITY;
  return v;
}

// ------------------------------------------------------------------ pass 1 --
template <int CTRL, int ROWS>
RGD_DEV float max_step(float v) {
  const int b = __float_as_int(v);
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(b, b, CTRL, ROWS, 0xf, false)));
}
// the maximum over 16 lanes, in all of them
RGD_DEV float row_max(float v) {
  v = max_step<0x128, 0xf>(v);  // row_ror 8, 4, 2, 1
  v = max_step<0x124, 0xf>(v);
  v = max_step<0x122, 0xf>(v);
  return max_step<0x121, 0xf>(v);
}
// the maximum over the wave, in its last lane
RGD_DEV float last_lane_max(float v) {
  v = max_step<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
  v = max_step<0x112, 0xf>(v);
  v = max_step<0x114, 0xf>(v);
  v = max_step<0x118, 0xf>(v);
  v = max_step<0x142, 0xa>(v);  // row_bcast 15, 31
  return max_step<0x143, 0xc>(v);
}

// 8 KB a wave in flight at once, then the quarters' maxima by rotations of 16 lanes.  311 MB: 47 us,
// 6.6 TB/s: memory bounds it (reads counted there: 1.00 times the bytes).  The loads are nontemporal: without
// that 54 us, and 5 us less in pass 2, which then finds some of its ids in the last-level cache.  One
// sequence of 4 drafts: 3.3 us, with 16 spans a wave 4.5.  Putting candidate ids aside here
// costs 19 us.
__global__ __launch_bounds__(256) void verify_max_kernel(Job j, int groups) {
  const long long r = blockIdx.x / groups;
  const int first = ((int)(blockIdx.x % groups) * 4 + (threadIdx.x >> 6)) * kWaveSpans, lane = threadIdx.x & 63;
  const float* z = row_logits(j.a, r);
  if (!z || first >= j.spans) return;
  f4 v[kWaveSpans];
  if ((first + kWaveSpans) * kSpan <= j.a.V) {
#pragma unroll
    for (int k = 0; k < kWaveSpans; ++k)
      v[k] = __builtin_nontemporal_load((const f4*)(z + (first + k) * kSpan + lane * 4));
  } else {
#pragma unroll
    for (int k = 0; k < kWaveSpans; ++k)
      v[k] = first + k < j.spans ? load_span(z, j.a.V, first + k) : f4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  }
  float mine = -INFINITY;
#pragma unroll
  for (int k = 0; k < kWaveSpans; ++k) {
    // NaN counts as -inf: fmaxf takes the other operand
    const float m = row_max(fmaxf(fmaxf(fmaxf(v[k][0], v[k][1]), fmaxf(v[k][2], v[k][3])), -INFINITY));
    mine = (lane & 15) == k ? m : mine;
  }
  const int sp = first + (lane & 15);
  if ((lane & 15) < kWaveSpans && sp < j.spans) j.quarter_max[(r * j.spans + sp) * 4 + lane / 16] = mine;
  mine = last_lane_max(mine);
  if (lane == 63) j.chunk_max[r * j.chunks + first * kSpan / kChunk] = mine;
}

// One row's distribution.
struct Dist {
  const float* z;
  float top, thr;
  double per_z, scale;  // p = 2^((z - top) per_z) * scale
  RGD_DEV double weight(float x) const { return x >= thr ? exp2_f64(((double)x - (double)top) * per_z) : 0.0; }
  // Rounded by itself: a product that went into the difference p - q unrounded would leave noise where p = q, and
  // the draw would come from that.
  RGD_DEV double p(float x) const {
#pragma clang fp contract(off)
    return weight(x) * scale;
  }
};

// Row r, of kept sum W.  A row without a finite maximum keeps nothing.
RGD_DEV Dist dist_of(const Job& j, const float* logits, long long r, double W) {
  Dist d;
  d.z = logits;
  d.top = j.top[r];
  d.per_z = j.per_z;
  const bool alive = finite_top(d.top);
  d.thr = alive ? threshold(d.top, j.low) : INFINITY;
  d.scale = alive ? 1.0 / W : 0.0;
  return d;
}

// The span maxima of a row, `per` neighbouring ones a thread of 256.
struct SpanMax {
  float m[kMaxSpans / 256];
  int per;
  RGD_DEV void load(const Job& j, long long r) {
    per = (j.spans + 255) / 256;
    const f4* row = (const f4*)j.quarter_max + r * j.spans;
#pragma unroll
    for (int k = 0; k < kMaxSpans / 256; ++k)
      if (k < per) {
        const f4 q = row[min(per * (int)threadIdx.x + k, j.spans - 1)];
        m[k] = fmaxf(fmaxf(q[0], q[1]), fmaxf(q[2], q[3]));
      }
  }
  // the spans that reach thr, in order, by the whole workgroup: list[0 .. n); red: 4 ints
  RGD_DEV int list(const Job& j, float thr, unsigned short* out, int* red) const {
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    unsigned hits = 0;
#pragma unroll
    for (int k = 0; k < kMaxSpans / 256; ++k)
      if (k < per) hits |= m[k] >= thr && per * t + k < j.spans ? 1u << k : 0u;
    const int mine = __popc(hits);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o, 64);
      if (lane >= o) incl += v;
    }
    if (lane == 63) red[w] = incl;
    __syncthreads();
    int at = incl - mine, n = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      at += k < w ? red[k] : 0;
      n += red[k];
    }
    for (; hits; hits &= hits - 1) out[at++] = (unsigned short)(per * t + __builtin_ctz(hits));
    __syncthreads();
    return n;
  }
};

// Listed spans are taken four at a time (a group), one group a wave.
constexpr int kGroup = 4;

RGD_DEV void load_group(const float* z, int V, const unsigned short* list, int n, int group, f4 (&v)[kGroup]) {
#pragma unroll
  for (int k = 0; k < kGroup; ++k) v[k] = load_span(z, V, list[min(group * kGroup + k, n - 1)]);
}

// Bit 4 k + e: v[k][e] is kept (and the group has a span k).
RGD_DEV unsigned kept_bits(const f4 (&v)[kGroup], float thr, int spans_left) {
  unsigned m = 0;
#pragma unroll
  for (int k = 0; k < kGroup; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) m |= v[k][e] >= thr && k < spans_left ? 1u << (4 * k + e) : 0u;
  return m;
}

// Whether some lane has so many kept logits of its 16 that all of them are weighed one after the other, in
// place of one kept logit per lane and turn, of which few lanes have more than one or two.  72 rows of
// 152064 ids that are all kept: pass 2 takes 20 us in place of 39, pass 3 20 in place of 27 (of pass 2 the weights
// alone take 16 and the loads alone 14); a bound of 4 is as fast as 6, 9 slower between few and all.
RGD_DEV bool dense(unsigned bits) { return __builtin_expect(__any(__popc(bits) > 6), 0); }

// v[i / 4][i % 4] by selects
RGD_DEV float pick(const f4 (&v)[kGroup], int i) {
  float a[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float lo = i & 1 ? v[k][1] : v[k][0], hi = i & 1 ? v[k][3] : v[k][2];
    a[k] = i & 2 ? hi : lo;
  }
  const float lo = i & 4 ? a[1] : a[0], hi = i & 4 ? a[3] : a[2];
  return i & 8 ? hi : lo;
}

// ------------------------------------------------------------------ pass 2 --
// A row's maximum, from those of its chunks, and the kept sum of j.part of its spans, by
// one wave, which puts their quarters with kept ids in a list and reads sixteen at a time.  Rows
// differ in kept ids by a factor of a hundred; small parts share that out: 512 rows of
// 152064 ids, 200 kept ones in the middle row and 4600 in the hundredth-largest: 27.5 us, 36 by whole
// spans, of which 39% hold kept ids (132 MB).  With those, 35 us for workgroups in place of waves
// where waves took 31, 39 for 64 spans a wave and 32 for 16.
__global__ __launch_bounds__(256, 5) void verify_sum_kernel(Job j, long long waves) {
  __shared__ unsigned char lists[4][4 * kMaxPart];
  const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (wave >= waves) return;
  const long long r = wave / j.parts2;
  const int part = (int)(wave - r * j.parts2), lane = threadIdx.x & 63, V = j.a.V, first = part * j.part;
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < 8; ++k)  // at most 512 chunks
    if (64 * k < j.chunks) top = fmaxf(top, j.chunk_max[r * j.chunks + min(64 * k + lane, j.chunks - 1)]);
  typedef float f2 __attribute__((ext_vector_type(2)));
  const int pair = first * 2 + lane, pairs = j.spans * 2;  // this lane's two quarters
  const f2 m = ((const f2*)j.quarter_max)[r * pairs + min(pair, pairs - 1)];
  const float* z = row_logits(j.a, r);
  if (!z) return;
  top = wave_max(top);
  if (part == 0 && lane == 0) j.top[r] = top;
  if (!finite_top(top)) return;
  const float thr = threshold(top, j.low);
  const bool mine = lane < 2 * j.part && pair < pairs, h0 = mine && m[0] >= thr, h1 = mine && m[1] >= thr;
  const unsigned long long b0 = __ballot(h0), b1 = __ballot(h1), below = (1ull << lane) - 1;
  const int n = __popcll(b0) + __popcll(b1), at = __popcll(b0 & below) + __popcll(b1 & below);
  unsigned char* list = lists[threadIdx.x >> 6];
  if (h0) list[at] = 2 * lane;
  if (h1) list[at + h0] = 2 * lane + 1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the wave's lanes read what its lanes wrote
  __builtin_amdgcn_wave_barrier();
  // sixteen quarters at a time, each by 16 lanes, the next ones on their way
  const bool whole = (first + j.part) * kSpan <= V;
  auto take = [&](int i0, f4 (&v)[kGroup]) {
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const int i = i0 + 4 * k + lane / 16, id = first * kSpan + list[min(i, n - 1)] * kQuarter + (lane & 15) * 4;
      if (i >= n) {
        v[k] = f4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      } else if (whole) {
        v[k] = *(const f4*)(z + id);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k][e] = id + e < V ? z[id + e] : -INFINITY;
      }
    }
  };
  double sum = 0.0;
  f4 v[kGroup], next[kGroup];
  if (n > 0) take(0, v);
  for (int i0 = 0; i0 < n; i0 += 4 * kGroup) {
    if (i0 + 4 * kGroup < n) take(i0 + 4 * kGroup, next);
    const unsigned bits = kept_bits(v, thr, kGroup);
    if (dense(bits)) {
#pragma unroll
      for (int k = 0; k < kGroup; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double w = exp2_f64(((double)v[k][e] - (double)top) * j.per_z);
          sum += bits >> (4 * k + e) & 1 ? w : 0.0;
        }
    } else {
      for (unsigned b = bits; b; b &= b - 1)
        sum += exp2_f64(((double)pick(v, __builtin_ctz(b)) - (double)top) * j.per_z);
    }
#pragma unroll
    for (int k = 0; k < kGroup; ++k) v[k] = next[k];
  }
  sum = wave_sum_f64(sum);
  if (lane == 0) j.sums[wave] = sum;
}

// ------------------------------------------------------------------ pass 3 --
// What one sequence draws from.
struct DrawInfo {
  float top[2], thr[2];  // of p and q
  double scale[2];
  int accepted;
  int without;  // the id that is left out (a certain draft), or -1
  int minus_q;
  int n;        // listed spans; 0: no distribution
};

struct Draw {
  Dist p, q;
  int without;
  bool minus_q;
  RGD_DEV Draw(const Job& j, int s, const DrawInfo& i) {
    const VerifyArgs& a = j.a;
    p = Dist{a.target + target_row(a, s, i.accepted) * a.V, i.top[0], i.thr[0], j.per_z, i.scale[0]};
    minus_q = i.minus_q;
    q = p;
    if (minus_q) q = Dist{a.draft + ((long long)s * a.K + i.accepted) * a.V, i.top[1], i.thr[1], j.per_z, i.scale[1]};
    without = i.without;
  }
  // (the rest of p over q, p) of one id
  RGD_DEV double2 rest(float zp, float zq, int id) const {
#pragma clang fp contract(off)
    const double x = p.p(zp);
    double r = x;
    if (minus_q) r = fmax(x - q.p(zq), 0.0);
    if (id == without) r = 0.0;
    return double2{r, x};
  }
};

// Accepted drafts of a sequence, one draft a thread (K <= 255), then the rest of the
// drawn row in this part's spans.  64 sequences in 12 parts: 19 us: 7 for two
// dependent chains (tokens and sums, accepted row, its maxima, its spans), 7 for 34 MB of reads, 4 for the
// weights; 3 us more where parts make more than three workgroups per CU.  By quarters it takes 19: fewer
// bytes, but fewer groups to share, each with more kept ids.
__global__ __launch_bounds__(256, 3) void verify_rest_kernel(Job j) {
  __shared__ int first[4], red[4];
  __shared__ unsigned short list[kMaxSpans];
  __shared__ DrawInfo info;
  __shared__ double sums[2 * 255 + 1];  // of the target's rows, then the drafts'
  const VerifyArgs& a = j.a;
  const int s = blockIdx.x / j.parts3, part = blockIdx.x % j.parts3, t = threadIdx.x, w = t >> 6;
  const int id = t < a.K ? a.tokens[(long long)s * a.K + t] : -1;
  const int nd = drafts_of(a, s);
  // 16 lanes a row; all K of them, so that the loads need not wait for the count
  for (int q = t / 16; q < (a.draft ? 2 * a.K + 1 : a.K + 1); q += 16) {
    const double* part = j.sums + (q <= a.K ? target_row(a, s, q) : draft_row(a, s, q - a.K - 1)) * j.parts2;
    double x = 0.0;
    for (int k0 = t % 16; k0 < j.parts2; k0 += 8 * 16) {  // eight loads at a time, whatever the number of parts
      double y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = part[min(k0 + 16 * i, j.parts2 - 1)];
#pragma unroll
      for (int i = 0; i < 8; ++i) x += k0 + 16 * i < j.parts2 ? y[i] : 0.0;
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor(x, o, 16);
    if (t % 16 == 0) sums[q] = x;
  }
  __syncthreads();
  bool ok = true;
  DrawInfo mine{};
  if (t <= nd) {  // row nd: no draft to refuse
    const bool inside = (unsigned)id < (unsigned)a.V, drafted = t < nd;
    const long long r = target_row(a, s, t);
    const float* zp = a.target + r * a.V;
    const float xp = zp[inside ? id : 0];
    const Dist p = dist_of(j, zp, r, sums[t]);
    Dist q = p;
    double qx = 1.0;
    if (a.draft && drafted) {
      const float* zq = a.draft + ((long long)s * a.K + t) * a.V;
      const float xq = zq[inside ? id : 0];
      q = dist_of(j, zq, draft_row(a, s, t), sums[a.K + 1 + t]);
      qx = q.p(xq);
    }
    if (drafted) ok = inside && (double)a.u[(long long)s * (a.K + 1) + t] * qx < p.p(xp);
    mine = DrawInfo{{p.top, q.top}, {p.thr, q.thr}, {p.scale, q.scale}, t, drafted && !a.draft ? id : -1,
                    drafted && a.draft, 0};
  }
  const unsigned long long no = __ballot(!ok);
  if ((t & 63) == 0) first[w] = no ? 64 * w + __builtin_ctzll(no) : 0x7FFFFFFF;
  __syncthreads();
  const int acc = min(min(min(first[0], first[1]), min(first[2], first[3])), nd);
  SpanMax spans;
  spans.load(j, target_row(a, s, acc));
  if (t == acc) info = mine;
  __syncthreads();
  DrawInfo di = info;
  di.n = finite_top(di.top[0]) ? spans.list(j, di.thr[0], list, red) : 0;
  if (part == 0) {  // for pass 4
    for (int i = t; i < di.n; i += 256) j.listed[(long long)s * j.spans + i] = list[i];
    if (t == 0) j.draws[s] = di;
  }
  const Draw d(j, s, di);
  const int step = 4 * j.parts3, g0 = part * 4 + w, n = di.n;
  f4 v[kGroup], q[kGroup] = {}, vn[kGroup], qn[kGroup] = {};
  auto load = [&](int g, f4 (&x)[kGroup], f4 (&y)[kGroup]) {
    load_group(d.p.z, a.V, list, n, g, x);
    if (d.minus_q) load_group(d.q.z, a.V, list, n, g, y);
  };
  if (g0 * kGroup < n) load(g0, v, q);
  for (int g = g0; g * kGroup < n; g += step) {
    if ((g + step) * kGroup < n) load(g + step, vn, qn);
    double2 sum{0.0, 0.0};
    const unsigned bits = kept_bits(v, d.p.thr, n - g * kGroup);
    if (dense(bits)) {
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        const int id = list[min(g * kGroup + k, n - 1)] * kSpan + (t & 63) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double2 x = d.rest(v[k][e], q[k][e], id + e);
          sum.x += bits >> (4 * k + e) & 1 ? x.x : 0.0;
          sum.y += bits >> (4 * k + e) & 1 ? x.y : 0.0;
        }
      }
    } else {
      for (unsigned m = bits; m; m &= m - 1) {
        const int i = __builtin_ctz(m);
        const double2 x = d.rest(pick(v, i), pick(q, i), list[g * kGroup + i / 4] * kSpan + (t & 63) * 4 + i % 4);
        sum.x += x.x;
        sum.y += x.y;
      }
    }
    sum.x = wave_sum_f64(sum.x);
    sum.y = wave_sum_f64(sum.y);
    if ((t & 63) == 0) j.rest[(long long)s * j.groups + g] = sum;
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      v[k] = vn[k];
      q[k] = qn[k];
    }
  }
}

// ------------------------------------------------------------------ pass 4 --
// Exclusive scans of N values each; red: 4 N doubles.
template <int N>
RGD_DEV void block_scan_f64(const double (&v)[N], double* red, double (&before)[N], double (&total)[N]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  double incl[N];
#pragma unroll
  for (int i = 0; i < N; ++i) incl[i] = v[i];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double x = __shfl_up(incl[i], o, 64);
      if (lane >= o) incl[i] += x;
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (lane == 63) red[4 * i + w] = incl[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    before[i] = incl[i] - v[i];
    total[i] = 0.0;
    double ahead = 0.0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      ahead += k < w ? red[4 * i + k] : 0.0;
      total[i] += red[4 * i + k];
    }
    before[i] = ahead + before[i];
  }
}

RGD_DEV int block_min_i(int v, int* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return min(min(red[0], red[1]), min(red[2], red[3]));
}
// The first thread's `hit` that is one (>= 0), or where there is none the last thread's `last`; both rise with
// the thread.  red: 8 ints.
RGD_DEV int first_or_last(int hit, int last, int* red) {
  const unsigned long long h = __ballot(hit >= 0), l = __ballot(last >= 0);
  const int hv = h ? __builtin_amdgcn_readlane(hit, __builtin_ctzll(h)) : -1;
  const int lv = l ? __builtin_amdgcn_readlane(last, 63 - __builtin_clzll(l)) : -1;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    red[threadIdx.x >> 6] = hv;
    red[4 + (threadIdx.x >> 6)] = lv;
  }
  __syncthreads();
  int first = -1, end = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    first = first < 0 ? red[w] : first;
    end = max(end, red[4 + w]);
  }
  return first >= 0 ? first : end;
}

// The draw: the group, then the id, whose running sum first exceeds u times the total;
// where rounding leaves none, the last one with weight.  4.0 to 6.0 us: one chain of two reads
// (the pass before's result with the groups' sums, a group's logits), two scans and two searches by ballots
// (4.4 to 6.8 with the groups' sums asked for after the result, and by minima over the workgroup).
__global__ __launch_bounds__(256) void verify_draw_kernel(Job j) {
  __shared__ double red[8];
  __shared__ int redi[8];
  __shared__ double sh_before;
  const VerifyArgs& a = j.a;
  const int s = blockIdx.x, t = threadIdx.x;
  double2 part[4];  // asked for before the number of groups is known
#pragma unroll
  for (int k = 0; k < 4; ++k) part[k] = j.rest[(long long)s * j.groups + min(4 * t + k, j.groups - 1)];
  const DrawInfo di = j.draws[s];
  const int acc = di.accepted, n = di.n;
  const float u = a.u[(long long)s * (a.K + 1) + a.K];
  int* out = a.out + (long long)s * (a.K + 1);
  if (t == 0) a.n_accepted[s] = acc;
  if (t <= a.K && t != acc) out[t] = t < acc ? a.tokens[(long long)s * a.K + t] : -1;
  if (n == 0) {
    if (t == 0) out[acc] = -1;
    return;
  }
  const Draw d(j, s, di);
  const int groups = (n + kGroup - 1) / kGroup;  // at most 1024
  double mine[2] = {0.0, 0.0}, total[2], before[2];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (4 * t + k >= groups) part[k] = double2{0.0, 0.0};
    mine[0] += part[k].x;
    mine[1] += part[k].y;
  }
  block_scan_f64<2>(mine, red, before, total);
  const int use = total[0] > 0.0 ? 0 : 1;  // nothing left by rounding: p itself
  const double goal = (double)u * total[use];
  double run = before[use], at[4];
  int hit = -1, last = -1;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const double x = use ? part[k].y : part[k].x;
    at[k] = run;
    if (x > 0.0) {
      run += x;
      last = 4 * t + k;
      if (hit < 0 && run > goal) hit = 4 * t + k;
    }
  }
  hit = first_or_last(hit, last, redi);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (hit == 4 * t + k) sh_before = at[k];
  __syncthreads();
  // one span a wave, four ids a thread
  const int sp = hit * kGroup + (t >> 6);
  const bool have = sp < n;
  const int id0 = j.listed[(long long)s * j.spans + (have ? sp : 0)] * kSpan + 4 * (t & 63);
  run = sh_before;
  double x[4], sum[1] = {0.0}, ahead[1], unused[1];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = 0.0;
    if (have && id0 + e < a.V) {
      const float zp = d.p.z[id0 + e];
      const double2 v = d.rest(zp, d.minus_q ? d.q.z[id0 + e] : zp, id0 + e);
      x[e] = use ? v.y : v.x;
    }
    sum[0] += x[e];
  }
  block_scan_f64<1>(sum, red, ahead, unused);
  run += ahead[0];
  int found = -1, end = -1;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (x[e] > 0.0) {
      run += x[e];
      end = id0 + e;
      if (found < 0 && run > goal) found = id0 + e;
    }
  const int id = first_or_last(found, end, redi);
  if (t == 0) out[acc] = id;
}

// ------------------------------------------------------------------ T == 0 --
// The first maximum of every row that is asked for, one row a wave; the drafts are
// kept while they are it.  One workgroup a sequence: it reads 4 bytes of 1 KB that pass 1 did.
__global__ __launch_bounds__(256) void verify_greedy_kernel(Job j) {
  __shared__ int best[256];
  __shared__ int redi[4];
  const VerifyArgs& a = j.a;
  const int s = blockIdx.x, t = threadIdx.x, lane = t & 63;
  const int nd = drafts_of(a, s);
  for (int i = t >> 6; i <= nd; i += 4) {
    const long long r = target_row(a, s, i);
    const f4* m = (const f4*)j.quarter_max + r * j.spans;
    auto span_max = [&](int k) { return fmaxf(fmaxf(m[k][0], m[k][1]), fmaxf(m[k][2], m[k][3])); };
    float top = -INFINITY;
    for (int k = lane; k < j.spans; k += 64) top = fmaxf(top, span_max(k));
    top = wave_max(top);
    int sp = 0x7FFFFFFF, id = 0x7FFFFFFF;
    for (int k = lane; k < j.spans; k += 64)
      if (span_max(k) == top) sp = min(sp, k);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sp = min(sp, __shfl_xor(sp, o, 64));
    if (finite_top(top)) {
      const f4 v = load_span(a.target + r * a.V, a.V, sp);
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if (v[e] == top) id = sp * kSpan + lane * 4 + e;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) id = min(id, __shfl_xor(id, o, 64));
    } else {
      id = -1;
    }
    if (lane == 0) best[i] = id;
  }
  __syncthreads();
  const int* x = a.tokens + (long long)s * a.K;
  const bool no = t < nd && (best[t] < 0 || best[t] != x[t]);
  const int acc = min(block_min_i(no ? t : 0x7FFFFFFF, redi), nd);
  int* out = a.out + (long long)s * (a.K + 1);
  if (t <= a.K) out[t] = t <= acc ? best[t] : -1;
  if (t == 0) a.n_accepted[s] = acc;
}

struct Sizes {
  long long rows;
  int spans, chunks, groups, part, parts2, parts3;
  size_t quarter_max, chunk_max, top, sums, rest, draws, listed, bytes;
};

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// parts3: few sequences are shared by several workgroups (768 in all: three per CU)
Sizes sizes_of(int S, int K, int V) {
  Sizes z;
  z.rows = (long long)S * (2 * K + 1);
  z.spans = (V + kSpan - 1) / kSpan;
  z.groups = (z.spans + kGroup - 1) / kGroup;
  z.chunks = (V + kChunk - 1) / kChunk;
  // smaller parts as long as all waves are resident at once: 72 rows with some thousand kept ids, 20.2 -> 14.8 us
  z.part = kMaxPart;
  while (z.part > 8 && z.rows * ((z.spans + z.part / 2 - 1) / (z.part / 2)) <= kResident) z.part /= 2;
  z.parts2 = (z.spans + z.part - 1) / z.part;
  z.parts3 = std::min(kMaxParts, (767 + S) / S);
  z.quarter_max = 0;
  z.chunk_max = up256((size_t)z.rows * z.spans * 16);
  z.top = z.chunk_max + up256((size_t)z.rows * z.chunks * 4);
  z.sums = z.top + up256((size_t)z.rows * 4);
  z.rest = z.sums + up256((size_t)z.rows * z.parts2 * 8);
  z.draws = z.rest + up256((size_t)S * z.groups * 16);
  z.listed = z.draws + up256((size_t)S * sizeof(DrawInfo));
  z.bytes = z.listed + up256((size_t)S * z.spans * 2);
  return z;
}

}  // namespace

size_t verify_workspace_bytes(int S, int K, int V) { return sizes_of(S, K, V).bytes; }

hipError_t verify_drafts(const VerifyArgs& a0, hipStream_t s) {
  const Sizes z = sizes_of(a0.S, a0.K, a0.V);
  Job j{};
  j.a = a0;
  if (a0.T == 0.f) j.a.draft = nullptr;
  const double T = a0.T;
  j.per_z = T > 0.0 ? 1.4426950408889634 / T : 0.0;
  j.low = a0.min_p > 0.f ? T * std::log((double)a0.min_p) : -(double)INFINITY;
  j.spans = z.spans;
  j.chunks = z.chunks;
  j.groups = z.groups;
  j.part = z.part;
  j.parts2 = z.parts2;
  j.parts3 = z.parts3;
  j.quarter_max = (float*)(a0.ws + z.quarter_max);
  j.chunk_max = (float*)(a0.ws + z.chunk_max);
  j.top = (float*)(a0.ws + z.top);
  j.sums = (double*)(a0.ws + z.sums);
  j.rest = (double2*)(a0.ws + z.rest);
  j.draws = (DrawInfo*)(a0.ws + z.draws);
  j.listed = (unsigned short*)(a0.ws + z.listed);
  const long long rows = (long long)a0.S * (j.a.draft ? 2 * a0.K + 1 : a0.K + 1);
  const int groups = (z.spans + 4 * kWaveSpans - 1) / (4 * kWaveSpans);
  const long long waves = rows * z.parts2;  // at most 2^23: rows x 8192 ids are bounded
  hipLaunchKernelGGL(verify_max_kernel, dim3((unsigned)(rows * groups)), dim3(256), 0, s, j, groups);
  if (T == 0.0) {
    hipLaunchKernelGGL(verify_greedy_kernel, dim3(a0.S), dim3(256), 0, s, j);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(verify_sum_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, j, waves);
  hipLaunchKernelGGL(verify_rest_kernel, dim3((unsigned)(a0.S * z.parts3)), dim3(256), 0, s, j);
  hipLaunchKernelGGL(verify_draw_kernel, dim3(a0.S), dim3(256), 0, s, j);
  return hipGetLastError();
}

}  // namespace rgd
