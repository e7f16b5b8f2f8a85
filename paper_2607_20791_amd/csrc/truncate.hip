// One draw per row under temperature, top-k, top-p and min-p.
//
// With the ids in the order of their logits (equal ones by id) each limit keeps a leading part, and the kept ids are the
// shortest of these.  Weights are whole multiples of 2^-43 of the largest one's, so that sums are exact in 64-bit integers
// and no order of adding them matters.
//
// One read of the logits bounds it, and, where nearly all ids count, their weights: fp64, as the id drawn hangs on sums of up
// to 2^20 of them.  Four passes: the maxima; the weights and counts of all ids in bins of 1/32 octave below the
// maximum, which tell the bins that the limits' borders lie in; the weights of the ids above these bins, summed by chunks of 2048
// ids, while those inside go to a list; and, one workgroup a row, the borders among the listed ones, the chunk that the
// draw falls in and its id.
#include <algorithm>
#include <cmath>

#include "paged.hpp"
#include "weights.hpp"

namespace rgd {

namespace {

typedef unsigned long long u64;
typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));  // rows need no alignment

constexpr double kOne = 8796093022208.0;  // 2^43: the largest weight; 2^20 of them stay below 2^63
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kSpan = 256;         // ids: one wave, four a lane
constexpr int kSpans = 8;          // spans of a chunk
constexpr int kChunk = kSpan * kSpans;
constexpr int kMaxChunks = 512;
constexpr int kPerOctave = 256;    // entries of the table of powers; bins are eight of them
constexpr int kOctaves = 45;       // below: a weight under 2^-44 is none
constexpr int kBins = kOctaves * 32;
constexpr int kItems = 16;         // listed ids of a thread of the last pass
constexpr int kList = kItems * kThreads;
constexpr int kSlab = 1024;        // rows at a time, for the workspace's sake

// The limits' part of a row, as the third pass finds it.
struct RowInfo {
  float top;
  uint32_t least;    // key of the lowest logit that min_p keeps
  int mode;          // below
  int p0, p1, kb;    // bins that top_p's border lies in, the bin of top_k's; -1: no such limit
  unsigned before_k; // ids ahead of bin kb
  u64 mass_k;        // weight ahead of bin kb
  u64 mass_p;        // weight ahead of bin p0
  u64 total;
};
enum { kNone, kGreedy, kDraw };

struct Job {
  TruncateArgs a;
  int spans, chunks, parts;
  bool merge;              // several parts add to a row's bins
  float* chunk_max;        // [R][chunks]
  u64* mass;               // [R][kBins]
  unsigned* count;         // [R][kBins]
  u64* chunk_sum;          // [R][chunks]
  RowInfo* info;           // [R]
  unsigned* listed;        // [R]
  uint2* list;             // [R][cap] (logit, id)
  int cap;
};

// ---------------------------------------------------------------- weights --
// An id's logit against its row: i, its distance below the maximum in 1/256 octaves, rounded (so that it never
// falls where logits rise), and its weight 2^(i/256) 2^(f/256) with the rest f, by the series of the second to its cube
// (1.4e-13 of the weight) and a table of the first.
struct Weigher {
  double top, scale;
  const double* table;  // 2^(j/256), LDS
  // -i; kOctaves * 256 and more: no weight (NaN and -inf among them)
  RGD_DEV int place(float z, double& f) const {
    const double y = fmax(((double)z - top) * scale, -(double)((kOctaves + 1) * kPerOctave));  // the other operand for NaN
    constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: the sum's last bit is 1
    const double t = y + kRound;
    f = y - (t - kRound);
    return -(int)(unsigned)__double2loint(t);
  }
  RGD_DEV u64 weight(int i, double f) const {
    constexpr double kLn = 0.6931471805599453 / kPerOctave;
    double s = fma(f, kLn * kLn * kLn / 6.0, kLn * kLn / 2.0);
    s = fma(s, f, kLn);
    s = fma(s, f, 1.0);
    s *= table[-i & (kPerOctave - 1)];
    s = ldexp(s, (-i >> 8) + 43) + 4503599627370496.0;  // 2^52: rounds to a whole number in the low bits
    return (u64)__double_as_longlong(s) & 0xFFFFFFFFFFFFFull;
  }
  RGD_DEV u64 of(float z) const {
    double f;
    const int i = place(z, f);
    return i < kOctaves * kPerOctave ? weight(i, f) : 0;
  }
};

RGD_DEV int bin_of(int i) { return i >> 3; }

RGD_DEV void fill_table(double* table) {
  if (threadIdx.x < kPerOctave) table[threadIdx.x] = 2.0 * exp2_f64((double)threadIdx.x / kPerOctave - 1.0);
}

RGD_DEV bool greedy(float T) { return !(T > 0.f); }
RGD_DEV float temperature(const TruncateArgs& a, int r) { return a.T ? a.T[r] : 1.f; }

RGD_DEV uint32_t key_of(float z) {
  z += 0.f;  // -0 is 0
  return ordered_u32(z != z ? -INFINITY : z);
}

// A place in the order of a row's ids: ascending here is descending by logit, then ascending by id.
RGD_DEV u64 order_of(uint32_t key, int id) { return (u64)(~key) << 20 | (unsigned)id; }

// The chunk's ids of this lane, 4 lane + {0..3} of each span; behind the row -inf.
RGD_DEV void load_chunk(const float* z, int V, int chunk, f4 (&v)[kSpans]) {
  const int lane = threadIdx.x & 63;
  if ((chunk + 1) * kChunk <= V) {
#pragma unroll
    for (int k = 0; k < kSpans; ++k) v[k] = *(const f4*)(z + chunk * kChunk + k * kSpan + lane * 4);
  } else {
#pragma unroll
    for (int k = 0; k < kSpans; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int id = chunk * kChunk + k * kSpan + lane * 4 + e;
        v[k][e] = id < V ? z[id] : -INFINITY;
      }
  }
}

// A row's maximum from its chunks', by every wave.
RGD_DEV float row_top(const Job& j, int r) {
  const int lane = threadIdx.x & 63;
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < kMaxChunks / 64; ++k)
    if (64 * k < j.chunks) top = fmaxf(top, j.chunk_max[(size_t)r * j.chunks + min(64 * k + lane, j.chunks - 1)]);
  return wave_max(top);
}

// ----------------------------------------------------------------- pass 1 --
// One wave a chunk, 8 KB in flight; rows that several workgroups weigh get their bins cleared.
__global__ __launch_bounds__(256) void truncate_max_kernel(Job j, int groups) {
  const int r = blockIdx.x / groups, g = blockIdx.x % groups, chunk = g * 4 + (threadIdx.x >> 6);
  if (j.merge)
    for (int i = g * 256 + threadIdx.x; i < kBins; i += groups * 256) {
      j.mass[(size_t)r * kBins + i] = 0;
      j.count[(size_t)r * kBins + i] = 0;
    }
  if (g == 0 && threadIdx.x == 0) j.listed[r] = 0;
  if (chunk >= j.chunks) return;
  const float* z = j.a.z + (size_t)r * j.a.ldz;
  f4 v[kSpans];
  load_chunk(z, j.a.V, chunk, v);
  float m = -INFINITY;  // NaN counts as -inf: fmaxf takes the other operand
#pragma unroll
  for (int k = 0; k < kSpans; ++k) m = fmaxf(m, fmaxf(fmaxf(v[k][0], v[k][1]), fmaxf(v[k][2], v[k][3])));
  m = wave_max(fmaxf(m, -INFINITY));
  if ((threadIdx.x & 63) == 0) j.chunk_max[(size_t)r * j.chunks + chunk] = m;
}

// ----------------------------------------------------------------- pass 2 --
RGD_DEV float min_p_least(const TruncateArgs& a, int r, float top) {
  const float p = a.min_p ? a.min_p[r] : 0.f;
  if (!(p > 0.f)) return -INFINITY;
  return threshold(top, p < 1.f ? (double)temperature(a, r) * log((double)p) : 0.0);
}
RGD_DEV bool has_top_p(const TruncateArgs& a, int r) { return a.top_p && a.top_p[r] < 1.f; }
RGD_DEV bool has_top_k(const TruncateArgs& a, int r) { return a.top_k && a.top_k[r] > 0 && a.top_k[r] < a.V; }

// Weight and number of the ids in each bin.  A row without top_k and top_p needs none.
__global__ __launch_bounds__(kThreads) void truncate_bins_kernel(Job j) {
  __shared__ u64 mass[kBins];
  __shared__ unsigned count[kBins];
  __shared__ double table[kPerOctave];
  const int r = blockIdx.x / j.parts, part = blockIdx.x % j.parts, wave = threadIdx.x >> 6;
  const TruncateArgs& a = j.a;
  const float top = row_top(j, r), T = temperature(a, r);
  const bool by_p = has_top_p(a, r), by_k = has_top_k(a, r);
  if (!finite_top(top) || greedy(T) || !(by_p || by_k)) return;
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    mass[i] = 0;
    count[i] = 0;
  }
  fill_table(table);
  __syncthreads();
  const float* z = a.z + (size_t)r * a.ldz;
  const Weigher w{top, kPerOctave * 1.4426950408889634 / (double)T, table};
  // without top_p, ids below min_p's border change nothing
  const float least = by_p ? -INFINITY : min_p_least(a, r, top);
  for (int c = part * kWaves + wave; c < j.chunks; c += j.parts * kWaves) {
    f4 v[kSpans];
    load_chunk(z, a.V, c, v);
#pragma unroll
    for (int k = 0; k < kSpans; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double f;
        const int i = w.place(v[k][e], f);
        if (i < kOctaves * kPerOctave && v[k][e] >= least) {
          atomicAdd(&mass[bin_of(i)], w.weight(i, f));
          if (by_k) atomicAdd(&count[bin_of(i)], 1u);
        }
      }
  }
  __syncthreads();
  u64* gm = j.mass + (size_t)r * kBins;
  unsigned* gc = j.count + (size_t)r * kBins;
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    if (!j.merge) {
      gm[i] = mass[i];
      gc[i] = count[i];
    } else {
      if (mass[i]) atomicAdd(&gm[i], mass[i]);
      if (count[i]) atomicAdd(&gc[i], count[i]);
    }
  }
}

// ------------------------------------------------------------ block scans --
struct Scan {
  u64 mass[kWaves];
  unsigned count[kWaves];
};
// Sums over the threads before this one; totals in all of them.
RGD_DEV void block_scan(u64 m, unsigned c, Scan& sh, u64& m_before, unsigned& c_before, u64& m_all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  u64 mi = m;
  unsigned ci = c;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 mt = __shfl_up(mi, o, 64);
    const unsigned ct = __shfl_up(ci, o, 64);
    if (lane >= o) {
      mi += mt;
      ci += ct;
    }
  }
  __syncthreads();
  if (lane == 63) {
    sh.mass[w] = mi;
    sh.count[w] = ci;
  }
  __syncthreads();
  m_before = mi - m;
  c_before = ci - c;
  m_all = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < w) {
      m_before += sh.mass[i];
      c_before += sh.count[i];
    }
    m_all += sh.mass[i];
  }
}

// ----------------------------------------------------------------- pass 3 --
// The bins of the borders, by a whole workgroup.
RGD_DEV RowInfo find_bins(const Job& j, int r, float top, RowInfo& sh, Scan& scan) {
  const TruncateArgs& a = j.a;
  if (threadIdx.x == 0) {
    sh.top = top;
    sh.least = 0;
    sh.mode = !finite_top(top) ? kNone : greedy(temperature(a, r)) ? kGreedy : kDraw;
    sh.p0 = sh.p1 = sh.kb = -1;
    sh.total = sh.mass_k = sh.mass_p = 0;
    sh.before_k = 0;
    if (sh.mode == kDraw) sh.least = key_of(min_p_least(a, r, top));
  }
  __syncthreads();
  const bool by_p = has_top_p(a, r), by_k = has_top_k(a, r);
  if (sh.mode != kDraw || !(by_p || by_k)) return sh;
  constexpr int PER = (kBins + kThreads - 1) / kThreads;
  u64 m[PER], mb, total, mine = 0;
  unsigned c[PER], cb, cmine = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = threadIdx.x * PER + i;
    m[i] = b < kBins ? j.mass[(size_t)r * kBins + b] : 0;
    c[i] = b < kBins && by_k ? j.count[(size_t)r * kBins + b] : 0;
    mine += m[i];
    cmine += c[i];
  }
  block_scan(mine, cmine, scan, mb, cb, total);
  // the bin in which the ids reach top_k (none: fewer weigh anything), and what lies ahead of it
  if (by_k) {
    const unsigned k = a.top_k[r];
    u64 x = mb;
    unsigned n = cb;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (n < k && n + c[i] >= k) {
        sh.kb = threadIdx.x * PER + i;
        sh.before_k = n;
        sh.mass_k = x;
        sh.total = x + m[i];  // the most that the first top_k ids weigh
      }
      n += c[i];
      x += m[i];
    }
    __syncthreads();
  }
  const u64 most = sh.kb >= 0 ? sh.total : total, fewest = sh.kb >= 0 ? sh.mass_k : total;
  if (by_p) {
    const double p = fmax((double)a.top_p[r], 0.0);
    u64 x = mb;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int b = threadIdx.x * PER + i;
      const double d0 = (double)x, d1 = (double)(x + m[i]);
      if (m[i]) {
        // the first bin whose end reaches the border, for the least and for the most that it may be
        if (d1 >= p * (double)fewest && (x == 0 || d0 < p * (double)fewest)) {
          sh.p0 = b;
          sh.mass_p = x;
        }
        if (d1 >= p * (double)most && (x == 0 || d0 < p * (double)most)) sh.p1 = b;
      }
      x += m[i];
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) sh.total = total;
  __syncthreads();
  return sh;
}

// Sums of the chunks' weights above the borders' bins; the ids in these bins are listed.
__global__ __launch_bounds__(kThreads) void truncate_sum_kernel(Job j) {
  __shared__ RowInfo sh;
  __shared__ Scan scan;
  __shared__ double table[kPerOctave];
  const int r = blockIdx.x / j.parts, part = blockIdx.x % j.parts, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const TruncateArgs& a = j.a;
  fill_table(table);
  const float top = row_top(j, r);
  const RowInfo in = find_bins(j, r, top, sh, scan);
  if (part == 0 && threadIdx.x == 0) j.info[r] = in;
  if (in.mode != kDraw) return;
  const float* z = a.z + (size_t)r * a.ldz;
  const Weigher w{top, kPerOctave * 1.4426950408889634 / (double)temperature(a, r), table};
  const int sure = in.p0 >= 0 ? in.p0 : in.kb >= 0 ? in.kb : kBins;  // bins ahead of it are kept
  const float least = from_ordered_u32(in.least);
  for (int c = part * kWaves + wave; c < j.chunks; c += j.parts * kWaves) {
    f4 v[kSpans];
    load_chunk(z, a.V, c, v);
    u64 sum = 0;
    unsigned hits = 0;
#pragma unroll
    for (int k = 0; k < kSpans; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double f;
        const int i = w.place(v[k][e], f), b = bin_of(i);
        if (i < kOctaves * kPerOctave) {
          if (b < sure && v[k][e] >= least) sum += w.weight(i, f);
          if ((b >= in.p0 && b <= in.p1) || b == in.kb) hits |= 1u << (4 * k + e);
        }
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane == 0) j.chunk_sum[(size_t)r * j.chunks + c] = sum;
    if (__any(hits)) {
      const unsigned n = __popc(hits);
      unsigned incl = n;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const unsigned t = __shfl_up(incl, o, 64);
        if (lane >= o) incl += t;
      }
      unsigned base = 0;
      if (lane == 63) base = atomicAdd(&j.listed[r], incl);
      base = __shfl(base, 63, 64) + incl - n;
#pragma unroll
      for (int k = 0; k < kSpans; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (hits >> (4 * k + e) & 1) {
            if (base < (unsigned)j.cap)
              j.list[(size_t)r * j.cap + base] = uint2{__float_as_uint(v[k][e]), (unsigned)(c * kChunk + k * kSpan + lane * 4 + e)};
            ++base;
          }
    }
  }
}

// ----------------------------------------------------------------- pass 4 --
// The last id that a limit keeps, as (key, id): kept are larger keys, and equal ones up to that id.
struct Last {
  uint32_t key;
  int id;
  RGD_DEV bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= id); }
};

struct Row {
  const float* z;
  int V;
  Weigher w;
  RGD_DEV float at(int i) const {
    const float v = z[i] + 0.f;  // -0 is 0
    return v != v ? -INFINITY : v;
  }
  RGD_DEV u64 weight(float v) const { return w.of(v); }
};

struct Shared {
  u64 mass[kThreads];
  unsigned count[kThreads];
  u64 chunk[kMaxChunks];
  Scan scan;
  u64 lo, hi;
  double table[kPerOctave];
  uint32_t key;
  int id;
  u64 left, reached;
  unsigned rank, found;
};

RGD_DEV u64 block_before(u64 v, Shared& sh) {
  u64 before, all;
  unsigned n;
  block_scan(v, 0, sh.scan, before, n, all);
  return before;
}
RGD_DEV u64 block_total(u64 v, Shared& sh) {
  u64 before, all;
  unsigned n;
  block_scan(v, 0, sh.scan, before, n, all);
  return all;
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

// The listed ids of a thread.
struct Items {
  float z[kItems];
  int id[kItems], bin[kItems];  // bin -1: none
  u64 weight[kItems];
};

// The place in the order at which the items in the bins [b0, b1] reach a count k (if > 0) or a weight, with so many ids and
// so much weight ahead of them; left: the weight up to there.  1024 parts of the range at a time, until one item is left.
RGD_DEV u64 reach(const Items& it, int n, int b0, int b1, unsigned k, double mass, unsigned ahead, u64 left, Shared& sh) {
  u64 lo = ~0ull, hi = 0;
#pragma unroll
  for (int x = 0; x < kItems; ++x)
    if (x * kThreads < n && it.bin[x] >= b0 && it.bin[x] <= b1) {
      const u64 o = order_of(key_of(it.z[x]), it.id[x]);
      lo = min(lo, o);
      hi = max(hi, o);
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o, 64));
    hi = max(hi, __shfl_xor(hi, o, 64));
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    sh.lo = ~0ull;
    sh.hi = 0;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    atomicMin(&sh.lo, lo);
    atomicMax(&sh.hi, hi);
  }
  __syncthreads();
  lo = sh.lo;
  hi = sh.hi;
  for (;;) {
    const int bits = hi > lo ? 64 - __clzll(hi - lo) : 0, shift = max(bits - 10, 0);
    sh.mass[threadIdx.x] = 0;
    sh.count[threadIdx.x] = 0;
    if (threadIdx.x == 0) sh.found = 0;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kItems; ++x)
      if (x * kThreads < n && it.bin[x] >= b0 && it.bin[x] <= b1) {
        const u64 o = order_of(key_of(it.z[x]), it.id[x]);
        if (o >= lo && o <= hi) {
          atomicAdd(&sh.mass[(o - lo) >> shift], it.weight[x]);
          atomicAdd(&sh.count[(o - lo) >> shift], 1u);
        }
      }
    __syncthreads();
    const u64 m = sh.mass[threadIdx.x];
    const unsigned c = sh.count[threadIdx.x];
    u64 mb, all;
    unsigned cb;
    block_scan(m, c, sh.scan, mb, cb, all);
    mb += left;
    cb += ahead;
    // the first part with items that gets there (the first id is kept in any case)
    const bool here = c && (k ? cb < k && cb + c >= k : (double)(mb + m) >= mass && (cb == 0 || (double)mb < mass));
    if (here) {
      sh.key = threadIdx.x;
      sh.rank = cb;
      sh.left = mb;
      sh.reached = mb + m;
      sh.found = c;
    }
    __syncthreads();
    const unsigned found = sh.found;
    if (!found) return ~0ull;  // never: the bins say that it is reached among the items
    lo += (u64)sh.key << shift;
    hi = lo + (1ull << shift) - 1;
    ahead = sh.rank;
    left = sh.left;
    if (found == 1 || shift == 0) break;
    __syncthreads();
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kItems; ++x)
    if (x * kThreads < n && it.bin[x] >= b0 && it.bin[x] <= b1) {
      const u64 o = order_of(key_of(it.z[x]), it.id[x]);
      if (o >= lo && o <= hi) sh.lo = o;
    }
  __syncthreads();
  return sh.lo;
}

__global__ __launch_bounds__(kThreads) void truncate_draw_kernel(Job j) {
  __shared__ Shared sh;
  const int r = blockIdx.x, t = threadIdx.x;
  const TruncateArgs& a = j.a;
  const RowInfo in = j.info[r];
  const unsigned listed = j.listed[r];
  fill_table(sh.table);
  if (in.mode == kNone) {
    if (t == 0) {
      a.out[r] = -1;
      if (a.logp) a.logp[r] = -INFINITY;
    }
    return;
  }
  const float T = temperature(a, r);
  Row row{a.z + (size_t)r * a.ldz, a.V, Weigher{in.top, kPerOctave * 1.4426950408889634 / (double)T, sh.table}};
  if (in.mode == kGreedy) {
    // the first chunk that holds the maximum, then its first id
    if (t == 0) {
      sh.key = ~0u;
      sh.id = a.V;
    }
    __syncthreads();
    for (int c = t; c < j.chunks; c += kThreads)
      if (j.chunk_max[(size_t)r * j.chunks + c] == in.top) atomicMin(&sh.key, (unsigned)c);
    __syncthreads();
    for (int i = (int)sh.key * kChunk + t; i < min((int)(sh.key + 1) * kChunk, a.V); i += kThreads)
      if (row.z[i] == in.top) atomicMin(&sh.id, i);
    __syncthreads();
    if (t == 0) {
      a.out[r] = sh.id;
      if (a.logp) a.logp[r] = 0.f;
    }
    return;
  }
  const float top_p = a.top_p ? a.top_p[r] : 1.f;
  const unsigned k = in.kb >= 0 ? a.top_k[r] : 0;
  u64 border = ~0ull;  // the last kept place
  for (int c = t; c < j.chunks; c += kThreads) sh.chunk[c] = j.chunk_sum[(size_t)r * j.chunks + c];
  if (listed > (unsigned)j.cap) {
    // more ids in the borders' bins than are listed (equal logits, limits of many thousands): from the row itself
    __syncthreads();
    Last last{0, a.V};
    if (k) last = find(row, last, k, 0.0, sh);
    if (in.p0 >= 0) {
      u64 mine = 0;
      for (int i = t; i < a.V; i += kThreads) {
        const float v = row.at(i);
        if (last.keeps(ordered_u32(v), i)) mine += row.weight(v);
      }
      const u64 total = block_total(mine, sh);
      last = find(row, last, 0, fmax((double)top_p, 0.0) * (double)total, sh);
    }
    border = order_of(last.key, last.id);
    // the chunks' sums again, a wave a chunk
    __syncthreads();
    for (int c = t >> 6; c < j.chunks; c += kWaves) {
      u64 sum = 0;
      for (int i = c * kChunk + (t & 63); i < min((c + 1) * kChunk, a.V); i += 64) {
        const float v = row.at(i);
        const uint32_t key = ordered_u32(v);
        if (key >= in.least && last.keeps(key, i)) sum += row.weight(v);
      }
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      if ((t & 63) == 0) sh.chunk[c] = sum;
    }
  } else {
    const int n = (int)listed;
    Items it;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kItems; ++x)
      if (x * kThreads < n) {
        const int i = x * kThreads + t;
        const uint2 e = j.list[(size_t)r * j.cap + min(i, n - 1)];
        it.z[x] = __uint_as_float(e.x);
        it.id[x] = (int)e.y;
        double f;
        const int place = row.w.place(it.z[x], f);
        it.bin[x] = i < n ? bin_of(place) : -1;
        it.weight[x] = row.w.weight(place, f);
      }
    u64 kept = in.total;
    if (k) {
      border = reach(it, n, in.kb, in.kb, k, 0.0, in.before_k, in.mass_k, sh);
      kept = sh.reached;
    }
    if (in.p0 >= 0)
      border = min(border, reach(it, n, in.p0, in.p1, 0, fmax((double)top_p, 0.0) * (double)kept, in.mass_p ? 1 : 0, in.mass_p, sh));
    __syncthreads();
    if (k || in.p0 >= 0) {
      const int first = in.p0 >= 0 ? in.p0 : in.kb;
#pragma unroll
      for (int x = 0; x < kItems; ++x)
        if (x * kThreads < n && it.bin[x] >= first) {
          const uint32_t key = key_of(it.z[x]);
          if (key >= in.least && order_of(key, it.id[x]) <= border) atomicAdd(&sh.chunk[it.id[x] / kChunk], it.weight[x]);
        }
    }
  }
  __syncthreads();
  // the chunk that the draw falls in
  const u64 mine = t < j.chunks ? sh.chunk[t] : 0;
  u64 before, total;
  unsigned none;
  block_scan(mine, 0, sh.scan, before, none, total);
  const double u = fmin(fmax((double)a.u[r], 0.0), 1.0 - 1.0 / 16777216.0), target = u * (double)total;
  if (mine && (double)before <= target && (double)(before + mine) > target) {
    sh.id = t;
    sh.left = before;
  }
  __syncthreads();
  const int id0 = sh.id * kChunk + 2 * t;
  u64 left = sh.left, w[2];
  float v[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    v[e] = id0 + e < a.V ? row.at(id0 + e) : -INFINITY;
    const uint32_t key = ordered_u32(v[e]);
    w[e] = key >= in.least && order_of(key, id0 + e) <= border ? row.weight(v[e]) : 0;
  }
  u64 all;
  block_scan(w[0] + w[1], 0, sh.scan, before, none, all);
  left += before;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (w[e] && (double)left <= target && (double)(left + w[e]) > target) {
      a.out[r] = id0 + e;
      if (a.logp) a.logp[r] = (float)(((double)v[e] - (double)in.top) / (double)T - log((double)total / kOne));
    }
    left += w[e];
  }
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// The workspace's parts for up to `rows` rows; returns its bytes.
size_t lay_out(Job& j, int rows, char* ws) {
  size_t at = 0;
  auto take = [&](size_t n) {
    char* p = ws + at;
    at += up256(n);
    return p;
  };
  const size_t R = rows;
  j.chunk_max = (float*)take(R * j.chunks * 4);
  j.mass = (u64*)take(R * kBins * 8);
  j.count = (unsigned*)take(R * kBins * 4);
  j.chunk_sum = (u64*)take(R * j.chunks * 8);
  j.info = (RowInfo*)take(R * sizeof(RowInfo));
  j.listed = (unsigned*)take(R * 4);
  j.list = (uint2*)take(R * j.cap * 8);
  return at;
}

Job job_of(int V) {
  Job j{};
  j.chunks = (V + kChunk - 1) / kChunk;
  j.cap = std::min(V, kList);
  return j;
}

}  // namespace

size_t sample_truncated_workspace_bytes(int R, int V) {
  Job j = job_of(V);
  return lay_out(j, std::min(R, kSlab), nullptr);
}

hipError_t sample_truncated(const TruncateArgs& a, hipStream_t s) {
  for (int r0 = 0; r0 < a.R; r0 += kSlab) {
    Job j = job_of(a.V);
    j.a = a;
    const int R = j.a.R = std::min(a.R - r0, kSlab);
    lay_out(j, R, a.ws);
    j.a.z = a.z + (size_t)r0 * a.ldz;
    j.a.u = a.u + r0;
    j.a.out = a.out + r0;
    if (a.T) j.a.T = a.T + r0;
    if (a.top_k) j.a.top_k = a.top_k + r0;
    if (a.top_p) j.a.top_p = a.top_p + r0;
    if (a.min_p) j.a.min_p = a.min_p + r0;
    if (a.logp) j.a.logp = a.logp + r0;
    const int groups = (j.chunks + 3) / 4, most = (j.chunks + kWaves - 1) / kWaves;
    j.parts = std::max(1, std::min(most, 512 / R));
    j.merge = j.parts > 1;
    hipLaunchKernelGGL(truncate_max_kernel, dim3(R * groups), dim3(256), 0, s, j, groups);
    if (a.top_k || a.top_p) hipLaunchKernelGGL(truncate_bins_kernel, dim3(R * j.parts), dim3(kThreads), 0, s, j);
    hipLaunchKernelGGL(truncate_sum_kernel, dim3(R * j.parts), dim3(kThreads), 0, s, j);
    hipLaunchKernelGGL(truncate_draw_kernel, dim3(R), dim3(kThreads), 0, s, j);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace rgd
