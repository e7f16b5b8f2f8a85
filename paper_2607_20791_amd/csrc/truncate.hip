// One draw per row under temperature, top-k, top-p and min-p.
//
// With the ids in the order of their logits (equal ones by id) each limit keeps a leading part, and the kept ids are the
// shortest of these.  Weights are whole multiples of 2^-43 of the largest one's, so that sums are exact in 64-bit integers
// and no order of adding them matters.
//
// One read of the logits bounds it, and, where nearly all ids count, their weights: fp64, as the id drawn hangs on sums of up
// to 2^20 of them.  Four passes.  The first streams the logits for the maxima and counts them in bins of 1/64 octave of
// weight; the second finds from the counts the few bins in which the limits' borders must lie.  The third weighs every id that
// it has to and sums those that are kept for certain by chunks of 512 ids; the ids in the borders' bins go to a list.  The
// last, one workgroup a row, finds the borders among the listed ids by exact sums, the chunk that the draw falls in and
// its id.  The bins only say where to look: a border that is not there, or more listed ids than there is room for, is
// noticed, and the row is searched as a whole; where min_p's border seems to be above top_p's that is certain by bounds of
// the bins' weights, or compared at the end by exact ones.
//
// Measured, the four in order: 256 rows of 152064 logits (156 MB), all of one limit on the sum, 29 + 7 + 60 + 20 us: the
// first is the stream at 5.4 TB/s, the third about 30 instructions an id, the last a chain of
// reads and sums a row.  One row of 128256 5 + 10 + 4 + 15: launches and chains.  (The whole row ordered by radix passes in
// place of the bins: 1137 and 481 us.)
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "paged.hpp"
#include "weights.hpp"

namespace rgd {

namespace {

typedef unsigned long long u64;
typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));  // rows need no alignment

constexpr double kOne = 8796093022208.0;  // 2^43: the largest weight; 2^20 of them stay below 2^63
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kSpan = 256;         // ids: one wave, four a lane
constexpr int kSpans = 2;          // spans of a chunk
constexpr int kChunk = kSpan * kSpans;
constexpr int kMaxChunks = 2048;
constexpr int kOctaves = 45;       // below: a weight under 2^-44 is none
constexpr int kFine = 64;          // bins per octave
constexpr int kBins = kOctaves * kFine;
constexpr int kReach = kBins + kFine;  // bins below its maximum that a workgroup counts
constexpr int kRing = 8192;        // bins are counted modulo this
constexpr float kLowest = -3.402823466e38f;  // -inf is never an id that weighs something, however large T is
constexpr float kFar = 524288.f;   // 2^19 bins from 0: up to there, three roundings of fp32 are within 1/8 of a bin
constexpr int kNear = 4096;        // listed ids that the last pass holds in LDS
constexpr int kList = 16384;       // of a row, about
constexpr int kRoom = 512;         // of a list, at least
constexpr int kMaxLists = 512;
constexpr int kSlab = 1024;        // rows at a time, for the workspace's sake
constexpr int kWide = 32;          // rows from which on a wave takes more chunks at a time
constexpr int kGroups = 512;       // workgroups of few rows
constexpr int kPerWave = 16;       // chunks of a wave of the third pass, at most

// What the second pass found of a row's limits.
struct RowInfo {
  float top, T;
  uint32_t least;      // key of the lowest logit that min_p keeps
  int mode;            // below
  int by_k, by_p;      // whether these limits cut anything; by_p of kBelow: only if what the others keep weighs too much
  float k_low, k_end;  // the ids from k_low up to below k_end are listed: top_k's border is among them
  float p_low, p_end;  // top_p's; infinite where there is no such limit, as top_k's
  float kept;          // ids from here on are kept for certain
  float whole;         // of what top_p refers to, ids from here on are not listed as top_k's
  float low;           // what is below concerns nothing
};
enum { kNone, kGreedy, kDraw };
constexpr int kBelow = 2;

struct Job {
  TruncateArgs a;
  int chunks;
  int parts;          // workgroups of a row in the first pass
  int lists, per_wave;  // in the third, and chunks of a wave there
  int room;           // of a list
  float* chunk_max;   // [R][chunks]
  int* top_bin;       // [R][parts]: bin of the part's maximum
  unsigned* bins;     // [R][parts][kReach], counts from there downwards
  RowInfo* info;      // [R]
  u64* chunk_sum;     // [R][chunks]: of the ids above the borders' bins
  u64* list_sum;      // [R][lists]: of what top_p's border refers to and is not listed
  unsigned* list_count;  // [R][lists]: ids above top_k's bin
  unsigned* listed;   // [R][lists]: ids listed, or more than there is room for
  uint2* list;        // [R][lists][room] (logit, id)
};

// ---------------------------------------------------------------- weights --
// An id's weight 2^y, y = (z - top) log2(e) / T: with n the whole number next to y, 2^(y - n) by a polynomial of degree 9 on
// [-1/2, 1/2] whose largest error is the least there is (2^-46 of the weight; of degree 8 2^-40, more than the rounding),
// rounded to a whole multiple of 2^-43, so that the largest one is 1.  (A table of powers takes four products less, and LDS more
// time than these.)
struct Weigher {
  double top, scale;
  float low;  // what is below weighs nothing
  // of a logit that weighs something (others: any)
  RGD_DEV double weight(float z) const {
    constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: a sum's last bit is 1
    constexpr double kUnit = 768.0;                // 1.5 * 2^9: a sum's last bit is 2^-43
    const double d = (double)z - top, t = fma(d, scale, kRound), f = fma(d, scale, -(t - kRound));
    double s = 1.0150336704816022e-07;
    s = fma(s, f, 1.325940560926017e-06);
    s = fma(s, f, 1.5252984838656468e-05);
    s = fma(s, f, 0.00015403434948072205);
    s = fma(s, f, 0.0013333557617604436);
    s = fma(s, f, 0.009618129192067245);
    s = fma(s, f, 0.05550410866868561);
    s = fma(s, f, 0.24022650695649653);
    s = fma(s, f, 0.693147180559871);
    s = fma(s, f, 1.0000000000000127);
    s = __hiloint2double(__double2hiint(s) + (__double2loint(t) << 20), __double2loint(s));
    return (s + kUnit) - kUnit;
  }
  RGD_DEV u64 of(float z) const { return z >= low ? (u64)(weight(z) * kOne) : 0; }
};

RGD_DEV Weigher weigher(float top, float T) {
  // ids below `low` weigh nothing: the float nearest to 46 octaves down has none beyond 45 above it, whatever T is
  return Weigher{top, 1.4426950408889634 / (double)T, fmaxf(top - 46.f * 0.6931472f * T, kLowest)};
}

// The sum over the wave, in its last lane (without LDS, which is short of time here).
template <int CTRL, int ROWS>
RGD_DEV double sum_step(double v) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xf, false);
  return v + __hiloint2double(hi, lo);
}
RGD_DEV double last_lane_sum(double v) {
  v = sum_step<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
  v = sum_step<0x112, 0xf>(v);
  v = sum_step<0x114, 0xf>(v);
  v = sum_step<0x118, 0xf>(v);
  v = sum_step<0x142, 0xa>(v);  // row_bcast 15, 31
  return sum_step<0x143, 0xc>(v);
}

RGD_DEV bool greedy(float T) { return !(T > 0.f); }
RGD_DEV float temperature(const TruncateArgs& a, int r) { return a.T ? a.T[r] : 1.f; }

RGD_DEV uint32_t key_of(float z) {
  z += 0.f;  // -0 is 0
  return ordered_u32(z != z ? -INFINITY : z);
}

// A place in the order of a row's ids: ascending here is descending by logit, then ascending by id.
RGD_DEV u64 order_of(uint32_t key, int id) { return (u64)(~key) << 20 | (unsigned)id; }

// This lane's ids of N chunks, 4 lane + {0..3} of each span; behind the row -inf.
template <int N>
RGD_DEV void load_chunks(const float* z, int V, int chunk, f4 (&v)[N * kSpans]) {
  const int lane = threadIdx.x & 63;
  if ((chunk + N) * kChunk <= V) {
#pragma unroll
    for (int k = 0; k < N * kSpans; ++k) v[k] = *(const f4*)(z + chunk * kChunk + k * kSpan + lane * 4);
  } else {
#pragma unroll
    for (int k = 0; k < N * kSpans; ++k)
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
#pragma unroll 1
  for (int k = 0; k < kMaxChunks / 64; k += 4)  // four loads at a time
    if (64 * k < j.chunks)
#pragma unroll
      for (int i = k; i < k + 4; ++i)
        top = fmaxf(top, j.chunk_max[(size_t)r * j.chunks + min(64 * i + lane, j.chunks - 1)]);
  return wave_max(top);
}

RGD_DEV float min_p_least(const TruncateArgs& a, int r, float top) {
  const float p = a.min_p ? a.min_p[r] : 0.f;
  if (!(p > 0.f)) return -INFINITY;
  return threshold(top, p < 1.f ? (double)temperature(a, r) * log((double)p) : 0.0);
}
RGD_DEV bool has_top_p(const TruncateArgs& a, int r) { return a.top_p && a.top_p[r] < 1.f; }
RGD_DEV bool has_top_k(const TruncateArgs& a, int r) { return a.top_k && a.top_k[r] > 0 && a.top_k[r] < a.V; }
RGD_DEV float bins_per_logit(float T) { return kFine * 1.4426950408889634f / T; }

// ----------------------------------------------------------------- pass 1 --
constexpr int kStream = 2;  // chunks of a wave at a time where rows are many

// Maxima of the chunks, and the numbers of ids by floor(z * bins per logit), modulo kRing: ids further below the maximum
// of what the workgroup reads first than they could matter are left out, so that no two bins that could are taken for one.
template <int N>
__global__ __launch_bounds__(kThreads, 8) void truncate_count_kernel(Job j) {
  __shared__ unsigned bins[kRing];
  __shared__ float red[2][kWaves];
  const int r = blockIdx.x / j.parts, part = blockIdx.x % j.parts, t = threadIdx.x, wave = t >> 6, lane = t & 63;
  const TruncateArgs& a = j.a;
  const float* z = a.z + (size_t)r * a.ldz;
  const float T = temperature(a, r), per = bins_per_logit(T);
  const bool binned = !greedy(T) && (has_top_p(a, r) || has_top_k(a, r)) && per < INFINITY;
  if (binned)
    for (int i = t; i < kRing; i += kThreads) bins[i] = 0;
  const int step = j.parts * kWaves * N;
  float first = -INFINITY, most = -INFINITY, low = INFINITY;
  for (int again = 0; again < 2; ++again) {
    for (int c0 = part * kWaves * N, c = c0 + wave * N; c0 < j.chunks; c0 += step, c += step) {
      f4 v[N * kSpans];
      if (c < j.chunks) {
        load_chunks<N>(z, a.V, c, v);
        if (!again) {
#pragma unroll
          for (int n = 0; n < N; ++n) {
            float m = -INFINITY;  // NaN counts as -inf: fmaxf takes the other operand
#pragma unroll
            for (int k = n * kSpans; k < (n + 1) * kSpans; ++k)
              m = fmaxf(m, fmaxf(fmaxf(v[k][0], v[k][1]), fmaxf(v[k][2], v[k][3])));
            m = wave_max(fmaxf(m, -INFINITY));
            if (lane == 0 && c + n < j.chunks) j.chunk_max[(size_t)r * j.chunks + c + n] = m;
            most = fmaxf(most, m);
          }
        }
      }
      if (!binned) continue;
      if (!again && c0 == part * kWaves * N) {
        if (lane == 0) red[0][wave] = most;
        __syncthreads();
        for (int i = 0; i < kWaves; ++i) first = fmaxf(first, red[0][i]);
        low = first > -INFINITY ? fmaxf(first - kReach / per, kLowest) : INFINITY;
      }
      if (c < j.chunks)
#pragma unroll
        for (int k = 0; k < N * kSpans; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (v[k][e] >= low) atomicAdd(&bins[(int)floorf(v[k][e] * per) & (kRing - 1)], 1u);
    }
    if (!binned) return;
    if (again) break;
    if (lane == 0) red[1][wave] = most;
    __syncthreads();
    for (int i = 0; i < kWaves; ++i) most = fmaxf(most, red[1][i]);
    if (!((most - first) * per > 2000.f)) break;  // (-inf - -inf: no)
    // what came first lies far below the rest: again, from the maximum
    low = fmaxf(most - kReach / per, kLowest);
    for (int i = t; i < kRing; i += kThreads) bins[i] = 0;
    __syncthreads();
  }
  __syncthreads();
  const float at = most * per;
  const bool near = fabsf(at) <= 4 * kFar;  // (not: the maximum's part of the row is given up, or this one does not matter)
  const int top = near ? (int)floorf(at) : -(1 << 30);
  if (t == 0) j.top_bin[r * j.parts + part] = top;
  if (near)
    for (int i = t; i < kReach; i += kThreads) j.bins[((size_t)r * j.parts + part) * kReach + i] = bins[(top - i) & (kRing - 1)];
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

// ----------------------------------------------------------------- pass 2 --
struct Found {
  unsigned bins[kBins];
  float mass[kWaves], square[kWaves];
  unsigned count[kWaves];
  int k, p0, p1;
  float ahead;    // estimate of what top_p's border refers to
  float most[kWaves];  // of what min_p keeps
};

// The bins of the borders, one workgroup a row, from the counts: a bin's weight is that of its middle, within half of 1/64
// octave.  The border of a count is where it is; that of a weight within the error of many such weights, which
// go either way.
RGD_DEV RowInfo find_bins(const Job& j, int r, Found& sh) {
  const TruncateArgs& a = j.a;
  RowInfo in{};
  in.T = temperature(a, r);
  const bool by_p = has_top_p(a, r), by_k = has_top_k(a, r), binned = !greedy(in.T) && (by_p || by_k);
  // all parts' counts are asked for before the first is looked at, up to kBatch parts
  constexpr int kBatch = 16, kPer = (kReach + kThreads - 1) / kThreads;
  unsigned c[kBatch][kPer];
  auto load = [&](int p0) {
#pragma unroll
    for (int x = 0; x < kBatch; ++x)
      if (p0 + x < j.parts)
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          c[x][i] = j.bins[((size_t)r * j.parts + p0 + x) * kReach + min(i * kThreads + (int)threadIdx.x, kReach - 1)];
  };
  if (binned) load(0);
  const float top = in.top = row_top(j, r);
  for (int i = threadIdx.x; i < kBins; i += kThreads) sh.bins[i] = 0;
  in.k_low = in.k_end = in.p_low = in.p_end = in.whole = INFINITY;
  in.mode = !finite_top(top) ? kNone : greedy(in.T) ? kGreedy : kDraw;
  if (in.mode != kDraw) return in;
  const float least = min_p_least(a, r, top), floor_z = weigher(top, in.T).low;
  in.least = key_of(least);
  in.kept = in.low = fmaxf(floor_z, least);
  if (!binned) return in;
  in.by_p = by_p;
  in.by_k = by_k;
  const float per = bins_per_logit(in.T), at = top * per;
  if (!(fabsf(at) <= kFar)) {
    // so low a temperature that bins are finer than logits: all ids of any weight are looked at
    if (by_k) in.k_low = floor_z;
    if (by_p) in.p_low = floor_z;
    in.kept = INFINITY;
    if (by_p && !by_k) in.whole = floor_z;
    in.low = floor_z;
    return in;
  }
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, top_bin = (int)floorf(at);
  __syncthreads();
  for (int p0 = 0; p0 < j.parts; p0 += kBatch) {
    if (p0) load(p0);
#pragma unroll
    for (int x = 0; x < kBatch; ++x)
      if (p0 + x < j.parts) {
        const int ahead = top_bin - j.top_bin[r * j.parts + p0 + x];  // 0 and more
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int b = i * kThreads + t;
          if (b < kReach && ahead < kBins - b && c[x][i]) atomicAdd(&sh.bins[b + ahead], c[x][i]);
        }
      }
  }
  __syncthreads();
  constexpr int PER = (kBins + kThreads - 1) / kThreads;
  unsigned count[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) count[i] = t * PER + i < kBins ? sh.bins[t * PER + i] : 0;
  float weight[PER], mass = 0.f, square = 0.f;
  unsigned n = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    weight[i] = __builtin_amdgcn_exp2f(-((at - floorf(at)) + (t * PER + i) - 0.5f) / kFine);
    mass += count[i] * weight[i];
    square += count[i] * weight[i] * weight[i];
    n += count[i];
  }
  float mi = mass, sq = square;
  unsigned ni = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const float x = __shfl_up(mi, o, 64), y = __shfl_up(sq, o, 64);
    const unsigned c = __shfl_up(ni, o, 64);
    if (lane >= o) {
      mi += x;
      sq += y;
      ni += c;
    }
  }
  if (lane == 63) {
    sh.mass[wave] = mi;
    sh.square[wave] = sq;
    sh.count[wave] = ni;
  }
  if (t == 0) {
    sh.k = -1;
    sh.p0 = sh.p1 = kBins - 1;
  }
  __syncthreads();
  float total = 0.f, squares = 0.f;
  mi -= mass;
  ni -= n;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) {
      mi += sh.mass[i];
      ni += sh.count[i];
    }
    total += sh.mass[i];
    squares += sh.square[i];
  }
  if (in.by_k) {
    const unsigned k = a.top_k[r];
    float x = mi;
    unsigned c = ni;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (c < k && c + count[i] >= k) {
        sh.k = t * PER + i;
        sh.ahead = x + (float)(k - c) * weight[i];
      }
      c += count[i];
      x += count[i] * weight[i];
    }
    __syncthreads();
    if (sh.k < 0) in.by_k = 0;  // no more ids than that weigh anything
    else total = sh.ahead;
  }
  if (in.by_p) {
    const float error = 1e-4f * total + 0.0128f * sqrtf(squares), target = fmaxf(a.top_p[r], 0.f) * total;
    float x = mi;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float y = x + count[i] * weight[i];
      if (count[i]) {
        if (y >= target - error && (x == 0.f || x < target - error)) atomicMin(&sh.p0, t * PER + i);
        if (y >= target + error && (x == 0.f || x < target + error)) atomicMin(&sh.p1, t * PER + i);
      }
      x = y;
    }
    __syncthreads();
  }
  // logits at the bins' ends and a fifth of a bin on (of three roundings, each within 1/16)
  const float step = 1.f / per;
  auto logit = [&](int bin, float off) { return ((float)(top_bin - bin) + off) * step; };
  if (in.by_k) {
    in.k_low = logit(sh.k, -0.2f);
    if (sh.k) in.k_end = logit(sh.k, 1.2f);
  }
  if (in.by_p) {
    in.p_low = fmaxf(logit(sh.p1, -0.2f), floor_z);
    if (sh.p0) in.p_end = logit(sh.p0, 1.2f);
  }
  if (!in.by_p && !in.by_k) return in;  // fewer than top_k weigh anything
  bool above = least >= (in.by_p ? in.p_end : in.k_end);  // min_p's border above the others
  if (above && in.by_p) {
    // For top_p that is an estimate, whose error equal logits share.  Certain is that an id weighs its bin's middle times 2^(1/128) at
    // most, or a little more (a fifth of a bin) for the roundings of z * per, and as much less at least: within 1%
    // with those of the sums.  Otherwise what min_p keeps is weighed and compared at the end.
    float most = 0.f;
    const float bin = (float)top_bin - (floorf(least * per) - 1.f);  // of the lowest id that it may keep
#pragma unroll
    for (int i = 0; i < PER; ++i) most += (float)(t * PER + i) <= bin ? count[i] * weight[i] : 0.f;
    most = wave_sum(most);
    if (lane == 0) sh.most[wave] = most;
    __syncthreads();
    most = 0.f;
    for (int i = 0; i < kWaves; ++i) most += sh.most[i];
    above = most * 1.01f < a.top_p[r] * (total * 0.99f) && (!in.by_k || least >= in.k_end);
    if (!above) {
      in.by_p = kBelow;
      in.p_low = in.p_end = INFINITY;
    }
  }
  if (above) {
    in.by_k = in.by_p = 0;
    in.k_low = in.k_end = in.p_low = in.p_end = INFINITY;
    return in;
  }
  if (in.by_p != kBelow) in.kept = fmaxf(in.kept, in.by_p ? in.p_end : in.k_end);
  else if (in.by_k) in.kept = fmaxf(in.kept, in.k_end);
  if (in.by_p) in.whole = in.by_k ? fmaxf(in.k_end, floor_z) : floor_z;
  in.low = fminf(fminf(in.kept, in.whole), fminf(in.p_low, in.k_low));
  return in;
}

__global__ __launch_bounds__(kThreads, 4) void truncate_bins_kernel(Job j) {
  __shared__ Found sh;
  const RowInfo in = find_bins(j, blockIdx.x, sh);
  if (threadIdx.x == 0) j.info[blockIdx.x] = in;
}

// ----------------------------------------------------------------- pass 3 --
// Sums of the chunks' weights above the borders' bins, and of all that top_p refers to; the ids in these bins are listed.
__global__ __launch_bounds__(256, 8) void truncate_sum_kernel(Job j) {
  __shared__ unsigned listed, count;
  __shared__ u64 sums;
  const int r = blockIdx.x / j.lists, part = blockIdx.x % j.lists, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const TruncateArgs& a = j.a;
  const float* z = a.z + (size_t)r * a.ldz;
  int c = (part * 4 + wave) * j.per_wave;
  const int end = min(c + j.per_wave, j.chunks);
  f4 v[kSpans];
  if (c < end) load_chunks<1>(z, a.V, c, v);
  const RowInfo& in = j.info[r];
  if (in.mode != kDraw) return;
  const Weigher w = weigher(in.top, in.T);
  const float kept = in.kept, whole = in.whole, low = in.low, p_low = in.p_low, p_end = in.p_end, k_low = in.k_low,
              k_end = in.k_end;
  const int by_k = in.by_k;
  if (threadIdx.x == 0) {
    listed = count = 0;
    sums = 0;
  }
  __syncthreads();
  // Multiples of 2^-43, none above 1: sums of up to 2^10 of them are exact in fp64.
  static_assert(kChunk <= 1 << 10 && kPerWave * kChunk / 64 <= 1 << 10, "a chunk's, a lane's");
  double all = 0.0;
  unsigned above = 0;
  uint2* list = j.list + ((size_t)r * j.lists + part) * j.room;
  auto chunks = [&](auto by_k) {
    while (c < end) {
      double sum = 0.0;
      unsigned hits = 0;
#pragma unroll
      for (int k = 0; k < kSpans; ++k) {
        const f4 x = v[k];
        if (!__any((x[0] >= low) | (x[1] >= low) | (x[2] >= low) | (x[3] >= low))) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double y = w.weight(x[e]);
          sum += x[e] >= kept ? y : 0.0;
          all += x[e] >= whole ? y : 0.0;
          bool hit = (x[e] >= p_low) & (x[e] < p_end);
          if constexpr (by_k) {
            above += x[e] >= k_end;
            hit |= (x[e] >= k_low) & (x[e] < k_end);
          }
          hits |= hit ? 1u << (4 * k + e) : 0u;
        }
      }
      if (__any(hits)) {
        unsigned at = hits ? atomicAdd(&listed, (unsigned)__popc(hits)) : 0;
#pragma unroll
        for (int k = 0; k < kSpans; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (hits >> (4 * k + e) & 1 && at < (unsigned)j.room)
              list[at++] = uint2{__float_as_uint(v[k][e]), (unsigned)(c * kChunk + k * kSpan + lane * 4 + e)};
      }
      const int done = c++;
      if (c < end) load_chunks<1>(z, a.V, c, v);
      sum = last_lane_sum(sum);
      if (lane == 63) j.chunk_sum[(size_t)r * j.chunks + done] = (u64)(sum * kOne);
    }
  };
  if (by_k) chunks(std::true_type{});
  else chunks(std::false_type{});
  u64 mine = (u64)(all * kOne);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    mine += __shfl_xor(mine, o, 64);
    above += __shfl_xor(above, o, 64);
  }
  if (lane == 63) {
    atomicAdd(&sums, mine);
    atomicAdd(&count, above);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const int at = r * j.lists + part;
    j.list_sum[at] = sums;
    j.list_count[at] = count;
    j.listed[at] = listed;
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

constexpr int kParts = 1024;  // of a range of the order
RGD_DEV int padded(int part) { return part + (part >> 4); }  // a lane's 16 parts start in banks of their own
struct Shared {
  u64 mass[kParts + kParts / 16];
  unsigned count[kParts + kParts / 16];
  u64 chunk[kMaxChunks];
  u64 order[kNear], weight[kNear];  // of the first listed ids
  u64 few_order[64], few_weight[64];
  Scan scan;
  u64 whole, kept;   // weight that top_p refers to, that is above its bins
  unsigned above;    // ids above top_k's bin
  u64 border;
  unsigned start[kMaxLists + 1];  // of each list's items among all
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

// The listed ids: places in the order and weights, the first kNear of them in LDS.
struct Items {
  const uint2* list;
  int n, room;
  const Weigher& w;
  Shared& sh;
  RGD_DEV uint2 far(int i) const {
    int p = 0;
    while (i >= (int)sh.start[p + 1]) ++p;
    return list[(size_t)p * room + i - sh.start[p]];
  }
  RGD_DEV u64 order_at(int i) const {
    if (i < kNear) return sh.order[i];
    const uint2 e = far(i);
    return order_of(key_of(__uint_as_float(e.x)), (int)e.y);
  }
  RGD_DEV u64 weight_at(int i) const { return i < kNear ? sh.weight[i] : w.of(__uint_as_float(far(i).x)); }
};

RGD_DEV u64 readlane_u64(u64 v, int lane) {
  const unsigned lo = __builtin_amdgcn_readlane((int)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
  return (u64)hi << 32 | lo;
}
RGD_DEV void wave_before(u64 m, unsigned c, u64& mb, unsigned& cb) {
  const int lane = threadIdx.x & 63;
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
  mb = mi - m;
  cb = ci - c;
}

// The place in the order at which the items in [lo, hi] reach a count k (if > 0) or a weight, with so many ids and
// so much weight ahead of them; sh.reached: the weight up to there.  1024 parts of the range, then the items of the one where it
// happens, ranked by one wave.
RGD_DEV u64 reach(const Items& it, u64 lo, u64 hi, unsigned k, double mass, unsigned ahead, u64 left, Shared& sh) {
  const int t = threadIdx.x;
  auto gets_there = [&](u64 mb, u64 m, unsigned cb, unsigned c) {  // (the first id is kept in any case)
    return c && (k ? cb < k && cb + c >= k : (double)(mb + m) >= mass && (cb == 0 || (double)mb < mass));
  };
  for (;;) {
    if (it.n <= 64) break;
    const int shift = max((hi > lo ? 64 - __clzll(hi - lo) : 0) - 10, 0);
    __syncthreads();
    for (int i = t; i < kParts + kParts / 16; i += kThreads) {
      sh.mass[i] = 0;
      sh.count[i] = 0;
    }
    if (t == 0) sh.found = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = t; i < it.n; i += kThreads) {
      const u64 o = it.order_at(i);
      if (o >= lo && o <= hi) {
        const int part = padded((int)((o - lo) >> shift));
        atomicAdd(&sh.mass[part], it.weight_at(i));
        atomicAdd(&sh.count[part], 1u);
      }
    }
    __syncthreads();
    if (t < 64) {
      constexpr int PER = kParts / 64;
      u64 m = 0, mb;
      unsigned c = 0, cb;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        m += sh.mass[padded(t * PER + i)];
        c += sh.count[padded(t * PER + i)];
      }
      wave_before(m, c, mb, cb);
      mb += left;
      cb += ahead;
      if (gets_there(mb, m, cb, c))
        for (int i = 0; i < PER; ++i) {
          const u64 x = sh.mass[padded(t * PER + i)];
          const unsigned y = sh.count[padded(t * PER + i)];
          if (gets_there(mb, x, cb, y)) {
            sh.key = t * PER + i;
            sh.found = y;
            sh.left = mb;
            sh.id = (int)cb;
            break;
          }
          mb += x;
          cb += y;
        }
    }
    __syncthreads();
    const unsigned found = sh.found;
    if (!found) return ~0ull;  // not among the items
    lo += (u64)sh.key << shift;
    hi = lo + (1ull << shift) - 1;
    ahead = (unsigned)sh.id;
    left = sh.left;
    if (found <= 64) break;
  }
  __syncthreads();
  if (t == 0) {
    sh.rank = 0;
    sh.border = ~0ull;
  }
  __syncthreads();
#pragma unroll 1
  for (int i = t; i < it.n; i += kThreads) {
    const u64 o = it.order_at(i);
    if (o >= lo && o <= hi) {
      const unsigned x = atomicAdd(&sh.rank, 1u);
      sh.few_order[x] = o;
      sh.few_weight[x] = it.weight_at(i);
    }
  }
  __syncthreads();
  if (t < 64) {
    const int found = (int)sh.rank;
    const bool mine = t < found;
    const u64 o = mine ? sh.few_order[t] : ~0ull, m = mine ? sh.few_weight[t] : 0;
    u64 mb = left;
    unsigned cb = ahead;
    for (int i = 0; i < found; ++i) {
      const u64 oi = readlane_u64(o, i), mi = readlane_u64(m, i);
      if (oi < o) {
        mb += mi;
        ++cb;
      }
    }
    if (mine && gets_there(mb, m, cb, 1)) {
      sh.border = o;
      sh.reached = mb + m;
    }
  }
  __syncthreads();
  return sh.border;
}

__global__ __launch_bounds__(kThreads) void truncate_draw_kernel(Job j) {
  __shared__ Shared sh;
  const int r = blockIdx.x, t = threadIdx.x;
  const TruncateArgs& a = j.a;
  const unsigned listed = t < j.lists ? j.listed[r * j.lists + t] : 0;
  const RowInfo in = j.info[r];
  if (in.mode == kNone) {
    if (t == 0) {
      a.out[r] = -1;
      if (a.logp) a.logp[r] = -INFINITY;
    }
    return;
  }
  const float T = in.T;
  Row row{a.z + (size_t)r * a.ldz, a.V, weigher(in.top, T)};
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
    const int i = (int)sh.key * kChunk + t;
    if (t < kChunk && i < a.V && row.z[i] == in.top) atomicMin(&sh.id, i);
    __syncthreads();
    if (t == 0) {
      a.out[r] = sh.id;
      if (a.logp) a.logp[r] = 0.f;
    }
    return;
  }
  const float top_p = a.top_p ? a.top_p[r] : 1.f;
  const unsigned k = in.by_k ? a.top_k[r] : 0;
  u64 border = ~0ull;  // the last kept place
  bool fine = true;
  if (in.by_k || in.by_p) {
    fine = !__syncthreads_or(listed > (unsigned)j.room);
    u64 none, all;
    unsigned start;
    block_scan(0, listed, sh.scan, none, start, all);
    if (t < j.lists) sh.start[t] = start;
    if (t == j.lists - 1) sh.start[j.lists] = start + listed;
    if (t == 0) {
      sh.whole = sh.kept = 0;
      sh.above = 0;
    }
    __syncthreads();
  }
  u64 sum = 0;
  for (int c = t; c < j.chunks; c += kThreads) sum += sh.chunk[c] = j.chunk_sum[(size_t)r * j.chunks + c];
  if ((in.by_k || in.by_p) && fine) {
    if (sum) atomicAdd(&sh.kept, sum);
    if (t < j.lists) {
      atomicAdd(&sh.whole, j.list_sum[r * j.lists + t]);
      atomicAdd(&sh.above, j.list_count[r * j.lists + t]);
    }
    const Items it{j.list + (size_t)r * j.lists * j.room, (int)sh.start[j.lists], j.room, row.w, sh};
#pragma unroll 1
    for (int l = t >> 6; l < j.lists; l += kWaves) {  // a wave a list
      const int start = sh.start[l], n = min((int)sh.start[l + 1], kNear) - start;
      for (int i = t & 63; i < n; i += 64) {
        const uint2 e = it.list[(size_t)l * j.room + i];
        const float z = __uint_as_float(e.x);
        sh.order[start + i] = order_of(key_of(z), (int)e.y);
        sh.weight[start + i] = row.w.of(z);
      }
    }
    __syncthreads();
    u64 whole = sh.whole;
    const u64 kept = sh.kept;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {  // top_k, top_p
      if (which ? !in.by_p || in.by_p == kBelow : !k) continue;
      const float z0 = which ? in.p_low : in.k_low, z1 = which ? in.p_end : in.k_end;
      const u64 lo = z1 <= in.top ? order_of(key_of(z1), 0xFFFFF) + 1 : order_of(key_of(in.top), 0),
                hi = order_of(key_of(z0), 0xFFFFF);
      const double mass = which ? fmax((double)top_p, 0.0) * (double)whole : 0.0;
      const unsigned ahead = which ? kept != 0 : sh.above;
      const u64 at = reach(it, lo, hi, which ? 0 : k, mass, ahead, which ? kept : whole, sh);
      fine = fine && at != ~0ull;
      if (!fine) break;
      border = min(border, at);
      whole = sh.reached;
    }
    if (fine) {
#pragma unroll 1
      for (int i = t; i < it.n; i += kThreads) {
        const u64 o = it.order_at(i);
        if (o <= border && (uint32_t)~(o >> 20) >= in.least) atomicAdd(&sh.chunk[(int)(o & 0xFFFFF) / kChunk], it.weight_at(i));
      }
      if (in.by_p == kBelow) {
        // top_p keeps all of what the other limits keep where that weighs less than it may
        __syncthreads();
        u64 all = 0;
        for (int c = t; c < j.chunks; c += kThreads) all += sh.chunk[c];
        fine = (double)block_total(all, sh) < (double)top_p * (double)whole;
      }
    }
  }
  if (!fine) {
    // more ids in the borders' bins than are listed (equal logits, limits near all of the weight), or a border
    // that is not among them: from the row itself
    __syncthreads();
    border = ~0ull;
    Last last{0, a.V};
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
      if (which ? !in.by_p : !k) continue;
      double mass = 0.0;
      if (which) {
        u64 mine = 0;
#pragma unroll 1
        for (int i = t; i < a.V; i += kThreads) {
          const float v = row.at(i);
          if (last.keeps(ordered_u32(v), i)) mine += row.weight(v);
        }
        mass = fmax((double)top_p, 0.0) * (double)block_total(mine, sh);
      }
      last = find(row, last, which ? 0 : k, mass, sh);
    }
    border = order_of(last.key, last.id);
    // the chunks' sums again, a wave a chunk
    __syncthreads();
#pragma unroll 1
    for (int c = t >> 6; c < j.chunks; c += kWaves) {
      u64 x = 0;
      for (int i = c * kChunk + (t & 63); i < min((c + 1) * kChunk, a.V); i += 64) {
        const float v = row.at(i);
        const uint32_t key = ordered_u32(v);
        if (key >= in.least && last.keeps(key, i)) x += row.weight(v);
      }
      for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
      if ((t & 63) == 0) sh.chunk[c] = x;
    }
  }
  __syncthreads();
  if (t >= 64) return;
  // the chunk that the draw falls in, by one wave
  const int per = (j.chunks + 63) / 64;
  u64 mine = 0, before, total;
  unsigned none;
  for (int i = 0; i < per; ++i)
    if (t * per + i < j.chunks) mine += sh.chunk[t * per + i];
  wave_before(mine, 0, before, none);
  total = readlane_u64(before + mine, 63);
  const double u = fmin(fmax((double)a.u[r], 0.0), 1.0 - 1.0 / 16777216.0), target = u * (double)total;
  auto falls_in = [&](u64 x) { return x && (double)before <= target && (double)(before + x) > target; };
  int chunk = 0;
  const unsigned long long in_lane = __ballot(falls_in(mine));
  if (falls_in(mine))
    for (int i = 0; i < per; ++i) {
      chunk = t * per + i;
      const u64 x = chunk < j.chunks ? sh.chunk[chunk] : 0;
      if (falls_in(x)) break;
      before += x;
    }
  const int lane = __builtin_ctzll(in_lane);
  chunk = __builtin_amdgcn_readlane(chunk, lane);
  before = readlane_u64(before, lane);
  // its id, of eight in a row a lane
  constexpr int PER = kChunk / 64;
  float v[PER];
  u64 x[PER], ahead;
  mine = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int id = chunk * kChunk + t * PER + e;
    v[e] = id < a.V ? row.z[id] : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int id = chunk * kChunk + t * PER + e;
    const uint32_t key = key_of(v[e]);
    x[e] = key >= in.least && order_of(key, id) <= border ? row.weight(v[e]) : 0;
    mine += x[e];
  }
  wave_before(mine, 0, ahead, none);
  before += ahead;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    if (falls_in(x[e])) {
      a.out[r] = chunk * kChunk + t * PER + e;
      if (a.logp) a.logp[r] = (float)(((double)v[e] - (double)in.top) / (double)T - log((double)total / kOne));
    }
    before += x[e];
  }
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// The first pass: few rows are shared out a chunk a wave, many two; about two workgroups per CU.
bool wide(int R) { return R >= kWide; }
int most_parts(int chunks, bool wide) {
  const int per = kWaves * (wide ? kStream : 1);
  return (chunks + per - 1) / per;
}
// The third: a wave takes up to kPerWave chunks where that leaves enough workgroups.
int lists_of(int chunks, int per_wave) { return (chunks + 4 * per_wave - 1) / (4 * per_wave); }
Job job_of(int R, int V) {
  Job j{};
  j.chunks = (V + kChunk - 1) / kChunk;
  j.parts = std::max(1, std::min(most_parts(j.chunks, wide(R)), kGroups / R));
  j.per_wave = std::max(1, std::min(kPerWave, (R * lists_of(j.chunks, 1) + 4 * kGroups - 1) / (4 * kGroups)));
  j.lists = lists_of(j.chunks, j.per_wave);
  j.room = std::max(kList / j.lists, kRoom);
  return j;
}

// The workspace's parts; returns its bytes.  What depends on how rows are shared out gets the most that R rows or
// fewer need, so that a workspace serves any smaller number, too.
size_t lay_out(Job& j, int rows, char* ws) {
  size_t at = 0;
  auto take = [&](size_t n) {
    char* p = ws + at;
    at += up256(n);
    return p;
  };
  const size_t R = rows, few = std::min(std::min(rows, kWide - 1) * most_parts(j.chunks, false), kGroups),
               many = wide(rows) ? std::min(rows * most_parts(j.chunks, true), kGroups) : 0,
               parts = std::max(R, std::max(few, many)), lists = R * lists_of(j.chunks, 1);
  j.chunk_max = (float*)take(R * j.chunks * 4);
  j.top_bin = (int*)take(parts * 4);
  j.bins = (unsigned*)take(parts * kReach * 4);
  j.info = (RowInfo*)take(R * sizeof(RowInfo));
  j.chunk_sum = (u64*)take(R * j.chunks * 8);
  j.list_sum = (u64*)take(lists * 8);
  j.list_count = (unsigned*)take(lists * 4);
  j.listed = (unsigned*)take(lists * 4);
  // up to 4 * kGroups + a row's lists of less than kPerWave chunks a wave, or any number of those with as many
  j.list = (uint2*)take((R * std::max(kList, lists_of(j.chunks, kPerWave) * kRoom) +
                         std::min(lists, (size_t)8 * kGroups + lists_of(j.chunks, 1)) * kRoom) * 8);
  return at;
}

}  // namespace

size_t sample_truncated_workspace_bytes(int R, int V) {
  const int rows = std::min(R, kSlab);
  Job j = job_of(rows, V);
  return lay_out(j, rows, nullptr);
}

hipError_t sample_truncated(const TruncateArgs& a, hipStream_t s) {
  for (int r0 = 0; r0 < a.R; r0 += kSlab) {
    const int R = std::min(a.R - r0, kSlab);
    Job j = job_of(R, a.V);
    j.a = a;
    j.a.R = R;
    lay_out(j, R, a.ws);
    j.a.z = a.z + (size_t)r0 * a.ldz;
    j.a.u = a.u + r0;
    j.a.out = a.out + r0;
    if (a.T) j.a.T = a.T + r0;
    if (a.top_k) j.a.top_k = a.top_k + r0;
    if (a.top_p) j.a.top_p = a.top_p + r0;
    if (a.min_p) j.a.min_p = a.min_p + r0;
    if (a.logp) j.a.logp = a.logp + r0;
    const dim3 grid(R * j.parts), block(kThreads);
    if (wide(R)) hipLaunchKernelGGL(truncate_count_kernel<kStream>, grid, block, 0, s, j);
    else hipLaunchKernelGGL(truncate_count_kernel<1>, grid, block, 0, s, j);
    hipLaunchKernelGGL(truncate_bins_kernel, dim3(R), block, 0, s, j);
    hipLaunchKernelGGL(truncate_sum_kernel, dim3(R * j.lists), dim3(256), 0, s, j);
    hipLaunchKernelGGL(truncate_draw_kernel, dim3(R), block, 0, s, j);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace rgd
