// Causal attention of a sequence's last few tokens over its pages.
//
// o = sum_j exp(a_j - lse) v_j with a_j = q . k_j / sqrt(D), lse = log sum_j exp(a_j): one pass over
// the keys and values with a running maximum and sum.  Each K and V is read
// from memory once for all query vectors of its KV head (tokens x query heads
// per KV head), a few operations a byte, so the reads bound it; the products
// go through MFMA, 16 query vectors to a tile, because the tile's unused
// columns cost less than the reads they wait for.
//
// A wave is the unit of work, without LDS or barriers.  The positions of all
// (sequence, KV head, query tile) items lie one behind the other in steps of
// 32, and every wave takes an equal run of steps, over the borders of items: short and
// long sequences fill the chip alike, whatever their order.  The waves work the
// runs out of the lengths on the device.  An item inside one run is finished by
// its wave; the pieces of one that is cut go to the workspace and a second kernel
// joins them by their maxima and sums, in order.
//
// Scores are computed transposed, S^T = K Q^T.  bf16: the K rows of a step are
// gathered so that a lane ends up with eight consecutive positions of one query
// vector, which are the B operand of O^T += V^T P^T as they stand, and the V^T
// fragments (pages hold V transposed) are plain 16-byte loads.  The weights
// enter that product as the sum of two bf16 (the second is the rounding error of
// the first, 2^-17 of the weight is lost), for which the matrix units have room;
// sums stay in fp32.  fp32: 16 positions at a time on the fp32 MFMA, whose operands have these
// layouts without a gather.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "paged.hpp"

namespace rgd {

namespace {

constexpr int kStep = 32;       // positions per step of the plan
constexpr int kMinSteps = 4;    // a wave's run is no shorter
constexpr int kMaxWaves = 2048; // 8 per CU
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;       // the running maximum moves when a score passes it by this (log2 units)
constexpr float kNoRef = -3.0e38f; // the maximum before any visible score: finite, so a masked one gives 0, never NaN

RGD_DEV int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// New tokens of sequence s.
RGD_DEV int new_tokens(const PagedAttnArgs& a, int s) { return a.n_new ? min(max(a.n_new[s], 0), a.n) : a.n; }

struct Seq {
  int len, m;   // positions, new tokens
  int steps;    // per item; at least one, so that tokens that see nothing get their zeros
  int items;    // KV heads x query tiles; 0 without new tokens
};

template <int COLS>
RGD_DEV Seq seq_of(const PagedAttnArgs& a, int s) {
  Seq q;
  q.len = paged_len(a.c, s);
  q.m = new_tokens(a, s);
  q.steps = max(1, (q.len + kStep - 1) / kStep);
  q.items = a.c.Hkv * ((q.m * (a.Hq / a.c.Hkv) + COLS - 1) / COLS);
  return q;
}

// Steps are counted in doubles (whole numbers far below 2^53).
RGD_DEV double wave_scan(double v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double t = __shfl_up(v, o, 64);
    if (lane >= o) v += t;
  }
  return v;
}

template <int COLS>
RGD_DEV double units_of(const PagedAttnArgs& a, int s) {
  if (s >= a.c.S) return 0.0;
  const Seq q = seq_of<COLS>(a, s);
  return (double)q.steps * (double)q.items;
}

// The steps of all sequences and of those before sequence `upto`.
template <int COLS>
RGD_DEV double count_units(const PagedAttnArgs& a, int upto, double& before) {
  const int lane = threadIdx.x & 63;
  double total = 0.0;
  before = 0.0;
  for (int s0 = 0; s0 < a.c.S; s0 += 64) {
    const double u = units_of<COLS>(a, s0 + lane), incl = wave_scan(u);
    if (upto >= s0 && upto < s0 + 64) before = total + __shfl(incl - u, upto - s0, 64);
    total += __shfl(incl, 63, 64);
  }
  return total;
}

// Steps per wave.
RGD_DEV double run_length(double total, int waves) { return fmax((double)kMinSteps, ceil(total / (double)waves)); }

// The sequence that holds step `at` and the steps before it.
template <int COLS>
RGD_DEV int find_seq(const PagedAttnArgs& a, double at, double& before) {
  const int lane = threadIdx.x & 63;
  double base = 0.0;
  for (int s0 = 0; s0 < a.c.S; s0 += 64) {
    const double u = units_of<COLS>(a, s0 + lane), incl = wave_scan(u);
    const unsigned long long hit = __ballot(base + incl > at);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      before = base + __shfl(incl - u, l, 64);
      return s0 + l;
    }
    base += __shfl(incl, 63, 64);
  }
  return -1;
}

RGD_DEV f32x4 mfma_bf16(const u32x4& x, const u32x4& y, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}
RGD_DEV f32x4 mfma_f32(float x, float y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, c, 0, 0, 0); }

RGD_DEV float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// The first n of the values packed in v (bf16 pairs or floats), zeros behind.
template <typename T>
RGD_DEV u32x4 keep_first(u32x4 v, int n) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (sizeof(T) == 4) v[j] = j < n ? v[j] : 0u;
    else v[j] = 2 * j + 1 < n ? v[j] : 2 * j < n ? v[j] & 0xFFFFu : 0u;
  }
  return v;
}

template <typename T>
RGD_DEV bool any_nonfinite(u32x4 v) {
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    bad = bad || (sizeof(T) == 4 ? (v[j] & 0x7F800000u) == 0x7F800000u
                                 : (v[j] & 0x7F80u) == 0x7F80u || (v[j] & 0x7F800000u) == 0x7F800000u);
  return bad;
}

// Walks a sequence's table 16 positions at a time, two times 64 entries in registers.
struct TableWalk {
  const int* row;
  int width, bpp;  // 16-position blocks per page
  int j, sub, jb, cur, nxt, lane;
  RGD_DEV void start(const PagedView& c, int s, int block) {
    row = c.pages + (size_t)s * c.width;
    width = c.width;
    bpp = c.ps >> 4;
    lane = threadIdx.x & 63;
    j = block / bpp;
    sub = block - j * bpp;
    jb = j;
    cur = row[min(jb + lane, width - 1)];
    nxt = row[min(jb + 64 + lane, width - 1)];
  }
  // the page of the next block (any value behind the table) and the block's place in it
  RGD_DEV int next(int& place) {
    if (j - jb >= 64) {
      cur = nxt;
      jb += 64;
      nxt = row[min(jb + 64 + lane, width - 1)];
    }
    const int p = __builtin_amdgcn_readlane(cur, j - jb);
    place = sub;
    if (++sub == bpp) {
      sub = 0;
      ++j;
    }
    return p;
  }
};

// D dimensions, NT tiles of 16 query vectors.
template <typename T, int D, int NT>
struct Piece {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int NB = BF ? 2 : 1;             // 16-position blocks per round
  static constexpr int KL = BF ? D / 32 : D / 16;   // 16-byte K loads per lane and block tile
  static constexpr int VL = D / 16;
  static constexpr int E = BF ? 8 : 4;              // consecutive positions of a lane
  static constexpr int COLS = 16 * NT;

  u32x4 q[NT][KL], k[NB][KL], v[VL];
  f32x4 o[NT][VL];
  float m[NT], l[NT];  // per column; l: this lane's part

  TableWalk walk;
  const char *kb[NB], *vb[NB];  // the blocks whose K is (being) loaded
  int ok;                       // bit b: block b is a page of the pool
  int lane, row, grp;

  RGD_DEV void load_k(const PagedAttnArgs& a, int g) {
    ok = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      int place;
      int p = walk.next(place);
      if (page_ok(a.c, p)) ok |= 1 << b;
      else p = 0;
      const size_t head = ((size_t)p * a.c.Hkv + g) * a.c.ps * D;
      kb[b] = (const char*)a.pool_k + (head + (size_t)place * 16 * D) * sizeof(T);
      vb[b] = (const char*)a.pool_v + (head + (size_t)place * 16) * sizeof(T);
    }
    if constexpr (BF) {
      // row r of tile e: position (r >> 2) * 8 + e * 4 + (r & 3) of the step's 32
      const char* base = row & 8 ? kb[1] : kb[0];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const char* at = base + (((row >> 2) & 1) * 8 + e * 4 + (row & 3)) * D * 2 + grp * 16;
#pragma unroll
        for (int c = 0; c < KL; ++c) k[e][c] = *(const u32x4*)(at + c * 64);
      }
    } else {
      const char* at = kb[0] + row * D * 4 + grp * 16;
#pragma unroll
      for (int c = 0; c < KL; ++c) k[0][c] = *(const u32x4*)(at + c * 64);
    }
  }

  RGD_DEV void load_v(const PagedAttnArgs& a) {
    const char* at;
    if constexpr (BF) at = (grp & 2 ? vb[1] : vb[0]) + (size_t)row * a.c.ps * 2 + (grp & 1) * 16;
    else at = vb[0] + (size_t)row * a.c.ps * 4 + grp * 16;
    const size_t step = (size_t)16 * a.c.ps * sizeof(T);
#pragma unroll
    for (int d = 0; d < VL; ++d) v[d] = *(const u32x4*)(at + d * step);
  }

  RGD_DEV void scores(f32x4 (&s)[NT][NB]) const {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < NB; ++e) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KL; ++c) {
          if constexpr (BF) {
            x = mfma_bf16(k[e][c], q[t][c], x);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x = mfma_f32(__uint_as_float(k[e][c][j]), __uint_as_float(q[t][c][j]), x);
          }
        }
        s[t][e] = x;
      }
  }

  // o[t] += V^T P^T for the given V
  RGD_DEV f32x4 weigh(const u32x4& vd, const float (&p)[E], const u32x4& hi, const u32x4& lo, f32x4 acc) const {
    if constexpr (BF) {
      acc = mfma_bf16(vd, hi, acc);
      return mfma_bf16(vd, lo, acc);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = mfma_f32(__uint_as_float(vd[j]), p[j], acc);
      return acc;
    }
  }

  // Steps [t0, t1) of one item.
  RGD_DEV void run(const PagedAttnArgs& a, const Seq& sq, int s, int g, int qb, int t0, int t1) {
    lane = threadIdx.x & 63;
    row = lane & 15;
    grp = lane >> 4;
    const int G = a.Hq / a.c.Hkv, cols = sq.m * G;
    walk.start(a.c, s, t0 * 2);
    // the tile's queries; columns behind the last one repeat it
    int lim[NT], least = 0x7FFFFFFF;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int col = min(qb * COLS + t * 16 + row, cols - 1), i = col / G;
      lim[t] = sq.len - sq.m + i + 1;
      const T* src = (const T*)a.q + ((size_t)s * a.n + i) * a.ldq + (size_t)(g * G + col - i * G) * D;
#pragma unroll
      for (int c = 0; c < KL; ++c) q[t][c] = *(const u32x4*)((const char*)src + c * 64 + grp * 16);
      m[t] = kNoRef;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < VL; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int first = (qb * COLS) / G;  // the tile's first token: all its columns see that much
    least = sq.len - sq.m + first + 1;
    const float scale = kLog2e / sqrtf((float)D);
    constexpr int PER = 16 * NB;
    const int p1 = min(t1 * kStep, max(sq.len, 1));
    int p0 = t0 * kStep;
    load_k(a, g);
    load_v(a);
    for (; p0 < p1; p0 += PER) {
      const int here = ok;
      f32x4 s4[NT][NB];
      scores(s4);
      const bool more = p0 + PER < p1;
      if (more) load_k(a, g);
      const bool whole = p0 + PER <= least && here == (1 << NB) - 1;
      const int pos = p0 + grp * E;  // of this lane's first score
      const bool there = BF ? (here >> (grp >> 1)) & 1 : here & 1;
      bool mixed = false;  // a position that some of the tile's tokens see and others do not is not finite
      if (!whole) {
        const int held = there ? sq.len - pos : 0;
        bool odd = false;
#pragma unroll
        for (int d = 0; d < VL; ++d) {
          v[d] = keep_first<T>(v[d], held);
          odd = odd || any_nonfinite<T>(v[d]);
        }
        mixed = __any(odd);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float x[E];
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] = s4[t][j / 4][j % 4] * scale;
        if (!whole) {
          const int seen = there ? lim[t] - pos : 0;
#pragma unroll
          for (int j = 0; j < E; ++j) x[j] = j < seen ? x[j] : -INFINITY;
        }
        float top = x[0];
#pragma unroll
        for (int j = 1; j < E; ++j) top = fmaxf(top, x[j]);
        if (__any(top > m[t] + kLazy)) {
          top = fmaxf(top, __shfl_xor(top, 16, 64));
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float nm = fmaxf(m[t], top), down = exp2_raw(m[t] - nm);
          m[t] = nm;
          l[t] *= down;
#pragma unroll
          for (int d = 0; d < VL; ++d) o[t][d] *= down;
        }
        float p[E];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) {
          p[j] = exp2_raw(x[j] - m[t]);
          sum += p[j];
        }
        l[t] += sum;
        u32x4 hi{}, lo{};
        if constexpr (BF) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            hi[j] = pack_bf16x2(p[2 * j], p[2 * j + 1]);
            lo[j] = pack_bf16x2(p[2 * j] - __uint_as_float(hi[j] << 16),
                                p[2 * j + 1] - __uint_as_float(hi[j] & 0xFFFF0000u));
          }
        }
        if (!mixed) {
#pragma unroll
          for (int d = 0; d < VL; ++d) o[t][d] = weigh(v[d], p, hi, lo, o[t][d]);
        } else {
          // 0 times such a value is not 0: each token's columns take the product with what it sees
          const int c0 = qb * COLS + t * 16, c1 = min(c0 + 16, cols) - 1;
          for (int i = min(c0, cols - 1) / G; i <= max(c1, 0) / G; ++i) {
            const int see = sq.len - sq.m + i + 1;
            const int n = there ? see - pos : 0;
#pragma unroll
            for (int d = 0; d < VL; ++d) {
              const f32x4 r = weigh(keep_first<T>(v[d], n), p, hi, lo, o[t][d]);
              if (lim[t] == see) o[t][d] = r;
            }
          }
        }
      }
      if (more) load_v(a);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      l[t] += __shfl_xor(l[t], 16, 64);
      l[t] += __shfl_xor(l[t], 32, 64);
    }
  }
};

RGD_DEV float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2; }

template <typename T>
RGD_DEV void store_row4(T* p, f32x4 v) {
  if constexpr (sizeof(T) == 2) *(u32x2*)p = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *(f32x4*)p = v;
}

// Pieces: slot 2 w + 1 holds the start of the item that wave w's run ends in, slot 2 w the
// part of an item that an earlier run began.  Per slot [COLS][D] weighted sums,
// then [COLS] (maximum, sum).
template <int D, int NT>
constexpr size_t slot_floats() {
  return (size_t)16 * NT * (D + 2);
}

template <typename T, int D, int NT>
__global__ __launch_bounds__(256, NT == 1 ? 2 : 1) void attn_run_kernel(PagedAttnArgs a, int waves) {
  using P = Piece<T, D, NT>;
  constexpr int COLS = P::COLS;
  const int w = uniform(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (w >= waves) return;
  const int lane = threadIdx.x & 63, row = lane & 15, grp = lane >> 4;
  double unused;
  const double total = count_units<COLS>(a, -1, unused);
  const double run = run_length(total, waves), start = (double)w * run;
  if (start >= total) return;
  double before = 0.0;
  int s = uniform(find_seq<COLS>(a, start, before));
  long long left = (long long)fmin(run, total - start);
  Seq sq = seq_of<COLS>(a, s);
  sq = Seq{uniform(sq.len), uniform(sq.m), uniform(sq.steps), uniform(sq.items)};
  const double inside = start - before;
  int item = uniform((int)(inside / (double)sq.steps));
  int t0 = uniform((int)(inside - (double)item * (double)sq.steps));
  const int G = a.Hq / a.c.Hkv;
  while (left > 0) {
    const int t1 = (int)min((long long)sq.steps, t0 + left), tiles = sq.items / a.c.Hkv;
    const int g = item / tiles, qb = item - g * tiles;
    P x;
    x.run(a, sq, s, g, qb, t0, t1);
    const bool done = t0 == 0 && t1 == sq.steps;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int col = qb * COLS + t * 16 + row;
      if (col >= sq.m * G) continue;
      if (done) {
        const size_t r = (size_t)s * a.n + col / G;
        const int h = g * G + col % G;
        const float inv = x.l[t] == 0.f ? 0.f : 1.f / x.l[t];
        T* out = (T*)a.out + (r * a.Hq + h) * D + grp * 4;
#pragma unroll
        for (int d = 0; d < P::VL; ++d) store_row4(out + d * 16, x.o[t][d] * inv);
        if (a.lse && grp == 0) a.lse[r * a.Hq + h] = lse_of(x.m[t], x.l[t]);
      } else {
        float* slot = a.ws + (size_t)(2 * w + (t0 == 0)) * slot_floats<D, NT>();
        const int c = t * 16 + row;
#pragma unroll
        for (int d = 0; d < P::VL; ++d) *(f32x4*)(slot + c * D + d * 16 + grp * 4) = x.o[t][d];
        if (grp == 0) *(float2*)(slot + COLS * D + 2 * c) = float2{x.m[t], x.l[t]};
      }
    }
    left -= t1 - t0;
    t0 = 0;
    if (left > 0 && ++item == sq.items) {
      item = 0;
      do {
        ++s;
        sq = seq_of<COLS>(a, s);  // steps are left, so a sequence with new tokens follows
        sq = Seq{uniform(sq.len), uniform(sq.m), uniform(sq.steps), uniform(sq.items)};
      } while (sq.items == 0);
    }
  }
}

// The outputs of the items that several runs share: one workgroup per (row,
// query head); each group of D threads sums every (256 / D)-th piece.
template <typename T, int D, int NT>
__global__ __launch_bounds__(256) void attn_join_kernel(PagedAttnArgs a, int waves) {
  constexpr int COLS = 16 * NT, PARTS = 256 / D;
  __shared__ float acc_s[256], top_s[4], sum_s[256];
  const int r = blockIdx.x, h = blockIdx.y, s = r / a.n, i = r - s * a.n;
  const Seq sq = seq_of<COLS>(a, s);
  if (i >= sq.m) return;
  const int G = a.Hq / a.c.Hkv, g = h / G, col = i * G + h - g * G, qb = col / COLS, c = col - qb * COLS;
  double before;
  const double total = count_units<COLS>(a, s, before);
  const double run = run_length(total, waves);
  const double from = before + (double)(g * (sq.items / a.c.Hkv) + qb) * (double)sq.steps;
  const int w0 = (int)(from / run), w1 = (int)((from + (double)sq.steps - 1.0) / run);
  if (w0 == w1) return;
  auto slot = [&](int w) { return a.ws + (size_t)(2 * w + (w == w0)) * slot_floats<D, NT>(); };
  const int t = threadIdx.x;
  float top = kNoRef;
  for (int w = w0 + t; w <= w1; w += 256) top = fmaxf(top, slot(w)[COLS * D + 2 * c]);
  top = block_max_once(top, top_s);
  const int d = t % D, part = t / D;
  float acc = 0.f, sum = 0.f;
#pragma unroll 8
  for (int w = w0 + part; w <= w1; w += PARTS) {
    const float* p = slot(w);
    const float f = exp2_raw(p[COLS * D + 2 * c] - top);
    acc += f * p[c * D + d];
    sum += f * p[COLS * D + 2 * c + 1];
  }
  acc_s[t] = acc;
  sum_s[t] = sum;
  __syncthreads();
  if (t >= D) return;
#pragma unroll
  for (int k = 1; k < PARTS; ++k) {
    acc += acc_s[k * D + t];
    sum += sum_s[k * D + t];
  }
  store_f((T*)a.out + ((size_t)r * a.Hq + h) * D + t, sum == 0.f ? 0.f : acc / sum);
  if (t == 0 && a.lse) a.lse[(size_t)r * a.Hq + h] = lse_of(top, sum);
}

// Query tiles a wave holds at once: all of a sequence's query vectors up to 64.
int tiles_for(int vectors) { return vectors <= 16 ? 1 : vectors <= 32 ? 2 : 4; }

int waves_for(const PagedView& c, int n, int Hq) {
  const int cols = 16 * tiles_for(n * (Hq / c.Hkv));
  const double items = (double)c.S * c.Hkv * ((n * (Hq / c.Hkv) + cols - 1) / cols);
  const double steps = items * std::max(1.0, std::ceil((double)c.width * c.ps / kStep));
  return (int)std::min((double)kMaxWaves, std::ceil(steps / kMinSteps));
}

template <typename T, int D, int NT>
hipError_t launch(const PagedAttnArgs& a, hipStream_t s) {
  const int waves = waves_for(a.c, a.n, a.Hq);
  hipLaunchKernelGGL((attn_run_kernel<T, D, NT>), dim3((waves + 3) / 4), dim3(256), 0, s, a, waves);
  if (hipError_t e = hipGetLastError()) return e;
  hipLaunchKernelGGL((attn_join_kernel<T, D, NT>), dim3(a.c.S * a.n, a.Hq), dim3(256), 0, s, a, waves);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_tiles(const PagedAttnArgs& a, hipStream_t s) {
  switch (tiles_for(a.n * (a.Hq / a.c.Hkv))) {
    case 1: return launch<T, D, 1>(a, s);
    case 2: return launch<T, D, 2>(a, s);
    default: return launch<T, D, 4>(a, s);
  }
}

template <typename T>
hipError_t launch_dim(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.c.D) {
    case 32: return launch_tiles<T, 32>(a, s);
    case 64: return launch_tiles<T, 64>(a, s);
    default: return launch_tiles<T, 128>(a, s);
  }
}

}  // namespace

size_t paged_attention_workspace_floats(const PagedView& c, int n, int Hq) {
  const int nt = tiles_for(n * (Hq / c.Hkv));
  return (size_t)2 * waves_for(c, n, Hq) * 16 * nt * (c.D + 2);
}

hipError_t paged_attention(const PagedAttnArgs& a, hipStream_t s) {
  return a.c.esz == 2 ? launch_dim<bf16_t>(a, s) : launch_dim<float>(a, s);
}

}  // namespace rgd
