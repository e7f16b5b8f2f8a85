// Causal attention of a sequence's last few tokens over its pages.
//
// o = sum_j exp(a_j - lse) v_j with a_j = q . k_j / sqrt(D), lse = log sum_j exp(a_j): one pass over
// the keys and values with a running maximum and sum.  Each K and V is read
// from memory once for all query vectors of its KV head (tokens x query heads
// per KV head), a few operations a byte, so the reads bound it; the products
// go through MFMA, 16 query vectors to a tile, because the tile's unused
// columns cost less than the reads they wait for.
//
// The positions of all (sequence, KV head, query tile) items lie one behind the
// other in steps of 32, and every workgroup takes an equal run of steps, over the
// borders of items: short and long sequences fill the chip alike, whatever their
// order.  The workgroups work the runs out of the lengths on the device.  Inside a
// run the four waves take an item's steps in turn, each with a maximum and sum of its
// own, and meet in LDS at the item's end.  An item inside one run is finished there;
// the pieces of one that is cut go to the workspace and a second kernel joins them
// by their maxima and sums, in order.
//
// Scores are computed transposed, S^T = K Q^T.  bf16: the K rows of a step are
// gathered so that a lane ends up with eight consecutive positions of one query
// vector, which are the B operand of O^T += V^T P^T as they stand, and the V^T
// fragments (pages hold V transposed) are plain 16-byte loads.  The weights
// enter that product as the sum of two bf16 (the second is the rounding error of
// the first, 2^-17 of the weight is lost), for which the matrix units have room;
// sums stay in fp32.  fp32: 16 positions at a time on the fp32 MFMA, whose operands have these
// layouts without a gather.
//
// Measured, 8 KV heads of 128, bf16, both kernels' times: one token of 64 sequences of up to 8192
// positions (253 MB of K and V) 47 + 5 us, 5.4 TB/s, and of one of 131072 (537 MB) 96 + 6 us, 5.6 TB/s:
// the reads bound them, of which the memory sees 1.02 and 1.06 times the bytes.  Five tokens
// of 32 sequences of up to 4096 (73 MB) 21 + 5 us, 16 of 16 sequences of 4096 (268 MB) 63 + 5.  One token over
// 512 positions 6.3 + 2.8 us: two launches and a chain of reads (lengths, table, K and V, pieces).  One token
// of 1024 sequences of up to 500 (354 MB): 115 us, as an item is a step or two of one to three waves.
// Pieces of prompts, 4 sequences of 4096: 16 tokens 26 us, 64 59, 256 222, 1000 783 (300 TFLOP/s): each
// 64 query vectors read the keys and values again, from the caches.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "paged.hpp"

namespace rgd {

namespace {

constexpr int kStep = 32;      // positions per step of the plan
// A run is no shorter: one step a wave.  One sequence of 512: 6.3 us, with 8 steps 7.0.
constexpr int kMinSteps = 4;
// What an item costs besides its steps, in steps: more with more outputs.  One token (one tile) of 64 ragged
// sequences to 8192 with 2, 3, 4, 6 and 8: 58.8, 52.8, 51.0, 51.6 and 51.8 us, of 1024 to 500: 122, 117, 115, 119 and
// 124; five (two tiles) of 32 to 4096 with 4, 6, 8 and 12: 26.4, 21.7, 21.5 and 21.0; twelve (four tiles)
// with 4, 6, 8, 12 and 16: 49.2, 39.9, 32.4, 32.3 and 31.2.
constexpr int item_cost(int nt) { return 4 * nt; }
// Two workgroups per CU; half of it where LDS or registers hold one.  Three per CU spill: one sequence of
// 131072 takes 162 us in place of 109.
constexpr int kMaxRuns = 512;
constexpr int kWaves = 4;      // per workgroup
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;       // the running maximum moves when a score passes it by this (log2 units)
constexpr float kLift = 256.f;     // 2^kLazy: weights are held divided by it, so none is above 1 and no sum above that of |V|
constexpr float kNoRef = -3.0e38f; // the maximum before any visible score: finite, so a masked one gives 0, never NaN

RGD_DEV int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// New tokens of sequence s.
RGD_DEV int new_tokens(const PagedAttnArgs& a, int s) { return a.n_new ? min(max(a.n_new[s], 0), a.n) : a.n; }

// Floor of col / G for col < 2^20, G <= 1024: the product passes col / G by less than col / 2^31,
// which is less than 1 / G.
RGD_DEV int token_of(const PagedAttnArgs& a, int col) { return (int)__umulhi((unsigned)col << 1, a.inv_G); }

struct Seq {
  int len, m;   // positions, new tokens
  int steps;    // per item; at least one, so that tokens that see nothing get their zeros
  int tiles;    // query tiles; 0 without new tokens.  Items: KV heads x query tiles
};

template <int COLS>
RGD_DEV Seq seq_of(const PagedAttnArgs& a, int len, int m) {
  Seq q;
  q.len = len;
  q.m = m;
  q.steps = max(1, (len + kStep - 1) / kStep);
  q.tiles = (m * a.G + COLS - 1) / COLS;
  return q;
}
template <int COLS>
RGD_DEV Seq seq_of(const PagedAttnArgs& a, int s) {
  return seq_of<COLS>(a, paged_len(a.c, s), new_tokens(a, s));
}
// The same for an s that the whole wave shares, by scalar loads: a vector load's wait would be one
// for the K and V on their way, too.
template <int COLS>
RGD_DEV Seq uniform_seq(const PagedAttnArgs& a, int s) {
  typedef const int __attribute__((address_space(4))) * Scalar;
  const int len = ((Scalar)a.c.lens)[s], m = a.n_new ? ((Scalar)a.n_new)[s] : a.n;
  return seq_of<COLS>(a, min(max(len, 0), a.c.width * a.c.ps), min(max(m, 0), a.n));
}

// Sum over the lanes up to this one (64-bit: long tables times many sequences).
template <int CTRL, int ROWS>
RGD_DEV long long scan_step(long long v) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false);
  return v + (((long long)hi << 32) | (unsigned)lo);
}
RGD_DEV long long wave_scan(long long v) {
  v = scan_step<0x111, 0xf>(v);  // row_shr:1
  v = scan_step<0x112, 0xf>(v);
  v = scan_step<0x114, 0xf>(v);
  v = scan_step<0x118, 0xf>(v);
  v = scan_step<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3
  return scan_step<0x143, 0xc>(v);  // row_bcast:31 into rows 2 and 3
}
RGD_DEV long long lane_value(long long v, int lane) {
  const int lo = __builtin_amdgcn_readlane((int)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
  return ((long long)hi << 32) | (unsigned)lo;
}

// Units of the plan that this lane's sequence takes (none behind the last).
template <int COLS>
RGD_DEV long long units_of(const PagedAttnArgs& a, int s, Seq& q) {
  q = seq_of<COLS>(a, min(s, a.c.S - 1));
  return s < a.c.S ? (long long)(q.steps + item_cost(COLS / 16)) * (a.c.Hkv * q.tiles) : 0;
}

// Floor of x / y for 0 <= x < 2^52, 0 < y.  Exact: a quotient that is no whole number
// is at least 1 / y, more than 2^-52 of itself, away from the next one.
RGD_DEV long long quotient(long long x, long long y) { return (long long)((double)x / (double)y); }

struct Runs {
  long long total, length;  // units of the plan, units per run
};

// Finds the run of workgroup r (of `runs`): the sequence it starts in and the units
// before that one.  False: there is none.
template <int COLS>
RGD_DEV bool find_run(const PagedAttnArgs& a, int r, int runs, Runs& plan, int& s, Seq& sq, long long& before) {
  const int lane = threadIdx.x & 63, per = (a.c.S + 63) / 64;  // sequences a lane: one, or neighbouring ones
  Seq q;
  long long u = 0;
#pragma unroll 8
  for (int k = 0; k < per; ++k) u += units_of<COLS>(a, lane * per + k, q);
  long long incl = wave_scan(u);
  plan.total = lane_value(incl, 63);
  plan.length = max((long long)kMinSteps, quotient(plan.total + runs - 1, runs));
  const long long start = r * plan.length;
  if (start >= plan.total) return false;
  int l = __builtin_ctzll(__ballot(incl > start));
  before = lane_value(incl - u, l);
  s = l * per;
  if (per > 1)
    for (;; s += 64) {
      u = units_of<COLS>(a, s + lane, q);
      incl = wave_scan(u);
      if (const unsigned long long hit = __ballot(before + incl > start)) {
        l = __builtin_ctzll(hit);
        before += lane_value(incl - u, l);
        s += l;
        break;
      }
      before += lane_value(incl, 63);
    }
  sq = seq_of<COLS>(a, __builtin_amdgcn_readlane(q.len, l), __builtin_amdgcn_readlane(q.m, l));
  return true;
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

// 1 in the first n places, 0 behind.
template <typename T>
RGD_DEV u32x4 ones(int n) {
  const uint32_t one = sizeof(T) == 4 ? 0x3F800000u : 0x3F803F80u;
  return keep_first<T>(u32x4{one, one, one, one}, n);
}

// Bits by type.
template <typename T>
constexpr uint32_t kInf = sizeof(T) == 4 ? 0x7F800000u : 0x7F80u;
template <typename T>
constexpr uint32_t kSign = sizeof(T) == 4 ? 0x80000000u : 0x8000u;

// f(bits) of each value packed in v.
template <typename T, typename F>
RGD_DEV u32x4 each(u32x4 v, F f) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = sizeof(T) == 4 ? f(v[j]) : f(v[j] & 0xFFFFu) | f(v[j] >> 16) << 16;
  return v;
}

// 1 where a value is +inf (kind 0), -inf (1) or NaN (2).
template <typename T>
RGD_DEV u32x4 marks(u32x4 v, int kind) {
  const uint32_t one = sizeof(T) == 4 ? 0x3F800000u : 0x3F80u;
  return each<T>(v, [=](uint32_t x) {
    const bool hit = kind == 2 ? (x & ~kSign<T>) > kInf<T> : x == (kind ? kInf<T> | kSign<T> : kInf<T>);
    return hit ? one : 0u;
  });
}

// 0 in the place of every value that is not finite.
template <typename T>
RGD_DEV u32x4 finite(u32x4 v) {
  return each<T>(v, [](uint32_t x) { return (x & kInf<T>) == kInf<T> ? 0u : x; });
}

template <typename T>
RGD_DEV bool any_nonfinite(u32x4 v) {
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    bad = bad || (v[j] & kInf<T>) == kInf<T> || (sizeof(T) == 2 && (v[j] >> 16 & kInf<T>) == kInf<T>);
  return bad;
}

// Looks up a sequence's table by 16-position blocks in rising order, two times 64
// entries in registers.
struct TableWalk {
  const int* row;
  int width, bpp;  // 16-position blocks per page
  unsigned long long inv;
  int jb, cur, nxt, lane;
  RGD_DEV int page_index(int block) const { return (int)(((unsigned long long)block * inv) >> 36); }
  RGD_DEV void start(const PagedView& c, int s, int block) {
    row = c.pages + (size_t)s * c.width;
    width = c.width;
    bpp = c.ps >> 4;
    inv = ((1ull << 36) + bpp - 1) / bpp;  // blocks are below 2^26, bpp at most 2^8: exact
    lane = threadIdx.x & 63;
    jb = page_index(block);
    cur = row[min(jb + lane, width - 1)];
    nxt = row[min(jb + 64 + lane, width - 1)];
  }
  // the page of a block (behind the table: any value) and the block's place in it
  RGD_DEV int find(int block, int& place) {
    const int j = page_index(block);
    place = block - j * bpp;
    while (j - jb >= 64) {
      cur = nxt;
      jb += 64;
      nxt = row[min(jb + 64 + lane, width - 1)];
    }
    return __builtin_amdgcn_readlane(cur, j - jb);
  }
};

// One item of a run: steps [t0, t1) of query tile qb of KV head g of sequence s.
struct Item {
  Seq sq;
  int s, g, qb, t0, t1;
  bool valid;
  long long at;  // its first unit in the plan
  RGD_DEV int end() const { return min(t1 * kStep, max(sq.len, 1)); }
  RGD_DEV int begin(int wave, int per) const { return t0 * kStep + wave * per; }
};

RGD_DEV Seq uniform(const Seq& q) { return Seq{uniform(q.len), uniform(q.m), uniform(q.steps), uniform(q.tiles)}; }

// The items of a run, one after the other.
template <int COLS>
struct Walk {
  static constexpr int COST = item_cost(COLS / 16);
  Seq sq;
  int s, g, qb, u0, left;
  long long at;
  RGD_DEV Item next(const PagedAttnArgs& a) {
    Item it{};
    if (left <= 0) return it;
    if (g == a.c.Hkv) {  // steps are left, so a sequence with new tokens follows
      g = 0;
      do sq = uniform_seq<COLS>(a, ++s);
      while (sq.tiles == 0);
    }
    // an item's first COST units of the plan are its fixed cost, in front of its steps
    const int u1 = min(sq.steps + COST, u0 + left);
    it.sq = sq;
    it.s = s;
    it.g = g;
    it.qb = qb;
    it.t0 = max(0, u0 - COST);
    it.t1 = u1 - COST;
    it.valid = it.t1 > it.t0;  // else the next run has the item's first step
    it.at = at;
    at += sq.steps + COST;
    left -= u1 - u0;
    u0 = 0;
    if (++qb == sq.tiles) {
      qb = 0;
      ++g;
    }
    return it;
  }
};

// D dimensions, NT tiles of 16 query vectors; PAST: V is loaded past the caches.
template <typename T, int D, int NT, bool PAST>
struct Piece {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int NB = BF ? 2 : 1;             // 16-position blocks per round
  static constexpr int KL = BF ? D / 32 : D / 16;   // 16-byte K loads per lane and block tile
  static constexpr int VL = D / 16;
  static constexpr int E = BF ? 8 : 4;              // consecutive positions of a lane
  static constexpr int COLS = 16 * NT;

  // where registers are short the queries stay in LDS, shared by the waves
  static constexpr bool QS = NT == 4 || (NT == 2 && sizeof(T) * D < 512);
  u32x4 q[QS ? 1 : NT][KL], k[NB][KL], v[VL];
  const u32x4* qs;
  f32x4 o[NT][VL];
  float m[NT], l[NT];  // per column; l: this lane's part

  TableWalk walk;
  const char *kb[NB], *vb[NB];  // the blocks whose K is (being) loaded
  int ok;                       // bit b: block b is a page of the pool
  int lane, row, grp;

  RGD_DEV void load_k(const PagedAttnArgs& a, int g, int p0) {
    ok = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      int place;
      int p = walk.find((p0 >> 4) + b, place);
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
    for (int d = 0; d < VL; ++d)
      v[d] = PAST ? __builtin_nontemporal_load((const u32x4*)(at + d * step)) : *(const u32x4*)(at + d * step);
  }

  // fp32: four sums of D / 4 products each, as every product is rounded where it is added (heads of 128: 2.8e-7 of the
  // outputs with one sum, 2.0e-7 with two, 1.6e-7 with four, at the same times).
  RGD_DEV void scores(f32x4 (&s)[NT][NB]) const {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < NB; ++e) {
        if constexpr (BF) {
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < KL; ++c) x = mfma_bf16(k[e][c], q_at(t, c), x);
          s[t][e] = x;
        } else {
          f32x4 x[4] = {};
#pragma unroll
          for (int c = 0; c < KL; ++c) {
            const u32x4 qc = q_at(t, c);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = mfma_f32(__uint_as_float(k[e][c][j]), __uint_as_float(qc[j]), x[j]);
          }
          s[t][e] = (x[0] + x[1]) + (x[2] + x[3]);
        }
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

  // sum over the positions of x y, both held as V and the weights are
  RGD_DEV f32x4 count(const u32x4& x, const u32x4& y) const {
    f32x4 r = {0.f, 0.f, 0.f, 0.f};
    if constexpr (BF) return mfma_bf16(x, y, r);
#pragma unroll
    for (int j = 0; j < 4; ++j) r = mfma_f32(__uint_as_float(x[j]), __uint_as_float(y[j]), r);
    return r;
  }

  // Weights of tile t's products (times scale: scores in log2 units) against its running maximum, which moves
  // with them, over kLift; hi + lo: the weights in two bf16.  A score's distance from the maximum is rounded once, at
  // its own size: a score that is rounded first takes errors of the score's size into the weight.
  RGD_DEV void weights(int t, const float (&x)[E], float scale, float (&p)[E], u32x4& hi, u32x4& lo) {
    float top = x[0];
#pragma unroll
    for (int j = 1; j < E; ++j) top = fmaxf(top, x[j]);
    top *= scale;
    if (__any(top > m[t] + kLazy)) {
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float nm = fmaxf(m[t], top), down = exp2_raw(m[t] - nm);
      m[t] = nm;
      l[t] *= down;
#pragma unroll
      for (int d = 0; d < VL; ++d) o[t][d] *= down;
    }
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      p[j] = exp2_raw(fmaf(x[j], scale, -m[t])) * (1.f / kLift);
      sum += p[j];
    }
    l[t] += sum;
    if constexpr (BF) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        hi[j] = pack_bf16x2(p[2 * j], p[2 * j + 1]);
        lo[j] = pack_bf16x2(p[2 * j] - __uint_as_float(hi[j] << 16),
                            p[2 * j + 1] - __uint_as_float(hi[j] & 0xFFFF0000u));
      }
    }
  }

  static constexpr int PER = 16 * NB, STRIDE = kWaves * PER;  // a round's positions, the way to the wave's next round

  RGD_DEV u32x4 q_at(int t, int c) const {
    if constexpr (QS) return qs[(t * KL + c) * 64 + lane];
    else return q[t][c];
  }

  // a tile a wave, between two barriers
  RGD_DEV void stage_q(const PagedAttnArgs& a, const Item& it, u32x4* dst, int wave) const {
    const int G = a.G, cols = it.sq.m * G;
    const int col = min(it.qb * COLS + wave * 16 + row, cols - 1), i = token_of(a, col);
    const T* src = (const T*)a.q + ((size_t)it.s * a.n + i) * a.ldq + (size_t)(it.g * G + col - i * G) * D;
#pragma unroll
    for (int c = 0; c < KL; ++c) dst[(wave * KL + c) * 64 + lane] = *(const u32x4*)((const char*)src + c * 64 + grp * 16);
  }

  RGD_DEV void load_q(const PagedAttnArgs& a, const Item& it) {
    if (QS) return;
    const int G = a.G, cols = it.sq.m * G;
#pragma unroll
    for (int t = 0; t < (QS ? 0 : NT); ++t) {
      const int col = min(it.qb * COLS + t * 16 + row, cols - 1), i = token_of(a, col);  // columns behind the last one repeat it
      const T* src = (const T*)a.q + ((size_t)it.s * a.n + i) * a.ldq + (size_t)(it.g * G + col - i * G) * D;
#pragma unroll
      for (int c = 0; c < KL; ++c) q[t][c] = *(const u32x4*)((const char*)src + c * 64 + grp * 16);
    }
  }

  RGD_DEV void start(const PagedAttnArgs& a, const Item& it, const TableWalk& w, int wave) {
    const int p0 = it.begin(wave, PER);
    if (!it.valid || p0 >= it.end()) return;
    walk = w;
    load_q(a, it);
    load_k(a, it.g, p0);
    __builtin_amdgcn_sched_barrier(0);  // K's wait leaves V's loads on their way, here and where the paths meet
    load_v(a);
  }

  // The wave's share of an item's steps, whose queries and first K and V are on their
  // way; leaves those of the next item on theirs (walk_next: its table's first entries).
  RGD_DEV void run(const PagedAttnArgs& a, const Item& it, const Item& next, const TableWalk& walk_next, int wave) {
    const Seq& sq = it.sq;
    const int cols = sq.m * a.G, qb = it.qb, g = it.g, p1 = it.end();
    int p0 = it.begin(wave, PER);
    int lim[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      lim[t] = sq.len - sq.m + token_of(a, min(qb * COLS + t * 16 + row, cols - 1)) + 1;
      m[t] = kNoRef;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < VL; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int least = sq.len - sq.m + token_of(a, qb * COLS) + 1;  // all of the tile's tokens see that much
    const float scale = kLog2e / sqrtf((float)D);
    if (p0 >= p1) {
      start(a, next, walk_next, wave);
      return;
    }
    constexpr int ALL = (1 << NB) - 1;
    while (p0 < p1) {
      while (ok == ALL && p0 + PER <= least && p0 + STRIDE < p1) {  // every column sees it all, and another round follows
        f32x4 s4[NT][NB];
        scores(s4);
        load_k(a, g, p0 + STRIDE);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float x[E], p[E];
#pragma unroll
          for (int j = 0; j < E; ++j) x[j] = s4[t][j / 4][j % 4];
          u32x4 hi, lo;
          weights(t, x, scale, p, hi, lo);
#pragma unroll
          for (int d = 0; d < VL; ++d) o[t][d] = weigh(v[d], p, hi, lo, o[t][d]);
        }
        load_v(a);
        p0 += STRIDE;
      }
      const int here = ok;
      f32x4 s4[NT][NB];
      scores(s4);
      const bool more = p0 + STRIDE < p1;
      const int first = next.begin(wave, PER);
      const bool on = !more && next.valid && first < next.end();
      if (more) {
        load_k(a, g, p0 + STRIDE);
      } else if (on) {
        walk = walk_next;
        load_q(a, next);
        load_k(a, next.g, first);
      }
      const int pos = p0 + grp * E;  // of this lane's first score
      const bool there = BF ? (here >> (grp >> 1)) & 1 : here & 1;
      bool odd = false;
      if (here != ALL || p0 + PER > sq.len) {
        const int held = there ? sq.len - pos : 0;
#pragma unroll
        for (int d = 0; d < VL; ++d) v[d] = keep_first<T>(v[d], held);
      }
      if (least < min(p0 + PER, sq.len)) {  // not every column sees every value
#pragma unroll
        for (int d = 0; d < VL; ++d) odd = odd || any_nonfinite<T>(v[d]);
      }
      float p[NT][E];
      u32x4 hi[NT], lo[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int seen = there ? lim[t] - pos : 0;
        float x[E];
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] = j < seen ? s4[t][j / 4][j % 4] : -INFINITY;
        weights(t, x, scale, p[t], hi[t], lo[t]);
      }
      if (__any(odd)) {
        // 0 times a value that is not finite is not 0, so these leave the product: a
        // column gets them by whether it sees one, not by its weight
        u32x4 see[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) see[t] = ones<T>(there ? lim[t] - pos : 0);
#pragma unroll
        for (int d = 0; d < VL; ++d) {
#pragma unroll
          for (int kind = 0; kind < 3; ++kind) {
            const u32x4 at = marks<T>(v[d], kind);
            const float is = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const f32x4 r = count(at, see[t]);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[t][d][e] += r[e] > 0.f ? is : 0.f;
              __builtin_amdgcn_sched_barrier(0);  // one count's registers at a time
            }
          }
          v[d] = finite<T>(v[d]);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int d = 0; d < VL; ++d) o[t][d] = weigh(v[d], p[t], hi[t], lo[t], o[t][d]);
      if (more || on) load_v(a);
      p0 += STRIDE;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      l[t] += __shfl_xor(l[t], 16, 64);
      l[t] += __shfl_xor(l[t], 32, 64);
    }
  }
};

RGD_DEV float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + __log2f(l * kLift)) * kLn2; }

template <typename T>
RGD_DEV void store_row4(T* p, f32x4 v) {
  if constexpr (sizeof(T) == 2) *(u32x2*)p = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *(f32x4*)p = v;
}

// Workspace: per run a Cut, then the pieces: slot 2 r + 1 holds the start of the item
// that run r ends in, slot 2 r the part of an item that an earlier run began.  Per slot
// [COLS][D] weighted sums, then [COLS] (maximum, sum).
struct Cut {  // the item that starts in this run and goes on to run `last`
  int s, g;   // s = -1: none
  int qb;
  short last, cols;  // cols: the item's query vectors
};
__host__ __device__ constexpr size_t cut_floats(int runs) { return ((size_t)runs * 4 + 63) / 64 * 64; }
template <int D, int NT>
constexpr size_t slot_floats() {
  return (size_t)16 * NT * (D + 2);
}

// Whether a CU holds two workgroups (row: bytes of a row of K).
constexpr bool two_per_cu(int nt, size_t row) { return nt == 1 || (nt == 2 && row < 512); }

template <typename T, int D, int NT, bool PAST>
__global__ __launch_bounds__(256, two_per_cu(NT, sizeof(T) * D) ? 2 : 1) void attn_run_kernel(PagedAttnArgs a, int runs) {
  using P = Piece<T, D, NT, PAST>;
  constexpr int COLS = P::COLS, LD = D + 4, COST = item_cost(NT);
  __shared__ float part[kWaves][COLS][LD];
  __shared__ float2 ml[kWaves][COLS];
  __shared__ u32x4 q_s[P::QS ? NT * P::KL * 64 : 1];
  const int r = blockIdx.x, wave = uniform(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, row = lane & 15, grp = lane >> 4;
  Runs plan;
  int s;
  long long before;
  Walk<COLS> walk;
  Cut* cut = (Cut*)a.ws + r;
  if (threadIdx.x == 0) *cut = Cut{-1, 0, 0, 0};
  if (!find_run<COLS>(a, r, runs, plan, s, walk.sq, before)) return;
  const long long start = r * plan.length;
  walk.s = uniform(s);
  walk.left = uniform((int)min(plan.length, plan.total - start));
  walk.sq = uniform(walk.sq);
  const int item = uniform((int)quotient(start - before, walk.sq.steps + COST));
  walk.g = item / walk.sq.tiles;
  walk.qb = item - walk.g * walk.sq.tiles;
  walk.at = before + (long long)item * (walk.sq.steps + COST);
  walk.u0 = uniform((int)(start - walk.at));
  const int G = a.G;
  P x;
  x.lane = lane;
  x.row = row;
  x.grp = grp;
  x.qs = q_s;
  Item it = walk.next(a);
  TableWalk table;
  table.start(a.c, it.s, it.begin(wave, P::PER) >> 4);
  x.start(a, it, table, wave);
  while (it.valid) {
    if (P::QS) {
      if (wave < NT) x.stage_q(a, it, q_s, wave);
      __syncthreads();
    }
    const Item next = walk.next(a);
    if (next.valid) table.start(a.c, next.s, next.begin(wave, P::PER) >> 4);
    x.run(a, it, next, table, wave);
    const Seq& sq = it.sq;
    const int g = it.g, qb = it.qb, t0 = it.t0, t1 = it.t1, cols = min(COLS, sq.m * G - qb * COLS);
    s = it.s;
#pragma unroll
    for (int t = 0; t < NT; ++t)
      if (t * 16 + row < cols) {
#pragma unroll
        for (int d = 0; d < P::VL; ++d) *(f32x4*)&part[wave][t * 16 + row][d * 16 + grp * 4] = x.o[t][d];
        if (grp == 0) ml[wave][t * 16 + row] = float2{x.m[t], x.l[t]};
      }
    __syncthreads();
    const bool done = t0 == 0 && t1 == sq.steps;
    if (t0 == 0 && !done && threadIdx.x == 0)
      *cut = Cut{s, g, qb, (short)quotient(it.at + COST + sq.steps - 1, plan.length), (short)cols};
    float* slot = a.ws + cut_floats(runs) + (size_t)(2 * r + (t0 == 0)) * slot_floats<D, NT>();
    for (int i = threadIdx.x; i < cols * (D / 4); i += 256) {
      const int c = i / (D / 4), d = i % (D / 4) * 4, col = qb * COLS + c;
      float top = ml[0][c].x, sum = 0.f;
#pragma unroll
      for (int w = 1; w < kWaves; ++w)
        top = fmaxf(top, ml[w][c].x);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        {
          const float f = exp2_raw(ml[w][c].x - top);
          sum += f * ml[w][c].y;
          o += f * *(const f32x4*)&part[w][c][d];
        }
      if (done) {
        const int i = token_of(a, col), h = g * G + col - i * G;
        const size_t row_out = (size_t)s * a.n + i;
        store_row4((T*)a.out + (row_out * a.Hq + h) * D + d, o * (sum == 0.f ? 0.f : 1.f / sum));
        if (a.lse && d == 0) a.lse[row_out * a.Hq + h] = lse_of(top, sum);
      } else {
        *(f32x4*)(slot + c * D + d) = o;
        if (d == 0) *(float2*)(slot + COLS * D + 2 * c) = float2{top, sum};
      }
    }
    it = next;
    __syncthreads();
  }
}

// Columns per workgroup of the joining kernel: one where an item has few (its pieces
// are then shared out over the workgroup), eight where it has many.  One sequence of 131072, cut into
// 64 pieces a head: 5.7 us, 12.8 with eight; 16 tokens of 16 sequences of 4096: 5.2, 13.3 with one.
constexpr int join_cols(int nt) { return nt == 1 ? 1 : 8; }

// The outputs of the items that several runs share, by the run that an item starts
// in: one workgroup per (run, join_cols columns), D / 4 threads to a piece.  2.8 to 5.7 us: a launch and
// one round trip, two where an item has more pieces than fit the threads (1 to 5 MB, which lie in the caches).
template <typename T, int D, int NT>
__global__ __launch_bounds__(256) void attn_join_kernel(PagedAttnArgs a, int runs) {
  constexpr int COLS = 16 * NT, W = D / 4, CB = join_cols(NT), PARTS = 256 / W / CB;
  __shared__ f32x4 acc_s[CB][PARTS][W];
  __shared__ float2 ml_s[CB][PARTS];
  const int r = blockIdx.x, t = threadIdx.x;
  const Cut cut = ((const Cut*)a.ws)[r];
  const int d = t % W, k = t / W / PARTS, part = t / W % PARTS, c = blockIdx.y * CB + k;
  const float* slots = a.ws + cut_floats(runs);
  auto slot = [&](int w) { return slots + (size_t)(2 * w + (w == r)) * slot_floats<D, NT>(); };
  // the first piece is asked for together with the cut; where there is none, it is not used
  const float* first = slot(min(r + part, runs - 1));
  f32x4 acc = *(const f32x4*)(first + c * D + 4 * d);
  const float2 ml0 = *(const float2*)(first + COLS * D + 2 * c);
  asm volatile("" ::"v"(acc), "v"(ml0.x), "v"(ml0.y));
  if (cut.s < 0) return;
  const int G = a.G, col = cut.qb * COLS + c, cols = cut.cols;
  float sum = ml0.y, top = ml0.x;
  if (c < cols) {
    if (r + part > cut.last) {
      acc = f32x4{0.f, 0.f, 0.f, 0.f};
      sum = 0.f;
      top = kNoRef;
    }
#pragma unroll 4
    for (int w = r + part + PARTS; w <= cut.last; w += PARTS) {
      const float* p = slot(w);
      const float2 ml = *(const float2*)(p + COLS * D + 2 * c);
      const float nt = fmaxf(top, ml.x), down = exp2_raw(top - nt), f = exp2_raw(ml.x - nt);
      acc = acc * down + f * *(const f32x4*)(p + c * D + 4 * d);
      sum = sum * down + f * ml.y;
      top = nt;
    }
    acc_s[k][part][d] = acc;
    if (d == 0) ml_s[k][part] = float2{top, sum};
  }
  if (PARTS > 1) __syncthreads();
  if (part > 0 || c >= cols) return;
  if (PARTS > 1) {
#pragma unroll
    for (int i = 0; i < PARTS; ++i) top = fmaxf(top, ml_s[k][i].x);
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
      const float f = exp2_raw(ml_s[k][i].x - top);
      acc += f * acc_s[k][i][d];
      sum += f * ml_s[k][i].y;
    }
  }
  const int i = token_of(a, col);
  const size_t at = ((size_t)cut.s * a.n + i) * a.Hq + cut.g * G + col - i * G;
  store_row4((T*)a.out + at * D + 4 * d, acc * (sum == 0.f ? 0.f : 1.f / sum));
  if (d == 0 && a.lse) a.lse[at] = lse_of(top, sum);
}

// Query tiles a wave holds at once: all of a sequence's query vectors up to 64 (fp32
// of 128 dimensions: 32, what the registers hold), as each further item reads K and V again.  20
// vectors of 32 sequences to 4096: 21.5 us in two tiles, 25.0 in two items of one; 64 vectors of 16
// sequences of 4096: 65 us in four, 82 in two items of two, 145 in four of one.  (48 vectors of 32
// sequences to 4096, 73 MB that the last-level cache holds: 31.2, 31.9 and 38.9.)
int tiles_for(const PagedView& c, int vectors) {
  return vectors <= 16 ? 1 : vectors <= 32 || (c.esz == 4 && c.D == 128) ? 2 : 4;
}

// Runs of a call whose sequences have up to `vectors` query vectors per KV head.
int runs_for(const PagedView& c, int vectors) {
  const int nt = tiles_for(c, vectors), cols = 16 * nt;
  const double items = (double)c.S * c.Hkv * ((vectors + cols - 1) / cols);
  const double steps = items * std::max(1.0, std::ceil((double)c.width * c.ps / kStep));
  const double most = two_per_cu(nt, c.esz * c.D) ? kMaxRuns : kMaxRuns / 2;
  return (int)std::min(most, std::ceil((steps + item_cost(nt) * items) / kMinSteps));
}

template <typename T, int D, int NT>
hipError_t launch(const PagedAttnArgs& a, hipStream_t s) {
  const int runs = runs_for(a.c, a.n * a.G);
  // PAST where a round of a wave takes all positions of a page's V row, and so whole cache lines; where waves share
  // lines, the second one is to find them.  64 ragged sequences to 8192, pages of 16: 47 us, 51 without; one of 131072,
  // pages of 64: 109 us, 96 without.  (K past the caches, too: 48 and 109; K alone: 50 and 99.)
  if (a.c.ps <= Piece<T, D, NT, true>::PER)
    hipLaunchKernelGGL((attn_run_kernel<T, D, NT, true>), dim3(runs), dim3(256), 0, s, a, runs);
  else
    hipLaunchKernelGGL((attn_run_kernel<T, D, NT, false>), dim3(runs), dim3(256), 0, s, a, runs);
  if (hipError_t e = hipGetLastError()) return e;
  const int cols = std::min(16 * NT, a.n * a.G);
  const dim3 grid(runs, (cols + join_cols(NT) - 1) / join_cols(NT));
  hipLaunchKernelGGL((attn_join_kernel<T, D, NT>), grid, dim3(256), 0, s, a, runs);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_tiles(const PagedAttnArgs& a, hipStream_t s) {
  switch (tiles_for(a.c, a.n * a.G)) {
    case 1: return launch<T, D, 1>(a, s);
    case 2: return launch<T, D, 2>(a, s);
  }
  if constexpr (sizeof(T) == 2 || D < 128) return launch<T, D, 4>(a, s);
  return hipErrorInvalidValue;
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

// the plan's units, whatever the lengths are, in numbers that it can count with
bool paged_attention_fits(const PagedView& c, int n, int Hq) {
  const int nt = tiles_for(c, n * (Hq / c.Hkv)), tiles = (n * (Hq / c.Hkv) + 16 * nt - 1) / (16 * nt);
  const double units = (double)c.S * c.Hkv * tiles * (std::ceil((double)c.width * c.ps / kStep) + item_cost(nt));
  return units < 274877906944.0;  // 2^38: a run's share of it is counted in ints
}

// Enough for every call of up to n tokens: fewer query vectors take fewer tiles, whose runs may be twice as many
// (two workgroups per CU in place of one), so the most that one to tiles_for of them need.
size_t paged_attention_workspace_floats(const PagedView& c, int n, int Hq) {
  const int vectors = n * (Hq / c.Hkv);
  size_t most = 0;
  for (const int upto : {16, 32, vectors}) {
    const int v = std::min(upto, vectors), runs = runs_for(c, v);
    most = std::max(most, cut_floats(runs) + (size_t)2 * runs * 16 * tiles_for(c, v) * (c.D + 2));
  }
  return most;
}

hipError_t paged_attention(const PagedAttnArgs& a0, hipStream_t s) {
  PagedAttnArgs a = a0;
  a.G = a.Hq / a.c.Hkv;
  a.inv_G = (unsigned)(((1ull << 31) + a.G - 1) / a.G);
  return a.c.esz == 2 ? launch_dim<bf16_t>(a, s) : launch_dim<float>(a, s);
}

}  // namespace rgd
