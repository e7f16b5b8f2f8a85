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
//
// By a plan of what sequences share the same kernels take only what is left of each one behind its shared positions, and
// join that with the parts that the groups' kernel left (fp32: the run kernel with a group's tokens as one sequence's; bf16:
// a kernel of its own).  Most of what is left is short, and is done in the joining launch.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "paged.hpp"
#include "paged_tiles.hpp"
#include "share.hpp"

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
// What a kernel attends to: whole sequences; by a plan, what groups of sequences share, each group a sequence of the
// tokens of all its members; or what is left of the sequences behind that, whose parts are joined with the shared ones:
// long ones as WHOLE, the others, of up to kTailSteps, a wave or a workgroup each.
enum Mode { WHOLE, SHARED, OWN, TAIL };
constexpr int kTailSteps = 24, kAloneSteps = 2, kManyTails = 768;  // (one load of page numbers covers a tail)
static_assert(2 * kTailSteps + 1 <= 64, "a tail's pages, of 16 positions at least, are looked up in one load");

// New tokens of sequence s.
RGD_DEV int new_tokens(const PagedAttnArgs& a, int s) { return a.n_new ? min(max(a.n_new[s], 0), a.n) : a.n; }

// Floor of col / G for col * G < 2^31: the product passes col / G by less than col / 2^31, which is less than 1 / G.
// (A sequence's: below 2^20 * 2^10.  A group's: what the entry point lets through.)
RGD_DEV int token_of(const PagedAttnArgs& a, int col) { return (int)__umulhi((unsigned)col << 1, a.inv_G); }

struct Seq {
  int len, m;   // positions, new tokens
  int from;     // first position of the steps: a multiple of 16
  int steps;    // per item; at least one, so that tokens that see nothing get their zeros
  int tiles;    // query tiles; 0 without new tokens.  Items: KV heads x query tiles
};

template <int COLS>
RGD_DEV Seq seq_of(const PagedAttnArgs& a, int len, int m, int from) {
  Seq q;
  q.len = len;
  q.m = m;
  q.from = from;
  q.steps = max(1, (len - from + kStep - 1) / kStep);
  q.tiles = (m * a.G + COLS - 1) / COLS;
  return q;
}
// What is left of a sequence behind its shared positions; no tiles where that is the other mode's.  The plan's tokens and
// shared positions may be any numbers where it is not this call's (most is 0): then there are no tokens, and no tiles.
template <int COLS, int MODE>
RGD_DEV Seq rest_of(const PagedAttnArgs& a, int len, int tokens, int shared) {
  Seq q = seq_of<COLS>(a, len, max(min(tokens, a.most), 0), min(max(shared, 0), len / 16 * 16));
  if ((q.steps <= kTailSteps) != (MODE == TAIL)) q.tiles = 0;
  return q;
}
template <int COLS, int MODE>
RGD_DEV Seq seq_of(const PagedAttnArgs& a, int s) {
  if constexpr (MODE == WHOLE) {
    return seq_of<COLS>(a, paged_len(a.c, s), new_tokens(a, s), 0);
  } else {
    const Plan p(a.plan, a.c.S);
    if constexpr (MODE == SHARED) {
      const PlanGroup g = p.group[s];
      return seq_of<COLS>(a, a.most ? g.shared : 0, a.most ? g.tokens : 0, 0);
    } else {
      return rest_of<COLS, MODE>(a, paged_len(a.c, s), p.tokens[s], p.shared[s]);
    }
  }
}
// The same for an s that the whole wave shares, by scalar loads: a vector load's wait would be one
// for the K and V on their way, too.
template <int COLS, int MODE>
RGD_DEV Seq uniform_seq(const PagedAttnArgs& a, int s) {
  typedef const int __attribute__((address_space(4))) * Scalar;
  if constexpr (MODE == WHOLE) {
    const int len = ((Scalar)a.c.lens)[s], m = a.n_new ? ((Scalar)a.n_new)[s] : a.n;
    return seq_of<COLS>(a, min(max(len, 0), a.c.width * a.c.ps), min(max(m, 0), a.n), 0);
  } else {
    const Plan p(a.plan, a.c.S);
    if constexpr (MODE == SHARED) {
      Scalar g = (Scalar)p.group + 4 * s;
      return seq_of<COLS>(a, a.most ? g[0] : 0, a.most ? g[1] : 0, 0);
    } else {
      const int len = min(max(((Scalar)a.c.lens)[s], 0), a.c.width * a.c.ps);
      return rest_of<COLS, MODE>(a, len, ((Scalar)p.tokens)[s], ((Scalar)p.shared)[s]);
    }
  }
}

// Units of the plan that this lane's sequence takes (none behind the last).
template <int COLS, int MODE>
RGD_DEV long long units_of(const PagedAttnArgs& a, int s, Seq& q) {
  q = seq_of<COLS, MODE>(a, min(s, a.c.S - 1));
  return s < a.c.S ? (long long)(q.steps + item_cost(COLS / 16)) * (a.c.Hkv * q.tiles) : 0;
}

struct Runs {
  long long total, length;  // units of the plan, units per run
};

// Finds the run of workgroup r (of `runs`): the sequence it starts in and the units
// before that one.  False: there is none.
template <int COLS, int MODE>
RGD_DEV bool find_run(const PagedAttnArgs& a, int r, int runs, Runs& plan, int& s, Seq& sq, long long& before) {
  const int lane = threadIdx.x & 63, per = (a.c.S + 63) / 64;  // sequences a lane: one, or neighbouring ones
  Seq q;
  long long u = 0;
#pragma unroll 8
  for (int k = 0; k < per; ++k) u += units_of<COLS, MODE>(a, lane * per + k, q);
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
      u = units_of<COLS, MODE>(a, s + lane, q);
      incl = wave_scan(u);
      if (const unsigned long long hit = __ballot(before + incl > start)) {
        l = __builtin_ctzll(hit);
        before += lane_value(incl - u, l);
        s += l;
        break;
      }
      before += lane_value(incl, 63);
    }
  sq = seq_of<COLS>(a, __builtin_amdgcn_readlane(q.len, l), __builtin_amdgcn_readlane(q.m, l),
                    MODE == OWN ? __builtin_amdgcn_readlane(q.from, l) : 0);
  return true;
}

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

// One item of a run: steps [t0, t1) of query tile qb of KV head g of sequence s.
struct Item {
  Seq sq;
  int s, g, qb, t0, t1;
  int row;     // SHARED: of its tokens in the plan's list
  int number;  // SHARED: among all items
  bool valid;
  long long at;  // its first unit in the plan
  RGD_DEV int end() const { return min(sq.from + t1 * kStep, max(sq.len, sq.from + 1)); }
  RGD_DEV int begin(int wave, int per) const { return sq.from + t0 * kStep + wave * per; }
};

RGD_DEV Seq same_for_all(const Seq& q) {
  return Seq{uniform(q.len), uniform(q.m), uniform(q.from), uniform(q.steps), uniform(q.tiles)};
}

// The token row of an item's token i: its q, and its outputs.
template <int MODE>
RGD_DEV size_t row_of(const PagedAttnArgs& a, const Item& it, int i) {
  if constexpr (MODE == SHARED) return Plan(a.plan, a.c.S).rows[it.row + i];
  else return (size_t)it.s * a.n + i;
}

// The items of a run, one after the other.
template <int COLS, int MODE>
struct Walk {
  static constexpr int COST = item_cost(COLS / 16);
  Seq sq;
  int s, g, qb, u0, left;
  int number;
  long long at;
  RGD_DEV Item next(const PagedAttnArgs& a) {
    Item it{};
    if (left <= 0) return it;
    if (g == a.c.Hkv) {  // steps are left, so a sequence with new tokens follows
      g = 0;
      do sq = uniform_seq<COLS, MODE>(a, ++s);
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
    if constexpr (MODE == SHARED) {
      typedef const int __attribute__((address_space(4))) * Scalar;
      it.row = ((Scalar)Plan(a.plan, a.c.S).group)[4 * s + 2];
      it.number = number++;
    }
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
template <typename T, int D, int NT, bool PAST, int MODE>
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
      int p = MODE == TAIL ? walk.find_near((p0 >> 4) + b, place) : walk.find((p0 >> 4) + b, place);
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
    const T* src = (const T*)a.q + row_of<MODE>(a, it, i) * a.ldq + (size_t)(it.g * G + col - i * G) * D;
#pragma unroll
    for (int c = 0; c < KL; ++c) dst[(wave * KL + c) * 64 + lane] = *(const u32x4*)((const char*)src + c * 64 + grp * 16);
  }

  RGD_DEV void load_q(const PagedAttnArgs& a, const Item& it) {
    if (QS) return;
    const int G = a.G, cols = it.sq.m * G;
#pragma unroll
    for (int t = 0; t < (QS ? 0 : NT); ++t) {
      const int col = min(it.qb * COLS + t * 16 + row, cols - 1), i = token_of(a, col);  // columns behind the last one repeat it
      const T* src = (const T*)a.q + row_of<MODE>(a, it, i) * a.ldq + (size_t)(it.g * G + col - i * G) * D;
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

  // One round of positions from p0 on, any of which may be masked, whose K and V are on their way; the next round's K is
  // asked for in between.  lim: positions that a column sees, least of all.
  template <class LoadK>
  RGD_DEV void take(const Seq& sq, const int (&lim)[NT], int least, int p0, float scale, LoadK&& next) {
    f32x4 s4[NT][NB];
    scores(s4);
    const int here = ok;
    __builtin_amdgcn_sched_barrier(0);
    next();
    __builtin_amdgcn_sched_barrier(0);
    const int pos = p0 + grp * E;  // of this lane's first score
    const bool there = BF ? (here >> (grp >> 1)) & 1 : here & 1;
    bool odd = false;
    if (here != (1 << NB) - 1 || p0 + PER > sq.len) {
      const int held = there ? sq.len - pos : 0;
#pragma unroll
      for (int d = 0; d < VL; ++d) v[d] = keep_first<T>(v[d], held);
    }
    if (least < min(p0 + PER, sq.len)) {  // not every column sees every value
#pragma unroll
      for (int d = 0; d < VL; ++d) odd |= any_nonfinite<T>(v[d]);
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
    if (__any(odd)) spread_nonfinite(v, lim, there, pos);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int d = 0; d < VL; ++d) o[t][d] = weigh(v[d], p[t], hi[t], lo[t], o[t][d]);
  }

  // 0 times a value that is not finite is not 0, so these leave the product: a
  // column gets them by whether it sees one, not by its weight
  RGD_DEV void spread_nonfinite(u32x4 (&v)[VL], const int (&lim)[NT], bool there, int pos) {
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

  // Every waves-th round of the item from the wave's own on.  The loads are the same on every path, so that a wait for some
  // leaves those behind them on their way: behind the end every lane asks for the last round's first bytes.
  RGD_DEV void run_alone(const PagedAttnArgs& a, const Item& it, const TableWalk& table, int wave, int waves) {
    const Seq& sq = it.sq;
    const int cols = sq.m * a.G, by = waves * PER, first = it.begin(wave, PER), end = it.end();
    int lim[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      lim[t] = sq.len - sq.m + token_of(a, min(it.qb * COLS + t * 16 + row, cols - 1)) + 1;
      m[t] = kNoRef;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < VL; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (first >= end) return;
    const int least = sq.len - sq.m + token_of(a, it.qb * COLS) + 1, row0 = row, grp0 = grp;
    const float scale = kLog2e / sqrtf((float)D);
    walk = table;
    load_q(a, it);
    load_k(a, it.g, first);
    __builtin_amdgcn_sched_barrier(0);
    load_v(a);
    for (int p0 = first; p0 < end; p0 += by) {
      const bool more = p0 + by < end;
      take(sq, lim, least, p0, scale, [&] {
        row = more ? row0 : 0;
        grp = more ? grp0 : 0;
        load_k(a, it.g, more ? p0 + by : p0);
        row = row0;
        grp = grp0;
      });
      row = more ? row0 : 0;
      grp = more ? grp0 : 0;
      load_v(a);
      row = row0;
      grp = grp0;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      l[t] += __shfl_xor(l[t], 16, 64);
      l[t] += __shfl_xor(l[t], 32, 64);
    }
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
      lim[t] = MODE == SHARED ? sq.len : sq.len - sq.m + token_of(a, min(qb * COLS + t * 16 + row, cols - 1)) + 1;
      m[t] = kNoRef;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < VL; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int least = MODE == SHARED ? sq.len : sq.len - sq.m + token_of(a, qb * COLS) + 1;  // all of the tile's tokens see that much
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
      const int pos = p0 + grp * E;
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
      if (__any(odd)) spread_nonfinite(v, lim, there, pos);
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

template <typename T>
RGD_DEV void store_row4(T* p, f32x4 v) {
  if constexpr (sizeof(T) == 2) *(u32x2*)p = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  else *(f32x4*)p = v;
}

// The parts of a sequence's shared positions, as the kernel before left them, joined with (top, sum, o) of a query vector of
// token i; four dimensions from d on.
struct SharedParts {
  const float* slots;
  long long length, unit;  // of a run; the group's first
  int col, tiles, steps, item, cols, cost, D;
  // (scalar loads: s is the wave's, and these loads do not queue behind K and V)
  RGD_DEV SharedParts(const PagedAttnArgs& a, int s) {
    typedef const int __attribute__((address_space(4))) * Scalar;
    typedef const long long __attribute__((address_space(4))) * Scalar64;
    const Plan p(a.plan, a.c.S);
    const int leader = ((Scalar)p.leader)[s], shared = leader < 0 ? 0 : ((Scalar)p.shared)[s];
    steps = (shared + a.s_step - 1) / a.s_step;
    if (!steps) return;
    Scalar g = (Scalar)p.group + 4 * leader, at = (Scalar)a.at + 4 * leader;
    length = *((Scalar64)a.at + 2 * a.c.S);
    unit = *(Scalar64)at;
    item = at[2];
    col = (((Scalar)p.row)[s] - g[2]) * a.G;
    cols = a.s_cols;
    cost = a.s_cost;
    tiles = (g[1] * a.G + cols - 1) / cols;
    slots = a.slots;
    D = a.c.D;
  }
  // the slots of query vector v of KV head g: [first, last], and its place there
  RGD_DEV const float* find(int g, int v, int& parts, int& c) const {
    const int qb = (col + v) / cols, k = g * tiles + qb;
    c = col + v - qb * cols;
    const long long u = unit + (long long)k * (steps + cost) + cost;
    const int r0 = (int)quotient(u, length);
    parts = (int)quotient(u + steps - 1, length) - r0 + 1;
    return slots + (size_t)(r0 + item + k) * cols * (D + 2);
  }
  // the query vector of KV head g that is `v` (token * G + head) among the sequence's
  RGD_DEV void join(int g, int v, int d, float& top, float& sum, f32x4& o) const {
    if (!steps) return;
    int parts, c;
    const float* slot = find(g, v, parts, c);
#pragma unroll 4
    for (int r = 0; r < parts; ++r) {
      const float* at = slot + (size_t)r * cols * (D + 2);
      const float2 ml = *(const float2*)(at + cols * D + 2 * c);
      const f32x4 x = *(const f32x4*)(at + c * D + d);
      const float nt = fmaxf(top, ml.x), down = exp2_raw(top - nt), f = exp2_raw(ml.x - nt);
      o = o * down + f * x;
      sum = sum * down + f * ml.y;
      top = nt;
    }
  }
  // all of a lane's dimensions, d * 16 + off; every `ways`-th part from `way` on
  template <int VL>
  RGD_DEV void join_all(int g, int v, int off, int way, int ways, float& top, float& sum, f32x4 (&o)[VL]) const {
    if (!steps) return;
    int parts, c;
    const float* slot = find(g, v, parts, c);
#pragma unroll 4
    for (int r = way; r < parts; r += ways) {
      const float* at = slot + (size_t)r * cols * (D + 2);
      const float2 ml = *(const float2*)(at + cols * D + 2 * c);
      f32x4 x[VL];
#pragma unroll
      for (int d = 0; d < VL; ++d) x[d] = *(const f32x4*)(at + c * D + d * 16 + off);
      const float nt = fmaxf(top, ml.x), down = exp2_raw(top - nt), f = exp2_raw(ml.x - nt);
#pragma unroll
      for (int d = 0; d < VL; ++d) o[d] = o[d] * down + f * x[d];
      sum = sum * down + f * ml.y;
      top = nt;
    }
  }
};

// Where each group's units and items begin, for the kernels that join; one wave.
template <int COLS>
RGD_DEV void list_groups(const PagedAttnArgs& a, long long length) {
  const int lane = threadIdx.x & 63;
  GroupAt* at = (GroupAt*)a.at;
  long long units = 0, items = 0;
  for (int s0 = 0; s0 < a.c.S; s0 += 64) {
    Seq q;
    const long long u = units_of<COLS, SHARED>(a, s0 + lane, q), n = s0 + lane < a.c.S ? a.c.Hkv * q.tiles : 0;
    const long long ui = wave_scan(u), ni = wave_scan(n);
    if (s0 + lane < a.c.S) at[s0 + lane] = GroupAt{units + ui - u, (int)(items + ni - n), 0};
    units += lane_value(ui, 63);
    items += lane_value(ni, 63);
  }
  if (lane == 0) at[a.c.S] = GroupAt{length, 0, 0};
}

template <int MODE>
RGD_DEV void check_plan(PagedAttnArgs& a) {
  if constexpr (MODE != WHOLE) a.most = *Plan(a.plan, a.c.S).head == PlanHead::of(a.c, a.n, a.Hq) ? a.n : 0;
}

template <typename T, int D, int NT, bool PAST, int MODE>
__global__ __launch_bounds__(256, two_per_cu(NT, sizeof(T) * D) ? 2 : 1) void attn_run_kernel(PagedAttnArgs a, int runs) {
  using P = Piece<T, D, NT, PAST, MODE>;
  constexpr int COLS = P::COLS, LD = D + 4, COST = item_cost(NT);
  __shared__ float part[kWaves][COLS][LD];
  __shared__ float2 ml[kWaves][COLS];
  __shared__ u32x4 q_s[P::QS ? NT * P::KL * 64 : 1];
  const int r = blockIdx.x, wave = uniform(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, row = lane & 15, grp = lane >> 4;
  Runs plan;
  int s;
  long long before;
  Walk<COLS, MODE> walk;
  Cut* cut = (Cut*)a.ws + r;
  check_plan<MODE>(a);
  if (MODE != SHARED && threadIdx.x == 0) *cut = Cut{-1, 0, 0, 0};
  const bool found = find_run<COLS, MODE>(a, min(r, runs - 1), runs, plan, s, walk.sq, before);
  if constexpr (MODE == SHARED)
    if (r == runs) {  // a workgroup beside the runs'
      if (wave == 0) list_groups<COLS>(a, plan.length);
      return;
    }
  if (!found) return;
  const long long start = r * plan.length;
  walk.s = uniform(s);
  walk.left = uniform((int)min(plan.length, plan.total - start));
  walk.sq = same_for_all(walk.sq);
  const int item = uniform((int)quotient(start - before, walk.sq.steps + COST));
  walk.g = item / walk.sq.tiles;
  walk.qb = item - walk.g * walk.sq.tiles;
  walk.at = before + (long long)item * (walk.sq.steps + COST);
  walk.u0 = uniform((int)(start - walk.at));
  if constexpr (MODE == SHARED) {
    long long ahead = 0;
    for (int s0 = 0; s0 < walk.s; s0 += 64) {
      const Seq q = seq_of<COLS, MODE>(a, min(s0 + lane, a.c.S - 1));
      ahead += lane_value(wave_scan(s0 + lane < walk.s ? a.c.Hkv * q.tiles : 0), 63);
    }
    walk.number = uniform((int)ahead + item);
  }
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
    const bool done = MODE != SHARED && t0 == 0 && t1 == sq.steps;
    if (MODE != SHARED && t0 == 0 && !done && threadIdx.x == 0)
      *cut = Cut{s, g, qb, (short)quotient(it.at + COST + sq.steps - 1, plan.length), (short)cols};
    float* slot = a.ws + cut_floats(runs) + (size_t)(2 * r + (t0 == 0)) * slot_floats<D, NT>();
    if constexpr (MODE == SHARED) slot = a.slots + (size_t)(r + it.number) * slot_floats<D, NT>();
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
        if constexpr (MODE == OWN) SharedParts(a, s).join(g, col, d, top, sum, o);
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

// Workgroups of the tails, four for each four items.
__host__ __device__ inline int tail_groups(const PagedAttnArgs& a) {
  return kWaves * a.c.S * ((a.c.Hkv * ((a.n * a.G + 15) / 16) + kWaves - 1) / kWaves);
}

// What is left of a sequence behind its shared positions, where that is short: 16 query vectors of a KV head are a
// workgroup's, whose waves take rounds and shared parts in turn, or, of up to kAloneSteps steps where there are more than
// the chip holds workgroups, a wave's.  What bounds it is a chain of loads: lengths and plan, pages, K and V, parts (64
// branches of one prompt 12 us).  256 branches, 4 to 300 positions left, 8 KV
// heads: 30 us, a wave for up to 0, 2, 3 and 6 steps 33, 31, 30 and 31; 64 x 5 tokens, 20 vectors: 16, 16, 19 and 21.
// Pieces of prompts were no part of that choice: each 16 query vectors read what is left of their sequence again (16 sequences of 64,
// 256 and 512 new tokens behind 4096 shared positions, 32 heads, 158, 570 and 1246 us with the groups' part).
// There are four workgroups for each four items, of which the first has work where waves do them; these come
// before all others, so that they meet all parts of the chip.
template <typename T, int D>
RGD_DEV void attend_tail(PagedAttnArgs a, int index, float (&part)[kWaves][16][D + 4], float2 (&ml)[kWaves][16]) {
  using P = Piece<T, D, 1, false, TAIL>;
  check_plan<TAIL>(a);
  const int wave = uniform(threadIdx.x >> 6);
  const int per = (a.n * a.G + 15) / 16, all = a.c.Hkv * per, fours = (all + kWaves - 1) / kWaves;
  const int nth = index / (a.c.S * fours), s = (index - nth * a.c.S * fours) / fours;
  Item it{};
  it.sq = uniform_seq<16, TAIL>(a, s);
  const bool alone = a.c.S * all > kManyTails && it.sq.steps <= kAloneSteps;
  if (alone && nth) return;
  const int rest = index % fours * kWaves + (alone ? wave : nth);
  if (rest >= all) return;
  it.s = s;
  it.g = rest / per;
  it.qb = rest - it.g * per;
  if (it.qb >= it.sq.tiles) return;
  it.t1 = it.sq.steps;
  it.valid = true;
  const SharedParts shared(a, s);
  P x;
  x.lane = threadIdx.x & 63;
  x.row = x.lane & 15;
  x.grp = x.lane >> 4;
  TableWalk table;
  table.start(a.c, s, it.begin(0, P::PER) >> 4);
  const int w0 = alone ? 0 : wave, waves = alone ? 1 : kWaves;
  x.run_alone(a, it, table, w0, waves);
  // where there are fewer than 16 columns, the lanes of the others take part of a column's shared parts
  const int here = min(it.sq.m * a.G - it.qb * 16, 16), width = here > 8 ? 16 : here > 4 ? 8 : here > 2 ? 4 : here;
  const int way = x.row / width, ways = 16 / width, col = it.qb * 16 + min(x.row % width, here - 1);
  float top = way ? kNoRef : x.m[0], sum = way ? 0.f : x.l[0];
#pragma unroll
  for (int d = 0; d < P::VL; ++d) x.o[0][d] = way ? f32x4{0.f, 0.f, 0.f, 0.f} : x.o[0][d];
  shared.join_all(it.g, col, x.grp * 4, way + ways * w0, ways * waves, top, sum, x.o[0]);
  for (int w = width; w < 16; w *= 2) {
    const float t2 = __shfl_xor(top, w, 64), s2 = __shfl_xor(sum, w, 64);
    const float nt = fmaxf(top, t2), down = exp2_raw(top - nt), f = exp2_raw(t2 - nt);
    sum = sum * down + f * s2;
    top = nt;
#pragma unroll
    for (int d = 0; d < P::VL; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) x.o[0][d][e] = x.o[0][d][e] * down + f * __shfl_xor(x.o[0][d][e], w, 64);
  }
  const int i = token_of(a, col);
  const size_t at = ((size_t)s * a.n + i) * a.Hq + it.g * a.G + col - i * a.G;
  if (alone) {
    if (x.row >= here) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < P::VL; ++d) store_row4((T*)a.out + at * D + d * 16 + x.grp * 4, x.o[0][d] * inv);
    if (a.lse && x.grp == 0) a.lse[at] = lse_of(top, sum);
    return;
  }
#pragma unroll
  for (int d = 0; d < P::VL; ++d) *(f32x4*)&part[wave][x.row][d * 16 + x.grp * 4] = x.o[0][d];
  if (x.grp == 0) ml[wave][x.row] = float2{top, sum};
  __syncthreads();
  if (x.row >= here) return;
  top = kNoRef;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][x.row].x);
  float f[kWaves];
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    f[w] = exp2_raw(ml[w][x.row].x - top);
    sum += f[w] * ml[w][x.row].y;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  for (int d = wave; d < P::VL; d += kWaves) {
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) o += f[w] * *(const f32x4*)&part[w][x.row][d * 16 + x.grp * 4];
    store_row4((T*)a.out + at * D + d * 16 + x.grp * 4, o * inv);
  }
  if (a.lse && x.grp == 0 && wave == 0) a.lse[at] = lse_of(top, sum);
}

// The outputs of the items that several runs share, by the run that an item starts
// in: one workgroup per (run, join_cols columns), D / 4 threads to a piece.  2.8 to 5.7 us: a launch and
// one round trip, two where an item has more pieces than fit the threads (1 to 5 MB, which lie in the caches).
template <typename T, int D, int NT, int MODE>
__global__ __launch_bounds__(256, MODE != OWN ? 1 : D == 32 || sizeof(T) * D == 512 ? 2 : 3) void attn_join_kernel(PagedAttnArgs a, int runs) {
  constexpr int COLS = 16 * NT, W = D / 4, CB = join_cols(NT), PARTS = 256 / W / CB;
  __shared__ f32x4 acc_s[CB][PARTS][W];
  __shared__ float2 ml_s[CB][PARTS];
  const int t = threadIdx.x;
  int block = blockIdx.x;
  if constexpr (MODE == OWN) {  // the tails' workgroups come first
    __shared__ float part_s[kWaves][16][D + 4];
    __shared__ float2 ml_w[kWaves][16];
    const int tails = tail_groups(a);
    if (block < tails) {
      attend_tail<T, D>(a, block, part_s, ml_w);
      return;
    }
    block -= tails;
  }
  const int r = block % runs, by = block / runs;
  const Cut cut = ((const Cut*)a.ws)[r];
  const int d = t % W, k = t / W / PARTS, part = t / W % PARTS, c = by * CB + k;
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
  if constexpr (MODE == OWN) SharedParts(a, uniform(cut.s)).join(cut.g, col, 4 * d, top, sum, acc);
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

template <typename T, int D, int NT, int MODE>
hipError_t launch(const PagedAttnArgs& a, int vectors, hipStream_t s) {
  // no runs where no own part can be too long for a tail: by the table's width, as lengths are on the device (2 sequences, 100
  // shared positions, a table of up to 768: 22 -> 20 us; wider tables pay 5 us a layer for a launch that may have nothing to do)
  const int runs = MODE == OWN && a.c.width * a.c.ps <= kTailSteps * kStep ? 0 : runs_for(a.c, vectors);
  // PAST where a round of a wave takes all positions of a page's V row, and so whole cache lines; where waves share
  // lines, the second one is to find them.  64 ragged sequences to 8192, pages of 16: 47 us, 51 without; one of 131072,
  // pages of 64: 109 us, 96 without.  (K past the caches, too: 48 and 109; K alone: 50 and 99.)
  if (MODE != SHARED && a.c.ps <= Piece<T, D, NT, true, MODE>::PER) {
    if (runs > 0) hipLaunchKernelGGL((attn_run_kernel<T, D, NT, true, MODE>), dim3(runs), dim3(256), 0, s, a, runs);
  } else if (runs > 0) {
    hipLaunchKernelGGL((attn_run_kernel<T, D, NT, false, MODE>), dim3(runs + (MODE == SHARED)), dim3(256), 0, s, a, runs);
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (MODE == SHARED) return hipSuccess;
  const int cols = std::min(16 * NT, a.n * a.G);
  const dim3 grid(runs * ((cols + join_cols(NT) - 1) / join_cols(NT)) + (MODE == OWN ? tail_groups(a) : 0));
  hipLaunchKernelGGL((attn_join_kernel<T, D, NT, MODE>), grid, dim3(256), 0, s, a, runs);
  return hipGetLastError();
}

template <int MODE, typename T, int D>
hipError_t launch_tiles(const PagedAttnArgs& a, int vectors, hipStream_t s) {
  switch (tiles_for(a.c, vectors)) {
    case 1: return launch<T, D, 1, MODE>(a, vectors, s);
    case 2: return launch<T, D, 2, MODE>(a, vectors, s);
  }
  if constexpr (sizeof(T) == 2 || D < 128) return launch<T, D, 4, MODE>(a, vectors, s);
  return hipErrorInvalidValue;
}

template <int MODE, typename T>
hipError_t launch_dim(const PagedAttnArgs& a, int vectors, hipStream_t s) {
  switch (a.c.D) {
    case 32: return launch_tiles<MODE, T, 32>(a, vectors, s);
    case 64: return launch_tiles<MODE, T, 64>(a, vectors, s);
    default: return launch_tiles<MODE, T, 128>(a, vectors, s);
  }
}

template <int MODE>
hipError_t launch_type(const PagedAttnArgs& a, int vectors, hipStream_t s) {
  return a.c.esz == 2 ? launch_dim<MODE, bf16_t>(a, vectors, s) : launch_dim<MODE, float>(a, vectors, s);
}

PagedAttnArgs with_groups(const PagedAttnArgs& a0) {
  PagedAttnArgs a = a0;
  a.G = a.Hq / a.c.Hkv;
  a.inv_G = (unsigned)(((1ull << 31) + a.G - 1) / a.G);
  return a;
}

// Most query vectors per KV head of a call's groups.
int group_vectors(const PagedView& c, int n, int Hq) { return c.S * n * (Hq / c.Hkv); }  // at most 2^22

// Items of the groups at most: full tiles, and one more for each group (of two sequences or more).
size_t group_items(const PagedView& c, int vectors, int cols) {
  return (size_t)c.Hkv * ((size_t)vectors / cols + (c.S + 1) / 2 + 1);
}

// One slot for each run that enters or leaves an item (of run r and item i: r + i).
size_t slots_floats(const PagedView& c, int vectors, const GroupShape& g) {
  return (g.runs + group_items(c, vectors, g.cols)) * g.cols * (c.D + 2);
}

size_t at_floats(const PagedView& c) { return ((size_t)(c.S + 1) * 4 + 63) / 64 * 64; }

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

hipError_t paged_attention(const PagedAttnArgs& a, hipStream_t s) {
  return launch_type<WHOLE>(with_groups(a), a.n * (a.Hq / a.c.Hkv), s);
}

static GroupShape shape_of(const PagedView& c, int vectors) {
  if (c.esz == 2) return group_shape(c, vectors);
  const int nt = tiles_for(c, vectors);
  return GroupShape{16 * nt, item_cost(nt), kStep, runs_for(c, vectors)};
}

bool paged_attention_shared_fits(const PagedView& c, int n, int Hq) {
  const int vectors = group_vectors(c, n, Hq);
  const GroupShape g = shape_of(c, vectors);
  const double units = (double)group_items(c, vectors, g.cols) * (std::ceil((double)c.width * c.ps / g.step) + g.cost);
  return paged_attention_fits(c, n, Hq) && units < 274877906944.0;
}

size_t paged_attention_shared_workspace_floats(const PagedView& c, int n, int Hq) {
  const int vectors = group_vectors(c, n, Hq);
  const GroupShape g = shape_of(c, vectors);
  return at_floats(c) + slots_floats(c, vectors, g) + paged_attention_workspace_floats(c, n, Hq);
}

hipError_t paged_attention_shared(const PagedAttnArgs& a0, const int* plan, hipStream_t s) {
  PagedAttnArgs a = with_groups(a0);
  const int vectors = group_vectors(a.c, a.n, a.Hq);
  const GroupShape g = shape_of(a.c, vectors);
  a.plan = (int*)plan;
  a.at = a.ws;
  a.slots = a.ws + at_floats(a.c);
  a.s_cols = g.cols;
  a.s_cost = g.cost;
  a.s_step = g.step;
  a.ws = a.slots + slots_floats(a.c, vectors, g);
  if (hipError_t e = a.c.esz == 2 ? paged_group(a, g.runs, s) : launch_dim<SHARED, float>(a, vectors, s)) return e;
  return launch_type<OWN>(a, a.n * a.G, s);
}

}  // namespace rgd
