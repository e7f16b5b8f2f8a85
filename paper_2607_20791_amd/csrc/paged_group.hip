// Attention of groups of sequences over the leading pages that they share, bf16: the first of the two parts of
// rgd_paged_attention_shared (paged_attention.hip has the second, and both for fp32).
//
// A group's query vectors (its sequences' tokens x query heads of a KV head) all see all of its shared positions, so no score is
// masked but those of pages that are not there.  128 of them are an item; the positions of all items lie one behind the
// other in steps of 64, and every workgroup takes an equal run of steps.  Where a run enters or leaves an item it leaves
// a piece: sums weighted against a reference of the piece's own, which the second part joins.
//
// Many query vectors read the same keys and values, so these come to LDS once for a workgroup, by copies that pass no
// register, three steps ahead of the products.  Of the eight waves four share out the query vectors, 32 each (two tiles
// for every fragment that is read from LDS), and two the positions, 32 each; they meet in LDS at an item's end.  Both
// arrays lie there in 16-byte chunks whose places are exchanged within a row, so that the 16 lanes that read at a time
// hit all banks.
//
// Measured, 32 query heads, 8 KV heads of 128: 64 branches of 8192 positions (34 MB of keys and values, 256 query vectors a
// KV head) 31 us; 32 prompts of 1024 with 8 branches each (134 MB) 31 us, 4.3 TB/s; 4 of 4095 with 16 branches of 5 tokens
// 47 us.  Of the first some 7 us pass until the first step is there (lengths, table, keys), a step takes 1.9, the
// end 3.  By counters over all of it a SIMD's matrix unit is at work for 23% of the clocks (16 a product of 16 x 16 x 32) and its
// vector instructions for 35% (4.3 each), 7% at the same time, LDS for 14% of a CU's; waves wait for copies or at barriers for
// 48% of their time and to be issued for 23%.  So no unit is what bounds a step, but that its parts follow each other: eight waves, two a
// SIMD, pass one barrier a step.  One kernel for all groups that read keys and values through registers, a wave for 16 to 64
// query vectors, took 44 and 45 us of the first two.
#include <algorithm>
#include <cmath>

#include "dma.hpp"
#include "paged.hpp"
#include "paged_tiles.hpp"
#include "share.hpp"

namespace rgd {

namespace {

constexpr int kCols = 128;  // query vectors of an item
constexpr int kTile = 64;   // positions of a step
constexpr int kCost = 4;    // what an item costs besides its steps, in steps
constexpr int kRuns = 256;  // one workgroup per CU
constexpr int kBlocks = kTile / 16;
constexpr int kRing = 4;    // steps in LDS: one at work, the others on their way

struct Group {
  int len, tokens, row, steps, tiles;
};
RGD_DEV Group group_of(const PagedAttnArgs& a, int len, int tokens, int row) {
  return Group{len, tokens, row, (len + kTile - 1) / kTile, (tokens * a.G + kCols - 1) / kCols};
}

// One item of a run: steps [t0, t1) of query vectors [kCols qb, ...) of KV head g of the group of leader s.
struct Item {
  Group gr;
  int s, g, qb, t0, t1, number;
  bool valid;
};

struct Walk {
  Group gr;
  int s, g, qb, u0, left, number;
  RGD_DEV Item next(const PagedAttnArgs& a) {
    typedef const int __attribute__((address_space(4))) * Scalar;
    Item it{};
    if (left <= 0) return it;
    if (g == a.c.Hkv) {  // steps are left, so a group with tokens follows
      g = 0;
      do {
        Scalar p = (Scalar)Plan(a.plan, a.c.S).group + 4 * ++s;
        gr = group_of(a, p[0], p[1], p[2]);
      } while (gr.tiles == 0);
    }
    // an item's first kCost units are its fixed cost, in front of its steps
    const int u1 = min(gr.steps + kCost, u0 + left);
    it.gr = gr;
    it.s = s;
    it.g = g;
    it.qb = qb;
    it.t0 = max(0, u0 - kCost);
    it.t1 = u1 - kCost;
    it.valid = it.t1 > it.t0;  // else the next run has the item's first step
    it.number = number++;
    left -= u1 - u0;
    u0 = 0;
    if (++qb == gr.tiles) {
      qb = 0;
      ++g;
    }
    return it;
  }
};

RGD_DEV const char* same_for_all(const char* p) {
  const unsigned long long v = (unsigned long long)p;
  const unsigned lo = uniform((int)v), hi = uniform((int)(v >> 32));
  return (const char*)((unsigned long long)hi << 32 | lo);
}

// Chunk places: the chunk of a row of K that position p of 32 has in place c, and back (its own inverse).
template <int D>
RGD_DEV int k_place(int p, int c) {
  const int r = (p & 3) | (p >> 1 & 12);  // the lane that reads it
  return D == 128 ? c ^ r : D == 64 ? c ^ (r >> 1) : c ^ (r >> 2);
}
// of a 16-position row of V^T, two chunks
RGD_DEV int v_place(int d, int half) { return half ^ (d >> 3 & 1); }

template <int D>
__global__ __launch_bounds__(512, 2) void group_run_kernel(PagedAttnArgs a, int runs) {
  constexpr int KL = D / 32, VL = D / 16, ROW = D * 2;
  constexpr int BLOCK = 16 * ROW, LOADS = BLOCK / 1024, BUF = 2 * kBlocks * BLOCK;  // bytes; K's blocks, then V's
  __shared__ __attribute__((aligned(1024))) unsigned char lds[kRing * BUF];
  __shared__ int ok_s[kRing][kBlocks];
  __shared__ float2 ml_s[kCols / 2];
  // Workgroups that are 8 apart share an XCD and its L2: these get neighbouring runs, which read the same keys and values for
  // other query vectors.
  const int b = blockIdx.x, r = runs % 8 || b == runs ? b : b % 8 * (runs / 8) + b / 8, lane = threadIdx.x & 63,
            row = lane & 15, grp = lane >> 4, S = a.c.S, G = a.G;
  const int wave = uniform(threadIdx.x >> 6), cg = wave >> 1, pg = wave & 1;
  const Plan plan(a.plan, S);
  const bool mine = *plan.head == PlanHead::of(a.c, a.n, a.Hq);

  // the run: its first group, the units and items ahead of that
  auto units = [&](int s, long long& items) {
    const PlanGroup p = plan.group[min(s, S - 1)];
    const Group q = group_of(a, p.shared, p.tokens, p.row);
    items = s < S && mine ? a.c.Hkv * q.tiles : 0;
    return items * (q.steps + kCost);
  };
  long long total = 0, n;
  for (int s = lane; s < S; s += 64) total += units(s, n);
  total = lane_value(wave_scan(total), 63);
  const long long length = max(1ll, quotient(total + runs - 1, runs)), start = r * length;
  if (r == runs) {  // a workgroup beside the runs': where each group's units and items begin
    if (wave > 0) return;
    GroupAt* at = (GroupAt*)a.at;
    long long before = 0, items = 0;
    for (int s0 = 0; s0 < S; s0 += 64) {
      const long long u = units(s0 + lane, n), ui = wave_scan(u), ni = wave_scan(n);
      if (s0 + lane < S) at[s0 + lane] = GroupAt{before + ui - u, (int)(items + ni - n), 0};
      before += lane_value(ui, 63);
      items += lane_value(ni, 63);
    }
    if (lane == 0) at[S] = GroupAt{length, 0, 0};
    return;
  }
  if (start >= total) return;
  Walk walk;
  long long before = 0, items = 0;
  for (int s0 = 0;; s0 += 64) {
    const long long u = units(s0 + lane, n), ui = wave_scan(u), ni = wave_scan(n);
    if (const unsigned long long hit = __ballot(before + ui > start)) {
      const int l = __builtin_ctzll(hit);
      before += lane_value(ui - u, l);
      items += lane_value(ni - n, l);
      walk.s = uniform(s0 + l);
      break;
    }
    before += lane_value(ui, 63);
    items += lane_value(ni, 63);
  }
  {
    typedef const int __attribute__((address_space(4))) * Scalar;
    Scalar p = (Scalar)plan.group + 4 * walk.s;
    walk.gr = group_of(a, p[0], p[1], p[2]);
    const int per = walk.gr.steps + kCost, item = uniform((int)quotient(start - before, per));
    walk.g = item / walk.gr.tiles;
    walk.qb = item - walk.g * walk.gr.tiles;
    walk.u0 = uniform((int)(start - before - (long long)item * per));
    walk.left = uniform((int)min(length, total - start));
    walk.number = uniform((int)items) + item;
  }

  // What a wave copies of a step: K (waves 0 to 3) or V of one block, chunk i * 64 + lane.
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  const int mine_b = wave & 3;
  const bool is_v = wave >= 4;
  uint32_t off[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int q = i * 64 + lane, p = q / (ROW / 16), d = q >> 1;
    off[i] = is_v ? (uint32_t)d * a.c.ps * 2 + v_place(d, q & 1) * 16 : p * ROW + k_place<D>((mine_b & 1) * 16 + p, q % (ROW / 16)) * 16;
  }
  // The steps of the run's items in their order, as far ahead as there is room; a block that is not there is copied
  // from the pool's first page, so that every step is as many copies.
  Walk ahead = walk;
  Item load = ahead.next(a);
  TableWalk table;
  int load_step = load.t0, to = 0, on_way = 0;
  auto copy = [&] {
    if (!load.valid) return;
    const int block = load_step * kBlocks + mine_b;
    int place = 0, page = 0;
    bool ok = block * 16 < load.gr.len;
    if (ok) {
      page = uniform(table.find(block, place));
      ok = page_ok(a.c, page);
      if (!ok) page = place = 0;
    }
    const size_t head = ((size_t)page * a.c.Hkv + uniform(load.g)) * a.c.ps * D;
    const char* base = same_for_all(is_v ? (const char*)a.pool_v + (head + (size_t)place * 16) * 2
                                         : (const char*)a.pool_k + (head + (size_t)place * 16 * D) * 2);
    const uint32_t dst = uniform(lds0 + to * BUF + wave * BLOCK);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) dma16<0, 0>(base, off[i], dst + i * 1024);
    if (lane == 0 && !is_v) ok_s[to][mine_b] = ok;
    to = (to + 1) % kRing;
    ++on_way;
    if (++load_step == load.t1) {
      load = ahead.next(a);
      load_step = load.t0;
      if (load.valid) {
        table.start(a.c, load.s, load.t0 * kBlocks + mine_b);
        asm volatile("" ::"v"(table.cur), "v"(table.nxt));
      }
    }
  };

  // the lane's query vectors of an item: rows and heads
  int rows[2], heads[2];
  auto find_rows = [&](const Item& it) {
    const int cols = it.gr.tokens * G;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int col = min(it.qb * kCols + cg * 32 + t * 16 + row, cols - 1), i = (int)__umulhi((unsigned)col << 1, a.inv_G);
      rows[t] = plan.rows[it.gr.row + i];
      heads[t] = it.g * G + col - i * G;
    }
  };

  // the oldest step on its way is there (in each wave's order of copies)
  auto arrive = [&] {
    if (on_way >= 3) dma_wait_barrier<2 * LOADS>();
    else if (on_way == 2) dma_wait_barrier<LOADS>();
    else dma_wait_barrier<0>();
    --on_way;
  };

  Item it = walk.next(a);
  if (it.valid) {
    find_rows(it);
    table.start(a.c, load.s, load.t0 * kBlocks + mine_b);
  }
  for (int i = 0; i < kRing - 1; ++i) copy();
  int buf = 0;
  const float scale = kLog2e / sqrtf((float)D);
  while (it.valid) {
    const int cols = min(kCols, it.gr.tokens * G - it.qb * kCols);  // of the item
    u32x4 q[2][KL];
    f32x4 o[2][VL];
    float m[2], l[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const char* src = (const char*)((const bf16_t*)a.q + (size_t)rows[t] * a.ldq + (size_t)heads[t] * D);
#pragma unroll
      for (int c = 0; c < KL; ++c) q[t][c] = *(const u32x4*)(src + c * 64 + grp * 16);
      m[t] = kNoRef;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < VL; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // waited for here: inside the loop it would be a wait for the copies on their way, too
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KL; ++c) asm volatile("" ::"v"(q[t][c]));
    const bool works = cg * 32 < cols;
    // the products of a step's keys with the wave's query vectors
    auto scores = [&](int slot, f32x4 (&s)[2][2]) {
      const unsigned char* kt = lds + slot * BUF + pg * 2 * BLOCK;
      u32x4 k[2][KL];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // row r of tile e: position (r >> 2) * 8 + e * 4 + (r & 3), so that a lane gets eight positions in a row
        const int p = (row >> 2) * 8 + e * 4 + (row & 3);
#pragma unroll
        for (int c = 0; c < KL; ++c) k[e][c] = *(const u32x4*)(kt + p * ROW + k_place<D>(p, c * 4 + grp) * 16);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) s[t][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KL; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) s[t][e] = mfma_bf16(k[e][c], q[t][c], s[t][e]);
    };
    f32x4 s[2][2];
    arrive();
    copy();
    if (works) scores(buf, s);
    for (int step = it.t0; step < it.t1; ++step) {
      // The next step is there, and every wave is done with the one before this; the first step of an item has no place to give.
      if (step + 1 < it.t1) arrive();
      else if (step > it.t0) lds_barrier();
      if (step > it.t0) copy();
      const int here = buf;
      buf = (buf + 1) % kRing;
      if (!works) continue;
      const int ok = uniform(ok_s[here][2 * pg] | ok_s[here][2 * pg + 1] << 1);  // this wave's two blocks
      const bool there = ok >> (grp >> 1) & 1;
      const unsigned char* vt = lds + here * BUF + pg * 2 * BLOCK + kBlocks * BLOCK;
      u32x4 v[VL];
#pragma unroll
      for (int d = 0; d < VL; ++d) {
        const int dim = d * 16 + row;
        v[d] = *(const u32x4*)(vt + (grp >> 1) * BLOCK + dim * 32 + v_place(dim, grp & 1) * 16);
      }
      float x[2][8];
      bool moves = false;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[t][j] = s[t][j / 4][j % 4];
        if (ok != 3)
#pragma unroll
          for (int j = 0; j < 8; ++j) x[t][j] = there ? x[t][j] : -INFINITY;
      }
      if (ok != 3)  // what an earlier step left in place of a block may be NaN
#pragma unroll
        for (int d = 0; d < VL; ++d) v[d] = there ? v[d] : u32x4{0, 0, 0, 0};
      float top[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float* y = x[t];
        top[t] = scale * fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
        moves = moves || top[t] > m[t];
      }
      if (__any(moves))
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          top[t] = fmaxf(top[t], __shfl_xor(top[t], 16, 64));
          top[t] = fmaxf(top[t], __shfl_xor(top[t], 32, 64));
          const float nm = fmaxf(m[t], top[t] + kLazy), down = exp2_raw(m[t] - nm);
          m[t] = nm;
          l[t] *= down;
#pragma unroll
          for (int d = 0; d < VL; ++d) o[t][d] *= down;
        }
      // The next step's products (behind the last step: of whatever lies there, not used), whose results are not waited for
      // then: this one's weights come in between.
      f32x4 s_next[2][2];
      scores(buf, s_next);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        // A weight is 2^(score - m), whose exponent is rounded once, at its own size; no score is above m, which moves to kLazy
        // above the one that passes it, so no weight is above 1.
        float w[8], sum = 0.f;
        u32x4 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          w[j] = exp2_raw(fmaf(x[t][j], scale, -m[t]));
          sum += w[j];
        }
        l[t] += sum;
        // a weight is the sum of two bf16, which leaves out 2^-17 of it
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          hi[j] = pack_bf16x2(w[2 * j], w[2 * j + 1]);
          lo[j] = pack_bf16x2(w[2 * j] - __uint_as_float(hi[j] << 16), w[2 * j + 1] - __uint_as_float(hi[j] & 0xFFFF0000u));
        }
#pragma unroll
        for (int d = 0; d < VL; ++d) o[t][d] = mfma_bf16(v[d], hi, o[t][d]);
#pragma unroll
        for (int d = 0; d < VL; ++d) o[t][d] = mfma_bf16(v[d], lo, o[t][d]);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) s[t][e] = s_next[t][e];
    }
    // The two halves of the positions meet in the step's place, which is free: of each pair of waves one takes the first
    // tile of query vectors, the other the second.
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      l[t] += __shfl_xor(l[t], 16, 64);
      l[t] += __shfl_xor(l[t], 32, 64);
    }
    float* part = (float*)(lds + (buf + kRing - 1) % kRing * BUF);
    const int c = cg * 16 + row;  // of 64 that meet at a time
    float* slot = a.slots + (size_t)(r + it.number) * kCols * (D + 2);
    const bool some = cg * 32 < cols;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      lds_barrier();
      if (pg != t && some) {
#pragma unroll
        for (int d = 0; d < VL; ++d) *(f32x4*)(part + c * D + ((d * 4 + grp) ^ (c & (D / 4 - 1) & 15)) * 4) = o[t][d];
        if (grp == 0) ml_s[c] = float2{m[t], l[t]};
      }
      lds_barrier();
      const int col = cg * 32 + t * 16 + row;
      if (pg == t && col < cols) {
        const float2 ml = ml_s[c];
        // (over kLift, as all pieces are)
        const float nm = fmaxf(m[t], ml.x), f0 = exp2_raw(m[t] - nm) * (1.f / kLift), f1 = exp2_raw(ml.x - nm) * (1.f / kLift);
#pragma unroll
        for (int d = 0; d < VL; ++d) {
          const f32x4 x = *(const f32x4*)(part + c * D + ((d * 4 + grp) ^ (c & (D / 4 - 1) & 15)) * 4);
          *(f32x4*)(slot + col * D + d * 16 + grp * 4) = o[t][d] * f0 + x * f1;
        }
        if (grp == 0) *(float2*)(slot + kCols * D + 2 * col) = float2{nm, l[t] * f0 + ml.y * f1};
      }
    }
    it = walk.next(a);
    if (it.valid) find_rows(it);
  }
}

}  // namespace

GroupShape group_shape(const PagedView& c, int vectors) {
  GroupShape g{kCols, kCost, kTile, 0};
  const double items = (double)c.Hkv * (vectors / kCols + (c.S + 1) / 2 + 1);
  g.runs = (int)std::min<double>(kRuns, std::max(1.0, items * (std::ceil((double)c.width * c.ps / kTile) + kCost)));
  return g;
}

hipError_t paged_group(const PagedAttnArgs& a, int runs, hipStream_t s) {
  const dim3 grid(runs + 1), block(512);
  switch (a.c.D) {
    case 32: hipLaunchKernelGGL(group_run_kernel<32>, grid, block, 0, s, a, runs); break;
    case 64: hipLaunchKernelGGL(group_run_kernel<64>, grid, block, 0, s, a, runs); break;
    default: hipLaunchKernelGGL(group_run_kernel<128>, grid, block, 0, s, a, runs);
  }
  return hipGetLastError();
}

}  // namespace rgd
