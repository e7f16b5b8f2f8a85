// What the attention kernels over pages share (internal): running softmax constants, the wave's sums of units, MFMA and
// page lookups.
#pragma once
#include "paged.hpp"

namespace rgd {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;       // the running maximum moves when a score passes it by this (log2 units)
constexpr float kLift = 256.f;     // 2^kLazy: weights are held divided by it, so none is above 1 and no sum above that of |V|
constexpr float kNoRef = -3.0e38f; // the maximum before any visible score: finite, so a masked one gives 0, never NaN

RGD_DEV int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

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

// Floor of x / y for 0 <= x < 2^52, 0 < y.  Exact: a quotient that is no whole number
// is at least 1 / y, more than 2^-52 of itself, away from the next one.
RGD_DEV long long quotient(long long x, long long y) { return (long long)((double)x / (double)y); }

RGD_DEV f32x4 mfma_bf16(const u32x4& x, const u32x4& y, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}
RGD_DEV f32x4 mfma_f32(float x, float y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, c, 0, 0, 0); }

RGD_DEV float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

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
  // of the first 64 pages: no load, for which those on their way would be waited for
  RGD_DEV int find_near(int block, int& place) const {
    const int j = page_index(block);
    place = block - j * bpp;
    return __builtin_amdgcn_readlane(cur, j - jb);
  }
};

RGD_DEV float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + __log2f(l * kLift)) * kLn2; }

}  // namespace rgd
