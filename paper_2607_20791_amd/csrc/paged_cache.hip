// Page operators of paged sequences: forking and rolling back (tables and
// reference counts), reserving pages with copy-on-write, compaction, and the
// append of new K/V rows.
#include <algorithm>

#include "paged.hpp"

namespace rgd {

namespace {

// ---------------------------------------------------------------- select ----
// What every sequence becomes, put aside before any table changes (a parent may
// itself become another sequence): its new length and its parent's entries.  A launch of its
// own, because all tables are read before one changes.  288 sequences: 3.9 us, and 3.1 us for
// the next kernel, a launch and two dependent reads each.
__global__ __launch_bounds__(256) void select_stage_kernel(PagedView c, const int* parent, const int* keep,
                                                           int* new_len, int* staged) {
  const int s = blockIdx.x;
  int p = parent[s];
  if ((unsigned)p >= (unsigned)c.S) p = s;
  int len = paged_len(c, p);
  if (keep && keep[s] >= 0) len = min(len, keep[s]);
  if (threadIdx.x == 0) new_len[s] = len;
  if (p == s) return;
  const int used = pages_of(c, len);
  for (int j = threadIdx.x; j < used; j += 256)
    staged[(size_t)s * c.width + j] = c.pages[(size_t)p * c.width + j];
}

// Reference counts move by one for each entry that changes: integer sums, whose
// order does not matter.
__global__ __launch_bounds__(256) void select_apply_kernel(PagedView c, const int* parent, const int* keep,
                                                           const int* new_len, const int* staged) {
  const int s = blockIdx.x;
  const int old = paged_len(c, s);
  bool self = true;
  int len = old;
  if (parent) {
    const int p = parent[s];
    self = (unsigned)p >= (unsigned)c.S || p == s;
    len = new_len[s];
  } else if (keep[s] >= 0) {
    len = min(len, keep[s]);
  }
  const int had = pages_of(c, old), used = pages_of(c, len);
  int* row = c.pages + (size_t)s * c.width;
  for (int j = (self ? used : 0) + threadIdx.x; j < max(had, used); j += 256) {
    const int was = j < had ? row[j] : -1;
    const int is = j < used ? staged[(size_t)s * c.width + j] : -1;
    row[j] = is;
    if (was == is) continue;
    if (page_ok(c, was)) atomicSub(c.refs + was, 1);
    if (page_ok(c, is)) atomicAdd(c.refs + is, 1);
  }
  __syncthreads();  // every thread has read the old length
  if (threadIdx.x == 0) c.lens[s] = len;
}

// --------------------------------------------------------------- reserve ----
constexpr int kPlan = 1024;  // threads of the one planning workgroup

// Sum of v over the threads before this one; total receives the whole sum.
// red: kPlan / 64 ints.
RGD_DEV int block_exclusive_scan(int v, int* red, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(incl, o, 64);
    if (lane >= o) incl += t;
  }
  __syncthreads();
  if (lane == 63) red[w] = incl;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kPlan / 64; ++i) {
    const int t = red[i];
    before += i < w ? t : 0;
    all += t;
  }
  total = all;
  return before + incl - v;
}

// Pages are looked through kLook * kPlan at a time, kLook loads of a thread in flight.
constexpr int kLook = 16;
struct PageLook {
  int refs[kLook];
  RGD_DEV void load(const PagedView& c, int p0) {
#pragma unroll
    for (int k = 0; k < kLook; ++k) refs[k] = c.refs[min(p0 + k * kPlan + (int)threadIdx.x, c.n_pages - 1)];
  }
};

struct LookCounts {
  int before[kLook * kPlan / 64];  // hits ahead of each 64 pages
  int total;
};

// Appends the pages of [p0, p0 + kLook * kPlan) whose bit k of `hits` is set (page
// p0 + k * kPlan + thread) to list[found ..), up to `most` entries in all; returns the
// new number of hits found.
RGD_DEV int list_pages(unsigned hits, int p0, int found, int most, int* list, LookCounts& n) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kLook; ++k) {
    const unsigned long long all = __ballot(hits >> k & 1);
    if (lane == 0) n.before[k * (kPlan / 64) + w] = __popcll(all);
  }
  __syncthreads();
  if (w == 0) {
    constexpr int PER = kLook * kPlan / 64 / 64;
    int c[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      c[i] = n.before[PER * lane + i];
      sum += c[i];
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o, 64);
      if (lane >= o) incl += v;
    }
    int at = incl - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      n.before[PER * lane + i] = at;
      at += c[i];
    }
    if (lane == 63) n.total = incl;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kLook; ++k) {
    const bool hit = hits >> k & 1;
    const unsigned long long all = __ballot(hit);
    const int at = found + n.before[k * (kPlan / 64) + w] + __popcll(all & ((1ull << lane) - 1));
    if (hit && at < most) list[at] = p0 + k * kPlan + (int)threadIdx.x;
  }
  return found + n.total;
}

// One workgroup: the pages every sequence needs, the lowest free ones, and the
// tables, counts and lengths that follow.  ws: [0] number of copies, then the
// (from, to) pairs [2 S], the sequences' first list entries [S], the page each
// gives up for a copy of its own or -1 [S], the list.  288 sequences and 4000 pages:
// 8.6 us, a chain of dependent reads (length, last page, its count, list entries) and seven
// barriers.  granted (or null) may be grow: a sequence's entries are read and written by one thread.
__global__ __launch_bounds__(kPlan) void reserve_plan_kernel(PagedView c, const int* grow, int* granted, int* ws) {
  __shared__ int red[kPlan / 64];
  __shared__ LookCounts counts;
  __shared__ int over, ncopy;
  int* pairs = ws + 4;
  int* first = pairs + 2 * c.S;
  int* given = first + c.S;
  int* list = given + c.S;
  PageLook look;
  look.load(c, 0);  // on its way while the needs are worked out
  if (threadIdx.x == 0) {
    over = 0;
    ncopy = 0;
  }
  __syncthreads();
  long long want = 0;
  for (int s0 = 0; s0 < c.S; s0 += kPlan) {
    const int s = s0 + threadIdx.x;
    int need = 0;
    if (s < c.S) {
      const int len = paged_len(c, s), g = max(grow[s], 0), used = pages_of(c, len);
      const int last = used ? c.pages[(size_t)s * c.width + used - 1] : -1;
      const bool copy = g > 0 && len % c.ps && page_ok(c, last) && c.refs[last] > 1;
      const long long end = (long long)len + g;
      if (end > (long long)c.width * c.ps) {
        over = 1;
      } else {
        need = pages_of(c, (int)end) - used + copy;
        if (need > c.n_pages) {
          over = 1;
          need = 0;
        }
      }
      given[s] = copy ? last : -1;
    }
    int total;
    const int at = block_exclusive_scan(need, red, total);  // 1024 needs of at most 2^20
    if (s < c.S) first[s] = (int)min(want + at, (long long)c.n_pages);
    want += total;
  }
  int found = 0;
  if (want <= c.n_pages)
    for (int p0 = 0; p0 < c.n_pages && found < want; p0 += kLook * kPlan) {
      if (p0) look.load(c, p0);
      unsigned hits = 0;
#pragma unroll
      for (int k = 0; k < kLook; ++k)
        hits |= look.refs[k] == 0 && p0 + k * kPlan + (int)threadIdx.x < c.n_pages ? 1u << k : 0u;
      found = list_pages(hits, p0, found, (int)want, list, counts);
    }
  __syncthreads();
  if (over || found < want) {
    if (threadIdx.x == 0) {
      ws[0] = 0;
      *c.status = 1;
    }
    if (granted)
      for (int s = threadIdx.x; s < c.S; s += kPlan) granted[s] = 0;
    return;
  }
  for (int s = threadIdx.x; s < c.S; s += kPlan) {  // the threads that wrote first and given
    const int g = max(grow[s], 0);
    if (granted) granted[s] = g;
    if (!g) continue;
    const int len = paged_len(c, s), used = pages_of(c, len), after = pages_of(c, len + g), from = given[s];
    int* row = c.pages + (size_t)s * c.width;
    int at = first[s];
    if (from >= 0) {
      const int to = list[at++], i = atomicAdd(&ncopy, 1);
      pairs[2 * i] = from;
      pairs[2 * i + 1] = to;
      row[used - 1] = to;
      c.refs[to] = 1;
      atomicSub(c.refs + from, 1);
    }
    for (int k = used; k < after; ++k) {
      const int p = list[at++];
      row[k] = p;
      c.refs[p] = 1;
    }
    c.lens[s] = len + g;
  }
  __syncthreads();
  if (threadIdx.x == 0) ws[0] = ncopy;
}

// Page `from` of one layer of one pool to page `to`: bytes (a multiple of 16) by
// the whole workgroup, eight requests of a thread in flight.  A page of one layer is 32 KB in the
// common sizes, enough for a workgroup; which pages are copied is known on the device only, so a fixed
// grid takes them in turn.  Stores go past the caches; so do loads where each page is read once (ONCE).
template <bool ONCE>
RGD_DEV void copy_page(char* pool, size_t page_bytes, size_t layer_page0, int from, int to) {
  const u32x4* src = (const u32x4*)(pool + (layer_page0 + from) * page_bytes);
  u32x4* dst = (u32x4*)(pool + (layer_page0 + to) * page_bytes);
  const size_t n = page_bytes / 16;
  auto load = [&](size_t i) { return ONCE ? __builtin_nontemporal_load(src + i) : src[i]; };
  size_t i = threadIdx.x;
  for (; i + 7 * 256 < n; i += 8 * 256) {
    u32x4 v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = load(i + 256 * k);
#pragma unroll
    for (int k = 0; k < 8; ++k) __builtin_nontemporal_store(v[k], dst + i + 256 * k);
  }
  for (; i < n; i += 256) __builtin_nontemporal_store(load(i), dst + i);
}

// The pages that reserve copies.  Branches of 32 prompts grow from their prompts' last pages, 8 layers of 32 KB
// K and V pages, 117 MB read and written: 12.4 us, 9 TB/s, as a prompt's page is read once for all its branches
// (20 us with cached stores or with loads past the caches, 17 with cached stores and eight requests in flight).
__global__ __launch_bounds__(256) void copy_pairs_kernel(PagedView c, const int* ws, size_t page_bytes) {
  const int n = ws[0];
  const int* pairs = ws + 4;
  const long long items = (long long)n * 2 * c.L;
  for (long long i = blockIdx.x; i < items; i += gridDim.x) {
    const int k = (int)(i / (2 * c.L)), which = (int)(i % (2 * c.L));
    copy_page<false>(which & 1 ? c.pool_v : c.pool_k, page_bytes, (size_t)(which >> 1) * c.n_pages, pairs[2 * k],
              pairs[2 * k + 1]);
  }
}

// --------------------------------------------------------------- compact ----
// One workgroup: the number n of live pages, then in order the free pages below
// n and the live ones at or above it (as many of each).  ws: [0] moves, map
// [n_pages], list [n_pages].  16384 pages: 8.1 us (29.6 with one
// load a thread in flight).
__global__ __launch_bounds__(kPlan) void compact_plan_kernel(PagedView c, int* live, int* ws) {
  __shared__ int red[kPlan / 64];
  __shared__ LookCounts counts;
  int* map = ws + 4;
  int* list = map + c.n_pages;
  constexpr int SPAN = kLook * kPlan;
  PageLook look;
  int n = 0;
  for (int p0 = 0; p0 < c.n_pages; p0 += SPAN) {
    look.load(c, p0);
    int mine = 0, total;
#pragma unroll
    for (int k = 0; k < kLook; ++k) mine += look.refs[k] > 0 && p0 + k * kPlan + (int)threadIdx.x < c.n_pages;
    block_exclusive_scan(mine, red, total);
    n += total;
  }
  int found = 0;
  for (int p0 = 0; p0 < c.n_pages; p0 += SPAN) {
    if (c.n_pages > SPAN) look.load(c, p0);
    unsigned hits = 0;
#pragma unroll
    for (int k = 0; k < kLook; ++k) {
      const int p = p0 + k * kPlan + (int)threadIdx.x;
      hits |= p < c.n_pages && (p < n) == (look.refs[k] <= 0) ? 1u << k : 0u;
      if (p < c.n_pages) map[p] = p;
    }
    found = list_pages(hits, p0, found, c.n_pages, list, counts);
  }
  __syncthreads();
  const int moves = found / 2;
  for (int i = threadIdx.x; i < moves; i += kPlan) {
    const int to = list[i], from = list[moves + i];
    map[from] = to;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    ws[0] = moves;
    *live = n;
  }
}

// The tables follow the map, then the pages move, each read and written once.  1.04 GB read and written:
// 194 us, 5.3 TB/s, what a large copy reaches, and no more at the memory than these bytes (198 us with
// cached loads, 203 with cached stores too, 207 with one request in flight).
__global__ __launch_bounds__(256) void compact_move_kernel(PagedView c, const int* ws, size_t page_bytes) {
  const int moves = ws[0];
  const int* map = ws + 4;
  const int* list = map + c.n_pages;
  for (int s = blockIdx.x; s < c.S; s += gridDim.x) {
    const int used = pages_of(c, paged_len(c, s));
    int* row = c.pages + (size_t)s * c.width;
    for (int j = threadIdx.x; j < used; j += 256) {
      const int p = row[j];
      if (page_ok(c, p) && map[p] != p) row[j] = map[p];
    }
  }
  const long long items = (long long)moves * 2 * c.L;
  for (long long i = blockIdx.x; i < items; i += gridDim.x) {
    const int k = (int)(i / (2 * c.L)), which = (int)(i % (2 * c.L));
    copy_page<true>(which & 1 ? c.pool_v : c.pool_k, page_bytes, (size_t)(which >> 1) * c.n_pages, list[moves + k], list[k]);
  }
}

// ---------------------------------------------------------------- append ----
// One workgroup per (16 positions that lie together in a page, KV head, sequence): K
// rows are copied as they come, V goes through LDS, whose columns are the rows of the
// pages' transposed V.  Whole runs are read and written 16 bytes at a time; the borders of a
// sequence's new positions one value at a time.  8 x 1000 tokens of 8 heads, bf16: 10.6 us
// (36 MB read and written, 22 us with a value a thread).
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(PagedView c, T* pk, T* pv, const T* k, const T* v, long long ldk,
                                                     long long ldv, int n, const int* n_new, int blocks) {
  constexpr int E = 16 / sizeof(T);  // values per 16 bytes
  __shared__ T vt[128][16 + E];
  const int s = blockIdx.x / blocks, h = blockIdx.y;
  const int m = n_new ? min(max(n_new[s], 0), n) : n;
  const int len = paged_len(c, s), base = len - m;  // position of token 0
  const int p0 = (max(base, 0) / 16 + (int)blockIdx.x % blocks) * 16;
  if (m == 0 || p0 >= len) return;
  const int lo = max(base - p0, 0), hi = min(len - p0, 16);  // the block's positions that are new
  const int page = c.pages[(size_t)s * c.width + p0 / c.ps];
  const int per = c.D / E;  // 16-byte pieces of a row
  const size_t row0 = (size_t)s * n + (p0 - base);  // token of the block's first position (from lo on)
  const bool ok = page_ok(c, page);
  const size_t head = ((size_t)(ok ? page : 0) * c.Hkv + h) * c.ps * c.D;
  const int slot = p0 % c.ps;
  for (int i = threadIdx.x; i < 16 * per; i += 256) {
    const int t = i / per, d = i % per * E;
    if (t < lo || t >= hi) continue;
    const size_t r = row0 + t;
    const u32x4 kk = *(const u32x4*)(k + r * ldk + h * c.D + d), vv = *(const u32x4*)(v + r * ldv + h * c.D + d);
    if (ok) *(u32x4*)(pk + head + (size_t)(slot + t) * c.D + d) = kk;
    const T* x = (const T*)&vv;
#pragma unroll
    for (int e = 0; e < E; ++e) vt[d + e][t] = x[e];
  }
  __syncthreads();
  if (!ok) return;
  for (int i = threadIdx.x; i < c.D * (16 / E); i += 256) {
    const int d = i / (16 / E), t = i % (16 / E) * E;
    T* dst = pv + head + (size_t)d * c.ps + slot + t;
    if (t >= lo && t + E <= hi) {
      *(u32x4*)dst = *(const u32x4*)&vt[d][t];
    } else {
      for (int e = 0; e < E; ++e)
        if (t + e >= lo && t + e < hi) dst[e] = vt[d][t + e];
    }
  }
}

}  // namespace

size_t paged_workspace_ints(const PagedView& c) {
  const size_t select = (size_t)c.S + (size_t)c.S * c.width;
  const size_t reserve = 4 + 4 * (size_t)c.S + c.n_pages;
  const size_t compact = 4 + 2 * (size_t)c.n_pages;
  return std::max(select, std::max(reserve, compact));
}

hipError_t paged_select(const PagedView& c, const int* parent, const int* keep, int* ws, hipStream_t s) {
  if (!parent && !keep) return hipSuccess;
  int* staged = ws ? ws + c.S : nullptr;
  if (parent) hipLaunchKernelGGL(select_stage_kernel, dim3(c.S), dim3(256), 0, s, c, parent, keep, ws, staged);
  hipLaunchKernelGGL(select_apply_kernel, dim3(c.S), dim3(256), 0, s, c, parent, keep, ws, staged);
  return hipGetLastError();
}

hipError_t paged_reserve(const PagedView& c, const int* grow, int* granted, int* ws, hipStream_t s) {
  hipLaunchKernelGGL(reserve_plan_kernel, dim3(1), dim3(kPlan), 0, s, c, grow, granted, ws);
  const int blocks = (int)std::min<long long>(4096, 2LL * c.L * c.S);
  hipLaunchKernelGGL(copy_pairs_kernel, dim3(blocks), dim3(256), 0, s, c, ws, c.page_elems() * c.esz);
  return hipGetLastError();
}

hipError_t paged_compact(const PagedView& c, int* live, int* ws, hipStream_t s) {
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kPlan), 0, s, c, live, ws);
  const int blocks = (int)std::min<long long>(4096, std::max<long long>(c.S, 2LL * c.L * c.n_pages));
  hipLaunchKernelGGL(compact_move_kernel, dim3(blocks), dim3(256), 0, s, c, ws, c.page_elems() * c.esz);
  return hipGetLastError();
}

hipError_t paged_append(const PagedView& c, int layer, const void* k, const void* v, long long ldk, long long ldv,
                        int n, const int* n_new, hipStream_t s) {
  const size_t at = (size_t)layer * c.n_pages * c.page_elems();
  const int blocks = (n + 14) / 16 + 1;  // that n positions can touch
  const dim3 grid(blocks * c.S, c.Hkv);
  if (c.esz == 2)
    hipLaunchKernelGGL(append_kernel<bf16_t>, grid, dim3(256), 0, s, c, (bf16_t*)c.pool_k + at,
                       (bf16_t*)c.pool_v + at, (const bf16_t*)k, (const bf16_t*)v, ldk, ldv, n, n_new, blocks);
  else
    hipLaunchKernelGGL(append_kernel<float>, grid, dim3(256), 0, s, c, (float*)c.pool_k + at, (float*)c.pool_v + at,
                       (const float*)k, (const float*)v, ldk, ldv, n, n_new, blocks);
  return hipGetLastError();
}

}  // namespace rgd
