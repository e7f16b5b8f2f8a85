// Page operators of paged sequences: forking and rolling back (tables and
// reference counts), reserving pages with copy-on-write, compaction, and the
// append of new K/V rows.
#include <algorithm>

#include "paged.hpp"

namespace rgd {

namespace {

// ---------------------------------------------------------------- select ----
// What every sequence becomes, put aside before any table changes (a parent may
// itself become another sequence): its new length and its parent's entries.
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

struct Need {
  int len, grow, used, after, copy, last;  // copy: the last page is another entry's too
};

RGD_DEV Need need_of(const PagedView& c, const int* grow, int s) {
  Need n;
  n.len = paged_len(c, s);
  n.grow = max(grow[s], 0);
  n.used = pages_of(c, n.len);
  const long long end = (long long)n.len + n.grow;
  n.after = end > (long long)c.width * c.ps ? -1 : pages_of(c, (int)end);  // -1: more than a table holds
  n.last = n.used ? c.pages[(size_t)s * c.width + n.used - 1] : -1;
  n.copy = n.grow > 0 && n.len % c.ps && page_ok(c, n.last) && c.refs[n.last] > 1;
  return n;
}

// One workgroup: the pages every sequence needs, the lowest free ones, and the
// tables, counts and lengths that follow.  ws: [0] number of copies, then the
// (from, to) pairs [2 S], the sequences' first list entries [S], the list.
__global__ __launch_bounds__(kPlan) void reserve_plan_kernel(PagedView c, const int* grow, int* ws) {
  __shared__ int red[kPlan / 64];
  __shared__ int over, ncopy;
  int* pairs = ws + 4;
  int* first = pairs + 2 * c.S;
  int* list = first + c.S;
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
      const Need n = need_of(c, grow, s);
      need = n.after - n.used + n.copy;
      if (n.after < 0 || need > c.n_pages) {
        over = 1;
        need = 0;
      }
    }
    int total;
    const int at = block_exclusive_scan(need, red, total);  // 1024 needs of at most 2^20
    if (s < c.S) first[s] = (int)min(want + at, (long long)c.n_pages);
    want += total;
  }
  int found = 0;
  if (want <= c.n_pages)
    for (int p0 = 0; p0 < c.n_pages && found < want; p0 += kPlan) {
      const int p = p0 + threadIdx.x;
      const int free = p < c.n_pages && c.refs[p] == 0;
      int total;
      const int at = block_exclusive_scan(free, red, total);
      if (free && found + at < want) list[found + at] = p;
      found += total;
    }
  __syncthreads();
  if (over || found < want) {
    if (threadIdx.x == 0) {
      ws[0] = 0;
      *c.status = 1;
    }
    return;
  }
  // the needs are taken again before any count changes (a page given up below
  // may be the last page of a sequence handled later)
  for (int s0 = 0; s0 < c.S; s0 += kPlan) {
    const int s = s0 + threadIdx.x;
    if (s < c.S) {
      const Need n = need_of(c, grow, s);
      if (n.copy) {
        const int i = atomicAdd(&ncopy, 1);
        pairs[2 * i] = n.last;
        pairs[2 * i + 1] = s;
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < ncopy; i += kPlan) {
    const int from = pairs[2 * i], s = pairs[2 * i + 1];
    const int to = list[first[s]];
    c.pages[(size_t)s * c.width + pages_of(c, paged_len(c, s)) - 1] = to;
    pairs[2 * i + 1] = to;
    c.refs[to] = 1;
    first[s] += 1;
    atomicSub(c.refs + from, 1);
  }
  __syncthreads();
  for (int s = threadIdx.x; s < c.S; s += kPlan) {
    const int len = paged_len(c, s), g = max(grow[s], 0);
    const int used = pages_of(c, len), after = pages_of(c, len + g);
    for (int j = used; j < after; ++j) {
      const int p = list[first[s] + j - used];
      c.pages[(size_t)s * c.width + j] = p;
      c.refs[p] = 1;
    }
    c.lens[s] = len + g;
  }
  if (threadIdx.x == 0) ws[0] = ncopy;
}

// Page `from` of one layer of one pool to page `to`: bytes (a multiple of 16) by
// the whole workgroup.
RGD_DEV void copy_page(char* pool, size_t page_bytes, size_t layer_page0, int from, int to) {
  const u32x4* src = (const u32x4*)(pool + (layer_page0 + from) * page_bytes);
  u32x4* dst = (u32x4*)(pool + (layer_page0 + to) * page_bytes);
  const size_t n = page_bytes / 16;
  for (size_t i = threadIdx.x; i < n; i += 256) dst[i] = src[i];
}

__global__ __launch_bounds__(256) void copy_pairs_kernel(PagedView c, const int* ws, size_t page_bytes) {
  const int n = ws[0];
  const int* pairs = ws + 4;
  const long long items = (long long)n * 2 * c.L;
  for (long long i = blockIdx.x; i < items; i += gridDim.x) {
    const int k = (int)(i / (2 * c.L)), which = (int)(i % (2 * c.L));
    copy_page(which & 1 ? c.pool_v : c.pool_k, page_bytes, (size_t)(which >> 1) * c.n_pages, pairs[2 * k],
              pairs[2 * k + 1]);
  }
}

// --------------------------------------------------------------- compact ----
// One workgroup: the number n of live pages, then in order the free pages below
// n and the live ones at or above it (as many of each).  ws: [0] moves, map
// [n_pages], list [n_pages].
__global__ __launch_bounds__(kPlan) void compact_plan_kernel(PagedView c, int* live, int* ws) {
  __shared__ int red[kPlan / 64];
  int* map = ws + 4;
  int* list = map + c.n_pages;
  int n = 0;
  for (int p0 = 0; p0 < c.n_pages; p0 += kPlan) {
    const int p = p0 + threadIdx.x;
    int total;
    block_exclusive_scan(p < c.n_pages && c.refs[p] > 0, red, total);
    n += total;
  }
  int found = 0;
  for (int p0 = 0; p0 < c.n_pages; p0 += kPlan) {
    const int p = p0 + threadIdx.x;
    const int hit = p < c.n_pages && (p < n) == (c.refs[p] <= 0);
    int total;
    const int at = block_exclusive_scan(hit, red, total);
    if (hit) list[found + at] = p;
    if (p < c.n_pages) map[p] = p;
    found += total;
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
    copy_page(which & 1 ? c.pool_v : c.pool_k, page_bytes, (size_t)(which >> 1) * c.n_pages, list[moves + k], list[k]);
  }
}

// ---------------------------------------------------------------- append ----
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(PagedView c, T* pk, T* pv, const T* k, const T* v, long long ldk,
                                                     long long ldv, int n, const int* n_new) {
  const int s = blockIdx.y, i = blockIdx.x;
  const int m = n_new ? min(max(n_new[s], 0), n) : n;
  if (i >= m) return;
  const int pos = paged_len(c, s) - m + i;
  if (pos < 0) return;
  const int page = c.pages[(size_t)s * c.width + pos / c.ps];
  if (!page_ok(c, page)) return;
  const int slot = pos % c.ps;
  const size_t at = (size_t)page * c.Hkv * c.ps * c.D;
  const size_t row = (size_t)s * n + i;
  for (int e = threadIdx.x; e < c.Hkv * c.D; e += 256) {
    const int h = e / c.D, d = e % c.D;
    pk[at + ((size_t)h * c.ps + slot) * c.D + d] = k[row * ldk + e];
    pv[at + ((size_t)h * c.D + d) * c.ps + slot] = v[row * ldv + e];
  }
}

}  // namespace

size_t paged_workspace_ints(const PagedView& c) {
  const size_t select = (size_t)c.S + (size_t)c.S * c.width;
  const size_t reserve = 4 + 3 * (size_t)c.S + c.n_pages;
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

hipError_t paged_reserve(const PagedView& c, const int* grow, int* ws, hipStream_t s) {
  hipLaunchKernelGGL(reserve_plan_kernel, dim3(1), dim3(kPlan), 0, s, c, grow, ws);
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
  const dim3 grid(n, c.S);
  if (c.esz == 2)
    hipLaunchKernelGGL(append_kernel<bf16_t>, grid, dim3(256), 0, s, c, (bf16_t*)c.pool_k + at,
                       (bf16_t*)c.pool_v + at, (const bf16_t*)k, (const bf16_t*)v, ldk, ldv, n, n_new);
  else
    hipLaunchKernelGGL(append_kernel<float>, grid, dim3(256), 0, s, c, (float*)c.pool_k + at, (float*)c.pool_v + at,
                       (const float*)k, (const float*)v, ldk, ldv, n, n_new);
  return hipGetLastError();
}

}  // namespace rgd
