// Paged sequences (internal): the kernels' view of an rgd_paged_cache and the
// launch interface of its operators and of the draft verification.
#pragma once
#include "common.hpp"

namespace rgd {

struct PagedView {
  int L, n_pages, Hkv, ps, D, S, width;  // layers, pages, KV heads, page size, head dim, sequences, table entries
  size_t esz;                            // bytes per K/V element
  char *pool_k, *pool_v;
  int *pages, *lens, *refs, *status;
  size_t page_elems() const { return (size_t)Hkv * ps * D; }
};

// length of sequence s, inside what its table can hold
RGD_DEV int paged_len(const PagedView& c, int s) { return min(max(c.lens[s], 0), c.width * c.ps); }
RGD_DEV int pages_of(const PagedView& c, int len) { return (len + c.ps - 1) / c.ps; }
RGD_DEV bool page_ok(const PagedView& c, int p) { return (unsigned)p < (unsigned)c.n_pages; }

size_t paged_workspace_ints(const PagedView& c);
hipError_t paged_select(const PagedView& c, const int* parent, const int* keep, int* ws, hipStream_t s);
hipError_t paged_reserve(const PagedView& c, const int* grow, int* granted, int* ws, hipStream_t s);
hipError_t paged_compact(const PagedView& c, int* live, int* ws, hipStream_t s);
// k, v: row s * n + i at k + (s * n + i) * ldk elements
hipError_t paged_append(const PagedView& c, int layer, const void* k, const void* v, long long ldk, long long ldv,
                        int n, const int* n_new, hipStream_t s);

struct PagedAttnArgs {
  PagedView c;
  const void *pool_k, *pool_v;  // of the layer
  const void* q; long long ldq;
  int n; const int* n_new; int Hq;
  void* out; float* lse;
  float* ws;
  int G;           // query heads per KV head
  unsigned inv_G;  // ceil(2^31 / G)
};
bool paged_attention_fits(const PagedView& c, int n, int Hq);
size_t paged_attention_workspace_floats(const PagedView& c, int n, int Hq);
hipError_t paged_attention(const PagedAttnArgs& a, hipStream_t s);

struct VerifyArgs {
  const float *target, *draft;  // [S][K+1][V], [S][K][V] or null
  const int *tokens, *n_draft;
  int S, K, V;
  float T, min_p;
  const float* u;
  int *out, *n_accepted;
  char* ws;
};
size_t verify_workspace_bytes(int S, int K, int V);
hipError_t verify_drafts(const VerifyArgs& a, hipStream_t s);

}  // namespace rgd
