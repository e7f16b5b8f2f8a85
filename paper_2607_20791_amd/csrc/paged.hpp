// Paged sequences (internal): the kernels' view of an rgd_paged_cache and the
// launch interface of its operators, of the draft verification and of the sampler with per-row limits.
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
  // by a plan: the groups' parts
  int* plan;
  void* at;                   // [S + 1]: where a group's units and items begin; units of a run
  float* slots;               // of run r and item i: r + i
  int s_cols, s_cost, s_step; // query vectors of a slot, units of an item besides its steps, positions of a step
  int most;                   // tokens of a sequence: n, or 0 where the plan is not this call's
};
bool paged_attention_fits(const PagedView& c, int n, int Hq);
size_t paged_attention_workspace_floats(const PagedView& c, int n, int Hq);
hipError_t paged_attention(const PagedAttnArgs& a, hipStream_t s);

constexpr int kRotaryLinear = 1, kRotaryBase = 2, kRotaryByRotations = 3, kRotaryByIndex = 4;
struct RotaryScaling {
  int kind;
  double factor, context, low, high;
};
void rotary_frequencies(int dim, double theta, const RotaryScaling* scaling, double* freq, float* scale);

struct RotateArgs {
  PagedView c;
  void *pool_k, *pool_v;  // of the layer
  const void *q, *k, *v; long long ldq, ldk, ldv;
  void* out; long long ldo;
  int n; const int *n_new, *positions;
  const float *q_norm, *k_norm; float eps;
  int dim, interleaved; float scale;
  double turns[64];  // of each pair, per position
  int G;       // query heads per KV head
  int blocks;  // 16-position blocks per sequence
  int heads;   // KV heads per workgroup
};
hipError_t paged_append_rotated(const RotateArgs& a, hipStream_t s);

// What the sequences of a group share (see rgd_paged_share); ints in the caller's plan.
struct ShareArgs {
  PagedView c;
  int n; const int *n_new, *group;
  int Hq;
  int* plan;
  int* shared;
};
size_t paged_share_ints(const PagedView& c, int n);
hipError_t paged_share(const ShareArgs& a, hipStream_t s);
// a.n_new is taken from the plan
hipError_t paged_attention_shared(const PagedAttnArgs& a, const int* plan, hipStream_t s);
// How the groups' part is cut: query vectors of an item, units of one besides its steps, positions of a step, runs.
struct GroupShape {
  int cols, cost, step, runs;
};
GroupShape group_shape(const PagedView& c, int vectors);
hipError_t paged_group(const PagedAttnArgs& a, int runs, hipStream_t s);  // bf16
bool paged_attention_shared_fits(const PagedView& c, int n, int Hq);
size_t paged_attention_shared_workspace_floats(const PagedView& c, int n, int Hq);

struct TruncateArgs {
  const float* z; long long ldz;
  int R, V;
  const float* T; const int* top_k; const float *top_p, *min_p, *u;
  int* out; float* logp;
  char* ws;
};
size_t sample_truncated_workspace_bytes(int R, int V);
hipError_t sample_truncated(const TruncateArgs& a, hipStream_t s);

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
