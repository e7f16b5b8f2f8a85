// C ABI of the paged sequences, of the draft verification and of the sampler with per-row limits: argument checks
// (before any HIP call), then the launches.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "entry.hpp"
#include "paged.hpp"
#include "rgd.h"

using namespace rgd;

namespace {

bool aligned(const void* p, uintptr_t n) { return (uintptr_t)p % n == 0; }

// The kernels' view of a description; null and a reason where it is refused.
const char* view_of(const rgd_paged_cache* c, PagedView& v) {
  if (!c) return "null cache";
  if (!c->pool_k || !c->pool_v || !c->pages || !c->lens || !c->refs || !c->status) return "null buffer in the cache";
  if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1 || c->max_pages < 1) return "cache sizes must be positive";
  if (c->max_seqs < 1 || c->max_seqs > 65536) return "max_seqs must be in [1, 65536]";
  if (c->page_size < 16 || c->page_size % 16 || c->page_size > 4096)
    return "page_size must be a multiple of 16, at most 4096";
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 32, 64 or 128";
  if (c->dtype != RGD_DTYPE_F32 && c->dtype != RGD_DTYPE_BF16) return "unknown dtype";
  if (c->n_layers > 65536 || c->n_kv_heads > 1024 || c->n_pages > (1 << 20)) return "cache sizes out of range";
  if ((int64_t)c->max_pages * c->page_size > (1 << 30)) return "a table may hold at most 2^30 positions";
  if (!aligned(c->pool_k, 16) || !aligned(c->pool_v, 16)) return "the pools must be 16-byte aligned";
  v.L = c->n_layers;
  v.n_pages = c->n_pages;
  v.Hkv = c->n_kv_heads;
  v.ps = c->page_size;
  v.D = c->head_dim;
  v.S = c->max_seqs;
  v.width = c->max_pages;
  v.esz = c->dtype == RGD_DTYPE_BF16 ? 2 : 4;
  v.pool_k = (char*)c->pool_k;
  v.pool_v = (char*)c->pool_v;
  v.pages = c->pages;
  v.lens = c->lens;
  v.refs = c->refs;
  v.status = c->status;
  return nullptr;
}

int32_t bad(const char* why) { return set_error(RGD_E_INVALID_ARG, why); }

// A buffer of n bytes (0 at null).
struct Range {
  uintptr_t at;
  uint64_t n;
  Range(const void* p, uint64_t n) : at((uintptr_t)p), n(p ? n : 0) {}
};
// n rows of `row` bytes, `ld` bytes apart; past what an address can be: up to there
Range rows_of(const void* p, int64_t n, int64_t ld, int64_t row) {
  return Range(p, (uint64_t)std::min((__int128)(n - 1) * ld + row, (__int128)1 << 62));
}
bool overlap(const Range& a, const Range& b) { return a.n && b.n && a.at < b.at + b.n && b.at < a.at + a.n; }

// Whether some output shares memory with an input or another output.
bool outputs_shared(std::initializer_list<Range> outputs, std::initializer_list<Range> inputs) {
  for (const Range* o = outputs.begin(); o != outputs.end(); ++o) {
    for (const Range& in : inputs)
      if (overlap(*o, in)) return true;
    for (const Range* p = outputs.begin(); p != o; ++p)
      if (overlap(*o, *p)) return true;
  }
  return false;
}

// Whether some of these buffers shares memory with the cache's.
bool shares_cache(const PagedView& c, std::initializer_list<Range> buffers) {
  const int64_t page = (int64_t)(c.page_elems() * c.esz), n = (int64_t)c.L * c.n_pages;
  return outputs_shared(buffers, {rows_of(c.pool_k, n, page, page), rows_of(c.pool_v, n, page, page),
                                  Range(c.pages, (uint64_t)c.S * c.width * 4), Range(c.lens, (uint64_t)c.S * 4),
                                  Range(c.refs, (uint64_t)c.n_pages * 4), Range(c.status, 4)});
}

// Why the workspace of a page operator is refused, or what it writes besides (or null): each apart from the
// other, from the cache and from the call's counts.
const char* work_ok(const PagedView& c, void* ws, const Range& written, const Range& in0, const Range& in1) {
  if (!aligned(ws, 256)) return "workspace must be 256-byte aligned";
  const Range work(ws, paged_workspace_ints(c) * sizeof(int));
  if (outputs_shared({work, written}, {in0, in1}) || shares_cache(c, {work, written}))
    return "the workspace or an output overlaps an input, the cache or each other";
  return nullptr;
}

int32_t launched(hipError_t e) { return e == hipSuccess ? (int32_t)RGD_OK : set_error(RGD_E_HIP, hipGetErrorString(e)); }

// rows of `width` elements, ld elements apart
const char* rows_ok(const PagedView& v, const void* p, int64_t ld, int64_t width) {
  if (ld < width || ld > ((int64_t)1 << 40)) return "row stride smaller than a row";
  if (!aligned(p, 16) || ld * (int64_t)v.esz % 16) return "rows must be 16-byte aligned";
  return nullptr;
}

const char* heads_ok(const PagedView& v, int32_t n, int32_t n_heads) {
  if (n < 1 || n > 1024) return "n must be in [1, 1024]";
  if (n_heads < 1 || n_heads > 1024 || n_heads % v.Hkv) return "n_heads must be a multiple of n_kv_heads, at most 1024";
  if ((int64_t)v.S * n > (1 << 24)) return "max_seqs * n must be at most 2^24";
  if (!paged_attention_fits(v, n, n_heads)) return "tables too long for so many sequences and heads";
  return nullptr;
}

int32_t reserve(const rgd_paged_cache* cache, const int32_t* grow, int32_t* granted, void* workspace,
                rgd_stream stream) {
  clear_error();
  PagedView v;
  if (const char* why = view_of(cache, v)) return bad(why);
  if (!grow || !workspace) return bad("null argument");
  const Range in(grow, (uint64_t)v.S * 4), out(granted, (uint64_t)v.S * 4), none(nullptr, 0);
  if (const char* why = work_ok(v, workspace, out, granted == grow ? none : in, none)) return bad(why);
  return launched(paged_reserve(v, grow, granted, (int*)workspace, (hipStream_t)stream));
}

// Whether rows at `out` share memory with rows at `in`, each of so many bytes, n rows.  Rows of one stride, as those of
// a fused projection, may lie between each other.
bool rows_overlap(const void* out, int64_t ld_out, int64_t row_out, const void* in, int64_t ld_in, int64_t row_in,
                  int64_t n) {
  if (!overlap(rows_of(out, n, ld_out, row_out), rows_of(in, n, ld_in, row_in))) return false;
  if (ld_out != ld_in || n == 1) return true;
  // the distance from an output row to the next input row that starts at or behind it, and from that one on
  const int64_t gap = (int64_t)((uintptr_t)in - (uintptr_t)out) % ld_out, ahead = gap < 0 ? gap + ld_out : gap;
  return ahead < row_out || ahead + row_in > ld_out;
}

const char* rotary_ok(const rgd_rotary* r, int D) {
  if (!r || r->dim == 0) return nullptr;
  if (r->dim < 0 || r->dim > D || r->dim % 2) return "a rotation's dim must be even, at most head_dim";
  if (!r->freq) return "null frequencies";
  if (!std::isfinite(r->scale)) return "a rotation's scale must be finite";
  for (int j = 0; j < r->dim / 2; ++j)
    if (!std::isfinite(r->freq[j])) return "frequencies must be finite";
  return nullptr;
}

// A plan's or a workspace's size is refused with the entry point's arguments.
const char* shared_ok(const PagedView& v, int32_t n, int32_t n_heads) {
  if (const char* why = heads_ok(v, n, n_heads)) return why;
  if ((int64_t)v.S * n * n_heads > (1 << 22)) return "max_seqs * n * n_heads must be at most 2^22";
  if ((int64_t)v.S * n * (n_heads / v.Hkv) * (n_heads / v.Hkv) >= ((int64_t)1 << 31))  // what query vectors are divided with
    return "max_seqs * n * (n_heads / n_kv_heads)^2 must be below 2^31";
  if (!paged_attention_shared_fits(v, n, n_heads)) return "tables too long for so many sequences and heads";
  return nullptr;
}

}  // namespace

extern "C" {

uint64_t rgd_paged_workspace_bytes(const rgd_paged_cache* cache) {
  clear_error();
  PagedView v;
  if (const char* why = view_of(cache, v)) {
    bad(why);
    return 0;
  }
  return paged_workspace_ints(v) * sizeof(int);
}

int32_t rgd_paged_select(const rgd_paged_cache* cache, const int32_t* parent, const int32_t* keep, void* workspace,
                         rgd_stream stream) {
  clear_error();
  PagedView v;
  if (const char* why = view_of(cache, v)) return bad(why);
  if (parent && !workspace) return bad("null workspace");
  if (const char* why = work_ok(v, workspace, Range(nullptr, 0), Range(parent, (uint64_t)v.S * 4), Range(keep, (uint64_t)v.S * 4)))
    return bad(why);
  return launched(paged_select(v, parent, keep, (int*)workspace, (hipStream_t)stream));
}

int32_t rgd_paged_reserve(const rgd_paged_cache* cache, const int32_t* grow, void* workspace, rgd_stream stream) {
  return reserve(cache, grow, nullptr, workspace, stream);
}

int32_t rgd_paged_reserve_granted(const rgd_paged_cache* cache, const int32_t* grow, int32_t* granted,
                                  void* workspace, rgd_stream stream) {
  clear_error();
  if (!granted) return bad("null argument");
  return reserve(cache, grow, granted, workspace, stream);
}

int32_t rgd_paged_compact(const rgd_paged_cache* cache, int32_t* live, void* workspace, rgd_stream stream) {
  clear_error();
  PagedView v;
  if (const char* why = view_of(cache, v)) return bad(why);
  if (!live || !workspace) return bad("null argument");
  if (const char* why = work_ok(v, workspace, Range(live, 4), Range(nullptr, 0), Range(nullptr, 0))) return bad(why);
  return launched(paged_compact(v, live, (int*)workspace, (hipStream_t)stream));
}

int32_t rgd_paged_append(const rgd_paged_cache* cache, int32_t layer, const void* k, const void* v, int64_t ldk,
                         int64_t ldv, int32_t n, const int32_t* n_new, rgd_stream stream) {
  clear_error();
  PagedView c;
  if (const char* why = view_of(cache, c)) return bad(why);
  if (!k || !v) return bad("null argument");
  if (layer < 0 || layer >= c.L) return bad("layer out of range");
  if (n < 1 || (int64_t)c.S * n > (1 << 24)) return bad("n out of range");
  if (const char* why = rows_ok(c, k, ldk, (int64_t)c.Hkv * c.D)) return bad(why);
  if (const char* why = rows_ok(c, v, ldv, (int64_t)c.Hkv * c.D)) return bad(why);
  return launched(paged_append(c, layer, k, v, ldk, ldv, n, n_new, (hipStream_t)stream));
}

uint64_t rgd_paged_attention_workspace_bytes(const rgd_paged_cache* cache, int32_t n, int32_t n_heads) {
  clear_error();
  PagedView v;
  const char* why = view_of(cache, v);
  if (!why) why = heads_ok(v, n, n_heads);
  if (why) {
    bad(why);
    return 0;
  }
  return paged_attention_workspace_floats(v, n, n_heads) * sizeof(float);
}

int32_t rgd_paged_attention(const rgd_paged_cache* cache, int32_t layer, const void* q, int64_t ldq, int32_t n,
                            const int32_t* n_new, int32_t n_heads, void* workspace, void* out, float* lse,
                            rgd_stream stream) {
  clear_error();
  PagedAttnArgs a{};
  if (const char* why = view_of(cache, a.c)) return bad(why);
  if (!q || !workspace || !out) return bad("null argument");
  if (layer < 0 || layer >= a.c.L) return bad("layer out of range");
  if (const char* why = heads_ok(a.c, n, n_heads)) return bad(why);
  const int64_t width = (int64_t)n_heads * a.c.D, rows = (int64_t)a.c.S * n;
  if (const char* why = rows_ok(a.c, q, ldq, width)) return bad(why);
  if (!aligned(out, 16) || !aligned(workspace, 256)) return bad("out must be 16-byte, the workspace 256-byte aligned");
  const int64_t esz = (int64_t)a.c.esz;
  const Range o(out, rows * width * esz), l(lse, rows * n_heads * 4),
      w(workspace, paged_attention_workspace_floats(a.c, n, n_heads) * sizeof(float));
  if (outputs_shared({o, l, w}, {rows_of(q, rows, ldq * esz, width * esz), Range(n_new, (uint64_t)a.c.S * 4)}) ||
      shares_cache(a.c, {o, l, w}))
    return bad("out, lse or the workspace overlaps an input, the cache or each other");
  const size_t layer0 = (size_t)layer * a.c.n_pages * a.c.page_elems() * a.c.esz;
  a.pool_k = a.c.pool_k + layer0;
  a.pool_v = a.c.pool_v + layer0;
  a.q = q;
  a.ldq = ldq;
  a.n = n;
  a.n_new = n_new;
  a.Hq = n_heads;
  a.out = out;
  a.lse = lse;
  a.ws = (float*)workspace;
  return launched(paged_attention(a, (hipStream_t)stream));
}

uint64_t rgd_verify_workspace_bytes(int32_t S, int32_t K, int32_t V) {
  if (S < 1 || S > 65536 || K < 1 || K > 255 || V < 2 || V > (1 << 20)) return 0;
  if ((int64_t)S * (2 * K + 1) * ((V + 8191) / 8192) > (1 << 23)) return 0;
  return verify_workspace_bytes(S, K, V);
}

int32_t rgd_verify_drafts(const float* target, const float* draft, const int32_t* draft_tokens,
                          const int32_t* n_draft, int32_t S, int32_t K, int32_t V, float T, float min_p,
                          const float* u, void* workspace, int32_t* out, int32_t* n_accepted, rgd_stream stream) {
  clear_error();
  if (!target || !draft_tokens || !u || !workspace || !out || !n_accepted) return bad("null argument");
  if (!rgd_verify_workspace_bytes(S, K, V)) return bad("S, K or V out of range");
  if (!(T >= 0.f && T < 3e38f)) return bad("T must be >= 0 and finite");
  if (!(min_p >= 0.f && min_p <= 1.f)) return bad("min_p must be in [0,1]");
  if (!aligned(workspace, 256)) return bad("workspace must be 256-byte aligned");
  const uint64_t s = S, k = K, kept = s * (k + 1) * 4, counts = s * 4;  // bytes of out, of n_accepted
  if (outputs_shared({Range(out, kept), Range(n_accepted, counts), Range(workspace, verify_workspace_bytes(S, K, V))},
                     {Range(target, kept * V), Range(draft, s * k * 4 * V), Range(draft_tokens, s * k * 4),
                      Range(n_draft, counts), Range(u, kept)}))
    return bad("an output or the workspace overlaps an input or another output");
  VerifyArgs a{target, draft, draft_tokens, n_draft, S, K, V, T, min_p, u, out, n_accepted, (char*)workspace};
  return launched(verify_drafts(a, (hipStream_t)stream));
}

int32_t rgd_rotary_frequencies(int32_t dim, double theta, const rgd_rotary_scaling* scaling, double* freq,
                               float* scale) {
  clear_error();
  if (!freq || !scale) return bad("null argument");
  if (dim < 2 || dim > 128 || dim % 2) return bad("dim must be even, 2 to 128");
  if (!(theta > 1.0 && std::isfinite(theta))) return bad("theta must be above 1 and finite");
  RotaryScaling how{};
  if (scaling) {
    how = RotaryScaling{scaling->kind, scaling->factor, scaling->context, scaling->low, scaling->high};
    if (how.kind < kRotaryLinear || how.kind > kRotaryByIndex) return bad("unknown kind of scaling");
    if (!(how.factor >= 1.0 && std::isfinite(how.factor))) return bad("factor must be at least 1 and finite");
    if (how.kind == kRotaryBase && dim < 4) return bad("dim must be above 2 where theta is scaled");
    if (how.kind >= kRotaryByRotations) {
      if (!(how.context > 0.0 && std::isfinite(how.context))) return bad("context must be positive and finite");
      if (!(how.low > 0.0 && how.low < how.high && std::isfinite(how.high))) return bad("0 < low < high is wanted");
    }
  }
  rotary_frequencies(dim, theta, scaling ? &how : nullptr, freq, scale);
  return RGD_OK;
}

int32_t rgd_paged_append_rotated(const rgd_paged_cache* cache, int32_t layer, const void* q, const void* k,
                                 const void* v, int64_t ldq, int64_t ldk, int64_t ldv, int32_t n,
                                 const int32_t* n_new, int32_t n_heads, const int32_t* positions,
                                 const rgd_rotary* rotary, const float* q_norm, const float* k_norm, float eps,
                                 void* q_out, int64_t ldo, rgd_stream stream) {
  clear_error();
  RotateArgs a{};
  if (const char* why = view_of(cache, a.c)) return bad(why);
  if (!q || !k || !v || !q_out) return bad("null argument");
  if (layer < 0 || layer >= a.c.L) return bad("layer out of range");
  if (n < 1 || (int64_t)a.c.S * n > (1 << 24)) return bad("n out of range");
  if (n_heads < 1 || n_heads > 1024 || n_heads % a.c.Hkv) return bad("n_heads must be a multiple of n_kv_heads, at most 1024");
  const int64_t rows = (int64_t)a.c.S * n, esz = (int64_t)a.c.esz, wq = (int64_t)n_heads * a.c.D, wk = (int64_t)a.c.Hkv * a.c.D;
  if (const char* why = rows_ok(a.c, q, ldq, wq)) return bad(why);
  if (const char* why = rows_ok(a.c, k, ldk, wk)) return bad(why);
  if (const char* why = rows_ok(a.c, v, ldv, wk)) return bad(why);
  if (const char* why = rows_ok(a.c, q_out, ldo, wq)) return bad(why);
  if (const char* why = rotary_ok(rotary, a.c.D)) return bad(why);
  if ((q_norm || k_norm) && !(eps >= 0.f && std::isfinite(eps))) return bad("eps must be at least 0 and finite");
  const bool in_place = q_out == q && ldo == ldq;
  const Range out = rows_of(q_out, rows, ldo * esz, wq * esz);
  if ((!in_place && rows_overlap(q_out, ldo * esz, wq * esz, q, ldq * esz, wq * esz, rows)) ||
      rows_overlap(q_out, ldo * esz, wq * esz, k, ldk * esz, wk * esz, rows) ||
      rows_overlap(q_out, ldo * esz, wq * esz, v, ldv * esz, wk * esz, rows))
    return bad("q_out overlaps q (other than in place), k or v");
  const Range counts(n_new, (uint64_t)a.c.S * 4), at(positions, (uint64_t)rows * 4), gq(q_norm, (uint64_t)a.c.D * 4),
      gk(k_norm, (uint64_t)a.c.D * 4);
  if (outputs_shared({out}, {counts, at, gq, gk}) || shares_cache(a.c, {out}))
    return bad("q_out overlaps an input or the cache");
  // (ranges of the inputs against the cache's one by one: they may share memory with each other)
  for (const Range& in : {rows_of(q, rows, ldq * esz, wq * esz), rows_of(k, rows, ldk * esz, wk * esz),
                          rows_of(v, rows, ldv * esz, wk * esz), counts, at, gq, gk})
    if (shares_cache(a.c, {in})) return bad("an input overlaps the cache");
  const size_t layer0 = (size_t)layer * a.c.n_pages * a.c.page_elems() * a.c.esz;
  a.pool_k = a.c.pool_k + layer0;
  a.pool_v = a.c.pool_v + layer0;
  a.q = q;
  a.k = k;
  a.v = v;
  a.ldq = ldq;
  a.ldk = ldk;
  a.ldv = ldv;
  a.out = q_out;
  a.ldo = ldo;
  a.n = n;
  a.n_new = n_new;
  a.positions = positions;
  a.q_norm = q_norm;
  a.k_norm = k_norm;
  a.eps = eps;
  a.G = n_heads / a.c.Hkv;
  if (rotary) {
    a.dim = rotary->dim;
    a.interleaved = rotary->interleaved != 0;
    a.scale = rotary->scale;
    for (int j = 0; j < a.dim / 2; ++j) a.turns[j] = rotary->freq[j] / 6.283185307179586;
  }
  return launched(paged_append_rotated(a, (hipStream_t)stream));
}

uint64_t rgd_paged_share_bytes(const rgd_paged_cache* cache, int32_t n, int32_t n_heads) {
  clear_error();
  PagedView v;
  const char* why = view_of(cache, v);
  if (!why) why = shared_ok(v, n, n_heads);
  if (why) {
    bad(why);
    return 0;
  }
  return paged_share_ints(v, n) * sizeof(int);
}

int32_t rgd_paged_share(const rgd_paged_cache* cache, int32_t n, const int32_t* n_new, int32_t n_heads,
                        const int32_t* group, void* plan, int32_t* shared, rgd_stream stream) {
  clear_error();
  ShareArgs a{};
  if (const char* why = view_of(cache, a.c)) return bad(why);
  if (!plan) return bad("null argument");
  if (const char* why = shared_ok(a.c, n, n_heads)) return bad(why);
  if (!aligned(plan, 256)) return bad("the plan must be 256-byte aligned");
  const uint64_t counts = (uint64_t)a.c.S * 4;
  const Range p(plan, paged_share_ints(a.c, n) * sizeof(int)), o(shared, counts);
  if (outputs_shared({p, o}, {Range(n_new, counts), Range(group, counts)}) || shares_cache(a.c, {p, o}))
    return bad("the plan or shared overlaps an input, the cache or each other");
  a.n = n;
  a.n_new = n_new;
  a.group = group;
  a.Hq = n_heads;
  a.plan = (int*)plan;
  a.shared = shared;
  return launched(paged_share(a, (hipStream_t)stream));
}

uint64_t rgd_paged_attention_shared_workspace_bytes(const rgd_paged_cache* cache, int32_t n, int32_t n_heads) {
  clear_error();
  PagedView v;
  const char* why = view_of(cache, v);
  if (!why) why = shared_ok(v, n, n_heads);
  if (why) {
    bad(why);
    return 0;
  }
  return paged_attention_shared_workspace_floats(v, n, n_heads) * sizeof(float);
}

int32_t rgd_paged_attention_shared(const rgd_paged_cache* cache, int32_t layer, const void* q, int64_t ldq, int32_t n,
                                   int32_t n_heads, const void* plan, void* workspace, void* out, float* lse,
                                   rgd_stream stream) {
  clear_error();
  PagedAttnArgs a{};
  if (const char* why = view_of(cache, a.c)) return bad(why);
  if (!q || !plan || !workspace || !out) return bad("null argument");
  if (layer < 0 || layer >= a.c.L) return bad("layer out of range");
  if (const char* why = shared_ok(a.c, n, n_heads)) return bad(why);
  const int64_t width = (int64_t)n_heads * a.c.D, rows = (int64_t)a.c.S * n;
  if (const char* why = rows_ok(a.c, q, ldq, width)) return bad(why);
  if (!aligned(out, 16) || !aligned(workspace, 256) || !aligned(plan, 256))
    return bad("out must be 16-byte, the plan and the workspace 256-byte aligned");
  const int64_t esz = (int64_t)a.c.esz;
  const Range o(out, rows * width * esz), l(lse, rows * n_heads * 4),
      w(workspace, paged_attention_shared_workspace_floats(a.c, n, n_heads) * sizeof(float)),
      p(plan, paged_share_ints(a.c, n) * sizeof(int));
  if (outputs_shared({o, l, w}, {rows_of(q, rows, ldq * esz, width * esz), p}) || shares_cache(a.c, {o, l, w}))
    return bad("out, lse or the workspace overlaps an input, the cache or each other");
  const size_t layer0 = (size_t)layer * a.c.n_pages * a.c.page_elems() * a.c.esz;
  a.pool_k = a.c.pool_k + layer0;
  a.pool_v = a.c.pool_v + layer0;
  a.q = q;
  a.ldq = ldq;
  a.n = n;
  a.Hq = n_heads;
  a.out = out;
  a.lse = lse;
  a.ws = (float*)workspace;
  return launched(paged_attention_shared(a, (const int*)plan, (hipStream_t)stream));
}

uint64_t rgd_sample_truncated_workspace_bytes(int32_t R, int32_t V) {
  if (R < 1 || R > 65536 || V < 1 || V > (1 << 20)) return 0;
  return sample_truncated_workspace_bytes(R, V);
}

int32_t rgd_sample_truncated(const float* z, int64_t ldz, int32_t R, int32_t V, const float* T, const int32_t* top_k,
                             const float* top_p, const float* min_p, const float* u, void* workspace, int32_t* out,
                             float* logp, rgd_stream stream) {
  clear_error();
  if (!z || !u || !workspace || !out) return bad("null argument");
  if (!rgd_sample_truncated_workspace_bytes(R, V)) return bad("R or V out of range");
  if (ldz < V || ldz > ((int64_t)1 << 40)) return bad("row stride smaller than a row");
  if (!aligned(workspace, 256)) return bad("workspace must be 256-byte aligned");
  const uint64_t r4 = (uint64_t)R * 4;
  if (outputs_shared({Range(out, r4), Range(logp, r4), Range(workspace, sample_truncated_workspace_bytes(R, V))},
                     {rows_of(z, R, ldz * 4, (int64_t)V * 4), Range(T, r4), Range(top_k, r4), Range(top_p, r4),
                      Range(min_p, r4), Range(u, r4)}))
    return bad("an output or the workspace overlaps an input or another output");
  TruncateArgs a{z, ldz, R, V, T, top_k, top_p, min_p, u, out, logp, (char*)workspace};
  return launched(sample_truncated(a, (hipStream_t)stream));
}

}  // extern "C"
