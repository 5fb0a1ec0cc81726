// C ABI entry points of the paged key/value cache: dv_rotary_freqs, dv_rope, dv_paged_append,
// dv_paged_attn, and dv_sparse_attn_paged (the sparsified attention on such a cache).
#include <math.h>

#include <algorithm>

#include "dv_paged.hpp"

namespace dv {

namespace {
bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Strides under which no two of the rows overlap: by increasing stride, each step passes all that the
// smaller ones reach. A dimension of one entry has no stride.
dv_status check_strides(const dv_paged_kv* kv) {
  int64_t stride[3] = {kv->row_stride, kv->head_stride, kv->page_stride};
  int64_t count[3] = {kv->page, kv->H, kv->n_pages};
  int order[3] = {0, 1, 2};
  std::stable_sort(order, order + 3, [&](int x, int y) { return stride[x] < stride[y]; });
  __int128 reach = kv->dh;
  for (int i : order) {
    if (count[i] == 1) continue;
    if (stride[i] % chunk_elems(kv->ktype) != 0) return DV_ERR_ALIGN;
    if (stride[i] < 1 || (__int128)stride[i] < reach) return DV_ERR_SHAPE;
    reach += (__int128)(count[i] - 1) * stride[i];
    if (reach > ((__int128)1 << 60)) return DV_ERR_SHAPE;
  }
  return DV_OK;
}

dv_status check_paged(const dv_paged_kv* kv) {
  if (kv == nullptr || kv->K == nullptr || kv->V == nullptr || kv->table == nullptr) return DV_ERR_NULL;
  if (!dtype_ok(kv->ktype)) return DV_ERR_DTYPE;
  if (kv->reserved != 0) return DV_ERR_ARG;
  if (kv->H <= 0 || kv->dh <= 0 || kv->page <= 0 || kv->n_pages <= 0 || kv->n_seq <= 0 || kv->max_pages <= 0)
    return DV_ERR_SHAPE;
  if ((kv->dh * elem_bytes(kv->ktype)) % 16 != 0) return DV_ERR_ALIGN;
  if (!aligned16(kv->K) || !aligned16(kv->V) || !aligned_to(kv->table, 4)) return DV_ERR_ALIGN;
  if (kv->dh > 256 || (int64_t)kv->max_pages * kv->page > INT32_MAX - 4096) return DV_ERR_UNSUPPORTED;
  return check_strides(kv);
}

dv_status check_rotary(const dv_rotary* r, int dh) {
  if (r->freq == nullptr) return DV_ERR_NULL;
  if (r->rot < 2 || r->rot > dh || r->rot % 2 != 0) return DV_ERR_SHAPE;
  if (r->layout != DV_ROPE_HALF && r->layout != DV_ROPE_INTERLEAVED) return DV_ERR_ARG;
  if (!isfinite(r->mscale) || r->reserved != 0) return DV_ERR_ARG;
  return aligned_to(r->freq, 8) ? DV_OK : DV_ERR_ALIGN;
}

// Tokens of n heads at a stride: inside the type's alignment, one token not reaching into the next.
dv_status check_tokens(const void* p, int64_t ld, int T, int64_t n, int type) {
  if (p == nullptr) return DV_ERR_NULL;
  if (!aligned_to(p, elem_bytes(type))) return DV_ERR_ALIGN;
  return T > 1 && (ld < n || ld > ((int64_t)1 << 40)) ? DV_ERR_SHAPE : DV_OK;
}

Pages pages_of(const dv_paged_kv* kv) {
  const int eb = elem_bytes(kv->ktype);
  auto bytes = [&](int64_t stride, int count) { return count == 1 ? 0 : stride * eb; };
  Pages g{};
  g.K = static_cast<char*>(kv->K); g.V = static_cast<char*>(kv->V);
  g.ps = bytes(kv->page_stride, kv->n_pages); g.hs = bytes(kv->head_stride, kv->H); g.rs = bytes(kv->row_stride, kv->page);
  g.table = kv->table; g.n_seq = kv->n_seq; g.max_pages = kv->max_pages; g.page = kv->page; g.n_pages = kv->n_pages;
  g.inv = 0xffffffffu / (uint32_t)kv->page;
  g.H = kv->H; g.dh = kv->dh;
  return g;
}

void set_rotary(RopeArgs* a, const dv_rotary* r) {
  if (r == nullptr) return;
  a->rot = r->rot; a->freq = r->freq; a->mscale = r->mscale;
}

constexpr int64_t kMaxPagedRows = 1 << 22;
constexpr int kMaxUnionHeads = 131072;               // heads of a batch's union (dv_sparse_attn's limit)

// The launch of T tokens with n query heads each (heads: non-NULL for head sets; seq: NULL or not) and its partials in w.
PagedAttnArgs attn_args(const dv_paged_kv* kv, int T, int Hq, const int32_t* heads, int n, const int32_t* seq, int max_len,
                        int shared_pages, Workspace& w) {
  PagedAttnArgs a{};
  a.g = pages_of(kv);
  a.T = T; a.n = n; a.G = Hq / kv->H; a.heads = heads; a.seq = seq; a.max_len = max_len; a.P = shared_pages * kv->page;
  plan_paged_attn(&a, kv->ktype);
  if (!a.direct) {
    const size_t shared = (size_t)T * n * a.SP, own = (size_t)a.items * a.U * a.RW;
    a.sml = w.take<float>(shared * 2 * sizeof(float));
    a.so = w.take<float>(shared * kv->dh * sizeof(float));
    a.oml = w.take<float>(own * 2 * sizeof(float));
    a.oo = w.take<float>(own * kv->dh * sizeof(float));
    a.meta = w.take<int4>((size_t)T * sizeof(int4));
  }
  return a;
}

dv_status enqueue_paged_attn(const PagedAttnArgs& a, int ktype, hipStream_t st) {
  DV_LAUNCH("paged_attn", st, launch_paged_attn(ktype, a, st));
  if (!a.direct) DV_LAUNCH("paged_combine", st, launch_paged_combine(a, st));
  return DV_OK;
}

dv_status validate_paged_sync(const dv_paged_kv* kv, const int32_t* seq, const int32_t* pos, int T, int max_len,
                              int shared_pages, int32_t* flag, hipStream_t st) {
  DV_LAUNCH("validate", st, launch_paged_validate(pages_of(kv), seq, pos, T, max_len, shared_pages, flag, st));
  int32_t bad = 0;
  if (hipMemcpyAsync(&bad, flag, sizeof(bad), hipMemcpyDeviceToHost, st) != hipSuccess) return DV_ERR_HIP;
  if (hipStreamSynchronize(st) != hipSuccess) return DV_ERR_HIP;
  return bad ? DV_ERR_INDEX : DV_OK;
}

// What dv_paged_attn and dv_sparse_attn_paged ask of the attended rows.
dv_status check_lengths(const dv_paged_kv* kv, const int32_t* seq, int T, int max_len, int shared_pages) {
  if (max_len < 1 || max_len > (int64_t)kv->max_pages * kv->page) return DV_ERR_SHAPE;
  if (shared_pages < 0 || (int64_t)shared_pages * kv->page > max_len) return DV_ERR_SHAPE;
  return seq == nullptr && T > kv->n_seq ? DV_ERR_SHAPE : DV_OK;
}
}  // namespace

size_t paged_step_ws(const dv_paged_kv* kv, int B, int n_heads, int max_len, int shared_pages) {
  if (n_heads == 0) return 0;
  Workspace w(nullptr);
  const int32_t some = 0;
  (void)attn_args(kv, B, kv->H, &some, n_heads, &some, max_len, shared_pages, w);
  return w.off;
}

dv_status paged_step(const PagedStep& p, int B, const int32_t* heads, int n_heads, float* q, const float* k, const float* v,
                     float* part, void* ws, hipStream_t st) {
  const int dh = p.kv->dh;
  RopeArgs r{};
  r.T = B; r.dh = dh; set_rotary(&r, p.r); r.pos = p.pos;
  r.q = q; r.qo = q; r.ldq = r.ldqo = (int64_t)n_heads * dh; r.nq = p.r != nullptr ? n_heads : 0;
  r.append = true; r.k = k; r.v = v; r.ldk = r.ldv = (int64_t)p.kv->H * dh; r.seq = p.seq; r.heads = heads; r.nk = n_heads;
  r.g = pages_of(p.kv);
  DV_LAUNCH("append", st, launch_rope(DV_F32, p.kv->ktype, p.r != nullptr ? p.r->layout : DV_ROPE_HALF, r, st));
  Workspace w(ws);
  PagedAttnArgs a = attn_args(p.kv, B, p.kv->H, heads, n_heads, p.seq, p.max_len, p.shared_pages, w);
  a.q = q; a.pos = p.pos; a.scale = p.scale * (float)M_LOG2E; a.out = part; a.ldo = dh + 2;
  return enqueue_paged_attn(a, p.kv->ktype, st);
}

}  // namespace dv

using namespace dv;

extern "C" dv_status dv_rotary_freqs(int32_t rule, int32_t rot, double base, double factor, double orig_len, double low,
                                     double high, double* freq) {
  if (freq == nullptr) return DV_ERR_NULL;
  if (rot < 2 || rot % 2 != 0) return DV_ERR_SHAPE;
  if (rule < DV_ROPE_PLAIN || rule > DV_ROPE_PARTS) return DV_ERR_ARG;
  if (!(base > 0) || !isfinite(base)) return DV_ERR_ARG;
  if (rule != DV_ROPE_PLAIN && (!(factor > 0) || !isfinite(factor))) return DV_ERR_ARG;
  if (rule == DV_ROPE_NTK) {
    if (rot == 2) return DV_ERR_SHAPE;
    base *= pow(factor, (double)rot / (rot - 2));
  }
  if (rule == DV_ROPE_PARTS && (!(orig_len > 0) || !isfinite(orig_len) || !(high > low) || !isfinite(high - low)))
    return DV_ERR_ARG;
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot);
    if (rule == DV_ROPE_LINEAR) f /= factor;
    if (rule == DV_ROPE_PARTS) {
      const double turns = orig_len * f / (2 * M_PI);
      const double g = std::min(std::max((turns - low) / (high - low), 0.0), 1.0);
      f *= g + (1 - g) / factor;
    }
    freq[i] = f;
  }
  return DV_OK;
}

extern "C" dv_status dv_rope(const dv_rotary* r, const void* x, int64_t ldx, int32_t xtype, int32_t T, int32_t H, int32_t dh,
                             const int32_t* pos, void* out, int64_t ldo, uint32_t flags, void* stream) {
  trace_reset();
  if (r == nullptr) return DV_ERR_NULL;
  if (!dtype_ok(xtype)) return DV_ERR_DTYPE;
  if (T < 0 || H < 0 || dh <= 0) return DV_ERR_SHAPE;
  if (dh > 256 || (int64_t)H * dh > INT32_MAX / 2) return DV_ERR_UNSUPPORTED;
  dv_status st = check_rotary(r, dh);
  if (st != DV_OK) return st;
  if (flags & ~(uint32_t)(DV_DETERMINISTIC | DV_ROPE_INVERSE)) return DV_ERR_ARG;
  if (T == 0 || H == 0) return DV_OK;
  if (pos == nullptr) return DV_ERR_NULL;
  if ((st = check_tokens(x, ldx, T, (int64_t)H * dh, xtype)) != DV_OK) return st;
  if ((st = check_tokens(out, ldo, T, (int64_t)H * dh, xtype)) != DV_OK) return st;
  if (x == out && T > 1 && ldx != ldo) return DV_ERR_ARG;
  RopeArgs a{};
  a.T = T; a.dh = dh; set_rotary(&a, r); a.inverse = (flags & DV_ROPE_INVERSE) != 0; a.pos = pos;
  a.q = x; a.ldq = ldx; a.qo = out; a.ldqo = ldo; a.nq = H;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  DV_LAUNCH("rope", hs, launch_rope(xtype, xtype, r->layout, a, hs));
  return DV_OK;
}

extern "C" dv_status dv_paged_append(const dv_paged_kv* kv, const dv_rotary* r, const void* k, int64_t ldk, const void* v,
                                     int64_t ldv, int32_t xtype, int32_t T, const int32_t* seq, const int32_t* pos,
                                     const int32_t* heads, int32_t n_heads, const void* q, int64_t ldq, int32_t Hq,
                                     void* q_out, int64_t ldqo, void* stream) {
  trace_reset();
  dv_status st = check_paged(kv);
  if (st != DV_OK) return st;
  if (!dtype_ok(xtype)) return DV_ERR_DTYPE;
  if (r != nullptr && (st = check_rotary(r, kv->dh)) != DV_OK) return st;
  if ((q == nullptr) != (q_out == nullptr)) return DV_ERR_NULL;
  if (T < 0 || (q != nullptr && Hq <= 0) || (heads != nullptr && (n_heads < 0 || n_heads > kv->H))) return DV_ERR_SHAPE;
  if ((int64_t)kv->H * kv->dh > INT32_MAX / 8 || (int64_t)(q != nullptr ? Hq : 0) * kv->dh > INT32_MAX / 8)
    return DV_ERR_UNSUPPORTED;
  if (T == 0) return DV_OK;
  if (pos == nullptr) return DV_ERR_NULL;
  if (seq == nullptr && T > kv->n_seq) return DV_ERR_SHAPE;
  if ((st = check_tokens(k, ldk, T, (int64_t)kv->H * kv->dh, xtype)) != DV_OK) return st;
  if ((st = check_tokens(v, ldv, T, (int64_t)kv->H * kv->dh, xtype)) != DV_OK) return st;
  if (q != nullptr) {
    if ((st = check_tokens(q, ldq, T, (int64_t)Hq * kv->dh, xtype)) != DV_OK) return st;
    if ((st = check_tokens(q_out, ldqo, T, (int64_t)Hq * kv->dh, xtype)) != DV_OK) return st;
    if (q == q_out && T > 1 && ldq != ldqo) return DV_ERR_ARG;
  }
  RopeArgs a{};
  a.T = T; a.dh = kv->dh; set_rotary(&a, r); a.pos = pos;
  a.q = q; a.ldq = ldq; a.qo = q_out; a.ldqo = ldqo; a.nq = q != nullptr ? Hq : 0;
  a.append = true; a.k = k; a.v = v; a.ldk = ldk; a.ldv = ldv; a.seq = seq; a.heads = heads;
  a.nk = heads != nullptr ? n_heads : kv->H;
  a.g = pages_of(kv);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  DV_LAUNCH("append", hs, launch_rope(xtype, kv->ktype, r != nullptr ? r->layout : DV_ROPE_HALF, a, hs));
  return DV_OK;
}

static const int32_t kSomeHeads = 0;   // stands for a head set where only its presence matters

extern "C" size_t dv_paged_attn_workspace_bytes(const dv_paged_kv* kv, int32_t T, int32_t Hq, int32_t n_heads,
                                                int32_t max_len, int32_t shared_pages) {
  if (check_paged(kv) != DV_OK || T < 0 || Hq <= 0 || Hq % kv->H != 0 || n_heads < 0 || n_heads > Hq ||
      check_lengths(kv, &kSomeHeads, T, max_len, shared_pages) != DV_OK)
    return 0;
  const int n = n_heads > 0 ? n_heads : Hq;
  if ((int64_t)T * n > kMaxPagedRows || (int64_t)T * kv->H > kMaxPagedRows) return 0;
  size_t most = 0;
  for (const int32_t* seq : {static_cast<const int32_t*>(nullptr), &kSomeHeads}) {   // (groups of drafts need seq)
    Workspace w(nullptr);
    w.take<int32_t>(sizeof(int32_t));
    if (T > 0) (void)attn_args(kv, T, Hq, n_heads > 0 ? &kSomeHeads : nullptr, n, seq, max_len, shared_pages, w);
    most = std::max(most, w.off);
  }
  return most;
}

extern "C" dv_status dv_paged_attn(const dv_paged_kv* kv, const float* q, int32_t T, int32_t Hq, const int32_t* heads,
                                   int32_t n_heads, const int32_t* seq, const int32_t* pos, int32_t max_len,
                                   int32_t shared_pages, float scale, float* out, float* lse, void* ws, size_t ws_bytes,
                                   uint32_t flags, void* stream) {
  trace_reset();
  dv_status st = check_paged(kv);
  if (st != DV_OK) return st;
  if (T < 0 || Hq <= 0 || Hq % kv->H != 0 || (heads != nullptr && (n_heads < 0 || n_heads > Hq))) return DV_ERR_SHAPE;
  if ((st = check_lengths(kv, seq, T, max_len, shared_pages)) != DV_OK) return st;
  if (flags & ~(uint32_t)(DV_DETERMINISTIC | DV_VALIDATE)) return DV_ERR_ARG;
  if (!isfinite(scale) || !isfinite(scale * (float)M_LOG2E)) return DV_ERR_ARG;
  const int n = heads != nullptr ? n_heads : Hq;
  if ((int64_t)T * n > kMaxPagedRows || (int64_t)T * kv->H > kMaxPagedRows) return DV_ERR_UNSUPPORTED;
  if (T == 0 || n == 0) return DV_OK;
  if (q == nullptr || out == nullptr || pos == nullptr) return DV_ERR_NULL;
  if (!aligned16(q) || !aligned16(out) || !aligned_to(lse, 4)) return DV_ERR_ALIGN;
  if (!ws_ok(ws)) return DV_ERR_WORKSPACE;
  Workspace w(ws);
  int32_t* flag = w.take<int32_t>(sizeof(int32_t));
  PagedAttnArgs a = attn_args(kv, T, Hq, heads, n, seq, max_len, shared_pages, w);
  if (w.off > ws_bytes) return DV_ERR_WORKSPACE;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (flags & DV_VALIDATE) {
    if (heads != nullptr && (st = validate_sets_sync(heads, T, n, Hq, flag, hs)) != DV_OK) return st;
    if ((st = validate_paged_sync(kv, seq, pos, T, max_len, shared_pages, flag, hs)) != DV_OK) return st;
  }
  a.q = q; a.pos = pos; a.scale = scale * (float)M_LOG2E; a.out = out; a.ldo = kv->dh; a.lse = lse;
  return enqueue_paged_attn(a, kv->ktype, hs);
}

// ------------------------------------------------- sparsified attention on pages
namespace {
struct PagedLayerWs {
  int32_t* heads; float *q, *k, *v, *part, *axp; uint32_t* axc; char* step;
};

size_t paged_layer_layout(const dv_attn* a, const dv_paged_kv* kv, int n_heads, int max_len, int shared_pages, Workspace& w,
                          PagedLayerWs* o) {
  const size_t rows = (size_t)a->H * a->dh * sizeof(float);
  o->heads = w.take<int32_t>((size_t)n_heads * sizeof(int32_t));
  o->q = w.take<float>((size_t)n_heads * a->dh * sizeof(float));
  o->k = w.take<float>(rows);
  o->v = w.take<float>(rows);
  o->part = w.take<float>((size_t)n_heads * (a->dh + 2) * sizeof(float));
  o->axp = w.take<float>(axpy_partial_bytes(a->d));
  o->axc = w.take<uint32_t>(kAxpyMaxSpans * sizeof(uint32_t));
  o->step = w.take<char>(paged_step_ws(kv, 1, n_heads, max_len, shared_pages));
  return w.off;
}

// One token: dv_sparse_attn's launches around the append and the attention over the pages.
dv_status paged_layer(const dv_attn* a, const float* x, const PagedStep& p, const int32_t* heads, int n_heads, float* out,
                      void* ws, size_t ws_bytes, hipStream_t hs) {
  Workspace w(ws);
  PagedLayerWs o;
  if (paged_layer_layout(a, p.kv, n_heads, p.max_len, p.shared_pages, w, &o) > ws_bytes) return DV_ERR_WORKSPACE;
  AxpyArgs ax{};
  ax.d = a->d; ax.M = a->WoT; ax.m_rows = a->H * a->dh; ax.set = o.heads; ax.bias = a->bo; ax.out = out;
  if (n_heads == 0) {
    ax.coef = o.q;
    DV_LAUNCH("oproj", hs, launch_axpy(a->wtype, ax, hs));
    return DV_OK;
  }
  // fresh keys and values: a buffer of one row a head, a cache of one row to the launch
  QkvArgs q{};
  q.d = a->d; q.H = a->H; q.dh = a->dh; q.cap = 1; q.pos = 0; q.n_heads = n_heads;
  q.x = x;
  q.Wq = a->Wq; q.Wk = a->Wk; q.Wv = a->Wv; q.bq = a->bq; q.bk = a->bk; q.bv = a->bv;
  q.K = o.k; q.V = o.v; q.q = o.q; q.heads_in = heads; q.heads_ws = o.heads;
  q.clear = o.axc; q.clear_n = kAxpyMaxSpans;
  DV_LAUNCH("qkv", hs, launch_qkv(a->wtype, DV_F32, q, hs));
  const dv_status st = paged_step(p, 1, o.heads, n_heads, o.q, o.k, o.v, o.part, o.step, hs);
  if (st != DV_OK) return st;
  ax.nrows = n_heads * a->dh; ax.dh = a->dh; ax.part = o.part; ax.n_split = 1; ax.partial = o.axp; ax.cnt = o.axc;
  DV_LAUNCH("oproj", hs, launch_axpy(a->wtype, ax, hs));
  return DV_OK;
}
}  // namespace

static size_t sparse_attn_paged_ws(const dv_attn* a, const dv_paged_kv* kv, int B, int n_heads, int max_len,
                                   int shared_pages) {
  size_t flag = 256;                                     // DV_VALIDATE's, first
  if (B > 1) return flag + batch_attn_paged_ws(a, kv, B, n_heads, max_len, shared_pages);
  Workspace w(nullptr);
  PagedLayerWs o;
  return flag + paged_layer_layout(a, kv, n_heads, max_len, shared_pages, w, &o);
}

extern "C" size_t dv_sparse_attn_paged_workspace_bytes(const dv_attn* a, const dv_paged_kv* kv, int32_t B, int32_t n_heads,
                                                       int32_t max_len, int32_t shared_pages) {
  if (check_attn(a) != DV_OK || check_paged(kv) != DV_OK || kv->H != a->H || kv->dh != a->dh || B <= 0 || B > kMaxBatch ||
      n_heads < 0 || n_heads > a->H || check_lengths(kv, &kSomeHeads, B, max_len, shared_pages) != DV_OK)
    return 0;
  return sparse_attn_paged_ws(a, kv, B, n_heads, max_len, shared_pages);
}

extern "C" dv_status dv_sparse_attn_paged(const dv_attn* a, const float* x, int32_t B, const dv_paged_kv* kv,
                                          const dv_rotary* r, const int32_t* seq, const int32_t* pos, int32_t max_len,
                                          int32_t shared_pages, const int32_t* heads, int32_t n_heads, float scale,
                                          float* out, void* ws, size_t ws_bytes, uint32_t flags, void* stream) {
  trace_reset();
  dv_status st = check_attn(a);
  if (st != DV_OK) return st;
  if ((st = check_paged(kv)) != DV_OK) return st;
  if (r != nullptr && (st = check_rotary(r, kv->dh)) != DV_OK) return st;
  if (x == nullptr || out == nullptr || pos == nullptr || (heads == nullptr && n_heads > 0)) return DV_ERR_NULL;
  if (B <= 0 || n_heads < 0 || n_heads > a->H || kv->H != a->H || kv->dh != a->dh) return DV_ERR_SHAPE;
  if ((st = check_lengths(kv, seq, B, max_len, shared_pages)) != DV_OK) return st;
  if (!aligned16(x) || !aligned16(out)) return DV_ERR_ALIGN;
  if (flags & ~(uint32_t)(DV_DETERMINISTIC | DV_VALIDATE)) return DV_ERR_ARG;
  if (!isfinite(scale) || !isfinite(scale * (float)M_LOG2E)) return DV_ERR_ARG;
  if (a->bo != nullptr && !aligned16(a->bo)) return DV_ERR_ALIGN;
  if (B > 1 && (B > kMaxBatch || a->wtype != DV_F16 || a->H > kMaxUnionHeads)) return DV_ERR_UNSUPPORTED;
  if (!ws_ok(ws)) return DV_ERR_WORKSPACE;
  if (sparse_attn_paged_ws(a, kv, B, n_heads, max_len, shared_pages) > ws_bytes) return DV_ERR_WORKSPACE;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  int32_t* flag = static_cast<int32_t*>(ws);
  if (flags & DV_VALIDATE) {
    if (n_heads > 0 && (st = validate_sets_sync(heads, B, n_heads, a->H, flag, hs)) != DV_OK) return st;
    if ((st = validate_paged_sync(kv, seq, pos, B, max_len, shared_pages, flag, hs)) != DV_OK) return st;
  }
  const PagedStep p{kv, r, seq, pos, max_len, shared_pages, scale};
  void* rest = static_cast<char*>(ws) + 256;
  if (B > 1) return batch_attn_paged(a, x, B, p, heads, n_heads, out, rest, ws_bytes - 256, hs);
  return paged_layer(a, x, p, heads, n_heads, out, rest, ws_bytes - 256, hs);
}
