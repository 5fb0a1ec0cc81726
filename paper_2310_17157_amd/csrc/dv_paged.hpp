// Argument structures and launchers of the paged key/value cache: rotary positions, the
// append, the attention over pages.
#pragma once

#include "dv_internal.hpp"

namespace dv {

// A cache in pages as the kernels see it: strides in bytes, page / rows by a reciprocal.
struct Pages {
  char* K; char* V;
  int64_t ps, hs, rs;               // page, head and row stride, bytes
  const int32_t* table; int n_seq, max_pages, page, n_pages;
  uint32_t inv;                     // floor((2^32 - 1) / page)
  int H, dh;
};

// t / page and the rest, 0 <= t < 2^31: the reciprocal's quotient is at most one too small.
__device__ __forceinline__ int page_of(const Pages& g, int t, int* row) {
  int p = (int)__umulhi((uint32_t)t, g.inv), r = t - p * g.page;
  if (r >= g.page) {
    ++p;
    r -= g.page;
  }
  *row = r;
  return p;
}

// What divides by a number that the host knows: a product and a shift.
struct Divisor {
  uint32_t m; int s;
};

// Rotation and append of T tokens: rotated (or copied) queries, keys and values into pages.
struct RopeArgs {
  int T, dh, rot; const double* freq; float mscale; bool inverse;
  const int32_t* pos;
  const void* q; int64_t ldq; void* qo; int64_t ldqo; int nq;        // heads of q (0: none)
  bool append;                      // keys and values as below; tokens with pos < 0 are left out
  const void* k; const void* v; int64_t ldk, ldv;
  const int32_t* seq; const int32_t* heads; int nk;                  // key/value heads written a token
  Pages g;
  // set by the launcher: tokens of a workgroup, parts of their work, units of a token, of a q or k head and of a v head
  int tpw, parts, per, uq, uv;
  Divisor by_parts, by_per, by_uq, by_uv;
};
hipError_t launch_rope(int xtype, int ktype, int layout, const RopeArgs& a, hipStream_t st);

// Attention of T tokens over the pages. Workgroups: first the shared rows' (key head, part, tile of query rows), then
// items x units of the tokens' own rows: an item is a run of a token's (a group's) rows, a unit a key head's tile of
// query rows, or a place of a head set. Partials: (max, sum) and a value sum each, of the shared rows by [row][part], of
// own rows by [workgroup][row of it].
struct PagedAttnArgs {
  Pages g;
  const float* q; const int32_t* heads; const int32_t* seq; const int32_t* pos;
  int T, n, G;                      // tokens, query heads a token, query heads a key head
  int max_len;
  float scale;                      // times log2(e)
  int RT, RTS;                      // query rows of a workgroup: of own rows, of the shared rows
  int U, row_tiles, group_tiles;    // units; tiles of a key head's shared and own work
  int P, SP, CP;                    // shared rows, parts of them, rows of a part
  int n_shared;                     // workgroups of the shared rows
  int target;                       // workgroups that the own rows are cut for (0: an item is a token)
  int items, cmin, cstep;           // items at most, least rows of one, what its rows are a multiple of
  int live;                         // units of a token that have query rows, at most
  int gmax, RW;                     // tokens of a group at most, rows that a workgroup keeps partials of
  bool direct;                      // one part each: written out by the attention itself
  float *sml, *so, *oml, *oo;       // partials of shared and own rows
  int4* meta;                       // [T] (target > 0) where a token's own partials are
  float* out; int ldo;              // row r at out + r ldo; ldo = dh + 2: (0, 1) before its dh values
  float* lse;
};
// How a launch is cut (all of the second block) for the sizes in g, n, G, T, max_len, P, with or without heads and seq.
void plan_paged_attn(PagedAttnArgs* a, int ktype);
hipError_t launch_paged_attn(int ktype, const PagedAttnArgs& a, hipStream_t st);
hipError_t launch_paged_combine(const PagedAttnArgs& a, hipStream_t st);
// 0 or 1 (a page, sequence, position or shared page that is not as documented) to *bad.
hipError_t launch_paged_validate(const Pages& g, const int32_t* seq, const int32_t* pos, int T, int max_len,
                                 int shared_pages, int32_t* bad, hipStream_t st);

// One step on a cache in pages inside a layer's attention (dv_paged_api.hip): B tokens' fresh keys and values k, v
// [B][H][dh] (fp32, the listed heads) and queries q [B][n][dh] (rotated in place) appended, then attended; the
// outputs go to part [B][n][dh + 2] in the partials' form (0, 1, values). ws: paged_step_ws bytes.
struct PagedStep {
  const dv_paged_kv* kv; const dv_rotary* r;
  const int32_t* seq; const int32_t* pos; int max_len, shared_pages;
  float scale;
};
size_t paged_step_ws(const dv_paged_kv* kv, int B, int n_heads, int max_len, int shared_pages);
dv_status paged_step(const PagedStep& p, int B, const int32_t* heads, int n_heads, float* q, const float* k, const float* v,
                     float* part, void* ws, hipStream_t st);
// The batched sparsified attention on pages (dv_batch_api.hip); arguments already validated.
size_t batch_attn_paged_ws(const dv_attn* a, const dv_paged_kv* kv, int B, int n_heads, int max_len, int shared_pages);
dv_status batch_attn_paged(const dv_attn* a, const float* x, int B, const PagedStep& p, const int32_t* heads, int n_heads,
                           float* out, void* ws, size_t ws_bytes, hipStream_t hs);

}  // namespace dv
