// Decode attention over a cache in pages, with a prefix that the batch shares attended once.
//
// For a query head of a token, over its rows p: s_p = scale q . K_p, out = sum_p e^{s_p - M} V_p / sum_p e^{s_p - M}.
// The sum is taken in parts (a running maximum, sum and value sum each) that are joined at the end.
//
// Units. A unit is a key head's query rows and a run of cache rows: a token's own query heads of that key head over a
// part of its own rows, or, for the shared rows, all tokens' query heads of that key head over a part of them, kept
// or read once for the whole batch. Both are the same work, a tile of up to RT query rows times cache rows, done by
// one workgroup of four wavefronts, each taking every fourth step of 32 (fp16) or 16 (fp32) cache rows.
//
// Products on the matrix cores, no cache element passing through LDS:
//   S^T = K Q^T  A: 16 cache rows, a lane holding 16 bytes of its row as loaded (any order of the contracted head
//                elements will do, as long as the queries have the same). D: lane = (query, four cache rows).
//   O^T = V^T P^T  B: the probabilities as D left them (the contracted cache rows in D's order: a lane's 4 + 4).
//                A: output row r of tile e is head element r E + e, so a lane needs element e of its r-th chunk
//                of those cache rows: it loads whole chunks of its eight cache rows (a row is
//                read by 16 lanes, contiguous) and picks pairs of elements with byte permutes.
// fp32's precision from fp16 matrix cores: cache elements are exact in fp16; a query row, scaled by a power of two
// to below 2^15, and the probabilities times 2^14 are each the sum of two fp16 numbers (22 bits; below 2^-25 of that scale
// nothing is left). With up to 8 query rows the second halves are columns 8..15 of the same products, so they
// cost nothing; with more they are products of their own. fp32 caches use the fp32 matrix instructions.
//
// Memory bounds it: at one query row per key head the matrix cores are busy about 4 % of the time. So a step's keys
// are loaded into the registers of the last step's as soon as its logits are taken, its values as soon as the last
// value product is, page indices two steps ahead: every wavefront has one to two steps' worth of loads in flight
// from one set of registers, and more wavefronts fit than with two sets.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dv_paged.hpp"

namespace dv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kPaNW = 4, kPaNT = 64 * kPaNW;
constexpr float kPaLn2 = 0.693147180559945309f;
constexpr int kPaMaxParts = 64;      // parts of the shared rows, and of a group's own, at most

// Rows that a position attends, and how many of them are shared ones (all of those, or none: a token that attends fewer
// takes what it attends by itself).
__device__ __forceinline__ int pa_rows_of(const PagedAttnArgs& a, int pos) { return min(max(pos, -1), a.max_len - 1) + 1; }
__device__ __forceinline__ int pa_len(const PagedAttnArgs& a, int t) { return pa_rows_of(a, a.pos[t]); }
__device__ __forceinline__ int pa_start(const PagedAttnArgs& a, int len) { return a.P > 0 && len >= a.P ? a.P : 0; }

// Over a wavefront without LDS: row shifts and rotations, then across its rows of 16.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int pa_dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int pa_wave_incl(int v) {      // inclusive prefix sum
  v += pa_dpp<0x111>(v);
  v += pa_dpp<0x112>(v);
  v += pa_dpp<0x114>(v);
  v += pa_dpp<0x118>(v);
  v += pa_dpp<0x142, 0xa>(v);
  v += pa_dpp<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ int pa_last(int v) { return __builtin_amdgcn_readlane(v, kWave - 1); }
__device__ __forceinline__ int pa_wave_max(int v) {       // of values >= 0, uniform
  v = max(v, pa_dpp<0x111>(v));
  v = max(v, pa_dpp<0x112>(v));
  v = max(v, pa_dpp<0x114>(v));
  v = max(v, pa_dpp<0x118>(v));
  v = max(v, pa_dpp<0x142, 0xa>(v));
  v = max(v, pa_dpp<0x143, 0xc>(v));
  return pa_last(v);
}

// Tokens next to each other that share a sequence (drafts) are a group, whose own rows are read once: up to gmax of
// them (aligned; a power of two), at ascending positions not far apart. A lane's token t:
struct PaTok {
  int len, seq;
  bool leads, ends;                  // the first, the last of its group
  int own;                           // a group's own rows, at its last token (0 at the others, and past the tokens)
};
constexpr int kPaGroupSpan = 64;
__device__ __forceinline__ PaTok pa_token(const PagedAttnArgs& a, int t) {
  const int c = min(t, a.T - 1), b = max(c - 1, 0), d = min(c + 1, a.T - 1);
  const int pb = a.pos[b], pc = a.pos[c], pd = a.pos[d];   // (one round of loads)
  int sb = 0, sc = c, sd = 0;
  if (a.seq != nullptr) sc = a.seq[c];
  if (a.gmax > 1) {
    sb = a.seq[b];
    sd = a.seq[d];
  }
  PaTok k;
  k.len = pa_rows_of(a, pc);
  k.seq = sc;
  const int start = pa_start(a, k.len);
  auto splits = [&](int s0, int p0, int s1, int p1) {
    return s0 != s1 || p0 < 0 || p1 < p0 || p1 - p0 > kPaGroupSpan ||
           pa_start(a, pa_rows_of(a, p0)) != pa_start(a, pa_rows_of(a, p1));
  };
  k.leads = (c & (a.gmax - 1)) == 0 || splits(sb, pb, sc, pc);
  k.ends = c + 1 == a.T || ((c + 1) & (a.gmax - 1)) == 0 || splits(sc, pc, sd, pd);
  k.own = t < a.T && k.ends ? k.len - start : 0;
  return k;
}

// How the groups' own rows are cut: runs of `chunk` rows, chosen from what the batch attends now (every wavefront
// computes the same), so that a.target workgroups share them evenly. Items are numbered: the whole
// runs of all groups, then the groups' rests (the short ones last, where the last workgroups are waited for).
// first: the lane's token of the first 64 (for more, the others are read in every pass).
struct PaCut { int chunk, whole; float inv; };
__device__ __forceinline__ int pa_runs(const PaCut& c, int n) {   // n / chunk (at most kPaMaxParts)
  int q = (int)((float)n * c.inv);
  q -= q * c.chunk > n ? 1 : 0;
  q += n - q * c.chunk >= c.chunk ? 1 : 0;
  return q;
}
__device__ __forceinline__ int pa_own(const PagedAttnArgs& a, const PaTok& first, int b, int lane) {
  return b == 0 ? first.own : pa_token(a, b + lane).own;
}
__device__ __forceinline__ PaCut pa_cut(const PagedAttnArgs& a, const PaTok& first, int lane) {
  float rows = 0.f;
  int most = 0;
  for (int b = 0; b < a.T; b += kWave) {
    // (sums of 64 lanes in units of 64 rows: below 2^31)
    const int n = pa_own(a, first, b, lane);
    rows += (float)pa_last(pa_wave_incl((n + 63) >> 6)) * 64.f;
    most = max(most, pa_wave_max(n));
  }
  const float even = fminf(rows * (float)a.live / (float)a.target + 1.f, 1e9f);
  PaCut c;
  int chunk = max(max(a.cmin, (int)even), most / (kPaMaxParts - 1) + 1);
  // An even share gives every group a rest beside it: where the card could hold all groups at once, a quarter more rows
  // at a time until it holds all runs and rests, which then need no second round.
  for (int k = 0; k < 8; ++k) {
    c.chunk = (chunk + a.cstep - 1) & -a.cstep;
    c.inv = 1.f / (float)c.chunk;
    c.whole = 0;
    int rests = 0, groups = 0;
    for (int b = 0; b < a.T; b += kWave) {
      const int n = pa_own(a, first, b, lane), w = pa_runs(c, n);
      c.whole += pa_last(pa_wave_incl(w));
      rests += __popcll(__ballot(n - w * c.chunk > 0));
      groups += __popcll(__ballot(n > 0));
    }
    if ((int64_t)(c.whole + rests) * a.live <= a.target || (int64_t)groups * a.live > a.target) break;
    chunk = c.chunk + (c.chunk >> 2);
  }
  return c;
}
// The group (its last token) and run of an item; -1: there is no such item.
__device__ __forceinline__ int pa_find(const PagedAttnArgs& a, const PaTok& first, const PaCut& c, int item, int lane, int* run) {
  int seen = item < c.whole ? 0 : c.whole;
  if (item >= c.whole && a.T <= kWave) {               // rests of up to 64 tokens: the longest first
    const int w = pa_runs(c, first.own), n = lane < a.T ? first.own - w * c.chunk : 0;
    int rank = 0;
    for (int l = 0; l < a.T; ++l) {
      const int o = __builtin_amdgcn_readlane(n, l);
      rank += o > n || (o == n && l < lane) ? 1 : 0;
    }
    const unsigned long long hit = __ballot(n > 0 && rank == item - c.whole);
    if (hit == 0) return -1;
    *run = __builtin_amdgcn_readlane(w, __builtin_ctzll(hit));
    return __builtin_ctzll(hit);
  }
  for (int b = 0; b < a.T; b += kWave) {
    const int n = pa_own(a, first, b, lane), w = pa_runs(c, n);
    const int mine = item < c.whole ? w : (n - w * c.chunk > 0 ? 1 : 0);
    const int incl = seen + pa_wave_incl(mine);
    const unsigned long long hit = __ballot(item < incl && item >= incl - mine);
    if (hit != 0) {
      const int l = __builtin_ctzll(hit);
      *run = item < c.whole ? item - __builtin_amdgcn_readlane(incl - mine, l) : __builtin_amdgcn_readlane(w, l);
      return b + l;
    }
    seen = pa_last(incl);
  }
  return -1;
}
// For the join: per token its group's first whole run, their number, the rest's item or -1, and the group's first token.
__device__ __forceinline__ void pa_write_meta(const PagedAttnArgs& a, const PaTok& first, const PaCut& c, int lane) {
  int whole = 0, rest = c.whole;
  for (int b = 0; b < a.T; b += kWave) {
    const int t = b + lane;
    const PaTok k = b == 0 ? first : pa_token(a, t);
    const int w = pa_runs(c, k.own), r = k.own - w * c.chunk > 0 ? 1 : 0;
    const int iw = whole + pa_wave_incl(w);
    int ir = rest + pa_wave_incl(r);
    if (a.T <= kWave) {
      const int n = t < a.T ? k.own - w * c.chunk : 0;
      ir = c.whole + 1;
      for (int l = 0; l < a.T; ++l) {
        const int o = __builtin_amdgcn_readlane(n, l);
        ir += o > n || (o == n && l < lane) ? 1 : 0;
      }
    }
    // (a group lies within 64 aligned tokens: its first is the last leading lane up to this one)
    const unsigned long long up = __ballot(k.leads && t < a.T) & (~0ull >> (kWave - 1 - lane));
    if (t < a.T && k.ends)
      for (int m = b + 63 - __builtin_clzll(up); m <= t; ++m)
        a.meta[m] = int4{iw - w, w, r ? ir - 1 : -1, b + 63 - __builtin_clzll(up)};
    whole = pa_last(iw);
    rest = pa_last(ir);
  }
}

// FULL: heads are DH elements wide (else up to DH, pieces past a row's end read its last bytes again).
template <typename KT, int DH, int QT, bool FULL, int SHARED = -1>
struct PaShape {
  static constexpr bool F16 = std::is_same<KT, _Float16>::value;
  static constexpr bool SPLIT = F16 && QT == 0;       // both halves of a query in one tile
  static constexpr int NT = QT == 0 ? 1 : QT;         // tiles of 16 query columns
  static constexpr int RT = SPLIT ? 8 : 16 * NT;      // query rows of a workgroup
  static constexpr int SK = F16 ? 32 : 16;            // cache rows of a wavefront's step
  static constexpr int KS = F16 ? DH / 32 : DH / 16;  // 64-byte pieces of a key
  static constexpr int CH = F16 ? (DH == 64 ? 4 : 8) : 4;   // elements of a lane's chunk of a value
  static constexpr int M = DH / (16 * CH);            // chunks of a lane
  static constexpr int DHP = DH + 4;                  // LDS row of the join
  // wavefronts a SIMD: as many as leave each its registers (a register spilled inside the loop would wait for all
  // loads before it, the next step's among them)
  static constexpr int WAVES = DH == 64 ? (QT == 0 ? 4 : 2) : DH == 128 ? (QT == 0 && FULL ? 3 : 2) : 1;
  // queries in LDS (the space of the join) instead of registers: their second halves, or all
  // (own rows, whose steps also tell the tokens of a group apart: all)
  static constexpr bool QLO = F16 && QT == 2 && DH >= 128;
  static constexpr bool QALL = QT == 2 && (DH == 256 || (F16 && DH == 128 && SHARED == 0));
  static constexpr size_t lds() { return (size_t)kPaNW * RT * (DHP + 2) * sizeof(float); }
};

// Between a wavefront's LDS writes and its lanes' reads of each other's words (LDS operations of a wavefront
// complete in order; this keeps the compiler's order).
__device__ __forceinline__ void pa_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Lane l and l ^ 8 of a row of 16; the maximum over the lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float pa_xor8(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));   // row_ror:8
}
__device__ __forceinline__ float pa_max_groups(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Product of a tile: acc += A B.
__device__ __forceinline__ f32x4 pa_mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 pa_mfma4(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// One unit: of the shared rows, or of own rows.
// SHARED: 1 or 0 where the kernel knows, -1 where the workgroup does.
template <typename KT, int DH, int QT, bool FULL, int SHARED>
__device__ __forceinline__ void pa_unit(const PagedAttnArgs& a, float* smem) {
  using Sh = PaShape<KT, DH, QT, FULL, SHARED>;
  constexpr bool F16 = Sh::F16, SPLIT = Sh::SPLIT;
  constexpr int NT = Sh::NT, RT = Sh::RT, SK = Sh::SK, KS = Sh::KS, CH = Sh::CH, M = Sh::M, DHP = Sh::DHP;
  constexpr int NK = F16 ? 8 : 4;                      // cache rows of a lane in the value product
  constexpr int EB = sizeof(KT);
  __shared__ int rows[RT];
  __shared__ int red[kPaNW + 1];
  __shared__ int glen[RT];                             // rows that the tokens of the group attend
  __shared__ float qfac[RT];
  __shared__ int64_t offs[kPaNW][2][SK];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;   // (a scalar: so are the steps)
  const int col = lane & 15, grp = lane >> 4;

  // ---- the unit: query rows (rows[0..nr): index t n + j, or -1), key head, cache rows [k0, k1), place of its partials
  int h, tile, k0, k1, c0 = 0, c1 = 0;                 // [c0, c1): candidates of head sets to look through
  int group = 1, lead = 0;                             // tokens of the unit (own rows), the first
  int sq = -1;                                         // its sequence (shared rows: any that attends them)
  int64_t place0;                                      // partials: row index * SP + part, or workgroup * RW + row
  const bool shared = SHARED < 0 ? (int)blockIdx.x < a.n_shared : SHARED == 1;
  if (shared) {
    // the row tiles of a part 8 workgroups apart: on one XCD, whose L2 then holds the part's keys and values
    const int b = blockIdx.x, x = b & 7, y = b >> 3;
    const int u = (y / a.row_tiles) * 8 + x;
    tile = y % a.row_tiles;
    if (u >= a.g.H * a.SP) return;
    h = u / a.SP;
    const int part = u - h * a.SP;
    place0 = part;
    k0 = part * a.CP;
    k1 = min(k0 + a.CP, a.P);
    if (a.heads != nullptr) c1 = a.T * a.n;
    if (a.heads == nullptr && tid < RT) {
      const int c = tile * RT + tid;
      int idx = -1;
      if (c < a.T * a.G) {
        const int t = c / a.G;
        if (pa_len(a, t) >= a.P) idx = t * a.n + h * a.G + (c - t * a.G);
      }
      rows[tid] = idx;
    }
  } else {
    const int id = (int)blockIdx.x - a.n_shared;
    const int item = id / a.U, u = id - item * a.U;
    int t = item, run = 0, chunk = INT32_MAX;
    if (a.target > 0) {
      const PaTok tok = pa_token(a, lane);
      const PaCut cut = pa_cut(a, tok, lane);
      if (id == 0 && wave == 0) pa_write_meta(a, tok, cut, lane);
      t = pa_find(a, tok, cut, item, lane, &run);
      if (t < 0) return;
      chunk = cut.chunk;
    }
    // lane k: token t - k (its group's first is the nearest that leads; t is its group's last, or there is nothing to do)
    const PaTok tok = pa_token(a, max(t - lane, 0));
    if (!__builtin_amdgcn_readfirstlane((int)tok.ends)) return;
    lead = t - (a.gmax > 1 ? __builtin_ctzll(__ballot(tok.leads)) : 0);
    group = t - lead + 1;
    sq = __builtin_amdgcn_readfirstlane(tok.seq);
    if (wave == 0 && lane < group) glen[group - 1 - lane] = tok.len;
    const bool single = a.heads != nullptr && a.G == 1;   // one row: the unit is (token, place in its set)
    if (single) {
      tile = 0;
      h = min(max(a.heads[(int64_t)t * a.n + u], 0), a.g.H - 1);
      if (tid < RT) rows[tid] = tid == 0 ? t * a.n + u : -1;
    } else {
      h = u / a.group_tiles;
      tile = u - h * a.group_tiles;
      if (a.heads == nullptr) {
        if (tid < RT) {
          const int r = tile * RT + tid, g = r / a.G;    // (group > 1: one tile)
          rows[tid] = r < group * a.G ? (lead + g) * a.n + h * a.G + (r - g * a.G) : -1;
        }
      } else {
        c0 = t * a.n;
        c1 = c0 + a.n;
      }
    }
    const int len = __builtin_amdgcn_readfirstlane(tok.len);
    k0 = pa_start(a, len) + run * (run > 0 ? chunk : 0);
    k1 = chunk < len - k0 ? k0 + chunk : len;
    place0 = (int64_t)id * a.RW;
    // nothing of its own to attend: the join does without, a direct output is still to be written
    if (k0 >= k1 && !a.direct) return;
  }
  if (c1 > c0) {
    // this tile's RT of the candidates whose query head belongs to key head h (and, for the shared rows, whose
    // token attends all of them), in order
    if (tid < RT) rows[tid] = -1;
    int seen = 0;
    for (int b = c0; b < c1 && seen < (tile + 1) * RT; b += kPaNT) {
      const int c = b + tid;
      bool mine = c < c1 && min(max(a.heads[c], 0), a.g.H * a.G - 1) / a.G == h;
      if (shared && mine) mine = pa_len(a, c / a.n) >= a.P;
      int total;
      const int at = seen + block_excl_scan<kPaNT>(mine ? 1 : 0, red, &total) - tile * RT;
      if (mine && at >= 0 && at < RT) rows[at] = c;
      seen += total;
    }
  }
  __syncthreads();
  // rows in use, and the sequence whose pages are read: that of the first
  int nr, first;
  {
    const int r = lane < RT ? rows[lane] : -1;
    const unsigned long long on = __ballot(r >= 0);
    if (on == 0) return;
    nr = 64 - __builtin_clzll(on);
    first = __builtin_amdgcn_readfirstlane(rows[__builtin_ctzll(on)]);
  }
  // (scalars: every thread has the same)
  k0 = __builtin_amdgcn_readfirstlane(k0);
  k1 = __builtin_amdgcn_readfirstlane(k1);
  h = __builtin_amdgcn_readfirstlane(h);
  lead = __builtin_amdgcn_readfirstlane(lead);
  group = __builtin_amdgcn_readfirstlane(group);
  if (k0 >= k1) {                                      // (direct only) nothing attended: 0, log of 0
    for (int x = tid; x < nr * a.ldo; x += kPaNT) {
      const int r = x / a.ldo, d = x - r * a.ldo;
      a.out[(int64_t)rows[r] * a.ldo + d] = a.ldo != a.g.dh && d == 1 ? 1.f : 0.f;
      if (d == 0 && a.lse != nullptr) a.lse[rows[r]] = -INFINITY;
    }
    return;
  }
  if (shared) sq = a.seq != nullptr ? a.seq[first / a.n] : first / a.n;
  sq = __builtin_amdgcn_readfirstlane(min(max(sq, 0), a.g.n_seq - 1));
  const int32_t* trow = a.g.table + (int64_t)sq * a.g.max_pages;
  const int rowb = FULL ? DH * EB : a.g.dh * EB;
  // this lane's piece of a key, chunk of a value (FULL: the others are at constant distances)
  const char* Kh = a.g.K + h * a.g.hs + (FULL ? grp * 16 : 0);
  const char* Vh = a.g.V + h * a.g.hs + (FULL ? col * CH * EB : 0);

  // ---- steps of this wavefront: cache rows key_of(i) .. + SK; at least one (rows past the end are masked, their loads
  // go to the last row: every wavefront and step runs the same path, so the waits count its own loads exactly)
  auto key_of = [&](int i) { return k0 + (i * kPaNW + wave) * SK; };
  const int nsteps = max(1, (k1 - key_of(0) + kPaNW * SK - 1) / (kPaNW * SK));
  auto page_load = [&](int i) {
    int row;
    return trow[page_of(a.g, min(key_of(i) + (lane & (SK - 1)), k1 - 1), &row)];
  };
  auto place = [&](int i, int id, int buf) {           // the step's row offsets (written twice where SK < 64)
    int row;
    (void)page_of(a.g, min(key_of(i) + (lane & (SK - 1)), k1 - 1), &row);
    offs[wave][buf][lane & (SK - 1)] = min(max(id, 0), a.g.n_pages - 1) * a.g.ps + row * a.g.rs;
  };
  using VT = typename std::conditional<F16 && CH == 4, u32x2, u32x4>::type;
  u32x4 kr[SK / 16][KS];
  VT vr[NK][M];
  // (pieces past the head width read its last bytes: their queries are zero, their outputs not written)
  auto load_k = [&](int buf) {
    pa_wave_sync();
#pragma unroll
    for (int u = 0; u < SK / 16; ++u) {
      const char* p = Kh + offs[wave][buf][u * 16 + col];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const char* pp = p + (FULL ? ks * 64 : min(ks * 64 + grp * 16, rowb - 16));
        kr[u][ks] = QT == 0 ? ld_stream(pp) : ld_plain(pp);
      }
    }
  };
  auto load_v = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const char* p = Vh + offs[wave][buf][(i >> 2) * 16 + grp * 4 + (i & 3)];
#pragma unroll
      for (int m = 0; m < M; ++m) {
        const VT* pp = reinterpret_cast<const VT*>(
            p + (FULL ? m * 16 * (int)sizeof(VT) : min((m * 16 + col) * (int)sizeof(VT), rowb - (int)sizeof(VT))));
        vr[i][m] = QT == 0 ? __builtin_nontemporal_load(pp) : *pp;
      }
    }
  };
  // ---- queries, asked for before the first keys and values (loads return in order). One tile: by every wavefront for
  // itself. More: tile w by wavefront w for all, through LDS (the space of the join)
  constexpr int Q4 = F16 ? 2 : 1;                      // float4 of a piece
  const bool mine = QT == 0 || wave < NT;
  f32x4 x[KS][Q4];
  if (mine) {
    const int idx = rows[SPLIT ? col & 7 : (QT == 0 ? 0 : wave) * 16 + col];
    const float* qp = a.q + (int64_t)max(idx, 0) * a.g.dh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < Q4; ++i) {
        const int d = ks * 16 * Q4 + grp * 4 * Q4 + i * 4;
        const f32x4 v = *reinterpret_cast<const f32x4*>(qp + (FULL ? d : min(d, a.g.dh - 4)));
        x[ks][i] = idx >= 0 && (FULL || d < a.g.dh) ? v : f32x4{0.f, 0.f, 0.f, 0.f};
      }
  }
  int klim[NT], ktok[NT];                              // end of a column's rows, its token in the group
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int idx = rows[SPLIT ? col & 7 : nt * 16 + col];
    klim[nt] = k1;
    ktok[nt] = 0;
    if (group > 1 && idx >= 0) {
      ktok[nt] = idx / a.n - lead;
      klim[nt] = min(k1, glen[ktok[nt]]);
    }
  }
  // (ascending: the first has the fewest)
  const int kmin = __builtin_amdgcn_readfirstlane(group > 1 ? min(k1, glen[0]) : k1);
  place(0, page_load(0), 0);
  int id1 = page_load(1);
  load_k(0);
  load_v(0);
  // scaled halves (fp16) or as they are, and the factor >= 0 from products to base-2 logits (a negative
  // scale's sign goes to the queries)
  const float sign = a.scale < 0.f ? -1.f : 1.f;
  u32x4 qh[Sh::QALL ? 1 : NT][Sh::QALL ? 1 : KS], ql[NT][SPLIT || !F16 || Sh::QLO ? 1 : KS];
  u32x4* qlds = reinterpret_cast<u32x4*>(smem) + lane;  // [first, second half][nt][ks][lane]
  float cf[NT];
  if (mine) {
    const int tq = QT == 0 ? 0 : wave;
    float c = fabsf(a.scale);
    int ex = 0;
    if constexpr (F16) {
      float mx = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf(x[ks][e >> 2][e & 3]));
      mx = pa_max_groups(mx);
      ex = 14 - ((int)((__float_as_uint(mx) >> 23) & 255u) - 127);   // largest element to [2^14, 2^15)
      c = ldexpf(c, -ex);
    }
    if constexpr (QT == 0)
      cf[0] = c;
    else if (grp == 0)
      qfac[tq * 16 + col] = c;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4 first, second;
      if constexpr (F16) {
        f16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = ldexpf(sign * x[ks][e >> 2][e & 3], ex);
          hi[e] = (_Float16)v;
          lo[e] = (_Float16)(v - (float)hi[e]);
        }
        first = __builtin_bit_cast(u32x4, hi);
        second = __builtin_bit_cast(u32x4, lo);
      } else {
        first = second = __builtin_bit_cast(u32x4, x[ks][0] * sign);
      }
      if constexpr (QT == 0) {
        qh[0][ks] = !SPLIT || col < 8 ? first : second;
      } else {
        qlds[(tq * KS + ks) * kWave] = first;
        if constexpr (F16) qlds[((NT + tq) * KS + ks) * kWave] = second;
      }
    }
  }
  if constexpr (QT > 0) {
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      cf[nt] = qfac[nt * 16 + col];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if constexpr (!Sh::QALL) qh[nt][ks] = qlds[(nt * KS + ks) * kWave];
        if constexpr (F16 && !Sh::QLO) ql[nt][ks] = qlds[((NT + nt) * KS + ks) * kWave];
      }
    }
  }

  // ---- a step: logits, running maximum, probabilities, values
  float m[NT], l[NT];
  f32x4 o[NT][M * CH];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = -INFINITY;
    l[nt] = 0.f;
#pragma unroll
    for (int e = 0; e < M * CH; ++e) o[nt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto step = [&](int i, auto last_c) {
    constexpr bool LAST = decltype(last_c)::value;
    const int base = key_of(i);
    // rows of the step are behind the end of a column's rows (of a group of one: in the last step alone)
    const bool tail = (SHARED != 1 || LAST) && base + SK > kmin;
    f32x4 s[NT][SK / 16];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int u = 0; u < SK / 16; ++u) {
        s[nt][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const u32x4 q0 = Sh::QALL ? qlds[(nt * KS + ks) * kWave] : qh[Sh::QALL ? 0 : nt][Sh::QALL ? 0 : ks];
          if constexpr (F16) {
            s[nt][u] = pa_mfma(kr[u][ks], q0, s[nt][u]);
            if constexpr (!SPLIT)
              s[nt][u] = pa_mfma(kr[u][ks], Sh::QLO ? qlds[((NT + nt) * KS + ks) * kWave] : ql[nt][Sh::QLO ? 0 : ks], s[nt][u]);
          } else {
            s[nt][u] = pa_mfma4(__builtin_bit_cast(f32x4, kr[u][ks]), __builtin_bit_cast(f32x4, q0), s[nt][u]);
          }
        }
      }
    // the next step's keys take the registers of this one's; its values follow behind the value products
    if constexpr (!LAST) {
      place(i + 1, id1, (i + 1) & 1);
      id1 = page_load(i + 2);
      load_k((i + 1) & 1);
    }
    u32x4 ph[NT], pl[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if constexpr (SPLIT) {
#pragma unroll
        for (int u = 0; u < SK / 16; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[nt][u][e] += pa_xor8(s[nt][u][e]);
      }
      // (scaled before the maximum is taken: a product needs no quieting of NaN, which would be an instruction each)
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < SK / 16; ++u) {
        s[nt][u] *= cf[nt];
        if (tail) {
#pragma unroll
          for (int e = 0; e < 4; ++e) s[nt][u][e] = base + u * 16 + grp * 4 + e < klim[nt] ? s[nt][u][e] : -INFINITY;
        }
        mx = fmaxf(fmaxf(mx, s[nt][u][0]), s[nt][u][1]);
        mx = fmaxf(fmaxf(mx, s[nt][u][2]), s[nt][u][3]);
      }
      mx = pa_max_groups(mx);
      if (__any(mx > m[nt])) {
        const float mn = fmaxf(m[nt], mx);
        const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[nt] - mn);
        m[nt] = mn;
        l[nt] *= f;
#pragma unroll
        for (int e = 0; e < M * CH; ++e) o[nt][e] *= f;
      }
      // (times 2^14 for fp16, so that small ones keep both halves; the sum has the same factor)
      const float mu = (m[nt] == -INFINITY ? 0.f : m[nt]) - (F16 ? 14.f : 0.f);
#pragma unroll
      for (int u = 0; u < SK / 16; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(s[nt][u][e] - mu);
          l[nt] += p;
          s[nt][u][e] = p;
        }
      if constexpr (F16) {
        // first halves rounded towards zero (one instruction a pair), second halves to nearest: 2^-22 in all
        u32x4 hi, lo;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p0 = s[nt][j >> 1][(j & 1) * 2], p1 = s[nt][j >> 1][(j & 1) * 2 + 1];
          const f16x2 h = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(p0, p1));
          const f16x2 r = {(_Float16)(p0 - (float)h[0]), (_Float16)(p1 - (float)h[1])};
          hi[j] = __builtin_bit_cast(uint32_t, h);
          lo[j] = __builtin_bit_cast(uint32_t, r);
        }
        if constexpr (SPLIT) {
#pragma unroll
          for (int j = 0; j < 4; ++j) ph[nt][j] = col < 8 ? hi[j] : lo[j];
        } else {
          ph[nt] = hi;
          pl[nt] = lo;
        }
      } else {
        ph[nt] = __builtin_bit_cast(u32x4, s[nt][0]);
      }
    }
    // Values behind a token's rows may be anything, and 0 times infinity is not 0: there token by token, from the
    // one with the most rows, with what is behind its rows zeroed and the other tokens' probabilities 0. What is not finite
    // would still reach their sums: such pieces are zeroed first, and the tokens that attend one of those rows get
    // probabilities of NaN.
    int first_bad = INT_MAX;
    if (tail && group > 1) {
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const int row = base + (k >> 2) * 16 + grp * 4 + (k & 3);
        uint32_t bad = 0;
#pragma unroll
        for (int mm = 0; mm < M; ++mm)
#pragma unroll
          for (int w = 0; w < (int)(sizeof(VT) / 4); ++w)
            if constexpr (F16)
              bad |= (vr[k][mm][w] & 0x7c007c00u) + 0x04000400u;   // bit 15 or 31: an exponent of all ones
            else
              bad |= (vr[k][mm][w] & 0x7f800000u) + 0x00800000u;   // bit 31
        if (bad & (F16 ? 0x80008000u : 0x80000000u)) {
          if (row < k1) first_bad = min(first_bad, row);
#pragma unroll
          for (int mm = 0; mm < M; ++mm) vr[k][mm] = VT{};
        }
      }
      for (int i = 1; i < kWave; i *= 2) first_bad = min(first_bad, __shfl_xor(first_bad, i, kWave));
      first_bad = __builtin_amdgcn_readfirstlane(first_bad);
    }
    for (int g = tail ? group - 1 : 0; g >= 0; --g) {
      uint32_t nan = 0;
      if (tail) {
        const int end = group > 1 ? min(k1, glen[g]) : k1;
        if (first_bad < end) nan = F16 ? 0x7e007e00u : 0x7fc00000u;
#pragma unroll
        for (int k = 0; k < NK; ++k)
          if (base + (k >> 2) * 16 + grp * 4 + (k & 3) >= end)
#pragma unroll
            for (int mm = 0; mm < M; ++mm) vr[k][mm] = VT{};
      }
      u32x4 th[NT], tl[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const uint32_t own = tail && ktok[nt] != g ? 0u : ~0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          th[nt][j] = (ph[nt][j] & own) | (nan & own);
          if constexpr (F16 && !SPLIT) tl[nt][j] = (pl[nt][j] & own) | (nan & own);
        }
      }
#pragma unroll
      for (int mm = 0; mm < M; ++mm)
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          if constexpr (F16) {
            // element e of the lane's chunks of its eight rows, two to a register
            u32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k)
              v[k] = __builtin_amdgcn_perm(vr[2 * k + 1][mm][e >> 1], vr[2 * k][mm][e >> 1],
                                           e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              o[nt][mm * CH + e] = pa_mfma(v, th[nt], o[nt][mm * CH + e]);
              if constexpr (!SPLIT) o[nt][mm * CH + e] = pa_mfma(v, tl[nt], o[nt][mm * CH + e]);
            }
          } else {
            f32x4 v;
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(vr[k][mm][e]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              o[nt][mm * CH + e] = pa_mfma4(v, __builtin_bit_cast(f32x4, th[nt]), o[nt][mm * CH + e]);
          }
        }
    }
    if constexpr (!LAST) load_v((i + 1) & 1);
  };
  for (int i = 0; i + 1 < nsteps; ++i) step(i, std::false_type{});
  step(nsteps - 1, std::true_type{});

  // ---- join the wavefronts: every one writes its sums (zeros where it had no step), then all threads add
  if constexpr (QT > 0) __syncthreads();               // (the queries lie there)
  float* sm_o = smem;                                  // [wave][RT][DHP]
  float* sm_m = smem + kPaNW * RT * DHP;               // [wave][RT]
  float* sm_l = sm_m + kPaNW * RT;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (nt > 0 && nt * 16 >= nr) break;
    l[nt] += __shfl_xor(l[nt], 16, kWave);
    l[nt] += __shfl_xor(l[nt], 32, kWave);
    if constexpr (SPLIT) {
#pragma unroll
      for (int e = 0; e < M * CH; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nt][e][i] += __shfl_xor(o[nt][e][i], 8, kWave);
    }
    const int r = nt * 16 + col;
    if (r < RT) {
      float* po = sm_o + (wave * RT + r) * DHP;
#pragma unroll
      for (int mm = 0; mm < M; ++mm)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < CH; e += 4) {
            const int k = mm * CH + e;
            *reinterpret_cast<f32x4*>(po + (mm * 16 + grp * 4 + i) * CH + e) =
                f32x4{o[nt][k][i], o[nt][k + 1][i], o[nt][k + 2][i], o[nt][k + 3][i]};
          }
      if (grp == 0) {
        sm_m[wave * RT + r] = m[nt];
        sm_l[wave * RT + r] = l[nt];
      }
    }
  }
  __syncthreads();
  // LPR threads a row, the rows of a pass next to each other
  constexpr int LPR = DH / 4, RP = kPaNT / LPR;
  const int d = tid % LPR * 4;
#pragma unroll
  for (int r0 = 0; r0 < RT; r0 += RP) {
    const int r = r0 + tid / LPR;
    const int idx = r < nr ? rows[r] : -1;             // (RT may be below RP)
    if (idx < 0 || (!FULL && d >= a.g.dh)) continue;
    float mw[kPaNW], lw[kPaNW], mt = -INFINITY, lt = 0.f;
    f32x4 v[kPaNW];
#pragma unroll
    for (int w = 0; w < kPaNW; ++w) {
      mw[w] = sm_m[w * RT + r];
      lw[w] = sm_l[w * RT + r];
      v[w] = *reinterpret_cast<const f32x4*>(sm_o + (w * RT + r) * DHP + d);
      mt = fmaxf(mt, mw[w]);
    }
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kPaNW; ++w) {
      const float f = mw[w] == -INFINITY ? (mt == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(mw[w] - mt);
      lt = fmaf(lw[w], f, lt);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(v[w][e], f, acc[e]);
    }
    const float me = mt - (F16 ? 14.f : 0.f);          // the sums' own factor
    if (a.direct) {
      const float rl = lt == 0.f ? 0.f : 1.f / lt;
      float* out = a.out + (int64_t)idx * a.ldo;
      if (a.ldo != a.g.dh) {                            // partials' form, for the out-projection
        if (d == 0) {
          out[0] = 0.f;
          out[1] = 1.f;
        }
        out += 2;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[d + e] = acc[e] * rl;
      } else {
        *reinterpret_cast<f32x4*>(out + d) = acc * rl;
      }
      if (d == 0 && a.lse != nullptr)
        a.lse[idx] = lt == 0.f ? -INFINITY : (me + __builtin_amdgcn_logf(lt)) * kPaLn2;
    } else {
      float* po = shared ? a.so + ((int64_t)idx * a.SP + place0) * a.g.dh : a.oo + (place0 + r) * a.g.dh;
      float* pm = shared ? a.sml + ((int64_t)idx * a.SP + place0) * 2 : a.oml + (place0 + r) * 2;
      *reinterpret_cast<f32x4*>(po + d) = acc;
      if (d == 0) {
        pm[0] = me;
        pm[1] = lt;
      }
    }
  }
}

// QS, QO: variants of the shared and the own rows' units (a batch has many query rows for the shared ones, a token few).
template <typename KT, int DH, int QS, int QO, bool FULL>
__global__ void __launch_bounds__(kPaNT, (PaShape<KT, DH, QS, FULL>::WAVES)) k_paged_attn(PagedAttnArgs a) {
  extern __shared__ float smem[];
  if constexpr (QS == 0) {
    pa_unit<KT, DH, 0, FULL, -1>(a, smem);
  } else {
    if ((int)blockIdx.x < a.n_shared)
      pa_unit<KT, DH, QS, FULL, 1>(a, smem);
    else
      pa_unit<KT, DH, QO, FULL, 0>(a, smem);
  }
}

// Rows' partials joined: a wavefront per row; the parts' weights in lanes, then their value sums, two parts at a
// time (half a wavefront each) where a row is at most 32 chunks of four.
__global__ void __launch_bounds__(kPaNT) k_paged_combine(PagedAttnArgs a) {
  const int idx = (int)blockIdx.x * kPaNW + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (idx >= a.T * a.n) return;
  const int t = idx / a.n, j = idx - t * a.n;
  const int len = pa_len(a, t), start = pa_start(a, len);
  // parts: [0, sp) of the shared rows, then the group's whole runs, then its rest
  int4 meta = a.target > 0 ? a.meta[t] : int4{t, len > start ? 1 : 0, -1, t};
  if (len == start) meta.y = 0, meta.z = -1;
  const int sp = start > 0 ? a.SP : 0, ns = sp + meta.y + (meta.z >= 0 ? 1 : 0);
  // the row's unit and place among the workgroup's rows
  int u = j, r = 0;
  if (a.heads == nullptr) {
    const int h = j / a.G, q = (t - meta.w) * a.G + (j - h * a.G), tile = q / a.RT;
    u = h * a.group_tiles + tile;
    r = q - tile * a.RT;
  } else if (a.G > 1) {
    const int32_t* set = a.heads + (int64_t)t * a.n;
    const int h = min(max(set[j], 0), a.g.H * a.G - 1) / a.G;
    int rank = 0;
    for (int b = 0; b < j; b += kWave)
      rank += __popcll(__ballot(b + lane < j && min(max(set[min(b + lane, j)], 0), a.g.H * a.G - 1) / a.G == h));
    u = h * a.group_tiles + rank / a.RT;
    r = rank % a.RT;
  }
  auto part_ml = [&](int s) {
    return s < sp ? a.sml + ((int64_t)idx * a.SP + s) * 2
                  : a.oml + (((int64_t)(s - sp < meta.y ? meta.x + s - sp : meta.z) * a.U + u) * a.RW + r) * 2;
  };
  auto part_o = [&](int s) {
    return s < sp ? a.so + ((int64_t)idx * a.SP + s) * a.g.dh
                  : a.oo + (((int64_t)(s - sp < meta.y ? meta.x + s - sp : meta.z) * a.U + u) * a.RW + r) * a.g.dh;
  };
  float w[2], m[2], l[2];
  float mt = -INFINITY;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = lane + 64 * i;
    m[i] = -INFINITY;
    l[i] = 0.f;
    if (s < ns) {
      const float* p = part_ml(s);
      m[i] = p[0];
      l[i] = p[1];
    }
    mt = fmaxf(mt, m[i]);
  }
  mt = wave_max(mt);
  float lt = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = m[i] == -INFINITY ? (mt == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(m[i] - mt);
    lt = fmaf(l[i], w[i], lt);
  }
  lt = wave_sum(lt);
  const bool two = a.g.dh <= 128;
  const int half = two ? lane >> 5 : 0, d = (two ? lane & 31 : lane) * 4, step = two ? 2 : 1;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < ns; s0 += 4 * step) {
    f32x4 v[4];
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = s0 + i * step + half, sc = min(s, ns - 1);
      v[i] = *reinterpret_cast<const f32x4*>(part_o(sc) + min(d, a.g.dh - 4));
      const float f0 = __shfl(w[0], sc & 63, kWave), f1 = __shfl(w[1], sc & 63, kWave);
      f[i] = sc < 64 ? f0 : f1;
      if (s >= ns) v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[k] = fmaf(v[i][k], f[i], acc[k]);
  }
  if (two) {
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] += __shfl_xor(acc[k], 32, kWave);
  }
  const float rl = lt == 0.f ? 0.f : 1.f / lt;
  float* out = a.out + (int64_t)idx * a.ldo;
  if (a.ldo != a.g.dh) {
    if (lane == 0) {
      out[0] = 0.f;
      out[1] = 1.f;
    }
    out += 2;
    if (half == 0 && d < a.g.dh)
      for (int k = 0; k < 4; ++k) out[d + k] = acc[k] * rl;
  } else if (half == 0 && d < a.g.dh) {
    *reinterpret_cast<f32x4*>(out + d) = acc * rl;
  }
  if (lane == 0 && a.lse != nullptr) a.lse[idx] = lt == 0.f ? -INFINITY : (mt + __builtin_amdgcn_logf(lt)) * kPaLn2;
}

hipError_t launch_paged_combine(const PagedAttnArgs& a, hipStream_t st) {
  launch_k(k_paged_combine, dim3((a.T * a.n + kPaNW - 1) / kPaNW), dim3(kPaNT), 0, st, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------ launch
// Query rows of a workgroup: the smaller tile if it holds a unit's rows (kernel variant QT).
// (8 rows with their second halves beside them against the tile of 32: 8 query heads a key head, 8000 to 50000 rows, 114 us
// against 132; 6 to 12 rows of drafts 11.8 against 15.4; 8 tokens of a shared prefix 37.5 against 38.8.)
static int pa_rows(int ktype, int qt) { return qt == 0 ? (ktype == DV_F16 ? 8 : 16) : 16 * qt; }
static int pa_variant(int ktype, int64_t most) { return most <= pa_rows(ktype, 0) ? 0 : 2; }

// Tokens that the table's sequences have on average (what is not known on the host is assumed), and query rows of the
// largest unit of own rows: those of a key head of so many tokens.
static int pa_drafts(const PagedAttnArgs& a) {
  return a.seq != nullptr && a.heads == nullptr ? min((a.T + a.g.n_seq - 1) / a.g.n_seq, 32) : 1;
}
static int pa_own_rows(const PagedAttnArgs& a) { return (a.heads != nullptr ? min(a.G, a.n) : a.G) * pa_drafts(a); }

// Least rows of a workgroup: 64 KB of keys, 64 to 256 of them. (One sequence of 2000 rows, 12 heads of 64 fp32, twelve workgroups
// a run: 12.0 us in 256, 10.4 in 128 with 1.5 more in the join, 15.2 in 512; where there are more heads or sequences
// the even share is longer. 2 tokens, 8 query on 2 heads of 256 fp32, 372 and 1206 rows: 26.7 us in 256, 21.9 in 64.
// 24 drafts of 5 heads of 192 fp32 on 1184 shared rows: 58 and 35.)
constexpr int kPaLeastBytes = 65536;
static int pa_least(const PagedAttnArgs& a, int ktype) {
  return min(max(kPaLeastBytes / (a.g.dh * (ktype == DV_F16 ? 2 : 4)), 64), 256);
}
// Lengths that one workgroup takes alone, its result needing no join: twice the least while the units do not fill the card,
// up to eight times it where they fill it four times over. (12 heads of 64 fp32: 512 rows 13.7 us, cut 18.6; 1000 rows 20.3, cut 16 to 19. 32
// tokens of 32 of 96 heads of 128 fp16, 1024 units: up to 1000 rows 78 us, cut 84; 12000 units of up to 1000 rows 491, cut 648.)
static int pa_alone(int least, int64_t units, int64_t resident) {
  return (units < resident ? 2 : units < 4 * resident ? 4 : 8) * least;
}
// Tokens up to which the rows are cut evenly: every wavefront looks at all positions. (64 query heads on 8 of 128 fp16, 100 to
// 6000 rows: 100 tokens 245 us, a workgroup a token 272; 300 tokens 703 and 680; 600 tokens of 100 to 4000 rows 911 and 840.)
constexpr int kPaMaxScan = 1024;

void plan_paged_attn(PagedAttnArgs* a, int ktype) {
  const int cus = device_cu_count();
  const int group = a->heads != nullptr ? min(a->G, a->n) : a->G;
  const int qs = a->P > 0 ? pa_variant(ktype, (int64_t)a->T * group) : 0;
  // (one token attends the shared rows with as many query rows as its own)
  const int qo = min(pa_variant(ktype, pa_own_rows(*a)), a->P > 0 ? qs : 2), qt = max(qs, qo);
  a->RT = pa_rows(ktype, qo);
  a->RTS = pa_rows(ktype, qs);
  // workgroups that a CU holds (PaShape::WAVES)
  const int per_cu = a->g.dh <= 64 ? (qt == 0 ? 4 : 2) : a->g.dh <= 128 ? (qt == 0 ? 3 : 2) : 1;
  const int64_t resident = (int64_t)per_cu * cus;
  const bool single = a->heads != nullptr && a->G == 1;
  a->row_tiles = a->P > 0 ? (int)(((int64_t)a->T * group + a->RTS - 1) / a->RTS) : 0;
  a->group_tiles = (group + a->RT - 1) / a->RT;
  a->U = single ? a->n : a->g.H * a->group_tiles;
  // units of a token that have query rows: of a set of grouped heads as many as it has heads at most (64 tokens of 1 of 8 heads
  // on 4, 4000 to 17600 rows: 103 us, cut as if all four had some 183)
  a->live = a->heads != nullptr ? min(a->U, a->n) : a->U;
  a->cmin = pa_least(*a, ktype);
  a->cstep = kPaNW * (ktype == DV_F16 ? 32 : 16);
  const int64_t units = (int64_t)a->T * a->live, own = a->max_len - a->P;
  // A workgroup a token: where each may be taken alone, and beside shared rows for more tokens than a wavefront's lanes that
  // are no drafts, which would lose their groups (32 heads of 128 fp16, 16 to 700 own rows: 100 tokens 158 us against 174,
  // 600 tokens 811 against 1118).
  const bool alone = own <= pa_alone(a->cmin, units, resident);
  const bool whole = a->T > kPaMaxScan || (alone && a->P > 0 && a->T > kWave && pa_drafts(*a) == 1);
  a->direct = a->P == 0 && (whole || alone);
  a->gmax = 1;
  if (a->seq != nullptr && a->heads == nullptr && (a->direct || !whole))
    while (2 * a->gmax * a->G <= a->RT) a->gmax *= 2;
  a->RW = min(a->RT, a->gmax * group);
  // The shared rows' parts: their share of the resident workgroups if all tokens had max_len (but no more than as many rows
  // of their own), one a CU at least, the least rows each at least.
  a->SP = 0;
  a->CP = 1;
  int64_t shared = 0;
  if (a->P > 0) {
    const int64_t tiles = (int64_t)a->g.H * a->row_tiles;
    const int64_t cost = tiles * a->P, others = units * min(own, (int64_t)a->P);
    const int64_t want = max((int64_t)cus, resident * cost / (cost + others));
    const int64_t parts = max((int64_t)1, min(min((int64_t)kPaMaxParts, (want + tiles - 1) / tiles), (int64_t)a->P / a->cmin));
    a->CP = (int)((a->P + parts - 1) / parts + a->cstep - 1) / a->cstep * a->cstep;
    a->SP = (a->P + a->CP - 1) / a->CP;
    shared = tiles * a->SP;
  }
  a->n_shared = a->P > 0 ? (a->g.H * a->SP + 7) / 8 * 8 * a->row_tiles : 0;
  a->target = a->direct || whole ? 0 : (int)max(resident - shared, (int64_t)cus);
  a->items = a->T + (a->target > 0 ? (a->target + a->live - 1) / a->live : 0);
}

template <typename KT, int DH, int QS, int QO, bool FULL>
static hipError_t launch_pa(const PagedAttnArgs& a, hipStream_t st) {
  const size_t lds = PaShape<KT, DH, QS, FULL>::lds();
  const hipError_t e = ensure_dyn_lds(reinterpret_cast<const void*>(k_paged_attn<KT, DH, QS, QO, FULL>), lds);
  if (e != hipSuccess) return e;
  launch_k((k_paged_attn<KT, DH, QS, QO, FULL>), dim3((unsigned)(a.n_shared + (int64_t)a.items * a.U)), dim3(kPaNT), lds, st, a);
  return hipGetLastError();
}

template <typename KT, int DH, int QS, int QO>
static hipError_t launch_pa_q(const PagedAttnArgs& a, hipStream_t st) {
  return a.g.dh == DH ? launch_pa<KT, DH, QS, QO, true>(a, st) : launch_pa<KT, DH, QS, QO, false>(a, st);
}

template <typename KT, int QS, int QO>
static hipError_t launch_pa_d(const PagedAttnArgs& a, hipStream_t st) {
  if (a.g.dh <= 64) return launch_pa_q<KT, 64, QS, QO>(a, st);
  return a.g.dh <= 128 ? launch_pa_q<KT, 128, QS, QO>(a, st) : launch_pa_q<KT, 256, QS, QO>(a, st);
}

template <typename KT>
static hipError_t launch_pa_k(int ktype, const PagedAttnArgs& a, hipStream_t st) {
  if (a.RT > pa_rows(ktype, 0)) return launch_pa_d<KT, 2, 2>(a, st);
  return a.P > 0 && a.RTS > pa_rows(ktype, 0) ? launch_pa_d<KT, 2, 0>(a, st) : launch_pa_d<KT, 0, 0>(a, st);
}

hipError_t launch_paged_attn(int ktype, const PagedAttnArgs& a, hipStream_t st) {
  return ktype == DV_F16 ? launch_pa_k<_Float16>(ktype, a, st) : launch_pa_k<float>(ktype, a, st);
}

// ------------------------------------------------------------------ DV_VALIDATE
// One workgroup over all tokens and their pages.
__global__ void __launch_bounds__(1024) k_paged_validate(Pages g, const int32_t* seq, const int32_t* pos, int T,
                                                         int max_len, int shared, int32_t* bad) {
  __shared__ int fail, lead;
  if (threadIdx.x == 0) {
    fail = 0;
    lead = T;
  }
  __syncthreads();
  const int P = shared * g.page;
  for (int t = threadIdx.x; t < T; t += 1024) {
    const int s = seq != nullptr ? seq[t] : t;
    if (pos[t] >= max_len || (pos[t] >= 0 && (s < 0 || s >= g.n_seq))) fail = 1;
    if (P > 0 && pos[t] + 1 >= P && pos[t] < max_len && s >= 0 && s < g.n_seq) atomicMin(&lead, t);
  }
  __syncthreads();
  if (fail == 0) {
    const int32_t* first = lead < T ? g.table + (int64_t)(seq != nullptr ? seq[lead] : lead) * g.max_pages : nullptr;
    for (int t = 0; t < T; ++t) {
      if (pos[t] < 0) continue;
      const int32_t* row = g.table + (int64_t)(seq != nullptr ? seq[t] : t) * g.max_pages;
      const int np = pos[t] / g.page + 1;
      for (int i = threadIdx.x; i < np; i += 1024) {
        const int id = row[i];
        if (id < 0 || id >= g.n_pages || (first != nullptr && pos[t] + 1 >= P && i < shared && id != first[i])) fail = 1;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) *bad = fail;
}

hipError_t launch_paged_validate(const Pages& g, const int32_t* seq, const int32_t* pos, int T, int max_len,
                                 int shared_pages, int32_t* bad, hipStream_t st) {
  launch_k(k_paged_validate, dim3(1), dim3(1024), 0, st, g, seq, pos, T, max_len, shared_pages, bad);
  return hipGetLastError();
}

}  // namespace dv
