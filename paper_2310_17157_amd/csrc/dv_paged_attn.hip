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

#include <type_traits>

#include "dv_paged.hpp"

namespace dv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kPaNW = 4, kPaNT = 64 * kPaNW;
constexpr float kPaLn2 = 0.693147180559945309f;
constexpr int kPaMaxSlots = 64;      // parts of the shared rows, and of a token's own, at most

// What a token attends: len rows in all, of which its own start at `start` (behind the shared rows, if it
// attends all of those), in `parts` parts of `chunk` rows.
struct Own { int len, start, chunk, parts; };
__device__ __forceinline__ Own own_rows(const PagedAttnArgs& a, int t) {
  Own o;
  o.len = min(max(a.pos[t], -1), a.max_len - 1) + 1;
  o.start = a.P > 0 && o.len >= a.P ? a.P : 0;
  const int n = o.len - o.start;
  o.chunk = max(a.cmin, ((n + a.S - 1) / a.S + 127) & ~127);
  o.parts = (n + o.chunk - 1) / o.chunk;
  return o;
}

template <typename KT, int DH, int QT>
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
  static constexpr int WAVES = DH == 64 ? (QT == 0 ? 4 : QT == 2 ? 3 : 2) : DH == 128 ? (QT == 0 ? 3 : QT == 2 ? 2 : 1) : 1;
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

template <typename KT, int DH, int QT>
__global__ void __launch_bounds__(kPaNT, (PaShape<KT, DH, QT>::WAVES)) k_paged_attn(PagedAttnArgs a) {
  using Sh = PaShape<KT, DH, QT>;
  constexpr bool F16 = Sh::F16, SPLIT = Sh::SPLIT;
  constexpr int NT = Sh::NT, RT = Sh::RT, SK = Sh::SK, KS = Sh::KS, CH = Sh::CH, M = Sh::M, DHP = Sh::DHP;
  constexpr int NK = F16 ? 8 : 4;                      // cache rows of a lane in the value product
  constexpr int EB = sizeof(KT);
  __shared__ int rows[RT];
  __shared__ int red[kPaNW + 1];
  __shared__ int64_t offs[kPaNW][2][SK];
  extern __shared__ float smem[];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int col = lane & 15, grp = lane >> 4;

  // ---- the unit: query rows (rows[0..nr): index t n + j, or -1), key head, cache rows [k0, k1), table row, slot
  int h, tile, k0, k1, slot, c0 = 0, c1 = 0;           // [c0, c1): candidates of head sets to look through
  bool shared = (int)blockIdx.x < a.n_shared;
  if (shared) {
    // the row tiles of a part 8 workgroups apart: on one XCD, whose L2 then holds the part's keys and values
    const int b = blockIdx.x, x = b & 7, y = b >> 3;
    const int u = (y / a.row_tiles) * 8 + x;
    tile = y % a.row_tiles;
    if (u >= a.g.H * a.SP) return;
    h = u / a.SP;
    slot = u - h * a.SP;
    k0 = slot * a.CP;
    k1 = min(k0 + a.CP, a.P);
    if (a.heads != nullptr) c1 = a.T * a.n;
    if (a.heads == nullptr && tid < RT) {
      const int c = tile * RT + tid;
      int idx = -1;
      if (c < a.T * a.G) {
        const int t = c / a.G;
        if (min(a.pos[t], a.max_len - 1) + 1 >= a.P) idx = t * a.n + h * a.G + (c - t * a.G);
      }
      rows[tid] = idx;
    }
  } else {
    int w = (int)blockIdx.x - a.n_shared;
    const int s = w % a.S;
    w /= a.S;
    tile = w % a.group_tiles;
    w /= a.group_tiles;
    const bool single = a.heads != nullptr && a.G == 1;   // one row: the unit is (token, place in its set)
    const int t = w / (single ? a.n : a.g.H), x = w - t * (single ? a.n : a.g.H);
    const Own o = own_rows(a, t);
    slot = a.SP + s;
    h = x;
    if (single) {
      h = min(max(a.heads[(int64_t)t * a.n + x], 0), a.g.H - 1);
      if (tid < RT) rows[tid] = tid == 0 ? t * a.n + x : -1;
    } else if (a.heads == nullptr) {
      if (tid < RT) rows[tid] = tile * RT + tid < a.G ? t * a.n + h * a.G + tile * RT + tid : -1;
    } else {
      c0 = t * a.n;
      c1 = c0 + a.n;
    }
    k0 = o.start + s * o.chunk;
    k1 = min(k0 + o.chunk, o.len);
    // a part that the token does not have; a token without rows is still to be written by its only part
    if (k0 >= k1 && (a.slots > 1 || a.P > 0)) return;
  }
  if (c1 > c0) {
    // this tile's RT of the candidates whose query head belongs to key head h (and, for the shared rows, whose
    // token attends all of them), in order
    if (tid < RT) rows[tid] = -1;
    int seen = 0;
    for (int b = c0; b < c1 && seen < (tile + 1) * RT; b += kPaNT) {
      const int c = b + tid;
      bool mine = c < c1 && min(max(a.heads[c], 0), a.g.H * a.G - 1) / a.G == h;
      if (shared && mine) mine = min(a.pos[c / a.n], a.max_len - 1) + 1 >= a.P;
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
    first = rows[__builtin_ctzll(on)];
  }
  const int t_first = first / a.n;
  const int sq = min(max(a.seq != nullptr ? a.seq[t_first] : t_first, 0), a.g.n_seq - 1);
  const int32_t* trow = a.g.table + (int64_t)sq * a.g.max_pages;
  const char* Kh = a.g.K + h * a.g.hs;
  const char* Vh = a.g.V + h * a.g.hs;
  const int rowb = a.g.dh * EB;

  // ---- steps of this wavefront: cache rows key_of(i) .. + SK
  auto key_of = [&](int i) { return k0 + (i * kPaNW + wave) * SK; };
  const int left = k1 - key_of(0);
  const int nsteps = left > 0 ? (left + kPaNW * SK - 1) / (kPaNW * SK) : 0;
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
        const char* pp = p + min(ks * 64 + grp * 16, rowb - 16);
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
        const VT* pp = reinterpret_cast<const VT*>(p + min((m * 16 + col) * (int)sizeof(VT), rowb - (int)sizeof(VT)));
        vr[i][m] = QT == 0 ? __builtin_nontemporal_load(pp) : *pp;
      }
    }
  };
  int id1 = 0;
  if (nsteps > 0) {
    place(0, page_load(0), 0);
    if (nsteps > 1) id1 = page_load(1);
    load_k(0);
    load_v(0);
  }

  // ---- queries: scaled halves (fp16) or as they are, and the factor >= 0 from products to base-2 logits (a negative
  // scale's sign goes to the queries)
  const float sign = a.scale < 0.f ? -1.f : 1.f;
  u32x4 qh[NT][KS], ql[NT][SPLIT || !F16 ? 1 : KS];
  float cf[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = SPLIT ? col & 7 : nt * 16 + col;
    const int idx = rows[r];
    const float* qp = a.q + (int64_t)max(idx, 0) * a.g.dh;
    constexpr int Q4 = F16 ? 2 : 1;                    // float4 of a piece
    f32x4 x[KS][Q4];
    float mx = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < Q4; ++i) {
        const int d = ks * 16 * Q4 + grp * 4 * Q4 + i * 4;
        const bool on = idx >= 0 && d < a.g.dh;
        const f32x4 v = *reinterpret_cast<const f32x4*>(qp + min(d, a.g.dh - 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[ks][i][e] = on ? v[e] : 0.f;
          mx = fmaxf(mx, fabsf(x[ks][i][e]));
        }
      }
    if constexpr (F16) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
      mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
      const int ex = 14 - ((int)((__float_as_uint(mx) >> 23) & 255u) - 127);   // largest element to [2^14, 2^15)
      cf[nt] = ldexpf(fabsf(a.scale), -ex);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        f16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = ldexpf(sign * x[ks][e >> 2][e & 3], ex);
          hi[e] = (_Float16)v;
          lo[e] = (_Float16)(v - (float)hi[e]);
        }
        if constexpr (SPLIT) {
          qh[nt][ks] = col < 8 ? __builtin_bit_cast(u32x4, hi) : __builtin_bit_cast(u32x4, lo);
        } else {
          qh[nt][ks] = __builtin_bit_cast(u32x4, hi);
          ql[nt][ks] = __builtin_bit_cast(u32x4, lo);
        }
      }
    } else {
      cf[nt] = fabsf(a.scale);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qh[nt][ks] = __builtin_bit_cast(u32x4, x[ks][0] * sign);
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
  for (int i = 0; i < nsteps; ++i) {
    const int base = key_of(i);
    const bool tail = base + SK > k1;
    f32x4 s[NT][SK / 16];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (nt > 0 && nt * 16 >= nr) break;
#pragma unroll
      for (int u = 0; u < SK / 16; ++u) {
        s[nt][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          if constexpr (F16) {
            s[nt][u] = pa_mfma(kr[u][ks], qh[nt][ks], s[nt][u]);
            if constexpr (!SPLIT) s[nt][u] = pa_mfma(kr[u][ks], ql[nt][ks], s[nt][u]);
          } else {
            s[nt][u] = pa_mfma4(__builtin_bit_cast(f32x4, kr[u][ks]), __builtin_bit_cast(f32x4, qh[nt][ks]), s[nt][u]);
          }
        }
      }
    }
    // the next step's keys take the registers of this one's; its values follow behind the value products
    if (i + 1 < nsteps) {
      place(i + 1, id1, (i + 1) & 1);
      if (i + 2 < nsteps) id1 = page_load(i + 2);
      load_k((i + 1) & 1);
    }
    u32x4 ph[NT], pl[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (nt > 0 && nt * 16 >= nr) break;
      if constexpr (SPLIT) {
#pragma unroll
        for (int u = 0; u < SK / 16; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[nt][u][e] += pa_xor8(s[nt][u][e]);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < SK / 16; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!tail || base + u * 16 + grp * 4 + e < k1) mx = fmaxf(mx, s[nt][u][e]);
      mx = pa_max_groups(mx) * cf[nt];
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
          float p = __builtin_amdgcn_exp2f(fmaf(s[nt][u][e], cf[nt], -mu));
          if (tail) p = base + u * 16 + grp * 4 + e < k1 ? p : 0.f;
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
          const f16x2 r = {(_Float16)fmaf((float)h[0], -1.f, p0), (_Float16)fmaf((float)h[1], -1.f, p1)};
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
    if (tail) {                                        // values behind the last row may be anything
#pragma unroll
      for (int k = 0; k < NK; ++k)
        if (base + (k >> 2) * 16 + grp * 4 + (k & 3) >= k1)
#pragma unroll
          for (int mm = 0; mm < M; ++mm) vr[k][mm] = VT{};
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
            if (nt > 0 && nt * 16 >= nr) break;
            o[nt][mm * CH + e] = pa_mfma(v, ph[nt], o[nt][mm * CH + e]);
            if constexpr (!SPLIT) o[nt][mm * CH + e] = pa_mfma(v, pl[nt], o[nt][mm * CH + e]);
          }
        } else {
          f32x4 v;
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(vr[k][mm][e]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0 && nt * 16 >= nr) break;
            o[nt][mm * CH + e] = pa_mfma4(v, __builtin_bit_cast(f32x4, ph[nt]), o[nt][mm * CH + e]);
          }
        }
      }
    if (i + 1 < nsteps) load_v((i + 1) & 1);
  }

  // ---- join the wavefronts: every one writes its sums (zeros where it had no step), then all threads add
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
  const bool direct = a.slots == 1 && a.P == 0;
  const int d4 = a.g.dh / 4;
  for (int x = tid; x < nr * d4; x += kPaNT) {
    const int r = x / d4, d = (x - r * d4) * 4;
    const int idx = rows[r];
    if (idx < 0) continue;
    float mw[kPaNW], mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int w = 0; w < kPaNW; ++w) {
      mw[w] = sm_m[w * RT + r];
      mt = fmaxf(mt, mw[w]);
    }
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kPaNW; ++w) {
      const float f = mw[w] == -INFINITY ? (mt == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(mw[w] - mt);
      lt = fmaf(sm_l[w * RT + r], f, lt);
      const f32x4 v = *reinterpret_cast<const f32x4*>(sm_o + (w * RT + r) * DHP + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(v[e], f, acc[e]);
    }
    const float me = mt - (F16 ? 14.f : 0.f);          // the sums' own factor
    if (direct) {
      const float rl = lt == 0.f ? 0.f : 1.f / lt;
      float* out = a.out + (int64_t)idx * a.ldo;
      if (a.ldo != a.g.dh) {                            // partials' form, for the out-projection
        if (d == 0) {
          out[0] = 0.f;
          out[1] = 1.f;
        }
        out += 2;
        for (int e = 0; e < 4; ++e) out[d + e] = acc[e] * rl;
      } else {
        *reinterpret_cast<f32x4*>(out + d) = acc * rl;
      }
      if (d == 0 && a.lse != nullptr)
        a.lse[idx] = lt == 0.f ? -INFINITY : (me + __builtin_amdgcn_logf(lt)) * kPaLn2;
    } else {
      const int64_t ps = (int64_t)idx * a.slots + slot;
      *reinterpret_cast<f32x4*>(a.o + ps * a.g.dh + d) = acc;
      if (d == 0) {
        a.ml[ps * 2] = me;
        a.ml[ps * 2 + 1] = lt;
      }
    }
  }
}

// Rows' partials joined: a wavefront per row; the slots' weights in lanes, then their value sums, two slots at a
// time (half a wavefront each) where a row is at most 32 chunks of four.
__global__ void __launch_bounds__(kPaNT) k_paged_combine(PagedAttnArgs a) {
  const int idx = (int)blockIdx.x * kPaNW + (int)(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (idx >= a.T * a.n) return;
  const Own own = own_rows(a, idx / a.n);
  const int b = own.start > 0 ? 0 : a.SP, e = a.SP + own.parts, ns = e - b;
  const int64_t base = (int64_t)idx * a.slots + b;
  float w[2], m[2], l[2];
  float mt = -INFINITY;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = lane + 64 * i;
    m[i] = s < ns ? a.ml[(base + s) * 2] : -INFINITY;
    l[i] = s < ns ? a.ml[(base + s) * 2 + 1] : 0.f;
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
      v[i] = *reinterpret_cast<const f32x4*>(a.o + (base + sc) * a.g.dh + min(d, a.g.dh - 4));
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
// Query rows of a workgroup: the smallest tile that holds a unit's rows (kernel variant QT), the largest otherwise.
static int pa_variant(int ktype, int dh, int most) {
  const bool f16 = ktype == DV_F16;
  if (most <= (f16 ? 8 : 16)) return 0;
  return 2;
}
static int pa_rows(int ktype, int qt) { return qt == 0 ? (ktype == DV_F16 ? 8 : 16) : 16 * qt; }

static int pa_most(const PagedAttnArgs& a) {           // query rows of the largest unit
  const int own = a.heads != nullptr ? min(a.G, a.n) : a.G;
  return a.P > 0 ? a.T * own : own;
}

void plan_paged_attn(PagedAttnArgs* a, int ktype) {
  const int rt = pa_rows(ktype, pa_variant(ktype, a->g.dh, pa_most(*a)));
  const int group = a->heads != nullptr ? min(a->G, a->n) : a->G;
  a->row_tiles = a->P > 0 ? max(1, (a->T * group + rt - 1) / rt) : 0;
  a->group_tiles = max(1, (group + rt - 1) / rt);
  const bool single = a->heads != nullptr && a->G == 1;
  const int64_t units = (int64_t)a->T * (single ? a->n : a->g.H) * a->group_tiles;
  const int64_t own = a->max_len - a->P;
  // Rows of a workgroup: the whole work over about four workgroups a CU, at least 256 rows (two steps of each
  // wavefront), so that the parts' sums stay small beside the cache rows.
  const int64_t total = units * own + (int64_t)a->g.H * a->row_tiles * a->P;
  const int64_t wgs = 4LL * device_cu_count();
  const int64_t chunk = max((int64_t)256, (total + wgs - 1) / wgs);
  auto parts = [&](int64_t n) { return (int)min((int64_t)kPaMaxSlots, max((int64_t)1, (n + chunk - 1) / chunk)); };
  a->S = parts(own);
  a->cmin = 128;
  a->SP = 0;
  a->CP = 1;
  if (a->P > 0) {
    a->CP = ((a->P + parts(a->P) - 1) / parts(a->P) + 127) / 128 * 128;
    a->SP = (a->P + a->CP - 1) / a->CP;
  }
  a->slots = a->SP + a->S;
  a->n_shared = a->P > 0 ? (a->g.H * a->SP + 7) / 8 * 8 * a->row_tiles : 0;
}

template <typename KT, int DH, int QT>
static hipError_t launch_pa(const PagedAttnArgs& a, hipStream_t st) {
  const size_t lds = PaShape<KT, DH, QT>::lds();
  const hipError_t e = ensure_dyn_lds(reinterpret_cast<const void*>(k_paged_attn<KT, DH, QT>), lds);
  if (e != hipSuccess) return e;
  const bool single = a.heads != nullptr && a.G == 1;
  const int64_t own = (int64_t)a.T * (single ? a.n : a.g.H) * a.group_tiles * a.S;
  launch_k((k_paged_attn<KT, DH, QT>), dim3((unsigned)(a.n_shared + own)), dim3(kPaNT), lds, st, a);
  return hipGetLastError();
}

template <typename KT>
static hipError_t launch_pa_k(int ktype, const PagedAttnArgs& a, hipStream_t st) {
  const int qt = pa_variant(ktype, a.g.dh, pa_most(a));
  if (a.g.dh <= 64) return qt == 0 ? launch_pa<KT, 64, 0>(a, st) : qt == 2 ? launch_pa<KT, 64, 2>(a, st) : launch_pa<KT, 64, 4>(a, st);
  if (a.g.dh <= 128)
    return qt == 0 ? launch_pa<KT, 128, 0>(a, st) : qt == 2 ? launch_pa<KT, 128, 2>(a, st) : launch_pa<KT, 128, 4>(a, st);
  return qt == 0 ? launch_pa<KT, 256, 0>(a, st) : launch_pa<KT, 256, 2>(a, st);
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
