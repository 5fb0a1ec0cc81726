// Rotary positions, and the append to a cache in pages with the rotation on the way.
//
//   (x0, x1) -> m (x0 cos a - x1 sin a, x0 sin a + x1 cos a),  a = p f_i   for pair i of a head at position p.
//
// One kernel serves both entry points: a token's queries are rotated from q to q_out, its keys are
// rotated and its values copied into their rows of the cache. Everything is read once and written once, so memory bounds it.
// The angles depend on (token, pair) alone and are computed once for all heads of a token that a workgroup
// takes: in 64 bits to turns, reduced to one turn, then sine and cosine in fp32 (an angle in
// fp32 is off by 0.03 rad at position 10^6). The work of a token is a list of units of 16 bytes of the input type (a pair of chunks
// where a chunk's partners lie rot/2 further), its queries', then its keys', then its values'. A workgroup takes whole
// tokens while they are short, a part of one token's list while it is long, at most kRopeU units a thread: their loads
// are in flight before the angles and the pages are looked up.
//
// Measured: 9600 tokens of 64 query and 8 key/value heads of 128 fp16, prompts of 100 to 1500, appended in 86 us:
// 393 MB at 4.57 TB/s, where a copy reaches 4.9. (With 2 units a thread 103 us, with 8, at half the waves,
// 129; with the loads behind the angles and a second round of them 117.) 32 tokens of a decode step 4.2 to 5.5 us, a launch.
#include <math.h>

#include "dv_paged.hpp"

namespace dv {

constexpr int kRopeNT = 256, kRopeU = 4;
constexpr int kRopePairs = 1024, kRopeTokens = 512;   // (cos, sin) pairs and tokens of a workgroup at most
constexpr int kRopeGridX = 65536;
// Results beyond what the L2s of the 8 XCDs hold together are stored past them: whoever reads them next
// finds them in memory anyhow. The prompts above 86 us against 92 through L2, 6000 tokens of 32 heads of 128 fp16 17
// against 22.5; results that fit stay where the next kernel reads them (the store itself takes as long either way).
constexpr double kL2Bytes = 32 << 20;

// E elements, moved as one.
template <typename T, int E>
struct alignas(E * sizeof(T)) Run {
  T e[E];
};
template <bool PAST, typename T, int E>
__device__ __forceinline__ void st_run(T* p, const float* f) {
  constexpr int W = E * (int)sizeof(T) > 16 ? 16 / (int)sizeof(T) : E;
#pragma unroll
  for (int c = 0; c < E; c += W) {
    Run<T, W> v;
#pragma unroll
    for (int e = 0; e < W; ++e) v.e[e] = (T)f[c + e];
    if constexpr (PAST) {
      typedef uint32_t Words __attribute__((ext_vector_type(W * sizeof(T) / 4)));
      __builtin_nontemporal_store(__builtin_bit_cast(Words, v), reinterpret_cast<Words*>(p + c));
    } else {
      *reinterpret_cast<Run<T, W>*>(p + c) = v;
    }
  }
}

// Unit u of a rotated head, as one or two runs of E elements (b < 0: one). Pairs across halves: the first rot/2/E
// units hold a run and its partners', the rest a run that stays. Adjacent pairs: runs in order;
// for E == 1 a pair is two runs of one element.
template <int E, bool HALF>
__device__ __forceinline__ void unit_place(int u, int rot, int* a, int* b) {
  if constexpr (HALF || E == 1) {
    const int np = rot / 2 / E;
    if (u < np) {
      *a = HALF ? u * E : 2 * u;
      *b = HALF ? rot / 2 + u * E : 2 * u + 1;
    } else {
      *a = rot + (u - np) * E;
      *b = -1;
    }
  } else {
    *a = u * E;
    *b = -1;
  }
}

__device__ __forceinline__ int div_by(const Divisor& d, int i) { return (int)(__umulhi((uint32_t)i << 1, d.m) >> d.s); }

template <typename IT, typename KT, int E, bool HALF, bool PAST>
__global__ void __launch_bounds__(kRopeNT) k_rope(RopeArgs a) {
  __shared__ float2 cs[kRopePairs];
  __shared__ int64_t place[kRopeTokens];   // a token's row in its page, in bytes; -1: none; -2: the token is left out
  const int tid = threadIdx.x;
  const int block = (int)(blockIdx.y * kRopeGridX + blockIdx.x), group = div_by(a.by_parts, block);
  const int64_t t0 = (int64_t)group * a.tpw;
  const int part = block - group * a.parts, nt = (int)min((int64_t)a.tpw, a.T - t0);
  if (nt <= 0) return;
  const int half = a.rot / 2, pairs = nt * half;
  auto pair_of = [&](int i, int* t) {
    *t = half == 0 ? 0 : i / half;
    return i - *t * half;
  };
  int at = 0;
  double f0 = 0;
  int p0 = 0;
  const int k0 = pair_of(min(tid, max(pairs - 1, 0)), &at);
  if (pairs > 0) {
    f0 = a.freq[k0];
    p0 = a.pos[t0 + at];
  }

  const int nq = a.nq * a.uq, nk = a.nk * a.uq;
  const int64_t total = (int64_t)nt * a.per;
  const int lo = (int)(part * total / a.parts), hi = (int)((part + 1) * total / a.parts);
  Run<IT, E> x[kRopeU][2];
  int tt[kRopeU], hd[kRopeU], pa[kRopeU], pb[kRopeU];   // token, cache head (of a query: its offset), runs of the unit
  int kind[kRopeU];                        // 0: none, 1: query, 2: key, 3: value
#pragma unroll
  for (int j = 0; j < kRopeU; ++j) {
    const int i = lo + j * kRopeNT + tid;
    kind[j] = 0;
    if (i >= hi) continue;
    const int t = div_by(a.by_per, i);
    const int64_t tok = t0 + t;
    int r = i - t * a.per;
    tt[j] = t;
    const IT* src;
    if (r < nq) {
      const int h = div_by(a.by_uq, r);
      unit_place<E, HALF>(r - h * a.uq, a.rot, &pa[j], &pb[j]);
      hd[j] = h * a.dh;
      src = static_cast<const IT*>(a.q) + tok * a.ldq + hd[j];
      kind[j] = 1;
    } else {
      const bool isv = r >= nq + nk;
      r -= isv ? nq + nk : nq;
      int h = div_by(isv ? a.by_uv : a.by_uq, r);
      const int u = r - h * (isv ? a.uv : a.uq);
      if (isv) {
        pa[j] = u * E;
        pb[j] = -1;
      } else {
        unit_place<E, HALF>(u, a.rot, &pa[j], &pb[j]);
      }
      if (a.heads != nullptr) {
        h = a.heads[tok * a.nk + h];
        if (h < 0 || h >= a.g.H) continue;
      }
      hd[j] = h;
      src = static_cast<const IT*>(isv ? a.v : a.k) + tok * (isv ? a.ldv : a.ldk) + h * a.dh;
      kind[j] = isv ? 3 : 2;
    }
    x[j][0] = *reinterpret_cast<const Run<IT, E>*>(src + pa[j]);
    if (pb[j] >= 0) x[j][1] = *reinterpret_cast<const Run<IT, E>*>(src + pb[j]);
  }

  if (a.append) {
    for (int t = tid; t < nt; t += kRopeNT) {
      const int p = a.pos[t0 + t], s = a.seq != nullptr ? a.seq[t0 + t] : (int)(t0 + t);
      int64_t at_row = p < 0 ? -2 : -1;
      if (p >= 0 && s >= 0 && s < a.g.n_seq) {
        int row;
        const int pg = page_of(a.g, p, &row);
        if (pg < a.g.max_pages) {
          const int id = a.g.table[(int64_t)s * a.g.max_pages + pg];
          if (id >= 0 && id < a.g.n_pages) at_row = id * a.g.ps + row * a.g.rs;
        }
      }
      place[t] = at_row;
    }
  }
  for (int i = tid; i < pairs; i += kRopeNT) {
    if (i != tid) {
      const int k = pair_of(i, &at);
      f0 = a.freq[k];
      p0 = a.pos[t0 + at];
    }
    double turns = (double)p0 * f0 * 0.15915494309189533577;   // 1 / 2 pi
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    cs[i] = float2{c * a.mscale, (a.inverse ? -s : s) * a.mscale};
  }
  __syncthreads();

#pragma unroll
  for (int j = 0; j < kRopeU; ++j) {
    if (kind[j] == 0) continue;
    const int64_t row = a.append ? place[tt[j]] : 0;
    if (row == -2 || (row < 0 && kind[j] != 1)) continue;
    float y[2 * E];
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = (float)x[j][0].e[e];
    if (pb[j] >= 0) {                      // two runs: partners
#pragma unroll
      for (int e = 0; e < E; ++e) y[E + e] = (float)x[j][1].e[e];
      const float2* c = cs + tt[j] * half + (HALF ? pa[j] : pa[j] >> 1);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 w = c[e];
        const float x0 = y[e], x1 = y[E + e];
        y[e] = x0 * w.x - x1 * w.y;
        y[E + e] = x0 * w.y + x1 * w.x;
      }
    } else if (!HALF && E > 1 && kind[j] != 3 && pa[j] < a.rot) {   // adjacent pairs of one run
      const float2* c = cs + tt[j] * half + (pa[j] >> 1);
#pragma unroll
      for (int e = 0; e + 1 < E; e += 2) {
        const float2 w = c[e >> 1];
        const float x0 = y[e], x1 = y[e + 1];
        y[e] = x0 * w.x - x1 * w.y;
        y[e + 1] = x0 * w.y + x1 * w.x;
      }
    }
    if (kind[j] == 1) {
      IT* dst = static_cast<IT*>(a.qo) + (t0 + tt[j]) * a.ldqo + hd[j];
      st_run<PAST, IT, E>(dst + pa[j], y);
      if (pb[j] >= 0) st_run<PAST, IT, E>(dst + pb[j], y + E);
    } else {
      KT* dst = reinterpret_cast<KT*>((kind[j] == 3 ? a.g.V : a.g.K) + row + hd[j] * a.g.hs);
      st_run<PAST, KT, E>(dst + pa[j], y);
      if (pb[j] >= 0) st_run<PAST, KT, E>(dst + pb[j], y + E);
    }
  }
}

// i / d for 0 <= i < 2^31 as (2 i m >> 32) >> s: m = ceil(2^(31+s) / d) with 2^(s-1) < d <= 2^s is at most d - 1 parts of
// 2^(31+s) too large, which i < 2^31 cannot lift to the next quotient.
static Divisor divisor(int d) {
  Divisor v{0, 0};
  if (d < 1) return v;
  while (((int64_t)1 << v.s) < d) ++v.s;
  v.m = (uint32_t)((((uint64_t)1 << (31 + v.s)) + d - 1) / d);
  return v;
}

template <typename IT, typename KT, int E, bool HALF>
static hipError_t launch_rope_t(RopeArgs a, hipStream_t st) {
  a.uq = HALF || E == 1 ? a.rot / 2 / E + (a.dh - a.rot) / E : a.dh / E;
  a.uv = a.dh / E;
  a.per = a.nq * a.uq + (a.append ? a.nk * (a.uq + a.uv) : 0);
  if (a.per == 0 || a.T == 0) return hipSuccess;
  // A workgroup's work: at most kRopeU units a thread, of several tokens where one has fewer (as many as their
  // angles fit in LDS), down to one unit a thread where there are not two workgroups a CU.
  const int most = kRopeNT * kRopeU, cus = device_cu_count();
  a.tpw = min(max(1, most / a.per), kRopeTokens);
  if (a.rot > 0) a.tpw = min(a.tpw, kRopePairs / (a.rot / 2));
  a.tpw = max(1, min(a.tpw, (a.T - 1) / cus + 1));
  const int64_t groups = ((int64_t)a.T + a.tpw - 1) / a.tpw, units = (int64_t)a.tpw * a.per;
  a.parts = (int)((units + most - 1) / most);
  while (groups * a.parts < 2 * cus && units > (int64_t)a.parts * kRopeNT) a.parts *= 2;
  const int64_t blocks = groups * a.parts;
  if (blocks > INT32_MAX / 2) return hipErrorInvalidValue;
  a.by_parts = divisor(a.parts); a.by_per = divisor(a.per); a.by_uq = divisor(a.uq); a.by_uv = divisor(a.uv);
  const int gx = (int)(blocks < kRopeGridX ? blocks : kRopeGridX);
  const dim3 grid(gx, (int)((blocks + gx - 1) / gx));
  if constexpr (E > 1) {
    if ((double)a.T * (a.nq + (a.append ? 2 * a.nk : 0)) * a.dh * sizeof(KT) > kL2Bytes) {
      launch_k((k_rope<IT, KT, E, HALF, true>), grid, dim3(kRopeNT), 0, st, a);
      return hipGetLastError();
    }
  }
  launch_k((k_rope<IT, KT, E, HALF, false>), grid, dim3(kRopeNT), 0, st, a);
  return hipGetLastError();
}

template <typename IT, typename KT>
static hipError_t launch_rope_i(int layout, const RopeArgs& a, hipStream_t st) {
  constexpr int E = Chunk<IT>::E;
  const bool half = layout == DV_ROPE_HALF;
  auto wide = [](const void* p, int64_t ld) { return p == nullptr || (aligned16(p) && ld % E == 0); };
  // 16 bytes at a time where every run of a unit is aligned and lies wholly inside or outside the rotated part;
  // else element by element
  const bool vec = a.dh % E == 0 && (half ? a.rot / 2 : a.rot) % E == 0 && wide(a.q, a.ldq) && wide(a.qo, a.ldqo) &&
                   wide(a.k, a.ldk) && wide(a.v, a.ldv);
  if (vec) return half ? launch_rope_t<IT, KT, E, true>(a, st) : launch_rope_t<IT, KT, E, false>(a, st);
  return half ? launch_rope_t<IT, KT, 1, true>(a, st) : launch_rope_t<IT, KT, 1, false>(a, st);
}

hipError_t launch_rope(int xtype, int ktype, int layout, const RopeArgs& a, hipStream_t st) {
  if (xtype == DV_F16)
    return ktype == DV_F16 ? launch_rope_i<_Float16, _Float16>(layout, a, st) : launch_rope_i<_Float16, float>(layout, a, st);
  return ktype == DV_F16 ? launch_rope_i<float, _Float16>(layout, a, st) : launch_rope_i<float, float>(layout, a, st);
}

}  // namespace dv
