// Rotary positions, and the append to a cache in pages with the rotation on the way.
//
//   (x0, x1) -> m (x0 cos a - x1 sin a, x0 sin a + x1 cos a),  a = p f_i   for pair i of a head at position p.
//
// One kernel serves both entry points: a token's queries are rotated from q to q_out, its keys are
// rotated and its values copied into their rows of the cache. Everything is read once and written once, so memory bounds it;
// the angles depend on (token, pair) alone and are computed once for all heads of a token that a workgroup
// takes: in 64 bits to turns, reduced to one turn, then sine and cosine in fp32 (an angle in
// fp32 is off by 0.03 rad at position 10^6). The work of a token is a list of units of 16 bytes of the input type (a pair of chunks
// where a chunk's partners lie rot/2 further), its queries', then its keys', then its values'; a
// workgroup takes whole tokens while they are many, a part of one token's list while they are few,
// and every thread has kRopeU units' loads in flight before it stores.
#include <math.h>

#include "dv_paged.hpp"

namespace dv {

constexpr int kRopeNT = 256, kRopeU = 4;
constexpr int kRopePairs = 1024;          // (cos, sin) pairs in LDS

// E elements as fp32, by the widest loads that E elements allow.
template <typename T, int E>
__device__ __forceinline__ void ld_vec(const T* p, float* f) {
  if constexpr (E == 1) {
    f[0] = (float)p[0];
  } else {
    typedef T V __attribute__((ext_vector_type(E)));
    const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = (float)v[e];
  }
}
template <typename T, int E>
__device__ __forceinline__ void st_vec(T* p, const float* f) {
  if constexpr (E == 1) {
    p[0] = (T)f[0];
  } else {
    constexpr int W = E * (int)sizeof(T) > 16 ? 16 / (int)sizeof(T) : E;
    typedef T V __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int c = 0; c < E; c += W) {
      V v;
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] = (T)f[c + e];
      *reinterpret_cast<V*>(p + c) = v;
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

template <typename IT, typename KT, int E, bool HALF>
__global__ void __launch_bounds__(kRopeNT) k_rope(RopeArgs a) {
  __shared__ float2 cs[kRopePairs];
  const int tid = threadIdx.x;
  const int t0 = (int)blockIdx.x * a.tpw, nt = min(a.tpw, a.T - t0);
  const int half = a.rot / 2;
  for (int i = tid; i < nt * half; i += kRopeNT) {
    const int t = i / half, k = i - t * half;
    double turns = (double)a.pos[t0 + t] * a.freq[k] * 0.15915494309189533577;   // 1 / 2 pi
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    cs[i] = float2{c * a.mscale, (a.inverse ? -s : s) * a.mscale};
  }
  __syncthreads();
  const int nq = a.nq * a.uq, nk = a.nk * a.uq, per = nq + nk + (a.append ? a.nk * a.uv : 0);
  const int total = nt * per;
  const int lo = (int)((int64_t)blockIdx.y * total / a.parts), hi = (int)((int64_t)(blockIdx.y + 1) * total / a.parts);
  for (int base = lo; base < hi; base += kRopeNT * kRopeU) {
    float x[kRopeU][2 * E];
    char* dst[kRopeU];
    int run[kRopeU];                       // bit 0: to pages, bit 2: rotated
    int pa[kRopeU], pb[kRopeU], tt[kRopeU];   // runs of the unit, its token
#pragma unroll
    for (int j = 0; j < kRopeU; ++j) {
      const int i = base + j * kRopeNT + tid;
      dst[j] = nullptr;
      if (i >= hi) continue;
      const int t = i / per;
      int r = i - t * per;
      tt[j] = t;
      const int tok = t0 + t;
      const int p = a.append ? a.pos[tok] : 0;
      if (p < 0) continue;
      const IT* src;
      if (r < nq) {
        const int h = r / a.uq;
        unit_place<E, HALF>(r - h * a.uq, a.rot, &pa[j], &pb[j]);
        src = static_cast<const IT*>(a.q) + tok * a.ldq + h * a.dh;
        dst[j] = reinterpret_cast<char*>(static_cast<IT*>(a.qo) + tok * a.ldqo + h * a.dh);
        run[j] = 4;
      } else {
        const bool isv = r >= nq + nk;
        const int uh = isv ? a.uv : a.uq;
        r -= isv ? nq + nk : nq;
        int h = r / uh;
        const int u = r - h * uh;
        if (isv) {
          pa[j] = u * E;
          pb[j] = -1;
        } else {
          unit_place<E, HALF>(u, a.rot, &pa[j], &pb[j]);
        }
        if (a.heads != nullptr) h = a.heads[(int64_t)tok * a.nk + h];
        const int s = a.seq != nullptr ? a.seq[tok] : tok;
        int row;
        const int pg = page_of(a.g, p, &row);
        if (h < 0 || h >= a.g.H || s < 0 || s >= a.g.n_seq || pg >= a.g.max_pages) continue;
        const int id = a.g.table[(int64_t)s * a.g.max_pages + pg];
        if (id < 0 || id >= a.g.n_pages) continue;
        src = static_cast<const IT*>(isv ? a.v : a.k) + tok * (isv ? a.ldv : a.ldk) + h * a.dh;
        dst[j] = (isv ? a.g.V : a.g.K) + id * a.g.ps + h * a.g.hs + row * a.g.rs;
        run[j] = isv ? 1 : 5;
      }
      ld_vec<IT, E>(src + pa[j], x[j]);
      if (pb[j] >= 0) ld_vec<IT, E>(src + pb[j], x[j] + E);
    }
#pragma unroll
    for (int j = 0; j < kRopeU; ++j) {
      if (dst[j] == nullptr) continue;
      const float2* c = cs + tt[j] * half;
      if (pb[j] >= 0) {                    // two runs: partners
        const int i0 = HALF ? pa[j] : pa[j] >> 1;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 w = c[i0 + e];
          const float x0 = x[j][e], x1 = x[j][E + e];
          x[j][e] = x0 * w.x - x1 * w.y;
          x[j][E + e] = x0 * w.y + x1 * w.x;
        }
      } else if (!HALF && E > 1 && (run[j] & 4) && pa[j] < a.rot) {   // adjacent pairs of one run
#pragma unroll
        for (int e = 0; e + 1 < E; e += 2) {
          const float2 w = c[(pa[j] + e) >> 1];
          const float x0 = x[j][e], x1 = x[j][e + 1];
          x[j][e] = x0 * w.x - x1 * w.y;
          x[j][e + 1] = x0 * w.y + x1 * w.x;
        }
      }
      if (run[j] & 1) {
        st_vec<KT, E>(reinterpret_cast<KT*>(dst[j]) + pa[j], x[j]);
        if (pb[j] >= 0) st_vec<KT, E>(reinterpret_cast<KT*>(dst[j]) + pb[j], x[j] + E);
      } else {
        st_vec<IT, E>(reinterpret_cast<IT*>(dst[j]) + pa[j], x[j]);
        if (pb[j] >= 0) st_vec<IT, E>(reinterpret_cast<IT*>(dst[j]) + pb[j], x[j] + E);
      }
    }
  }
}

template <typename IT, typename KT, int E, bool HALF>
static hipError_t launch_rope_t(RopeArgs a, hipStream_t st) {
  a.uq = HALF || E == 1 ? a.rot / 2 / E + (a.dh - a.rot) / E : a.dh / E;
  a.uv = a.dh / E;
  const int per = a.nq * a.uq + (a.append ? a.nk * (a.uq + a.uv) : 0);
  if (per == 0 || a.T == 0) return hipSuccess;
  // A workgroup's work: about kRopeU units a thread, of several tokens where one has fewer (as many as their
  // angles fit in LDS); parts of one token where the tokens do not fill the CUs.
  const int want = kRopeNT * kRopeU, cus = device_cu_count();
  a.tpw = max(1, want / per);
  if (a.rot > 0) a.tpw = min(a.tpw, kRopePairs / (a.rot / 2));
  a.tpw = max(1, min(a.tpw, (a.T + cus - 1) / cus));
  const int groups = (a.T + a.tpw - 1) / a.tpw;
  a.parts = 1;
  while (groups * a.parts < 2 * cus && a.tpw * per > a.parts * kRopeNT) a.parts *= 2;
  launch_k((k_rope<IT, KT, E, HALF>), dim3(groups, a.parts), dim3(kRopeNT), 0, st, a);
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
