// Rotary positions with several axes on query and key rows, with the per-head
// RMS norm of queries and keys in front where weights are given, forward and
// backward, on gfx950. The packed foreground tokens keep the positions of the
// full multi-view grid (paper Sec. 3.2): a token reads its coordinates through
// its kept index.
//
//   angle a_p = pos[row, axis(p)] theta^(-2 i(p) / d_axis), pair p the i-th of
//   its axis; (u, v) -> (u cos a - v sin a, v cos a + u sin a) on the pair's two
//   elements; elements past the axes' sum pass through.
//   norm      u = x rstd w,  rstd = 1 / sqrt(mean(x^2) + eps) over the head
//   backward  g = the rotation by -a of dy; without the norm dx = g; with it
//             h = x rstd,  dw = sum over rows and heads of g h,
//             dx = rstd (g w - h mean(g w h))
//
// Bytes bound it: a row is read and written once, about 150 vector instructions of
// the built loop (forward with the norm; 163 with the table's share, by the counters)
// stand beside 32 bytes a lane. The angles are shared by all heads: a
// workgroup takes a few tokens, one thread computes one cos and sin (the
// angle in turns and in 64 bits, so that a far position loses nothing), and the
// heads read them from LDS. A group of P2 lanes holds one head, 8 elements (4
// pairs) a lane, so that the norm's sums are exchanges between lanes; all sums
// are fp32 and the result is rounded once.
//
// The weights' gradients: every workgroup adds its rows in registers, then its
// head slots in LDS, and writes one partial row; a second launch adds the
// partial rows in a fixed order (no atomics, equal results on every run).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "common.h"

namespace ut {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTok = 16;    // most tokens of a workgroup's turn
constexpr int kTable = 256;    // cos and sin of a turn: one a thread

struct RopeArgs {
  RopeSide side[2];
  float* part;
  const float* pos;
  const int32_t* idx;
  int64_t n;
  uint32_t pos_rows;
  int32_t D, half, tok, n_axes;
  float eps;
  bool w_bf16;
  double rev[kRopeMaxDim / 2];    // turns per unit of position
  uint8_t axis[kRopeMaxDim / 2];
};

template <typename T>
struct Vec;
template <>
struct Vec<__bf16> {
  typedef __bf16 x4 __attribute__((ext_vector_type(4)));
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
};
template <>
struct Vec<float> {
  typedef float x4 __attribute__((ext_vector_type(4)));
};

// Eight elements of a head: two runs of four, one run of eight where the pairs
// are neighbours.
template <typename T, bool FAR>
struct Chunk {
  typename Vec<T>::x4 a, b;
  __device__ inline void load(const T* p, int o0, int o1) {
    if constexpr (!FAR && sizeof(T) == 2) {
      const typename Vec<T>::x8 v = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T>::x8*>(p + o0));
      a = v.lo;
      b = v.hi;
    } else {
      a = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T>::x4*>(p + o0));
      b = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T>::x4*>(p + o1));
    }
  }
  __device__ inline void get(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)a[e], x[4 + e] = (float)b[e];
  }
  __device__ static inline void store(T* p, int o0, int o1, const float (&x)[8]) {
    typename Vec<T>::x4 u, v;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = (T)x[e], v[e] = (T)x[4 + e];
    if constexpr (!FAR && sizeof(T) == 2) {
      typename Vec<T>::x8 w;
      w.lo = u;
      w.hi = v;
      __builtin_nontemporal_store(w, reinterpret_cast<typename Vec<T>::x8*>(p + o0));
    } else {
      __builtin_nontemporal_store(u, reinterpret_cast<typename Vec<T>::x4*>(p + o0));
      __builtin_nontemporal_store(v, reinterpret_cast<typename Vec<T>::x4*>(p + o1));
    }
  }
};

// The rotation of a chunk's four pairs by cs = (cos, sin) each, backwards with BWD.
template <bool FAR, bool BWD>
__device__ inline void rotate(float (&x)[8], const float2 (&cs)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int i = FAR ? e : 2 * e, j = FAR ? 4 + e : 2 * e + 1;
    const float c = cs[e].x, s = BWD ? -cs[e].y : cs[e].y;
    const float u = x[i], v = x[j];
    x[i] = u * c - v * s;
    x[j] = v * c + u * s;
  }
}

template <int P2>
__device__ inline float lanes_sum(float x) {
#pragma unroll
  for (int m = 1; m < P2; m <<= 1) x += __shfl_xor(x, m, 64);
  return x;
}

template <typename T, int P2, bool FAR, bool NORM, bool BWD>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeArgs a) {
  constexpr int kSlots = kThreads / P2;
  constexpr int U = sizeof(T) == 2 ? 2 : 1;   // rows of 16 or 32 bytes a lane in flight; more cost occupancy
  __shared__ float2 table[kTable];
  const int tid = threadIdx.x, slot = tid / P2, j = tid % P2;
  const int H = a.side[0].H + a.side[1].H, lph = a.D / 8;
  const int hp = (a.half + 3) & ~3;             // table entries of a token
  const bool live = j < lph, turned = 4 * j < a.half;
  const int o0 = FAR && turned ? 4 * j : 8 * j;
  const int o1 = FAR && turned ? a.half + 4 * j : 8 * j + 4;

  float w[2][8], dw[2][8];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[s][e] = dw[s][e] = 0.f;
      if (NORM && live && a.side[s].w) {
        const int i = e < 4 ? o0 + e : o1 + e - 4;
        w[s][e] = a.w_bf16 ? (float)static_cast<const __bf16*>(a.side[s].w)[i]
                           : static_cast<const float*>(a.side[s].w)[i];
      }
    }

  const int dt = kSlots / H, dh = kSlots % H;   // from one item of a slot to its next
  for (int64_t t0 = (int64_t)blockIdx.x * a.tok; t0 < a.n; t0 += (int64_t)gridDim.x * a.tok) {
    const int tn = (int)min((int64_t)a.tok, a.n - t0);
    __syncthreads();                            // the turn before has read its table
    for (int i = tid; i < tn * hp; i += kThreads) {
      const int lt = i / hp, p = i - lt * hp;
      float2 cs = make_float2(1.f, 0.f);
      if (p < a.half) {
        const uint32_t t = (uint32_t)(t0 + lt);
        const int64_t row = a.idx ? (int64_t)a.idx[t] : (int64_t)(t < a.pos_rows ? t : t % a.pos_rows);
        if (row >= 0 && row < (int64_t)a.pos_rows) {   // others are not turned
          double r = (double)a.pos[row * a.n_axes + a.axis[p]] * a.rev[p];
          r -= rint(r);                         // turns in [-1/2, 1/2]
          sincospif(2.f * (float)r, &cs.y, &cs.x);
        }
      }
      table[i] = cs;
    }
    __syncthreads();

    // The turn's first rows, scalar; a row from there is one 64-bit multiply-add.
    const T *x0 = static_cast<const T*>(a.side[0].x) + t0 * a.side[0].sx,
            *x1 = static_cast<const T*>(a.side[1].x) + t0 * a.side[1].sx,
            *dy0 = static_cast<const T*>(a.side[0].dy) + t0 * a.side[0].sdy,
            *dy1 = static_cast<const T*>(a.side[1].dy) + t0 * a.side[1].sdy;
    T *out0 = static_cast<T*>(a.side[0].out) + t0 * a.side[0].so, *out1 = static_cast<T*>(a.side[1].out) + t0 * a.side[1].so;
    const int sx0 = (int)a.side[0].sx, sx1 = (int)a.side[1].sx, sdy0 = (int)a.side[0].sdy, sdy1 = (int)a.side[1].sdy,
              so0 = (int)a.side[0].so, so1 = (int)a.side[1].so;

    const int items = tn * H;
    int lt = slot / H, hh = slot - lt * H;
    for (int it = slot; it < items; it += U * kSlots) {
      Chunk<T, FAR> cx[U], cd[U];
      int at_t[U], at_h[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        at_t[u] = lt, at_h[u] = hh;
        if (live && it + u * kSlots < items) {
          const bool s = hh >= a.side[0].H;
          const int h = (hh - (s ? a.side[0].H : 0)) * a.D;
          if constexpr (BWD) cd[u].load((s ? dy1 : dy0) + (int64_t)lt * (s ? sdy1 : sdy0) + h, o0, o1);
          if constexpr (!BWD || NORM) cx[u].load((s ? x1 : x0) + (int64_t)lt * (s ? sx1 : sx0) + h, o0, o1);
        }
        lt += dt, hh += dh;
        if (hh >= H) hh -= H, ++lt;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (it + u * kSlots >= items) break;    // whole lane groups leave together
        const int s = at_h[u] >= a.side[0].H;
        float2 cs[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) cs[e] = live && turned ? table[at_t[u] * hp + 4 * j + e] : make_float2(1.f, 0.f);
        float x[8], y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = y[e] = 0.f;
        if (live) {
          if constexpr (!BWD || NORM) cx[u].get(x);
          if constexpr (BWD) cd[u].get(y);
        }
        if constexpr (BWD) rotate<FAR, true>(y, cs);
        if constexpr (NORM) {
          float sq = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) sq += x[e] * x[e];
          const float rstd = rsqrtf(lanes_sum<P2>(sq) / (float)a.D + a.eps);
          float ws[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) ws[e] = s ? w[1][e] : w[0][e];
          if constexpr (BWD) {
            float dot = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              x[e] *= rstd;
              const float gh = y[e] * x[e];
              dw[0][e] += s ? 0.f : gh;
              dw[1][e] += s ? gh : 0.f;
              y[e] *= ws[e];
              dot += y[e] * x[e];
            }
            dot = lanes_sum<P2>(dot) / (float)a.D;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = rstd * (y[e] - x[e] * dot);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= rstd * ws[e];
          }
        }
        if constexpr (!BWD) {
          rotate<FAR, false>(x, cs);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = x[e];
        }
        if (live) {
          const int h = (at_h[u] - (s ? a.side[0].H : 0)) * a.D;
          Chunk<T, FAR>::store((s ? out1 : out0) + (int64_t)at_t[u] * (s ? so1 : so0) + h, o0, o1, y);
        }
      }
    }
  }

  if constexpr (BWD && NORM) {
    __shared__ float red[kThreads * 8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) red[e * kThreads + tid] = dw[s][e];
      __syncthreads();
      if (slot < 8 && live)                     // element `slot` of chunk j, in the order of the slots
        for (int e = slot; e < 8; e += kSlots) {
          float sum = 0.f;
          for (int k = 0; k < kSlots; ++k) sum += red[e * kThreads + k * P2 + j];
          const int i = e < 4 ? o0 + e : o1 + e - 4;
          a.part[((int64_t)blockIdx.x * 2 + s) * a.D + i] = sum;
        }
    }
  }
}

// out[s][c] = the sum of `parts` partial rows in a fixed order: 64 threads a
// column, each over every 64th row, then a tree.
__global__ __launch_bounds__(kThreads) void rope_weight_sum_kernel(const float* __restrict__ part, int parts, int D,
                                                                   float* dwq, float* dwk) {
  __shared__ float red[kThreads];
  const int col = blockIdx.x * 4 + (threadIdx.x & 3), r = threadIdx.x >> 2;
  float sum = 0.f;
  if (col < 2 * D)
    for (int i = r; i < parts; i += 64) sum += part[(int64_t)i * 2 * D + col];
  red[threadIdx.x] = sum;
  __syncthreads();
  for (int m = 32; m >= 1; m >>= 1) {
    if (r < m) red[threadIdx.x] += red[threadIdx.x + 4 * m];
    __syncthreads();
  }
  if (r == 0 && col < 2 * D) {
    float* out = col < D ? dwq : dwk;
    if (out) out[col < D ? col : col - D] = red[threadIdx.x];
  }
}

// Persistent workgroups, as many as fit at once (the gradients' partial rows too
// are at most kRopeParts), six a CU at most: the runtime's figure leaves scalar
// registers out, and a grid that does not fit at once ends in a second round. At
// 77,586 x 48 x 128 the forward with the norm takes 385 us with 1,536, 409 with 1,280
// and 462 with 2,048 (four rows in flight, of which 1,280 fit: 404); without the norm
// 363 with 1,536 and 441 with 2,048. A turn holds as many tokens as the table has room
// for, fewer where the last round would be mostly idle; a turn costs about half a
// token's time besides.
template <typename T, int P2, bool FAR, bool NORM, bool BWD>
unsigned launch(RopeArgs& a, hipStream_t s) {
  static const int per_cu = [] {
    int n = 0;
    return hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, rope_kernel<T, P2, FAR, NORM, BWD>, kThreads, 0) ==
                       hipSuccess && n > 0 ? std::min(n, 6) : 4;
  }();
  const int64_t fit = std::min<int64_t>(256 * per_cu, BWD && NORM ? kRopeParts : 1 << 20);
  const int hp = (a.half + 3) & ~3, most = std::max(1, std::min(kMaxTok, kTable / hp));
  int64_t best = 0;
  for (int tok = most; tok >= 1; --tok) {
    const int64_t turns = (a.n + tok - 1) / tok, cost = (turns + fit - 1) / fit * (2 * tok + 1);
    if (best == 0 || cost < best) best = cost, a.tok = tok;
  }
  const unsigned wgs = (unsigned)std::min<int64_t>((a.n + a.tok - 1) / a.tok, fit);
  TraceScope ts_(s, BWD ? "qk_rope_bwd" : "qk_rope_fwd", a.D, NORM);
  hipLaunchKernelGGL((rope_kernel<T, P2, FAR, NORM, BWD>), dim3(wgs), dim3(kThreads), 0, s, a);
  return wgs;
}

template <typename T, bool FAR, bool NORM, bool BWD>
unsigned launch_p(RopeArgs& a, hipStream_t s) {
  return a.D <= 64 ? launch<T, 8, FAR, NORM, BWD>(a, s) : a.D <= 128 ? launch<T, 16, FAR, NORM, BWD>(a, s)
                                                                      : launch<T, 32, FAR, NORM, BWD>(a, s);
}

template <typename T>
unsigned launch_t(RopeArgs& a, bool far_pairs, bool norm, bool bwd, hipStream_t s) {
  if (far_pairs) {
    if (norm) return bwd ? launch_p<T, true, true, true>(a, s) : launch_p<T, true, true, false>(a, s);
    return bwd ? launch_p<T, true, false, true>(a, s) : launch_p<T, true, false, false>(a, s);
  }
  if (norm) return bwd ? launch_p<T, false, true, true>(a, s) : launch_p<T, false, true, false>(a, s);
  return bwd ? launch_p<T, false, false, true>(a, s) : launch_p<T, false, false, false>(a, s);
}

}  // namespace

hipError_t launch_qk_rope(const RopeShape& sh, const RopeSide (&side)[2], bool bwd, float* part,
                          float* dwq, float* dwk, hipStream_t s) {
  const bool norm = side[0].w || side[1].w;
  unsigned wgs = 0;
  if (sh.n > 0) {
    RopeArgs a{};
    for (int i = 0; i < 2; ++i) a.side[i] = side[i];
    a.part = part;
    a.pos = sh.pos;
    a.idx = sh.idx;
    a.n = sh.n;
    a.pos_rows = (uint32_t)sh.pos_rows;
    a.D = sh.D;
    a.n_axes = sh.n_axes;
    a.eps = sh.eps;
    a.w_bf16 = sh.w_bf16;
    for (int x = 0; x < sh.n_axes; ++x) {
      // one power an axis: the products are off by at most 128 steps of 2^-53, and 64
      // powers would take the call longer than its launch
      const double ratio = std::pow(sh.theta, -2.0 / sh.dims[x]);
      double rev = 1 / (2 * 3.14159265358979323846);
      for (int i = 0; i < sh.dims[x] / 2; ++i, rev *= ratio) {
        a.axis[a.half] = (uint8_t)x;
        a.rev[a.half++] = rev;
      }
    }
    wgs = sh.bf16 ? launch_t<__bf16>(a, sh.far_pairs, norm, bwd, s) : launch_t<float>(a, sh.far_pairs, norm, bwd, s);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (bwd && norm) {
    TraceScope ts_(s, "qk_rope_weight_sum", sh.D);
    hipLaunchKernelGGL(rope_weight_sum_kernel, dim3((unsigned)((2 * sh.D + 3) / 4)), dim3(kThreads), 0, s, part,
                       (int)wgs, sh.D, dwq, dwk);
  }
  return hipGetLastError();
}

}  // namespace ut
