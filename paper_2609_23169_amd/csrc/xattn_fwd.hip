// Attention of image tokens to an encoder's states of another length, forward,
// on gfx950: O = softmax(Q K^T scale) V over the keys in use, and the rows'
// log-sum-exp. Every query of a sample reads every key in use of its sample.
//
// One workgroup takes 32 NW query rows of a key head (NW waves of 32; a row is a
// token and one of the G heads that share the key head) and walks the sample's
// 64-key tiles, K and V double-buffered in LDS by direct loads. As in the
// block-sparse forward the scores are formed transposed, S^T = K Q^T on 32x32x16
// bf16 MFMA, so that a lane holds one row's scores and the softmax needs no
// exchange but one; the exponentials run against the maximum of the first tile,
// which is replaced when a lane's tile sum leaves fp32's safe range; then
// O^T += V^T P^T on 16x16x32 after one v_permlane16_swap per register. Sums,
// maxima and O are fp32; P is rounded to bf16 for the second product (half a
// step, 2^-9 relative, as large as that of V itself).
//
// With few rows the grid would leave the chip idle, and one workgroup would
// read a long sequence alone: then the keys are split over workgroups, each
// writes its unnormalised fp32 O with its maximum and sum, and a second launch
// joins them in a fixed order. No atomics: equal results on every run.
#include <algorithm>
#include <type_traits>

#include "xattn_util.h"

namespace ut {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSumGuard = 18446744073709551616.0f;   // 2^64: per-lane tile sum bound

// Partial results of split s: sums[s][stat] = {maximum (log2 units), sum} and
// O[s][stat][D], stat a row's index in the LSE tensor.
struct Parts {
  float2* sums;
  float* o;
  int64_t stats;
};

template <int DP, int NW, bool SPLIT>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 2 : 1) void xattn_fwd_kernel(const XArgs a, const unsigned rtiles,
                                                               const unsigned splits, const bool by_xcd,
                                                               const Parts parts) {
  constexpr int ROWB = DP * 2, CPR = DP / 8, TILEB = kXKeys * ROWB, KS = DP / 16, DT = DP / 16;
  __shared__ __attribute__((aligned(1024))) char k_lds0[TILEB];
  __shared__ __attribute__((aligned(1024))) char k_lds1[TILEB];
  __shared__ __attribute__((aligned(1024))) char v_lds0[TILEB];
  __shared__ __attribute__((aligned(1024))) char v_lds1[TILEB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g = lane >> 5, c16 = lane & 15, gq = lane >> 4;

  const unsigned item = xcd_item(blockIdx.x, gridDim.x, by_xcd);
  const unsigned rt = item % rtiles, sp = SPLIT ? item / rtiles % splits : 0;
  const unsigned bh = item / rtiles / (SPLIT ? splits : 1);
  const int hk = (int)(bh % (unsigned)a.Hk), b = (int)(bh / (unsigned)a.Hk);
  const XSample sm = x_sample(a, b);
  const int rows = sm.nq * a.G;
  const int row0 = (int)rt * 32 * NW;
  if (row0 >= rows) return;   // uniform over the workgroup

  // This split's tiles.
  const int ntiles = (sm.nk + kXKeys - 1) / kXKeys;
  int t_begin = 0, t_end = ntiles;
  if constexpr (SPLIT) {
    const int per = (ntiles + (int)splits - 1) / (int)splits;
    t_begin = min((int)sp * per, ntiles);
    t_end = min(t_begin + per, ntiles);
  }
  KeyTiles tiles(a.mask ? a.mask + sm.k0 : nullptr, sm.nk, t_begin, t_end);

  // Q operand (B of S^T = K Q^T): lane holds Q[row][16 ks + 8 g .. +7].
  bf16x8 qop[KS];
  const int row = min(row0 + 32 * w + l32, rows - 1);
  {
    const int tok = row / a.G;
    const __bf16* qp = static_cast<const __bf16*>(a.q) + (sm.q0 + tok) * a.sq + (hk * a.G + row - tok * a.G) * a.D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qop[ks] = bf16x8{};
      if (16 * ks + 8 * g < a.D) qop[ks] = *reinterpret_cast<const bf16x8*>(qp + 16 * ks + 8 * g);
    }
  }
  const TileLoad<DP, NW> load_k(lane, a.D, a.sk), load_v(lane, a.D, a.sv);
  const __bf16* const kb = static_cast<const __bf16*>(a.k) + sm.k0 * a.sk + hk * a.D;
  const __bf16* const vb = static_cast<const __bf16*>(a.v) + sm.k0 * a.sv + hk * a.D;
  auto load_tile = [&](int t, uint64_t bits, char* kd, char* vd) __attribute__((always_inline)) {
    load_k(kb + (int64_t)t * kXKeys * a.sk, a.sk, bits, kd, w, lane);
    load_v(vb + (int64_t)t * kXKeys * a.sv, a.sv, bits, vd, w, lane);
  };

  // LDS lane offsets of the two products, as in the block-sparse forward.
  int koff[KS], voff[DT];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) koff[ks] = lds_off<CPR>(l32, 2 * ks + g);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    const int d = 16 * dt + 4 * (c16 & 3);
    voff[dt] = lds_off<CPR>(8 * (gq & 1) + 4 * (gq >> 1) + (c16 >> 2), d >> 3) + 2 * (d & 7);
  }
  const float c2 = a.scale * kLog2e;   // scores in log2 units
  // oacc[dt][qg]: lane holds O^T[16 dt + 4 gq + (0..3)][row 32 w + 16 qg + c16]
  f32x4 oacc[DT][2];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt][0] = oacc[dt][1] = f32x4{};
  float m_run = -INFINITY, l_run = 0.f;

  auto step = [&](uint64_t bits, const char* kt_lds, const char* vt_lds) __attribute__((always_inline)) {
    f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const bf16x8 av = *reinterpret_cast<const bf16x8*>(kt_lds + koff[ks] + kt * 32 * ROWB);
        s[kt] = mfma32(av, qop[ks], s[kt]);
      }
    if (bits != ~(uint64_t)0) {   // uniform
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const unsigned mine = (unsigned)(bits >> (32 * kt)) >> (4 * g);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[kt][e] = mine >> (8 * (e >> 2) + (e & 3)) & 1 ? s[kt][e] : -INFINITY;
      }
    }
    u32x4 pq[2][2];
    float lsum = 0.f;
    auto expo = [&]() __attribute__((always_inline)) {
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
      lsum = 0.f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float p0 = fast_exp2(__builtin_fmaf(s[kt][e], c2, -m_use));
          const float p1 = fast_exp2(__builtin_fmaf(s[kt][e + 1], c2, -m_use));
          lsum += p0;
          lsum += p1;
          pq[kt][(e >> 2) & 1][((e & 3) >> 1) + 2 * (e >> 3)] = pack_bf16x2(p0, p1);
        }
    };
    constexpr int kPairs = 2 * DT, kPre = 4;
    bf16x8 vop[kPre];
    auto read_v = [&](int pp) __attribute__((always_inline)) {
      const char* vbuf = vt_lds + 32 * (pp & 1) * ROWB + voff[pp >> 1];
      const s16x4 lo = lds_read_tr16(vbuf);
      const s16x4 hi = lds_read_tr16(vbuf + 16 * ROWB);
      const s16x8 v8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(bf16x8, v8);
    };
#pragma unroll
    for (int pp = 0; pp < kPre; ++pp) vop[pp] = read_v(pp);
    bool redo = __ballot(m_run == -INFINITY) != 0;
    if (!redo) {
      expo();
      redo = __ballot(!(lsum <= kSumGuard)) != 0;   // also catches inf and NaN
    }
    if (redo) {
      float mx = s[0][0];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = (kt == 0 ? 1 : 0); e < 16; ++e) mx = fmaxf(mx, s[kt][e]);
      mx = pair_max(mx) * c2;
      float alpha = 1.f;
      if (mx > m_run) {
        alpha = fast_exp2(m_run - mx);   // 0 on the first tile
        l_run *= alpha;
        m_run = mx;
      }
      const auto ar = __builtin_amdgcn_permlane16_swap(__float_as_uint(alpha), __float_as_uint(alpha), false, false);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        oacc[dt][0] *= __uint_as_float(ar[0]);
        oacc[dt][1] *= __uint_as_float(ar[1]);
      }
      expo();
    }
    l_run += lsum;
    bf16x8 pop[2][2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const u32x4 x = pq[kt][0], y = pq[kt][1];
      u32x4 nx, ny;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const auto r = __builtin_amdgcn_permlane16_swap(x[v], y[v], false, false);
        nx[v] = r[0];
        ny[v] = r[1];
      }
      pop[kt][0] = __builtin_bit_cast(bf16x8, nx);
      pop[kt][1] = __builtin_bit_cast(bf16x8, ny);
    }
#pragma unroll
    for (int pp = 0; pp < kPairs; ++pp) {
      const bf16x8 av = vop[pp % kPre];
      if (pp + kPre < kPairs) vop[pp % kPre] = read_v(pp + kPre);
      oacc[pp >> 1][0] = mfma16(av, pop[pp & 1][0], oacc[pp >> 1][0]);
      oacc[pp >> 1][1] = mfma16(av, pop[pp & 1][1], oacc[pp >> 1][1]);
    }
#pragma unroll
    for (int pp = 0; pp + kPre < kPairs; ++pp) {
      __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);   // MFMA
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);   // DS read
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 2 * kPre, 0);
  };

  // Tile in stage P: its successor's loads into the other stage (read in the
  // iteration before, behind the last barrier), its products, the wait.
  int tile = 0;
  uint64_t bits = 0;
  bool more = tiles.next(tile, bits);
  auto iter = [&](auto par) __attribute__((always_inline)) {
    constexpr int P = decltype(par)::value;
    const uint64_t now = bits;
    more = tiles.next(tile, bits);
    if (more) load_tile(tile, bits, P ? k_lds0 : k_lds1, P ? v_lds0 : v_lds1);
    step(now, P ? k_lds1 : k_lds0, P ? v_lds1 : v_lds0);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
  };
  if (more) {
    load_tile(tile, bits, k_lds0, v_lds0);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    while (true) {
      iter(std::integral_constant<int, 0>{});
      if (!more) break;
      iter(std::integral_constant<int, 1>{});
      if (!more) break;
    }
  }

  // O = O^T / l, LSE = (m + log2 l) ln 2; a row without keys: 0 and -inf.
  const float l_tot = pair_sum(l_run);
  const bool none = l_tot == 0.f;
  if (row0 + 32 * w + l32 < rows && g == 0) {
    const int tok = row / a.G;
    const int64_t stat = sm.stat0 + (hk * a.G + row - tok * a.G) * sm.hstep + tok;
    if constexpr (SPLIT) parts.sums[sp * parts.stats + stat] = make_float2(m_run, l_tot);
    else a.lse[stat] = none ? -INFINITY : (m_run + __log2f(l_tot)) * kLn2;
  }
  const float inv = SPLIT ? 1.f : none ? 0.f : 1.f / l_tot;
  const auto ir = __builtin_amdgcn_permlane16_swap(__float_as_uint(inv), __float_as_uint(inv), false, false);
#pragma unroll
  for (int qg = 0; qg < 2; ++qg) {
    const int ro = row0 + 32 * w + 16 * qg + c16;
    if (ro >= rows) continue;
    const int tok = ro / a.G, head = hk * a.G + ro - tok * a.G;
    const float iv = __uint_as_float(ir[qg]);
    if constexpr (SPLIT) {
      float* op = parts.o + (sp * parts.stats + sm.stat0 + head * sm.hstep + tok) * a.D + 4 * gq;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        if (16 * dt + 4 * gq < a.D) *reinterpret_cast<f32x4*>(op + 16 * dt) = oacc[dt][qg];
    } else {
      __bf16* op = static_cast<__bf16*>(a.o) + (sm.q0 + tok) * a.so + head * a.D + 4 * gq;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        bf16x4 v4;
#pragma unroll
        for (int e = 0; e < 4; ++e) v4[e] = (__bf16)(oacc[dt][qg][e] * iv);
        if (16 * dt + 4 * gq < a.D) *reinterpret_cast<bf16x4*>(op + 16 * dt) = v4;
      }
    }
  }
}

// Joins the splits of a row: GPR groups of 32 lanes take every GPR-th split,
// four columns a lane, and the groups' sums are added in LDS.
template <int GPR>
__global__ __launch_bounds__(256) void xattn_join_kernel(const XArgs a, const int splits, const Parts parts) {
  __shared__ float4 red[256];
  __shared__ float red_l[8];
  constexpr int kRows = 8 / GPR;
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5, sub = grp % GPR;
  for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < parts.stats; r0 += (int64_t)gridDim.x * kRows) {
    const int64_t r = r0 + grp / GPR;
    // row r: the statistics are laid out [B, Hq, Nq] or [Hq, Tq]
    bool live = r < parts.stats;
    int64_t tok = 0;
    int head = 0;
    if (live) {
      if (a.cuq) {
        head = (int)(r / a.Tq);
        tok = r - (int64_t)head * a.Tq;
        live = in_sample(a.cuq, a.Tq, a.B, a.Nq, tok);
      } else {
        const int64_t bh = r / a.Nq;
        head = (int)(bh % a.Hq);
        tok = bh / a.Hq * a.Nq + (r - bh * a.Nq);
      }
    }
    float M = -INFINITY;
    if (live)
      for (int s = lane; s < splits; s += 32) {
        const float2 p = parts.sums[s * parts.stats + r];
        M = p.y != 0.f ? fmaxf(M, p.x) : M;
      }
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) M = fmaxf(M, __shfl_xor(M, m, 64));
    float L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live) {
#pragma unroll 4
      for (int s = sub; s < splits; s += GPR) {
        const float2 p = parts.sums[s * parts.stats + r];
        if (p.y == 0.f) continue;   // no keys in use here
        const float f = fast_exp2(p.x - M);
        L += p.y * f;
        if (4 * lane < a.D) {
          const float4 o = *reinterpret_cast<const float4*>(parts.o + (s * parts.stats + r) * a.D + 4 * lane);
          acc.x += o.x * f, acc.y += o.y * f, acc.z += o.z * f, acc.w += o.w * f;
        }
      }
    }
    if constexpr (GPR > 1) {
      __syncthreads();
      red[threadIdx.x] = acc;
      if (lane == 0) red_l[grp] = L;
      __syncthreads();
      if (sub == 0)
        for (int k = 1; k < GPR; ++k) {
          const float4 o = red[threadIdx.x + 32 * k];
          acc.x += o.x, acc.y += o.y, acc.z += o.z, acc.w += o.w;
          L += red_l[grp + k];
        }
    }
    if (!live || sub != 0) continue;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (lane == 0) a.lse[r] = L == 0.f ? -INFINITY : (M + __log2f(L)) * kLn2;
    if (4 * lane < a.D) {
      const bf16x4 v = {(__bf16)(acc.x * inv), (__bf16)(acc.y * inv), (__bf16)(acc.z * inv), (__bf16)(acc.w * inv)};
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.o) + tok * a.so + head * a.D + 4 * lane) = v;
    }
  }
}

// Waves of a workgroup: as many as there are tiles of 32 rows, up to four.
int fwd_waves(const XArgs& a) {
  const int64_t rows = (int64_t)a.Nq * a.G;
  return rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
}
int64_t fwd_groups(const XArgs& a) {
  const int64_t per = 32 * fwd_waves(a);
  return (int64_t)a.B * a.Hk * (((int64_t)a.Nq * a.G + per - 1) / per);
}
int64_t stats_of(const XArgs& a) { return a.Tq * a.Hq; }

template <int DP, int NW>
void launch_fwd(const XArgs& a, int splits, const Parts& parts, hipStream_t s) {
  const unsigned rtiles = (unsigned)(((int64_t)a.Nq * a.G + 32 * NW - 1) / (32 * NW));
  const dim3 grid((unsigned)(fwd_groups(a) * splits));
  const bool by_xcd = (int64_t)a.Nk * a.D * 4 <= kXcdHeadBytes;
  TraceScope ts_(s, splits > 1 ? "xattn_fwd_split" : "xattn_fwd", DP, NW);
  if (splits > 1)
    hipLaunchKernelGGL((xattn_fwd_kernel<DP, NW, true>), grid, dim3(64 * NW), 0, s, a, rtiles, (unsigned)splits, by_xcd, parts);
  else
    hipLaunchKernelGGL((xattn_fwd_kernel<DP, NW, false>), grid, dim3(64 * NW), 0, s, a, rtiles, 1u, by_xcd, parts);
}
template <int GPR>
void launch_join(const XArgs& a, int splits, const Parts& parts, hipStream_t s) {
  TraceScope ts_(s, "xattn_join", GPR);
  const int64_t per = 8 / GPR;
  hipLaunchKernelGGL((xattn_join_kernel<GPR>), dim3((unsigned)std::min<int64_t>((parts.stats + per - 1) / per, 1 << 20)),
                     dim3(256), 0, s, a, splits, parts);
}

}  // namespace

int xattn_fwd_splits(const XArgs& a) {
  const int64_t groups = fwd_groups(a), tiles = ((int64_t)a.Nk + kXKeys - 1) / kXKeys;
  if (groups == 0) return 1;
  return (int)std::max<int64_t>(1, std::min(512 / groups, tiles / 4));
}
size_t xattn_fwd_workspace(const XArgs& a) {
  const int splits = xattn_fwd_splits(a);
  return splits > 1 ? (size_t)splits * stats_of(a) * (sizeof(float2) + (size_t)a.D * sizeof(float)) : 0;
}

hipError_t launch_xattn_fwd(const XArgs& a, void* workspace, hipStream_t s) {
  const int splits = xattn_fwd_splits(a);
  Parts parts{};
  parts.stats = stats_of(a);
  if (splits > 1) {   // O first: its rows are 16-byte aligned
    parts.o = static_cast<float*>(workspace);
    parts.sums = reinterpret_cast<float2*>(parts.o + (size_t)splits * parts.stats * a.D);
  }
  const int nw = fwd_waves(a);
  if (a.D <= 64)
    nw == 1 ? launch_fwd<64, 1>(a, splits, parts, s) : nw == 2 ? launch_fwd<64, 2>(a, splits, parts, s) : launch_fwd<64, 4>(a, splits, parts, s);
  else
    nw == 1 ? launch_fwd<128, 1>(a, splits, parts, s) : nw == 2 ? launch_fwd<128, 2>(a, splits, parts, s) : launch_fwd<128, 4>(a, splits, parts, s);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (splits > 1) splits >= 16 ? launch_join<8>(a, splits, parts, s) : launch_join<1>(a, splits, parts, s);
  return hipGetLastError();
}

}  // namespace ut
