// Attention of image tokens to an encoder's states of another length, forward,
// on gfx950: O = softmax(Q K^T scale) V over the keys in use, and the rows'
// log-sum-exp. Every query of a sample reads every key in use of its sample.
//
// One workgroup takes 32 NW query rows of a key head (NW waves of 32; a row is a
// token and one of the G heads that share the key head) and walks the sample's
// 64-key tiles, K and V double-buffered in LDS by direct loads. As in the
// block-sparse forward the scores are formed transposed, S^T = K Q^T on 32x32x16
// bf16 MFMA, so that a lane holds one row's scores and the softmax needs no
// exchange but one. The exponentials run against the maximum of the item's first
// 32 keys; another one is taken (O and the sum rescaled, the half tile's
// exponentials formed again) only when a lane's sum of a half tile leaves fp32's
// safe range, above 2^64: O and the sum always use the same reference, so the
// result is exact in real arithmetic. Then
// O^T += V^T P^T on 16x16x32 after one v_permlane16_swap per register. Sums,
// maxima and O are fp32; P is rounded to bf16 for the second product (half a
// step, 2^-9 relative, as large as that of V itself).
//
// With few rows the grid would leave the chip idle, and one workgroup would
// read a long sequence alone: then the keys are split over workgroups, each
// writes its unnormalised fp32 O with its maximum and sum, and a second launch
// joins them in a fixed order. No atomics: equal results on every run. Parts for
// one round of the chip: two rounds of half the length (which would even out
// unequal samples) took 56.5 + 8.2 us against 52.5 + 6.7 at 4 x 32 query heads on
// 16,391 keys.
//
// What bounds it: 22,879 queries on 4,097 keys, 24 heads of 128, take 1,060 to 1,080
// us, 1,070 TFLOP/s: matrix cores 51% busy, vector work 43%, LDS reads (a wave reads
// the tile for its 32 rows) about as long as the products, at the clock that the
// board's power limit leaves (1.75 of 2.4 GHz; rows of zeros run 16% faster). 77,586
// queries on 512 keys take 560 us, 870 TFLOP/s: a change of item every eight tiles
// (about 5,000 of 37,000 cycles) and 0.19 ms of rows at the copy rate come on top. One
// query each of 32 heads on 16,391 keys: 4.3 TB/s.
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
__global__ __launch_bounds__(64 * NW, NW < 4 ? 1 : DP == 64 ? 3 : 2) void xattn_fwd_kernel(const XArgs a, const XOrder order,
                                                                                           const Parts parts) {
  constexpr int ROWB = DP * 2, CPR = DP / 8, TILEB = kXKeys * ROWB, KS = DP / 16, DT = DP / 16;
  __shared__ __attribute__((aligned(1024))) char k_lds0[TILEB];
  __shared__ __attribute__((aligned(1024))) char k_lds1[TILEB];
  __shared__ __attribute__((aligned(1024))) char v_lds0[TILEB];
  __shared__ __attribute__((aligned(1024))) char v_lds1[TILEB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g = lane >> 5, c16 = lane & 15, gq = lane >> 4;

  if (a.zero_rest) {   // here, not in a launch of its own, which costs 6 us
    x_clear_rest(a.cuq, a.B, a.Tq, a.Hq * a.D, a.o, a.so);
    const int64_t end = min(max((int64_t)x_cu(a.cuq, a.B), (int64_t)0), a.Tq), rest = a.Tq - end;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + tid; i < rest * a.Hq; i += (int64_t)gridDim.x * blockDim.x)
      a.lse[i / rest * a.Tq + end + i % rest] = -INFINITY;
  }

  // Q operand (B of S^T = K Q^T), once turned: lane holds Q[row][16 ks + 8 g .. +7].
  bf16x8 qop[KS];
  auto load_rows = [&](const XItem& at) __attribute__((always_inline)) {
    const XArgs& x = *x_args_again();
    const XSample sm = x_sample(x, at.b);
    x_load_rows<DP>(qop, x.q, sm.q0, x.sq, (int64_t)at.hk * x.G * x.D, at.tile * 32 * NW + 32 * w, sm.nq, x.G, x.D);
  };
  const TileLoad<DP, NW> load_k(lane, a.sk), load_v(lane, a.sv);

  // LDS offsets of the two products: chunk 2 ks + g of row l32, and V^T's operand
  // as in the block-sparse forward.
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
  float m_run = 0.f, l_run = 0.f;
  bool fresh = true;                   // no key of the item seen yet: no reference (uniform)

  TileSeq seq;

  // One tile in two 32-key halves, so that a wave's vector work has matrix work of
  // its own beside it: S of half 1 runs beside the exponentials of half 0, and the
  // second product of half 0 beside the exponentials of half 1. With `swap` the
  // rows of the next item take the place of this one's once the scores are formed.
  // The next tile's loads (load(u), u < 2 IPW) stand between the first products.
  using Load = TileLoad<DP, NW>;
  auto step = [&](uint64_t bits, const char* kt_lds, const char* vt_lds, bool swap, bool loads,
                  auto load) __attribute__((always_inline)) {
    constexpr int kAhead = 4, kPre = 4;
    bf16x8 kop[kAhead], vop[kPre];
    auto read_k = [&](int n) __attribute__((always_inline)) {   // product n: half n / KS, ks n % KS
      return *reinterpret_cast<const bf16x8*>(kt_lds + koff[n % KS] + n / KS * 32 * ROWB);
    };
    auto read_v = [&](int n) __attribute__((always_inline)) {   // half n / DT, d tile n % DT
      const char* vbuf = vt_lds + n / DT * 32 * ROWB + voff[n % DT];
      const s16x4 lo = lds_read_tr16(vbuf);
      const s16x4 hi = lds_read_tr16(vbuf + 16 * ROWB);
      const s16x8 v8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(bf16x8, v8);
    };
    f32x16 s[2];
    u32x4 pq[2];      // a half's P as bf16 pairs, as in the block-sparse forward
    float lsum = 0.f, x[2], m_use = 0.f;
    // Elements 2 i and 2 i + 1 of half h: their exponents, and their P with its sums.
    auto expo0 = [&](int h, int i) __attribute__((always_inline)) {
      x[0] = __builtin_fmaf(s[h][2 * i], c2, -m_use);
      x[1] = __builtin_fmaf(s[h][2 * i + 1], c2, -m_use);
    };
    auto expo1 = [&](int i) __attribute__((always_inline)) {
      const float p0 = fast_exp2(x[0]), p1 = fast_exp2(x[1]);
      lsum += p0;
      lsum += p1;
      const int e = 2 * i;
      unsigned q = pack_bf16x2(p0, p1);
      pin_value(q);      // here, not at its use behind the matrix instructions
      pin_value(lsum);
      pq[(e >> 2) & 1][((e & 3) >> 1) + 2 * (e >> 3)] = q;
    };
    auto half_max = [&](int h) __attribute__((always_inline)) {   // of this lane's keys
      float mx = s[h][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[h][e]);
      return fmaxf(mx * c2, -3.0e38f);
    };
    // Before half h's exponentials: unused keys, and the item's reference.
    auto prepare = [&](int h) __attribute__((always_inline)) {
      const unsigned half = (unsigned)(bits >> (32 * h));
      if (half != ~0u) {   // uniform
        const unsigned mine = half >> (4 * g);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[h][e] = mine >> (8 * (e >> 2) + (e & 3)) & 1 ? s[h][e] : -INFINITY;
      }
      if (fresh && half) {   // uniform
        m_run = pair_max(half_max(h));
        fresh = false;
      }
      m_use = m_run;
      lsum = 0.f;
    };
    // After them: another reference where a lane's sum left fp32's safe range (or
    // is inf or NaN), then P to the operand layout of two 16-row groups.
    bf16x8 pop[2];
    auto settle = [&](int h) __attribute__((always_inline)) {
      const bool over = !(lsum <= kSumGuard);
      if (__ballot(over) != 0) {
        // from the lanes whose sum it is: other rows keep theirs, so that no row's
        // result depends on its neighbours
        const float to = fmaxf(pair_max(over ? half_max(h) : -3.0e38f), m_run), alpha = fast_exp2(m_run - to);
        l_run *= alpha;
        m_run = m_use = to;
        const auto ar = __builtin_amdgcn_permlane16_swap(__float_as_uint(alpha), __float_as_uint(alpha), false, false);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          oacc[dt][0] *= __uint_as_float(ar[0]);
          oacc[dt][1] *= __uint_as_float(ar[1]);
        }
        lsum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          expo0(h, i);
          expo1(i);
        }
      }
      l_run += lsum;
      u32x4 nx, ny;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const auto r = __builtin_amdgcn_permlane16_swap(pq[0][v], pq[1][v], false, false);
        nx[v] = r[0];
        ny[v] = r[1];
      }
      pop[0] = __builtin_bit_cast(bf16x8, nx);
      pop[1] = __builtin_bit_cast(bf16x8, ny);
    };

#pragma unroll
    for (int n = 0; n < kAhead; ++n) kop[n] = read_k(n);
    pin_order();
    // S^T of half 0, its K operands read kAhead products before their use. Between here
    // and the last products a wave goes before one in these two phases, which have no
    // vector work (image case 1,071 -> 1,062 us, training forward 567 -> 557; the other
    // way round 1,070 and 562).
    __builtin_amdgcn_s_setprio(0);
    s[0] = f32x16{};
    if (loads) {   // uniform
#pragma unroll
      for (int n = 0; n < KS; ++n) {
        s[0] = mfma32(kop[n % kAhead], qop[n], s[0]);
        kop[n % kAhead] = read_k(n + kAhead);
#pragma unroll
        for (int u = n * 2 * Load::IPW / KS; u < (n + 1) * 2 * Load::IPW / KS; ++u) load(u);
        pin_order();
      }
    } else {
#pragma unroll
      for (int n = 0; n < KS; ++n) {
        s[0] = mfma32(kop[n % kAhead], qop[n], s[0]);
        kop[n % kAhead] = read_k(n + kAhead);
        pin_order();
      }
    }
    __builtin_amdgcn_s_setprio(1);
    prepare(0);
    pin_order();
    // S^T of half 1 beside the exponentials of half 0
    s[1] = f32x16{};
#pragma unroll
    for (int n = 0; n < KS; ++n) {
      s[1] = mfma32(kop[n % kAhead], qop[n], s[1]);
      if (n + kAhead < KS) kop[n % kAhead] = read_k(KS + n + kAhead);
      else if (n + kAhead - KS < kPre) vop[n + kAhead - KS] = read_v(n + kAhead - KS);
#pragma unroll
      for (int i = n * 8 / KS; i < (n + 1) * 8 / KS; ++i) {
        expo0(0, i);
        expo1(i);
      }
      pin_order();
    }
    if (swap) load_rows(seq.item(seq.at, order));   // uniform
    settle(0);
    prepare(1);
    pin_order();
    // O^T += V^T P^T of half 0 beside the exponentials of half 1
#pragma unroll
    for (int n = 0; n < DT; ++n) {
      const bf16x8 av = vop[n % kPre];
      oacc[n][0] = mfma16(av, pop[0], oacc[n][0]);
      oacc[n][1] = mfma16(av, pop[1], oacc[n][1]);
      vop[n % kPre] = read_v(n + kPre);
#pragma unroll
      for (int i = n * 8 / DT; i < (n + 1) * 8 / DT; ++i) {
        expo0(1, i);
        expo1(i);
      }
      pin_order();
    }
    settle(1);
    __builtin_amdgcn_s_setprio(0);
    pin_order();
#pragma unroll
    for (int n = 0; n < DT; ++n) {
      const bf16x8 av = vop[n % kPre];
      oacc[n][0] = mfma16(av, pop[0], oacc[n][0]);
      oacc[n][1] = mfma16(av, pop[1], oacc[n][1]);
      if (n + kPre < DT) vop[n % kPre] = read_v(DT + n + kPre);
      pin_order();
    }
    __builtin_amdgcn_s_setprio(1);
  };

  // O = O^T / l, LSE = (m + log2 l) ln 2; a row without keys: 0 and -inf.
  auto finish = [&](const XItem& at, char* lds0, char* lds1) __attribute__((always_inline)) {
    const XArgs& x = *x_args_again();
    const XSample sm = x_sample(x, at.b);
    const int rows = sm.nq * x.G, r0 = at.tile * 32 * NW + 32 * w;
    const float l_tot = pair_sum(l_run);
    const bool none = l_tot == 0.f;
    if (r0 + l32 < rows && g == 0) {
      const int row = r0 + l32, tok = row_token(row, x.G);
      const int64_t stat = sm.stat0 + (at.hk * x.G + row - tok * x.G) * sm.hstep + tok;
      if constexpr (SPLIT) parts.sums[at.part * parts.stats + stat] = make_float2(m_run, l_tot);
      else x.lse[stat] = none ? -INFINITY : (m_run + __log2f(l_tot)) * kLn2;
    }
    const float inv = SPLIT ? 1.f : none ? 0.f : 1.f / l_tot;
    const auto ir = __builtin_amdgcn_permlane16_swap(__float_as_uint(inv), __float_as_uint(inv), false, false);
    if constexpr (SPLIT) {
#pragma unroll
      for (int qg = 0; qg < 2; ++qg) {
        const int row = r0 + 16 * qg + c16, tok = row_token(row, x.G);
        if (row >= rows) continue;
        const int64_t stat = sm.stat0 + (at.hk * x.G + row - tok * x.G) * sm.hstep + tok;
        float* op = parts.o + (at.part * parts.stats + stat) * x.D + 4 * gq;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
          if (16 * dt + 4 * gq < x.D) *reinterpret_cast<f32x4*>(op + 16 * dt) = oacc[dt][qg];
      }
    } else {
      x_store_rows<DP>(x.o, sm.q0, x.so, (int64_t)at.hk * x.G * x.D, r0, sm.nq, x.G, x.D, lds0, lds1,
                       [&](int dt, int qg) { return oacc[dt][qg] * __uint_as_float(ir[qg]); });
    }
  };

  // A workgroup's items in turn, their tiles as one sequence: a tile's loads are
  // issued while the tile before it is worked on, across items too.
  seq.begin(x_items((unsigned)a.B * order.tiles * order.splits * (unsigned)a.Hk));
  bool have = false;   // a tile lies in the current stage
  auto iter = [&](auto par) __attribute__((always_inline)) {   // false: done
    constexpr int P = decltype(par)::value;
    const uint64_t now = seq.bits;
    bool changed;
    const bool more = seq.next(order, 32 * NW, changed);
    if (!have && !more) return false;
    char* const kn = P ? k_lds0 : k_lds1;
    char* const vn = P ? v_lds0 : v_lds1;
    const int64_t key = seq.k0 + (int64_t)seq.tile * kXKeys;
    const __amdgpu_buffer_rsrc_t rk = load_k.tile(static_cast<const __bf16*>(a.k) + key * a.sk + seq.hk * a.D, a.sk);
    const __amdgpu_buffer_rsrc_t rv = load_v.tile(static_cast<const __bf16*>(a.v) + key * a.sv + seq.hk * a.D, a.sv);
    const bool all = more && seq.bits == ~(uint64_t)0;
    if (more && !all) {
      load_k.masked(rk, a.sk, seq.bits, kn, w, lane, a.D);
      load_v.masked(rv, a.sv, seq.bits, vn, w, lane, a.D);
    }
    auto load = [&](int u) __attribute__((always_inline)) {
      if (u < Load::IPW) load_k.one(rk, a.sk, kn, w, u, a.D);
      else load_v.one(rv, a.sv, vn, w, u - Load::IPW, a.D);
    };
    // At 128 columns before the first tile too, beside its loads: what it leaves is not
    // used, and a branch around it costs the loop more (packed case 259 -> 275 us). At
    // 64 the branch takes 1 us off a call's 10.
    if (DP == 128 || have) {
      step(now, P ? k_lds1 : k_lds0, P ? v_lds1 : v_lds0, changed && more, all, load);
    } else {
      if (all)
#pragma unroll
        for (int u = 0; u < 2 * Load::IPW; ++u) load(u);
      load_rows(seq.item(seq.at, order));
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (changed) {
      // through the wave's part of the consumed stage; the stores end beside the
      // next item's first tile
      char* const lds0 = (P ? k_lds1 : k_lds0) + w * Load::IPW * 1024;
      char* const lds1 = (P ? v_lds1 : v_lds0) + w * Load::IPW * 1024;
      if (have) finish(seq.item(seq.cur, order), lds0, lds1);
      if (more) XTurn<DP>(x_lane_again()).turn(qop, lds0, lds1);
      seq.cur = seq.at;
      m_run = l_run = 0.f;
      fresh = true;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) oacc[dt][0] = oacc[dt][1] = f32x4{};
    }
    have = true;
    return more;
  };
  while (iter(std::integral_constant<int, 0>{}) && iter(std::integral_constant<int, 1>{})) {
  }
}

// Joins the parts of a row: GPR groups of 32 lanes take every GPR-th part, four
// columns a lane, and the groups' sums are added in LDS.
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

// Parts of the keys, and waves of a workgroup: four, or one where up to 32 rows meet
// split keys (4 rows of 4 x 8 key heads on 16,391 keys: 49 us against 51 with three
// idle waves beside; unsplit keys the other way round, 14.2 against 13.0 for 16
// samples of 20 rows and 300 keys). Parts below four tiles: the last case split in two
// takes 11.7 + 6.4, 16 samples of 60 rows 15.9 + 7.5 against 16.2.
struct Shape {
  int splits, waves;
};
Shape fwd_shape(const XArgs& a) {
  const int64_t rows = (int64_t)a.Nq * a.G, heads = (int64_t)a.B * a.Hk, tiles = ((int64_t)a.Nk + kXKeys - 1) / kXKeys;
  auto splits = [&](int nw) {
    const int64_t groups = heads * ((rows + 32 * nw - 1) / (32 * nw));
    return groups == 0 ? 1 : (int)std::max<int64_t>(1, std::min(x_resident(x_padded(a), nw) / groups, tiles / 4));
  };
  if (rows <= 32 && splits(1) > 1) return Shape{splits(1), 1};
  return Shape{splits(4), 4};
}
int64_t stats_of(const XArgs& a) { return a.Tq * a.Hq; }

template <int DP, int NW>
void launch_fwd(const XArgs& a, int splits, const Parts& parts, hipStream_t s) {
  const XOrder order{head_group(a), (unsigned)(((int64_t)a.Nq * a.G + 32 * NW - 1) / (32 * NW)), (unsigned)splits};
  const int64_t items = (int64_t)a.B * a.Hk * order.tiles * splits;
  const dim3 grid((unsigned)(std::min<int64_t>(std::max<int64_t>(items, 1), x_resident(DP, NW)) + 7) / 8 * 8);
  TraceScope ts_(s, splits > 1 ? "xattn_fwd_split" : "xattn_fwd", DP, NW);
  if (splits > 1) {
    hipLaunchKernelGGL((xattn_fwd_kernel<DP, NW, true>), grid, dim3(64 * NW), 0, s, a, order, parts);
  } else {
    if constexpr (NW == 4)
      hipLaunchKernelGGL((xattn_fwd_kernel<DP, NW, false>), grid, dim3(64 * NW), 0, s, a, order, parts);
  }
}
template <int GPR>
void launch_join(const XArgs& a, int splits, const Parts& parts, hipStream_t s) {
  TraceScope ts_(s, "xattn_join", GPR);
  const int64_t per = 8 / GPR;
  hipLaunchKernelGGL((xattn_join_kernel<GPR>), dim3((unsigned)std::min<int64_t>((parts.stats + per - 1) / per, 1 << 20)),
                     dim3(256), 0, s, a, splits, parts);
}

}  // namespace

size_t xattn_fwd_workspace(const XArgs& a) {
  const int splits = fwd_shape(a).splits;
  return splits > 1 ? (size_t)splits * stats_of(a) * (sizeof(float2) + (size_t)a.D * sizeof(float)) : 0;
}

hipError_t launch_xattn_fwd(const XArgs& a, void* workspace, hipStream_t s) {
  const auto [splits, waves] = fwd_shape(a);
  Parts parts{};
  parts.stats = stats_of(a);
  if (splits > 1) {   // O first: its rows are 16-byte aligned
    parts.o = static_cast<float*>(workspace);
    parts.sums = reinterpret_cast<float2*>(parts.o + (size_t)splits * parts.stats * a.D);
  }
  if (a.D <= 64)
    waves == 1 ? launch_fwd<64, 1>(a, splits, parts, s) : launch_fwd<64, 4>(a, splits, parts, s);
  else
    waves == 1 ? launch_fwd<128, 1>(a, splits, parts, s) : launch_fwd<128, 4>(a, splits, parts, s);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  // Eight groups of lanes a row where many parts are to be read for few rows: 320 rows
  // of 11 parts 6.9 us against 11.3 with one, 1,024 of 8 7.0 against 9.0; but 8,000 of
  // 8 18.9 against 13.1, and 8,000 of 3 17.3 against 9.5.
  if (splits > 1)
    splits >= 8 && parts.stats <= 4096 ? launch_join<8>(a, splits, parts, s) : launch_join<1>(a, splits, parts, s);
  return hipGetLastError();
}

}  // namespace ut
