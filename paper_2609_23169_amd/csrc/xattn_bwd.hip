// Attention of image tokens to an encoder's states of another length, backward,
// on gfx950. With P = exp(S scale - LSE) over the keys in use, delta =
// rowsum(dO o O) and dS = P o (dO V^T - delta):
//   dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO,
// dK and dV summed over the query heads that share the key head. Launches:
//
//   dQ    : query-stationary, first: it forms the rows' statistics LSE log2(e) and
//           -delta (fp32, two planes of the workspace) from LSE, O and the dO
//           rows that it holds anyway. S and dP on 32x32x16 bf16 MFMA,
//           dQ^T += K^T dS^T on 16x16x32; with few rows the keys are split as
//           below. The workgroups are persistent: the rows and the first tile of
//           the next item load beside the last tile of the one before;
//   dK/dV : key-stationary. A workgroup owns 128 keys of a key head, one wave
//           per 32, and walks the 32-token tiles of every query head of the
//           group: S and dP on 32x32x16 bf16 MFMA, dV^T += dO^T P and
//           dK^T += Q^T dS on 16x16x32, accumulators in fp32 registers. Few keys
//           (an encoder's states against a picture's tokens) make few
//           workgroups, so the query tiles are split over workgroups, each
//           writes fp32 partial sums, and a join adds them in a fixed order.
//
// Rounding: P and dS to bf16 before their second products (half a step each,
// 2^-9 relative), all sums in fp32. delta comes from O as stored (half a step
// of it), or as rowsum(P o dP) in fp32 where a row's keys in use lie in one tile.
// No atomics: equal results on every run. Keys not in use: the dQ pass reads
// zeros in their place and sets their P to 0; in the dK/dV pass a key is a
// column of its own, whatever it holds, and is stored as 0; waves whose 32 keys
// are all unused only load.
//
// What bounds it (77,060 queries, 512 keys, 24 heads of 128: dQ 795 us, dK/dV 840,
// 915 and 1,150 TFLOP/s of the products that they form): the matrix cores are 44 and
// 57% busy, vector work and LDS reads fill most of the rest, and the board's power
// limit sets the clock (1.8 to 1.9 of 2.4 GHz): with rows of zeros the same
// instructions run 17% faster. dQ also moves 1.9 GB, 0.39 ms at the copy rate, beside it.
#include <algorithm>
#include <type_traits>

#include "xattn_util.h"

namespace ut {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kBwdKeys = 128;   // keys of a dK/dV workgroup
constexpr int kRowTile = 32;    // query tokens of a dK/dV step
constexpr int kDqWaves = 4;     // of 32 rows each

// ---------------------------------------------------------------------------
// dQ
// ---------------------------------------------------------------------------
// part: fp32 [split][token][Hq][D], null with one split.
template <int DP>
__global__ __launch_bounds__(256, DP == 64 ? 3 : 2) void xattn_dq_kernel(const XArgs a, float* __restrict__ aux,
                                                                         const XOrder order, float* __restrict__ part) {
  constexpr int NW = kDqWaves, ROWB = DP * 2, CPR = DP / 8, TILEB = kXKeys * ROWB, KS = DP / 16, DT = DP / 16;
  __shared__ __attribute__((aligned(1024))) char k_lds0[TILEB];
  __shared__ __attribute__((aligned(1024))) char k_lds1[TILEB];
  __shared__ __attribute__((aligned(1024))) char v_lds0[TILEB];
  __shared__ __attribute__((aligned(1024))) char v_lds1[TILEB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g = lane >> 5, c16 = lane & 15, gq = lane >> 4;

  if (a.zero_rest) x_clear_rest(a.cuq, a.B, a.Tq, a.Hq * a.D, a.dq, a.sdq);

  bf16x8 qop[KS], doop[KS];   // Q and dO (operands, once turned)
  float lse2, l2, ndl;        // the row's LSE log2 e, that less log2(scale), and -delta
  // What only the statistics need: O as loaded, and LSE. (Set between a change of
  // item and its use alone: held in the loop otherwise.)
  struct Extra {
    bf16x8 o[KS];
    float lse;
  };
  auto load_rows = [&](const XItem& at, Extra& ex) __attribute__((always_inline)) {
    const XArgs& x = *x_args_again();
    const XSample sm = x_sample(x, at.b);
    const int r0 = at.tile * 32 * NW + 32 * w, rows = sm.nq * x.G;
    const int64_t head0 = (int64_t)at.hk * x.G * x.D;
    x_load_rows<DP>(qop, x.q, sm.q0, x.sq, head0, r0, sm.nq, x.G, x.D);
    x_load_rows<DP>(doop, x.dout, sm.q0, x.sdo, head0, r0, sm.nq, x.G, x.D);
    x_load_rows<DP>(ex.o, x.o_in, sm.q0, x.so, head0, r0, sm.nq, x.G, x.D);
    const int row = min(r0 + l32, rows - 1), tok = row_token(row, x.G);
    ex.lse = x.lse[sm.stat0 + (at.hk * x.G + row - tok * x.G) * sm.hstep + tok];
  };
  // The statistics of those rows before they are turned: a lane has pieces of rows,
  // and their sums pass through LDS. A row without keys has LSE -inf; any finite
  // value keeps its P at 0.
  auto row_stats = [&](const Extra& ex, char* lds) __attribute__((always_inline)) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const int ln = x_lane_again();
    float* const piece = reinterpret_cast<float*>(lds) + ln;   // [row][CPR]
#pragma unroll
    for (int u = 0; u < KS; ++u) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e += 2)   // products of bf16 are exact in fp32, the sums fp32
        sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{ex.o[u][e], ex.o[u][e + 1]}, bf16x2{doop[u][e], doop[u][e + 1]}, sum,
                                              false);
      piece[64 * u] = sum;
    }
    __builtin_amdgcn_wave_barrier();
    const f32x4* const mine = reinterpret_cast<const f32x4*>(lds + (ln & 31) * CPR * 4 + (ln >> 5) * CPR * 2);
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CPR / 8; ++c) {
      const f32x4 y = mine[c];
      sum += (y[0] + y[1]) + (y[2] + y[3]);
    }
    ndl = -pair_sum(sum);
    const float scale = x_args_again()->scale;
    lse2 = ex.lse == -INFINITY ? 0.f : ex.lse * kLog2e;
    l2 = lse2 - __log2f(scale);   // P scale in place of P: dS comes out scaled (2^-21 off at most)
  };
  // For the dK/dV pass too: one part writes them.
  auto put_stats = [&](const XItem& at, bool writes) __attribute__((always_inline)) {
    const int ln = x_lane_again();
    const XArgs& x = *x_args_again();
    const XSample sm = x_sample(x, at.b);
    const int row = at.tile * 32 * NW + 32 * w + (ln & 31), tok = row_token(row, x.G);
    if (writes && ln < 32 && row < sm.nq * x.G) {
      const int64_t stat = sm.stat0 + (at.hk * x.G + row - tok * x.G) * sm.hstep + tok;
      aux[stat] = lse2;
      aux[x.Tq * x.Hq + stat] = ndl;
    }
  };
  const TileLoad<DP, NW> load_k(lane, a.sk), load_v(lane, a.sv);
  // LDS offsets, as in the forward: chunk 2 ks + g of row l32, and K^T's operand.
  // The swizzle is an exclusive or, and so is the step to another ks or dt: one
  // register each and an instruction a use, where sixteen would not fit.
  const int koff0 = lds_off<CPR>(l32, g);
  const int ktr0 = lds_off<CPR>(8 * (gq & 1) + 4 * (gq >> 1) + (c16 >> 2), (c16 & 3) >> 1) + 8 * (c16 & 1);
  const float c2 = a.scale * kLog2e;
  // dq[dt][qg]: lane holds dQ^T[16 dt + 4 gq + (0..3)][row 32 w + 16 qg + c16]
  f32x4 dq[DT][2];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dq[dt][0] = dq[dt][1] = f32x4{};

  TileSeq seq;

  // A tile as two 32-key halves: S^T and dP^T, dS^T, its exchange to the
  // 16x16 operand layout, and the half's dQ product. With `swap` the next item's
  // rows take the place of this one's after the last score products. The next
  // tile's loads (load(u), u < 2 IPW) stand between the first products.
  using Load = TileLoad<DP, NW>;
  auto step = [&](uint64_t bits, const char* kt_lds, const char* vt_lds, bool swap, Extra& ex, bool loads,
                  auto load)
      __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      f32x16 s = f32x16{}, dp = f32x16{};
      int ko = koff0, kx = ktr0;
      pin_value(ko);
      pin_value(kx);
      // S^T and dP^T in turn, operands read kAhead products before their use
      constexpr int kAhead = 4, kPre = 4;
      bf16x8 op[kAhead];
      auto read_op = [&](int n) __attribute__((always_inline)) {
        return *reinterpret_cast<const bf16x8*>((n & 1 ? vt_lds : kt_lds) + (ko ^ (32 * (n >> 1))) + kt * 32 * ROWB);
      };
#pragma unroll
      for (int n = 0; n < kAhead; ++n) op[n] = read_op(n);
      // a wave in its products goes before one in its vector work (dQ of 77,060 queries on 512 keys
      // 820 -> 793 us; the other way round 823)
      __builtin_amdgcn_s_setprio(1);
      pin_order();
      auto product = [&](int n) __attribute__((always_inline)) {
        if (n & 1) dp = mfma32(op[n % kAhead], doop[n >> 1], dp);
        else s = mfma32(op[n % kAhead], qop[n >> 1], s);
        if (n + kAhead < 2 * KS) op[n % kAhead] = read_op(n + kAhead);
      };
      if (kt == 0 && loads) {   // uniform
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n) {
          product(n);
#pragma unroll
          for (int u = n * Load::IPW / KS; u < (n + 1) * Load::IPW / KS; ++u) load(u);
          pin_order();
        }
      } else {
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n) {
          product(n);
          pin_order();
        }
      }
      __builtin_amdgcn_s_setprio(0);
      const float ls = l2, nd = ndl;
      if (kt == 1 && swap) load_rows(seq.item(seq.at, order), ex);   // uniform
      if (bits != ~(uint64_t)0) {             // uniform
        const unsigned mine = (unsigned)(bits >> (32 * kt)) >> (4 * g);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[e] = mine >> (8 * (e >> 2) + (e & 3)) & 1 ? s[e] : -INFINITY;
      }
      u32x4 pq[2];
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float p0 = fast_exp2(__builtin_fmaf(s[e], c2, -ls));
        const float p1 = fast_exp2(__builtin_fmaf(s[e + 1], c2, -ls));
        pq[(e >> 2) & 1][((e & 3) >> 1) + 2 * (e >> 3)] = pack_bf16x2(p0 * (dp[e] + nd), p1 * (dp[e + 1] + nd));
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const auto r = __builtin_amdgcn_permlane16_swap(pq[0][v], pq[1][v], false, false);
        pq[0][v] = r[0];
        pq[1][v] = r[1];
      }
      pin_order();
      auto read_kt = [&](int dt) __attribute__((always_inline)) {
        const char* kbuf = kt_lds + 32 * kt * ROWB + (kx ^ (32 * dt));
        const s16x4 lo = lds_read_tr16(kbuf);
        const s16x4 hi = lds_read_tr16(kbuf + 16 * ROWB);
        const s16x8 k8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8, k8);
      };
#pragma unroll
      for (int dt = 0; dt < kPre; ++dt) op[dt] = read_kt(dt);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        dq[dt][0] = mfma16(op[dt % kPre], __builtin_bit_cast(bf16x8, pq[0]), dq[dt][0]);
        dq[dt][1] = mfma16(op[dt % kPre], __builtin_bit_cast(bf16x8, pq[1]), dq[dt][1]);
        if (dt + kPre < DT) op[dt % kPre] = read_kt(dt + kPre);
        pin_order();
      }
      __builtin_amdgcn_s_setprio(0);
    }
  };
  // delta of rows whose keys in use all lie in one tile, as rowsum(P o dP) in fp32: with
  // few keys dP - delta is a small difference, and the rounding of the O that is stored
  // would show in it (2 keys: dQ 0.0039 off in relative norm, 0.0024 with this).
  auto tile_delta = [&](uint64_t bits, const char* kt_lds, const char* vt_lds) __attribute__((always_inline)) {
    float sum = 0.f;
#pragma unroll 1
    for (int kt = 0; kt < 2; ++kt) {
      f32x16 s = f32x16{}, dp = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int off = (koff0 ^ (32 * ks)) + kt * 32 * ROWB;
        s = mfma32(*reinterpret_cast<const bf16x8*>(kt_lds + off), qop[ks], s);
        dp = mfma32(*reinterpret_cast<const bf16x8*>(vt_lds + off), doop[ks], dp);
      }
      const unsigned mine = (unsigned)(bits >> (32 * kt)) >> (4 * g);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float p = fast_exp2(__builtin_fmaf(s[e], c2, -lse2));
        sum += mine >> (8 * (e >> 2) + (e & 3)) & 1 ? p * dp[e] : 0.f;
      }
    }
    return pair_sum(sum);
  };
  auto finish = [&](const XItem& at, char* lds0, char* lds1) __attribute__((always_inline)) {
    const XArgs& x = *x_args_again();
    const XSample sm = x_sample(x, at.b);
    const int rows = sm.nq * x.G, r0 = at.tile * 32 * NW + 32 * w;
    if (!part) {
      x_store_rows<DP>(x.dq, sm.q0, x.sdq, (int64_t)at.hk * x.G * x.D, r0, sm.nq, x.G, x.D, lds0, lds1,
                       [&](int dt, int qg) { return dq[dt][qg]; });
      return;
    }
#pragma unroll
    for (int qg = 0; qg < 2; ++qg) {
      const int row = r0 + 16 * qg + c16, tok = row_token(row, x.G);
      if (row >= rows) continue;
      float* const pp =
          part + ((at.part * x.Tq + sm.q0 + tok) * x.Hq + at.hk * x.G + row - tok * x.G) * x.D + 4 * gq;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        if (16 * dt + 4 * gq < x.D) *reinterpret_cast<f32x4*>(pp + 16 * dt) = dq[dt][qg];
    }
  };

  // A workgroup's items in turn, their tiles as one sequence, as in the forward.
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
    Extra ex;
    auto load = [&](int u) __attribute__((always_inline)) {
      if (u < Load::IPW) load_k.one(rk, a.sk, kn, w, u, a.D);
      else load_v.one(rv, a.sv, vn, w, u - Load::IPW, a.D);
    };
    // At 128 columns before the first tile too, beside its loads: what it leaves is not
    // used, and a branch around it would spill 29 registers.
    if (DP == 128 || have) {
      step(now, P ? k_lds1 : k_lds0, P ? v_lds1 : v_lds0, changed && more, ex, all, load);
    } else {
      if (all)
#pragma unroll
        for (int u = 0; u < 2 * Load::IPW; ++u) load(u);
      load_rows(seq.item(seq.at, order), ex);
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (changed) {
      // through the wave's part of the consumed stage; the stores end beside the
      // next item's first tile
      char* const lds0 = (P ? k_lds1 : k_lds0) + w * Load::IPW * 1024;
      char* const lds1 = (P ? v_lds1 : v_lds0) + w * Load::IPW * 1024;
      if (have) finish(seq.item(seq.cur, order), lds0, lds1);
      const XItem at = seq.item(seq.at, order);
      seq.cur = seq.at;
      if (more) {
        row_stats(ex, lds0);
        const XTurn<DP> rows(x_lane_again());
        rows.turn(qop, lds0, lds1);
        rows.turn(doop, lds0, lds1);
        const bool one = seq.one_tile(order);   // uniform
        if (one) ndl = -tile_delta(seq.bits, kn, vn);
        put_stats(at, one ? seq.bits != 0 : at.part == 0);   // where delta is known
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) dq[dt][0] = dq[dt][1] = f32x4{};
    }
    have = true;
    return more;
  };
  while (iter(std::integral_constant<int, 0>{}) && iter(std::integral_constant<int, 1>{})) {
  }
}

// ---------------------------------------------------------------------------
// dK, dV
// ---------------------------------------------------------------------------
// part: fp32 [dK, dV][split][token][Hk][D], null with one split.
template <int DP>
__global__ __launch_bounds__(256, 2) void xattn_dkdv_kernel(const XArgs a, const float* __restrict__ aux,
                                                            const XOrder order, float* __restrict__ part) {
  constexpr int NW = 4, ROWB = DP * 2, CPR = DP / 8, KS = DP / 16, DT = DP / 16;
  constexpr int TILEB = kRowTile * ROWB, RPI = 1024 / ROWB, IPW = TILEB / 1024 / NW, VIPW = kBwdKeys * ROWB / 1024 / NW;
  __shared__ __attribute__((aligned(1024))) char q_lds0[TILEB];
  __shared__ __attribute__((aligned(1024))) char q_lds1[TILEB];
  __shared__ __attribute__((aligned(1024))) char o_lds0[TILEB];
  __shared__ __attribute__((aligned(1024))) char o_lds1[TILEB];
  __shared__ __attribute__((aligned(1024))) char a_lds0[2048];
  __shared__ __attribute__((aligned(1024))) char a_lds1[2048];
  __shared__ __attribute__((aligned(1024))) char vblk_lds[kBwdKeys * ROWB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g = lane >> 5, c16 = lane & 15, gq = lane >> 4;

  if (a.zero_rest) {
    x_clear_rest(a.cuk, a.B, a.Tk, a.Hk * a.D, a.dk, a.sdk);
    x_clear_rest(a.cuk, a.B, a.Tk, a.Hk * a.D, a.dv, a.sdv);
  }
  const XItems items = x_items((unsigned)a.B * order.tiles * order.splits * (unsigned)a.Hk);
  if (items.first >= items.end) return;
  const XItem at = x_item(items.first, (unsigned)a.B, order);
  const unsigned kt = at.tile, sp = at.part;
  const int hk = at.hk;
  const XSample sm = x_sample(a, at.b);
  const int key0 = (int)kt * kBwdKeys;
  if (key0 >= sm.nk) return;   // uniform over the workgroup

  // Steps: the 32-token tiles of each head of the group; this split's share.
  const int ttiles = (sm.nq + kRowTile - 1) / kRowTile, all = ttiles * a.G;
  const int per = (all + (int)order.splits - 1) / (int)order.splits;
  const int s_begin = min((int)sp * per, all), s_end = min(s_begin + per, all);

  f32x4 dk[DT][2], dv[DT][2];   // [dt][kg]: lane holds X^T[16 dt + 4 gq + (0..3)][key 32 w + 16 kg + c16]
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dk[dt][0] = dk[dt][1] = dv[dt][0] = dv[dt][1] = f32x4{};

  if (s_begin < s_end) {
    const __bf16* const kb = static_cast<const __bf16*>(a.k) + sm.k0 * a.sk + hk * a.D;
    bf16x8 kop[KS];
    {
      const __bf16* kp = kb + (int64_t)min(key0 + 32 * w + l32, sm.nk - 1) * a.sk + 8 * g;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        kop[ks] = bf16x8{};
        if (16 * ks + 8 * g < a.D) kop[ks] = *reinterpret_cast<const bf16x8*>(kp + 16 * ks);
      }
    }
    int qoff[IPW], ooff[IPW];
#pragma unroll
    for (int u = 0; u < IPW; ++u) {
      const int r = (w * IPW + u) * RPI + lane / CPR, c = (lds_off<CPR>(r, lane % CPR) >> 4) & (CPR - 1);
      qoff[u] = c < a.D / 8 ? r * a.sq * 2 + 16 * c : kXOut;
      ooff[u] = c < a.D / 8 ? r * a.sdo * 2 + 16 * c : kXOut;
    }
    {   // the workgroup's V rows (rows past the sample's keys read zeros)
      const int left = min(sm.nk - key0, kBwdKeys);
      const __amdgpu_buffer_rsrc_t rv = buffer_rsrc(
          static_cast<const __bf16*>(a.v) + (sm.k0 + key0) * a.sv + hk * a.D, (left - 1) * a.sv * 2 + 2 * a.D);
#pragma unroll
      for (int u = 0; u < VIPW; ++u) {
        const int r = (w * VIPW + u) * RPI + lane / CPR, c = (lds_off<CPR>(r, lane % CPR) >> 4) & (CPR - 1);
        buffer_load_lds16(rv, vblk_lds + (w * VIPW + u) * 1024, c < a.D / 8 ? r * a.sv * 2 + 16 * c : kXOut);
      }
    }
    const char* const vrow = vblk_lds + 32 * w * ROWB;   // this wave's keys
    // LDS offsets, the swizzle's steps by exclusive or as in the dQ pass.
    const int roff0 = lds_off<CPR>(l32, g);
    const int rtr0 = lds_off<CPR>(8 * (gq & 1) + 4 * (gq >> 1) + (c16 >> 2), (c16 & 3) >> 1) + 8 * (c16 & 1);
    // Step i: 32 rows of Q and dO and their statistics (rows past the sample read zeros).
    const __bf16* const qb = static_cast<const __bf16*>(a.q) + sm.q0 * a.sq + hk * a.G * a.D;
    const __bf16* const ob = static_cast<const __bf16*>(a.dout) + sm.q0 * a.sdo + hk * a.G * a.D;
    auto load_step = [&](int head, int tt, char* qd, char* od, char* ad) __attribute__((always_inline)) {
      const int t0 = tt * kRowTile, left = min(sm.nq - t0, kRowTile);
      const __amdgpu_buffer_rsrc_t rq = buffer_rsrc(qb + (int64_t)t0 * a.sq + head * a.D, (left - 1) * a.sq * 2 + 2 * a.D);
      const __amdgpu_buffer_rsrc_t ro = buffer_rsrc(ob + (int64_t)t0 * a.sdo + head * a.D, (left - 1) * a.sdo * 2 + 2 * a.D);
#pragma unroll
      for (int u = 0; u < IPW; ++u) {
        buffer_load_lds16(rq, qd + (w * IPW + u) * 1024, qoff[u]);
        buffer_load_lds16(ro, od + (w * IPW + u) * 1024, ooff[u]);
      }
      if (w == 0) {
        const float* const st = aux + sm.stat0 + (hk * a.G + head) * sm.hstep + t0;
        buffer_load_lds16(buffer_rsrc(st, left * 4), ad, 16 * lane);
        buffer_load_lds16(buffer_rsrc(st + a.Tq * a.Hq, left * 4), ad + 1024, 16 * lane);
      }
    };
    const float c2 = a.scale * kLog2e;
    auto step = [&](const char* qt_lds, const char* ot_lds, const char* at_lds) __attribute__((always_inline)) {
      const float* const a_pl = reinterpret_cast<const float*>(at_lds) + 4 * g;
      f32x16 s = f32x16{}, dp;
#pragma unroll
      for (int x = 0; x < 4; ++x) {   // dP - delta directly: start at -delta
        const f32x4 y = *reinterpret_cast<const f32x4*>(a_pl + 256 + 8 * x);
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[4 * x + e] = y[e];
      }
      // S and dP in turn, operands read kAhead pairs of products before their use. The
      // order is held at 128 columns, where two waves a SIMD are to cover each other
      // (77,060 rows, 512 keys, 24 heads: 920 -> 875 us); at 64 there are three, and
      // the compiler's own order is the faster one (192 us against 201).
      constexpr int kAhead = 3, kPre = 3;
      // Likewise a wave in its vector work goes before one in its products (856 -> 830;
      // the other way round 845; at 64 188 -> 195, so not there).
      auto hold = []() __attribute__((always_inline)) {
        if constexpr (DP == 128) pin_order();
      };
      auto vector_first = [](bool on) __attribute__((always_inline)) {
        if constexpr (DP == 128) on ? __builtin_amdgcn_s_setprio(1) : __builtin_amdgcn_s_setprio(0);
      };
      int ro = roff0, rt = rtr0;
      if constexpr (DP == 128) {   // at 64 the offsets fit into registers of their own
        pin_value(ro);
        pin_value(rt);
      }
      bf16x8 op[3 * kAhead];
      auto read_ops = [&](int ks) __attribute__((always_inline)) {
        bf16x8* const to = op + 3 * (ks % kAhead);
        to[0] = *reinterpret_cast<const bf16x8*>(qt_lds + (ro ^ (32 * ks)));
        to[1] = *reinterpret_cast<const bf16x8*>(ot_lds + (ro ^ (32 * ks)));
        to[2] = *reinterpret_cast<const bf16x8*>(vrow + (ro ^ (32 * ks)));
      };
#pragma unroll
      for (int ks = 0; ks < kAhead; ++ks) read_ops(ks);
      vector_first(false);
      hold();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8* const x = op + 3 * (ks % kAhead);
        s = mfma32(x[0], kop[ks], s);
        dp = mfma32(x[1], x[2], dp);
        if (ks + kAhead < KS) read_ops(ks + kAhead);
        hold();
      }
      vector_first(true);
      auto read_tr = [&](int dt) __attribute__((always_inline)) {
        bf16x8* const to = op + 2 * (dt % kPre);
        const int off = rt ^ (32 * dt);
        const s16x4 o_lo = lds_read_tr16(ot_lds + off), o_hi = lds_read_tr16(ot_lds + off + 16 * ROWB);
        const s16x4 q_lo = lds_read_tr16(qt_lds + off), q_hi = lds_read_tr16(qt_lds + off + 16 * ROWB);
        const s16x8 o8 = {o_lo[0], o_lo[1], o_lo[2], o_lo[3], o_hi[0], o_hi[1], o_hi[2], o_hi[3]};
        const s16x8 q8 = {q_lo[0], q_lo[1], q_lo[2], q_lo[3], q_hi[0], q_hi[1], q_hi[2], q_hi[3]};
        to[0] = __builtin_bit_cast(bf16x8, o8);
        to[1] = __builtin_bit_cast(bf16x8, q8);
      };
#pragma unroll
      for (int dt = 0; dt < kPre; ++dt) read_tr(dt);
      u32x4 pp[2], pd[2];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const f32x4 ls = *reinterpret_cast<const f32x4*>(a_pl + 8 * x);
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const int i = 4 * x + e;
          const float p0 = fast_exp2(__builtin_fmaf(s[i], c2, -ls[e]));
          const float p1 = fast_exp2(__builtin_fmaf(s[i + 1], c2, -ls[e + 1]));
          const int r = (i >> 2) & 1, c = ((i & 3) >> 1) + 2 * (i >> 3);
          pp[r][c] = pack_bf16x2(p0, p1);
          pd[r][c] = pack_bf16x2(p0 * dp[i], p1 * dp[i + 1]);
        }
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const auto r0 = __builtin_amdgcn_permlane16_swap(pp[0][v], pp[1][v], false, false);
        pp[0][v] = r0[0];
        pp[1][v] = r0[1];
        const auto r1 = __builtin_amdgcn_permlane16_swap(pd[0][v], pd[1][v], false, false);
        pd[0][v] = r1[0];
        pd[1][v] = r1[1];
      }
      vector_first(false);
      hold();
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const bf16x8* const x = op + 2 * (dt % kPre);
#pragma unroll
        for (int kg = 0; kg < 2; ++kg) {
          dv[dt][kg] = mfma16(x[0], __builtin_bit_cast(bf16x8, pp[kg]), dv[dt][kg]);
          dk[dt][kg] = mfma16(x[1], __builtin_bit_cast(bf16x8, pd[kg]), dk[dt][kg]);
        }
        if (dt + kPre < DT) read_tr(dt + kPre);
        hold();
      }
      vector_first(true);
    };
    int head = s_begin / ttiles, tt = s_begin - head * ttiles;
    auto advance = [&]() __attribute__((always_inline)) {
      if (++tt == ttiles) tt = 0, ++head;
    };
    auto iter = [&](int i, auto par, auto used) __attribute__((always_inline)) {
      constexpr int P = decltype(par)::value;
      advance();
      if (i + 1 < s_end) load_step(head, tt, P ? q_lds0 : q_lds1, P ? o_lds0 : o_lds1, P ? a_lds0 : a_lds1);
      if constexpr (decltype(used)::value) step(P ? q_lds1 : q_lds0, P ? o_lds1 : o_lds0, P ? a_lds1 : a_lds0);
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
    };
    load_step(head, tt, q_lds0, o_lds0, a_lds0);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    auto walk = [&](auto used) __attribute__((always_inline)) {
      int i = s_begin;
      for (; i + 1 < s_end; i += 2) {
        iter(i, std::integral_constant<int, 0>{}, used);
        iter(i + 1, std::integral_constant<int, 1>{}, used);
      }
      if (i < s_end) iter(i, std::integral_constant<int, 0>{}, used);
    };
    // a wave without keys in use loads its part of the steps and leaves the matrix
    // cores to the others
    const int mine = key0 + 32 * w + l32;
    if (__ballot(mine < sm.nk && (!a.mask || a.mask[sm.k0 + mine]))) walk(std::true_type{});
    else walk(std::false_type{});
  }

#pragma unroll
  for (int kg = 0; kg < 2; ++kg) {
    const int key = key0 + 32 * w + 16 * kg + c16;
    if (key >= sm.nk) continue;
    const bool used = !a.mask || a.mask[sm.k0 + key];
    const int64_t tok = sm.k0 + key;
    float* const pk = part + ((sp * a.Tk + tok) * a.Hk + hk) * a.D + 4 * gq;
    float* const pv = pk + order.splits * a.Tk * a.Hk * a.D;
    __bf16* const ok = static_cast<__bf16*>(a.dk) + tok * a.sdk + hk * a.D + 4 * gq;
    __bf16* const ov = static_cast<__bf16*>(a.dv) + tok * a.sdv + hk * a.D + 4 * gq;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      if (16 * dt + 4 * gq >= a.D) continue;
      const f32x4 x = used ? dk[dt][kg] * a.scale : f32x4{}, y = used ? dv[dt][kg] : f32x4{};
      if (part) {
        *reinterpret_cast<f32x4*>(pk + 16 * dt) = x;
        *reinterpret_cast<f32x4*>(pv + 16 * dt) = y;
      } else {
        *reinterpret_cast<bf16x4*>(ok + 16 * dt) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
        *reinterpret_cast<bf16x4*>(ov + 16 * dt) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
      }
    }
  }
}

// ---------------------------------------------------------------------------
// join: out[token][row of the token's heads] = the sum of the parts, in order, of up
// to three tensors in one launch. Four elements a thread; tokens of no sample are
// left as they are.
// ---------------------------------------------------------------------------
struct Join {
  const float* part;   // [parts][T][width]
  int parts;
  int64_t T;
  int width;
  void* out;
  int stride;
  const int32_t* cu;   // [B + 1], or null
  int N;               // most tokens of a sample
};
__global__ __launch_bounds__(256) void xattn_sum_kernel(const Join j0, const Join j1, const Join j2, int B) {
  const Join j = blockIdx.y == 0 ? j0 : blockIdx.y == 1 ? j1 : j2;
  const int64_t total = j.T * j.width, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= total) return;
  const int64_t tok = i / j.width;
  if (j.cu && !in_sample(j.cu, j.T, B, j.N, tok)) return;
  f32x4 x = f32x4{};
#pragma unroll 4
  for (int s = 0; s < j.parts; ++s) x += *reinterpret_cast<const f32x4*>(j.part + s * total + i);
  *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(j.out) + tok * j.stride + (i - tok * j.width)) =
      bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
}

int64_t dq_tiles(const XArgs& a) { return ((int64_t)a.Nq * a.G + 32 * kDqWaves - 1) / (32 * kDqWaves); }
int64_t dq_groups(const XArgs& a) { return (int64_t)a.B * a.Hk * dq_tiles(a); }
int64_t dkdv_groups(const XArgs& a) {
  return (int64_t)a.B * a.Hk * (((int64_t)a.Nk + kBwdKeys - 1) / kBwdKeys);
}
// As many parts as fit the chip at once, of four tiles or eight steps at least: at 300
// queries and keys, 8 heads of 64, half of that takes dQ from 14.9 to 13.0 us and dK/dV
// from 14.5 to 11.7, and their join adds 7.
int dq_splits(const XArgs& a) {
  const int64_t groups = dq_groups(a), tiles = ((int64_t)a.Nk + kXKeys - 1) / kXKeys;
  return groups == 0 ? 1 : (int)std::max<int64_t>(1, std::min(x_resident(x_padded(a), kDqWaves) / groups, tiles / 4));
}
int dkdv_splits(const XArgs& a) {
  const int64_t groups = dkdv_groups(a), steps = (int64_t)a.G * (((int64_t)a.Nq + kRowTile - 1) / kRowTile);
  return groups == 0 ? 1 : (int)std::max<int64_t>(1, std::min(x_resident(x_padded(a), 4) / groups, steps / 8));
}
size_t aux_bytes(const XArgs& a) { return ((size_t)a.Tq * a.Hq * 2 * sizeof(float) + 255) / 256 * 256; }
size_t dq_part(const XArgs& a) {
  const int n = dq_splits(a);
  return n > 1 ? (size_t)n * a.Tq * a.Hq * a.D * sizeof(float) : 0;
}
size_t dkdv_part(const XArgs& a) {
  const int n = dkdv_splits(a);
  return n > 1 ? (size_t)n * a.Tk * a.Hk * a.D * 2 * sizeof(float) : 0;
}

template <int DP>
void launch_dq(const XArgs& a, float* aux, int splits, float* part, hipStream_t s) {
  const XOrder order{head_group(a), (unsigned)dq_tiles(a), (unsigned)splits};
  const int64_t items = dq_groups(a) * splits;
  const dim3 grid((unsigned)(std::min<int64_t>(std::max<int64_t>(items, 1), x_resident(DP, kDqWaves)) + 7) / 8 * 8);
  TraceScope ts_(s, "xattn_dq", DP);
  hipLaunchKernelGGL((xattn_dq_kernel<DP>), grid, dim3(64 * kDqWaves), 0, s, a, aux, order, part);
}
template <int DP>
void launch_dkdv(const XArgs& a, const float* aux, int splits, float* part, hipStream_t s) {
  const XOrder order{head_group(a), (unsigned)(((int64_t)a.Nk + kBwdKeys - 1) / kBwdKeys), (unsigned)splits};
  TraceScope ts_(s, "xattn_dkdv", DP);
  const dim3 grid((unsigned)(std::max<int64_t>(dkdv_groups(a) * splits, 1) + 7) / 8 * 8);
  hipLaunchKernelGGL((xattn_dkdv_kernel<DP>), grid, dim3(256), 0, s, a, aux, order, part);
}
void launch_sums(const Join* j, int n, int B, hipStream_t s) {
  int64_t most = 0;
  for (int i = 0; i < n; ++i) most = std::max(most, j[i].T * j[i].width);
  if (most == 0) return;
  TraceScope ts_(s, "xattn_sum");
  hipLaunchKernelGGL(xattn_sum_kernel, dim3((unsigned)((most / 4 + 255) / 256), (unsigned)n), dim3(256), 0, s, j[0],
                     j[n > 1 ? 1 : 0], j[n > 2 ? 2 : 0], B);
}

}  // namespace

bool xattn_bwd_launchable(const XArgs& a) {
  constexpr int64_t kMost = (int64_t)1 << 24;   // workgroups of 256 threads
  const int64_t sums = std::max(dq_part(a) > 0 ? a.Tq * a.Hq : 0, dkdv_part(a) > 0 ? a.Tk * a.Hk : 0) * a.D;
  return (dkdv_groups(a) + 7) / 8 * 8 < kMost && (sums / 4 + 255) / 256 < kMost;
}

size_t xattn_bwd_workspace(const XArgs& a) { return aux_bytes(a) + dq_part(a) + dkdv_part(a); }

hipError_t launch_xattn_bwd(const XArgs& a, void* workspace, hipStream_t s) {
  float* const aux = static_cast<float*>(workspace);
  float* const qpart = reinterpret_cast<float*>(static_cast<char*>(workspace) + aux_bytes(a));
  float* const kpart = qpart + dq_part(a) / sizeof(float);
  Join joins[3];
  int n = 0;
  if (dq_groups(a) > 0 || (a.zero_rest && a.Tq > 0)) {
    const int splits = dq_splits(a);
    float* const p = splits > 1 ? qpart : nullptr;
    a.D <= 64 ? launch_dq<64>(a, aux, splits, p, s) : launch_dq<128>(a, aux, splits, p, s);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (p) joins[n++] = Join{p, splits, a.Tq, a.Hq * a.D, a.dq, a.sdq, a.cuq, a.Nq};
  }
  if (dkdv_groups(a) > 0 || (a.zero_rest && a.Tk > 0)) {
    const int splits = dkdv_splits(a);
    float* const p = splits > 1 ? kpart : nullptr;
    a.D <= 64 ? launch_dkdv<64>(a, aux, splits, p, s) : launch_dkdv<128>(a, aux, splits, p, s);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (p) {
      joins[n++] = Join{p, splits, a.Tk, a.Hk * a.D, a.dk, a.sdk, a.cuk, a.Nk};
      joins[n++] = Join{p + (size_t)splits * a.Tk * a.Hk * a.D, splits, a.Tk, a.Hk * a.D, a.dv, a.sdv, a.cuk, a.Nk};
    }
  }
  if (n > 0) launch_sums(joins, n, a.B, s);
  return hipGetLastError();
}

}  // namespace ut
