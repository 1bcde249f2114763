// Attention over a cache with few rows a key head (a token, or a small tree, times the
// heads of the group: up to 32), on gfx950: what serving does for every token. Keys and
// values pass once and bound it; the products are a twentieth of the time.
//
// A workgroup of four waves takes a share of the tiles of all samples and groups of key
// heads (cache_share), a wave every fourth 32 keys of an item, and they run without
// barriers until the item's end. Of long caches a group is four heads, which a wave takes
// in turn: the memory gives some heads less (of 8 x 256 bytes a token, heads 1 and 5:
// 48 us where the others took 40), and so every wave has its part of them. To keep enough
// bytes under way (two microseconds of the chip's bandwidth are some 10 MB, 40 KB a CU) a
// wave loads four steps of 32 keys ahead: K into registers, in the operand's layout, V
// into its own LDS by direct loads. One token on four caches of 16,500 slots, 32 heads on
// 8 of 128, 230 MB: 44 us, 5.2 TB/s (the last-level cache holds some of it from call to
// call; with other caches each time 4.3). S^T = K Q^T and
// O^T += V^T P^T on 16x16x32 bf16 MFMA: the contraction over the keys is taken in the
// order that the scores' layout leaves (keys 4 g .. of both 16-key tiles in lane
// group g), so P needs no exchange, and V's transposing reads follow it. The softmax
// keeps a running maximum and sum; P is rounded to bf16 for the second product (half a
// step, 2^-8 relative at most, as V's own), everything else is fp32.
//
// At an item's end the waves' results meet in LDS. A whole item is finished there;
// of others the workgroup's part goes to the workspace, and a second launch joins the
// parts in a fixed order. No atomics: equal results on every run.
#include <algorithm>
#include <type_traits>

#include "xattn_util.h"

namespace ut {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kStages = 4;   // steps of a wave under way or at work

// RG: groups of 16 rows; HG: key heads of an item.
template <int DP, int RG, int HG>
__global__ __launch_bounds__(256, 1) void cache_one_kernel(const XArgs a, const CacheParts parts, const CacheWeights wt,
                                                           const bool weights_here) {
  constexpr int ROWB = DP * 2, CPR = DP / 8, KS = DP / 32, DT = DP / 16, STEPB = 32 * ROWB, VI = STEPB / 1024;
  __shared__ __attribute__((aligned(1024))) char v_lds0[4 * STEPB];
  __shared__ __attribute__((aligned(1024))) char v_lds1[4 * STEPB];
  __shared__ __attribute__((aligned(1024))) char v_lds2[4 * STEPB];
  __shared__ __attribute__((aligned(1024))) char v_lds3[4 * STEPB];
  static_assert(RG * HG <= 4, "a stage for the results of every 16 rows");
  __shared__ float2 ml_lds[HG][4][16 * RG];
  __shared__ float lse_lds[HG][16 * RG];
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, gq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // 16 rows of a wave's O, in its part of stage i, which is read by then: 16-byte pieces,
  // swizzled by row.
  static_assert(16 * DP * 4 == STEPB, "a step's values and 16 rows of O take the same room");
  auto o_lds = [&](int i, int wave, int r, int d) __attribute__((always_inline)) {
    char* const stage = i == 0 ? v_lds0 : i == 1 ? v_lds1 : i == 2 ? v_lds2 : v_lds3;
    return reinterpret_cast<f32x4*>(stage + wave * STEPB + r * DP * 4 + ((d / 4 ^ r) << 4));
  };
  const int rows = a.Nq * a.G;
  const float c2 = a.scale * kLog2e;
  CacheShare share = cache_share(a, (int)blockIdx.x, (int)gridDim.x, a.Hk / HG, blockIdx.x == 0 && w == 0 ? parts.cuts : nullptr);

  // V of a step: instruction i writes 1 KB of rows, this lane's row and column in it.
  int v_row[VI], v_off[VI];
#pragma unroll
  for (int i = 0; i < VI; ++i) {
    v_row[i] = i * (1024 / ROWB) + lane / CPR;
    const int c = swz_off<CPR>(v_row[i], lane % CPR) / 16 % CPR;
    v_off[i] = 8 * c < a.D ? v_row[i] * a.sv * 2 + 16 * c : kXOut;
  }
  int k_off[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_off[ks] = 32 * ks + 8 * gq < a.D ? c16 * a.sk * 2 + 64 * ks + 16 * gq : kXOut;
  // V^T's operand: rows 4 gq + 0..3 and 16 further on, columns 16 dt + 4 (c16 & 3) ..
  int v_tr[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    v_tr[dt] = w * STEPB + swz_off<CPR>(4 * gq + (c16 >> 2), 2 * dt + ((c16 & 3) >> 1)) + 8 * (c16 & 1);

  for (bool first = true; share.items > 0; first = false) {   // uniform over the workgroup
    const int b = share.b, hk = share.g * HG;   // the first of its heads
    const XSample sm = x_sample<kSeeCache>(a, b);
    const XSpan span = x_span<kSeeCache>(a, sm, 0, rows);
    const int off = sm.nk - sm.nq, t0 = first ? share.t0 : 0, t1 = share.items == 1 ? share.t1 : span.count;
    const int part = first ? share.part : 0;
    const bool all_here = t0 == 0 && t1 == span.count;
    auto key_of = [&](int s) __attribute__((always_inline)) {
      const int i = s >> 1;
      return kXKeys * (i + (i >= span.first ? span.skip : 0)) + 32 * (s & 1);
    };
    // the wave's steps: s0, 4 further on each, below s_end (the last tile's second half may be
    // behind the slots in use)
    const int s0 = 2 * t0 + w, s_end = 2 * t1 - (t1 > t0 && key_of(2 * t1 - 1) >= sm.nk ? 1 : 0);
    const __bf16* const kb = static_cast<const __bf16*>(a.k) + sm.k0 * a.sk + hk * a.D;
    const __bf16* const vb = static_cast<const __bf16*>(a.v) + sm.k0 * a.sv + hk * a.D;
    bf16x8 kop[kStages][2][KS];
    // Keys s of head h; slots that the sample lacks read zeros, and so do values of
    // slots that no row sees.
    auto load = [&](int s, int h, bf16x8 (&k)[2][KS], char* v) __attribute__((always_inline)) {
      if (s >= s_end) return;   // uniform
      const int key = key_of(s), left = min(sm.nk - key, 32);
      const __amdgpu_buffer_rsrc_t rk = buffer_rsrc(kb + (int64_t)key * a.sk + h * a.D, ((left - 1) * a.sk + a.D) * 2);
      const __amdgpu_buffer_rsrc_t rv = buffer_rsrc(vb + (int64_t)key * a.sv + h * a.D, ((left - 1) * a.sv + a.D) * 2);
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)   // kXOut and 16 slots further on is past the range too
          k[kt][ks] = __builtin_bit_cast(   // in the vector offset: the range's check leaves scalar ones out
              bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rk, k_off[ks] + 16 * kt * a.sk * 2, 0, kXStream));
      char* const to = v + w * STEPB;
      if ((key >= span.lo && key + 32 <= span.hi) || key + 32 <= span.send) {   // uniform
#pragma unroll
        for (int i = 0; i < VI; ++i) buffer_load_lds16(rv, to + i * 1024, v_off[i]);
      } else {
#pragma unroll
        for (int i = 0; i < VI; ++i) {
          const int at = key + v_row[i];
          const bool in = ((at >= span.lo) & (at < span.hi)) | (at < span.send);
          buffer_load_lds16(rv, to + i * 1024, in ? v_off[i] : kXOut);
        }
      }
    };
    bf16x8 qop[HG][RG][KS];
    RowWindow<kSeeCache> see[RG];
    float m[HG][RG], l[HG][RG];
    f32x4 o[HG][RG][DT];
#pragma unroll
    for (int rg = 0; rg < RG; ++rg) {
      const int r = 16 * rg + c16, tok = row_token(min(r, rows - 1), a.G);
      see[rg].open(a, sm, b, r);
#pragma unroll
      for (int h = 0; h < HG; ++h) {
        const __bf16* const qp = static_cast<const __bf16*>(a.q) + (sm.q0 + tok) * a.sq +
                                 ((hk + h) * a.G + min(r, rows - 1) - tok * a.G) * a.D + 8 * gq;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          qop[h][rg][ks] = bf16x8{};
          if (r < rows && 32 * ks + 8 * gq < a.D) qop[h][rg][ks] = *reinterpret_cast<const bf16x8*>(qp + 32 * ks);
        }
        m[h][rg] = -INFINITY;
        l[h][rg] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[h][rg][dt] = f32x4{};
      }
    }
    // Steps in order: the heads of 32 keys, then the next keys. Step i of four from keys s on.
    auto keys_of = [](int s, int i) __attribute__((always_inline)) { return s + 4 * (i / HG); };
    load(keys_of(s0, 0), 0, kop[0], v_lds0);
    load(keys_of(s0, 1), 1 % HG, kop[1], v_lds1);
    load(keys_of(s0, 2), 2 % HG, kop[2], v_lds2);
    // The queries' rows, loaded first, are waited for here: in the loop the compiler would
    // wait for every load under way.
#pragma unroll
    for (int h = 0; h < HG; ++h)
#pragma unroll
      for (int rg = 0; rg < RG; ++rg)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) pin_value(qop[h][rg][ks]);
    auto step = [&](int s, auto head, bf16x8 (&k)[2][KS], const char* v) __attribute__((always_inline)) {
      constexpr int h = decltype(head)::value;
      const int key = key_of(s);
      const int end = a.tree ? off : off + 1, last = a.tree ? off + sm.nq : off + sm.nq - 1;
      const bool whole = (key >= last - a.left && key + 32 <= end) || key + 32 <= min(a.sinks, end);   // uniform
      bf16x8 pop[RG];
#pragma unroll
      for (int rg = 0; rg < RG; ++rg) {
        f32x4 x[2] = {f32x4{}, f32x4{}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) x[kt] = mfma16(k[kt][ks], qop[h][rg][ks], x[kt]);
        x[0] *= c2, x[1] *= c2;
        if (!whole) {
          unsigned mine = see[rg].bits(a, key) & bits32_from_to(0, sm.nk - key);
          mine >>= 4 * gq;
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[kt][e] = mine >> (16 * kt + e) & 1 ? x[kt][e] : -INFINITY;
        }
        if (a.scores && 16 * rg + c16 < rows) {
          float* const to = parts.scores + (((int64_t)b * a.Hk + hk + h) * rows + 16 * rg + c16) * score_keys(a) + key + 4 * gq;
          *reinterpret_cast<f32x4*>(to) = x[0];
          *reinterpret_cast<f32x4*>(to + 16) = x[1];
        }
        float mx = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                         fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
        const float to = fmaxf(m[h][rg], quad_max(mx));
        const float ref = to == -INFINITY ? 0.f : to, alpha = fast_exp2(m[h][rg] - ref);
        float sum = 0.f, p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = fast_exp2(x[e >> 2][e & 3] - ref);
          sum += p[e];
        }
        m[h][rg] = to;
        l[h][rg] = l[h][rg] * alpha + sum;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[h][rg][dt] *= alpha;
        const u32x4 y = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
        pop[rg] = __builtin_bit_cast(bf16x8, y);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const s16x4 lo = lds_read_tr16(v + v_tr[dt]), hi = lds_read_tr16(v + v_tr[dt] + 16 * ROWB);
        const s16x8 v8 = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
        for (int rg = 0; rg < RG; ++rg) o[h][rg][dt] = mfma16(__builtin_bit_cast(bf16x8, v8), pop[rg], o[h][rg][dt]);
      }
    };
    // Stage by stage, the fourth step ahead loaded while one is worked on. Loads return in
    // order, 2 KS + VI a step, so a step's are there when only the later steps' are under
    // way (the scores' stores count too: then the wait is for a little more).
    auto wait = [](auto steps) __attribute__((always_inline)) {
      constexpr int n = decltype(steps)::value * (2 * KS + VI);
      __builtin_amdgcn_s_waitcnt(0x0f70 | (n & 15) | (n >> 4) << 14);   // vmcnt(n)
    };
    for (int s = s0; s < s_end; s += 16 / HG) {
      auto turn = [&](auto at, bf16x8 (&k)[2][KS], const char* v, bf16x8 (&kn)[2][KS], char* vn) __attribute__((always_inline)) {
        constexpr int i = decltype(at)::value;
        if (keys_of(s, i) >= s_end) return;   // uniform
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the stage to be loaded is read
        pin_order();
        load(keys_of(s, i + 3), (i + 3) % HG, kn, vn);
        if (keys_of(s, i + 3) < s_end) wait(std::integral_constant<int, 3>{});
        else if (keys_of(s, i + 2) < s_end) wait(std::integral_constant<int, 2>{});
        else if (keys_of(s, i + 1) < s_end) wait(std::integral_constant<int, 1>{});
        else wait(std::integral_constant<int, 0>{});
        pin_order();
        step(keys_of(s, i), std::integral_constant<int, i % HG>{}, k, v);
      };
      turn(std::integral_constant<int, 0>{}, kop[0], v_lds0, kop[3], v_lds3);
      turn(std::integral_constant<int, 1>{}, kop[1], v_lds1, kop[0], v_lds0);
      turn(std::integral_constant<int, 2>{}, kop[2], v_lds2, kop[1], v_lds1);
      turn(std::integral_constant<int, 3>{}, kop[3], v_lds3, kop[2], v_lds2);
    }

    // The waves' results together.
#pragma unroll
    for (int h = 0; h < HG; ++h)
#pragma unroll
      for (int rg = 0; rg < RG; ++rg) {
        const float sum = quad_sum(l[h][rg]);
        if (gq == 0) ml_lds[h][w][16 * rg + c16] = make_float2(m[h][rg], sum);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *o_lds(h * RG + rg, w, c16, 16 * dt + 4 * gq) = o[h][rg][dt];
      }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < HG; ++h)
#pragma unroll
      for (int rg = 0; rg < RG; ++rg) {
        const int n = min(rows - 16 * rg, 16);
        for (int i = tid; i < n * (DP / 4); i += 256) {
          const int r = i / (DP / 4), d = i % (DP / 4) * 4, row = 16 * rg + r, tok = row_token(row, a.G);
          const int head = (hk + h) * a.G + row - tok * a.G;
          float M = -INFINITY, L = 0.f;
#pragma unroll
          for (int x = 0; x < 4; ++x) M = fmaxf(M, ml_lds[h][x][row].x);
          f32x4 y = f32x4{};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float2 ml = ml_lds[h][x][row];
            const float f = ml.y == 0.f ? 0.f : fast_exp2(ml.x - M);
            L += ml.y * f;
            y += *o_lds(h * RG + rg, x, r, d) * f;
          }
          const int64_t stat = ((int64_t)b * a.Hq + head) * a.Nq + tok;
          if (all_here) {
            const float inv = L == 0.f ? 0.f : 1.f / L, lse2 = M + __log2f(L);
            if (d == 0) {
              a.lse[stat] = L == 0.f ? -INFINITY : lse2 * kLn2;
              lse_lds[h][row] = L == 0.f ? INFINITY : lse2;   // no slots: P = 0
            }
            if (d < a.D)
              *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.o) + (sm.q0 + tok) * a.so + head * a.D + d) =
                  bf16x4{(__bf16)(y[0] * inv), (__bf16)(y[1] * inv), (__bf16)(y[2] * inv), (__bf16)(y[3] * inv)};
          } else {
            if (d == 0) parts.sums[part * parts.stats + stat] = make_float2(M, L);
            if (d < a.D) *reinterpret_cast<f32x4*>(parts.o + (part * parts.stats + stat) * a.D + d) = y;
          }
        }
      }
    if (weights_here) {   // uniform: the item is whole, its scores are this workgroup's
      __syncthreads();
      for (int h = 0; h < HG; ++h) {
        const float* const sc = parts.scores + ((int64_t)b * a.Hk + hk + h) * rows * score_keys(a);
        const int64_t to = ((int64_t)b * a.Hk + hk + h) * a.Nk;
        for (int key = tid; key < a.Nk; key += 256) {
          float sum = 0.f;
          if (key < sm.nk && span.has(key / kXKeys))
            for (int r = 0; r < rows; ++r) sum += fast_exp2(sc[r * score_keys(a) + key] - lse_lds[h][r]);
          wt.out[to + key] = (wt.in ? wt.in[to + key] : 0.f) + sum;
        }
      }
    }
    if (++share.g == a.Hk / HG) share.g = 0, ++share.b;
    if (--share.items > 0) __syncthreads();   // before the stages are loaded again
  }
}

}  // namespace

hipError_t launch_cache_one(const XArgs& a, const CacheParts& parts, const CacheWeights& w, bool weights_here, hipStream_t s) {
  const int rows = a.Nq * a.G;
  const dim3 grid(kCacheOneGroups);
  TraceScope ts_(s, "cache_one", x_padded(a), parts.heads);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, parts, w, weights_here); };
  if (parts.heads == 4) a.D <= 64 ? launch(cache_one_kernel<64, 1, 4>) : launch(cache_one_kernel<128, 1, 4>);
  else if (rows <= 16) a.D <= 64 ? launch(cache_one_kernel<64, 1, 1>) : launch(cache_one_kernel<128, 1, 1>);
  else a.D <= 64 ? launch(cache_one_kernel<64, 2, 1>) : launch(cache_one_kernel<128, 2, 1>);
  return hipGetLastError();
}

}  // namespace ut
