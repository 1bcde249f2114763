// What a cache of keys and values needs beside the attention that reads it, on
// gfx950: the end of a split attention call, the attention weight that every slot
// receives, summed over the queries, and eviction of the slots that received least.
//
// Weights: out[b, hk, j] = in[b, hk, j] + sum over the tokens t and the heads h of the
// group of P = exp(S scale - LSE). The attention knows a row's LSE only at its end, so
// this pass forms the scores again (of few rows the attention leaves them instead): a
// workgroup keeps the rows of the group in LDS, up to 192 at once, and a wave takes tiles
// of 32 keys: whole rows into its own part of LDS by direct loads (as operands, straight
// from memory, an instruction touches 32 rows: twice the time), from there into
// registers, the next tile's loads beside the products; S = Q K^T on 32x32x16 bf16 MFMA
// in the layout where a lane holds one key, so that the sum over the rows is the lane's
// own but for one exchange. fp32 throughout, a fixed order: no atomics. 192 rows on four
// caches of 8,300 slots, 8 key heads of 128: 39 us with the joins of the attention's parts
// (28 alone), vector work and the latency of a workgroup's start and few steps.
//
// Eviction: of a row of weights the middle slots (behind the sinks, before the recent
// ones) are searched by value for the smallest weight that stays: its order as an
// unsigned number is bracketed, and the next number is taken where the counts at the
// ends would have it on a straight line, every fourth time in the middle (that number
// grows with the float's logarithm): some five steps leave 64 slots, which are ranked
// against each other, where bisection took over twenty. A workgroup holds the row in
// registers, and longer ones in LDS too (up to 69,632 slots; beyond they are read again), a
// step is a compare and an add a register and one barrier. Then ballots give every kept slot its place in ascending order, equal
// weights the lowest slots first, and a second launch copies the rows of K and V.
#include <algorithm>
#include <type_traits>

#include "xattn_util.h"

namespace ut {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// How the rows of a cache call lie in its items: tiles of `per` rows of a key head.
struct CacheRows {
  int tiles, per;
};
// Parts of sample b's row `row` of key head hk, and its place in the statistics.
__device__ inline int row_parts(const XArgs& a, const CacheParts& parts, const CacheRows& at, int b, int hk, int row) {
  const int g = parts.heads > 0 ? hk / parts.heads : hk * at.tiles + row / at.per;
  return cache_parts(parts.cuts[0], parts.cuts[1 + b], cache_tiles(a, b), g);
}
__device__ inline int64_t row_stat(const XArgs& a, int b, int hk, int row) {
  const int t = row_token(row, a.G);
  return ((int64_t)b * a.Hq + hk * a.G + row - t * a.G) * a.Nq + t;
}
// A row's LSE in log2 units (-inf: no keys) from the sums of its n parts, by `lanes`
// neighbouring lanes, this one the sub-th; parts that hold nothing are left out.
__device__ inline float part_lse(const CacheParts& parts, int64_t stat, int n, int sub, int lanes) {
  float m = -INFINITY, l = 0.f;
  auto add = [&](float mo, float lo) __attribute__((always_inline)) {
    const float to = lo == 0.f ? m : fmaxf(m, mo);
    l = (l == 0.f ? 0.f : l * fast_exp2(m - to)) + (lo == 0.f ? 0.f : lo * fast_exp2(mo - to));
    m = to;
  };
#pragma unroll 4
  for (int s = sub; s < n; s += lanes) {
    const float2 p = parts.sums[s * parts.stats + stat];
    add(p.x, p.y);
  }
  for (int x = 1; x < lanes; x <<= 1) add(__shfl_xor(m, x, 64), __shfl_xor(l, x, 64));
  return l == 0.f ? -INFINITY : m + __log2f(l);
}

// The parts of rows joined: GPR groups of 32 lanes a row take every GPR-th part, four
// columns a lane, and the groups' sums are added in LDS. Of blocks of T / 32 / GPR rows:
// `block` and, R = 2, the one a grid further on, whose loads are under way together.
template <int GPR, int T, int R = 1>
__device__ inline void join_rows(const XArgs& a, const CacheParts& parts, const CacheRows& at, int block, float4* red) {
  constexpr int kRows = T / 32 / GPR;
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5, sub = grp % GPR;
  const bool col = 4 * lane < a.D;
  int64_t r[R], tok[R];   // row [B, Hq, T], its token
  bool live[R];
  int head[R], splits[R];
#pragma unroll
  for (int y = 0; y < R; ++y) {
    r[y] = ((int64_t)block + y * (int64_t)gridDim.x) * kRows + grp / GPR;
    live[y] = r[y] < parts.stats;
    tok[y] = 0;
    head[y] = splits[y] = 0;
    if (live[y]) {
      const int64_t bh = r[y] / a.Nq;
      const int b = (int)(bh / a.Hq), t = (int)(r[y] - bh * a.Nq);
      head[y] = (int)(bh - (int64_t)b * a.Hq);
      tok[y] = (int64_t)b * a.Nq + t;
      const int hk = head[y] / a.G;
      splits[y] = row_parts(a, parts, at, b, hk, t * a.G + head[y] - hk * a.G);
    }
    if (splits[y] == 1 && parts.heads > 0) live[y] = false, splits[y] = 0;   // cache_one finishes these
  }
  // O of the first parts is loaded beside their sums, of which each lane has one.
  constexpr int kEarly = GPR == 1 ? 8 : 4;
  float4 o[R][kEarly];
  auto load = [&](int y, int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kEarly; ++u) {
      const int s = s0 + u * GPR;
      o[y][u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s < splits[y] && col)
        o[y][u] = *reinterpret_cast<const float4*>(parts.o + (s * parts.stats + r[y]) * a.D + 4 * lane);
    }
  };
  float2 mine[R];
#pragma unroll
  for (int y = 0; y < R; ++y) {
    mine[y] = make_float2(-INFINITY, 0.f);
    if (lane < splits[y]) mine[y] = parts.sums[lane * parts.stats + r[y]];
    load(y, sub);
  }
#pragma unroll
  for (int y = 0; y < R; ++y) {
    float M = mine[y].y != 0.f ? mine[y].x : -INFINITY;
    for (int s = lane + 32; s < splits[y]; s += 32) {
      const float2 p = parts.sums[s * parts.stats + r[y]];
      M = p.y != 0.f ? fmaxf(M, p.x) : M;
    }
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) M = fmaxf(M, __shfl_xor(M, m, 64));
    auto factor = [&](const float2& p) { return p.y == 0.f ? 0.f : fast_exp2(p.x - M); };   // 0: no keys in use there
    const float f_mine = factor(mine[y]);
    float L = mine[y].y * f_mine;
    for (int s = lane + 32; s < splits[y]; s += 32) {
      const float2 p = parts.sums[s * parts.stats + r[y]];
      L += p.y * factor(p);
    }
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) L += __shfl_xor(L, m, 64);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = sub; s0 < splits[y]; s0 += kEarly * GPR) {
      if (s0 != sub) load(y, s0);
#pragma unroll
      for (int u = 0; u < kEarly; ++u) {
        const int s = s0 + u * GPR;
        if (s >= splits[y]) break;
        const float f = s < 32 ? __shfl(f_mine, s, 32) : factor(parts.sums[s * parts.stats + r[y]]);
        if (f != 0.f) acc.x += o[y][u].x * f, acc.y += o[y][u].y * f, acc.z += o[y][u].z * f, acc.w += o[y][u].w * f;
      }
    }
    if constexpr (GPR > 1) {
      red[threadIdx.x] = acc;
      __syncthreads();
      if (sub == 0)
        for (int k = 1; k < GPR; ++k) {
          const float4 x = red[threadIdx.x + 32 * k];
          acc.x += x.x, acc.y += x.y, acc.z += x.z, acc.w += x.w;
        }
    }
    if (!live[y] || sub != 0) continue;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (lane == 0) a.lse[r[y]] = L == 0.f ? -INFINITY : (M + __log2f(L)) * kLn2;
    if (col) {
      const bf16x4 v = {(__bf16)(acc.x * inv), (__bf16)(acc.y * inv), (__bf16)(acc.z * inv), (__bf16)(acc.w * inv)};
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(a.o) + tok[y] * a.so + head[y] * a.D + 4 * lane) = v;
    }
  }
}

// The end of a cache call: its rows joined (the first `joins` workgroups), and with the
// scores of few rows the weights that the slots receive, a workgroup 256 slots of a key
// head; a row's maximum and sum come from its parts again, or from its LSE. The scores
// are loaded beside them.
template <int GPR, bool SPLIT>
__global__ __launch_bounds__(256) void cache_finish_kernel(const XArgs a, const CacheRows rows_at, const int joins,
                                                           const CacheParts parts, const CacheWeights wt) {
  __shared__ float4 red[256];
  if (SPLIT && (int)blockIdx.x < joins) return join_rows<GPR, 256>(a, parts, rows_at, blockIdx.x, red);
  float* const lse2 = reinterpret_cast<float*>(red);
  const unsigned at = blockIdx.x - (SPLIT ? joins : 0), chunks = (unsigned)((a.Nk + 255) / 256);
  const unsigned bh = at / chunks;
  const int b = (int)(bh / (unsigned)a.Hk), hk = (int)(bh - b * a.Hk), rows = a.Nq * a.G;
  const int key = (int)(at - bh * chunks) * 256 + threadIdx.x;
  const float* const sc = parts.scores + (int64_t)bh * rows * score_keys(a) + min(key, a.Nk - 1);
  const int64_t to = (int64_t)bh * a.Nk + key;
  constexpr int kEarly = 8;   // rows whose scores are loaded at once; what lies there may be anything
  float early[kEarly];
#pragma unroll
  for (int r = 0; r < kEarly; ++r) early[r] = sc[(int64_t)min(r, rows - 1) * score_keys(a)];
  const float before = wt.in && key < a.Nk ? wt.in[to] : 0.f;
  const int row = threadIdx.x >> 3, sub = threadIdx.x & 7;   // eight lanes a row
  if (row < rows) {
    const int64_t stat = row_stat(a, b, hk, row);
    const int n = SPLIT ? row_parts(a, parts, rows_at, b, hk, row) : 1;
    float m;
    if (n > 1) {
      m = part_lse(parts, stat, n, sub, 8);
    } else {   // finished by its workgroup
      m = a.lse[stat] * kLog2e;
    }
    if (sub == 0) lse2[row] = m == -INFINITY ? INFINITY : m;   // no keys: P = 0
  }
  __syncthreads();
  if (key >= a.Nk) return;
  const XSample sm = x_sample<kSeeCache>(a, b);
  const XSpan span = x_span<kSeeCache>(a, sm, 0, rows);
  float sum = 0.f;
  if (key < sm.nk && span.has(key / kXKeys)) {
#pragma unroll
    for (int r = 0; r < kEarly; ++r) sum += r < rows ? fast_exp2(early[r] - lse2[r]) : 0.f;
#pragma unroll 4
    for (int r = kEarly; r < rows; ++r) sum += fast_exp2(sc[(int64_t)r * score_keys(a)] - lse2[r]);
  }
  wt.out[to] = before + sum;
}

constexpr int kWWaves = 8;    // of a workgroup: at 128 columns 64 KB of keys and 48 KB of rows, one workgroup a CU
constexpr int kWRows = 192;   // rows in LDS, a multiple of 64
constexpr int kWTiles = 8;    // most tiles of 32 keys of a wave

// JOIN: the rows' parts are not joined yet. Each workgroup joins some first (as workgroups
// of their own they would wait for a place, one a CU: 36 us in place of 29 at 4 x 1,536
// rows), those behind the first `weigh` nothing else, and the rows' LSE come from the
// parts' sums.
// SHARED: the steps of four tiles that are seen are shared out; else a workgroup has `per`
// steps of one sample and key head, seen or not.
template <int DP, bool JOIN, bool SHARED>
__global__ __launch_bounds__(64 * kWWaves, 2) void cache_weights_kernel(const XArgs a, const CacheWeights c,
                                                                        const CacheRows rows_at, const CacheParts parts,
                                                                        const int weigh, const int per, const int joins, const bool many) {
  constexpr int ROWB = DP * 2, CPR = DP / 8, KS = DP / 16;
  constexpr int KI = 32 * ROWB / 1024;   // direct loads of a tile
  __shared__ __attribute__((aligned(1024))) char k_lds[kWWaves * 32 * ROWB];
  __shared__ __attribute__((aligned(16))) char q_lds[kWRows * ROWB];
  __shared__ __attribute__((aligned(16))) float lse_lds[kWRows];
  __shared__ int p_lds[kWRows];
  __shared__ uint64_t tree_lds[kWRows];
  __shared__ unsigned see_lds[kWWaves][64];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int T = 64 * kWWaves;
  if constexpr (JOIN) {
    if (many) {   // uniform: a row a turn
      for (int i = blockIdx.x; i < joins; i += gridDim.x) {
        join_rows<T / 32, T>(a, parts, rows_at, i, reinterpret_cast<float4*>(k_lds));
        __syncthreads();
      }
    } else {
      for (int i = blockIdx.x; i < joins; i += 2 * gridDim.x) join_rows<1, T, 2>(a, parts, rows_at, i, nullptr);
    }
  }
  const int rows = a.Nq * a.G;
  if (SHARED && c.in != c.out) {   // tiles that no row sees keep what they had
    const int chunks = (a.Nk + T - 1) / T;
    for (int i = blockIdx.x; i < a.B * a.Hk * chunks; i += gridDim.x) {
      const int bh = i / chunks, b = bh / a.Hk, key = (i - bh * chunks) * T + tid;
      const XSample sm = x_sample<kSeeCache>(a, b);
      if (key >= a.Nk || x_span<kSeeCache>(a, sm, 0, rows).has(key / kXKeys)) continue;
      const int64_t at = (int64_t)bh * a.Nk + key;
      c.out[at] = c.in ? c.in[at] : 0.f;
    }
  }
  if ((int)blockIdx.x >= weigh) return;
  const float c2 = a.scale * kLog2e;
  char* const k_mine = k_lds + w * 32 * ROWB;
  int k_off[KI];   // row and column of this lane's piece of direct load i
#pragma unroll
  for (int i = 0; i < KI; ++i) {
    const int r = i * (1024 / ROWB) + lane / CPR, ch = lds_off<CPR>(r, lane % CPR) / 16 % CPR;
    k_off[i] = 8 * ch < a.D ? r * a.sk * 2 + 16 * ch : kXOut;
  }
  bool again = false;   // the rows in LDS are in use (uniform)
  CacheShare share;
  if constexpr (SHARED) {
    share = cache_share<4>(a, (int)blockIdx.x, weigh, a.Hk, nullptr);
  } else {
    const unsigned rest = blockIdx.x / (unsigned)a.Hk, chunks = (unsigned)((a.Nk + 4 * kXKeys * per - 1) / (4 * kXKeys * per));
    const int b = (int)(rest / chunks), t0 = (int)(rest % chunks) * per;
    share = CacheShare{b, (int)(blockIdx.x % (unsigned)a.Hk), t0, t0 + per, 1, 0};
  }
  for (bool first = true; share.items > 0; first = false) {   // uniform over the workgroup
    const int b = share.b, hk = share.g;
    const XSample sm = x_sample<kSeeCache>(a, b);
    const int off = sm.nk - sm.nq;
    const XSpan span = x_span<kSeeCache>(a, sm, 0, rows);
    // The tiles in turn: all of them, or those that some row sees.
    const int tiles = SHARED ? span.count : (a.Nk + kXKeys - 1) / kXKeys;
    const int all = (tiles + 3) / 4, end = share.items == 1 ? min(share.t1, all) : all;
    for (int step0 = first ? share.t0 : 0; step0 < end; step0 += kWTiles) {
      const int per_wave = min(end - step0, kWTiles);
      // The wave's half of one of the four tiles of step i; behind the last tile no row sees it.
      auto tile_of = [&](int i) __attribute__((always_inline)) { return 4 * (step0 + i) + (w >> 1); };
      auto tile_key = [&](int i) __attribute__((always_inline)) {
        const int t = tile_of(i);
        return kXKeys * (t + (SHARED && t >= span.first ? span.skip : 0)) + 32 * (w & 1);
      };
      auto seen = [&](int k) __attribute__((always_inline)) {   // keys from k on, by some row
        return (k < span.hi && k + 32 > span.lo) || k < span.send;
      };
      auto load = [&](int k) __attribute__((always_inline)) {   // slots that the sample lacks read zeros
        const int left = min(sm.nk - k, 32);
        const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(static_cast<const __bf16*>(a.k) + (sm.k0 + min(k, sm.nk - 1)) * a.sk + hk * a.D,
                                                      left > 0 ? ((left - 1) * a.sk + a.D) * 2 : 0);
#pragma unroll
        for (int i = 0; i < KI; ++i) buffer_load_lds16(rs, k_mine + i * 1024, k_off[i]);
      };
      float sum[kWTiles];
#pragma unroll
      for (int i = 0; i < kWTiles; ++i) sum[i] = 0.f;
      const int key0 = 4 * kXKeys * step0;
      const bool any = SHARED || (key0 < span.hi && key0 + 4 * kXKeys * per_wave > span.lo) || key0 < span.send;   // uniform
      for (int r0 = 0; any && r0 < rows; r0 += kWRows) {
        const int n = min(rows - r0, kWRows);
        if (again) __syncthreads();
        again = true;
        constexpr int kLoads = kWRows * CPR / T;   // 16-byte pieces a thread, loaded together
        bf16x8 piece[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
          const int i = u * T + tid, r = i / CPR, ch = i % CPR, tok = row_token(r0 + r, a.G);
          piece[u] = bf16x8{};
          if (r < n && 8 * ch < a.D)
            piece[u] = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + (sm.q0 + tok) * a.sq +
                                                        (hk * a.G + r0 + r - tok * a.G) * a.D + 8 * ch);
        }
        load(tile_key(0));
        const int pad = (n + 63) / 64 * 64;
        if (tid < pad) {
          const int row = r0 + tid, tok = row_token(min(row, rows - 1), a.G);
          RowWindow<kSeeCache> see;
          see.open(a, sm, b, row);
          p_lds[tid] = see.p;
          tree_lds[tid] = see.tree;
          if constexpr (!JOIN) {   // rows that are not counted, and rows without keys: P = 0
            float l = INFINITY;
            if (row < rows && (!c.tokens || c.tokens[b] >> tok & 1)) l = a.lse[row_stat(a, b, hk, row)] * kLog2e;
            lse_lds[tid] = l == -INFINITY ? INFINITY : l;
          }
        }
        if constexpr (JOIN) {   // all lanes: parts may be many where rows are few
          static_assert(2 * kWRows <= T);
          const int shift = pad <= T / 8 ? 3 : pad <= T / 4 ? 2 : 1, at = tid >> shift, row = r0 + at;
          if (at < pad) {
            float l = INFINITY;
            if (row < rows)
              l = part_lse(parts, row_stat(a, b, hk, row), row_parts(a, parts, rows_at, b, hk, row), tid - (at << shift), 1 << shift);
            lse_lds[at] = l == -INFINITY ? INFINITY : l;
          }
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
          const int i = u * T + tid;
          *reinterpret_cast<bf16x8*>(q_lds + lds_off<CPR>(i / CPR, i % CPR)) = piece[u];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWTiles; ++i) {
          if (i >= per_wave) break;   // uniform
          __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): the tile is there
          bf16x8 kop[KS];
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) kop[ks] = *reinterpret_cast<const bf16x8*>(k_mine + lds_off<CPR>(l32, 2 * ks + g));
          __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): and read
          pin_order();
          if (i + 1 < per_wave) load(tile_key(i + 1));
          const int k = tile_key(i);
          if (!seen(k)) continue;     // uniform
          // every row sees every key of the tile, whatever its place in the chunk or tree
          const bool whole = k + 32 <= off && (k >= off + sm.nq - a.left || k + 32 <= a.sinks);
          float add = 0.f;
          auto walk = [&](auto all_seen) __attribute__((always_inline)) {
            for (int r = 0; r < n; r += 64) {   // 64 rows, so that products and exponentials overlap
              if constexpr (!decltype(all_seen)::value) {   // which of the keys a row sees, a lane a row
                const int row = r + lane, p = p_lds[row];
                const RowWindow<kSeeCache> see{p, a.tree ? off : p + 1, tree_lds[row]};
                see_lds[w][lane] = see.bits(a, k) & bits32_from_to(0, sm.nk - k);
                __builtin_amdgcn_wave_barrier();
              }
              f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
              for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                  s[y] = mfma32(*reinterpret_cast<const bf16x8*>(q_lds + lds_off<CPR>(r + 32 * y + l32, 2 * ks + g)), kop[ks],
                                s[y]);
#pragma unroll
              for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  const int row0 = r + 32 * y + 8 * x + 4 * g;
                  const f32x4 ls = *reinterpret_cast<const f32x4*>(lse_lds + row0);
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    const float p = fast_exp2(__builtin_fmaf(s[y][4 * x + e], c2, -ls[e]));
                    if constexpr (decltype(all_seen)::value) add += p;
                    else add += see_lds[w][row0 - r + e] >> l32 & 1 ? p : 0.f;
                  }
                }
            }
          };
          if (whole) walk(std::true_type{});   // uniform
          else walk(std::false_type{});
          sum[i] += add;
        }
      }
#pragma unroll
      for (int i = 0; i < kWTiles; ++i) {
        if (i >= per_wave) break;   // uniform
        const int key = tile_key(i) + l32;
        const float x = pair_sum(sum[i]);
        const int64_t at = ((int64_t)b * a.Hk + hk) * a.Nk + key;
        if (g == 0 && tile_of(i) < tiles && key < a.Nk) c.out[at] = (c.in ? c.in[at] : 0.f) + x;
      }
      if (!SHARED) return;   // per <= kWTiles
    }
    if (++share.g == a.Hk) share.g = 0, ++share.b;
    --share.items;
  }
}

// ---------------------------------------------------------------------------
// Eviction
// ---------------------------------------------------------------------------
// Weights as unsigned numbers of the same order, 1 or above; NaN below all, -0 as +0.
__device__ inline unsigned weight_key(float x) {
  const unsigned u = __float_as_uint(x);
  if (x != x) return 1u;
  if (u == 0x80000000u) return 0x80000000u;
  return u >> 31 ? ~u : u | 0x80000000u;
}

// One workgroup of W waves a row (sample and key head). R: registers a lane for the row's
// middle, L: words of LDS a lane for more of it; R = 0: it is read again in every pass. Few
// waves where they hold the row: the arithmetic of a step is done by each of them (300
// slots 5.7 us with 4, 9.3 with 16; 16,000 slots 22 and 16).
template <int W, int R, int L = 0>
__global__ __launch_bounds__(64 * W) void cache_select_kernel(const CacheEvict a) {
  __shared__ __attribute__((aligned(16))) unsigned cnt[2][W], cnt2[W], ends[4][W];
  __shared__ unsigned few[64], found;
  __shared__ unsigned key_lds[L ? L * 64 * W : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = blockIdx.x;
  const int b = (int)(row / a.Hk);
  const float* const wt = a.weights + row * a.cap;
  float* const wo = a.weights_out + row * a.cap_out;
  int32_t* const idx = a.idx + row * a.keep;
  // Wave w holds the slots [begin, begin + per) of the middle, in order of register and
  // lane: by the capacity, so that they load beside the length.
  const float* const mid = wt + a.sinks;
  const int room = max(a.cap - a.sinks - a.recent, 0), per = ((room + W - 1) / W + 63) / 64 * 64, begin = w * per;
  float x[R ? R : 1];
  if constexpr (R > 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int at = begin + 64 * i + lane;
      x[i] = 64 * i < per && at < room ? mid[at] : 0.f;
    }
  }
  const int n = min(max(x_cu(a.lens, b), 0), a.cap), count = min(n, a.keep);
  if (tid == 0 && row % a.Hk == 0) a.len_out[b] = count;
  for (int i = count + tid; i < a.keep; i += 64 * W) idx[i] = -1;
  for (int i = count + tid; i < a.cap_out; i += 64 * W) wo[i] = 0.f;
  if (n <= a.keep) {   // uniform
    for (int i = tid; i < n; i += 64 * W) idx[i] = i;
    return;
  }
  // The first and the last slots stay; `need` >= 0 of the m > need between them.
  for (int i = tid; i < a.sinks; i += 64 * W) idx[i] = i;
  for (int i = tid; i < a.recent; i += 64 * W) idx[a.keep - a.recent + i] = n - a.recent + i;
  const int m = n - a.sinks - a.recent, need = a.keep - a.sinks - a.recent;
  if (need == 0) return;   // uniform
  const int end = min(m, begin + per);
  unsigned key[R ? R : 1];   // behind the middle 0: below every key
  if constexpr (R > 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) key[i] = begin + 64 * i + lane < end ? weight_key(x[i]) : 0u;
  }
#pragma unroll 12
  for (int i = 0; i < L; ++i) {   // a lane reads what it wrote: no barrier
    const int at = begin + 64 * (R + i) + lane;
    key_lds[i * 64 * W + tid] = at < end ? weight_key(mid[at]) : 0u;
  }
  // f(slot of the lane, its key) over the wave's slots
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (R > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i) f(begin + 64 * i + lane, key[i]);
#pragma unroll 12
      for (int i = 0; i < L; ++i) f(begin + 64 * (R + i) + lane, key_lds[i * 64 * W + tid]);
    } else {
      constexpr int U = 8;   // loaded together
      for (int at = begin + lane; at - lane < end; at += 64 * U) {
        float y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) y[u] = at + 64 * u < end ? mid[at + 64 * u] : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) f(at + 64 * u, at + 64 * u < end ? weight_key(y[u]) : 0u);
      }
    }
  };
  int turn = 0;
  auto total = [&](unsigned mine) __attribute__((always_inline)) {   // over the waves; one barrier
    if (lane == 0) cnt[turn][w] = mine;
    __syncthreads();
    unsigned sum = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) sum += cnt[turn][i];
    turn ^= 1;
    return sum;
  };
  // [t, last] holds the largest key that `need` slots or more have or exceed: at_t of
  // them have t or more, at_last more than `last`. At first all keys, or those above 0:
  // many slots have received nothing, and no key lies between 0 and the rest.
  constexpr unsigned kZero = 0x80000000u;
  unsigned t = ~0u, from = ~0u, last = 0;
  int positive = 0;
  each([&](int, unsigned k) {
    t = min(t, k - 1);   // 0: the largest
    from = min(from, k > kZero ? k : ~0u);
    positive += k > kZero ? 1 : 0;
    last = max(last, k);
  });
  t = wave_min(t);
  from = wave_min(from);
  last = ~wave_min(~last);
  positive = wave_sum(positive);
  if (lane == 0) ends[0][w] = t, ends[1][w] = last, ends[2][w] = from, ends[3][w] = positive;
  __syncthreads();
  positive = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    t = min(t, ends[0][i]), last = max(last, ends[1][i]), from = min(from, ends[2][i]);
    positive += ends[3][i];
  }
  const bool above_0 = positive >= need;
  t = above_0 ? from : t + 1;
  unsigned at_t = above_0 ? positive : m, at_last = 0;
  for (int step = 1; at_t != (unsigned)need && last > t && at_t - at_last > 64; ++step) {   // uniform
    const unsigned width = last - t;
    unsigned by = width / 2;
    if (step % 4 != 0)   // any number within the bracket will do
      by = (unsigned)((float)width * ((float)(at_t - need) + 0.5f) * __builtin_amdgcn_rcpf((float)(at_t - at_last)));
    const unsigned limit = t + 1 + min(by, width - 1);
    int c = 0;
    each([&](int, unsigned k) { c += k >= limit ? 1 : 0; });
    const unsigned all = total((unsigned)wave_sum(c));
    if (all >= (unsigned)need) t = limit, at_t = all;
    else last = limit - 1, at_last = all;
  }
  if (at_t != (unsigned)need && last > t) {   // uniform: the last 64 or fewer, each against all others
    if (tid == 0) found = 0;
    __syncthreads();
    each([&](int, unsigned k) {
      if (k >= t && k <= last) few[atomicAdd(&found, 1u)] = k;   // values alone: any order
    });
    __syncthreads();
    const int n_few = at_t - at_last;
    const unsigned mine = lane < n_few ? few[lane] : 0u;
    unsigned more = 0, same = 0;   // of them above the lane's, and equal to it
    for (int i = 0; i < n_few; ++i) {
      const unsigned other = (unsigned)__builtin_amdgcn_readlane((int)mine, i);
      more += other > mine;
      same += other == mine;
    }
    // the one with which `need` is reached
    const bool is = lane < n_few && at_last + more < (unsigned)need && (unsigned)need <= at_last + more + same;
    t = (unsigned)__builtin_amdgcn_readlane((int)mine, __builtin_ctzll(__ballot(is)));
  }
  // Slots above t, and of those equal to it the first ones.
  int over_mine = 0, same_mine = 0;
  each([&](int, unsigned k) {
    over_mine += k > t ? 1 : 0;
    same_mine += k == t ? 1 : 0;
  });
  const unsigned over = wave_sum(over_mine), same = wave_sum(same_mine);
  if (lane == 0) cnt2[w] = same;
  const unsigned above = total(over);   // its barrier covers cnt2 too
  unsigned before_over = 0, before_same = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    before_over += i < w ? cnt[turn ^ 1][i] : 0;
    before_same += i < w ? cnt2[i] : 0;
  }
  const unsigned ties = (unsigned)need - above;
  if (same == 0) {   // uniform: as a rule
    each([&](int at, unsigned k) {
      const uint64_t o = __ballot(k > t);
      const unsigned mo = __builtin_amdgcn_mbcnt_hi((unsigned)(o >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)o, before_over));
      if (k > t) idx[a.sinks + (int)(mo + min(before_same, ties))] = a.sinks + at;
      before_over += __builtin_popcountll(o);
    });
    return;
  }
  each([&](int at, unsigned k) {
    const uint64_t o = __ballot(k > t), s = __ballot(k == t);
    const unsigned mo = __builtin_amdgcn_mbcnt_hi((unsigned)(o >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)o, before_over));
    const unsigned ms = __builtin_amdgcn_mbcnt_hi((unsigned)(s >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)s, before_same));
    if (k > t || (k == t && ms < ties)) idx[a.sinks + (int)(mo + min(ms, ties))] = a.sinks + at;
    before_over += __builtin_popcountll(o);
    before_same += __builtin_popcountll(s);
  });
}

// Rows of K and V to their places, 16 bytes a thread of each, and the slots' weights
// (written beside the selection they would wait for a load each: 23 us in place of 10);
// rows behind the kept ones 0 up to `rows`.
__global__ __launch_bounds__(256) void cache_move_kernel(const CacheEvict a, const int rows) {
  const int per = a.Hk * a.D / 8, b = blockIdx.y;
  const int count = min(min(max(x_cu(a.lens, b), 0), a.cap), a.keep);
  const int64_t total = (int64_t)rows * per;
  constexpr int U = 4;
  for (int64_t i0 = (int64_t)blockIdx.x * (256 * U) + threadIdx.x; i0 < total; i0 += (int64_t)gridDim.x * (256 * U)) {
    u32x4 k[U], v[U];
    int64_t to_k[U], to_v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + 256 * u;
      const int place = (int)(i / per), col = (int)(i - (int64_t)place * per) * 8, hk = col / a.D;
      k[u] = v[u] = u32x4{};
      to_k[u] = ((int64_t)b * a.cap_out + place) * a.sko + col;
      to_v[u] = ((int64_t)b * a.cap_out + place) * a.svo + col;
      if (i < total && place < count) {
        const int64_t row = (int64_t)b * a.Hk + hk;
        const int from = a.idx[row * a.keep + place];
        if (col == hk * a.D) a.weights_out[row * a.cap_out + place] = a.weights[row * a.cap + from];
        const int64_t slot = (int64_t)b * a.cap + from;
        k[u] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(static_cast<const __bf16*>(a.k) + slot * a.sk + col));
        v[u] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(static_cast<const __bf16*>(a.v) + slot * a.sv + col));
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + 256 * u >= total) break;
      __builtin_nontemporal_store(k[u], reinterpret_cast<u32x4*>(static_cast<__bf16*>(a.k_out) + to_k[u]));
      __builtin_nontemporal_store(v[u], reinterpret_cast<u32x4*>(static_cast<__bf16*>(a.v_out) + to_v[u]));
    }
  }
}

}  // namespace

// Workspace of a cache call: the parts' O and sums, how items are cut, the scores.
namespace {
struct CacheSpace {
  size_t o, sums, cuts, scores;   // bytes
};
CacheSpace cache_space(const XArgs& a) {
  const int splits = cache_shape(a).splits;
  const int64_t stats = a.Tq * a.Hq;
  CacheSpace c{};
  if (splits > 1) {
    c.o = (size_t)splits * stats * a.D * sizeof(float);
    c.sums = ((size_t)splits * stats * sizeof(float2) + 15) / 16 * 16;
    c.cuts = ((size_t)a.B + 1 + 3) / 4 * 4 * sizeof(int);
  }
  if (a.scores) c.scores = (size_t)stats * score_keys(a) * sizeof(float);
  return c;
}

// Workgroups of the weights' launch. Steps of four tiles: as many a workgroup (`per`) as
// leave one for each CU, by the capacity, or where a window leaves most of it unseen (0)
// shared out by what is seen (48 tokens of 32 heads, four samples: 24,576 slots with a
// window of 4,096 57 -> 39 us, but 4,096 slots seen whole 31 -> 34).
struct WeightsGrid {
  int64_t per, weigh;
};
WeightsGrid weights_grid(const XArgs& a) {
  const int64_t heads = (int64_t)a.B * a.Hk, all = ((int64_t)a.Nk + 4 * kXKeys - 1) / (4 * kXKeys);
  const int64_t steps = (x_item_tiles(a, a.Nq * a.G) + 3) / 4;
  const int64_t per = 2 * steps <= all ? 0 : std::max<int64_t>(1, std::min<int64_t>(kWTiles, (heads * all + 255) / 256));
  return WeightsGrid{per, per ? heads * ((all + per - 1) / per) : std::min<int64_t>(heads * steps, 256)};
}
// Workgroups behind the attention: of the joins, and of the weights from the scores.
int64_t finish_joins(const XArgs& a, bool many) { return (a.Tq * a.Hq + (many ? 0 : 7)) / (many ? 1 : 8); }
int64_t finish_chunks(const XArgs& a) { return a.scores ? (int64_t)a.B * a.Hk * (((int64_t)a.Nk + 255) / 256) : 0; }
constexpr int64_t kMostThreads = (int64_t)1 << 32;   // of a launch: fewer

template <bool JOIN>
hipError_t launch_weights(const XArgs& a, const CacheWeights& c, const CacheRows& rows, const CacheParts& parts, bool many,
                          hipStream_t s) {
  const auto [per, weigh] = weights_grid(a);
  const int64_t joins = !JOIN ? 0 : many ? parts.stats : (parts.stats + 2 * kWWaves - 1) / (2 * kWWaves);
  const int64_t grid = std::max<int64_t>(weigh, std::min<int64_t>(joins, 256));
  TraceScope ts_(s, "cache_weights", x_padded(a));
  const int most = (int)weigh, each = (int)per;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kWWaves), 0, s, a, c, rows, parts, most, each, (int)joins, many);
  };
  if (per > 0) a.D <= 64 ? launch(cache_weights_kernel<64, JOIN, false>) : launch(cache_weights_kernel<128, JOIN, false>);
  else a.D <= 64 ? launch(cache_weights_kernel<64, JOIN, true>) : launch(cache_weights_kernel<128, JOIN, true>);
  return hipGetLastError();
}
}  // namespace

bool cache_weights_launchable(const XArgs& a) { return weights_grid(a).weigh * (64 * kWWaves) < kMostThreads; }

bool cache_attn_launchable(const XArgs& a, bool weights) {
  if (weights && !a.scores && !cache_weights_launchable(a)) return false;
  const int64_t joins = cache_shape(a).splits > 1 ? finish_joins(a, false) : 0;   // `many` are few enough
  return (joins + finish_chunks(a)) * 256 < kMostThreads;
}

size_t cache_attn_workspace(const XArgs& a) {
  const CacheSpace c = cache_space(a);
  return c.o + c.sums + c.cuts + c.scores;
}

hipError_t launch_cache_attn(const XArgs& a, const CacheWeights& w, void* workspace, hipStream_t s) {
  const XShape shape = cache_shape(a);
  const CacheSpace c = cache_space(a);
  char* const at = static_cast<char*>(workspace);
  const bool few = a.Nq * a.G <= kScoreRows, split = shape.splits > 1;
  const CacheParts parts{reinterpret_cast<float2*>(at + c.o), reinterpret_cast<float*>(at), a.Tq * a.Hq,
                         split ? reinterpret_cast<int*>(at + c.o + c.sums) : nullptr,
                         reinterpret_cast<float*>(at + c.o + c.sums + c.cuts),
                         few ? cache_heads(a) : 0};
  // Eight groups of lanes a row where many parts are to be read for few rows, as in
  // cross attention. Beside the weights sixteen where a workgroup's turns, a row each, pay
  // for themselves (80 rows of up to 235 parts 84 -> 29 us, 256 of 17 14 -> 12; but 1,024 of
  // 17 18 -> 22, 4,096 of 9 26 -> 51).
  const bool many = few || !w.out ? shape.splits >= 8 && parts.stats <= 4096
                                  : shape.splits >= 16 * ((parts.stats + 255) / 256);
  const int per = few ? kScoreRows : 32 * shape.waves;
  const CacheRows rows{(int)(((int64_t)a.Nq * a.G + per - 1) / per), per};
  if (few) {
    // no item is cut, and the weights are few enough for the workgroup that has the scores
    const bool weights_here = !split && a.scores && a.Nk <= 2048;
    if (hipError_t e = launch_cache_one(a, parts, w, weights_here, s); e != hipSuccess) return e;
    if (!split && (!a.scores || weights_here)) return hipSuccess;
  } else {
    if (hipError_t e = launch_cache_fwd(a, shape, parts, s); e != hipSuccess) return e;
    if (w.out) return split ? launch_weights<true>(a, w, rows, parts, many, s) : launch_weights<false>(a, w, rows, parts, false, s);
    if (!split) return hipSuccess;
  }
  const int64_t joins = split ? finish_joins(a, many) : 0, chunks = finish_chunks(a);
  TraceScope ts_(s, "cache_finish");
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(joins + chunks)), dim3(256), 0, s, a, rows, (int)joins, parts, w);
  };
  !split ? launch(cache_finish_kernel<1, false>) : many ? launch(cache_finish_kernel<8, true>) : launch(cache_finish_kernel<1, true>);
  return hipGetLastError();
}

hipError_t launch_cache_weights(const XArgs& a, const CacheWeights& c, hipStream_t s) {
  return launch_weights<false>(a, c, CacheRows{}, CacheParts{}, false, s);
}

hipError_t launch_cache_evict(const CacheEvict& a, hipStream_t s) {
  const int64_t room = std::max<int64_t>((int64_t)a.cap - a.sinks - a.recent, 0);   // slots of a row's middle, at most
  {
    TraceScope ts_(s, "cache_select");
    const dim3 grid((unsigned)(a.B * a.Hk));
    if (room <= 1024) hipLaunchKernelGGL((cache_select_kernel<4, 4>), grid, dim3(256), 0, s, a);
    else if (room <= 4096) hipLaunchKernelGGL((cache_select_kernel<4, 16>), grid, dim3(256), 0, s, a);
    else if (room <= 16384) hipLaunchKernelGGL((cache_select_kernel<16, 16>), grid, dim3(1024), 0, s, a);
    else if (room <= 32768) hipLaunchKernelGGL((cache_select_kernel<16, 32>), grid, dim3(1024), 0, s, a);
    else if (room <= 1024 * 68) hipLaunchKernelGGL((cache_select_kernel<16, 32, 36>), grid, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((cache_select_kernel<16, 0>), grid, dim3(1024), 0, s, a);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  const int rows = a.zero_rest ? a.cap_out : a.keep;
  TraceScope ts_(s, "cache_move");
  const int64_t groups = ((int64_t)rows * (a.Hk * a.D / 8) + 1023) / 1024;
  hipLaunchKernelGGL(cache_move_kernel, dim3((unsigned)std::min<int64_t>(groups, 1 << 16), (unsigned)a.B), dim3(256), 0, s,
                     a, rows);
  return hipGetLastError();
}

}  // namespace ut
