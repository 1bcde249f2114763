// What a cache of keys and values needs beside the attention that reads it, on
// gfx950: the attention weight that every slot receives, summed over the queries,
// and eviction of the slots that received least.
//
// Weights: out[b, hk, j] = in[b, hk, j] + sum over the tokens t and the heads h of the
// group of P = exp(S scale - LSE). The attention knows a row's LSE only at its end, so
// this pass forms the scores again (of few rows the attention leaves them instead): a
// workgroup keeps the rows of the group in LDS, up to 192 at once, a wave takes tiles of
// 32 keys, whose rows pass through its registers, the next tile's loads beside the
// products; S = Q K^T on 32x32x16 bf16 MFMA in the layout where a lane holds one key, so
// that the sum over the rows is the lane's own but for one exchange. fp32 throughout, a
// fixed order: no atomics.
//
// Eviction: of a row of weights the middle slots (behind the sinks, before the recent
// ones) are bisected by value for the smallest weight that stays. A workgroup holds the
// row in registers (up to 32,768 slots, longer rows are read again), a step is a
// compare and a ballot a register and one barrier, and it ends as soon as the count
// fits. Then ballots give every kept slot its place in ascending order, equal weights
// the lowest slots first, and a second launch copies the rows of K and V.
#include <algorithm>

#include "xattn_util.h"

namespace ut {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWRows = 192;   // rows in LDS: 48 KB at 128 columns, three workgroups a CU
constexpr int kWTiles = 4;    // most tiles of 32 keys of a wave

template <int DP>
__global__ __launch_bounds__(256, 3) void cache_weights_kernel(const XArgs a, const CacheWeights c, const int per_wave) {
  constexpr int ROWB = DP * 2, CPR = DP / 8, KS = DP / 16;
  __shared__ __attribute__((aligned(16))) char q_lds[kWRows * ROWB];
  __shared__ __attribute__((aligned(16))) float lse_lds[kWRows];
  __shared__ int p_lds[kWRows];
  __shared__ uint64_t tree_lds[kWRows];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned hk = blockIdx.x % (unsigned)a.Hk, rest = blockIdx.x / (unsigned)a.Hk;
  const int keys = 128 * per_wave;   // of the workgroup
  const unsigned chunks = (unsigned)((a.Nk + keys - 1) / keys);
  const int b = (int)(rest / chunks), key0 = (int)(rest % chunks) * keys;
  const XSample sm = x_sample<kSeeCache>(a, b);
  const int off = sm.nk - sm.nq, rows = sm.nq * a.G;
  const XSpan span = x_span<kSeeCache>(a, sm, 0, rows);
  const float c2 = a.scale * kLog2e;
  // The wave's tiles: one of every four in turn. Whether some row sees keys from k on.
  auto tile_key = [&](int i) __attribute__((always_inline)) { return key0 + 32 * (4 * i + w); };
  auto seen = [&](int k) __attribute__((always_inline)) {
    return (k < span.hi && k + 32 > span.lo) || k < span.send;
  };
  auto load = [&](bf16x8 (&kop)[KS], int k) __attribute__((always_inline)) {
    const __bf16* const kp =
        static_cast<const __bf16*>(a.k) + (sm.k0 + min(k + l32, a.Nk - 1)) * a.sk + hk * a.D + 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kop[ks] = bf16x8{};
      if (16 * ks + 8 * g < a.D) kop[ks] = *reinterpret_cast<const bf16x8*>(kp + 16 * ks);
    }
  };
  float sum[kWTiles];
#pragma unroll
  for (int i = 0; i < kWTiles; ++i) sum[i] = 0.f;
  // uniform over the workgroup
  const bool any = (key0 < span.hi && key0 + keys > span.lo) || key0 < span.send;
  for (int r0 = 0; any && r0 < rows; r0 += kWRows) {
    const int n = min(rows - r0, kWRows);
    if (r0 > 0) __syncthreads();
    constexpr int kLoads = kWRows * CPR / 256;   // 16-byte pieces a thread, loaded together
    bf16x8 piece[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = u * 256 + tid, r = i / CPR, ch = i % CPR, tok = row_token(r0 + r, a.G);
      piece[u] = bf16x8{};
      if (r < n && 8 * ch < a.D)
        piece[u] = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(a.q) + (sm.q0 + tok) * a.sq +
                                                    (hk * a.G + r0 + r - tok * a.G) * a.D + 8 * ch);
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = u * 256 + tid;
      *reinterpret_cast<bf16x8*>(q_lds + lds_off<CPR>(i / CPR, i % CPR)) = piece[u];
    }
    if (tid < (n + 31) / 32 * 32) {
      const int row = r0 + tid, tok = row_token(min(row, rows - 1), a.G);
      RowWindow<kSeeCache> see;
      see.open(a, sm, b, row);
      p_lds[tid] = see.p;
      tree_lds[tid] = see.tree;
      // rows that are not counted, and rows without keys: P = 0
      float l = INFINITY;
      if (row < rows && (!c.tokens || c.tokens[b] >> tok & 1)) {
        l = a.lse[sm.stat0 + (hk * a.G + row - tok * a.G) * sm.hstep + tok] * kLog2e;
        if (l == -INFINITY) l = INFINITY;
      }
      lse_lds[tid] = l;
    }
    bf16x8 next[KS];
    load(next, tile_key(0));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWTiles; ++i) {
      if (i >= per_wave) break;   // uniform
      bf16x8 kop[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kop[ks] = next[ks];
      if (i + 1 < per_wave) load(next, tile_key(i + 1));
      const int k = tile_key(i), key = k + l32;
      if (!seen(k)) continue;     // uniform
      // every row sees every key of the tile, whatever its place in the chunk or tree
      const bool whole = k + 32 <= off && (k >= off + sm.nq - a.left || k + 32 <= a.sinks);
      for (int r = 0; r < n; r += 32) {
        f32x16 s = f32x16{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          s = mfma32(*reinterpret_cast<const bf16x8*>(q_lds + lds_off<CPR>(r + l32, 2 * ks + g)), kop[ks], s);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const f32x4 ls = *reinterpret_cast<const f32x4*>(lse_lds + r + 8 * x + 4 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = fast_exp2(__builtin_fmaf(s[4 * x + e], c2, -ls[e]));
            if (whole) {   // uniform
              sum[i] += p;
            } else {
              const int row = r + 8 * x + 4 * g + e, pos = p_lds[row], end = a.tree ? off : pos + 1;
              const bool in = (key < end && (key >= pos - a.left || key < a.sinks)) ||
                              (a.tree && key >= off && key < sm.nk && (tree_lds[row] >> (key - off) & 1));
              sum[i] += in ? p : 0.f;
            }
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kWTiles; ++i) {
    if (i >= per_wave) break;
    const int key = tile_key(i) + l32;
    const float x = pair_sum(sum[i]);
    const int64_t at = ((int64_t)b * a.Hk + hk) * a.Nk + key;
    if (g == 0 && key < a.Nk) c.out[at] = (c.in ? c.in[at] : 0.f) + x;
  }
}

// ---------------------------------------------------------------------------
// Eviction
// ---------------------------------------------------------------------------
constexpr int kEvictWaves = 16;

// Weights as unsigned numbers of the same order; NaN below all, -0 as +0.
__device__ inline unsigned weight_key(float x) {
  const unsigned u = __float_as_uint(x);
  if (x != x) return 0u;
  if (u == 0x80000000u) return 0x80000000u;
  return u >> 31 ? ~u : u | 0x80000000u;
}

// One workgroup a row (sample and key head). R: registers a lane for the row's middle,
// 0: it is read again in every pass.
template <int R>
__global__ __launch_bounds__(64 * kEvictWaves) void cache_select_kernel(const CacheEvict a) {
  constexpr int W = kEvictWaves;
  __shared__ unsigned cnt[2][W], cnt2[W];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = blockIdx.x;
  const int b = (int)(row / a.Hk);
  const int n = min(max(x_cu(a.lens, b), 0), a.cap), count = min(n, a.keep);
  const float* const wt = a.weights + row * a.cap;
  float* const wo = a.weights_out + row * a.cap_out;
  int32_t* const idx = a.idx + row * a.keep;
  if (tid == 0 && row % a.Hk == 0) a.len_out[b] = count;
  for (int i = count + tid; i < a.keep; i += 64 * W) idx[i] = -1;
  for (int i = count + tid; i < a.cap_out; i += 64 * W) wo[i] = 0.f;
  auto put = [&](int place, int slot) __attribute__((always_inline)) { idx[place] = slot; };
  if (n <= a.keep) {   // uniform
    for (int i = tid; i < n; i += 64 * W) put(i, i);
    return;
  }
  // The first and the last slots stay; `need` >= 0 of the m > need between them.
  for (int i = tid; i < a.sinks; i += 64 * W) put(i, i);
  for (int i = tid; i < a.recent; i += 64 * W) put(a.keep - a.recent + i, n - a.recent + i);
  const int m = n - a.sinks - a.recent, need = a.keep - a.sinks - a.recent;
  const float* const mid = wt + a.sinks;
  if (need == 0) return;   // uniform

  // Wave w holds the slots [begin, end) of the middle, in order of register and lane.
  const int per = ((m + W - 1) / W + 63) / 64 * 64, begin = w * per, end = min(m, begin + per);
  unsigned key[R ? R : 1];
  if constexpr (R > 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int at = begin + 64 * i + lane;
      key[i] = at < end ? weight_key(mid[at]) : 0u;
    }
  }
  // f(slot of the lane, its key) over the wave's slots (R > 0: its registers, slots
  // behind `end` with key 0)
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (R > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i) f(begin + 64 * i + lane, key[i]);
    } else {
      for (int at = begin + lane; at - lane < end; at += 64) f(at, at < end ? weight_key(mid[at]) : 0u);
    }
  };
  int turn = 0;
  auto total = [&](unsigned mine) __attribute__((always_inline)) {   // over the waves; one barrier
    if (lane == 0) cnt[turn][w] = mine;
    __syncthreads();
    unsigned t = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) t += cnt[turn][i];
    turn ^= 1;
    return t;
  };
  // The largest t such that `need` slots or more have a key of t or above.
  unsigned t = 0;
  bool exact = false;   // just `need` have one
  for (unsigned bit = 0x80000000u; bit != 0 && !exact; bit >>= 1) {   // uniform
    const unsigned to = t | bit;
    unsigned c = 0;
    each([&](int, unsigned k) { c += __builtin_popcountll(__ballot(k >= to)); });
    const unsigned all = total(c);
    if (all >= (unsigned)need) t = to, exact = all == (unsigned)need;
  }
  // Slots above t, and of those equal to it the first ones (behind the row's end keys
  // are 0: no slot, where t is 0).
  unsigned over = 0, same = 0;
  each([&](int at, unsigned k) {
    over += __builtin_popcountll(__ballot(k > t && at < end));
    same += __builtin_popcountll(__ballot(k == t && at < end));
  });
  if (lane == 0) cnt2[w] = same;
  const unsigned above = total(over);   // its barrier covers cnt2 too
  unsigned before_over = 0, before_same = 0;
  for (int i = 0; i < w; ++i) before_over += cnt[turn ^ 1][i], before_same += cnt2[i];
  const unsigned ties = (unsigned)need - above;
  each([&](int at, unsigned k) {
    const uint64_t o = __ballot(k > t && at < end), s = __ballot(k == t && at < end);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    const unsigned mo = before_over + __builtin_popcountll(o & below), ms = before_same + __builtin_popcountll(s & below);
    const bool in = (o >> lane & 1) || ((s >> lane & 1) && ms < ties);
    if (in) put(a.sinks + (int)(mo + min(ms, ties)), a.sinks + at);
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

hipError_t launch_cache_weights(const XArgs& a, const CacheWeights& c, hipStream_t s) {
  // as many tiles a wave as leave a workgroup for each place on the chip
  const int64_t heads = (int64_t)a.B * a.Hk, blocks = ((int64_t)a.Nk + 127) / 128;
  const int per_wave = (int)std::max<int64_t>(1, std::min<int64_t>(kWTiles, (heads * blocks + 767) / 768));
  const int64_t chunks = ((int64_t)a.Nk + 128 * per_wave - 1) / (128 * per_wave);
  TraceScope ts_(s, "cache_weights", x_padded(a));
  const dim3 grid((unsigned)(heads * chunks));
  if (a.D <= 64) hipLaunchKernelGGL(cache_weights_kernel<64>, grid, dim3(256), 0, s, a, c, per_wave);
  else hipLaunchKernelGGL(cache_weights_kernel<128>, grid, dim3(256), 0, s, a, c, per_wave);
  return hipGetLastError();
}

hipError_t launch_cache_evict(const CacheEvict& a, hipStream_t s) {
  const int64_t most = ((int64_t)a.cap - a.sinks - a.recent + 64 * kEvictWaves - 1) / (64 * kEvictWaves);   // a lane's
  {
    TraceScope ts_(s, "cache_select");
    const dim3 grid((unsigned)(a.B * a.Hk)), block(64 * kEvictWaves);
    if (most <= 4) hipLaunchKernelGGL(cache_select_kernel<4>, grid, block, 0, s, a);
    else if (most <= 16) hipLaunchKernelGGL(cache_select_kernel<16>, grid, block, 0, s, a);
    else if (most <= 32) hipLaunchKernelGGL(cache_select_kernel<32>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(cache_select_kernel<0>, grid, block, 0, s, a);
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
