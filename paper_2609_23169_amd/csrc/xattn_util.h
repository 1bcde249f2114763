// Device helpers shared by the cross-attention kernels: rows of queries and
// tiles of keys. A key head's queries are rows r of one list, token r / G and
// head r % G of its group of G, so that few tokens with many heads fill a tile
// and all of them read the key head's tiles once.
#pragma once

#include "attn_util.h"

namespace ut {

constexpr int kXKeys = 64;                 // keys of a tile
constexpr int kXOut = 0x40000000;          // a byte offset past every descriptor's range: reads zeros

// Work item of workgroup wg: the items are numbered so that neighbours share
// keys, and each XCD (workgroups go to the eight in turn) takes one run of them.
// With by_xcd false they are taken in plain order.
__device__ inline unsigned xcd_item(unsigned wg, unsigned n, bool by_xcd) {
  if (!by_xcd) return wg;
  const unsigned x = wg & 7, q = n >> 3, r = n & 7;
  return x * q + min(x, r) + (wg >> 3);
}

// The key tiles of one sample that hold a key in use, and which keys of each:
// 64 tiles at a time, one a lane, as 64-bit masks, so that a step to the next
// tile costs a few scalar instructions and unused tiles none. Tiles
// [begin, end); n keys; mask: a byte a key, or null.
struct KeyTiles {
  const uint8_t* mask;
  int n, end, base;
  uint64_t mine, left;   // this lane's tile; the group's tiles not yet visited

  __device__ inline KeyTiles(const uint8_t* m, int keys, int begin, int stop)
      : mask(m), n(keys), end(stop), base(begin - 64), mine(0), left(0) {}

  __device__ inline void group() {
    const int lane = threadIdx.x & 63, t = base + lane;
    mine = 0;
    if (mask) {
      if (t < end && kXKeys * (t + 1) <= n) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          u32x4 v;
          __builtin_memcpy(&v, mask + (int64_t)kXKeys * t + 16 * c, 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            unsigned b = v[e];   // a nonzero byte to its lowest bit, the four bits to one nibble
            b |= b >> 4;
            b |= b >> 2;
            b |= b >> 1;
            b = ((b & 0x01010101u) * 0x10204080u) >> 28;
            mine |= (uint64_t)b << (16 * c + 4 * e);
          }
        }
      }
    } else if (t < end) {
      mine = kXKeys * (t + 1) <= n ? ~(uint64_t)0 : 0;
    }
    const int last = n / kXKeys, rest = n % kXKeys;   // the short last tile
    if (rest && last < end && last >= base && last < base + 64) {
      const bool in = lane < rest && (!mask || mask[(int64_t)kXKeys * last + lane]);
      const uint64_t bits = __ballot(in);
      if (t == last) mine = bits;
    }
    left = __ballot(mine != 0);
  }
  // The next tile with keys in use and their bits; false at the end.
  __device__ inline bool next(int& tile, uint64_t& bits) {
    while (left == 0) {
      base += 64;
      if (base >= end) return false;
      group();
    }
    const int i = __builtin_ctzll(left);
    left &= left - 1;
    tile = base + i;
    const unsigned lo = __builtin_amdgcn_readlane((unsigned)mine, i);
    const unsigned hi = __builtin_amdgcn_readlane((unsigned)(mine >> 32), i);
    bits = (uint64_t)hi << 32 | lo;
    return true;
  }
};

// Sample b of B: its query rows and its keys.
struct XSample {
  int64_t q0, k0;     // first tokens
  int nq, nk;         // lengths
  int64_t stat0;      // statistics of (head 0, the first token)
  int64_t hstep;      // statistics from one head to the next
};
__device__ inline XSample x_sample(const XArgs& a, int b) {
  const SampleRows q = sample_rows(a.cuq, a.Tq, b, 0, a.Hq, a.Nq);
  const SampleRows k = sample_rows(a.cuk, a.Tk, b, 0, 1, a.Nk);
  return XSample{q.tok0, k.tok0, q.n, k.n, q.stat0, a.cuq ? a.Tq : (int64_t)a.Nq};
}

// Whether packed token `tok` belongs to one of the B samples (lengths up to N).
__device__ inline bool in_sample(const int32_t* __restrict__ cu, int64_t T, int B, int N, int64_t tok) {
  for (int b = 0; b < B; ++b) {
    const SampleRows r = sample_rows(cu, T, b, 0, 1, N);
    if (tok >= r.tok0 && tok < r.tok0 + r.n) return true;
  }
  return false;
}

// Direct loads of 64-row tiles into LDS by NW waves, in rows of DP elements:
// instruction u of wave w writes 1 KB of rows. The swizzle repeats every 16
// rows, so a lane keeps one offset for each of the instructions of 16 rows, and
// the rest of the row's offset is a scalar.
template <int DP, int NW>
struct TileLoad {
  static constexpr int ROWB = DP * 2, CPR = DP / 8;
  static constexpr int RPI = 1024 / ROWB;                      // rows per instruction
  static constexpr int IPW = kXKeys * ROWB / 1024 / NW;        // instructions per wave
  static constexpr int REP = 16 / RPI;                         // instructions of 16 rows
  static_assert(IPW % REP == 0, "a wave takes whole runs of 16 rows");
  int off[REP];

  __device__ inline TileLoad(int lane, int D, int stride) {
#pragma unroll
    for (int u = 0; u < REP; ++u) {
      const int r = u * RPI + lane / CPR, p = lane % CPR;
      const int c = (lds_off<CPR>(r, p) >> 4) & (CPR - 1);
      off[u] = c < D / 8 ? r * stride * 2 + 16 * c : kXOut;    // columns past D read zeros
    }
  }
  // Tile at `src` (its first key's row of this head), keys in `bits`; other rows
  // become zeros, whatever memory holds there, and are not read.
  __device__ inline void operator()(const __bf16* src, int stride, uint64_t bits, char* dst, int w, int lane) const {
    const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(src, (kXKeys - 1) * stride * 2 + DP * 2);
    if (bits == ~(uint64_t)0) {
#pragma unroll
      for (int u = 0; u < IPW; ++u) {
        const int i = w * IPW + u;
        buffer_load_lds16(rs, dst + i * 1024, off[u % REP], i / REP * 16 * stride * 2);
      }
    } else {
#pragma unroll
      for (int u = 0; u < IPW; ++u) {
        const int i = w * IPW + u;
        const unsigned run = (unsigned)(bits >> (i / REP * 16)) >> (u % REP * RPI);   // scalar
        buffer_load_lds16(rs, dst + i * 1024, run >> (lane / CPR) & 1 ? off[u % REP] : kXOut,
                          i / REP * 16 * stride * 2);
      }
    }
  }
};

}  // namespace ut
