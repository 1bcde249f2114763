// Device helpers shared by the cross-attention kernels: rows of queries and
// tiles of keys. A key head's queries are rows r of one list, token r / G and
// head r % G of its group of G, so that few tokens with many heads fill a tile
// and all of them read the key head's tiles once.
#pragma once

#include "attn_util.h"

namespace ut {

constexpr int kXKeys = 64;                 // keys of a tile
constexpr int kXOut = 0x40000000;          // a byte offset past every descriptor's range: reads zeros

// The kernel's arguments (an XArgs in front of the others), read again where they
// are used: work done once an item would otherwise hold some fifty more scalar
// registers through the loop over the tiles. The compiler still keeps 25 to 48 in
// lanes of vector registers (145 in the one-wave form at 128 columns) and reads them
// back in the loop; none go to memory.
__device__ inline const XArgs* x_args_again() {
#if defined(__HIP_DEVICE_COMPILE__)
  auto p = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return (const XArgs*)p;
#else
  return nullptr;
#endif
}

// The lane, read again where it is used: the offsets that work done once an item
// forms from it would otherwise be kept in registers through the loop.
__device__ inline int x_lane_again() {
  int lane = threadIdx.x & 63;
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(lane));
#endif
  return lane;
}

// The work items of a persistent workgroup: first, then `step` and `turn` - `step`
// further in turn, below end. Each XCD (workgroups go to the eight in turn) takes
// one run of the items, its n workgroups n items a turn, so that they share keys in
// their L2 (20,000 rows and keys, 24 heads: 5,014 us against 5,110 with one run for
// all; 60,000 keys: 15,517 against 15,217). Every other turn goes backwards: a
// workgroup would otherwise meet the same sample whenever the samples divide n, the
// longest each time (two samples of 1,370 and 822 keys: forward 136 us, now 124).
// The grid is a multiple of 8.
struct XItems {
  unsigned first, step, turn, end;
};
__device__ inline XItems x_items(unsigned total) {
  const unsigned x = blockIdx.x & 7, at = blockIdx.x >> 3, n = gridDim.x >> 3;
  const unsigned q = total >> 3, r = total & 7, start = x * q + min(x, r);
  return XItems{start + at, 2 * (n - at) - 1, 2 * n, start + q + (x < r ? 1 : 0)};
}
// How item numbers are read: `heads` key heads of a group fastest (their rows lie
// side by side), then samples, whose lengths may differ, so that every run holds
// alike parts of all of them, then tiles, parts of a split, groups of heads.
struct XOrder {
  unsigned heads, tiles, splits;
};
// Heads of a group: an eighth of them, so that each XCD has a group of its own
// and the runs are alike whatever the samples' lengths (eight samples of 17 to 512
// keys: forward and backward 1,708 us with one head a group, 1,380 with three).
inline unsigned head_group(const XArgs& a) { return a.Hk % 8 == 0 ? (unsigned)a.Hk / 8 : 1; }
// Workgroups of nw waves that fit 256 CUs at once, by LDS (64 KB at 128 columns, 32
// to 36 at 64) and by registers (two waves a SIMD at 128 columns, three at 64): what
// a grid needs to fill the chip.
constexpr int64_t x_resident(int DP, int nw) { return 256 * (DP == 128 ? 2 : nw == 4 ? 3 : 4); }
inline int x_padded(const XArgs& a) { return a.D <= 64 ? 64 : 128; }
struct XItem {
  int b, tile, part, hk;
};
__device__ inline XItem x_item(unsigned it, unsigned B, const XOrder& o) {
  const unsigned r = it / o.heads, s = r / B, t = s / o.tiles, u = t / o.splits;
  return XItem{(int)(r - s * B), (int)(s - t * o.tiles), (int)(t - u * o.splits), (int)(u * o.heads + it - r * o.heads)};
}

// The key tiles of one sample that hold a key in use, and which keys of each:
// 64 tiles at a time, one a lane, as 64-bit masks, so that a step to the next
// tile costs a few scalar instructions and unused tiles none. Tiles
// [begin, end); n keys; mask: a byte a key, or null.
struct KeyTiles {
  const uint8_t* mask;
  int n, end, base;
  uint64_t mine, left;   // this lane's tile; the group's tiles not yet visited

  __device__ inline void open(const uint8_t* m, int keys, int begin, int stop) {
    mask = m;
    n = keys;
    end = stop;
    base = begin - 64;
    mine = left = 0;
  }

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
// Offset i of a sample array, as a scalar load (the array is not written while the
// kernel runs).
__device__ inline int x_cu(const int32_t* cu, int i) {
#if defined(__HIP_DEVICE_COMPILE__)
  return ((const __attribute__((address_space(4))) int32_t*)cu)[i];
#else
  return cu[i];
#endif
}
__device__ inline XSample x_sample(const XArgs& a, int b) {
  if (!a.cuq)
    return XSample{(int64_t)b * a.Nq, (int64_t)b * a.Nk, a.Nq, a.Nk, (int64_t)b * a.Hq * a.Nq, (int64_t)a.Nq};
  // clamped as in sample_rows: no offsets can send an access outside the tensors
  const int64_t q0 = min(max((int64_t)x_cu(a.cuq, b), (int64_t)0), a.Tq);
  const int64_t q1 = min(max((int64_t)x_cu(a.cuq, b + 1), q0), a.Tq);
  const int64_t k0 = min(max((int64_t)x_cu(a.cuk, b), (int64_t)0), a.Tk);
  const int64_t k1 = min(max((int64_t)x_cu(a.cuk, b + 1), k0), a.Tk);
  return XSample{q0, k0, (int)min(q1 - q0, (int64_t)a.Nq), (int)min(k1 - k0, (int64_t)a.Nk), q0, a.Tq};
}
// Token of row `row` (the division is skipped where every head has its own keys).
__device__ inline int row_token(int row, int G) {
  if (G == 1) return row;
  return (int)((unsigned)row / (unsigned)G);
}

// Whether packed token `tok` belongs to one of the B samples (lengths up to N).
__device__ inline bool in_sample(const int32_t* __restrict__ cu, int64_t T, int B, int N, int64_t tok) {
  for (int b = 0; b < B; ++b) {
    const SampleRows r = sample_rows(cu, T, b, 0, 1, N);
    if (tok >= r.tok0 && tok < r.tok0 + r.n) return true;
  }
  return false;
}

// Rows of x at and past the last sample's end to 0, the grid's threads in turn.
__device__ inline void x_clear_rest(const int32_t* cu, int B, int64_t T, int width, void* x, int stride) {
  const int64_t end = min(max((int64_t)x_cu(cu, B), (int64_t)0), T);
  const int per = width / 8;
  for (int64_t i = end * per + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < T * per;
       i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t tok = i / per;
    *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(x) + tok * stride + 8 * (i - tok * per)) = bf16x8{};
  }
}

// The tiles of a persistent workgroup's items as one sequence. The items are worked
// out kTurns at a time, one a lane, so that a change of item costs some readlanes in
// place of three divisions, and the scalar registers are left to the loop over the
// tiles. The code of a change stands once in the loop: an item whose keys are not in
// use yields one tile without keys (bits 0), so that it is finished like the others.
struct TileSeq {
  static constexpr int kTurns = 62;             // even: every group begins with a forward turn
  static constexpr int kKept = 63;              // the lane that keeps an item over the groups
  KeyTiles tiles;
  int b, rtile, hkpart;                         // a lane's item: sample, tile of rows, key head and part
  unsigned first, step, turn, end;              // the next group's items (XItems)
  uint64_t todo;                                // items of the group not begun
  int at, cur;                                  // lanes of the item of the last tile given, and of the caller's
  int tile;
  uint64_t bits;
  bool fresh;                                   // that item has given no tile yet
  int64_t k0;                                   // its sample's first key
  int hk, keys;                                 // its key head and number of keys

  __device__ inline void begin(const XItems& i) {
    first = i.first, step = i.step, turn = i.turn, end = i.end;
    tiles.open(nullptr, 0, 0, 0);
    tile = hk = keys = b = rtile = hkpart = 0;
    k0 = 0;
    bits = todo = 0;
    at = cur = kKept;
    fresh = false;
  }
  // Item of lane i.
  __device__ inline XItem item(int i, const XOrder& order) const {
    const int hp = __builtin_amdgcn_readlane(hkpart, i);
    return XItem{__builtin_amdgcn_readlane(b, i), __builtin_amdgcn_readlane(rtile, i),
                 order.splits > 1 ? hp >> 16 : 0, order.splits > 1 ? hp & 0xffff : hp};
  }
  // The next group of items, those with rows; false at the end. The caller's item
  // moves to the lane that keeps it.
  __device__ inline bool group(const XOrder& order, int rows_per_item) {
    const XArgs& x = *x_args_again();
    const int lane = x_lane_again();
    const int cb = __builtin_amdgcn_readlane(b, cur), ct = __builtin_amdgcn_readlane(rtile, cur),
              ch = __builtin_amdgcn_readlane(hkpart, cur);
    while (first < end) {
      cur = at = kKept;
      const unsigned it = first + (lane >> 1) * turn + (lane & 1 ? step : 0);
      const bool in = lane < kTurns && it < end;
      const XItem m = x_item(in ? it : 0, (unsigned)x.B, order);
      int nq = x.Nq;
      if (x.cuq) {   // as x_sample
        const int64_t q0 = min(max((int64_t)x.cuq[m.b], (int64_t)0), x.Tq);
        nq = (int)min(min(max((int64_t)x.cuq[m.b + 1], q0), x.Tq) - q0, (int64_t)x.Nq);
      }
      b = lane == kKept ? cb : m.b;
      rtile = lane == kKept ? ct : m.tile;
      hkpart = lane == kKept ? ch : order.splits > 1 ? m.hk | m.part << 16 : m.hk;
      todo = __ballot(in && (int64_t)m.tile * rows_per_item < (int64_t)nq * x.G);
      first += kTurns / 2 * turn;
      if (todo) return true;
    }
    return false;
  }
  // The next tile; false at the end. changed: it is another item's than the one before.
  __device__ inline bool next(const XOrder& order, int rows_per_item, bool& changed) {
    changed = false;
    while (true) {
      if (tiles.next(tile, bits)) break;
      if (fresh) {
        bits = 0;
        break;
      }
      changed = true;
      if (todo == 0 && !group(order, rows_per_item)) return false;
      at = __builtin_ctzll(todo);
      todo &= todo - 1;
      const XItem m = item(at, order);
      const XArgs& x = *x_args_again();
      const XSample sm = x_sample(x, m.b);
      const int n = (sm.nk + kXKeys - 1) / kXKeys;
      int t0 = 0, t1 = n;
      if (order.splits > 1) {
        const int per = (n + (int)order.splits - 1) / (int)order.splits;
        t0 = min(m.part * per, n);
        t1 = min(t0 + per, n);
      }
      tiles.open(x.mask ? x.mask + sm.k0 : nullptr, sm.nk, t0, t1);
      k0 = sm.k0;
      hk = m.hk;
      keys = sm.nk;
      fresh = true;
    }
    fresh = false;
    return true;
  }
  // After an item's first tile: whether its sample has keys in use in one tile alone
  // (of which a split item may hold nothing: bits 0). Split items look through the
  // mask until they meet a second such tile: 1 us of a call where there is one in the
  // first 4,096 keys (dQ of 40 rows on 700 keys 16.8 -> 17.9 us), 8 us at 20 keys of
  // 16,391; unsplit ones have it from the walk.
  __device__ inline bool one_tile(const XOrder& order) const {
    const int n = (keys + kXKeys - 1) / kXKeys;
    if (n <= 1) return bits != 0;
    if (!tiles.mask) return false;
    KeyTiles t;   // the tiles not yet looked at; of a split item, all of the sample's
    int count = 0, from = 0;
    if (order.splits == 1) {
      if (tiles.left != 0) return false;
      count = bits != 0;
      from = tiles.base + 64;
    }
    t.open(tiles.mask, keys, from, n);
    for (t.base = from; t.base < n && count <= 1; t.base += 64) {
      t.group();
      count += __builtin_popcountll(t.left);
    }
    return count == 1;
  }
};

// 16 bytes a lane, or zeros for an offset of kXOut and more; stores from there on are
// dropped. Query rows and results pass once, so they are non-temporal and leave the
// L2 to the keys and values (packed case: dQ 443 -> 427 us, forward 305 -> 299).
constexpr int kXStream = 2;
__device__ inline bf16x8 x_load16(__amdgpu_buffer_rsrc_t rs, int off) {
  return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, kXStream));
}
__device__ inline void x_store16(bf16x8 v, __amdgpu_buffer_rsrc_t rs, int off) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rs, off, 0, kXStream);
}

// Byte offsets of a wave's rows r0 + lane / CPR + u RPI, u = 0 .., at the lane's 16-byte
// column: row r is token r / G and head r % G, which the step of RPI rows moves on
// without another division. Offsets count from the first row's token and head0 of
// it. Rows past the sample's nq tokens lie past the descriptor's range, and columns
// past D too: loads give zeros there, stores are dropped.
template <int DP>
struct XRows {
  static constexpr int CPR = DP / 8, RPI = 64 / CPR, N = DP / 16;   // N instructions of RPI rows
  int off[N];
  __amdgpu_buffer_rsrc_t rs;

  __device__ inline XRows(int lane, const void* base, int64_t tok0, int stride, int64_t head0, int r0, int nq, int G,
                          int D) {
    const int c = 8 * (lane % CPR), row0 = r0 + lane / CPR;
    int first = r0, tok = row0, head = 0;
    if (G != 1) {   // uniform
      first = (int)((unsigned)first / (unsigned)G);
      tok = (int)((unsigned)row0 / (unsigned)G), head = row0 - tok * G;
    }
    first = __builtin_amdgcn_readfirstlane(min(first, nq - 1));
    // at most 31 tokens behind the first of the wave (4 waves: 127 behind the last of
    // the sample): with strides up to kXMaxStride all of it stays below 2^31
    rs = buffer_rsrc(static_cast<const __bf16*>(base) + (tok0 + first) * stride + head0,
                     (min(nq - 1 - first, 32) * stride + G * D) * 2);
    off[0] = c < D ? ((tok - first) * stride + head * D + c) * 2 : kXOut;
    if (G == 1) {   // uniform
#pragma unroll
      for (int u = 1; u < N; ++u) off[u] = off[u - 1] + RPI * stride * 2;
    } else {
      const int dtok = RPI / G, dhead = RPI - dtok * G;
      const int step = (dtok * stride + dhead * D) * 2, wrap = (stride - G * D) * 2;
#pragma unroll
      for (int u = 1; u < N; ++u) {
        head += dhead;
        const bool over = head >= G;
        head -= over ? G : 0;
        off[u] = off[u - 1] + step + (over ? wrap : 0);
      }
    }
  }
};

// LDS offsets of a wave's 32 rows in its own part of a stage: row group 0 or 1 of 16
// rows in lds0 or lds1, swizzled as the tiles. As whole rows, lane / CPR + u RPI at the
// lane's column: the swizzle of the later ones differs by the bits of u alone.
template <int DP>
struct XTurn {
  static constexpr int CPR = DP / 8, ROWB = DP * 2, RPI = 64 / CPR, N = DP / 16, REP = 16 / RPI;
  int lane, row, column;
  __device__ inline explicit XTurn(int ln) : lane(ln) {
    row = lane / CPR * ROWB;
    column = lds_off<CPR>(lane / CPR, lane % CPR) & (ROWB - 1);
  }
  __device__ inline int whole(int u) const {
    const int k = u % REP;
    return row + (column ^ (CPR == 16 ? k << 4 : (4 * k) << 4)) + k * RPI * ROWB;
  }
  // Rows loaded whole to operands: op[ks] = columns 16 ks + 8 g .. of row l32.
  __device__ inline void turn(bf16x8 (&x)[N], char* lds0, char* lds1) const {
#pragma unroll
    for (int u = 0; u < N; ++u) *reinterpret_cast<bf16x8*>((u < REP ? lds0 : lds1) + whole(u)) = x[u];
    pin_order();
    const char* const from = (lane & 16) ? lds1 : lds0;
    const int op = lds_off<CPR>(lane & 15, lane >> 5);
#pragma unroll
    for (int ks = 0; ks < N; ++ks) x[ks] = *reinterpret_cast<const bf16x8*>(from + (op ^ (32 * ks)));
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the reads are done before the next writes
  }
};

// A wave's 32 operand rows r0 .. loaded as whole rows, 16 bytes a lane, to be turned
// into operands (XTurn): loaded as operands, an instruction would touch a line of
// every row.
template <int DP>
__device__ inline void x_load_rows(bf16x8 (&x)[DP / 16], const void* src, int64_t tok0, int stride, int64_t head0, int r0,
                                   int nq, int G, int D) {
  const XRows<DP> at(x_lane_again(), src, tok0, stride, head0, r0, nq, G, D);
#pragma unroll
  for (int u = 0; u < DP / 16; ++u) x[u] = x_load16(at.rs, at.off[u]);
}

// Stores a wave's 32 result rows, rounded to bf16, as whole rows, where the
// accumulators' layout would write pieces of 32 bytes: through the wave's own part of a
// consumed stage, which only the wave's own next loads write. val(dt, qg): columns
// 16 dt + 4 gq + (0..3) of row 16 qg + c16 of the rows r0 ...
template <int DP, class Val>
__device__ inline void x_store_rows(void* dst, int64_t tok0, int stride, int64_t head0, int r0, int nq, int G, int D,
                                    char* lds0, char* lds1, Val val) {
  constexpr int N = DP / 16;
  const XTurn<DP> t(x_lane_again());
  const int c16 = t.lane & 15, gq = t.lane >> 4, piece = lds_off<DP / 8>(c16, gq >> 1) + 8 * (gq & 1);
#pragma unroll
  for (int qg = 0; qg < 2; ++qg) {
#pragma unroll
    for (int dt = 0; dt < N; ++dt) {
      const f32x4 y = val(dt, qg);
      *reinterpret_cast<bf16x4*>((qg ? lds1 : lds0) + (piece ^ (32 * dt))) =
          bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
    }
    pin_order();
  }
  bf16x8 v[N];
#pragma unroll
  for (int u = 0; u < N; ++u) v[u] = *reinterpret_cast<const bf16x8*>((u < t.REP ? lds0 : lds1) + t.whole(u));
  const XRows<DP> at(t.lane, dst, tok0, stride, head0, r0, nq, G, D);   // beside the reads
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the reads are done before the next loads
#pragma unroll
  for (int u = 0; u < N; ++u) x_store16(v[u], at.rs, at.off[u]);
}

// Direct loads of 64-row tiles into LDS by NW waves, in rows of DP elements:
// instruction u of wave w writes 1 KB of rows. Within 16 rows the swizzle only
// flips bits of the column that the instruction's number gives, so a lane keeps
// its row's offset and its column, and the rest is scalar.
template <int DP, int NW>
struct TileLoad {
  static constexpr int ROWB = DP * 2, CPR = DP / 8;
  static constexpr int RPI = 1024 / ROWB;                      // rows per instruction
  static constexpr int IPW = kXKeys * ROWB / 1024 / NW;        // instructions per wave
  static constexpr int REP = 16 / RPI;                         // instructions of 16 rows
  static_assert(IPW % REP == 0, "a wave takes whole runs of 16 rows");
  int row;      // bytes from the instruction's first row to this lane's
  int column;   // this lane's byte in it, instruction 0

  __device__ inline TileLoad(int lane, int stride) {
    row = lane / CPR * stride * 2;
    column = (lds_off<CPR>(lane / CPR, lane % CPR) & (ROWB - 1));
  }
  // Instruction u's column: rows u RPI further on differ in the swizzle by u's
  // bits (CPR 16: rows 4 u + r, CPR 8: rows 8 u + r).
  static constexpr int flip(int u) { return CPR == 16 ? u << 4 : (4 * u) << 4; }

  // A tile's descriptor, from its first key's row of this head.
  __device__ inline __amdgpu_buffer_rsrc_t tile(const __bf16* src, int stride) const {
    const uint64_t p = (uint64_t)src;   // uniform: kept in scalar registers
    const uint64_t u = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((unsigned)(p >> 32)) << 32 |
                       (unsigned)__builtin_amdgcn_readfirstlane((unsigned)p);
    return buffer_rsrc((const void*)u, (kXKeys - 1) * stride * 2 + DP * 2);
  }
  // Instruction u of wave w of a tile whose keys are all in use. Columns past D
  // become zeros.
  __device__ inline void one(__amdgpu_buffer_rsrc_t rs, int stride, char* dst, int w, int u, int D) const {
    const int i = w * IPW + u, c = column ^ flip(u % REP);
    int step = RPI * stride * 2;   // not kept in a register for each instruction
    UT_DEV_ASM("" : "+s"(step));
    buffer_load_lds16(rs, dst + i * 1024, c < 2 * D ? row + c : kXOut, i * step);
  }
  // All of them, keys in `bits`: other rows become zeros too, whatever memory holds
  // there, and are not read.
  __device__ inline void masked(__amdgpu_buffer_rsrc_t rs, int stride, uint64_t bits, char* dst, int w, int lane,
                                int D) const {
#pragma unroll
    for (int u = 0; u < IPW; ++u) {
      const int i = w * IPW + u, c = column ^ flip(u % REP);
      const unsigned run = (unsigned)(bits >> (i * RPI));   // scalar: this instruction's rows
      buffer_load_lds16(rs, dst + i * 1024, run >> (lane / CPR) & 1 && c < 2 * D ? row + c : kXOut,
                        i * RPI * stride * 2);
    }
  }
};

}  // namespace ut
