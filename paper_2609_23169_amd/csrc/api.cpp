// Host side of the C ABI declared in include/ultratex.h: argument validation,
// workspace sizing, status codes and the per-thread error message. Every
// check runs before any launch; no exception leaves this file.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <exception>
#include <vector>

#include "common.h"

namespace ut {
namespace {
thread_local char g_last_error[512] = "";

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
}  // namespace

ut_status fail(ut_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
  va_end(ap);
  return st;
}

ut_status check_hip(hipError_t e, const char* what) {
  if (e == hipSuccess) return UT_OK;
  return fail(UT_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// ptr[0] = 0, ptr non-decreasing, ptr[rows] = the number of entries given, and
// each row's entries strictly ascending in [0, limit).
ut_status check_lists(const char* fn, const char* what, const int32_t* ptr, const int32_t* idx,
                      int64_t n_idx, int64_t rows, int32_t limit) {
  if (ptr[0] != 0)
    return fail(UT_ERR_INVALID_ARG, "%s: %s: pointers start at %d, not 0", fn, what, ptr[0]);
  for (int64_t r = 0; r < rows; ++r)
    if (ptr[r + 1] < ptr[r])
      return fail(UT_ERR_INVALID_ARG, "%s: %s: pointers decrease at row %lld", fn, what,
                  (long long)r);
  if (!idx) return UT_OK;   // pointers only
  if (ptr[rows] != n_idx)
    return fail(UT_ERR_INVALID_ARG, "%s: %s: pointers end at %d, not at the %lld entries", fn,
                what, ptr[rows], (long long)n_idx);
  for (int64_t r = 0; r < rows; ++r)
    for (int64_t e = ptr[r]; e < ptr[r + 1]; ++e) {
      if (idx[e] < 0 || idx[e] >= limit)
        return fail(UT_ERR_INVALID_ARG, "%s: %s: row %lld holds %d, outside [0, %d)", fn, what,
                    (long long)r, idx[e], limit);
      if (e > ptr[r] && idx[e] <= idx[e - 1])
        return fail(UT_ERR_INVALID_ARG, "%s: %s: row %lld is not strictly ascending", fn, what,
                    (long long)r);
    }
  return UT_OK;
}

ut_status check_cu_seqlens(const char* fn, const int32_t* cu, int32_t B, int64_t T,
                           int32_t max_seqlen) {
  if (cu[0] != 0 || cu[B] != T)
    return fail(UT_ERR_INVALID_ARG, "%s: cu_seqlens must run from 0 to T = %lld (got %d .. %d)",
                fn, (long long)T, cu[0], cu[B]);
  for (int32_t b = 0; b < B; ++b) {
    if (cu[b + 1] < cu[b])
      return fail(UT_ERR_INVALID_ARG, "%s: cu_seqlens decreases at sample %d", fn, b);
    if (cu[b + 1] - cu[b] > max_seqlen)
      return fail(UT_ERR_INVALID_ARG, "%s: sample %d has %d tokens > max_seqlen %d", fn, b,
                  cu[b + 1] - cu[b], max_seqlen);
  }
  return UT_OK;
}

namespace {

ut_status check_attn_common(const char* fn, int32_t B, int32_t N, int32_t H, int32_t D,
                            int32_t block, float scale) {
  if (B < 1 || N < 1 || H < 1)
    return fail(UT_ERR_INVALID_ARG, "%s: B, N, H must be >= 1 (got %d, %d, %d)", fn, B, N, H);
  if (D != 64 && D != 128)
    return fail(UT_ERR_UNSUPPORTED, "%s: head_dim %d unsupported (64 or 128)", fn, D);
  if (block != 64 && block != 128)
    return fail(UT_ERR_UNSUPPORTED, "%s: block %d unsupported (64 or 128)", fn, block);
  // the kernels keep a running maximum of the scaled scores and mask keys with
  // -inf scores; both need a positive scale
  if (!std::isfinite(scale) || !(scale > 0.f))
    return fail(UT_ERR_INVALID_ARG, "%s: softmax_scale must be finite and > 0 (got %g)", fn,
                (double)scale);
  const int64_t nblk = (N + block - 1) / block;
  if ((int64_t)B * H * nblk >= (int64_t)1 << 31 || (int64_t)B * N * H * D >= (int64_t)1 << 40)
    return fail(UT_ERR_INVALID_ARG, "%s: problem too large", fn);
  // the kernels bound their tile loads with 32-bit buffer ranges over one
  // sample's rows
  if ((int64_t)N * H * D * 2 >= (int64_t)1 << 31)
    return fail(UT_ERR_UNSUPPORTED, "%s: one sample's Q/K/V of %d x %d x %d bf16 reach 2 GiB", fn,
                N, H, D);
  return UT_OK;
}

ut_status check_ptr(const char* fn, const char* name, const void* p, uintptr_t align) {
  if (!p) return fail(UT_ERR_INVALID_ARG, "%s: %s is NULL", fn, name);
  if (!aligned(p, align))
    return fail(UT_ERR_INVALID_ARG, "%s: %s must be %zu-byte aligned", fn, name, (size_t)align);
  return UT_OK;
}

#define UT_TRY(x)                     \
  do {                                \
    ut_status _s = (x);               \
    if (_s != UT_OK) return _s;       \
  } while (0)

// ---- backward workspace: statistics planes, then the stored dS tiles ----
// Layout past the statistics (each part 256-byte aligned): a flag per query
// block row, the row-list entry -> tile map, then the tiles of 2 block^2 bytes.
constexpr size_t kDsAlign = 256;
size_t align_up(size_t x) { return (x + kDsAlign - 1) / kDsAlign * kDsAlign; }
size_t tiles_bytes(int64_t m, int32_t block) {
  return align_up((size_t)m * 4) + (size_t)m * 2 * block * block;
}

// Size with room for the dS tiles of nnz pairs (0 for invalid arguments).
size_t stored_size(size_t stats_bytes, int64_t rows, int32_t block, int64_t nnz) {
  if (stats_bytes == 0 || rows < 1 || (block != 64 && block != 128) || nnz < 0 ||
      nnz > ((int64_t)1 << 31) - 1)
    return 0;
  return align_up(stats_bytes) + align_up((size_t)rows * 4) + tiles_bytes(nnz, block);
}

// The tiles a workspace of `bytes` holds past the statistics (none: recompute dQ).
DsTiles ds_region(void* workspace, size_t bytes, size_t stats_bytes, int64_t rows, int32_t block) {
  DsTiles r;
  const size_t off = align_up(stats_bytes), flags = align_up((size_t)rows * 4);
  if (!workspace || bytes <= off + flags) return r;
  const size_t rem = bytes - off - flags;
  int64_t m = std::min<int64_t>((int64_t)(rem / ((size_t)2 * block * block + 4)),
                                ((int64_t)1 << 31) - 1);
  while (m > 0 && tiles_bytes(m, block) > rem) --m;
  if (m <= 0) return r;
  char* base = static_cast<char*>(workspace) + off;
  r.row_ok = reinterpret_cast<int32_t*>(base);
  r.map = reinterpret_cast<int32_t*>(base + flags);
  r.tiles = base + flags + align_up((size_t)m * 4);
  r.max_pairs = m;
  return r;
}
}  // namespace
}  // namespace ut

using namespace ut;

extern "C" {

const char* ut_last_error(void) { return g_last_error; }

int ut_abi_version(void) { return UT_ABI_VERSION; }

size_t ut_drop_background_workspace_size(int64_t L) {
  if (L < 1) return 0;
  return (size_t)compact_tiles(L) * sizeof(int32_t);
}

ut_status ut_drop_background(const uint8_t* fg_mask, int64_t L, const void* x_full,
                             int64_t row_bytes, void* x_packed, int64_t capacity,
                             int32_t* kept_idx, int32_t* inv_idx, int32_t* n_kept,
                             int64_t* n_kept_host, void* workspace, size_t workspace_bytes,
                             hipStream_t stream) {
  static const char* fn = "ut_drop_background";
  g_last_error[0] = 0;
  if (L < 1 || L >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: L must be in [1, 2^31) (got %lld)", fn, (long long)L);
  if (capacity < 0) return fail(UT_ERR_INVALID_ARG, "%s: capacity < 0", fn);
  UT_TRY(check_ptr(fn, "fg_mask", fg_mask, 1));
  UT_TRY(check_ptr(fn, "n_kept", n_kept, 4));
  if (capacity > 0) UT_TRY(check_ptr(fn, "kept_idx", kept_idx, 4));
  if (inv_idx) UT_TRY(check_ptr(fn, "inv_idx", inv_idx, 4));
  if ((x_full == nullptr) != (x_packed == nullptr))
    return fail(UT_ERR_INVALID_ARG, "%s: x_full and x_packed must both be NULL or both set", fn);
  if (x_full) {
    if (row_bytes <= 0 || row_bytes % 16 != 0)
      return fail(UT_ERR_INVALID_ARG, "%s: row_bytes must be a positive multiple of 16 (got %lld)",
                  fn, (long long)row_bytes);
    UT_TRY(check_ptr(fn, "x_full", x_full, 16));
    UT_TRY(check_ptr(fn, "x_packed", x_packed, 16));
  }
  const size_t need = ut_drop_background_workspace_size(L);
  if (!workspace || workspace_bytes < need)
    return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                workspace ? workspace_bytes : (size_t)0);
  UT_TRY(check_ptr(fn, "workspace", workspace, 4));

  UT_TRY(check_hip(launch_compact(fg_mask, L, capacity, kept_idx, inv_idx, n_kept,
                                  static_cast<int32_t*>(workspace), stream),
                   "compaction launch"));
  if (x_full)
    UT_TRY(check_hip(launch_gather(x_full, row_bytes, x_packed, capacity, kept_idx, n_kept, stream),
                     "gather launch"));
  if (n_kept_host) {
    int32_t n = 0;
    UT_TRY(check_hip(hipMemcpyAsync(&n, n_kept, sizeof(n), hipMemcpyDeviceToHost, stream),
                     "n_kept copy"));
    UT_TRY(check_hip(hipStreamSynchronize(stream), "stream sync"));
    *n_kept_host = n;
    if (n > capacity)
      return fail(UT_ERR_CAPACITY, "%s: %d kept positions exceed capacity %lld", fn, n,
                  (long long)capacity);
  }
  return UT_OK;
}

ut_status ut_scatter_foreground(const void* x_packed, const int32_t* kept_idx, int64_t n_kept,
                                int64_t row_bytes, void* x_full, hipStream_t stream) {
  static const char* fn = "ut_scatter_foreground";
  g_last_error[0] = 0;
  if (n_kept < 0 || n_kept >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: n_kept out of range", fn);
  if (row_bytes <= 0 || row_bytes % 16 != 0)
    return fail(UT_ERR_INVALID_ARG, "%s: row_bytes must be a positive multiple of 16", fn);
  if (n_kept == 0) return UT_OK;
  UT_TRY(check_ptr(fn, "x_packed", x_packed, 16));
  UT_TRY(check_ptr(fn, "x_full", x_full, 16));
  UT_TRY(check_ptr(fn, "kept_idx", kept_idx, 4));
  return check_hip(launch_scatter(x_packed, kept_idx, n_kept, row_bytes, x_full, stream),
                   "scatter launch");
}

size_t ut_build_block_index_workspace_size(int32_t B, int32_t H, int32_t Nq, int32_t Nk) {
  // the counts are scanned in place inside q_rowptr / kv_colptr: no scratch
  (void)B, (void)H, (void)Nq, (void)Nk;
  return 0;
}

ut_status ut_build_block_index(const uint8_t* block_mask, int32_t B, int32_t H, int32_t Nq,
                               int32_t Nk, int32_t* q_rowptr, int32_t* q_cols,
                               int32_t* kv_colptr, int32_t* kv_rows, int64_t cap,
                               int64_t* nnz_host, void* workspace, size_t workspace_bytes,
                               hipStream_t stream) {
  static const char* fn = "ut_build_block_index";
  g_last_error[0] = 0;
  if (B < 1 || H < 1 || Nq < 1 || Nk < 1)
    return fail(UT_ERR_INVALID_ARG, "%s: B, H, Nq, Nk must be >= 1", fn);
  if ((int64_t)B * H > 65535)
    return fail(UT_ERR_INVALID_ARG, "%s: B*H must be <= 65535 (got %lld)", fn,
                (long long)B * H);
  // list offsets are int32: the mask may not hold 2^31 entries
  if ((int64_t)B * H * Nq * Nk >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: B*H*Nq*Nk = %lld reaches 2^31 (int32 offsets)", fn,
                (long long)B * H * Nq * Nk);
  if (cap < 0) return fail(UT_ERR_INVALID_ARG, "%s: cap < 0", fn);
  UT_TRY(check_ptr(fn, "block_mask", block_mask, 1));
  UT_TRY(check_ptr(fn, "q_rowptr", q_rowptr, 4));
  UT_TRY(check_ptr(fn, "kv_colptr", kv_colptr, 4));
  if (cap > 0) {
    UT_TRY(check_ptr(fn, "q_cols", q_cols, 4));
    UT_TRY(check_ptr(fn, "kv_rows", kv_rows, 4));
  }
  const size_t need = ut_build_block_index_workspace_size(B, H, Nq, Nk);
  if (workspace_bytes < need || (need > 0 && !workspace))
    return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                workspace ? workspace_bytes : (size_t)0);
  UT_TRY(check_hip(launch_block_index(block_mask, B, H, Nq, Nk, q_rowptr, q_cols, kv_colptr,
                                      kv_rows, cap, stream),
                   "block index launch"));
  if (nnz_host) {
    int32_t nnz = 0;
    UT_TRY(check_hip(hipMemcpyAsync(&nnz, q_rowptr + (int64_t)B * H * Nq, sizeof(nnz),
                                    hipMemcpyDeviceToHost, stream),
                     "nnz copy"));
    UT_TRY(check_hip(hipStreamSynchronize(stream), "stream sync"));
    *nnz_host = nnz;
    if (nnz < 0 || nnz > cap)
      return fail(UT_ERR_CAPACITY, "%s: %d retained pairs exceed cap %lld", fn, nnz,
                  (long long)cap);
  }
  return UT_OK;
}

namespace {
// Opt-in checking of the block lists' contents (environment UT_VALIDATE set to
// anything but "0"): a debugging aid, since it waits for the stream.
bool validate_mode() {
  const char* e = std::getenv("UT_VALIDATE");
  return e && e[0] && !(e[0] == '0' && e[1] == 0);
}

// `count` device values to the host, when the stream has come there. No exception
// leaves the C entries: host memory that runs out is an error like the device's.
ut_status validate_copy(const int32_t* src, size_t count, std::vector<int32_t>* out, hipStream_t stream) {
  try {
    out->resize(count);
  } catch (const std::exception&) {   // bad_alloc, length_error
    return check_hip(hipErrorOutOfMemory, "validate copy");
  }
  if (count == 0) return UT_OK;
  UT_TRY(check_hip(hipMemcpyAsync(out->data(), src, count * sizeof(int32_t), hipMemcpyDeviceToHost, stream),
                   "validate copy"));
  return check_hip(hipStreamSynchronize(stream), "validate sync");
}

// Copies a compressed list pair to the host and checks it with check_lists.
ut_status validate_lists(const char* fn, const char* what, const int32_t* ptr, const int32_t* idx,
                         int64_t rows, int32_t limit, hipStream_t stream) {
  std::vector<int32_t> p, v;
  UT_TRY(validate_copy(ptr, (size_t)rows + 1, &p, stream));
  // well-formed pointers first, so that p[rows] is a sane entry count
  UT_TRY(check_lists(fn, what, p.data(), nullptr, 0, rows, limit));
  UT_TRY(validate_copy(idx, (size_t)p[rows], &v, stream));
  return check_lists(fn, what, p.data(), v.data(), (int64_t)v.size(), rows, limit);
}
}  // namespace

ut_status ut_bsattn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                        int32_t B, int32_t N, int32_t H, int32_t D, int32_t block,
                        const int32_t* q_rowptr, const int32_t* q_cols, float softmax_scale,
                        hipStream_t stream) {
  static const char* fn = "ut_bsattn_fwd";
  g_last_error[0] = 0;
  UT_TRY(check_attn_common(fn, B, N, H, D, block, softmax_scale));
  UT_TRY(check_ptr(fn, "q", q, 16));
  UT_TRY(check_ptr(fn, "k", k, 16));
  UT_TRY(check_ptr(fn, "v", v, 16));
  UT_TRY(check_ptr(fn, "o", o, 16));
  UT_TRY(check_ptr(fn, "lse", lse, 4));
  UT_TRY(check_ptr(fn, "q_rowptr", q_rowptr, 4));
  UT_TRY(check_ptr(fn, "q_cols", q_cols, 4));
  const AttnShape sh{B, N, H, D, block, (N + block - 1) / block, softmax_scale, nullptr,
                     (int64_t)B * N};
  if (validate_mode())
    UT_TRY(validate_lists(fn, "row lists", q_rowptr, q_cols, (int64_t)B * H * sh.nblk, sh.nblk,
                          stream));
  return check_hip(launch_bsattn_fwd(q, k, v, o, lse, sh, q_rowptr, q_cols, stream),
                   "forward launch");
}

size_t ut_bsattn_bwd_workspace_size(int32_t B, int32_t N, int32_t H) {
  if (B < 1 || N < 1 || H < 1) return 0;
  return (size_t)B * H * N * 2 * sizeof(float);   // {LSE log2 e, delta} per query row
}


size_t ut_bsattn_bwd_workspace_size_stored(int32_t B, int32_t N, int32_t H, int32_t block,
                                           int64_t nnz) {
  if (block < 1) return 0;
  return stored_size(ut_bsattn_bwd_workspace_size(B, N, H),
                     (int64_t)B * H * (((int64_t)N + block - 1) / block), block, nnz);
}

ut_status ut_bsattn_bwd(const void* q, const void* k, const void* v, const void* o,
                        const void* dout, const float* lse, void* dq, void* dk, void* dv,
                        int32_t B, int32_t N, int32_t H, int32_t D, int32_t block,
                        const int32_t* q_rowptr, const int32_t* q_cols,
                        const int32_t* kv_colptr, const int32_t* kv_rows, float softmax_scale,
                        void* workspace, size_t workspace_bytes, hipStream_t stream) {
  static const char* fn = "ut_bsattn_bwd";
  g_last_error[0] = 0;
  UT_TRY(check_attn_common(fn, B, N, H, D, block, softmax_scale));
  const struct { const char* n; const void* p; uintptr_t a; } ptrs[] = {
      {"q", q, 16},   {"k", k, 16},   {"v", v, 16},         {"o", o, 16},
      {"dout", dout, 16}, {"lse", lse, 4}, {"dq", dq, 16},   {"dk", dk, 16},
      {"dv", dv, 16}, {"q_rowptr", q_rowptr, 4}, {"q_cols", q_cols, 4},
      {"kv_colptr", kv_colptr, 4}, {"kv_rows", kv_rows, 4}};
  for (const auto& p : ptrs) UT_TRY(check_ptr(fn, p.n, p.p, p.a));
  const size_t need = ut_bsattn_bwd_workspace_size(B, N, H);
  if (!workspace || workspace_bytes < need)
    return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                workspace ? workspace_bytes : (size_t)0);
  UT_TRY(check_ptr(fn, "workspace", workspace, 16));
  const AttnShape sh{B, N, H, D, block, (N + block - 1) / block, softmax_scale, nullptr,
                     (int64_t)B * N};
  if (validate_mode()) {
    UT_TRY(validate_lists(fn, "row lists", q_rowptr, q_cols, (int64_t)B * H * sh.nblk, sh.nblk,
                          stream));
    UT_TRY(validate_lists(fn, "column lists", kv_colptr, kv_rows, (int64_t)B * H * sh.nblk,
                          sh.nblk, stream));
  }
  const DsTiles ds = ds_region(workspace, workspace_bytes, need, (int64_t)B * H * sh.nblk, block);
  return check_hip(launch_bsattn_bwd(q, k, v, o, dout, lse, dq, dk, dv, sh, q_rowptr, q_cols,
                                     kv_colptr, kv_rows, static_cast<float*>(workspace), ds,
                                     stream),
                   "backward launch");
}

ut_status ut_bsattn_bwd_noalloc(const void* q, const void* k, const void* v, const void* o,
                                const void* dout, const float* lse, void* dq, void* dk, void* dv,
                                int32_t B, int32_t N, int32_t H, int32_t D, int32_t block,
                                const int32_t* q_rowptr, const int32_t* q_cols,
                                const int32_t* kv_colptr, const int32_t* kv_rows,
                                float softmax_scale, hipStream_t stream) {
  static const char* fn = "ut_bsattn_bwd_noalloc";
  g_last_error[0] = 0;
  UT_TRY(check_attn_common(fn, B, N, H, D, block, softmax_scale));
  const struct { const char* n; const void* p; uintptr_t a; } ptrs[] = {
      {"q", q, 16},   {"k", k, 16},   {"v", v, 16},         {"o", o, 16},
      {"dout", dout, 16}, {"lse", lse, 4}, {"dq", dq, 16},   {"dk", dk, 16},
      {"dv", dv, 16}, {"q_rowptr", q_rowptr, 4}, {"q_cols", q_cols, 4},
      {"kv_colptr", kv_colptr, 4}, {"kv_rows", kv_rows, 4}};
  for (const auto& p : ptrs) UT_TRY(check_ptr(fn, p.n, p.p, p.a));
  const size_t need = ut_bsattn_bwd_workspace_size(B, N, H);
  if (need > kNoallocScratchBytes)
    return fail(UT_ERR_WORKSPACE,
                "%s: B*H*N = %lld query rows need %zu bytes of scratch; the built-in scratch "
                "holds %zu bytes (%zu rows): use ut_bsattn_bwd with a workspace",
                fn, (long long)B * H * N, need, kNoallocScratchBytes,
                kNoallocScratchBytes / (2 * sizeof(float)));
  float* ws = nullptr;
  UT_TRY(check_hip(noalloc_scratch(stream, &ws), "scratch address"));
  const AttnShape sh{B, N, H, D, block, (N + block - 1) / block, softmax_scale, nullptr,
                     (int64_t)B * N};
  return check_hip(launch_bsattn_bwd(q, k, v, o, dout, lse, dq, dk, dv, sh, q_rowptr, q_cols,
                                     kv_colptr, kv_rows, ws, DsTiles{}, stream),
                   "backward launch");
}

namespace {
// Sample offsets of the variable-length calls: B + 1 device int32 values.
// Under UT_VALIDATE they are copied to the host and must start at 0, end at
// T and never decrease, with no sample longer than max_seqlen.
ut_status check_varlen(const char* fn, const int32_t* cu_seqlens, int32_t B, int64_t T,
                       int32_t max_seqlen, hipStream_t stream) {
  UT_TRY(check_ptr(fn, "cu_seqlens", cu_seqlens, 4));
  if (T < 0 || T >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: T = %lld outside [0, 2^31)", fn, (long long)T);
  if (!validate_mode()) return UT_OK;
  std::vector<int32_t> cu;
  UT_TRY(validate_copy(cu_seqlens, (size_t)B + 1, &cu, stream));
  return check_cu_seqlens(fn, cu.data(), B, T, max_seqlen);
}
}  // namespace

ut_status ut_bsattn_fwd_varlen(const void* q, const void* k, const void* v, void* o, float* lse,
                               const int32_t* cu_seqlens, int32_t B, int64_t T,
                               int32_t max_seqlen, int32_t H, int32_t D, int32_t block,
                               const int32_t* q_rowptr, const int32_t* q_cols,
                               float softmax_scale, hipStream_t stream) {
  static const char* fn = "ut_bsattn_fwd_varlen";
  g_last_error[0] = 0;
  UT_TRY(check_attn_common(fn, B, max_seqlen, H, D, block, softmax_scale));
  UT_TRY(check_varlen(fn, cu_seqlens, B, T, max_seqlen, stream));
  if (T * H * D >= (int64_t)1 << 40) return fail(UT_ERR_INVALID_ARG, "%s: problem too large", fn);
  if (T == 0) return UT_OK;
  UT_TRY(check_ptr(fn, "q", q, 16));
  UT_TRY(check_ptr(fn, "k", k, 16));
  UT_TRY(check_ptr(fn, "v", v, 16));
  UT_TRY(check_ptr(fn, "o", o, 16));
  UT_TRY(check_ptr(fn, "lse", lse, 4));
  UT_TRY(check_ptr(fn, "q_rowptr", q_rowptr, 4));
  UT_TRY(check_ptr(fn, "q_cols", q_cols, 4));
  const AttnShape sh{B, max_seqlen, H, D, block, (max_seqlen + block - 1) / block,
                     softmax_scale, cu_seqlens, T};
  if (validate_mode())
    UT_TRY(validate_lists(fn, "row lists", q_rowptr, q_cols, (int64_t)B * H * sh.nblk, sh.nblk,
                          stream));
  return check_hip(launch_bsattn_fwd(q, k, v, o, lse, sh, q_rowptr, q_cols, stream),
                   "forward launch");
}

size_t ut_bsattn_bwd_varlen_workspace_size(int64_t T, int32_t H) {
  if (T < 1 || H < 1) return 0;
  return (size_t)T * H * 2 * sizeof(float);
}

size_t ut_bsattn_bwd_varlen_workspace_size_stored(int32_t B, int64_t T, int32_t max_seqlen,
                                                  int32_t H, int32_t block, int64_t nnz) {
  if (B < 1 || max_seqlen < 1 || block < 1) return 0;
  return stored_size(ut_bsattn_bwd_varlen_workspace_size(T, H),
                     (int64_t)B * H * (((int64_t)max_seqlen + block - 1) / block), block, nnz);
}

ut_status ut_bsattn_bwd_varlen(const void* q, const void* k, const void* v, const void* o,
                               const void* dout, const float* lse, void* dq, void* dk, void* dv,
                               const int32_t* cu_seqlens, int32_t B, int64_t T,
                               int32_t max_seqlen, int32_t H, int32_t D, int32_t block,
                               const int32_t* q_rowptr, const int32_t* q_cols,
                               const int32_t* kv_colptr, const int32_t* kv_rows,
                               float softmax_scale, void* workspace, size_t workspace_bytes,
                               hipStream_t stream) {
  static const char* fn = "ut_bsattn_bwd_varlen";
  g_last_error[0] = 0;
  UT_TRY(check_attn_common(fn, B, max_seqlen, H, D, block, softmax_scale));
  UT_TRY(check_varlen(fn, cu_seqlens, B, T, max_seqlen, stream));
  if (T * H * D >= (int64_t)1 << 40) return fail(UT_ERR_INVALID_ARG, "%s: problem too large", fn);
  if (T == 0) return UT_OK;
  const struct { const char* n; const void* p; uintptr_t a; } ptrs[] = {
      {"q", q, 16},   {"k", k, 16},   {"v", v, 16},         {"o", o, 16},
      {"dout", dout, 16}, {"lse", lse, 4}, {"dq", dq, 16},   {"dk", dk, 16},
      {"dv", dv, 16}, {"q_rowptr", q_rowptr, 4}, {"q_cols", q_cols, 4},
      {"kv_colptr", kv_colptr, 4}, {"kv_rows", kv_rows, 4}};
  for (const auto& p : ptrs) UT_TRY(check_ptr(fn, p.n, p.p, p.a));
  const size_t need = ut_bsattn_bwd_varlen_workspace_size(T, H);
  if (!workspace || workspace_bytes < need)
    return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                workspace ? workspace_bytes : (size_t)0);
  UT_TRY(check_ptr(fn, "workspace", workspace, 16));
  const AttnShape sh{B, max_seqlen, H, D, block, (max_seqlen + block - 1) / block,
                     softmax_scale, cu_seqlens, T};
  if (validate_mode()) {
    UT_TRY(validate_lists(fn, "row lists", q_rowptr, q_cols, (int64_t)B * H * sh.nblk, sh.nblk,
                          stream));
    UT_TRY(validate_lists(fn, "column lists", kv_colptr, kv_rows, (int64_t)B * H * sh.nblk,
                          sh.nblk, stream));
  }
  const DsTiles ds = ds_region(workspace, workspace_bytes, need, (int64_t)B * H * sh.nblk, block);
  return check_hip(launch_bsattn_bwd(q, k, v, o, dout, lse, dq, dk, dv, sh, q_rowptr, q_cols,
                                     kv_colptr, kv_rows, static_cast<float*>(workspace), ds,
                                     stream),
                   "backward launch");
}

size_t ut_topk_block_mask_workspace_size(int32_t B, int32_t N, int32_t H, int32_t D,
                                         int32_t block) {
  if (B < 1 || N < 1 || H < 1 || D < 1 || block < 1) return 0;
  const int64_t nblk = ((int64_t)N + block - 1) / block;
  return (size_t)2 * B * H * nblk * D * sizeof(float);   // pooled Q and K
}

ut_status ut_topk_block_mask(const void* q, const void* k, int32_t B, int32_t N, int32_t H,
                             int32_t D, int32_t block, int32_t k_keep, int32_t prefix_blocks,
                             uint8_t* block_mask, void* workspace, size_t workspace_bytes,
                             hipStream_t stream) {
  static const char* fn = "ut_topk_block_mask";
  g_last_error[0] = 0;
  if (B < 1 || N < 1 || H < 1 || block < 1)
    return fail(UT_ERR_INVALID_ARG, "%s: B, N, H, block must be >= 1 (got %d, %d, %d, %d)", fn,
                B, N, H, block);
  if (D < 8 || D > 512 || D % 8 != 0)
    return fail(UT_ERR_INVALID_ARG, "%s: head_dim must be a multiple of 8 in [8, 512] (got %d)",
                fn, D);
  if (B > 65535) return fail(UT_ERR_INVALID_ARG, "%s: B must be <= 65535 (got %d)", fn, B);
  if (k_keep < 1) return fail(UT_ERR_INVALID_ARG, "%s: k_keep must be >= 1 (got %d)", fn, k_keep);
  const int64_t nblk = ((int64_t)N + block - 1) / block;
  if ((int64_t)B * N * H * D >= (int64_t)1 << 40 || (int64_t)B * H * nblk >= (int64_t)1 << 31)
    return fail(UT_ERR_INVALID_ARG, "%s: problem too large", fn);
  if (prefix_blocks < 0 || prefix_blocks > nblk)
    return fail(UT_ERR_INVALID_ARG, "%s: prefix_blocks must be in [0, %lld] (got %d)", fn,
                (long long)nblk, prefix_blocks);
  if (topk_rows_per_group(D, (int)nblk) == 0)
    return fail(UT_ERR_UNSUPPORTED, "%s: %lld blocks per row do not fit one workgroup", fn,
                (long long)nblk);
  UT_TRY(check_ptr(fn, "q", q, 16));
  UT_TRY(check_ptr(fn, "k", k, 16));
  UT_TRY(check_ptr(fn, "block_mask", block_mask, 1));
  const size_t need = ut_topk_block_mask_workspace_size(B, N, H, D, block);
  if (!workspace || workspace_bytes < need)
    return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                workspace ? workspace_bytes : (size_t)0);
  UT_TRY(check_ptr(fn, "workspace", workspace, 16));
  return check_hip(launch_topk_block_mask(q, k, B, N, H, D, block, k_keep, prefix_blocks,
                                          block_mask, static_cast<float*>(workspace), stream),
                   "top-k launch");
}

namespace {
ut_status check_fg_common(const char* fn, int64_t L, int64_t C, int64_t n, const void* v,
                          ut_dtype vt) {
  if (L < 1 || L >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: L must be in [1, 2^31) (got %lld)", fn, (long long)L);
  if (C < 4 || C % 4 != 0 || C > (1 << 20))
    return fail(UT_ERR_INVALID_ARG, "%s: C must be a positive multiple of 4 (got %lld)", fn,
                (long long)C);
  if (n < 0 || n > L)
    return fail(UT_ERR_INVALID_ARG, "%s: n_kept must be in [0, L] (got %lld)", fn, (long long)n);
  if (vt != UT_BF16 && vt != UT_F32)
    return fail(UT_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, (int)vt);
  if (n > 0) UT_TRY(check_ptr(fn, "v", v, vt == UT_BF16 ? 8 : 16));
  return UT_OK;
}
}  // namespace

ut_status ut_euler_update_foreground(float* z, int64_t L, int64_t C, const void* v,
                                     ut_dtype v_dtype, const int32_t* kept_idx,
                                     int64_t n_kept, float dt, hipStream_t stream) {
  static const char* fn = "ut_euler_update_foreground";
  g_last_error[0] = 0;
  UT_TRY(check_fg_common(fn, L, C, n_kept, v, v_dtype));
  if (!std::isfinite(dt)) return fail(UT_ERR_INVALID_ARG, "%s: dt must be finite", fn);
  if (n_kept == 0) return UT_OK;
  UT_TRY(check_ptr(fn, "z", z, 16));
  UT_TRY(check_ptr(fn, "kept_idx", kept_idx, 4));
  return check_hip(launch_euler_fg(z, L, C, v, v_dtype == UT_BF16, kept_idx, n_kept, dt, stream),
                   "euler launch");
}

size_t ut_fg_flow_loss_workspace_size(void) { return (size_t)kLossParts * sizeof(double); }

ut_status ut_fg_flow_loss(const void* v, ut_dtype v_dtype, const void* eps, const void* z0,
                          ut_dtype x_dtype, int64_t L, int64_t C, const int32_t* kept_idx,
                          int64_t n_kept, float* loss, float* grad, void* workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  static const char* fn = "ut_fg_flow_loss";
  g_last_error[0] = 0;
  UT_TRY(check_fg_common(fn, L, C, n_kept, v, v_dtype));
  if (x_dtype != UT_BF16 && x_dtype != UT_F32)
    return fail(UT_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, (int)x_dtype);
  UT_TRY(check_ptr(fn, "loss", loss, 4));
  if (n_kept > 0) {
    const uintptr_t xa = x_dtype == UT_BF16 ? 8 : 16;
    UT_TRY(check_ptr(fn, "eps", eps, xa));
    UT_TRY(check_ptr(fn, "z0", z0, xa));
    UT_TRY(check_ptr(fn, "kept_idx", kept_idx, 4));
    if (grad) UT_TRY(check_ptr(fn, "grad", grad, 16));
  }
  const size_t need = ut_fg_flow_loss_workspace_size();
  if (!workspace || workspace_bytes < need)
    return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                workspace ? workspace_bytes : (size_t)0);
  UT_TRY(check_ptr(fn, "workspace", workspace, 8));
  return check_hip(launch_fg_loss(v, v_dtype == UT_BF16, eps, z0, x_dtype == UT_BF16, L, C,
                                  kept_idx, n_kept, loss, grad, static_cast<double*>(workspace),
                                  stream),
                   "loss launch");
}

ut_status ut_composite_latent(const void* x_packed, int64_t n_kept, const int32_t* inv_idx,
                              int64_t L, const void* z_bg, int64_t bg_rows, int64_t row_bytes,
                              void* z_mix, hipStream_t stream) {
  static const char* fn = "ut_composite_latent";
  g_last_error[0] = 0;
  if (L < 1 || L >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: L must be in [1, 2^31) (got %lld)", fn, (long long)L);
  if (bg_rows < 1)
    return fail(UT_ERR_INVALID_ARG, "%s: bg_rows must be >= 1 (got %lld)", fn, (long long)bg_rows);
  if (n_kept < 0 || n_kept > L)
    return fail(UT_ERR_INVALID_ARG, "%s: n_kept must be in [0, L] (got %lld)", fn, (long long)n_kept);
  if (row_bytes <= 0 || row_bytes % 16 != 0)
    return fail(UT_ERR_INVALID_ARG, "%s: row_bytes must be a positive multiple of 16 (got %lld)",
                fn, (long long)row_bytes);
  if (n_kept > 0) UT_TRY(check_ptr(fn, "x_packed", x_packed, 16));
  UT_TRY(check_ptr(fn, "inv_idx", inv_idx, 4));
  UT_TRY(check_ptr(fn, "z_bg", z_bg, 16));
  UT_TRY(check_ptr(fn, "z_mix", z_mix, 16));
  return check_hip(launch_composite(x_packed, n_kept, inv_idx, L, z_bg, bg_rows, row_bytes, z_mix,
                                    stream),
                   "composite launch");
}

size_t ut_token_mask_workspace_size(int32_t V, int32_t Hp, int32_t Wp, int32_t patch) {
  if (V < 1 || Hp < 1 || Wp < 1 || patch < 1) return 0;
  return (size_t)V * (Hp / patch) * (Wp / patch);
}

ut_status ut_token_mask_from_alpha(const uint8_t* alpha, int32_t V, int32_t Hp, int32_t Wp,
                                   int32_t patch, int32_t threshold, int32_t radius,
                                   uint8_t* token_mask, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
  static const char* fn = "ut_token_mask_from_alpha";
  g_last_error[0] = 0;
  if (V < 1 || Hp < 1 || Wp < 1)
    return fail(UT_ERR_INVALID_ARG, "%s: V, Hp, Wp must be >= 1", fn);
  if (patch < 16 || patch % 16 != 0 || Hp % patch != 0 || Wp % patch != 0)
    return fail(UT_ERR_INVALID_ARG,
                "%s: patch must be a positive multiple of 16 dividing Hp and Wp (got %d for %d x %d)",
                fn, patch, Hp, Wp);
  if (threshold < 0 || threshold > 255)
    return fail(UT_ERR_INVALID_ARG, "%s: threshold must be in [0, 255] (got %d)", fn, threshold);
  if (radius < 0 || radius > 16)
    return fail(UT_ERR_INVALID_ARG, "%s: radius must be in [0, 16] (got %d)", fn, radius);
  if ((int64_t)V * Hp * Wp >= ((int64_t)1 << 40))
    return fail(UT_ERR_INVALID_ARG, "%s: alpha too large", fn);
  UT_TRY(check_ptr(fn, "alpha", alpha, 16));
  UT_TRY(check_ptr(fn, "token_mask", token_mask, 1));
  if (radius > 0) {
    const size_t need = ut_token_mask_workspace_size(V, Hp, Wp, patch);
    if (!workspace || workspace_bytes < need)
      return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                  workspace ? workspace_bytes : (size_t)0);
  }
  return check_hip(launch_token_mask(alpha, V, Hp, Wp, patch, threshold, radius, token_mask,
                                     static_cast<uint8_t*>(workspace), stream),
                   "token mask launch");
}

namespace {
// Shape, strides and positions shared by the two rotary calls; fills sh.
ut_status check_rope(const char* fn, int64_t n, int32_t Hq, int32_t Hk, int32_t D, ut_dtype dtype,
                     const float* pos, int64_t pos_rows, const int32_t* token_idx,
                     const int32_t* axis_dims_host, int32_t n_axes, double theta,
                     ut_rope_pairs pairs, const void* q_weight, const void* k_weight,
                     ut_dtype w_dtype, float eps, RopeShape* sh) {
  if (n < 0 || n >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: n must be in [0, 2^31) (got %lld)", fn, (long long)n);
  if (Hq < 1 || Hk < 0)
    return fail(UT_ERR_INVALID_ARG, "%s: Hq must be >= 1 and Hk >= 0 (got %d, %d)", fn, Hq, Hk);
  if (Hq > 65536 || Hk > 65536)
    return fail(UT_ERR_INVALID_ARG, "%s: more than 65536 heads (%d, %d)", fn, Hq, Hk);
  if (D < 8 || D % 8 != 0 || D > kRopeMaxDim)
    return fail(UT_ERR_UNSUPPORTED, "%s: head_dim %d unsupported (a multiple of 8 up to %d)", fn, D,
                kRopeMaxDim);
  if (dtype != UT_BF16 && dtype != UT_F32)
    return fail(UT_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, (int)dtype);
  if (pairs != UT_ROPE_NEAR && pairs != UT_ROPE_FAR)
    return fail(UT_ERR_INVALID_ARG, "%s: unknown pair layout %d", fn, (int)pairs);
  if (!axis_dims_host || n_axes < 1 || n_axes > kRopeMaxAxes)
    return fail(UT_ERR_INVALID_ARG, "%s: 1 to %d axes and their sizes are needed (got %d)", fn,
                kRopeMaxAxes, n_axes);
  int64_t sum = 0;
  for (int x = 0; x < n_axes; ++x) {
    if (axis_dims_host[x] < 2 || axis_dims_host[x] % 2 != 0)
      return fail(UT_ERR_INVALID_ARG, "%s: axis %d: size must be positive and even (got %d)", fn, x,
                  axis_dims_host[x]);
    sh->dims[x] = axis_dims_host[x];
    sum += axis_dims_host[x];
  }
  if (sum > D)
    return fail(UT_ERR_INVALID_ARG, "%s: the axes take %lld elements of a head of %d", fn,
                (long long)sum, D);
  if (pairs == UT_ROPE_FAR && sum % 8 != 0)
    return fail(UT_ERR_UNSUPPORTED, "%s: far pairs need axes of a multiple of 8 in all (got %lld)",
                fn, (long long)sum);
  if (!std::isfinite(theta) || !(theta > 0.0))
    return fail(UT_ERR_INVALID_ARG, "%s: theta must be finite and > 0 (got %g)", fn, theta);
  if (pos_rows < 1 || pos_rows >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: pos_rows must be in [1, 2^31) (got %lld)", fn,
                (long long)pos_rows);
  UT_TRY(check_ptr(fn, "pos", pos, 4));
  if (token_idx && !aligned(token_idx, 4))
    return fail(UT_ERR_INVALID_ARG, "%s: token_idx must be 4-byte aligned", fn);
  if (Hk > 0 && (q_weight == nullptr) != (k_weight == nullptr))
    return fail(UT_ERR_INVALID_ARG, "%s: q_weight and k_weight must both be NULL or both set", fn);
  if (q_weight) {
    if (w_dtype != UT_BF16 && w_dtype != UT_F32)
      return fail(UT_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, (int)w_dtype);
    const uintptr_t wa = w_dtype == UT_BF16 ? 2 : 4;
    UT_TRY(check_ptr(fn, "q_weight", q_weight, wa));
    if (Hk > 0) UT_TRY(check_ptr(fn, "k_weight", k_weight, wa));
    if (!std::isfinite(eps) || !(eps > 0.f))
      return fail(UT_ERR_INVALID_ARG, "%s: eps must be finite and > 0 (got %g)", fn, (double)eps);
  }
  sh->n = n;
  sh->D = D;
  sh->bf16 = dtype == UT_BF16;
  sh->w_bf16 = w_dtype == UT_BF16;
  sh->far_pairs = pairs == UT_ROPE_FAR;
  sh->pos = pos;
  sh->pos_rows = pos_rows;
  sh->idx = token_idx;
  sh->n_axes = n_axes;
  sh->theta = theta;
  sh->eps = eps;
  return UT_OK;
}

// Token stride i of `strides_host` (NULL: rows of H heads back to back): whole
// rows apart, and in steps of `step` elements, so that rows stay aligned.
ut_status check_stride(const char* fn, const char* name, const int64_t* strides_host, int i,
                       int64_t row, int64_t step, int64_t limit, int64_t* out) {
  *out = strides_host ? strides_host[i] : row;
  if (*out < row || *out % step != 0)
    return fail(UT_ERR_INVALID_ARG,
                "%s: stride of %s must be a multiple of %lld and at least a row of %lld (got %lld)", fn,
                name, (long long)step, (long long)row, (long long)*out);
  if (*out >= limit)
    return fail(UT_ERR_UNSUPPORTED, "%s: stride of %s must be below %lld elements (got %lld)", fn,
                name, (long long)limit, (long long)*out);
  return UT_OK;
}
constexpr int64_t kRopeMaxStride = (int64_t)1 << 31;
}  // namespace

ut_status ut_qk_rope_fwd(const void* q, const void* k, void* q_out, void* k_out,
                         const int64_t* strides_host, ut_dtype dtype, int64_t n, int32_t Hq,
                         int32_t Hk, int32_t D, const float* pos, int64_t pos_rows,
                         const int32_t* token_idx, const int32_t* axis_dims_host, int32_t n_axes,
                         double theta, ut_rope_pairs pairs, const void* q_weight,
                         const void* k_weight, ut_dtype w_dtype, float eps, hipStream_t stream) {
  static const char* fn = "ut_qk_rope_fwd";
  g_last_error[0] = 0;
  RopeShape sh{};
  UT_TRY(check_rope(fn, n, Hq, Hk, D, dtype, pos, pos_rows, token_idx, axis_dims_host, n_axes, theta,
                    pairs, q_weight, k_weight, w_dtype, eps, &sh));
  const int64_t step = dtype == UT_BF16 ? 8 : 4;
  RopeSide side[2] = {};
  side[0] = RopeSide{q, nullptr, q_out, q_weight, 0, 0, 0, Hq};
  UT_TRY(check_stride(fn, "q", strides_host, 0, (int64_t)Hq * D, step, kRopeMaxStride, &side[0].sx));
  UT_TRY(check_stride(fn, "q_out", strides_host, 2, (int64_t)Hq * D, step, kRopeMaxStride, &side[0].so));
  if (Hk > 0) {
    side[1] = RopeSide{k, nullptr, k_out, k_weight, 0, 0, 0, Hk};
    UT_TRY(check_stride(fn, "k", strides_host, 1, (int64_t)Hk * D, step, kRopeMaxStride, &side[1].sx));
    UT_TRY(check_stride(fn, "k_out", strides_host, 3, (int64_t)Hk * D, step, kRopeMaxStride, &side[1].so));
  }
  if (n == 0) return UT_OK;
  UT_TRY(check_ptr(fn, "q", q, 16));
  UT_TRY(check_ptr(fn, "q_out", q_out, 16));
  if (Hk > 0) {
    UT_TRY(check_ptr(fn, "k", k, 16));
    UT_TRY(check_ptr(fn, "k_out", k_out, 16));
  }
  return check_hip(launch_qk_rope(sh, side, false, nullptr, nullptr, nullptr, stream), "rotary launch");
}

size_t ut_qk_rope_bwd_workspace_size(int32_t D) {
  if (D < 1 || D > kRopeMaxDim) return 0;
  return (size_t)kRopeParts * 2 * D * sizeof(float);
}

ut_status ut_qk_rope_bwd(const void* dq_out, const void* dk_out, const void* q, const void* k,
                         void* dq, void* dk, const int64_t* strides_host, ut_dtype dtype, int64_t n,
                         int32_t Hq, int32_t Hk, int32_t D, const float* pos, int64_t pos_rows,
                         const int32_t* token_idx, const int32_t* axis_dims_host, int32_t n_axes,
                         double theta, ut_rope_pairs pairs, const void* q_weight,
                         const void* k_weight, ut_dtype w_dtype, float eps, float* dq_weight,
                         float* dk_weight, void* workspace, size_t workspace_bytes,
                         hipStream_t stream) {
  static const char* fn = "ut_qk_rope_bwd";
  g_last_error[0] = 0;
  RopeShape sh{};
  UT_TRY(check_rope(fn, n, Hq, Hk, D, dtype, pos, pos_rows, token_idx, axis_dims_host, n_axes, theta,
                    pairs, q_weight, k_weight, w_dtype, eps, &sh));
  const int64_t step = dtype == UT_BF16 ? 8 : 4;
  const bool norm = q_weight != nullptr;
  RopeSide side[2] = {};
  side[0] = RopeSide{q, dq_out, dq, q_weight, 0, 0, 0, Hq};
  UT_TRY(check_stride(fn, "dq_out", strides_host, 0, (int64_t)Hq * D, step, kRopeMaxStride, &side[0].sdy));
  if (norm) UT_TRY(check_stride(fn, "q", strides_host, 2, (int64_t)Hq * D, step, kRopeMaxStride, &side[0].sx));
  UT_TRY(check_stride(fn, "dq", strides_host, 4, (int64_t)Hq * D, step, kRopeMaxStride, &side[0].so));
  if (Hk > 0) {
    side[1] = RopeSide{k, dk_out, dk, k_weight, 0, 0, 0, Hk};
    UT_TRY(check_stride(fn, "dk_out", strides_host, 1, (int64_t)Hk * D, step, kRopeMaxStride, &side[1].sdy));
    if (norm) UT_TRY(check_stride(fn, "k", strides_host, 3, (int64_t)Hk * D, step, kRopeMaxStride, &side[1].sx));
    UT_TRY(check_stride(fn, "dk", strides_host, 5, (int64_t)Hk * D, step, kRopeMaxStride, &side[1].so));
  }
  if (n > 0) {
    UT_TRY(check_ptr(fn, "dq_out", dq_out, 16));
    UT_TRY(check_ptr(fn, "dq", dq, 16));
    if (norm) UT_TRY(check_ptr(fn, "q", q, 16));
    if (Hk > 0) {
      UT_TRY(check_ptr(fn, "dk_out", dk_out, 16));
      UT_TRY(check_ptr(fn, "dk", dk, 16));
      if (norm) UT_TRY(check_ptr(fn, "k", k, 16));
    }
  }
  if (norm) {
    UT_TRY(check_ptr(fn, "dq_weight", dq_weight, 4));
    if (Hk > 0) UT_TRY(check_ptr(fn, "dk_weight", dk_weight, 4));
    const size_t need = ut_qk_rope_bwd_workspace_size(D);
    if (!workspace || workspace_bytes < need)
      return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                  workspace ? workspace_bytes : (size_t)0);
    UT_TRY(check_ptr(fn, "workspace", workspace, 16));
  } else if (n == 0) {
    return UT_OK;
  }
  return check_hip(launch_qk_rope(sh, side, true, static_cast<float*>(workspace), dq_weight,
                                  Hk > 0 ? dk_weight : nullptr, stream),
                   "rotary backward launch");
}

namespace {
// Sizes shared by the cross-attention calls; fills a (T = 0 and null cu: uniform).
ut_status check_xattn(const char* fn, int32_t B, int64_t Tq, int64_t Tk, int32_t Nq, int32_t Nk,
                      int32_t Hq, int32_t Hk, int32_t D, float scale, XArgs* a) {
  if (B < 1 || Nq < 0 || Nk < 0 || Hq < 1 || Hk < 1)
    return fail(UT_ERR_INVALID_ARG, "%s: B, Hq, Hk must be >= 1, lengths >= 0 (got %d, %d, %d, %d, %d)",
                fn, B, Hq, Hk, Nq, Nk);
  if (Hq % Hk != 0)
    return fail(UT_ERR_INVALID_ARG, "%s: Hq = %d is no multiple of Hk = %d", fn, Hq, Hk);
  if (D < 8 || D % 8 != 0 || D > 128)
    return fail(UT_ERR_UNSUPPORTED, "%s: head_dim %d unsupported (a multiple of 8 up to 128)", fn, D);
  // as in the block-sparse calls: a running maximum of the scaled scores
  if (!std::isfinite(scale) || !(scale > 0.f))
    return fail(UT_ERR_INVALID_ARG, "%s: softmax_scale must be finite and > 0 (got %g)", fn,
                (double)scale);
  if (Tq < 0 || Tk < 0 || Tq >= ((int64_t)1 << 31) || Tk >= ((int64_t)1 << 31))
    return fail(UT_ERR_INVALID_ARG, "%s: token counts %lld, %lld outside [0, 2^31)", fn,
                (long long)Tq, (long long)Tk);
  // 32-bit row numbers, and launches over rows of less than 2^32 threads
  const int64_t most = (int64_t)1 << 27;
  if (Tq * Hq >= most || Tk * Hk >= most || (int64_t)B * Nq * Hq >= most || (int64_t)B * Nk * Hk >= most)
    return fail(UT_ERR_INVALID_ARG, "%s: problem too large (2^27 rows of a head or more)", fn);
  a->B = B;
  a->Nq = Nq;
  a->Nk = Nk;
  a->Hq = Hq;
  a->Hk = Hk;
  a->G = Hq / Hk;
  a->D = D;
  a->Tq = Tq;
  a->Tk = Tk;
  a->scale = scale;
  return UT_OK;
}

// The backward's dK/dV pass and its joins launch by size, not by what fits the chip.
ut_status check_xattn_bwd(const char* fn, const XArgs& a) {
  if (!xattn_bwd_launchable(a))
    return fail(UT_ERR_INVALID_ARG,
                "%s: problem too large (2^24 workgroups: B Hk ceil(Nk / 128), or T H D / 1024 of split work)",
                fn);
  return UT_OK;
}

// Sample offsets of one side; under UT_VALIDATE copied to the host and checked
// (they may end before T: the tokens behind belong to no sample).
ut_status check_cu(const char* fn, const char* name, const int32_t* cu, int32_t B, int64_t T,
                   int32_t max_seqlen, hipStream_t stream) {
  UT_TRY(check_ptr(fn, name, cu, 4));
  if (!validate_mode()) return UT_OK;
  std::vector<int32_t> v;
  UT_TRY(validate_copy(cu, (size_t)B + 1, &v, stream));
  if (v[(size_t)B] > T)
    return fail(UT_ERR_INVALID_ARG, "%s: %s ends at %d, past T = %lld", fn, name, v[(size_t)B],
                (long long)T);
  return check_cu_seqlens(fn, v.data(), B, v[(size_t)B], max_seqlen);
}

struct XTensor {
  const char* name;
  const void* p;
  int* stride;      // in XArgs
  bool keys;        // rows of Hk heads for Tk tokens, else Hq and Tq
};
ut_status check_xtensors(const char* fn, const XTensor* t, int count, const int64_t* strides_host,
                         const XArgs& a) {
  for (int i = 0; i < count; ++i) {
    int64_t s = 0;
    UT_TRY(check_stride(fn, t[i].name, strides_host, i, (int64_t)(t[i].keys ? a.Hk : a.Hq) * a.D, 8,
                        kXMaxStride, &s));
    *t[i].stride = (int)s;
    if ((t[i].keys ? a.Tk : a.Tq) > 0) UT_TRY(check_ptr(fn, t[i].name, t[i].p, 16));
  }
  return UT_OK;
}

ut_status check_space(const char* fn, size_t need, const void* workspace, size_t bytes) {
  if (need == 0) return UT_OK;
  if (!workspace || bytes < need)
    return fail(UT_ERR_WORKSPACE, "%s: workspace of %zu bytes required (got %zu)", fn, need,
                workspace ? bytes : (size_t)0);
  return check_ptr(fn, "workspace", workspace, 16);
}

ut_status xattn_fwd(const char* fn, XArgs& a, const void* q, const void* k, const void* v, void* o,
                    float* lse, const int64_t* strides_host, const uint8_t* key_mask, void* workspace,
                    size_t workspace_bytes, bool zero_rest, hipStream_t stream) {
  const XTensor t[] = {{"q", q, &a.sq, false}, {"k", k, &a.sk, true}, {"v", v, &a.sv, true},
                       {"o", o, &a.so, false}};
  UT_TRY(check_xtensors(fn, t, 4, strides_host, a));
  if (a.Tq > 0) UT_TRY(check_ptr(fn, "lse", lse, 4));
  UT_TRY(check_space(fn, xattn_fwd_workspace(a), workspace, workspace_bytes));
  a.q = q, a.k = k, a.v = v, a.o = o, a.lse = lse, a.mask = key_mask;
  if (a.Tq == 0) return UT_OK;
  a.zero_rest = zero_rest;
  if (a.Nq == 0 && !zero_rest) return UT_OK;
  return check_hip(launch_xattn_fwd(a, workspace, stream), "cross attention launch");
}

ut_status xattn_bwd(const char* fn, XArgs& a, const void* q, const void* k, const void* v,
                    const void* o, const void* dout, const float* lse, void* dq, void* dk, void* dv,
                    const int64_t* strides_host, const uint8_t* key_mask, void* workspace,
                    size_t workspace_bytes, bool zero_rest, hipStream_t stream) {
  const XTensor t[] = {{"q", q, &a.sq, false},     {"k", k, &a.sk, true},    {"v", v, &a.sv, true},
                       {"o", o, &a.so, false},     {"dout", dout, &a.sdo, false},
                       {"dq", dq, &a.sdq, false},  {"dk", dk, &a.sdk, true}, {"dv", dv, &a.sdv, true}};
  UT_TRY(check_xtensors(fn, t, 8, strides_host, a));
  if (a.Tq > 0) UT_TRY(check_ptr(fn, "lse", lse, 4));
  UT_TRY(check_space(fn, xattn_bwd_workspace(a), workspace, workspace_bytes));
  a.q = q, a.k = k, a.v = v, a.o_in = o, a.dout = dout, a.dq = dq, a.dk = dk, a.dv = dv;
  a.lse = const_cast<float*>(lse), a.mask = key_mask;
  if (a.Tq == 0 && a.Tk == 0) return UT_OK;
  a.zero_rest = zero_rest;
  return check_hip(launch_xattn_bwd(a, workspace, stream), "cross attention backward launch");
}

// Workspace sizes: 0 for sizes that the calls refuse.
bool xattn_sizes(int32_t B, int64_t Tq, int64_t Tk, int32_t Nq, int32_t Nk, int32_t Hq, int32_t Hk,
                 int32_t D, XArgs* a) {
  const bool ok = check_xattn("ut_xattn", B, Tq, Tk, Nq, Nk, Hq, Hk, D, 1.f, a) == UT_OK;
  g_last_error[0] = 0;
  return ok;
}
}  // namespace

size_t ut_xattn_fwd_workspace_size(int32_t B, int32_t Nq, int32_t Nk, int32_t Hq, int32_t Hk, int32_t D) {
  XArgs a{};
  return xattn_sizes(B, (int64_t)B * Nq, (int64_t)B * Nk, Nq, Nk, Hq, Hk, D, &a) ? xattn_fwd_workspace(a) : 0;
}

ut_status ut_xattn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                       const int64_t* strides_host, const uint8_t* key_mask, int32_t B, int32_t Nq,
                       int32_t Nk, int32_t Hq, int32_t Hk, int32_t D, float softmax_scale,
                       void* workspace, size_t workspace_bytes, hipStream_t stream) {
  static const char* fn = "ut_xattn_fwd";
  g_last_error[0] = 0;
  XArgs a{};
  UT_TRY(check_xattn(fn, B, (int64_t)B * Nq, (int64_t)B * Nk, Nq, Nk, Hq, Hk, D, softmax_scale, &a));
  return xattn_fwd(fn, a, q, k, v, o, lse, strides_host, key_mask, workspace, workspace_bytes, false,
                   stream);
}

size_t ut_xattn_fwd_varlen_workspace_size(int32_t B, int64_t Tq, int32_t max_seqlen_q,
                                          int32_t max_seqlen_k, int32_t Hq, int32_t Hk, int32_t D) {
  XArgs a{};
  return xattn_sizes(B, Tq, 0, max_seqlen_q, max_seqlen_k, Hq, Hk, D, &a) ? xattn_fwd_workspace(a) : 0;
}

ut_status ut_xattn_fwd_varlen(const void* q, const void* k, const void* v, void* o, float* lse,
                              const int64_t* strides_host, const uint8_t* key_mask,
                              const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t B,
                              int64_t Tq, int64_t Tk, int32_t max_seqlen_q, int32_t max_seqlen_k,
                              int32_t Hq, int32_t Hk, int32_t D, float softmax_scale,
                              int32_t zero_rest, void* workspace, size_t workspace_bytes,
                              hipStream_t stream) {
  static const char* fn = "ut_xattn_fwd_varlen";
  g_last_error[0] = 0;
  XArgs a{};
  UT_TRY(check_xattn(fn, B, Tq, Tk, max_seqlen_q, max_seqlen_k, Hq, Hk, D, softmax_scale, &a));
  UT_TRY(check_cu(fn, "cu_seqlens_q", cu_seqlens_q, B, Tq, max_seqlen_q, stream));
  UT_TRY(check_cu(fn, "cu_seqlens_k", cu_seqlens_k, B, Tk, max_seqlen_k, stream));
  a.cuq = cu_seqlens_q, a.cuk = cu_seqlens_k;
  return xattn_fwd(fn, a, q, k, v, o, lse, strides_host, key_mask, workspace, workspace_bytes,
                   zero_rest != 0, stream);
}

size_t ut_xattn_bwd_workspace_size(int32_t B, int32_t Nq, int32_t Nk, int32_t Hq, int32_t Hk, int32_t D) {
  XArgs a{};
  return xattn_sizes(B, (int64_t)B * Nq, (int64_t)B * Nk, Nq, Nk, Hq, Hk, D, &a) && xattn_bwd_launchable(a)
             ? xattn_bwd_workspace(a)
             : 0;
}

ut_status ut_xattn_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                       const float* lse, void* dq, void* dk, void* dv, const int64_t* strides_host,
                       const uint8_t* key_mask, int32_t B, int32_t Nq, int32_t Nk, int32_t Hq,
                       int32_t Hk, int32_t D, float softmax_scale, void* workspace,
                       size_t workspace_bytes, hipStream_t stream) {
  static const char* fn = "ut_xattn_bwd";
  g_last_error[0] = 0;
  XArgs a{};
  UT_TRY(check_xattn(fn, B, (int64_t)B * Nq, (int64_t)B * Nk, Nq, Nk, Hq, Hk, D, softmax_scale, &a));
  UT_TRY(check_xattn_bwd(fn, a));
  return xattn_bwd(fn, a, q, k, v, o, dout, lse, dq, dk, dv, strides_host, key_mask, workspace,
                   workspace_bytes, false, stream);
}

size_t ut_xattn_bwd_varlen_workspace_size(int32_t B, int64_t Tq, int64_t Tk, int32_t max_seqlen_q,
                                          int32_t max_seqlen_k, int32_t Hq, int32_t Hk, int32_t D) {
  XArgs a{};
  return xattn_sizes(B, Tq, Tk, max_seqlen_q, max_seqlen_k, Hq, Hk, D, &a) && xattn_bwd_launchable(a)
             ? xattn_bwd_workspace(a)
             : 0;
}

ut_status ut_xattn_bwd_varlen(const void* q, const void* k, const void* v, const void* o,
                              const void* dout, const float* lse, void* dq, void* dk, void* dv,
                              const int64_t* strides_host, const uint8_t* key_mask,
                              const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t B,
                              int64_t Tq, int64_t Tk, int32_t max_seqlen_q, int32_t max_seqlen_k,
                              int32_t Hq, int32_t Hk, int32_t D, float softmax_scale,
                              int32_t zero_rest, void* workspace, size_t workspace_bytes,
                              hipStream_t stream) {
  static const char* fn = "ut_xattn_bwd_varlen";
  g_last_error[0] = 0;
  XArgs a{};
  UT_TRY(check_xattn(fn, B, Tq, Tk, max_seqlen_q, max_seqlen_k, Hq, Hk, D, softmax_scale, &a));
  UT_TRY(check_xattn_bwd(fn, a));
  UT_TRY(check_cu(fn, "cu_seqlens_q", cu_seqlens_q, B, Tq, max_seqlen_q, stream));
  UT_TRY(check_cu(fn, "cu_seqlens_k", cu_seqlens_k, B, Tk, max_seqlen_k, stream));
  a.cuq = cu_seqlens_q, a.cuk = cu_seqlens_k;
  return xattn_bwd(fn, a, q, k, v, o, dout, lse, dq, dk, dv, strides_host, key_mask, workspace,
                   workspace_bytes, zero_rest != 0, stream);
}

}  // extern "C"
