// da_paged.hpp -- launch arguments of the paged cache, the attention over it and
// the block selection, shared by the C-ABI layer (da_paged_api.cpp) and the
// kernels.  Not part of the public interface.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "da_internal.hpp"
#include "delta_attn.h"

namespace da {

constexpr int kPage = DA_PAGE_TOKENS;  // tokens per page: the attention kernels' key tile
// Most candidates of a group: their ranks and, in the prefill, their scores are in LDS.
constexpr int kMaxCandPages = 131072, kMaxCandBlocks = 24576;
// Candidate pages that one launch scores and picks from, without a workspace.
constexpr int kFewCandPages = 1024;
// Longest list of pages: places in it, and a workgroup's step past them, are 32-bit in the kernels.
constexpr int kMaxList = 1 << 30;
constexpr int kMaxRequests = DA_PAGES_MAX_REQUESTS;

// The integers of a cache: page table [S][M], lengths [S], reference counts [P].
struct Table {
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  int S, M, P;
};

// Its pages [layers][P][Hkv][64][d] (bf16).
struct Pages {
  uint16_t* k;
  uint16_t* v;
  int layers, Hkv, d;
};

hipError_t launch_pages_fork(const Table& t, const int32_t* src, const int32_t* dst, int n,
                             int32_t* result, hipStream_t s);
hipError_t launch_pages_resize(const Table& t, const Pages& p, const int32_t* slots,
                               const int32_t* new_lens, int n, int32_t* result, hipStream_t s);
hipError_t launch_pages_append(const Table& t, const Pages& p, const uint16_t* k,
                               const uint16_t* v, int64_t T, const int32_t* slots,
                               const int32_t* cu, int B, int N, const int32_t* new_lens, hipStream_t s);
hipError_t launch_pages_compact(const Table& t, const Pages& p, const int32_t* slots,
                                const int32_t* start, const int32_t* keep, int64_t n_keep,
                                const int32_t* cu_keep, int n, int32_t* result, hipStream_t s);

// Where the keys of a summary lie: rows of a packed or fixed-length batch
// (table == nullptr), or pages.
struct SummaryArgs {
  const uint16_t* k;
  const int32_t* cu;     // [B + 1], or nullptr for B sequences of N tokens
  const int32_t* table;  // [S][M], or nullptr
  const int32_t* lens;   // [S]
  const int32_t* slots;  // [B], or nullptr: sequence b is slot b
  const int32_t* first;  // [B], or nullptr: 0
  int8_t* codes;         // [blocks][Hkv][d]
  float* scales;         // [blocks][Hkv]
  int B, N, Hkv, d, S, M, P;
  int nblk;              // blocks per sequence that the grid covers
};
hipError_t launch_summary(const SummaryArgs& a, hipStream_t s);

// Selection of blocks by score (prefill: per query block; decode: per token).
struct SelectArgs {
  const uint16_t* q;     // [T][Hq][d]
  const int8_t* codes;
  const float* scales;
  const int32_t* cu;     // [B + 1], or nullptr for B sequences of N rows
  const int32_t* table;  // decode only
  const int32_t* lens;
  const int32_t* slots;
  int B, N, Hq, Hkv, d, S, M, P;
  int top_k, n_sink, n_recent;
  int G;                 // Hq / Hkv
  FastDiv fd_G;
  int block_q, nqb;      // prefill
  int32_t* block_ptr;
  int32_t* block_idx;
  int64_t total;         // list entries of one (sequence, kv head)
  int max_blocks;        // candidates any group can have
  int32_t* pages;        // decode: [T][Hkv][top_k]
  uint32_t* keys;        // decode: workspace [B * N][Hkv][max_blocks], past kFewCandPages of them
};
// Entries of the lists of one (sequence, kv head) before query block qb: min(top_k, j * R) for
// each block j, R key tiles long.  In 64 bits: top_k may be the largest int, "all of them".
__host__ __device__ __forceinline__ int64_t list_entries_before(int64_t qb, int top_k, int R) {
  const int64_t whole = (int64_t)(top_k / R) + 1;  // lists with j * R <= top_k
  const int64_t m = qb < whole ? qb : whole;
  return m * (m - 1) / 2 * R + (qb - m) * top_k;
}
hipError_t launch_select_blocks(const SelectArgs& a, hipStream_t s);
hipError_t launch_select_pages(const SelectArgs& a, hipStream_t s);

// Attention over the pages.
struct PagedArgs {
  const uint16_t* q;     // [T][Hq][d]
  const uint16_t* k;     // [P][Hkv][64][d]
  const uint16_t* v;
  uint16_t* out;         // [T][Hq][d]
  float* lse;            // [T][Hq], or nullptr
  const int32_t* table;  // [S][M]
  const int32_t* lens;   // [S]
  const int32_t* slots;  // [B], or nullptr
  const int32_t* cu;     // [B + 1], or nullptr for B sequences of N rows
  const uint64_t* mask;  // [T][mask_words], or nullptr: causal
  const int32_t* lists;  // [T][Hkv][n_list] page positions, or nullptr: every page
  int B, N, Hq, Hkv, d, S, M, P;
  int max_len, mask_words, n_list;
  int G;                 // Hq / Hkv
  FastDiv fd_G, fd_Hkv, fd_Hq, fd_N;
  float scale_log2;
  // How the work is shared (da_paged_api.cpp): n_wgs workgroups of row_tiles tiles of 32
  // rows, at least min_units pages each; or, with `whole`, segments (a kv head's rows of
  // a sequence, a workgroup's worth of them) as they are, min_units of them each.
  // Workgroups begin at segments where that costs at most align_pages pages each.
  // row_groups: of the sequence with most rows, where workgroups may team up (1: they do not).
  int row_tiles, n_wgs, min_units, whole, align_pages, row_groups;
  // Workspace (nullptr where no rows are cut)
  int32_t* units;        // [B + 3] pages before each sequence's, the share, whether aligned, team
  float* part_o;         // [n_wgs][2][row_tiles * 32][d] partial results of cut segments
  float* part_ml;        // [n_wgs][2][row_tiles * 32][2]
};
// Units per workgroup or team, of `total` for n of them (up to the largest int: the sum is unsigned).
__host__ __device__ __forceinline__ int share_of(int min_units, int total, int n) {
  const int even = (int)(((uint32_t)total + (uint32_t)n - 1) / (uint32_t)n);
  return even > min_units ? even : min_units;
}
hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t s);

}  // namespace da
