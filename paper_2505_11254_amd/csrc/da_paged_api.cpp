// da_paged_api.cpp -- the C ABI of the paged cache, the attention over it and the
// block selection: argument checks and launch plans.
#include <stdint.h>

#include "da_internal.hpp"
#include "da_paged.hpp"

namespace da {
namespace {

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Whether a launch can have so many workgroups: its threads are counted in 32 bits.
bool fits(int64_t wgs, int threads) { return wgs <= (int64_t)UINT32_MAX / threads; }

da_status check_table(const Table& t) {
  if (!t.table || !t.lens) return DA_ERR_NULL;
  if (t.S < 1 || t.M < 1 || t.P < 1) return DA_ERR_SHAPE;
  // positions are 32-bit inside the kernels
  if ((int64_t)t.M * kPage > INT32_MAX) return DA_ERR_SHAPE;
  if (!aligned(t.table, 4) || !aligned(t.lens, 4) || !aligned(t.refs, 4)) return DA_ERR_ALIGN;
  return DA_OK;
}

da_status check_pages(const void* k, const void* v, int layers, int Hkv, int d) {
  if (!k || !v) return DA_ERR_NULL;
  if (layers < 1 || layers > 32767 || Hkv < 1) return DA_ERR_SHAPE;
  if (d != 64 && d != 128) return DA_ERR_UNSUPPORTED;
  if (!aligned(k, 16) || !aligned(v, 16)) return DA_ERR_ALIGN;
  return DA_OK;
}

// A batch of B sequences of up to N tokens with Hq heads on Hkv.
da_status check_batch(int B, int N, int Hq, int Hkv, int d) {
  if (B < 1 || N < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return DA_ERR_SHAPE;
  if (d != 64 && d != 128) return DA_ERR_UNSUPPORTED;
  return DA_OK;
}
// The same where a workgroup or a partial result goes with each of its rows (256 threads
// merge eight of them).
da_status check_rows(int B, int N, int Hq, int Hkv, int d) {
  const da_status st = check_batch(B, N, Hq, Hkv, d);
  if (st != DA_OK) return st;
  const int64_t tokens = (int64_t)B * N;
  return tokens > INT32_MAX || tokens * Hq > INT32_MAX || !fits((tokens * Hq + 7) / 8, 256) ? DA_ERR_SHAPE : DA_OK;
}

da_status launched(hipError_t e) { return e == hipSuccess ? DA_OK : fail_hip(e); }

int64_t pages_of(int64_t tokens) { return (tokens + kPage - 1) / kPage; }

// How the attention over pages is shared: rows in tiles of 32, up to row_tiles of them
// per workgroup, and as many workgroups as run at once (kSlots: by LDS and registers; at
// d = 64 more would fit, but make more partial results than they gain), each with an
// even share of all pages.  A workgroup alone takes kPageUs per page.
//  - Segments are left whole where their even shares would gain less than the cuts cost:
//    kCutUs for a second start in a workgroup, two tiles of partial results written and
//    read, and the merge's launch.  Whole against shared (us; d 128 unless said).  One row
//    tile, equal lengths: 8 segments of 7 pages 11.4, 13.2, of 16 pages 16.0, 13.3; 64 of 118
//    pages 72, 46; 384 of 161 pages 343, 343.  Two: 28 of 6 pages 12.9, 16.5; 24 of 34 pages 33, 19.
//    Four: 21 of 11 pages 18.8, 27.7; 136 of 74 pages 88, 54; d 64, 240 of 27 pages 28, 34, 82
//    of 29 pages 28, 19.  Eight: 32 of 19 pages 35, 47; 24 of 50 pages 78, 38; 408 of 23 pages
//    79, 99.  (Over 290 drawn sizes the rule's choices average within 1 % of the better of
//    the two; at worst 18 % above, one row tile, d 64, 18 segments of 22 pages.)
//  - Workgroups begin at segments (and some stay idle) where that costs each at most
//    kAlignPages pages, less than a second start and its partial results: one sequence of
//    9000 keys, 14 drafts 26.5 -> 21.8 us; six of them 40.4 -> 37.3; 16 of 24 drafts, 6000
//    keys 60.5 -> 58.7; eight of 2000 keys, 8 heads on 2, d 64, one token 13.0 -> 10.6.
constexpr int kAlignPages = 8;
struct PagedPlan {
  int row_tiles, n_wgs, min_units, whole, align_pages, row_groups;
  size_t units_bytes, part_rows, bytes;
};
da_status paged_plan(int B, int N, int Hq, int Hkv, int d, int64_t pages, int n_list, PagedPlan* p) {
  if (n_list > kMaxList) return DA_ERR_SHAPE;
  const int G = Hq / Hkv;
  const int64_t rows = n_list ? G : (int64_t)N * G;
  const int rt = rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 || d == 64 || n_list ? 4 : 8;
  const int c = rt == 1 ? 0 : rt == 2 ? 1 : rt == 4 ? 2 : 3;
  static const int kSlots[2][4] = {{256, 256, 512, 256}, {256, 256, 512, 512}};
  static const double kPageUs[2][4] = {{0.46, 0.9, 1.08, 1.54}, {0.29, 0.55, 0.8, 0.8}};
  static const double kCutUs[4] = {6., 8., 17., 35.};
  const int64_t groups = (rows + 32 * rt - 1) / (32 * rt);
  const int64_t segs = (n_list ? (int64_t)B * N : B) * Hkv * groups;
  if (n_list) pages = (int64_t)n_list + 1;
  if (pages < 1) pages = 1;
  if ((double)segs * (double)pages > (double)INT32_MAX) return DA_ERR_SHAPE;
  const int64_t slots = kSlots[d == 64][c];
  const double page_us = kPageUs[d == 64][c], seg_us = (double)pages * page_us;
  // (lengths below the longest are taken to make four fifths of the work)
  const double rounds = (double)segs / (double)slots;
  p->row_tiles = rt;
  p->whole = fits(segs, 512) &&
             ((seg_us < 12. && rounds >= 0.25) ||
              seg_us * (double)((segs + slots - 1) / slots) < 0.8 * seg_us * rounds + kCutUs[c]);
  if (p->whole) {
    p->min_units = 1;
    p->n_wgs = (int)segs;
  } else {
    p->min_units = 2 * rt;
    const int64_t most = (segs * pages + p->min_units - 1) / p->min_units;
    p->n_wgs = (int)(most < slots ? most : slots);
  }
  p->align_pages = kAlignPages;
  p->row_groups = !n_list && !p->whole && B <= 64 && groups <= p->n_wgs ? (int)groups : 1;
  p->part_rows = p->whole || p->n_wgs == 1 ? 0 : (size_t)p->n_wgs * 2 * rt * 32;
  p->units_bytes = p->part_rows ? ((size_t)B + 3 + 63) / 64 * 256 : 0;  // (the merge's alone)
  p->bytes = p->units_bytes + p->part_rows * (size_t)(d + 2) * 4;
  return DA_OK;
}

// Entries of the lists of one (sequence, kv head).
int64_t list_total(int max_seqlen, int top_k, int block_q) {
  return list_entries_before(((int64_t)max_seqlen + block_q - 1) / block_q, top_k, block_q / kPage);
}

da_status paged_attn(PagedArgs a, int n_list, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a.q || !a.k || !a.v || !a.out) return DA_ERR_NULL;
  da_status st = check_table({const_cast<int32_t*>(a.table), const_cast<int32_t*>(a.lens), nullptr, a.S, a.M, a.P});
  if (st != DA_OK) return st;
  st = check_rows(a.B, a.N, a.Hq, a.Hkv, a.d);
  if (st != DA_OK) return st;
  if (!a.slots && a.B > a.S) return DA_ERR_SHAPE;
  if (!aligned(a.q, 16) || !aligned(a.k, 16) || !aligned(a.v, 16) || !aligned(a.out, 16) ||
      !aligned(a.cu, 4) || !aligned(a.slots, 4) || !aligned(a.lse, 4) || !aligned(a.mask, 8) ||
      !aligned(a.lists, 4))
    return DA_ERR_ALIGN;
  const int64_t room = (int64_t)a.M * kPage;
  if (a.max_len > room) a.max_len = (int)room;
  PagedPlan p;
  st = paged_plan(a.B, a.N, a.Hq, a.Hkv, a.d, pages_of(a.max_len), n_list, &p);
  if (st != DA_OK) return st;
  if (p.bytes && (!workspace || workspace_bytes < p.bytes)) return DA_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return DA_ERR_ALIGN;
  st = check_device();
  if (st != DA_OK) return st;
  a.scale_log2 = 1.4426950408889634f / (a.d == 128 ? 11.313708498984761f : 8.f);
  a.G = a.Hq / a.Hkv;
  a.fd_G = make_fastdiv(a.G);
  a.fd_Hkv = make_fastdiv(a.Hkv);
  a.fd_Hq = make_fastdiv(a.Hq);
  a.fd_N = make_fastdiv(a.N);
  a.row_tiles = p.row_tiles;
  a.n_wgs = p.n_wgs;
  a.min_units = p.min_units;
  a.whole = p.whole;
  a.align_pages = p.align_pages;
  a.row_groups = p.row_groups;
  a.units = p.bytes ? (int32_t*)workspace : nullptr;
  a.part_o = (float*)((char*)workspace + p.units_bytes);
  a.part_ml = a.part_o + p.part_rows * a.d;
  return launched(launch_paged_attn(a, (hipStream_t)stream));
}

}  // namespace
}  // namespace da

using namespace da;

extern "C" {

da_status da_pages_fork(int32_t* table, int32_t* lens, int32_t* refs, int S, int M, int P,
                        const int32_t* src, const int32_t* dst, int n, int32_t* result, void* stream) {
  const Table t{table, lens, refs, S, M, P};
  if (!refs || !src || !dst || !result) return DA_ERR_NULL;
  da_status st = check_table(t);
  if (st != DA_OK) return st;
  if (n < 1 || n > kMaxRequests) return DA_ERR_SHAPE;
  if (!aligned(src, 4) || !aligned(dst, 4) || !aligned(result, 4)) return DA_ERR_ALIGN;
  st = check_device();
  if (st != DA_OK) return st;
  return launched(launch_pages_fork(t, src, dst, n, result, (hipStream_t)stream));
}

da_status da_pages_resize(void* k_pages, void* v_pages, int layers, int Hkv, int d, int32_t* table,
                          int32_t* lens, int32_t* refs, int S, int M, int P, const int32_t* slots,
                          const int32_t* new_lens, int n, int32_t* result, void* stream) {
  const Table t{table, lens, refs, S, M, P};
  if (!refs || !slots || !result) return DA_ERR_NULL;
  da_status st = check_table(t);
  if (st != DA_OK) return st;
  st = check_pages(k_pages, v_pages, layers, Hkv, d);
  if (st != DA_OK) return st;
  if (n < 1 || n > kMaxRequests || Hkv > INT32_MAX / 2 / n / layers || !fits((int64_t)n * layers * 2 * Hkv, 256))
    return DA_ERR_SHAPE;
  if (!aligned(slots, 4) || !aligned(new_lens, 4) || !aligned(result, 16)) return DA_ERR_ALIGN;
  st = check_device();
  if (st != DA_OK) return st;
  const Pages p{(uint16_t*)k_pages, (uint16_t*)v_pages, layers, Hkv, d};
  return launched(launch_pages_resize(t, p, slots, new_lens, n, result, (hipStream_t)stream));
}

da_status da_pages_append(const void* k, const void* v, int64_t T, void* k_pages, void* v_pages,
                          int layers, int Hkv, int d, const int32_t* table, const int32_t* lens, int S,
                          int M, int P, const int32_t* slots, const int32_t* cu_seqlens, int B,
                          int max_seqlen, void* stream) {
  return da_pages_append_to(k, v, T, k_pages, v_pages, layers, Hkv, d, table, lens, S, M, P, slots, cu_seqlens, B,
                            max_seqlen, nullptr, stream);
}

da_status da_pages_append_to(const void* k, const void* v, int64_t T, void* k_pages, void* v_pages,
                             int layers, int Hkv, int d, const int32_t* table, const int32_t* lens, int S,
                             int M, int P, const int32_t* slots, const int32_t* cu_seqlens, int B,
                             int max_seqlen, const int32_t* new_lens, void* stream) {
  const Table t{const_cast<int32_t*>(table), const_cast<int32_t*>(lens), nullptr, S, M, P};
  if (!k || !v) return DA_ERR_NULL;
  da_status st = check_table(t);
  if (st != DA_OK) return st;
  st = check_pages(k_pages, v_pages, layers, Hkv, d);
  if (st != DA_OK) return st;
  if (B < 1 || max_seqlen < 1 || T < 0 || (!slots && B > S)) return DA_ERR_SHAPE;
  if (!cu_seqlens && (int64_t)B * max_seqlen != T) return DA_ERR_SHAPE;
  // chunks of 16 bytes per sequence and layer, and workgroups of at least 1024 of them
  const int64_t row = (int64_t)Hkv * (d / 8);
  if (row > INT32_MAX / max_seqlen || !fits((max_seqlen * row / 1024 + 1) * B, 256)) return DA_ERR_SHAPE;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4) || !aligned(cu_seqlens, 4) || !aligned(new_lens, 4))
    return DA_ERR_ALIGN;
  st = check_device();
  if (st != DA_OK) return st;
  const Pages p{(uint16_t*)k_pages, (uint16_t*)v_pages, layers, Hkv, d};
  return launched(launch_pages_append(t, p, (const uint16_t*)k, (const uint16_t*)v, T, slots, cu_seqlens, B,
                                      max_seqlen, new_lens, (hipStream_t)stream));
}

da_status da_pages_compact(void* k_pages, void* v_pages, int layers, int Hkv, int d, int32_t* table,
                           int32_t* lens, int32_t* refs, int S, int M, int P, const int32_t* slots,
                           const int32_t* start, const int32_t* keep, int64_t n_keep,
                           const int32_t* cu_keep, int n, int32_t* result, void* stream) {
  const Table t{table, lens, refs, S, M, P};
  if (!refs || !slots || !start || !keep || !cu_keep || !result) return DA_ERR_NULL;
  da_status st = check_table(t);
  if (st != DA_OK) return st;
  st = check_pages(k_pages, v_pages, layers, Hkv, d);
  if (st != DA_OK) return st;
  if (n < 1 || n > kMaxRequests || n_keep < 0 || Hkv > INT32_MAX / 2 / n / layers ||
      !fits((int64_t)n * layers * 2 * Hkv, 256))
    return DA_ERR_SHAPE;
  if (!aligned(slots, 4) || !aligned(start, 4) || !aligned(keep, 4) || !aligned(cu_keep, 4) ||
      !aligned(result, 16))
    return DA_ERR_ALIGN;
  st = check_device();
  if (st != DA_OK) return st;
  const Pages p{(uint16_t*)k_pages, (uint16_t*)v_pages, layers, Hkv, d};
  return launched(launch_pages_compact(t, p, slots, start, keep, n_keep, cu_keep, n, result, (hipStream_t)stream));
}

da_status da_page_summary(const void* k_pages, int Hkv, int d, const int32_t* table, const int32_t* lens,
                          int S, int M, int P, const int32_t* slots, const int32_t* first, int B,
                          int max_new, void* codes, float* scales, void* stream) {
  if (!k_pages || !codes || !scales) return DA_ERR_NULL;
  da_status st = check_table({const_cast<int32_t*>(table), const_cast<int32_t*>(lens), nullptr, S, M, P});
  if (st != DA_OK) return st;
  if (B < 1 || Hkv < 1 || max_new < 1 || (!slots && B > S)) return DA_ERR_SHAPE;
  if (d != 64 && d != 128) return DA_ERR_UNSUPPORTED;
  if (!aligned(k_pages, 16) || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(slots, 4) || !aligned(first, 4))
    return DA_ERR_ALIGN;
  SummaryArgs a{};
  // max_new tokens from anywhere in a page on end up to this many pages
  int64_t nblk = pages_of(max_new) + (first ? 1 : 0);
  if (nblk > M) nblk = M;
  if ((int64_t)B * nblk > INT32_MAX || !fits((int64_t)B * nblk * Hkv / 4 + 1, 256)) return DA_ERR_SHAPE;
  st = check_device();
  if (st != DA_OK) return st;
  a.k = (const uint16_t*)k_pages;
  a.table = table;
  a.lens = lens;
  a.slots = slots;
  a.first = first;
  a.codes = (int8_t*)codes;
  a.scales = scales;
  a.B = B;
  a.Hkv = Hkv;
  a.d = d;
  a.S = S;
  a.M = M;
  a.P = P;
  a.nblk = (int)nblk;
  return launched(launch_summary(a, (hipStream_t)stream));
}

da_status da_key_summary(const void* k, const int32_t* cu_seqlens, int B, int max_seqlen, int Hkv, int d,
                         void* codes, float* scales, void* stream) {
  if (!k || !codes || !scales) return DA_ERR_NULL;
  if (B < 1 || max_seqlen < 1 || Hkv < 1) return DA_ERR_SHAPE;
  if (d != 64 && d != 128) return DA_ERR_UNSUPPORTED;
  if (!cu_seqlens && (int64_t)B * max_seqlen > INT32_MAX) return DA_ERR_SHAPE;
  const int64_t nblk = max_seqlen / kPage;
  if ((int64_t)B * nblk > INT32_MAX || !fits((int64_t)B * nblk * Hkv / 4 + 1, 256)) return DA_ERR_SHAPE;
  if (!aligned(k, 16) || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(cu_seqlens, 4)) return DA_ERR_ALIGN;
  da_status st = check_device();
  if (st != DA_OK) return st;
  if (nblk == 0) return DA_OK;  // no whole block
  SummaryArgs a{};
  a.k = (const uint16_t*)k;
  a.cu = cu_seqlens;
  a.codes = (int8_t*)codes;
  a.scales = scales;
  a.B = B;
  a.N = max_seqlen;
  a.Hkv = Hkv;
  a.d = d;
  a.nblk = (int)nblk;
  return launched(launch_summary(a, (hipStream_t)stream));
}

int64_t da_key_summary_blocks(int64_t T, int B) { return T < 0 || B < 1 ? 0 : T / kPage + B; }

int64_t da_select_blocks_entries(int B, int max_seqlen, int Hkv, int top_k, int block_q) {
  if (B < 1 || max_seqlen < 1 || Hkv < 1 || top_k < 1 || (block_q != 64 && block_q != 128 && block_q != 256))
    return 0;
  const int64_t n = list_total(max_seqlen, top_k, block_q);
  return n > INT32_MAX || (double)n * B * Hkv > (double)INT32_MAX ? 0 : n * B * Hkv;
}

da_status da_select_blocks(const void* q, const void* codes, const float* scales, const int32_t* cu_seqlens,
                           int B, int max_seqlen, int Hq, int Hkv, int d, int top_k, int n_sink,
                           int n_recent, int block_q, int32_t* block_ptr, int32_t* block_idx,
                           void* stream) {
  if (!q || !codes || !scales || !block_ptr || !block_idx) return DA_ERR_NULL;
  da_status st = check_batch(B, max_seqlen, Hq, Hkv, d);
  if (st != DA_OK) return st;
  if (!cu_seqlens && (int64_t)B * max_seqlen > INT32_MAX) return DA_ERR_SHAPE;
  if (top_k < 1 || n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > top_k) return DA_ERR_PARAM;
  if (block_q != 64 && block_q != 128 && block_q != 256) return DA_ERR_PARAM;
  const int64_t nqb = ((int64_t)max_seqlen + block_q - 1) / block_q;
  if (nqb * block_q / kPage > kMaxCandBlocks) return DA_ERR_UNSUPPORTED;
  const int64_t total = list_total(max_seqlen, top_k, block_q);
  if (total > 0 && da_select_blocks_entries(B, max_seqlen, Hkv, top_k, block_q) == 0) return DA_ERR_SHAPE;
  if ((int64_t)B * Hkv > INT32_MAX || !fits((int64_t)B * Hkv * (nqb + 1), 256)) return DA_ERR_SHAPE;
  // (byte offsets inside a query block are 32-bit)
  if ((int64_t)block_q * Hq > (int64_t)UINT32_MAX / (2 * d)) return DA_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(cu_seqlens, 4) ||
      !aligned(block_ptr, 4) || !aligned(block_idx, 4))
    return DA_ERR_ALIGN;
  st = check_device();
  if (st != DA_OK) return st;
  SelectArgs a{};
  a.q = (const uint16_t*)q;
  a.codes = (const int8_t*)codes;
  a.scales = scales;
  a.cu = cu_seqlens;
  a.B = B;
  a.N = max_seqlen;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.G = Hq / Hkv;
  a.fd_G = make_fastdiv(a.G);
  a.top_k = top_k;
  a.n_sink = n_sink;
  a.n_recent = n_recent;
  a.block_q = block_q;
  a.nqb = (int)nqb;
  a.block_ptr = block_ptr;
  a.block_idx = block_idx;
  a.total = total;
  a.max_blocks = (int)((nqb - 1) * (block_q / kPage));
  return launched(launch_select_blocks(a, (hipStream_t)stream));
}

size_t da_select_pages_workspace_bytes(int B, int max_seqlen, int Hkv, int max_len) {
  if (B < 1 || max_seqlen < 1 || Hkv < 1 || max_len < 1 || max_len / kPage <= kFewCandPages) return 0;
  return (size_t)B * max_seqlen * Hkv * (size_t)(max_len / kPage) * 4;
}

da_status da_select_pages(const void* q, const void* codes, const float* scales, const int32_t* table,
                          const int32_t* lens, int S, int M, int P, const int32_t* slots,
                          const int32_t* cu_seqlens, int B, int max_seqlen, int max_len, int Hq, int Hkv,
                          int d, int top_k, int n_sink, int n_recent, int32_t* pages, void* workspace,
                          size_t workspace_bytes, void* stream) {
  if (!q || !codes || !scales || !pages) return DA_ERR_NULL;
  da_status st = check_table({const_cast<int32_t*>(table), const_cast<int32_t*>(lens), nullptr, S, M, P});
  if (st != DA_OK) return st;
  st = check_rows(B, max_seqlen, Hq, Hkv, d);
  if (st != DA_OK) return st;
  if (max_len < 1 || (!slots && B > S)) return DA_ERR_SHAPE;
  if (top_k < 1 || n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > top_k) return DA_ERR_PARAM;
  if (top_k > kMaxList) return DA_ERR_SHAPE;
  // (places inside a token's heads of one kv head are 32-bit)
  if (Hq / Hkv > INT32_MAX / d) return DA_ERR_SHAPE;
  const int64_t room = (int64_t)M * kPage;
  if (max_len > room) max_len = (int)room;
  if (max_len / kPage > kMaxCandPages) return DA_ERR_UNSUPPORTED;
  const int blocks = max_len / kPage;
  if (!fits((int64_t)B * max_seqlen * Hkv, blocks > 4096 ? 1024 : blocks > kFewCandPages ? 256 : 512)) return DA_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(cu_seqlens, 4) ||
      !aligned(slots, 4) || !aligned(pages, 4) || !aligned(workspace, 4))
    return DA_ERR_ALIGN;
  const size_t need = da_select_pages_workspace_bytes(B, max_seqlen, Hkv, max_len);
  if (need && max_len / kPage > top_k && (!workspace || workspace_bytes < need)) return DA_ERR_WORKSPACE;
  st = check_device();
  if (st != DA_OK) return st;
  SelectArgs a{};
  a.q = (const uint16_t*)q;
  a.codes = (const int8_t*)codes;
  a.scales = scales;
  a.cu = cu_seqlens;
  a.table = table;
  a.lens = lens;
  a.slots = slots;
  a.B = B;
  a.N = max_seqlen;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.S = S;
  a.M = M;
  a.P = P;
  a.G = Hq / Hkv;
  a.fd_G = make_fastdiv(a.G);
  a.top_k = top_k;
  a.n_sink = n_sink;
  a.n_recent = n_recent;
  a.max_blocks = max_len / kPage;
  a.pages = pages;
  a.keys = (uint32_t*)workspace;
  return launched(launch_select_pages(a, (hipStream_t)stream));
}

size_t da_paged_workspace_bytes(int B, int max_seqlen, int Hq, int Hkv, int d, int max_len, int n_list) {
  PagedPlan p;
  if (check_rows(B, max_seqlen, Hq, Hkv, d) != DA_OK || max_len < 1 || n_list < 0) return 0;
  if (paged_plan(B, max_seqlen, Hq, Hkv, d, pages_of(max_len), n_list, &p) != DA_OK) return 0;
  return p.bytes;
}

da_status tree_attn_paged(const void* q, const void* k_pages, const void* v_pages, void* out, float* lse,
                          const int32_t* table, const int32_t* lens, int S, int M, int P,
                          const int32_t* slots, const int32_t* cu_seqlens, int B, int max_seqlen,
                          int max_len, int Hq, int Hkv, int d, const uint64_t* mask, int mask_words,
                          void* workspace, size_t workspace_bytes, void* stream) {
  if (max_len < 1) return DA_ERR_SHAPE;
  if (mask && (mask_words < 1 || (int64_t)mask_words * 64 < max_seqlen)) return DA_ERR_PARAM;
  PagedArgs a{};
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k_pages;
  a.v = (const uint16_t*)v_pages;
  a.out = (uint16_t*)out;
  a.lse = lse;
  a.table = table;
  a.lens = lens;
  a.slots = slots;
  a.cu = cu_seqlens;
  a.mask = mask;
  a.mask_words = mask_words;
  a.B = B;
  a.N = max_seqlen;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.S = S;
  a.M = M;
  a.P = P;
  a.max_len = max_len;
  return paged_attn(a, 0, workspace, workspace_bytes, stream);
}

da_status selected_attn_paged(const void* q, const void* k_pages, const void* v_pages, void* out, float* lse,
                              const int32_t* table, const int32_t* lens, int S, int M, int P,
                              const int32_t* slots, const int32_t* cu_seqlens, int B, int max_seqlen,
                              int Hq, int Hkv, int d, const int32_t* pages, int top_k, void* workspace,
                              size_t workspace_bytes, void* stream) {
  if (!pages) return DA_ERR_NULL;
  if (top_k < 1) return DA_ERR_PARAM;
  PagedArgs a{};
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k_pages;
  a.v = (const uint16_t*)v_pages;
  a.out = (uint16_t*)out;
  a.lse = lse;
  a.table = table;
  a.lens = lens;
  a.slots = slots;
  a.cu = cu_seqlens;
  a.lists = pages;
  a.n_list = top_k;
  a.B = B;
  a.N = max_seqlen;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.d = d;
  a.S = S;
  a.M = M;
  a.P = P;
  a.max_len = INT32_MAX;
  return paged_attn(a, top_k, workspace, workspace_bytes, stream);
}

}  // extern "C"
