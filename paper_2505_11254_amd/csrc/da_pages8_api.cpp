// da_pages8_api.cpp -- the C ABI of the cache in 8 bits, and of the attention over either cache under
// changed scores: argument checks and calls.
#include <stdint.h>

#include "da_internal.hpp"
#include "da_paged.hpp"

namespace da {
namespace {

da_status check_scales(const float* k_scales, const float* v_scales) {
  if (!k_scales || !v_scales) return DA_ERR_NULL;
  return aligned(k_scales, 4) && aligned(v_scales, 4) ? DA_OK : DA_ERR_ALIGN;
}

// Rows of bf16 that go into pages of codes, or come from them; `ints` [B] or NULL.
da_status check_rows8(const Table& t, const Pages8& p, const void* k, const void* v, int64_t T,
                      const int32_t* slots, const int32_t* cu, int B, int N, const int32_t* ints) {
  if (!k || !v) return DA_ERR_NULL;
  da_status st = check_scales(p.k_scales, p.v_scales);
  if (st != DA_OK) return st;
  st = check_table(t);
  if (st != DA_OK) return st;
  st = check_pages(p.k, p.v, p.layers, p.Hkv, p.d);
  if (st != DA_OK) return st;
  if (B < 1 || N < 1 || T < 0 || (!slots && B > t.S)) return DA_ERR_SHAPE;
  if (!cu && (int64_t)B * N != T) return DA_ERR_SHAPE;
  // Pieces of 16 values of a sequence and layer are counted in 32 bits, and a launch has less than 2^32
  // threads: a read's one for each of them, an append's 256 for each page that may be touched, layer, keys
  // or values, and kv head.
  const int64_t row = (int64_t)p.Hkv * (p.d / 16);
  if (row > INT32_MAX / N) return DA_ERR_SHAPE;
  const double most = (double)(UINT32_MAX / 256);
  const double of_pages = (double)B * pages8_parts(N) * p.layers * 2 * p.Hkv;
  const double of_pieces = (double)B * ((N * row + 255) / 256) * p.layers * 2;
  if (of_pages > most || of_pieces > most) return DA_ERR_SHAPE;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4) || !aligned(cu, 4) || !aligned(ints, 4))
    return DA_ERR_ALIGN;
  return check_device();
}

}  // namespace
}  // namespace da

using namespace da;

extern "C" {

da_status da_pages8_resize(void* k_pages, void* v_pages, float* k_scales, float* v_scales, int layers, int Hkv,
                           int d, int32_t* table, int32_t* lens, int32_t* refs, int S, int M, int P,
                           const int32_t* slots, const int32_t* new_lens, int n, int32_t* result, void* stream) {
  const da_status st = check_scales(k_scales, v_scales);
  if (st != DA_OK) return st;
  // (a row of codes is as long as one of half as many bf16 values)
  const Pages p{(uint16_t*)k_pages, (uint16_t*)v_pages, layers, Hkv, d / 2, k_scales, v_scales};
  return resize_pages(p, d, {table, lens, refs, S, M, P}, slots, new_lens, n, result, stream);
}
da_status da_pages8_compact(void* k_pages, void* v_pages, float* k_scales, float* v_scales, int layers, int Hkv,
                            int d, int32_t* table, int32_t* lens, int32_t* refs, int S, int M, int P,
                            const int32_t* slots, const int32_t* start, const int32_t* keep, int64_t n_keep,
                            const int32_t* cu_keep, int n, int32_t* result, void* stream) {
  const Table t{table, lens, refs, S, M, P};
  const Pages8 p{(uint8_t*)k_pages, (uint8_t*)v_pages, k_scales, v_scales, layers, Hkv, d};
  da_status st = check_scales(k_scales, v_scales);
  if (st != DA_OK) return st;
  st = check_compact(t, k_pages, v_pages, layers, Hkv, d, slots, start, keep, n_keep, cu_keep, n, result);
  if (st != DA_OK) return st;
  return launched(launch_pages8_compact(t, p, slots, start, keep, n_keep, cu_keep, n, result, (hipStream_t)stream));
}

da_status da_pages8_append(const void* k, const void* v, int64_t T, void* k_pages, void* v_pages, float* k_scales,
                           float* v_scales, int layers, int Hkv, int d, const int32_t* table, const int32_t* lens,
                           int S, int M, int P, const int32_t* slots, const int32_t* cu_seqlens, int B,
                           int max_seqlen, const int32_t* new_lens, void* stream) {
  const Table t{const_cast<int32_t*>(table), const_cast<int32_t*>(lens), nullptr, S, M, P};
  const Pages8 p{(uint8_t*)k_pages, (uint8_t*)v_pages, k_scales, v_scales, layers, Hkv, d};
  const da_status st = check_rows8(t, p, k, v, T, slots, cu_seqlens, B, max_seqlen, new_lens);
  if (st != DA_OK) return st;
  return launched(launch_pages8_append(t, p, (const uint16_t*)k, (const uint16_t*)v, T, slots, cu_seqlens, B,
                                       max_seqlen, new_lens, (hipStream_t)stream));
}

da_status da_pages8_read(void* k, void* v, int64_t T, const void* k_pages, const void* v_pages,
                         const float* k_scales, const float* v_scales, int layers, int Hkv, int d,
                         const int32_t* table, const int32_t* lens, int S, int M, int P, const int32_t* slots,
                         const int32_t* cu_seqlens, int B, int max_seqlen, const int32_t* first, void* stream) {
  const Table t{const_cast<int32_t*>(table), const_cast<int32_t*>(lens), nullptr, S, M, P};
  const Pages8 p{(uint8_t*)const_cast<void*>(k_pages), (uint8_t*)const_cast<void*>(v_pages),
                 const_cast<float*>(k_scales), const_cast<float*>(v_scales), layers, Hkv, d};
  const da_status st = check_rows8(t, p, k, v, T, slots, cu_seqlens, B, max_seqlen, first);
  if (st != DA_OK) return st;
  return launched(launch_pages8_read(t, p, (uint16_t*)k, (uint16_t*)v, T, slots, cu_seqlens, B, max_seqlen, first,
                                     (hipStream_t)stream));
}

da_status da_page8_summary(const void* k_pages, const float* k_scales, int Hkv, int d, const int32_t* table,
                           const int32_t* lens, int S, int M, int P, const int32_t* slots, const int32_t* first,
                           int B, int max_new, void* codes, float* scales, void* stream) {
  const da_status st = check_scales(k_scales, k_scales);
  if (st != DA_OK) return st;
  return summarise_pages(k_pages, k_scales, Hkv, d,
                         {const_cast<int32_t*>(table), const_cast<int32_t*>(lens), nullptr, S, M, P}, slots, first, B,
                         max_new, codes, scales, stream);
}

size_t da_paged8_workspace_bytes(int B, int max_seqlen, int Hq, int Hkv, int d, int max_len, int n_list) {
  return paged_bytes(B, max_seqlen, Hq, Hkv, d, max_len, n_list, true);
}

da_status tree_attn_paged_scored(const void* q, const void* k_pages, const void* v_pages, void* out, float* lse,
                                 const int32_t* table, const int32_t* lens, int S, int M, int P,
                                 const int32_t* slots, const int32_t* cu_seqlens, int B, int max_seqlen,
                                 int max_len, int Hq, int Hkv, int d, const uint64_t* mask, int mask_words,
                                 float cap, const float* slopes, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  PagedArgs a = paged_args(q, k_pages, v_pages, out, lse, table, lens, S, M, P, slots, cu_seqlens, B, max_seqlen, Hq,
                           Hkv, d);
  a.slopes = slopes;
  a.mask = mask;
  a.mask_words = mask_words;
  return attend_pages(a, max_len, cap, workspace, workspace_bytes, stream);
}

da_status tree_attn_paged8(const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
                           const float* v_scales, void* out, float* lse, const int32_t* table,
                           const int32_t* lens, int S, int M, int P, const int32_t* slots,
                           const int32_t* cu_seqlens, int B, int max_seqlen, int max_len, int Hq, int Hkv, int d,
                           const uint64_t* mask, int mask_words, float cap, const float* slopes, void* workspace,
                           size_t workspace_bytes, void* stream) {
  const da_status st = check_scales(k_scales, v_scales);
  if (st != DA_OK) return st;
  PagedArgs a = paged_args(q, k_pages, v_pages, out, lse, table, lens, S, M, P, slots, cu_seqlens, B, max_seqlen, Hq,
                           Hkv, d);
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.slopes = slopes;
  a.mask = mask;
  a.mask_words = mask_words;
  return attend_pages(a, max_len, cap, workspace, workspace_bytes, stream);
}

da_status selected_attn_paged8(const void* q, const void* k_pages, const void* v_pages, const float* k_scales,
                               const float* v_scales, void* out, float* lse, const int32_t* table,
                               const int32_t* lens, int S, int M, int P, const int32_t* slots,
                               const int32_t* cu_seqlens, int B, int max_seqlen, int Hq, int Hkv, int d,
                               const int32_t* pages, int top_k, void* workspace, size_t workspace_bytes,
                               void* stream) {
  const da_status st = check_scales(k_scales, v_scales);
  if (st != DA_OK) return st;
  PagedArgs a = paged_args(q, k_pages, v_pages, out, lse, table, lens, S, M, P, slots, cu_seqlens, B, max_seqlen, Hq,
                           Hkv, d);
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  return attend_lists(a, pages, top_k, workspace, workspace_bytes, stream);
}

}  // extern "C"
