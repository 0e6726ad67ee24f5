// The host layer of the cache in 8 bits and of attention over it (da_pages8_api.cpp on top of
// da_paged_api.cpp, compiled for the host only) with stub launchers that keep what a kernel would get.
// Built under AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_sanitizers_pages8.py: sizes
// at the ends of what the calls take must neither wrap nor pass as others.
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "da_paged.hpp"
#include "delta_attn.h"

namespace da {
static int g_launched = 0;
static int64_t g_n = 0;
static PagedArgs g_paged;
da_status check_device() { return DA_OK; }
da_status fail_hip(hipError_t) { return DA_ERR_HIP; }
static hipError_t went(int64_t n) { ++g_launched; g_n = n; return hipSuccess; }
hipError_t launch_pages_fork(const Table&, const int32_t*, const int32_t*, int, int32_t*, hipStream_t) { return went(0); }
hipError_t launch_pages_resize(const Table&, const Pages& p, const int32_t*, const int32_t*, int, int32_t*, hipStream_t) { return went(p.d); }
hipError_t launch_pages_append(const Table&, const Pages&, const uint16_t*, const uint16_t*, int64_t, const int32_t*, const int32_t*, int, int, const int32_t*, hipStream_t) { return went(0); }
hipError_t launch_pages_compact(const Table&, const Pages&, const int32_t*, const int32_t*, const int32_t*, int64_t, const int32_t*, int, int32_t*, hipStream_t) { return went(0); }
hipError_t launch_pages8_append(const Table&, const Pages8& p, const uint16_t*, const uint16_t*, int64_t, const int32_t*, const int32_t*, int B, int N, const int32_t*, hipStream_t) {
  return went((int64_t)B * pages8_parts(N) * p.layers * 2 * p.Hkv);
}
hipError_t launch_pages8_read(const Table&, const Pages8& p, uint16_t*, uint16_t*, int64_t, const int32_t*, const int32_t*, int B, int N, const int32_t*, hipStream_t) {
  return went((int64_t)B * (((int64_t)N * p.Hkv * (p.d / 16) + 255) / 256) * p.layers * 2);
}
hipError_t launch_pages8_compact(const Table&, const Pages8&, const int32_t*, const int32_t*, const int32_t*, int64_t, const int32_t*, int, int32_t*, hipStream_t) { return went(0); }
hipError_t launch_summary(const SummaryArgs&, hipStream_t) { return went(0); }
hipError_t launch_select_blocks(const SelectArgs&, hipStream_t) { return went(0); }
hipError_t launch_select_pages(const SelectArgs&, hipStream_t) { return went(0); }
hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t) { g_paged = a; return went(0); }
}  // namespace da

using namespace da;

static int failures = 0;
static void expect(int64_t got, int64_t want, const char* what, int64_t at = 0) {
  if (got != want) {
    fprintf(stderr, "%s (%lld): %lld, expected %lld\n", what, (long long)at, (long long)got, (long long)want);
    ++failures;
  }
}

alignas(16) static char room[16];
static char* const p = room;
static int32_t* const i32 = (int32_t*)room;
static float* const f32 = (float*)room;

static int append(int layers, int Hkv, int d, int B, int N, int S) {
  return da_pages8_append(p, p, 0, p, p, f32, f32, layers, Hkv, d, i32, i32, S, 4, 4, i32, i32, B, N, nullptr, nullptr);
}
static int read(int layers, int Hkv, int d, int B, int N, int S) {
  return da_pages8_read(p, p, 0, p, p, f32, f32, layers, Hkv, d, i32, i32, S, 4, 4, i32, i32, B, N, nullptr, nullptr);
}

// A launch's workgroups of 256 threads fit 32 bits, or the call is refused: no size wraps into that.
static void sizes_of_rows() {
  const int64_t sizes[] = {1, 2, 63, 64, 65, 1000, 4096, 32767, 65536, 1 << 20, (1 << 20) + 1, INT32_MAX / 2, INT32_MAX - 63, INT32_MAX};
  for (int64_t layers : {1, 2, 32767})
    for (int64_t Hkv : sizes)
      for (int d : {64, 128})
        for (int64_t B : sizes)
          for (int64_t N : sizes) {
            const __int128 row = (__int128)Hkv * (d / 16);
            const __int128 by_page = (__int128)B * layers * 2 * Hkv * ((N + 62) / 64 + 1);
            const __int128 by_piece = (__int128)B * layers * 2 * ((N * row + 255) / 256);
            const bool ok = row * N <= INT32_MAX && by_page < 1 << 24 && by_piece < 1 << 24;
            const int before = g_launched;
            expect(append((int)layers, (int)Hkv, d, (int)B, (int)N, 4), ok ? DA_OK : DA_ERR_SHAPE, "append", N);
            if (ok) expect(g_n, (int64_t)by_page, "workgroups of an append", N);
            expect(read((int)layers, (int)Hkv, d, (int)B, (int)N, 4), ok ? DA_OK : DA_ERR_SHAPE, "read", N);
            if (ok) expect(g_n, (int64_t)by_piece, "workgroups of a read", N);
            expect(g_launched - before, ok ? 2 : 0, "launches", N);
          }
  expect(append(1, 8, 96, 1, 1, 4), DA_ERR_UNSUPPORTED, "d 96");
  expect(append(0, 8, 64, 1, 1, 4), DA_ERR_SHAPE, "no layer");
  expect(da_pages8_append(p, p, 5, p, p, f32, f32, 1, 1, 64, i32, i32, 4, 4, 4, i32, nullptr, 2, 3, nullptr, nullptr), DA_ERR_SHAPE, "tokens that are not B * N");
}

// A row of codes is moved as half as many words of 16 bits.
static void resize_moves_half() {
  for (int d : {64, 128}) {
    expect(da_pages8_resize(p, p, f32, f32, 1, 2, d, i32, i32, i32, 4, 4, 4, i32, i32, 1, i32, nullptr), DA_OK, "resize");
    expect(g_n, d / 2, "words of a row", d);
  }
  for (int d : {32, 96, 256})
    expect(da_pages8_resize(p, p, f32, f32, 1, 2, d, i32, i32, i32, 4, 4, 4, i32, i32, 1, i32, nullptr), DA_ERR_UNSUPPORTED, "resize", d);
}

static int attend(float cap, const float* slopes, const uint64_t* mask, int words, int B, int N, int max_len, int Hq, int Hkv, size_t bytes) {
  return tree_attn_paged8(p, p, p, f32, f32, p, nullptr, i32, i32, INT32_MAX, INT32_MAX / 64, INT32_MAX, i32, i32, B, N,
                          max_len, Hq, Hkv, 128, mask, words, cap, slopes, p, bytes, nullptr);
}

// Plans at the ends: whatever passes has a workspace of the size that is told, and is refused one byte less.
static void plans() {
  for (int B : {1, 3, 64, 1000, 100000})
    for (int N : {1, 2, 24, 64, 2000})
      for (int max_len : {1, 64, 65, 5000, 1 << 20, INT32_MAX - 63})
        for (int G : {1, 4, 16}) {
          const size_t bytes = da_paged8_workspace_bytes(B, N, 8 * G, 8, 128, max_len, 0);
          const int st = attend(0.f, nullptr, nullptr, 0, B, N, max_len, 8 * G, 8, bytes);
          if (bytes) {
            expect(st, DA_OK, "attend", max_len);
            expect(attend(0.f, nullptr, nullptr, 0, B, N, max_len, 8 * G, 8, bytes - 1), DA_ERR_WORKSPACE, "a byte less", max_len);
          } else {
            expect(st == DA_OK || st == DA_ERR_SHAPE, 1, "attend without a workspace", max_len);
          }
        }
  for (int k : {INT32_MIN, -1, INT32_MAX}) (void)da_paged8_workspace_bytes(k, k, k, k, 128, k, k);
}

static void caps() {
  for (float cap : {0.f, -0.f, 9.765625e-4f, 1.f, 50.f, 1024.f}) expect(attend(cap, f32, nullptr, 0, 1, 1, 64, 8, 8, 0), DA_OK, "cap", (int64_t)cap);
  for (float cap : {-1.f, 9.76e-4f, 1.4e-45f, 1025.f, 3.4e38f, INFINITY, -INFINITY, NAN})
    expect(attend(cap, nullptr, nullptr, 0, 1, 1, 64, 8, 8, 0), DA_ERR_PARAM, "cap that is refused");
  expect(attend(0.f, f32, (const uint64_t*)p, 1, 1, 4, 64, 8, 8, 0), DA_ERR_PARAM, "slopes with a mask");
}

int main() {
  sizes_of_rows();
  resize_moves_half();
  plans();
  caps();
  if (failures) return 1;
  printf("pages8 driver ok\n");
  return 0;
}
