// da_pages8.hip -- a key/value cache held in 8 bits: quantising tokens as they are
// written, reading them back, compacting (gfx950).
//
// A page holds e4m3 codes of 64 tokens for each kv head, keys and values apart, and for
// each (page, kv head) a power of two 2^e that its codes count in:
//   code = x 2^-e rounded to e4m3 (to nearest, ties to even), value = code 2^e
//   e = the least with max |x| <= 448 2^e, held to [kLeastExp, kMostExp], over all tokens since the page was
//       last begun, those among them that have left it too: to lower it would take a pass over the page
//       and give back no bit that its codes have lost
// A floating point code loses nothing by a scale that is only a power of two, its values are
// bf16 without rounding, and codes that have to count in a larger scale, because a later token
// of the page needs it or because they move into another page, only shift their exponents:
// nothing is lost until they fall below e4m3's normal range (2^-14 of the page's largest).
// So the error of a cached value is its own rounding, 2^-4 of it at most, whatever came later, while it
// is 2^-6 of its scale or more.  Below, each growth rounds it to a multiple of 2^-9 of the new scale, by 2^-10
// of it at most; a growth doubles the scale or more, so all of them together stay under 2^-9 of the last one.
//
// A workgroup takes the rows that one page and kv head has of the keys or of the values: it
// alone writes them and their scale.  Bound by HBM where there are many, by a chain of reads
// (length, page entry, rows, scale) where there are few.
#include "da_device.hpp"
#include "da_paged.hpp"

namespace da {
namespace {

constexpr int kLeastExp = -110, kMostExp = 119;  // (codes times these are normal and finite in bf16)
constexpr uint32_t kInf = 0x7f80;                // bits of a bf16 infinity

typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bool page_ok(int e, int P) { return (unsigned)e < (unsigned)P; }
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The exponent of a page's scale, and what fits if something else stands there.
__device__ __forceinline__ int exp_of(float scale) {
  return min(max((int)(__float_as_uint(scale) >> 23 & 255u) - 127, kLeastExp), kMostExp);
}

// Largest magnitude (bf16 bits) of two values.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  const u16x2 m = __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b));
  return __builtin_bit_cast(uint32_t, m);
}
// Two values of a word: magnitudes that are finite, else 0.
__device__ __forceinline__ uint32_t finite2(uint32_t w) {
  const uint32_t lo = w & 0x7fffu, hi = w >> 16 & 0x7fffu;
  return (lo < kInf ? lo : 0u) | (hi < kInf ? hi : 0u) << 16;
}
// The least e with top <= 448 2^e = 1.75 2^(e + 8), for a magnitude's bf16 bits.
__device__ __forceinline__ int needed_exp(uint32_t top) {
  return min(max((int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0), kLeastExp), kMostExp);
}

// Four values (two words) to codes counted in `scale`, a power of two that brings them within 448.
__device__ __forceinline__ uint32_t codes_of(uint32_t w0, uint32_t w1, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
  i16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, w0), scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, w1), scale, true);
  return __builtin_bit_cast(uint32_t, r);
#else
  return 0u;
#endif
}
// The same of any values: those past 448 scale count as that, what is not finite becomes NaN.
__device__ __forceinline__ uint32_t codes_of_any(uint32_t w0, uint32_t w1, int e) {
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = ((i < 2 ? w0 : w1) >> (16 * (i & 1))) & 0xffffu;
    const float f = fminf(fmaxf(__uint_as_float(x << 16) * pow2(-e), -448.f), 448.f);
    const uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f, f, 0, false) & 0xffu;
    out |= ((x & 0x7fffu) < kInf ? c : 0x7fu) << (8 * i);
  }
  return out;
}

// Four codes as two words of bf16 values.
__device__ __forceinline__ void values_of(uint32_t c, float scale, uint32_t& w0, uint32_t& w1) {
#if defined(__HIP_DEVICE_COMPILE__)
  w0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false));
  w1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true));
#endif
}
// Codes that counted in 2^e count in 2^(e + up) from here on, up >= 0.
__device__ __forceinline__ u32x4 recoded(u32x4 c, int up) {
  const float down = pow2(-min(up, 64));  // (past 2^18 everything is 0)
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w0 = 0, w1 = 0;
    values_of(c[i], down, w0, w1);
    r[i] = codes_of(w0, w1, 1.f);
  }
  return r;
}

// The maximum over a workgroup of NT threads, in every thread (all of them call it; `lds` is not
// in use by another call).
template <int NT>
__device__ __forceinline__ int block_max(int x, int* lds) {
  x = wave_reduce(x, INT32_MIN, [](int a, int b) { return max(a, b); });
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) x = max(x, lds[w]);
  }
  return x;
}

// What a workgroup does: (layer, keys or values, sequence, page of its range, kv head).
struct Item {
  int b, part, h;
  int64_t layer;
  bool values;
};
__device__ __forceinline__ Item item_of(uint32_t i, int Hkv, int B, int parts) {
  Item x;
  x.h = (int)(i % (uint32_t)Hkv);
  i /= (uint32_t)Hkv;
  x.part = (int)(i % (uint32_t)parts);
  i /= (uint32_t)parts;
  x.b = (int)(i % (uint32_t)B);
  i /= (uint32_t)B;
  x.values = i & 1u;
  x.layer = i >> 1;
  return x;
}

// New tokens become the last ones of their sequences, as codes; a page gets up to ROWS of them.  Bound by
// HBM: 87302 tokens of 8 kv heads, d 128, 0.36 GB read and 0.18 GB written in 101 us, 5.3 TB/s (104 with keys
// and values in turn; 111 with 512 threads).  A few tokens per sequence take a wavefront for 16 rows, so
// that all of a batch's run at once: 64 sequences of 16 drafts, 4 layers 15.1 -> 7.6 us.
template <int D, int NT, int ROWS>
__global__ __launch_bounds__(NT) void append8_kernel(Table t, Pages8 p, const uint16_t* __restrict__ k,
                                                     const uint16_t* __restrict__ v, int64_t T,
                                                     const int32_t* __restrict__ slots,
                                                     const int32_t* __restrict__ cu, int B, int N, int parts,
                                                     const int32_t* __restrict__ new_lens) {
  constexpr int kPer = D / 16, kRows = NT / kPer, kSteps = (ROWS + kRows - 1) / kRows;  // 16 values per thread and step
  __shared__ int red[NT / 64];
  const Item it = item_of(blockIdx.x, p.Hkv, B, parts);
  const int tid = threadIdx.x, b = it.b;
  const int64_t base = cu ? cu[b] : (int64_t)b * N;
  const int m = min(cu ? cu[b + 1] - cu[b] : N, N);
  const int s = slots ? slots[b] : b;
  if ((unsigned)s >= (unsigned)t.S || m <= 0 || base < 0 || base + m > T) return;
  const int len = t.lens[s];
  if (new_lens && len != new_lens[b]) return;
  const int64_t start = (int64_t)len - m, end = min((int64_t)len, (int64_t)t.M * kPage);
  const int64_t page0 = (max(start, (int64_t)0) / kPage + it.part) * kPage;
  const int r0 = (int)(max(start, page0) - page0), r1 = (int)min(end - page0, (int64_t)kPage);
  if (r0 >= r1) return;
  const int e = t.table[(int64_t)s * t.M + page0 / kPage];
  if (!page_ok(e, t.P)) return;

  const int64_t place = (it.layer * t.P + e) * p.Hkv + it.h;
  float* const scale = (it.values ? p.v_scales : p.k_scales) + place;
  uint8_t* const tile = (it.values ? p.v : p.k) + place * (kPage * D);
  const int rr = tid / kPer, c = tid % kPer;
  const uint16_t* const src = (it.values ? v : k) + ((it.layer * T + base + (page0 + r0 - start)) * p.Hkv + it.h) * D + c * 16;
  const int64_t stride = (int64_t)p.Hkv * D;
  const float held = r0 ? *scale : 0.f;
  u32x4 x[kSteps][2];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int row = i * kRows + rr;
    x[i][0] = x[i][1] = u32x4{};
    if (row < r1 - r0) {
      x[i][0] = *(const u32x4*)(src + row * stride);
      x[i][1] = *(const u32x4*)(src + row * stride + 8);
    }
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
#pragma unroll
    for (int q = 0; q < 8; ++q) top = max2(top, x[i][q / 4][q % 4] & 0x7fff7fffu);
  top = max(top & 0xffffu, top >> 16);
  bool odd = top >= kInf;  // something is not finite: the largest of the rest
  if (odd) {
    top = 0;
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int q = 0; q < 8; ++q) top = max2(top, finite2(x[i][q / 4][q % 4]));
    top = max(top & 0xffffu, top >> 16);
  }
  top = (uint32_t)block_max<NT>((int)top, red);
  int exp = needed_exp(top);
  const int was = r0 ? exp_of(held) : exp;
  exp = max(exp, was);
  odd = odd || exp == kMostExp;
  const float unit = pow2(exp);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int row = i * kRows + rr;
    if (row >= r1 - r0) break;
    u32x4 y;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t w0 = x[i][q / 2][2 * (q % 2)], w1 = x[i][q / 2][2 * (q % 2) + 1];
      y[q] = odd ? codes_of_any(w0, w1, exp) : codes_of(w0, w1, unit);
    }
    *(u32x4*)(tile + (r0 + row) * D + c * 16) = y;
  }
  // the tokens that the page held before
  if (exp > was)
    for (int u = tid; u < r0 * kPer; u += NT) {
      u32x4* const at = (u32x4*)(tile + u * 16);
      *at = recoded(*at, exp - was);
    }
  if (tid == 0) *scale = unit;
}

// Tokens of the cache as rows of bf16.  A thread turns 16 codes into 32 bytes, in the order of the rows, a
// sequence after the other: a workgroup's stores are one stretch of memory, its loads the rows that a
// few tokens have in their pages.  Bound by HBM: 64 sequences of up to 8192 tokens, 8 kv heads, d 128, 0.68
// GB read and 1.37 GB written in 358 us, 5.7 TB/s (a page and head per workgroup, as in the append, 437; two
// and four pieces per thread 373, the sequences' workgroups in turn 424).
template <int D>
__global__ __launch_bounds__(256) void read8_kernel(Table t, Pages8 p, uint16_t* __restrict__ k,
                                                    uint16_t* __restrict__ v, int64_t T,
                                                    const int32_t* __restrict__ slots,
                                                    const int32_t* __restrict__ cu, int N, unsigned parts,
                                                    const int32_t* __restrict__ first) {
  constexpr int kPer = D / 16;
  const int b = (int)(blockIdx.x / parts);
  const unsigned u = blockIdx.x % parts * 256 + threadIdx.x;
  const int64_t layer = blockIdx.y >> 1;
  const bool values = blockIdx.y & 1;
  const int64_t base = cu ? cu[b] : (int64_t)b * N;
  const int m = min(cu ? cu[b + 1] - cu[b] : N, N);
  const int s = slots ? slots[b] : b;
  if ((unsigned)s >= (unsigned)t.S || m <= 0 || base < 0 || base + m > T) return;
  const unsigned row = (unsigned)p.Hkv * kPer;  // pieces of a token
  const int i = (int)(u / row);
  const unsigned w = u % row;
  const int start = first ? first[b] : 0;
  const int64_t pos = (int64_t)start + i;
  if (i >= m || start < 0 || pos >= min((int64_t)t.lens[s], (int64_t)t.M * kPage)) return;
  const int e = t.table[(int64_t)s * t.M + pos / kPage];
  if (!page_ok(e, t.P)) return;
  const int64_t place = (layer * t.P + e) * p.Hkv + w / kPer;
  const u32x4 x = *(const u32x4*)((values ? p.v : p.k) + (place * kPage + pos % kPage) * D + w % kPer * 16);
  const float scale = (values ? p.v_scales : p.k_scales)[place];
  u32x4 y[2];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t w0 = 0, w1 = 0;
    values_of(x[q], scale, w0, w1);
    y[q / 2][2 * (q % 2)] = w0;
    y[q / 2][2 * (q % 2) + 1] = w1;
  }
  u32x4* const at = (u32x4*)((values ? v : k) + ((layer * T + base + i) * p.Hkv * (int64_t)D + w * 16));
  at[0] = y[0];
  at[1] = y[1];
}

// Compacting, behind the check that the bf16 cache has: a workgroup per (request, layer, keys or
// values, kv head) moves its rows up, one page that takes rows after the other.  That page counts
// in the largest of the scales that its rows had, those that stay in it among them.  A row never
// moves down, so a page's rows come from itself and later ones: all are read before any is
// written, and the pages written before are read no more.
template <int D>
__global__ __launch_bounds__(256) void compact8_kernel(Table t, Pages8 p, const int32_t* __restrict__ slots,
                                                       const int32_t* __restrict__ start,
                                                       const int32_t* __restrict__ keep,
                                                       const int32_t* __restrict__ cu_keep, int n,
                                                       int32_t* __restrict__ result) {
  constexpr int kPer = D / 16, kRows = 256 / kPer, kSteps = kPage / kRows;
  __shared__ int red[4];
  __shared__ int left;
  uint32_t blk = blockIdx.x;
  const int i = (int)(blk % (uint32_t)n);
  blk /= (uint32_t)n;
  const int4 r = ((const int4*)result)[i];
  if (r.x < 0) return;  // refused
  const int h = (int)(blk % (uint32_t)p.Hkv);
  blk /= (uint32_t)p.Hkv;
  const bool values = blk & 1u;
  const int64_t layer = blk >> 1;
  const int st = start[i], slot = slots[i], tid = threadIdx.x;
  const int32_t* const kp = keep + cu_keep[i];
  int32_t* const row = t.table + (int64_t)slot * t.M;
  float* const scales = (values ? p.v_scales : p.k_scales) + layer * t.P * p.Hkv + h;
  uint8_t* const tiles = (values ? p.v : p.k) + (layer * t.P * p.Hkv + h) * (int64_t)(kPage * D);
  const int64_t page_bytes = (int64_t)p.Hkv * kPage * D;
  const int rr = tid / kPer, c = tid % kPer;
  for (int j0 = r.y; j0 < r.x;) {
    const int to0 = (st + j0) % kPage;                 // first row that is written
    const int count = min(r.x - j0, kPage - to0);      // rows
    const int to = row[(st + j0) / kPage];             // (a page: the check has seen it)
    u32x4 x[kSteps];
    int from_exp[kSteps], top = kLeastExp;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int j = j0 + min(u * kRows + rr, count - 1);
      const int from = st + kp[j];
      const int e = row[from / kPage];
      x[u] = u32x4{};
      from_exp[u] = kLeastExp;
      if (page_ok(e, t.P)) {
        x[u] = *(const u32x4*)(tiles + e * page_bytes + (from % kPage) * D + c * 16);
        from_exp[u] = exp_of(scales[(int64_t)e * p.Hkv]);
      }
      top = max(top, from_exp[u]);
    }
    uint8_t* const tile = tiles + to * page_bytes;
    float* const scale = scales + (int64_t)to * p.Hkv;
    const int was = to0 ? exp_of(*scale) : kLeastExp;
    top = max(block_max<256>(top, red), was);  // (with a barrier: every row is read)
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int w = u * kRows + rr;
      if (w >= count) break;
      *(u32x4*)(tile + (to0 + w) * D + c * 16) = top > from_exp[u] ? recoded(x[u], top - from_exp[u]) : x[u];
    }
    if (to0 && top > was)
      for (int u = tid; u < to0 * kPer; u += 256) {
        u32x4* const at = (u32x4*)(tile + u * 16);
        *at = recoded(*at, top - was);
      }
    if (tid == 0) *scale = pow2(top);
    j0 += count;
    __syncthreads();  // (red is read; and the rows written are this page's last)
  }
  // The last of a request's workgroups, which all have read the table by then, gives back the
  // pages past the new end (result[i].w counts them from 0).
  const int c0 = (st + r.x + kPage - 1) / kPage, c1 = (r.z + kPage - 1) / kPage;
  if (c0 >= c1) return;
  __syncthreads();
  if (tid == 0) left = p.layers * 2 * p.Hkv - 1 - atomicAdd(result + 4 * i + 3, 1);
  __syncthreads();
  if (left == 0)
    for (int q = c0 + tid; q < c1; q += 256) {
      const int e = row[q];
      if (page_ok(e, t.P)) atomicSub(t.refs + e, 1);
      row[q] = -1;
    }
}

}  // namespace

hipError_t launch_pages8_append(const Table& t, const Pages8& p, const uint16_t* k, const uint16_t* v,
                                int64_t T, const int32_t* slots, const int32_t* cu, int B, int N,
                                const int32_t* new_lens, hipStream_t s) {
  const int parts = pages8_parts(N);
  const dim3 g((unsigned)((int64_t)B * parts * p.layers * 2 * p.Hkv));
#define DA_APPEND8(NT, ROWS)                                                                             \
  do {                                                                                                   \
    if (p.d == 128)                                                                                      \
      hipLaunchKernelGGL((append8_kernel<128, NT, ROWS>), g, dim3(NT), 0, s, t, p, k, v, T, slots, cu, B, N, parts, new_lens); \
    else                                                                                                 \
      hipLaunchKernelGGL((append8_kernel<64, NT, ROWS>), g, dim3(NT), 0, s, t, p, k, v, T, slots, cu, B, N, parts, new_lens);  \
  } while (0)
  if (N <= 16)
    DA_APPEND8(64, 16);
  else
    DA_APPEND8(256, 64);
#undef DA_APPEND8
  return hipGetLastError();
}

hipError_t launch_pages8_read(const Table& t, const Pages8& p, uint16_t* k, uint16_t* v, int64_t T,
                              const int32_t* slots, const int32_t* cu, int B, int N, const int32_t* first,
                              hipStream_t s) {
  const int64_t parts = ((int64_t)N * p.Hkv * (p.d / 16) + 255) / 256;
  const dim3 g((unsigned)(parts * B), p.layers * 2);
  if (p.d == 128)
    hipLaunchKernelGGL(read8_kernel<128>, g, dim3(256), 0, s, t, p, k, v, T, slots, cu, N, (unsigned)parts, first);
  else
    hipLaunchKernelGGL(read8_kernel<64>, g, dim3(256), 0, s, t, p, k, v, T, slots, cu, N, (unsigned)parts, first);
  return hipGetLastError();
}

hipError_t launch_pages8_compact(const Table& t, const Pages8& p, const int32_t* slots, const int32_t* start,
                                 const int32_t* keep, int64_t n_keep, const int32_t* cu_keep, int n,
                                 int32_t* result, hipStream_t s) {
  const hipError_t e = launch_compact_check(t, slots, start, keep, n_keep, cu_keep, n, result, s);
  if (e != hipSuccess) return e;
  const dim3 g((unsigned)(n * p.layers * 2 * p.Hkv));
  if (p.d == 128)
    hipLaunchKernelGGL(compact8_kernel<128>, g, dim3(256), 0, s, t, p, slots, start, keep, cu_keep, n, result);
  else
    hipLaunchKernelGGL(compact8_kernel<64>, g, dim3(256), 0, s, t, p, slots, start, keep, cu_keep, n, result);
  return hipGetLastError();
}

}  // namespace da
