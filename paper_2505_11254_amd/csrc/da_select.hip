// da_select.hip -- which key blocks a group of queries attends to (gfx950):
// 8-bit summaries of blocks of 64 keys, scores of queries against them, and the
// top_k blocks of each group.
//
//   summary of a block:  S_c = sum of its 64 keys' channel c,  A = max_c |S_c|,
//     code_c = round(127 S_c / A),  scale = A / (127 * 64)   (the mean key is about
//     code * scale)
//   a group's queries:   a = max |q| over all its rows and channels,
//     q8 = round(127 q / a)
//   score of a block:    scale * max over the group's rows of sum_c q8_c code_c
//
// Rounding is to nearest, ties to even.  The inner sums are whole numbers below
// 2^21, exact in 32 bits in any order, and the scale enters by one multiplication:
// scores do not depend on how the work is cut, so neither do the blocks chosen.
// (a is common to the group and drops out of the order of its scores.)  The sums
// S_c are taken in 64-bit floats, where 64 bf16 values of one channel add exactly
// unless their magnitudes lie more than 2^38 apart.
//
// The products run on v_mfma_i32_32x32x32_i8 with the queries' rows down the
// accumulator and the blocks across it, so that a lane holds 16 rows' products with
// one block and their maximum takes eight 3-input instructions, no exchange.
#include "da_device.hpp"
#include "da_paged.hpp"

#include <type_traits>

namespace da {
namespace {

typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float bf16_float(uint32_t bits) { return __uint_as_float(bits << 16); }

__device__ __forceinline__ i32x16 mfma_i8(i32x4 a, i32x4 b, i32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

// ---------------------------------------------------------------- summaries
//
// A wavefront per (block, kv head): D/8 lanes read a key's row, 16 bytes each, so
// that 512/D keys arrive per load.  The lanes that hold the same eight channels then
// halve the sums they keep as they add them up, and each finishes one or two channels.
// Every key is read once, 1/64 of that written; the conversions and sums in 64 bits
// take about as long as the loads.
template <int D>
__global__ __launch_bounds__(256) void summary_kernel(SummaryArgs a) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes, kSteps = kPage / kRows;
  const int lane = threadIdx.x & 63;
  const uint32_t item = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const uint32_t x = item / (uint32_t)a.Hkv;
  const int h = (int)(item - x * (uint32_t)a.Hkv);
  const int b = (int)(x / (uint32_t)a.nblk);
  int j = (int)(x - (uint32_t)b * (uint32_t)a.nblk);
  if (b >= a.B) return;
  int64_t block;  // where the summary goes
  const uint16_t* k;
  int64_t stride;
  if (a.table) {
    const int s = a.slots ? a.slots[b] : b;
    if ((unsigned)s >= (unsigned)a.S) return;
    const int first = a.first ? a.first[b] : 0;
    if (first < 0) return;
    j += first / kPage;
    if (j >= a.M || (j + 1) * (int64_t)kPage > a.lens[s]) return;
    const int e = a.table[(int64_t)s * a.M + j];
    if ((unsigned)e >= (unsigned)a.P) return;
    block = e;
    k = a.k + ((int64_t)e * a.Hkv + h) * kPage * D;
    stride = D;
  } else {
    const int64_t base = a.cu ? a.cu[b] : (int64_t)b * a.N;
    const int L = a.cu ? a.cu[b + 1] - a.cu[b] : a.N;
    if ((j + 1) * (int64_t)kPage > L) return;
    block = base / kPage + b + j;
    stride = (int64_t)a.Hkv * D;
    k = a.k + (base + (int64_t)j * kPage) * stride + h * D;
  }
  const int c = lane % kLanes, r = lane / kLanes;
  u32x4 w[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) w[i] = *(const u32x4*)(k + (i * kRows + r) * stride + c * 8);
  double sum[8] = {};
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[2 * q] += (double)bf16_float(w[i][q] & 0xffffu);
      sum[2 * q + 1] += (double)__uint_as_float(w[i][q] & 0xffff0000u);
    }
  // Lanes a power of two apart exchange the halves that the other keeps: those with the
  // bit set keep the upper one.
  int q0 = 0;
  auto halve = [&](auto width, int d) {
    constexpr int kKept = decltype(width)::value;
    const bool up = lane & d;
    q0 += up ? kKept : 0;
#pragma unroll
    for (int q = 0; q < kKept; ++q) {
      const double other = __shfl_xor(up ? sum[q] : sum[q + kKept], d);
      sum[q] = (up ? sum[q + kKept] : sum[q]) + other;
    }
  };
  halve(std::integral_constant<int, 4>{}, 32);
  halve(std::integral_constant<int, 2>{}, 16);
  if (kLanes == 8) halve(std::integral_constant<int, 1>{}, 8);
  constexpr int kMine = 8 * kLanes / 64;  // channels that this lane finishes, from q0 on
  double top = fabs(sum[0]);
  if (kMine == 2) top = fmax(top, fabs(sum[1]));
  top = wave_dmax(top);
  auto code = [&](double x) { return (uint32_t)((top > 0. ? (int)rint(x * 127. / top) : 0) & 0xff); };
  uint8_t* const out = (uint8_t*)a.codes + (block * a.Hkv + h) * D + c * 8 + q0;
  if (kMine == 2)
    *(uint16_t*)out = (uint16_t)(code(sum[0]) | code(sum[1]) << 8);
  else
    *out = (uint8_t)code(sum[0]);
  if (lane == 0) a.scales[block * a.Hkv + h] = (float)(top / (127. * kPage));
}

// ------------------------------------------------------------------- top_k
//
// The top_k of n keys by value, ties to the lowest index.  Rounds narrow the range of
// values that holds the smallest chosen one: its keys' least and greatest value, a
// histogram of kBins equal steps between them (in LDS, by atomics; steps of a range
// that fits the keys spread them, where their leading bits alone would pile them up on
// few counters), and the step that the count from above ends in, until that step holds
// one value or just as many keys as are chosen.  32-bit keys need at most three
// rounds of 2048 steps, scores two as a rule.  Then one pass ranks the chosen ones in
// ascending order: stripes of NT keys, each wave's counts in a table, a prefix sum
// over (stripe, wave).  Thread tid owns keys tid, tid + NT, ...; each(f) calls
// f(stripe, index, key) for those of all stripes, index >= n where there is none.
// emit(rank, index) is called once per chosen key.
constexpr uint32_t kForced = 0xffffffffu;  // always chosen (never more than top_k are)
constexpr uint32_t kAbsent = 0u;           // chosen last

template <int NT, int MAX>
struct TopK {
  static constexpr int kWaves = NT / 64;
  static constexpr int kBins = 2048;
  static constexpr int kPer = kBins / NT;  // of a thread
  static constexpr int kMaxStripes = (MAX + NT - 1) / NT;
  int hist[kBins];
  int table[2][kMaxStripes * kWaves];
  int scan[3][kWaves];
  uint32_t ends[2][kWaves];
  uint32_t bin;
  int need, all;
};

template <int NT, int MAX, typename Each, typename Emit>
__device__ __forceinline__ void select_top(TopK<NT, MAX>& t, int n, int top_k, Each each, Emit emit) {
  using TK = TopK<NT, MAX>;
  constexpr int W = TK::kWaves;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (n <= top_k) {
    for (int i = tid; i < n; i += NT) emit(i, i);
    return;
  }
  // members: keys in [lo, hi]; `need` of them are chosen, and every key above
  uint32_t lo = 1, hi = kForced - 1;
  int need = top_k;
  for (bool first = true;; first = false) {
    uint32_t mn = ~0u, mx = 0;
    int forced = 0, members = 0;
    each([&](int, int i, uint32_t x) {
      if (i >= n) return;
      const bool in = x >= lo && x <= hi;
      mn = in ? min(mn, x) : mn;
      mx = in ? max(mx, x) : mx;
      members += in;
      forced += x == kForced;
    });
    mn = (uint32_t)wave_reduce((int)mn, -1, [](int x, int y) { return (int)min((uint32_t)x, (uint32_t)y); });
    mx = (uint32_t)wave_reduce((int)mx, 0, [](int x, int y) { return (int)max((uint32_t)x, (uint32_t)y); });
    members = wave_add(members);
    forced = wave_add(forced);
    if (lane == 0) {
      t.ends[0][wave] = mn;
      t.ends[1][wave] = mx;
      t.scan[0][wave] = members;
      t.scan[1][wave] = forced;
    }
#pragma unroll
    for (int j = 0; j < TK::kPer; ++j) t.hist[j * NT + tid] = 0;
    __syncthreads();
    members = forced = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      mn = min(mn, t.ends[0][w]);
      mx = max(mx, t.ends[1][w]);
      members += t.scan[0][w];
      forced += t.scan[1][w];
    }
    if (first) {
      if (forced >= need) {  // (scores past the range of floats count as forced: the first of them)
        lo = kForced;
        break;
      }
      need -= forced;
      if (members < need) {  // all of them, and the first absent ones
        lo = kAbsent;
        need -= members;
        break;
      }
    }
    const int bits = 32 - __clz((int)(mx - mn));  // 0 for a single value
    const int sh = max(0, bits - (31 - __clz(TK::kBins)));
    each([&](int, int i, uint32_t x) {
      if (i < n && x >= lo && x <= hi) atomicAdd(&t.hist[(x - mn) >> sh], 1);
    });
    __syncthreads();
    // thread tid holds kPer steps, the highest of all threads' first
    int c[TK::kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < TK::kPer; ++j) sum += c[j] = t.hist[TK::kBins - 1 - TK::kPer * tid - j];
    int upto = wave_scan_add(sum);
    if (lane == 63) t.scan[2][wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += t.scan[2][w];
    int before = upto - sum;
    if (before < need && upto >= need) {
#pragma unroll
      for (int j = 0; j < TK::kPer; ++j) {
        if (before < need && before + c[j] >= need) {
          t.bin = TK::kBins - 1 - TK::kPer * tid - j;
          t.need = need - before;
          t.all = before + c[j] == need;
        }
        before += c[j];
      }
    }
    __syncthreads();
    need = t.need;
    lo = mn + (t.bin << sh);
    if (t.all) {  // every key of the step is chosen
      --lo;
      need = 0;
      break;
    }
    if (sh == 0) break;
    hi = lo + min(mx - lo, (1u << sh) - 1u);
  }
  // keys above lo are chosen, and the first `need` equal to it
  each([&](int s, int i, uint32_t x) {
    const uint64_t above = __ballot(i < n && x > lo), same = __ballot(i < n && x == lo);
    if (lane == 0) {
      t.table[0][s * W + wave] = __popcll(above);
      t.table[1][s * W + wave] = __popcll(same);
    }
  });
  __syncthreads();
  // exclusive prefix sums of the tables: a thread per run of entries
  const int entries = (n + NT - 1) / NT * W, per = (entries + NT - 1) / NT;
  int sum[2] = {0, 0};
  for (int j = 0; j < per; ++j) {
    const int e = tid * per + j;
    if (e < entries) {
      sum[0] += t.table[0][e];
      sum[1] += t.table[1][e];
    }
  }
  int before[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int x = wave_scan_add(sum[q]);
    if (lane == 63) t.scan[q][wave] = x;
    before[q] = x - sum[q];
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    for (int w = 0; w < wave; ++w) before[q] += t.scan[q][w];
    for (int j = 0; j < per; ++j) {
      const int e = tid * per + j;
      if (e < entries) {
        const int x = t.table[q][e];
        t.table[q][e] = before[q];
        before[q] += x;
      }
    }
  }
  __syncthreads();
  each([&](int s, int i, uint32_t x) {
    const bool above = i < n && x > lo, same = i < n && x == lo;
    const uint64_t lower = (1ull << lane) - 1;
    const int na = t.table[0][s * W + wave] + __popcll(__ballot(above) & lower);
    const int ns = t.table[1][s * W + wave] + __popcll(__ballot(same) & lower);
    if (above || (same && ns < need)) emit(na + min(ns, need), i);
  });
}

// A score as a whole number that orders as it does (+0 and -0 alike).
__device__ __forceinline__ uint32_t order_bits(float x) {
  const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Codes round(127 x / top) of a group's queries.  The quotient q0 = 127 x / top comes from
// the hardware's reciprocal and one correction, whose relative error is below 2^-22.
// That rounds as the exact quotient does: 127 x / top is 127 a / (b 2^e) with bf16
// significands a, b < 256, so it lies on a tie or at least 1 / (2 b 2^e) from it, 2^-16
// of itself; and where it is a tie it is a float, to which the correction comes exactly.
// (Outside [2^-100, 2^100] products may leave the range of floats: true division.)
struct Coder {
  float top, inv;
  bool fast;
  __device__ __forceinline__ explicit Coder(float t)
      : top(t), inv(__builtin_amdgcn_rcpf(t)), fast(t > 7.9e-31f && t < 1.2e30f) {}
  template <bool FAST>
  __device__ __forceinline__ int code(float x) const {
    const float y = x * 127.f;
    float q;
    if (FAST) {
      q = y * inv;
      q = __builtin_fmaf(__builtin_fmaf(-q, top, y), inv, q);
    } else {
      q = top > 0.f ? y / top : 0.f;
    }
    return (int)rintf(q);
  }
  template <bool FAST>
  __device__ __forceinline__ i32x4 codes16(u32x4 lo, u32x4 hi) const {
    i32x4 out;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t packed = 0;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t x = w < 2 ? lo[2 * w + j] : hi[2 * (w - 2) + j];
        packed |= (uint32_t)(code<FAST>(bf16_float(x & 0xffffu)) & 0xff) << (16 * j) |
                  (uint32_t)(code<FAST>(__uint_as_float(x & 0xffff0000u)) & 0xff) << (16 * j + 8);
      }
      out[w] = (int)packed;
    }
    return out;
  }
  // 16 channels
  __device__ __forceinline__ i32x4 codes(u32x4 lo, u32x4 hi) const {
    return fast ? codes16<true>(lo, hi) : codes16<false>(lo, hi);
  }
};

__device__ __forceinline__ float abs_max8(u32x4 w) {
  float m = 0.f;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    m = fmaxf(m, fmaxf(fabsf(bf16_float(w[q] & 0xffffu)), fabsf(__uint_as_float(w[q] & 0xffff0000u))));
  return m;
}

// The largest of a lane's 16 products and m.
__device__ __forceinline__ int max16(const i32x16& c, int m) {
#pragma unroll
  for (int i = 0; i < 16; i += 2) m = max(m, max(c[i], c[i + 1]));
  return m;
}

constexpr int kSelThreads = 256;
using BlockTopK = TopK<kSelThreads, kMaxCandBlocks>;

// ------------------------------------------------ prefill: a list per query block
//
// One workgroup per (sequence, kv head, query block), the late blocks first, which
// have the most candidates.  The block's rows (block_q rows of G heads) pass
// through LDS as codes, kRowTiles tiles of 32 at a time, and from there into
// registers: each wave holds all of them and takes every fourth tile of 32
// blocks, so a block's codes are read once per workgroup and pass.  Scores stay in
// LDS.  Bound by the matrix unit where rows are many (256 rows: 32 MFMAs per 4 KB of
// codes).
template <int D>
struct SelTiles {
  static constexpr int kRowTiles = 1024 / D;       // row tiles per pass (128 registers)
  static constexpr int kRowBytes = D + 16;         // LDS row of codes, padded against conflicts
  static constexpr int kCodeBytes = kRowTiles * 32 * kRowBytes;
};

template <int D>
__global__ __launch_bounds__(kSelThreads, 2) void select_blocks_kernel(SelectArgs a) {
  using ST = SelTiles<D>;
  extern __shared__ __attribute__((aligned(16))) uint8_t sel_smem[];
  BlockTopK& topk = *(BlockTopK*)sel_smem;
  uint8_t* const rows_lds = sel_smem + (sizeof(BlockTopK) + 15) / 16 * 16;
  int* const best = (int*)(rows_lds + ST::kCodeBytes);
  __shared__ float red[kSelThreads / 64];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int half = lane >> 5, col = lane & 31;
  const int G = a.Hq / a.Hkv;
  int64_t x = blockIdx.x;
  const int g = (int)(x % a.Hkv);
  x /= a.Hkv;
  const int b = (int)(x % a.B);
  const int qb = a.nqb - 1 - (int)(x / a.B);
  const int64_t base = a.cu ? a.cu[b] : (int64_t)b * a.N;
  const int L = min(a.cu ? a.cu[b + 1] - a.cu[b] : a.N, a.N);
  const int R = a.block_q / kPage;
  const int n_qb = max(0, (L + a.block_q - 1) / a.block_q);

  // list sizes are known ahead: min(top_k, qb * R) each
  auto before = [&](int qb_) -> int64_t {  // entries of the lists before qb_
    const int64_t m = min((int64_t)qb_, (int64_t)a.top_k / R + 1);  // lists with j * R <= top_k
    return m * (m - 1) / 2 * R + (qb_ - m) * a.top_k;
  };
  const int64_t list0 = ((int64_t)b * a.Hkv + g) * a.total;
  int32_t* const ptr = a.block_ptr + ((int64_t)b * a.Hkv + g) * (a.nqb + 1);
  if (tid == 0) {
    ptr[qb] = (int32_t)(list0 + before(min(qb, n_qb)));
    if (qb == a.nqb - 1) ptr[a.nqb] = (int32_t)(list0 + before(n_qb));
  }
  const int n = qb * R;  // candidates
  int32_t* const list = a.block_idx + list0 + before(qb);
  if (qb >= n_qb) {  // no rows: the room of its list stays empty
    for (int i = tid; i < min(n, a.top_k); i += kSelThreads) list[i] = -1;
    return;
  }
  if (n == 0) return;
  if (n <= a.top_k) {
    for (int i = tid; i < n; i += kSelThreads) list[i] = i;
    return;
  }

  const int r0 = qb * a.block_q, n_tok = min(a.block_q, L - r0);
  const int n_rows = n_tok * G;  // row r: token r / G, head g * G + r % G (contiguous in q)
  const uint16_t* const q0 = a.q + ((base + r0) * a.Hq + (int64_t)g * G) * D;
  auto row_at = [&](int r) { return q0 + ((int64_t)(r / G) * a.Hq + r % G) * D; };
  // The first pass's rows stay in registers from the maximum to their codes.  (Rows past
  // the last repeat it, which changes no maximum.)
  constexpr int kItems = ST::kRowTiles * 32 * (D / 16) / kSelThreads;  // 16 channels each
  u32x4 held[kItems][2];
  float top = 0.f;
#pragma unroll
  for (int u = 0; u < kItems; ++u) {
    const int c = u * kSelThreads + tid;
    const u32x4* p = (const u32x4*)(row_at(min(c / (D / 16), n_rows - 1)) + c % (D / 16) * 16);
    held[u][0] = p[0];
    held[u][1] = p[1];
  }
#pragma unroll
  for (int u = 0; u < kItems; ++u) top = fmaxf(top, fmaxf(abs_max8(held[u][0]), abs_max8(held[u][1])));
  for (int c = ST::kRowTiles * 32 * (D / 8) + tid; c < n_rows * (D / 8); c += kSelThreads)
    top = fmaxf(top, abs_max8(*(const u32x4*)(row_at(c / (D / 8)) + c % (D / 8) * 8)));
  top = wave_fmax(top);
  if (lane == 0) red[wave] = top;
  __syncthreads();
  const Coder coder(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));

  const int64_t blk0 = base / kPage + b;
  for (int p0 = 0; p0 < n_rows; p0 += ST::kRowTiles * 32) {
    const int rows = min(n_rows - p0, ST::kRowTiles * 32);
    const int tiles = (rows + 31) / 32;
    if (p0) __syncthreads();
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int c = u * kSelThreads + tid, r = c / (D / 16), w = c % (D / 16);
      if (p0) {
        const u32x4* p = (const u32x4*)(row_at(p0 + min(r, rows - 1)) + w * 16);
        held[u][0] = p[0];
        held[u][1] = p[1];
      }
      if (r < tiles * 32) *(i32x4*)(rows_lds + r * ST::kRowBytes + w * 16) = coder.codes(held[u][0], held[u][1]);
    }
    __syncthreads();
    i32x4 qf[ST::kRowTiles][D / 32];
#pragma unroll
    for (int t = 0; t < ST::kRowTiles; ++t)
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk)
        qf[t][kk] = *(const i32x4*)(rows_lds + (min(t, tiles - 1) * 32 + col) * ST::kRowBytes + kk * 32 + half * 16);
    for (int t0 = wave * 32; t0 < n; t0 += kSelThreads / 64 * 32) {
      const int j = min(t0 + col, n - 1);
      const int8_t* cp = a.codes + ((blk0 + j) * a.Hkv + g) * D + half * 16;
      i32x4 kf[D / 32];
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) kf[kk] = *(const i32x4*)(cp + kk * 32);
      int m = INT32_MIN;
#pragma unroll
      for (int t = 0; t < ST::kRowTiles; ++t) {
        if (t < tiles) {
          i32x16 acc = i32x16{};
#pragma unroll
          for (int kk = 0; kk < D / 32; ++kk) acc = mfma_i8(qf[t][kk], kf[kk], acc);
          m = max16(acc, m);
        }
      }
      m = max(m, __shfl_xor(m, 32));
      if (half == 0 && t0 + col < n) best[t0 + col] = p0 ? max(best[t0 + col], m) : m;
    }
  }
  __syncthreads();
  uint32_t* const keys = (uint32_t*)best;
  for (int i = tid; i < n; i += kSelThreads) {
    const float score = (float)best[i] * a.scales[(blk0 + i) * a.Hkv + g];
    keys[i] = i < a.n_sink || i >= n - a.n_recent ? kForced : order_bits(score);
  }
  __syncthreads();
  select_top(
      topk, n, a.top_k,
      [&](auto f) {
        for (int s = 0; s * kSelThreads < n; ++s) {
          const int i = s * kSelThreads + tid;
          f(s, i, i < n ? keys[i] : kAbsent);
        }
      },
      [&](int rank, int i) { list[rank] = i; });
}

// ------------------------------------------------- decode: a list per query token
//
// Candidates are the whole pages before the token's own.  Scores first, a workgroup
// of four waves per (token, kv head, kScoreTiles tiles of 32 pages), then a
// workgroup per (token, kv head) picks.  Bound by HBM in the first (one byte per key
// channel and 64 keys), by latency in the second.
constexpr int kScoreTiles = 16;

struct Token {
  int b, s, pos;
  int64_t t;  // row of q
};
__device__ __forceinline__ bool token_of(const SelectArgs& a, int64_t item, Token* x) {
  x->b = (int)(item / a.N);
  const int i = (int)(item % a.N);
  const int64_t base = a.cu ? a.cu[x->b] : (int64_t)x->b * a.N;
  const int m = min(a.cu ? a.cu[x->b + 1] - a.cu[x->b] : a.N, a.N);
  if (i >= m) return false;
  x->s = a.slots ? a.slots[x->b] : x->b;
  x->t = base + i;
  x->pos = (unsigned)x->s < (unsigned)a.S ? min(a.lens[x->s], a.M * kPage) - m + i : -1;
  return true;
}

// The codes of the token's rows are made once per workgroup, through LDS, while the
// first pages' codes are on their way.
template <int D>
__global__ __launch_bounds__(kSelThreads) void score_pages_kernel(SelectArgs a) {
  constexpr int kPer = kScoreTiles / (kSelThreads / 64);  // tiles of a wave
  __shared__ __attribute__((aligned(16))) uint8_t rows_lds[32 * SelTiles<D>::kRowBytes];
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31, wave = tid >> 6;
  const int G = a.Hq / a.Hkv;
  const int64_t item = blockIdx.x / (unsigned)a.Hkv;
  const int g = blockIdx.x % (unsigned)a.Hkv;
  Token tk;
  if (!token_of(a, item, &tk)) return;
  const int n = min(max(tk.pos, 0) / kPage, a.max_blocks);
  const int t0 = blockIdx.y * (kScoreTiles * 32);
  if (t0 >= n || n <= a.top_k) return;  // (all are chosen without scores)
  const uint16_t* const q0 = a.q + (tk.t * a.Hq + (int64_t)g * G) * D;
  const int32_t* const row = a.table + (int64_t)tk.s * a.M;
  uint32_t* const keys = a.keys + ((int64_t)item * a.Hkv + g) * a.max_blocks;
  int page[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) page[i] = row[min(t0 + (i * (kSelThreads / 64) + wave) * 32 + col, n - 1)];
  float top = 0.f;
  for (int c = lane; c < G * (D / 8); c += 64) top = fmaxf(top, abs_max8(*(const u32x4*)(q0 + c * 8)));
  float scale[kPer];
  i32x4 kf[kPer][D / 32];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int64_t e = (unsigned)page[i] < (unsigned)a.P ? page[i] : 0;
    const int8_t* cp = a.codes + (e * a.Hkv + g) * D + half * 16;
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) kf[i][kk] = *(const i32x4*)(cp + kk * 32);
    scale[i] = a.scales[e * a.Hkv + g];
  }
  const Coder coder(wave_fmax(top));
  int m[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) m[i] = INT32_MIN;
  for (int u = 0; u < G; u += 32) {  // (more than one turn for more than 32 heads only)
    if (u) __syncthreads();
    // (rows past the last repeat it, which changes no maximum)
    for (int c = tid; c < 32 * (D / 16); c += kSelThreads) {
      const u32x4* p = (const u32x4*)(q0 + min(u + c / (D / 16), G - 1) * D + c % (D / 16) * 16);
      *(i32x4*)(rows_lds + c / (D / 16) * SelTiles<D>::kRowBytes + c % (D / 16) * 16) = coder.codes(p[0], p[1]);
    }
    __syncthreads();
    i32x4 qf[D / 32];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk)
      qf[kk] = *(const i32x4*)(rows_lds + col * SelTiles<D>::kRowBytes + kk * 32 + half * 16);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      i32x16 acc = i32x16{};
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) acc = mfma_i8(qf[kk], kf[i][kk], acc);
      m[i] = max16(acc, m[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    m[i] = max(m[i], __shfl_xor(m[i], 32));
    const int j = t0 + (i * (kSelThreads / 64) + wave) * 32 + col;
    if (half == 0 && j < n) {
      // (a page that the table does not name comes last: nothing of it is attended to)
      const uint32_t key = (unsigned)page[i] < (unsigned)a.P ? order_bits((float)m[i] * scale[i]) : kAbsent;
      keys[j] = j < a.n_sink || j >= n - a.n_recent ? kForced : key;
    }
  }
}

// Workgroups of 256 threads take up to 4096 candidates, whose keys they hold in
// registers, 1024 up to 16384 likewise, and more from memory: barriers of four waves
// cost less than those of sixteen.
constexpr int kPickHeld = 16;  // keys per thread held in registers
template <int NT, bool HELD>
__global__ __launch_bounds__(NT) void pick_pages_kernel(SelectArgs a) {
  __shared__ TopK<NT, HELD ? NT * kPickHeld : kMaxCandPages> topk;
  const int tid = threadIdx.x;
  const int64_t item = blockIdx.x / (unsigned)a.Hkv;
  const int g = blockIdx.x % (unsigned)a.Hkv;
  Token tk;
  if (!token_of(a, item, &tk)) return;
  const int n = min(max(tk.pos, 0) / kPage, a.max_blocks);
  int32_t* const list = a.pages + (tk.t * a.Hkv + g) * a.top_k;
  for (int i = min(n, a.top_k) + tid; i < a.top_k; i += NT) list[i] = -1;
  const uint32_t* const keys = a.keys + ((int64_t)item * a.Hkv + g) * a.max_blocks;
  auto emit = [&](int rank, int i) { list[rank] = i; };
  if constexpr (HELD) {
    uint32_t x[kPickHeld];
    if (n > a.top_k) {
#pragma unroll
      for (int s = 0; s < kPickHeld; ++s) x[s] = s * NT + tid < n ? keys[s * NT + tid] : kAbsent;
    }
    select_top(
        topk, n, a.top_k,
        [&](auto f) {
#pragma unroll
          for (int s = 0; s < kPickHeld; ++s)
            if (s * NT < n) f(s, s * NT + tid, x[s]);
        },
        emit);
  } else {
    select_top(
        topk, n, a.top_k,
        [&](auto f) {
          for (int s = 0; s * NT < n; ++s) {
            const int i = s * NT + tid;
            f(s, i, i < n ? keys[i] : kAbsent);
          }
        },
        emit);
  }
}

}  // namespace

hipError_t launch_summary(const SummaryArgs& a, hipStream_t s) {
  const int64_t items = (int64_t)a.B * a.nblk * a.Hkv;
  const dim3 grid((unsigned)((items + 3) / 4));
  if (a.d == 128)
    hipLaunchKernelGGL(summary_kernel<128>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(summary_kernel<64>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_select_blocks(const SelectArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.nqb * a.B * a.Hkv));
  const size_t head = (sizeof(BlockTopK) + 15) / 16 * 16;
  if (a.d == 128)
    hipLaunchKernelGGL(select_blocks_kernel<128>, grid, dim3(kSelThreads),
                       head + SelTiles<128>::kCodeBytes + (size_t)a.max_blocks * 4, s, a);
  else
    hipLaunchKernelGGL(select_blocks_kernel<64>, grid, dim3(kSelThreads),
                       head + SelTiles<64>::kCodeBytes + (size_t)a.max_blocks * 4, s, a);
  return hipGetLastError();
}

hipError_t launch_select_pages(const SelectArgs& a, hipStream_t s) {
  const int64_t items = (int64_t)a.B * a.N * a.Hkv;
  if (a.max_blocks > a.top_k) {
    const dim3 grid((unsigned)items, (unsigned)((a.max_blocks + kScoreTiles * 32 - 1) / (kScoreTiles * 32)));
    if (a.d == 128)
      hipLaunchKernelGGL(score_pages_kernel<128>, grid, dim3(kSelThreads), 0, s, a);
    else
      hipLaunchKernelGGL(score_pages_kernel<64>, grid, dim3(kSelThreads), 0, s, a);
  }
  const dim3 grid((unsigned)items);
  if (a.max_blocks <= 256 * kPickHeld)
    hipLaunchKernelGGL((pick_pages_kernel<256, true>), grid, dim3(256), 0, s, a);
  else if (a.max_blocks <= 1024 * kPickHeld)
    hipLaunchKernelGGL((pick_pages_kernel<1024, true>), grid, dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL((pick_pages_kernel<1024, false>), grid, dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace da
