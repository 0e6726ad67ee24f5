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
// Every key is read once, 1/64 of that written: 16384 tokens of 8 kv heads, d 128 (34 MB) in
// 8.1 us, 87302 (179 MB) in 50 us, 3.6 TB/s, right after the pages were written; with sums
// in 32 bits the same: not the arithmetic bounds it, but that a wave ends with its block and
// reads nothing while it reduces.
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
// one value or just as many keys as are chosen.  The first round's steps are of the
// scores themselves; where its step holds 64 keys or fewer, as a rule, one wave ranks
// those and there is no second round (8000 keys: 19.0 us against 20.3, scores included).
// Then one pass ranks the chosen ones in ascending order: stripes of NT keys, each wave's
// counts in a table, a prefix sum over (stripe, wave).  Thread tid owns keys tid,
// tid + NT, ...; each(f) calls
// f(stripe, index, key) for those of all stripes, index >= n where there is none.
// emit(rank, index) is called once per chosen key.
constexpr uint32_t kForced = 0xffffffffu;  // always chosen (never more than top_k are)
constexpr uint32_t kAbsent = 0u;           // chosen last

// A score as a whole number that orders as it does (+0 and -0 alike).
__device__ __forceinline__ uint32_t order_bits(float x) {
  const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_float(uint32_t x) {
  return __uint_as_float(x & 0x80000000u ? x ^ 0x80000000u : ~x);
}

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
  int need, all, held;       // of the step that was found, and how many keys it holds
  uint32_t list[2][64], cut[2];  // its keys and their places; the last chosen one
  int listed;
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
  // members: keys in [lo, hi]; `need` of them are chosen, and every key above.  The first
  // round's steps are equal ones of the scores themselves, where their range allows
  // (`lin`), later ones of the keys, whose spacing is by octaves.
  uint32_t lo = 1, hi = kForced - 1;
  float f0 = 0.f, per_step = 0.f;
  bool lin = false;
  auto lin_step = [&](uint32_t x) { return (uint32_t)((order_float(x) - f0) * per_step); };
  int need = top_k;
  uint32_t bin = 0;
  bool all = false, cut = false;  // cut: t.cut is the last chosen key
  for (int round = 0;; ++round) {
    uint32_t mn = ~0u, mx = 0;
    int forced = 0, members = 0;
    each([&](int, int i, uint32_t x) {
      if (i >= n) return;
      const bool in = x >= lo && x <= hi && (!lin || lin_step(x) == bin);
      mn = in ? min(mn, x) : mn;
      mx = in ? max(mx, x) : mx;
      members += in;
      forced += x == kForced;
    });
    mn = (uint32_t)wave_reduce((int)mn, -1, [](int x, int y) { return (int)min((uint32_t)x, (uint32_t)y); });
    mx = (uint32_t)wave_reduce((int)mx, 0, [](int x, int y) { return (int)max((uint32_t)x, (uint32_t)y); });
    if (round == 0) {
      members = wave_add(members);
      forced = wave_add(forced);
    }
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
    if (round == 0) {
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
    lo = mn;
    hi = mx;
    if (all) {  // every key of the last round's step is chosen
      --lo;
      need = 0;
      break;
    }
    int sh = 0;
    if (round == 0) {
      f0 = order_float(mn);
      const float range = order_float(mx) - f0;  // (steps 0 .. kBins - 1: the product may round up)
      lin = range > 1e-30f && range < 1e30f;
      per_step = lin ? (float)(TK::kBins - 1) * 0.9999f / range : 0.f;
    } else {
      lin = false;
    }
    if (!lin) sh = max(0, 32 - __clz((int)(mx - mn)) - (31 - __clz(TK::kBins)));  // (0 for a single value)
    each([&](int, int i, uint32_t x) {
      if (i < n && x >= lo && x <= hi) atomicAdd(&t.hist[lin ? lin_step(x) : (x - mn) >> sh], 1);
    });
    __syncthreads();
    // thread tid holds kPer steps, the highest of all threads' first
    int c[TK::kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < TK::kPer; ++j) sum += c[j] = t.hist[TK::kBins - 1 - TK::kPer * tid - j];
    int upto = wave_scan_add(sum);
    if (lane == 63) t.scan[2][wave] = upto;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) upto += w < wave ? t.scan[2][w] : 0;
    int before = upto - sum;
    if (before < need && upto >= need) {
#pragma unroll
      for (int j = 0; j < TK::kPer; ++j) {
        if (before < need && before + c[j] >= need) {
          t.bin = TK::kBins - 1 - TK::kPer * tid - j;
          t.need = need - before;
          t.all = before + c[j] == need;
          t.held = c[j];
          t.listed = 0;
        }
        before += c[j];
      }
    }
    __syncthreads();
    need = t.need;
    bin = t.bin;
    all = t.all;
    if (lin && t.held <= 64) {
      // One wave ranks the step's keys: the need-th of them is the last one chosen.
      each([&](int, int i, uint32_t x) {
        if (i < n && x >= lo && x <= hi && lin_step(x) == bin) {
          const int at = atomicAdd(&t.listed, 1);
          t.list[0][at] = x;
          t.list[1][at] = i;
        }
      });
      __syncthreads();
      if (wave == 0) {
        const int m = t.held;
        const uint32_t key = lane < m ? t.list[0][lane] : 0u, at = lane < m ? t.list[1][lane] : ~0u;
        int rank = 0;
        for (int j = 0; j < m; ++j) {
          const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)key, j), i = (uint32_t)__builtin_amdgcn_readlane((int)at, j);
          rank += k > key || (k == key && i < at);
        }
        if (lane < m && rank == need - 1) {
          t.cut[0] = key;
          t.cut[1] = at;
        }
      }
      __syncthreads();
      cut = true;
      break;
    }
    if (lin) continue;  // the step's keys: those whose score falls into it
    lo = mn + (bin << sh);
    if (all) {
      --lo;
      need = 0;
      break;
    }
    if (sh == 0) break;
    hi = lo + min(mx - lo, (1u << sh) - 1u);
  }
  // Keys above lo are chosen, and the first `need` equal to it (with `cut`, those up to
  // place cut_at), in ascending order of their places.
  uint32_t cut_at = 0;
  if (cut) {
    lo = t.cut[0];
    cut_at = t.cut[1];
    need = 0;
  }
  auto is_above = [&](int i, uint32_t x) { return i < n && (x > lo || (cut && x == lo && (uint32_t)i <= cut_at)); };
  auto is_same = [&](int i, uint32_t x) { return !cut && i < n && x == lo; };
  each([&](int s, int i, uint32_t x) {
    const uint64_t above = __ballot(is_above(i, x)), same = __ballot(is_same(i, x));
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
#pragma unroll
    for (int w = 0; w < W; ++w) before[q] += w < wave ? t.scan[q][w] : 0;
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
  const uint64_t lower = (1ull << lane) - 1;
  each([&](int s, int i, uint32_t x) {
    const bool above = is_above(i, x), same = is_same(i, x);
    const uint64_t ups = __ballot(above), sames = __ballot(same);
    if (!(ups | sames)) return;
    const int na = t.table[0][s * W + wave] + __popcll(ups & lower);
    const int ns = t.table[1][s * W + wave] + __popcll(sames & lower);
    if (above || (same && ns < need)) emit(na + min(ns, need), i);
  });
}

// The same by one wavefront for at most 64 RK keys, which it holds in registers (key s *
// 64 + lane in x[s], kAbsent past the last): the smallest chosen key bit by bit below those
// that all keys share, counting the keys that are as large by ballots, without LDS or
// barriers.  Ends early where just top_k keys are as large.  (A histogram in LDS, or
// guesses by interpolation, take a single wave longer: 780 keys 17.2 and 21.5 us against
// 13.6, scores included.)
template <int RK, typename Emit>
__device__ __forceinline__ void select_wave(const uint32_t (&x)[RK], int n, int top_k, Emit emit) {
  const int lane = threadIdx.x & 63;
  auto count = [&](auto holds) {
    int c = 0;
#pragma unroll
    for (int s = 0; s < RK; ++s) c += __popcll(__ballot(holds(s)));  // (never true of absent keys below)
    return c;
  };
  uint32_t least = 0;
  int above = 0;  // keys above it that are chosen
  bool exact = n <= top_k;
  int bit = 31;
  if (!exact) {
    uint32_t mn = kForced, mx = kAbsent;  // of the keys that are neither forced nor absent
#pragma unroll
    for (int s = 0; s < RK; ++s) {
      const bool in = x[s] != kForced && x[s] != kAbsent;
      mn = in ? min(mn, x[s]) : mn;
      mx = in ? max(mx, x[s]) : mx;
    }
    mn = (uint32_t)wave_reduce((int)mn, -1, [](int p, int q) { return (int)min((uint32_t)p, (uint32_t)q); });
    mx = (uint32_t)wave_reduce((int)mx, 0, [](int p, int q) { return (int)max((uint32_t)p, (uint32_t)q); });
    // the bits that all of them share are the key's, unless it is a forced or an absent one
    if (count([&](int s) { return x[s] > mx; }) < top_k && count([&](int s) { return x[s] >= mn; }) >= top_k) {
      bit = 31 - __clz((int)(mn ^ mx));  // (-1 for a single value)
      least = bit < 0 ? mn : bit == 31 ? 0u : mn & ~((2u << bit) - 1u);
    }
  }
  for (; bit >= 0 && !exact; --bit) {
    const uint32_t t = least | 1u << bit;
    const int c = count([&](int s) { return x[s] >= t; });
    if (c >= top_k) least = t;
    exact = c == top_k;
  }
  if (!exact) above = count([&](int s) { return x[s] > least; });
  const int need = exact ? 0 : top_k - above;  // of those equal to it, the first
  int before = 0, same_before = 0;
  const uint64_t lower = (1ull << lane) - 1;
#pragma unroll
  for (int s = 0; s < RK; ++s) {
    const bool in = s * 64 + lane < n;
    const bool up = in && (exact ? x[s] >= least : x[s] > least), same = in && !exact && x[s] == least;
    const uint64_t ups = __ballot(up), sames = __ballot(same);
    const int ns = same_before + __popcll(sames & lower);
    if (up || (same && ns < need)) emit(before + __popcll(ups & lower) + min(ns, need), s * 64 + lane);
    before += __popcll(ups);
    same_before += __popcll(sames);
  }
}

// One wavefront alone takes up to 64 keys times this, with as few registers of them as n
// needs; key(i) is that of place i < n.
constexpr int kWaveKeys = 16;
template <typename Key, typename Emit>
__device__ __forceinline__ void select_few(int n, int top_k, Key key, Emit emit) {
  const int lane = threadIdx.x & 63;
  auto run = [&](auto keys) {
    constexpr int RK = decltype(keys)::value;
    uint32_t x[RK];
#pragma unroll
    for (int s = 0; s < RK; ++s) x[s] = s * 64 + lane < n ? key(s * 64 + lane) : kAbsent;
    select_wave(x, n, top_k, emit);
  };
  if (n <= 128)
    run(std::integral_constant<int, 2>{});
  else if (n <= 256)
    run(std::integral_constant<int, 4>{});
  else if (n <= 512)
    run(std::integral_constant<int, 8>{});
  else
    run(std::integral_constant<int, kWaveKeys>{});
}

// Codes round(127 x / top) of a group's queries, top its largest magnitude, ties to even.
// With bf16 significands a and b of x and top, 128 to 255, the quotient is 127 a / (b 2^e).
//  - It is a tie n + 1/2 where 254 a = (2n + 1) b 2^e.  127 is prime, so either 2n + 1 =
//    127 and a = b, x = +-top / 2, whose code is +-64, or 127 divides b, which is 254.
//  - Else it lies at least 1 / (2 b 2^e) from a tie, 2^-16 of itself.
// So unless b is 254, round(k x) with k above 127 / top by a 2^-19th of it is the code: too
// little to cross a tie, enough to round 63.5 to 64.  That takes one fma, onto 1.5 * 2^23, where
// floats are whole numbers: the low byte of the sum is the code.
//  - With b = 254, or top outside [2^-100, 2^100], where k or k x may not be normal: true
//    division.
struct Coder {
  float top, k;
  bool fast;
  __device__ __forceinline__ explicit Coder(float t)
      : top(t),
        k(127.f * __builtin_amdgcn_rcpf(t) * (1.f + 0x1p-19f)),
        fast(t > 0x1p-100f && t < 0x1p100f && (__float_as_uint(t) & 0x7f0000u) != 0x7e0000u) {}
  template <bool FAST>
  __device__ __forceinline__ uint32_t code(uint32_t bits) const {  // (the low byte)
    const float x = __uint_as_float(bits);
    if (FAST) return __float_as_uint(__builtin_fmaf(x, k, 12582912.f));
    // (scaled by a power of two, so that 127 x neither overflows nor loses bits)
    const float s = top > 1.f ? 0x1p-64f : 0x1p64f;
    return (uint32_t)(int)rintf(top > 0.f ? x * s * 127.f / (top * s) : 0.f);
  }
  template <bool FAST>
  __device__ __forceinline__ uint2 codes8(u32x4 x) const {
    uint32_t out[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      uint32_t pair[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        pair[j] = __builtin_amdgcn_perm(code<FAST>(x[2 * w + j] & 0xffff0000u), code<FAST>(x[2 * w + j] << 16), 0x0c0c0400u);
      out[w] = __builtin_amdgcn_perm(pair[1], pair[0], 0x05040100u);
    }
    return uint2{out[0], out[1]};
  }
  // 8 channels
  __device__ __forceinline__ uint2 codes(u32x4 x) const { return fast ? codes8<true>(x) : codes8<false>(x); }
};

// The larger magnitudes of two times two bf16 values (whose bits, without the sign, order as
// they do), and the largest of a wavefront's.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 max_bits(u16x2 m, u32x4 w) {
#pragma unroll
  for (int q = 0; q < 4; ++q) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[q] & 0x7fff7fffu));
  return m;
}
__device__ __forceinline__ float wave_top(u16x2 m) {
  return __uint_as_float((uint32_t)wave_reduce(max((int)m[0], (int)m[1]), 0, [](int x, int y) { return max(x, y); }) << 16);
}

// The largest of a lane's 16 products and m.
__device__ __forceinline__ int max16(const i32x16& c, int m) {
#pragma unroll
  for (int i = 0; i < 16; i += 2) m = max(m, max(c[i], c[i + 1]));
  return m;
}

constexpr int kSelThreads = 256;
using BlockTopK = TopK<kSelThreads, kMaxCandBlocks>;
constexpr int kScoreThreads = 256;

// ------------------------------------------------ prefill: a list per query block
//
// One workgroup per (sequence, kv head, query block), the late blocks first, which
// have the most candidates.  Each of its four waves holds kTiles tiles of 32 of the
// block's rows (block_q rows of G heads) as codes in registers and takes every tile of 32
// blocks; the waves' maxima meet in LDS.  Rows are loaded whole, neighbouring lanes
// neighbouring chunks, and their codes pass through the wave's part of LDS into the
// operand's layout.  (Loaded straight into that layout, each instruction took 16 bytes
// of each of 64 lines, which the L1 cache did not keep for the next one: 52 us with
// 16384 tokens, 32 heads on 8, against 45 to 49.)  More rows take further passes.  Bound by the
// queries, which are read once, and by the selection; of the products there are 8 MFMAs per
// wave and 32 blocks.
template <int D>
struct SelTiles {
  static constexpr int kTiles = 256 / D;     // row tiles of a wave (32 registers of codes)
  static constexpr int kRows = kTiles * 32;  // rows of a wave per pass
  static constexpr int kRowBytes = D + 16;   // of codes in LDS, padded against bank conflicts
  static constexpr int kBytes = kSelThreads / 64 * kRows * kRowBytes;
};

template <int D>
__global__ __launch_bounds__(kSelThreads, 3) void select_blocks_kernel(SelectArgs a) {
  using ST = SelTiles<D>;
  constexpr int kWaves = kSelThreads / 64;
  extern __shared__ __attribute__((aligned(16))) uint8_t sel_smem[];
  BlockTopK& topk = *(BlockTopK*)sel_smem;
  uint8_t* const rows_lds = sel_smem + (sizeof(BlockTopK) + 15) / 16 * 16;
  int* const best = (int*)(rows_lds + ST::kBytes);
  __shared__ float red[kWaves];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int half = lane >> 5, col = lane & 31;
  const int G = a.G;
  const uint32_t x = blockIdx.x / (uint32_t)a.Hkv;
  const int g = (int)(blockIdx.x - x * (uint32_t)a.Hkv);
  const int b = (int)(x % (uint32_t)a.B);
  const int qb = a.nqb - 1 - (int)(x / (uint32_t)a.B);
  const int64_t base = a.cu ? a.cu[b] : (int64_t)b * a.N;
  const int L = min(a.cu ? a.cu[b + 1] - a.cu[b] : a.N, a.N);
  const int R = a.block_q / kPage;
  const int n_qb = max(0, (L + a.block_q - 1) / a.block_q);

  // list sizes are known ahead
  auto before = [&](int j) { return list_entries_before(j, a.top_k, R); };
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
  // (byte offsets inside a query block fit 32 bits)
  auto row_at = [&](int r) {
    const uint32_t i = fdiv((uint32_t)r, a.fd_G);
    return (const uint16_t*)((const char*)q0 + (i * (uint32_t)a.Hq + ((uint32_t)r - i * (uint32_t)G)) * (uint32_t)(2 * D));
  };
  // (Rows past the last repeat it, which changes no maximum.)
  constexpr int kLanes = D / 8, kLoads = ST::kRows * kLanes / 64;
  u32x4 held[kLoads];
  auto load_row = [&](int p0, int u) {
    const int r = p0 + wave * ST::kRows + u * (64 / kLanes) + lane / kLanes;
    return *(const u32x4*)(row_at(min(r, n_rows - 1)) + lane % kLanes * 8);
  };
  auto load_rows = [&](int p0) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) held[u] = load_row(p0, u);
  };
  load_rows(0);
  const int64_t blk0 = base / kPage + b;
  const int8_t* const codes = a.codes + (blk0 * a.Hkv + g) * D + half * 16;
  const int64_t stride = (int64_t)a.Hkv * D;
  auto load_block = [&](i32x4* kf, int t0) {
    const i32x4* p = (const i32x4*)(codes + min(t0 + col, n - 1) * stride);
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) kf[kk] = p[2 * kk];
  };
  for (int i = tid; i < n; i += kSelThreads) best[i] = INT32_MIN;
  u16x2 most = {0, 0};
#pragma unroll
  for (int u = 0; u < kLoads; ++u) most = max_bits(most, held[u]);
  for (int c = kWaves * ST::kRows * (D / 8) + tid; c < n_rows * (D / 8); c += kSelThreads)
    most = max_bits(most, *(const u32x4*)(row_at(c / (D / 8)) + c % (D / 8) * 8));
  float top = wave_top(most);
  if (lane == 0) red[wave] = top;
  __syncthreads();
  top = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, red[w]);
  const Coder coder(top);

  for (int p0 = 0; p0 < n_rows; p0 += kWaves * ST::kRows) {
    if (p0) load_rows(p0);
    if (p0 + wave * ST::kRows >= n_rows) break;  // (uniform over the wave; no barrier in the loop)
    uint8_t* const mine = rows_lds + wave * (ST::kRows * ST::kRowBytes);
    wave_lds_exchange();  // (the pass before has read its rows)
    auto place = [&](int u) {
      return (uint2*)(mine + (u * (64 / kLanes) + lane / kLanes) * ST::kRowBytes + lane % kLanes * 8);
    };
    if (coder.fast) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) *place(u) = coder.codes8<true>(held[u]);
    } else {  // (rare: rolled up, from memory again, so that it takes no registers of the other)
#pragma unroll 1
      for (int u = 0; u < kLoads; ++u) *place(u) = coder.codes8<false>(load_row(p0, u));
    }
    i32x4 kf[D / 32], next[D / 32];
    load_block(next, 0);
    wave_lds_exchange();
    i32x4 qf[ST::kTiles][D / 32];
#pragma unroll
    for (int t = 0; t < ST::kTiles; ++t)
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk)
        qf[t][kk] = *(const i32x4*)(mine + (t * 32 + col) * ST::kRowBytes + kk * 32 + half * 16);
    for (int t0 = 0; t0 < n; t0 += 32) {
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) kf[kk] = next[kk];
      if (t0 + 32 < n) load_block(next, t0 + 32);
      int m = INT32_MIN;
#pragma unroll
      for (int t = 0; t < ST::kTiles; ++t) {
        i32x16 acc = i32x16{};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) acc = mfma_i8(qf[t][kk], kf[kk], acc);
        m = max16(acc, m);
      }
      m = max(m, __shfl_xor(m, 32));
      if (half == 0 && t0 + col < n) atomicMax(&best[t0 + col], m);
    }
  }
  __syncthreads();
  auto emit = [&](int rank, int i) { list[rank] = i; };
  auto key_of = [&](int i) {
    const float score = (float)best[i] * a.scales[(blk0 + i) * a.Hkv + g];
    return i < a.n_sink || i >= n - a.n_recent ? kForced : order_bits(score);
  };
  if (n <= 64 * kWaveKeys) {
    if (wave) return;
    select_few(n, a.top_k, key_of, emit);
    return;
  }
  uint32_t* const keys = (uint32_t*)best;
  for (int i = tid; i < n; i += kSelThreads) keys[i] = key_of(i);
  __syncthreads();
  select_top(
      topk, n, a.top_k,
      [&](auto f) {
        for (int s = 0; s * kSelThreads < n; ++s) {
          const int i = s * kSelThreads + tid;
          f(s, i, i < n ? keys[i] : kAbsent);
        }
      },
      emit);
}

// ------------------------------------------------- decode: a list per query token
//
// Candidates are the whole pages before the token's own.  Up to kFewCandPages of them a
// workgroup per (token, kv head) scores and picks; with more, scores come first, a
// workgroup of four waves per 512 pages, then a workgroup per (token, kv head) picks.  Bound
// by HBM in the scores (one byte per key channel and 64 keys), by latency otherwise: 16
// tokens over up to 50000 keys, 32 heads on 8, d 128: 14 us (as two launches 16 and the gap
// between, and 3 us more on the host); one over 1048576 keys: 8.4 and 20.4.
struct Token {
  int b, s, pos;
  int64_t t;  // row of q
};
__device__ __forceinline__ bool token_of(const SelectArgs& a, uint32_t item, Token* x) {
  x->b = (int)(item / (uint32_t)a.N);
  const int i = (int)(item - (uint32_t)x->b * (uint32_t)a.N);
  const int64_t base = a.cu ? a.cu[x->b] : (int64_t)x->b * a.N;
  const int m = min(a.cu ? a.cu[x->b + 1] - a.cu[x->b] : a.N, a.N);
  if (i >= m) return false;
  x->s = a.slots ? a.slots[x->b] : x->b;
  x->t = base + i;
  x->pos = (unsigned)x->s < (unsigned)a.S ? min(a.lens[x->s], a.M * kPage) - m + i : -1;
  return true;
}

// Keys of the candidates t0 to t0 + 2 NT - 1 of n, by the NT threads of a workgroup: put(j, key)
// for each.  The codes of the token's rows are made once, through LDS, while the first
// pages' codes are on their way.
constexpr int kTilesPerWave = 4;
template <int D>
constexpr int kCodeRowBytes = D + 16;  // padded against bank conflicts
template <int D, int NT, typename Put>
__device__ __forceinline__ void score_pages(const SelectArgs& a, const Token& tk, int g, int n, int t0,
                                            uint8_t* rows_lds, Put put) {
  constexpr int kPer = kTilesPerWave, kRowBytes = kCodeRowBytes<D>;
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31, wave = tid >> 6;
  const int G = a.Hq / a.Hkv;
  const uint16_t* const q0 = a.q + (tk.t * a.Hq + (int64_t)g * G) * D;
  const int32_t* const row = a.table + (int64_t)tk.s * a.M;
  int page[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) page[i] = row[min(t0 + (i * (NT / 64) + wave) * 32 + col, n - 1)];
  u16x2 most = {0, 0};
  for (int c = lane; c < G * (D / 8); c += 64) most = max_bits(most, *(const u32x4*)(q0 + c * 8));
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
  const Coder coder(wave_top(most));
  int m[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) m[i] = INT32_MIN;
  for (int u = 0; u < G; u += 32) {  // (more than one turn for more than 32 heads only)
    if (u) __syncthreads();
    // (rows past the last repeat it, which changes no maximum)
    for (int c = tid; c < 32 * (D / 8); c += NT)
      *(uint2*)(rows_lds + c / (D / 8) * kRowBytes + c % (D / 8) * 8) =
          coder.codes(*(const u32x4*)(q0 + min(u + c / (D / 8), G - 1) * D + c % (D / 8) * 8));
    __syncthreads();
    i32x4 qf[D / 32];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk)
      qf[kk] = *(const i32x4*)(rows_lds + col * kRowBytes + kk * 32 + half * 16);
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
    const int j = t0 + (i * (NT / 64) + wave) * 32 + col;
    if (half == 0 && j < n) {
      // (a page that the table does not name comes last: nothing of it is attended to)
      const uint32_t key = (unsigned)page[i] < (unsigned)a.P ? order_bits((float)m[i] * scale[i]) : kAbsent;
      put(j, j < a.n_sink || j >= n - a.n_recent ? kForced : key);
    }
  }
}

template <int D>
__global__ __launch_bounds__(kScoreThreads) void score_pages_kernel(SelectArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t rows_lds[32 * kCodeRowBytes<D>];
  const uint32_t item = blockIdx.x / (unsigned)a.Hkv;
  const int g = blockIdx.x % (unsigned)a.Hkv;
  Token tk;
  if (!token_of(a, item, &tk)) return;
  const int n = min(max(tk.pos, 0) / kPage, a.max_blocks);
  const int t0 = blockIdx.y * (kScoreThreads * 2);
  if (t0 >= n || n <= a.top_k) return;  // (all are chosen without scores)
  uint32_t* const keys = a.keys + ((int64_t)item * a.Hkv + g) * a.max_blocks;
  score_pages<D, kScoreThreads>(a, tk, g, n, t0, rows_lds, [&](int j, uint32_t key) { keys[j] = key; });
}

// Up to 1024 candidates: one launch, whose workgroups score them, keys in LDS, and whose first
// waves then pick.
constexpr int kFewThreads = 512;
static_assert(kFewThreads * 2 == kFewCandPages && kFewCandPages == 64 * kWaveKeys, "as many as one wave takes");
template <int D>
__global__ __launch_bounds__(kFewThreads) void few_pages_kernel(SelectArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t rows_lds[32 * kCodeRowBytes<D>];
  __shared__ uint32_t keys[64 * kWaveKeys];
  const int tid = threadIdx.x;
  const uint32_t item = blockIdx.x / (unsigned)a.Hkv;
  const int g = blockIdx.x % (unsigned)a.Hkv;
  Token tk;
  if (!token_of(a, item, &tk)) return;
  const int n = min(max(tk.pos, 0) / kPage, a.max_blocks);
  int32_t* const list = a.pages + (tk.t * a.Hkv + g) * a.top_k;
  for (int i = min(n, a.top_k) + tid; i < a.top_k; i += kFewThreads) list[i] = -1;
  if (n <= a.top_k) {
    for (int i = tid; i < n; i += kFewThreads) list[i] = i;
    return;
  }
  score_pages<D, kFewThreads>(a, tk, g, n, 0, rows_lds, [&](int j, uint32_t key) { keys[j] = key; });
  __syncthreads();
  if (tid >= 64) return;
  select_few(n, a.top_k, [&](int i) { return keys[i]; }, [&](int rank, int i) { list[rank] = i; });
}

// More: workgroups of 256 threads take up to 4096, whose keys they hold in registers, 1024 up
// to 16384 likewise, and more from memory: barriers of four waves cost less than those of
// sixteen.
constexpr int kPickHeld = 16;  // keys per thread held in registers
template <int NT, bool HELD>
__global__ __launch_bounds__(NT) void pick_pages_kernel(SelectArgs a) {
  __shared__ TopK<NT, HELD ? NT * kPickHeld : kMaxCandPages> topk;
  const int tid = threadIdx.x;
  const uint32_t item = blockIdx.x / (unsigned)a.Hkv;
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
                       head + SelTiles<128>::kBytes + (size_t)a.max_blocks * 4, s, a);
  else
    hipLaunchKernelGGL(select_blocks_kernel<64>, grid, dim3(kSelThreads),
                       head + SelTiles<64>::kBytes + (size_t)a.max_blocks * 4, s, a);
  return hipGetLastError();
}

hipError_t launch_select_pages(const SelectArgs& a, hipStream_t s) {
  const dim3 items((unsigned)((int64_t)a.B * a.N * a.Hkv));
  if (a.max_blocks <= kFewCandPages) {
    if (a.d == 128)
      hipLaunchKernelGGL(few_pages_kernel<128>, items, dim3(kFewThreads), 0, s, a);
    else
      hipLaunchKernelGGL(few_pages_kernel<64>, items, dim3(kFewThreads), 0, s, a);
    return hipGetLastError();
  }
  if (a.max_blocks > a.top_k) {
    const dim3 grid(items.x, (unsigned)((a.max_blocks + kScoreThreads * 2 - 1) / (kScoreThreads * 2)));
    if (a.d == 128)
      hipLaunchKernelGGL(score_pages_kernel<128>, grid, dim3(kScoreThreads), 0, s, a);
    else
      hipLaunchKernelGGL(score_pages_kernel<64>, grid, dim3(kScoreThreads), 0, s, a);
  }
  if (a.max_blocks <= 256 * kPickHeld)
    hipLaunchKernelGGL((pick_pages_kernel<256, true>), items, dim3(256), 0, s, a);
  else if (a.max_blocks <= 1024 * kPickHeld)
    hipLaunchKernelGGL((pick_pages_kernel<1024, true>), items, dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL((pick_pages_kernel<1024, false>), items, dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace da
