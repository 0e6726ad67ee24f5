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
// that 512/D keys arrive per load; the lanes of one channel chunk are then added
// up by exchanges.  Bound by HBM: every key is read once, 1/64 of that written.
template <int D>
__global__ __launch_bounds__(256) void summary_kernel(SummaryArgs a) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes, kSteps = kPage / kRows;
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int h = (int)(item % a.Hkv);
  const int64_t x = item / a.Hkv;
  int j = (int)(x % a.nblk);
  const int b = (int)(x / a.nblk);
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
  double top = 0.;
#pragma unroll
  for (int q = 0; q < 8; ++q) {
#pragma unroll
    for (int d = kLanes; d < 64; d *= 2) sum[q] += __shfl_xor(sum[q], d);
    top = fmax(top, fabs(sum[q]));
  }
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) top = fmax(top, __shfl_xor(top, d));
  if (r == 0) {
    uint32_t out[2] = {};
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int code = top > 0. ? (int)rint(sum[q] * 127. / top) : 0;
      out[q / 4] |= (uint32_t)(code & 0xff) << (8 * (q % 4));
    }
    *(uint2*)(a.codes + (block * a.Hkv + h) * D + c * 8) = uint2{out[0], out[1]};
    if (c == 0) a.scales[block * a.Hkv + h] = (float)(top / (127. * kPage));
  }
}

// ------------------------------------------------------------------- top_k
//
// The top_k of n keys by value, ties to the lowest index, found by their bits: four
// rounds fix eight bits each of the smallest chosen key from a histogram of the
// keys that share the bits above.  Then one pass ranks the chosen ones in
// ascending order: stripes of NT keys, each wave's counts in a table, a prefix sum
// over (stripe, wave).  emit(rank, index) is called once per chosen key.
template <int NT>
struct TopK {
  static constexpr int kWaves = NT / 64;
  static constexpr int kMaxStripes = (NT == 1024 ? kMaxCandPages : kMaxCandBlocks) / NT;
  int hist[256];
  int table[2][kMaxStripes * kWaves];
  int scan[2][kWaves];
  uint32_t prefix;
  int need;
};

template <int NT, typename Emit>
__device__ __forceinline__ void select_top(TopK<NT>& t, const uint32_t* keys, int n, int top_k,
                                           Emit emit) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int W = NT / 64;
  if (n <= top_k) {
    for (int i = tid; i < n; i += NT) emit(i, i);
    return;
  }
  uint32_t prefix = 0, mask = 0;
  int need = top_k;  // of the keys that share the prefix, this many are chosen
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += NT) t.hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
      const uint32_t x = keys[i];
      if ((x & mask) == prefix) atomicAdd(&t.hist[(x >> shift) & 255], 1);
    }
    __syncthreads();
    if (wave == 0) {
      // lane l holds digits 255-4l .. 252-4l, the highest first
      int c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j] = t.hist[255 - 4 * lane - j];
      int upto = sum;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(upto, d);
        if (lane >= d) upto += y;
      }
      int before = upto - sum;
      if (before < need && upto >= need) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (before < need && before + c[j] >= need) {
            t.prefix = prefix | (uint32_t)(255 - 4 * lane - j) << shift;
            t.need = need - before;
          }
          before += c[j];
        }
      }
    }
    __syncthreads();
    prefix = t.prefix;
    need = t.need;
    mask |= 255u << shift;
  }
  // keys above `prefix` are chosen, and the first `need` equal to it
  const int stripes = (n + NT - 1) / NT;
  for (int s = 0; s < stripes; ++s) {
    const int i = s * NT + tid;
    const uint32_t x = i < n ? keys[i] : 0;
    const uint64_t above = __ballot(i < n && x > prefix), same = __ballot(i < n && x == prefix);
    if (lane == 0) {
      t.table[0][s * W + wave] = __popcll(above);
      t.table[1][s * W + wave] = __popcll(same);
    }
  }
  __syncthreads();
  // exclusive prefix sums of the tables: a thread per run of entries
  const int entries = stripes * W, per = (entries + NT - 1) / NT;
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
    int x = sum[q];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
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
  for (int s = 0; s < stripes; ++s) {
    const int i = s * NT + tid;
    const uint32_t x = i < n ? keys[i] : 0;
    const bool above = i < n && x > prefix, same = i < n && x == prefix;
    const uint64_t lower = (1ull << lane) - 1;
    const int na = t.table[0][s * W + wave] + __popcll(__ballot(above) & lower);
    const int ns = t.table[1][s * W + wave] + __popcll(__ballot(same) & lower);
    if (above || (same && ns < need)) emit(na + min(ns, need), i);
  }
}

// A score as a whole number that orders as it does (+0 and -0 alike).
__device__ __forceinline__ uint32_t order_bits(float x) {
  const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kForced = 0xffffffffu;  // blocks that are always chosen

// 16 channels of a query row as codes.
__device__ __forceinline__ i32x4 quantise(const uint16_t* q, float top) {
  const u32x4 lo = *(const u32x4*)q, hi = *(const u32x4*)(q + 8);
  i32x4 out;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t packed = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t x = w < 2 ? lo[2 * w + j] : hi[2 * (w - 2) + j];
      const float f0 = bf16_float(x & 0xffffu), f1 = __uint_as_float(x & 0xffff0000u);
      const int c0 = top > 0.f ? (int)rintf(f0 * 127.f / top) : 0;
      const int c1 = top > 0.f ? (int)rintf(f1 * 127.f / top) : 0;
      packed |= (uint32_t)(c0 & 0xff) << (16 * j) | (uint32_t)(c1 & 0xff) << (16 * j + 8);
    }
    out[w] = (int)packed;
  }
  return out;
}

__device__ __forceinline__ float abs_max8(u32x4 w) {
  float m = 0.f;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    m = fmaxf(m, fmaxf(fabsf(bf16_float(w[q] & 0xffffu)), fabsf(__uint_as_float(w[q] & 0xffff0000u))));
  return m;
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

// The largest of a lane's 16 products and m.
__device__ __forceinline__ int max16(const i32x16& c, int m) {
#pragma unroll
  for (int i = 0; i < 16; i += 2) m = max(m, max(c[i], c[i + 1]));
  return m;
}

constexpr int kSelThreads = 256;

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
__global__ __launch_bounds__(kSelThreads) void select_blocks_kernel(SelectArgs a) {
  using ST = SelTiles<D>;
  extern __shared__ __attribute__((aligned(16))) uint8_t sel_smem[];
  TopK<kSelThreads>& topk = *(TopK<kSelThreads>*)sel_smem;
  uint8_t* const rows_lds = sel_smem + (sizeof(TopK<kSelThreads>) + 15) / 16 * 16;
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
  float top = 0.f;
  for (int c = tid; c < n_rows * (D / 8); c += kSelThreads)
    top = fmaxf(top, abs_max8(*(const u32x4*)(row_at(c / (D / 8)) + c % (D / 8) * 8)));
  top = wave_max(top);
  if (lane == 0) red[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));

  const int64_t blk0 = base / kPage + b;
  for (int p0 = 0; p0 < n_rows; p0 += ST::kRowTiles * 32) {
    if (p0) __syncthreads();
    const int rows = min(n_rows - p0, ST::kRowTiles * 32);
    const int tiles = (rows + 31) / 32;
    // (rows past the last repeat it, which changes no maximum)
    for (int c = tid; c < tiles * 32 * (D / 16); c += kSelThreads) {
      const int r = c / (D / 16), w = c % (D / 16);
      *(i32x4*)(rows_lds + r * ST::kRowBytes + w * 16) = quantise(row_at(p0 + min(r, rows - 1)) + w * 16, top);
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
  select_top<kSelThreads>(topk, keys, n, a.top_k, [&](int rank, int i) { list[rank] = i; });
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

template <int D>
__global__ __launch_bounds__(kSelThreads) void score_pages_kernel(SelectArgs a) {
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int wave = threadIdx.x >> 6;
  const int G = a.Hq / a.Hkv;
  const int64_t item = blockIdx.x / (unsigned)a.Hkv;
  const int g = blockIdx.x % (unsigned)a.Hkv;
  Token tk;
  if (!token_of(a, item, &tk)) return;
  const int n = min(max(tk.pos, 0) / kPage, a.max_blocks);
  const int t0 = blockIdx.y * (kScoreTiles * 32);
  if (t0 >= n || n <= a.top_k) return;  // (all are chosen without scores)
  const uint16_t* const q0 = a.q + (tk.t * a.Hq + (int64_t)g * G) * D;
  float top = 0.f;
  for (int c = lane; c < G * (D / 8); c += 64) top = fmaxf(top, abs_max8(*(const u32x4*)(q0 + c * 8)));
  top = wave_max(top);
  const int32_t* const row = a.table + (int64_t)tk.s * a.M;
  uint32_t* const keys = a.keys + ((int64_t)item * a.Hkv + g) * a.max_blocks;
  constexpr int kPer = kScoreTiles / (kSelThreads / 64);  // tiles of a wave
  int m[kPer];
  for (int u = 0; u < G; u += 32) {  // (more than one turn for more than 32 heads only)
    const uint16_t* qr = q0 + (int64_t)min(u + col, G - 1) * D + half * 16;
    i32x4 qf[D / 32];
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) qf[kk] = quantise(qr + kk * 32, top);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int j = min(t0 + (i * (kSelThreads / 64) + wave) * 32 + col, n - 1);
      int e = row[j];
      e = (unsigned)e < (unsigned)a.P ? e : 0;
      const int8_t* cp = a.codes + ((int64_t)e * a.Hkv + g) * D + half * 16;
      i32x16 acc = i32x16{};
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) acc = mfma_i8(qf[kk], *(const i32x4*)(cp + kk * 32), acc);
      m[i] = max16(acc, u ? m[i] : INT32_MIN);
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    m[i] = max(m[i], __shfl_xor(m[i], 32));
    const int j = t0 + (i * (kSelThreads / 64) + wave) * 32 + col;
    if (half == 0 && j < n) {
      // (a page that the table does not name comes last: nothing of it is attended to)
      const int e = row[j];
      uint32_t key = 0u;
      if ((unsigned)e < (unsigned)a.P) key = order_bits((float)m[i] * a.scales[(int64_t)e * a.Hkv + g]);
      keys[j] = j < a.n_sink || j >= n - a.n_recent ? kForced : key;
    }
  }
}

constexpr int kPickThreads = 1024;
__global__ __launch_bounds__(kPickThreads) void pick_pages_kernel(SelectArgs a) {
  __shared__ TopK<kPickThreads> topk;
  const int64_t item = blockIdx.x / (unsigned)a.Hkv;
  const int g = blockIdx.x % (unsigned)a.Hkv;
  Token tk;
  if (!token_of(a, item, &tk)) return;
  const int n = min(max(tk.pos, 0) / kPage, a.max_blocks);
  int32_t* const list = a.pages + (tk.t * a.Hkv + g) * a.top_k;
  for (int i = min(n, a.top_k) + threadIdx.x; i < a.top_k; i += kPickThreads) list[i] = -1;
  const uint32_t* keys = a.keys + ((int64_t)item * a.Hkv + g) * a.max_blocks;
  select_top<kPickThreads>(topk, keys, n, a.top_k, [&](int rank, int i) { list[rank] = i; });
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
  const size_t head = (sizeof(TopK<kSelThreads>) + 15) / 16 * 16;
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
  hipLaunchKernelGGL(pick_pages_kernel, dim3((unsigned)items), dim3(kPickThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace da
