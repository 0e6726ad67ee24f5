// da_paged_attn.hip -- attention of new tokens over a paged cache (gfx950): trees
// of drafted tokens, single tokens and causal chunks over every page, or single
// rows over lists of selected pages.
//
//   out_r = sum_j w_rj v_j / sum_j w_rj,  w_rj = exp(q_r.k_j / sqrt d), over the
//   keys j that row r sees; a row that sees none is 0
//
// A row is one query head of one token; the n * G rows of a sequence's tokens that
// share a kv head read the same keys.  Tile core as in the prefill kernels: S^T =
// K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16_bf16, a lane owning one row.
// Keys and values arrive by LDS DMA in units of 32 keys (half a page).
//
// What bounds it: with few rows every key and value is read from HBM once and used
// by few MFMAs, so that HBM bounds; the workgroup then keeps as many bytes in flight
// as LDS holds.  Each of its four waves takes units of its own (4 key streams, no
// barrier in the loop), and the waves' partial results meet at the end.  With more
// rows, tiles of 32 rows share a unit: 2 tiles x 2 streams, 4 x 1, or 8 x 1.
// The pages of all rows' keys, sequence by sequence and head by head, are one line of
// work that the workgroups share evenly, as many of them as run at once: each takes a
// stretch of it, whatever sequences that touches.  Rows whose keys several workgroups
// have are merged by a second launch.
//
// Measured (32 heads on 8, d 128): 64 single tokens over up to 8192 keys, 1.37 GB in 239 us,
// 5.7 TB/s; one over 131072 keys, 0.54 GB in 97 us; 16 trees of 24 over up to 6000 keys, 0.25 GB
// and 20 GFLOP in 50 us; 64 heads on 8, 4 trees of 64 over up to 40000 keys, 0.50 GB and 238
// GFLOP in 234 to 256 us, 0.93 to 1.02 PFLOP/s, the matrix cores busy half the time.  (There
// rings of 3 and 4 stages took as long as 2: not the latency of the transfers.)  With keys
// that stay in the L2 it takes a fifth less.
#include "da_device.hpp"
#include "da_paged.hpp"

#include <math.h>

#include <type_traits>

namespace da {
namespace {

constexpr int kIdPages = 1024;  // page ids that a workgroup holds in LDS at a time

// RT tiles of 32 rows and KS key streams per workgroup of NW waves.
template <int D, int RT>
struct Shape {
  static constexpr int NW = RT > 4 ? RT : 4;
  static constexpr int KS = NW / RT;
  // Keys per unit: half a page where four streams share LDS, else a whole page.
  static constexpr int UNIT = KS == 4 ? 32 : 64;
  static constexpr int UPP = kPage / UNIT;  // units per page
  static constexpr int NB = UNIT / 32;      // 32-key blocks of scores
  static constexpr int unitElems = 2 * UNIT * D;  // keys, then values
  // ring of each stream: 128 KB together at d = 128 where several stream, 64 KB for one
  static constexpr int DEPTH = 2;
  static constexpr int ringElems = KS * DEPTH * unitElems;
  static constexpr int regions = UNIT * D * 2 / 1024;  // 1 KB DMA regions per tile
  static constexpr int RPW = regions / RT;             // of a wave
  static constexpr int ldsBytes = ringElems * 2 + kIdPages * 4 + 256;
  // Weights as two bf16 parts, the nearest value and what it leaves (2^-16 of a weight is lost
  // instead of 2^-8): the root mean square error of the outputs is that of their own rounding.
  // One row tile has matrix cores to spare behind HBM: 64 single tokens over 8192 keys 239.8 -> 241.1
  // us, one over 131072 104.9 -> 105.6, 16 over 64 pages each 64.1 -> 65.3 (at worst, bound by
  // latency, one over 448: 10.5 -> 11.3).  More tiles do not: two
  // 52.9 -> 58.8 (16 trees of 12), 31.5 -> 36.1 (d = 64), four 58.5 -> 73.1 (16 of 24), eight 255 ->
  // 353 (4 of 64, 64 heads); their weights are rounded once.
  static constexpr bool TWO_PARTS = RT == 1;
  // waves per SIMD that LDS has room for
  static constexpr int WAVES = ldsBytes > 81920 ? 1 : 2;
  __device__ static constexpr int kswz(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
  __device__ static constexpr int vswz(int r) {
    return D == 128 ? ((r & 3) << 2) : (((r >> 1) & 1) << 2);
  }
};

template <int N>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70);
}

// One sequence: its new tokens, its keys, and its share of the work.
struct SeqWork {
  int64_t base;  // first row of q
  int m;         // new tokens
  int s;         // slot
  int L;         // keys
  int np;        // pages that each of its segments reads, at least 1
  int n_rg;      // row groups per kv head (and token, with lists)
  int segs;      // segments: (token with lists,) kv head, row group
};
template <bool LISTS>
__device__ __forceinline__ SeqWork seq_work(const PagedArgs& a, int b, int group_rows) {
  SeqWork x;
  x.base = a.cu ? a.cu[b] : (int64_t)b * a.N;
  x.m = max(0, min(a.cu ? a.cu[b + 1] - a.cu[b] : a.N, a.N));
  x.s = a.slots ? a.slots[b] : b;
  x.L = (unsigned)x.s < (unsigned)a.S ? min(max(a.lens[x.s], 0), min(a.max_len, a.M * kPage)) : 0;
  x.np = LISTS ? a.n_list + 1 : max(1, (x.L + kPage - 1) / kPage);
  x.n_rg = (unsigned)((LISTS ? a.G : x.m * a.G) + group_rows - 1) / (unsigned)group_rows;
  x.segs = (LISTS ? x.m : 1) * a.Hkv * x.n_rg;
  return x;
}
// Units of work that count for a sequence: pages of its segments, or whole segments.
__device__ __forceinline__ int units_of(const PagedArgs& a, const SeqWork& x) {
  return a.whole ? x.segs : x.segs * x.np;
}

template <int D, int RT, bool LISTS>
__global__ __launch_bounds__((64 * Shape<D, RT>::NW), (Shape<D, RT>::WAVES)) void paged_attn_kernel(PagedArgs a) {
  using SH = Shape<D, RT>;
  constexpr int NW = SH::NW, KS = SH::KS, DEPTH = SH::DEPTH, RPW = SH::RPW, MB = D / 32;
  constexpr int UNIT = SH::UNIT, UPP = SH::UPP, NB = SH::NB;
  constexpr int kThreads = 64 * NW;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];
  int* const ids = (int*)(smem + SH::ringElems);

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int rt = wave % RT, ks = wave / RT;
  const int G = a.G;

  // ---- this workgroup's share: units [x0, x1) of all sequences' in a row.  Neighbours
  // in that order run on one XCD (block i goes to XCD i % 8): row groups of the same keys
  // meet in its L2.
  const int w = gridDim.x % 8 == 0 ? (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8) : (int)blockIdx.x;
  // Up to 64 sequences each wave holds in its lanes, one each, and looks up there;
  // more are counted by the whole workgroup and loaded one by one.
  const bool few = a.B <= 64;
  auto from_lane = [](const SeqWork& x, int j) {
    SeqWork y;
    y.base = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)x.base, j) |
             (int64_t)__builtin_amdgcn_readlane((int)(x.base >> 32), j) << 32;
    y.m = __builtin_amdgcn_readlane(x.m, j);
    y.s = __builtin_amdgcn_readlane(x.s, j);
    y.L = __builtin_amdgcn_readlane(x.L, j);
    y.np = __builtin_amdgcn_readlane(x.np, j);
    y.n_rg = __builtin_amdgcn_readlane(x.n_rg, j);
    y.segs = __builtin_amdgcn_readlane(x.segs, j);
    return y;
  };
  SeqWork held{};
  int b, off, left;
  bool aligned = false;  // segments begin with workgroups
  int team = 1;          // workgroups that take one stretch, a row group each
  if (few) {
    if (lane < a.B) held = seq_work<LISTS>(a, lane, RT * 32);
    int mine = lane < a.B ? units_of(a, held) : 0;
    if (!LISTS && a.row_groups > 1) {
      // The row groups of a kv head read the same pages: workgroups next to each other take
      // one stretch of them in step and meet in the L2, where sequences with fewer row groups
      // than others leave at most a sixteenth of the workgroups' time idle.  (4 trees of 64 over
      // 40000 keys, 64 heads on 8: 0.50 GB fetched instead of 1.00, 308 us a call instead of 348
      // in a row; contexts that the cache behind the L2 holds as before.)
      const int columns = lane < a.B && held.segs ? a.Hkv * held.np : 0;
      if ((int64_t)wave_add(columns) * a.row_groups * 16 <= (int64_t)wave_add(mine) * 17) {
        team = a.row_groups;
        held.segs = held.segs ? a.Hkv : 0;
        mine = columns;
      }
    }
    const int n_wgs = a.n_wgs / team, wt = w / team;
    int upto = wave_scan_add(mine), units = mine;
    int total = __builtin_amdgcn_readlane(upto, 63);
    int share = share_of(a.min_units, total, n_wgs);
    if (!a.whole) {
      // Where segments are few against workgroups, whole workgroups go to each: a
      // second segment would cost a workgroup another start, more than the pages that
      // the even share saves.
      const int segs = wave_add(lane < a.B ? held.segs : 0);
      if (segs < n_wgs && (double)total * segs < (double)a.align_pages * n_wgs * (n_wgs - segs)) {
        aligned = true;
        share = share_of(a.min_units, total, n_wgs - segs);
        units = lane < a.B ? held.segs * ((held.np + share - 1) / share * share) : 0;
        upto = wave_scan_add(units);
        total = __builtin_amdgcn_readlane(upto, 63);
      }
    }
    const int before = upto - units;
    const int64_t x0 = (int64_t)wt * share;
    if (w == 0 && tid < 64 && a.units) {  // (for the merge)
      if (lane < a.B) a.units[lane] = before;
      if (lane == 0) {
        a.units[a.B] = share;
        a.units[a.B + 1] = aligned;
        a.units[a.B + 2] = team;
      }
    }
    if (wt >= n_wgs || x0 >= total) return;
    left = min(share, total - (int)x0);
    b = __builtin_ctzll(__ballot(before <= x0 && x0 < upto));
    off = (int)x0 - __builtin_amdgcn_readlane(before, b);
  } else {
    int* const red = ids + kIdPages;  // [NW] sums, then what is found
    auto block_scan = [&](int x, int* total) {
      x = wave_scan_add(x);
      __syncthreads();
      if (lane == 63) red[wave] = x;
      __syncthreads();
      int before = 0, all = 0;
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        before += v < wave ? red[v] : 0;
        all += red[v];
      }
      *total = all;
      return x + before;
    };
    auto units_at = [&](int j) { return j < a.B ? units_of(a, seq_work<LISTS>(a, j, RT * 32)) : 0; };
    int mine = units_at(tid), sum, total;
    int upto = block_scan(mine, &sum);
    total = sum;
    for (int b0 = kThreads; b0 < a.B; b0 += kThreads) {
      int more;
      block_scan(units_at(b0 + tid), &more);
      total += more;
    }
    total = __builtin_amdgcn_readfirstlane(total);
    const int share = share_of(a.min_units, total, a.n_wgs);
    const int64_t x0 = (int64_t)w * share;
    if (w == 0 && tid == 0 && a.units) {
      a.units[a.B] = share;
      a.units[a.B + 1] = 0;
      a.units[a.B + 2] = 1;
    }
    if (x0 >= total) return;
    left = min(share, total - (int)x0);
    for (int b0 = 0, carry = 0; b0 < a.B; b0 += kThreads) {
      if (b0) {
        mine = units_at(b0 + tid);
        upto = block_scan(mine, &sum);
      }
      const int64_t before = (int64_t)carry + upto - mine;
      if (w == 0 && b0 + tid < a.B && a.units) a.units[b0 + tid] = (int)before;
      if (before <= x0 && x0 < before + mine) {
        red[NW] = b0 + tid;
        red[NW + 1] = (int)(x0 - before);
      }
      carry += sum;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane(red[NW]);
    off = __builtin_amdgcn_readfirstlane(red[NW + 1]);
  }
  auto seq_at = [&](int j) {
    return few ? from_lane(held, j) : from_lane(seq_work<LISTS>(a, j, RT * 32), 0);
  };
  SeqWork sq = seq_at(b);
  int seg = off, p0 = 0;
  if (!a.whole) {
    const int np = aligned ? (sq.np + left - 1) / left * left : sq.np;  // (`left` is the share there)
    seg = (unsigned)off / (unsigned)np;
    p0 = off - seg * np;
  }

  // ---- segment after segment
  while (true) {
  const int head = sq.n_rg == 1 || team > 1 ? seg : (unsigned)seg / (unsigned)sq.n_rg;
  const int rg = team > 1 ? w % team : seg - head * sq.n_rg;
  const int tok = LISTS ? (int)fdiv(head, a.fd_Hkv) : 0;  // the token of a list
  const int g = head - tok * a.Hkv;
  const int p1 = a.whole ? sq.np : min(sq.np, p0 + left);
  const bool direct = p0 == 0 && p1 == sq.np;  // no other workgroup has keys of these rows
  const int64_t base = sq.base;
  const int m = sq.m;
  const int n_rows = LISTS ? G : m * G;
  const int row0 = rg * (RT * 32);
  const int first = sq.L - m;  // the position of the first new token
  // (with lists a row whose own position is missing reads nothing)
  const int own = LISTS ? max(first + tok, 0) / kPage : 0;
  // keys: up to the last that some row sees
  const int last_key = LISTS ? first + tok : sq.L - 1;

  // ---- this lane's row
  const int r = row0 + rt * 32 + col;
  const int rc = min(r, n_rows - 1);
  const int i_tok = LISTS ? tok : (int)fdiv(rc, a.fd_G);
  const int64_t t = base + i_tok;
  const int h = g * G + (LISTS ? rc : rc - i_tok * G);
  const int pos = first + i_tok;
  bf16x8 qf[D / 16];
  {
    const uint16_t* qp = a.q + (t * a.Hq + h) * (int64_t)D + half * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *(const bf16x8*)(qp + kk * 16);
  }

  // ---- state of the rows
  f32x16 o[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) o[mb] = f32x16{};
  // Online softmax against a lagging reference, as in the prefill kernels: `ref` in
  // base-2 units of the logits, -ref / c in every register of nref, from which the score
  // accumulators start, so that c times them is logit - ref.
  const float c2 = a.scale_log2, inv_c2 = 1.f / a.scale_log2;
  float ref = 0.f, l = 0.f;
  bool has_ref = false;
  f32x16 nref = f32x16{};
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 ones2 = {(__bf16)1.0f, (__bf16)1.0f};

  // ---- the segment's pages, as many at a time as there is room for ids
  const int p_end = last_key < 0 || row0 >= n_rows ? p0 : p1;
  for (int q0 = p0; q0 < p_end; q0 += kIdPages) {
  const int q1 = min(q0 + kIdPages, p_end), n_pages = q1 - q0;
  if (q0 > p0) __syncthreads();  // (the ids before are read)
  for (int j = tid; j < n_pages; j += kThreads) {
    int at = q0 + j;
    if (LISTS) {
      at = at < a.n_list ? a.lists[((base + tok) * a.Hkv + g) * a.n_list + at] : own;
      if (at < 0 || at > own || (at == own && q0 + j < a.n_list)) at = -1;
    }
    const int e = at >= 0 ? a.table[(int64_t)sq.s * a.M + at] : -1;
    ids[j] = (unsigned)e < (unsigned)a.P ? e : -1;  // (-1: no such page, its keys are not seen)
  }
  // the queries have landed: the loop's products must not wait for them behind the
  // transfers issued there
  wait_vm<0>();
  __syncthreads();

  // ---- units of this wave's stream: ks, ks + KS, ... of these pages'
  // (with lists the last page of all is the own one)
  const bool ends = q1 == sq.np;
  const int tail_pos = LISTS ? own * kPage : (q1 - 1) * kPage;  // position of the last page
  const int n_units = (n_pages - 1) * UPP + (ends ? min(UPP, (last_key - tail_pos) / UNIT + 1) : UPP);
  const int tail_keys = ends ? last_key + 1 - tail_pos - (n_units - 1) % UPP * UNIT : UNIT;  // of the last unit
  const int n_it = (n_units + KS - 1) / KS;
  const uint32_t smem_lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)smem;
  const uint32_t ring = smem_lds + (uint32_t)(ks * DEPTH * SH::unitElems) * 2;
  const uint64_t page_bytes = (uint64_t)a.Hkv * kPage * D * 2;
  const uint64_t head_off = (uint64_t)g * kPage * D * 2;
  const uint64_t k0_addr = (uint64_t)a.k + head_off, v0_addr = (uint64_t)a.v + head_off;
  int dma_row[RPW], dma_kc[RPW], dma_vc[RPW];
#pragma unroll
  for (int i = 0; i < RPW; ++i) {
    const int byte = (rt * RPW + i) * 1024 + 16 * lane;
    dma_row[i] = byte / (2 * D);
    const int pc = (byte % (2 * D)) / 16;
    dma_kc[i] = (pc ^ SH::kswz(dma_row[i])) * 16;
    dma_vc[i] = (pc ^ SH::vswz(dma_row[i])) * 16;
  }
  auto page_of = [&](int it) -> int {  // -1: nothing to read (a vector register until dma)
    const int u = it * KS + ks;
    const int e = ids[min(u, n_units - 1) / UPP];
    return u < n_units ? e : -1;
  };
  // Every call issues 2 * RPW transfers, so that waits can count them; a unit
  // without keys reads page 0.  Rows past the last key read that key: what lies
  // behind it in the page may be anything, and a weight of zero times it could be
  // NaN.
  auto dma = [&](int it, int stage, int page) -> int {
    const int e = __builtin_amdgcn_readfirstlane(page);
    const int u = it * KS + ks;
    const int keys = e < 0 ? 1 : u == n_units - 1 ? tail_keys : UNIT;
    const uint64_t off = (uint64_t)max(e, 0) * page_bytes + (uint64_t)(u % UPP * UNIT * D * 2);
    const uint64_t ka = k0_addr + off, va = v0_addr + off;
    i32x4 kr = {(int)(uint32_t)ka, (int)((uint32_t)(ka >> 32) & 0xffffu), UNIT * D * 2, 0x00020000};
    i32x4 vr = {(int)(uint32_t)va, (int)((uint32_t)(va >> 32) & 0xffffu), UNIT * D * 2, 0x00020000};
    uint32_t dst = ring + (uint32_t)(stage * SH::unitElems) * 2;
    settle_sgprs(kr, vr, dst);
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
      const uint32_t region = (uint32_t)((rt * RPW + i) * 1024);
      const int row = min(dma_row[i], keys - 1) * (2 * D);
      dma16(kr, dst + region, row + dma_kc[i]);
      dma16(vr, dst + UNIT * D * 2 + region, row + dma_vc[i]);
    }
    return e;
  };

  // ---- LDS offsets of the operands (elements inside the stream's ring; the stage is a
  // constant of the loop's unrolled halves)
  const int ring0 = ks * DEPTH * SH::unitElems;
  int kread[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) kread[kk] = ring0 + col * D + (((2 * kk + half) ^ SH::kswz(col)) * 8);
  const int tr_g1 = (lane >> 4) & 1, tr_k = (lane >> 2) & 3, tr_m = lane & 3;
  const int vsw = SH::vswz(4 * half + tr_k);
  int vread[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
    vread[mb] = ring0 + (4 * half + tr_k) * D + (((4 * mb + 2 * tr_g1 + (tr_m >> 1)) ^ vsw) * 8) + (tr_m & 1) * 4;

  // Which of 32 keys from position k0 on this lane's row sees, bit by bit.
  auto visible = [&](int k0) -> uint32_t {
    if (LISTS || !a.mask) {
      const int c = pos - k0;  // sees keys 0 .. c
      return c < 0 ? 0u : c >= 31 ? ~0u : (2u << c) - 1u;
    }
    const int j0 = k0 - first;  // place of the first key among the new tokens
    // (the context is seen whole: ones below place 0; nothing past the last word)
    uint64_t lo = 0, hi = 0;
    const uint64_t* w = a.mask + t * a.mask_words;
    if (j0 <= -32) return ~0u;
    if (j0 < 0) return (uint32_t)(w[0] << -j0) | ((1u << -j0) - 1u);
    const int word = j0 >> 6, sh = j0 & 63;
    if (word < a.mask_words) lo = w[word];
    if (word + 1 < a.mask_words) hi = w[word + 1];
    return (uint32_t)(sh ? (lo >> sh) | (hi << (64 - sh)) : lo);
  };

  auto compute = [&](int it, auto stage) {
    const int u = it * KS + ks;
    const uint16_t* ku = smem + decltype(stage)::value * SH::unitElems;
    const uint16_t* vu = ku + UNIT * D;
    f32x16 sc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) sc[nb] = nref;
    // K reads kAhead MFMAs ahead of their use, an order that the scheduling barriers hold
    // (left to itself the compiler pairs each MFMA with its own read and a wait)
    constexpr int kAhead = 4, kProducts = NB * D / 16;
    auto kfrag = [&](int i) { return *(const bf16x8*)(ku + kread[i / NB] + (i % NB) * 32 * D); };
    bf16x8 kf[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) kf[i] = kfrag(i);
#pragma unroll
    for (int i = 0; i < kProducts; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      sc[i % NB] = mfma32(kf[i % kAhead], qf[i / NB], sc[i % NB]);
      if (i + kAhead < kProducts) kf[i % kAhead] = kfrag(i + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0);
    // mask the units that some row does not see whole
    const int at = q0 + u / UPP;
    const int k0 = (LISTS ? own : at) * kPage + u % UPP * UNIT;
    if (LISTS ? at >= a.n_list : k0 + UNIT > first) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int keys = last_key + 1 - (k0 + nb * 32);
        uint32_t vis = keys > 0 ? visible(k0 + nb * 32) : 0u;
        if (keys < 32 && keys > 0) vis &= (1u << keys) - 1u;
        vis >>= 4 * half;
#pragma unroll
        for (int q = 0; q < 16; ++q) sc[nb][q] = (vis >> (8 * (q >> 2) + (q & 3))) & 1u ? sc[nb][q] : -INFINITY;
      }
    }
    // Weights are bf16 in the second product: two parts of each, and the normaliser sums the
    // fp32 ones; or the nearest value, and the normaliser sums those, so that the rounding
    // cancels where one key dominates.
    bf16x8 pf[2 * NB], rest[2 * NB];
    auto weights = [&]() {
      f32x16 p[NB];
#pragma unroll
      for (int q = 0; q < 16; ++q)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) p[nb][q] = fast_exp2(c2 * sc[nb][q]);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        pf[2 * nb] = __builtin_convertvector(p[nb].lo, bf16x8);
        pf[2 * nb + 1] = __builtin_convertvector(p[nb].hi, bf16x8);
      }
      float ta = 0.f, tb = 0.f;
      if constexpr (SH::TWO_PARTS) {
        auto left = [](f32x8 x, bf16x8 y) { return __builtin_convertvector(x - __builtin_convertvector(y, f32x8), bf16x8); };
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          rest[2 * nb] = left(p[nb].lo, pf[2 * nb]);
          rest[2 * nb + 1] = left(p[nb].hi, pf[2 * nb + 1]);
#pragma unroll
          for (int q = 0; q < 16; q += 2) {
            ta += p[nb][q];
            tb += p[nb][q + 1];
          }
        }
        return ta + tb;
      }
#pragma unroll
      for (int f = 0; f < 2 * NB; ++f) {
        ta = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(pf[f], pf[f], 0, 1), ones2, ta, false);
        tb = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(pf[f], pf[f], 2, 3), ones2, tb, false);
        ta = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(pf[f], pf[f], 4, 5), ones2, ta, false);
        tb = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(pf[f], pf[f], 6, 7), ones2, tb, false);
      }
      return ta + tb;
    };
    // While every score lies within 8 of the reference, a lane's 16 NB weights sum to at
    // most 16 NB 2^8; only past that is the row's maximum taken, and the reference moves up
    // if a weight passes 2^8.  The result is the same whatever the reference.
    float tsum = INFINITY;
    if (!__any(!has_ref)) tsum = weights();
    if (__any(!(tsum <= 4096.f * NB))) {
      float mx = sc[0][0];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int q = 0; q < 16; ++q) mx = fmaxf(mx, sc[nb][q]);
      const auto pr = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = c2 * fmaxf(__uint_as_float(pr[0]), __uint_as_float(pr[1]));
      // a lane without a reference takes the unit's maximum (if it sees a key); one with a
      // reference moves only up
      const bool seen = mx != -INFINITY;
      if (__any(has_ref ? mx > 8.f : seen)) {
        const float dm = has_ref ? fmaxf(mx, 0.f) : (seen ? mx : 0.f);
        const float alpha = has_ref ? fast_exp2(-dm) : 0.f;  // l and O are still zero without one
        ref += dm;
        has_ref = has_ref || seen;
        l *= alpha;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) o[mb] *= alpha;
        const float dr = dm * inv_c2;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) sc[nb][q] -= dr;
          nref[q] = -ref * inv_c2;
        }
      }
      tsum = weights();
    }
    l += tsum;
    // V^T reads (two per MFMA) likewise
    constexpr int kSums = 2 * NB * MB;
    auto vfrag = [&](int i) {
      const uint16_t* p = vu + vread[i % MB] + (16 * (i / MB)) * D;
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lds_read_tr(p), lds_read_tr(p + 8 * D), 0, 1, 2, 3, 4, 5, 6, 7));
    };
    bf16x8 vf[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) vf[i] = vfrag(i);
#pragma unroll
    for (int i = 0; i < kSums; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      o[i % MB] = mfma32(vf[i % kAhead], pf[i / MB], o[i % MB]);
      if constexpr (SH::TWO_PARTS) o[i % MB] = mfma32(vf[i % kAhead], rest[i / MB], o[i % MB]);
      if (i + kAhead < kSums) vf[i % kAhead] = vfrag(i + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  // ---- the loop.  Streams of one wave need no barrier: a stage is filled again when
  // the wave's own reads of it are done.  Waves that share a unit publish its parts
  // with one barrier per unit, which also says that the unit before it is read.  Page
  // ids are read one unit ahead of the transfers that need them.
  static_assert(DEPTH == 2, "the loop is unrolled by stage");
  int now = dma(0, 0, page_of(0)), next = page_of(1);
  auto step = [&](int it, auto stage) {
    constexpr int kOther = 1 - decltype(stage)::value;
    int after;
    if (RT == 1) {
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the reads of the stage that fills next
      asm volatile("" ::: "memory");
      after = dma(it + 1, kOther, next);
      wait_vm<2 * RPW>();
      asm volatile("" ::: "memory");
    } else {
      wait_vm<0>();
      __syncthreads();
      after = dma(it + 1, kOther, next);
    }
    next = page_of(it + 2);
    if (now >= 0) compute(it, stage);
    now = after;
  };
  for (int it = 0; it < n_it; it += 2) {
    step(it, std::integral_constant<int, 0>{});
    if (it + 1 < n_it) step(it + 1, std::integral_constant<int, 1>{});
  }
  wait_vm<0>();
  }  // (pages)
  __syncthreads();  // every transfer has landed and every read is done: the ring is free
  // A row that has seen nothing has the reference kNone, whose share of any sum is 0.
  constexpr float kNone = -1e30f;
  if (!has_ref) ref = kNone;

  // ---- the streams' partial results meet: stream ks takes dims of block mb = ks
  if (KS > 1) {
    f32x4* const xo = (f32x4*)smem;                       // [rt][ks][mb][4][64]
    f32x2* const xml = (f32x2*)(smem + SH::ringElems);    // [rt][ks][64] (over the ids)
    const int slot = (rt * KS + ks) * MB;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        xo[((slot + mb) * 4 + q) * 64 + lane] = f32x4{o[mb][4 * q], o[mb][4 * q + 1], o[mb][4 * q + 2], o[mb][4 * q + 3]};
    xml[(rt * KS + ks) * 64 + lane] = f32x2{ref, l};
    __syncthreads();
    float top = kNone;
#pragma unroll
    for (int w = 0; w < KS; ++w) top = fmaxf(top, xml[(rt * KS + w) * 64 + lane][0]);
    float sum = 0.f;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) o[mb] = f32x16{};
#pragma unroll
    for (int w = 0; w < KS; ++w) {
      const f32x2 ml = xml[(rt * KS + w) * 64 + lane];
      const float f = fast_exp2(ml[0] - top);
      sum += f * ml[1];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        if (mb % KS != ks) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 x = xo[(((rt * KS + w) * MB + mb) * 4 + q) * 64 + lane];
#pragma unroll
          for (int z = 0; z < 4; ++z) o[mb][4 * q + z] += f * x[z];
        }
      }
    }
    ref = top;
    l = sum;
  }
  {  // the normaliser's other share
    const auto pr = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(pr[0]) + __uint_as_float(pr[1]);
  }
  const int64_t orow = t * a.Hq + h;
  if (direct && r < n_rows) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      if (mb % KS != ks) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        const f32x4 x = {o[mb][4 * q] * inv, o[mb][4 * q + 1] * inv, o[mb][4 * q + 2] * inv, o[mb][4 * q + 3] * inv};
        *(bf16x4*)(a.out + orow * D + 32 * mb + 8 * q + 4 * half) = __builtin_convertvector(x, bf16x4);
      }
    }
    if (a.lse && ks == 0 && half == 0) a.lse[orow] = l > 0.f ? (ref + __log2f(l)) * 0.6931471805599453f : -INFINITY;
  } else if (r < n_rows) {
    // A workgroup cuts at most the first and the last of its segments: place 1 holds one
    // that begins with its rows' first page, place 0 one that does not.
    const int64_t prow = (int64_t)(2 * w + (p0 == 0 ? 1 : 0)) * (RT * 32) + rt * 32 + col;
    float* const po = a.part_o + prow * D;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      if (mb % KS != ks) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(f32x4*)(po + 32 * mb + 8 * q + 4 * half) =
            f32x4{o[mb][4 * q], o[mb][4 * q + 1], o[mb][4 * q + 2], o[mb][4 * q + 3]};
    }
    if (ks == 0 && half == 0) *(f32x2*)(a.part_ml + prow * 2) = f32x2{ref, l};
  }

  // ---- on to the next segment
  left -= a.whole ? 1 : p1 - p0;
  if (left <= 0 || aligned) break;
  p0 = 0;
  if (++seg == sq.segs) {
    seg = 0;
    do {
      if (++b >= a.B) return;  // (not reached: `left` counts the units that follow)
      sq = seq_at(b);
    } while (sq.segs == 0);
  }
  __syncthreads();  // (the ring is read)
  }  // (segments)
}

// Merge of the partial results of rows whose keys several workgroups had.  Groups of
// D/4 lanes, kRowGroups of them per row: one where rows are many, or all of a
// workgroup's, which take workgroups' parts in turn and meet in LDS.  Four loads are
// in flight per group.  Bound by the partial results, which the L2 and the cache behind it
// still hold: 12288 rows of 16 trees 8.2 us, 16384 rows of 4 trees 12.
constexpr int kMergeThreads = 256;
constexpr int kManyRows = 2048;  // from here on a group of lanes per row
template <int D, bool LISTS, bool MANY>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedArgs a) {
  constexpr int kLanes = D / 4, kAll = kMergeThreads / kLanes;
  constexpr int kRows = MANY ? kAll : 1, kRowGroups = kAll / kRows, kFlight = 4;
  __shared__ f32x4 xo[kRowGroups][kLanes];
  __shared__ float xl[kRowGroups];
  const int tid = threadIdx.x, grp = MANY ? 0 : tid / kLanes, c = tid % kLanes;
  const unsigned row = blockIdx.x * kRows + (MANY ? tid / kLanes : 0);
  const unsigned item = fdiv(row, a.fd_Hq);
  const int h = row - item * a.Hq;
  const int b = fdiv(item, a.fd_N), i = item - b * a.N;
  if (b >= a.B) return;  // (past the last row; whole groups only, and no barrier where kRows > 1)
  const unsigned group_rows = a.row_tiles * 32;
  const SeqWork sq = seq_work<LISTS>(a, b, group_rows);
  if (i >= sq.m) return;
  const int g = fdiv(h, a.fd_G);
  const unsigned in_head = (LISTS ? 0 : i * a.G) + h - g * a.G;  // row of the (token and) kv head
  const int team = a.units[a.B + 2], member = team > 1 ? in_head / group_rows : 0;
  const int seg = team > 1 ? g : ((LISTS ? i * a.Hkv : 0) + g) * sq.n_rg + in_head / group_rows;
  const unsigned share = a.units[a.B];
  const int np = a.units[a.B + 1] ? (sq.np + share - 1) / share * share : sq.np;
  const unsigned u0 = a.units[b] + seg * np;
  const int w0 = u0 / share, n = (int)((u0 + sq.np - 1) / share) - w0 + 1;
  if (n <= 1) return;  // written by the one workgroup that has all its keys
  const int64_t orow = (sq.base + i) * a.Hq + h;
  // part 0 lies in place 1 of workgroup (or team) w0, part j in place 0 of w0 + j
  auto place = [&](int j) {
    return (int64_t)(2 * ((w0 + j) * team + member) + (j == 0 ? 1 : 0)) * group_rows + in_head % group_rows;
  };
  const f32x2* ml = (const f32x2*)a.part_ml;
  float top = -1e30f;
  if (MANY) {
    for (int j = c; j < n; j += kLanes) top = fmaxf(top, ml[place(j)][0]);
#pragma unroll
    for (int d = 1; d < kLanes; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  } else {
    for (int j = tid & 63; j < n; j += 64) top = fmaxf(top, ml[place(j)][0]);
    top = wave_fmax(top);
  }
  f32x4 acc = f32x4{};
  float l = 0.f;
  for (int j0 = grp; j0 < n; j0 += kRowGroups * kFlight) {
    f32x2 x[kFlight];
    f32x4 y[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {  // (past the last part: that one again, unused)
      const int64_t at = place(min(j0 + u * kRowGroups, n - 1));
      x[u] = ml[at];
      y[u] = *(const f32x4*)(a.part_o + at * D + c * 4);
    }
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const float f = j0 + u * kRowGroups < n ? fast_exp2(x[u][0] - top) : 0.f;
      l += f * x[u][1];
      acc += f * y[u];
    }
  }
  if (!MANY) {
    xo[grp][c] = acc;
    if (c == 0) xl[grp] = l;
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int w = 1; w < kRowGroups; ++w) {
      acc += xo[w][c];
      l += xl[w];
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *(bf16x4*)(a.out + orow * D + c * 4) = __builtin_convertvector(acc * inv, bf16x4);
  if (a.lse && c == 0) a.lse[orow] = l > 0.f ? (top + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace

hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.n_wgs);
#define DA_PAGED(DD, RT, LS)                                                                       \
  hipLaunchKernelGGL((paged_attn_kernel<DD, RT, LS>), grid, dim3(64 * Shape<DD, RT>::NW),          \
                     (Shape<DD, RT>::ldsBytes), s, a)
#define DA_PAGED_RT(DD, LS)                                                                        \
  switch (a.row_tiles) {                                                                           \
    case 1: DA_PAGED(DD, 1, LS); break;                                                            \
    case 2: DA_PAGED(DD, 2, LS); break;                                                            \
    default: DA_PAGED(DD, 4, LS); break;                                                           \
  }
  if (a.lists) {
    if (a.d == 128) {
      DA_PAGED_RT(128, true)
    } else {
      DA_PAGED_RT(64, true)
    }
  } else if (a.d == 128) {
    if (a.row_tiles == 8)
      DA_PAGED(128, 8, false);
    else
      DA_PAGED_RT(128, false)
  } else {
    DA_PAGED_RT(64, false)
  }
#undef DA_PAGED_RT
#undef DA_PAGED
  if (!a.units) return hipGetLastError();  // no rows are cut
  const int64_t rows = (int64_t)a.B * a.N * a.Hq;
  const bool many = rows >= kManyRows;
  const int per = many ? kMergeThreads / (a.d / 4) : 1;
  const dim3 g((unsigned)((rows + per - 1) / per));
#define DA_MERGE(DD, LS, MANY)                                                                     \
  hipLaunchKernelGGL((paged_merge_kernel<DD, LS, MANY>), g, dim3(kMergeThreads), 0, s, a)
#define DA_MERGE_LS(DD, LS)                                                                        \
  if (many)                                                                                        \
    DA_MERGE(DD, LS, true);                                                                        \
  else                                                                                             \
    DA_MERGE(DD, LS, false)
  if (a.lists) {
    if (a.d == 128) {
      DA_MERGE_LS(128, true);
    } else {
      DA_MERGE_LS(64, true);
    }
  } else if (a.d == 128) {
    DA_MERGE_LS(128, false);
  } else {
    DA_MERGE_LS(64, false);
  }
#undef DA_MERGE_LS
#undef DA_MERGE
  return hipGetLastError();
}

}  // namespace da
