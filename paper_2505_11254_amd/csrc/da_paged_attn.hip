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
// The key axis is split over workgroups; partial results are merged by a second
// launch.
#include "da_device.hpp"
#include "da_paged.hpp"

#include <math.h>

namespace da {
namespace {

constexpr int kMaxSplitPages = 1024;  // page ids of a split, held in LDS

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
  static constexpr int ldsBytes = ringElems * 2 + kMaxSplitPages * 4;
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

// The keys of one row group: pages of the sequence and how they are split.
struct Span {
  int L;      // keys of the sequence
  int first;  // the position of the first new token
  int n;      // pages (list entries and the own page, where there are lists)
  int per;    // pages per split
};
__device__ __forceinline__ Span span_of(const PagedArgs& a, int b, int m, int i) {
  Span x;
  const int s = a.slots ? a.slots[b] : b;
  x.L = (unsigned)s < (unsigned)a.S ? min(max(a.lens[s], 0), min(a.max_len, a.M * kPage)) : 0;
  x.first = x.L - m;
  const int pages = (x.L + kPage - 1) / kPage;
  // with lists a row reads the list's pages and the page of its own position
  x.n = a.lists ? (x.first + i >= 0 ? a.n_list + 1 : 0) : pages;
  x.per = max(1, (x.n + a.n_split - 1) / a.n_split);
  return x;
}
__device__ __forceinline__ int splits_of(const Span& x) { return (x.n + x.per - 1) / x.per; }

template <int D, int RT, bool LISTS>
__global__ __launch_bounds__((64 * Shape<D, RT>::NW), (Shape<D, RT>::WAVES)) void paged_attn_kernel(PagedArgs a, uint32_t n_items) {
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

  // Row groups of the same keys run side by side on one XCD (block i goes to XCD
  // i % 8).
  const uint32_t y = blockIdx.x / 8;
  const uint32_t rg = y % (uint32_t)a.n_rowgroups;
  uint32_t item = (y / (uint32_t)a.n_rowgroups) * 8 + blockIdx.x % 8;
  if (item >= n_items) return;
  const int split = item % (uint32_t)a.n_split;
  item /= (uint32_t)a.n_split;
  const int g = item % (uint32_t)a.Hkv;
  item /= (uint32_t)a.Hkv;
  const int b = LISTS ? item / (uint32_t)a.N : item;
  const int tok = LISTS ? item % (uint32_t)a.N : 0;  // the token of a list
  const int64_t base = a.cu ? a.cu[b] : (int64_t)b * a.N;
  const int m = min(a.cu ? a.cu[b + 1] - a.cu[b] : a.N, a.N);
  if (tok >= m) return;
  const int G = a.Hq / a.Hkv;
  const int n_rows = LISTS ? G : m * G;
  const int row0 = rg * (RT * 32);
  if (row0 >= n_rows) return;
  const Span sp = span_of(a, b, m, tok);
  const int n_eff = splits_of(sp);
  // (a sequence without keys: the first split writes its rows)
  const int p0 = __builtin_amdgcn_readfirstlane(split * sp.per);
  const int p1 = __builtin_amdgcn_readfirstlane(min(p0 + sp.per, sp.n));
  if (p0 >= p1 && split > 0) return;
  const int n_pages = max(p1 - p0, 0);
  const int first = __builtin_amdgcn_readfirstlane(sp.first);

  // ---- page ids of the split (-1: no such page, its keys are not seen)
  const int s = a.slots ? a.slots[b] : b;
  const int own = LISTS ? (first + tok) / kPage : 0;
  for (int j = tid; j < n_pages; j += kThreads) {
    int at = p0 + j;
    if (LISTS) {
      at = at < a.n_list ? a.lists[((base + tok) * a.Hkv + g) * a.n_list + at] : own;
      if (at < 0 || at > own || (at == own && p0 + j < a.n_list)) at = -1;
    }
    const int e = at >= 0 ? a.table[(int64_t)s * a.M + at] : -1;
    ids[j] = (unsigned)e < (unsigned)a.P ? e : -1;
  }

  // ---- this lane's row
  const int r = row0 + rt * 32 + col;
  const int rc = min(r, n_rows - 1);
  const int i_tok = LISTS ? tok : rc / G;
  const int64_t t = base + i_tok;
  const int h = g * G + (LISTS ? rc : rc % G);
  const int pos = first + i_tok;
  bf16x8 qf[D / 16];
  {
    const uint16_t* qp = a.q + (t * a.Hq + h) * (int64_t)D + half * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *(const bf16x8*)(qp + kk * 16);
  }
  // the queries have landed: the loop's products must not wait for them behind the
  // transfers issued there
  wait_vm<0>();
  __syncthreads();

  // ---- units of this wave's stream: ks, ks + KS, ... of the split's
  // the last key that some row of the sequence may see, and the units that hold keys up
  // to there
  const int last_key = __builtin_amdgcn_readfirstlane(LISTS ? first + tok : sp.L - 1);
  // (with lists the last page is the own one, where the split has it)
  const bool ends = p1 == sp.n;
  const int tail_pos = LISTS ? own * kPage : (p1 - 1) * kPage;  // position of the last page
  const int n_units = __builtin_amdgcn_readfirstlane(
      n_pages == 0 ? 0 : (n_pages - 1) * UPP + (ends ? min(UPP, (last_key - tail_pos) / UNIT + 1) : UPP));
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
  auto page_of = [&](int it) -> int {  // -1: nothing to read
    const int u = it * KS + ks;
    const int e = ids[min(u, max(n_units - 1, 0)) / UPP];
    return __builtin_amdgcn_readfirstlane(u < n_units ? e : -1);
  };
  // Every call issues 2 * RPW transfers, so that waits can count them; a unit
  // without keys reads page 0.  Rows past the last key read that key: what lies
  // behind it in the page may be anything, and a weight of zero times it could be
  // NaN.
  auto dma = [&](int it, int e) {
    const int u = it * KS + ks;
    const int keys = e < 0 ? 1 : u == n_units - 1 ? tail_keys : UNIT;
    const uint64_t off = (uint64_t)max(e, 0) * page_bytes + (uint64_t)(u % UPP * UNIT * D * 2);
    const uint64_t ka = k0_addr + off, va = v0_addr + off;
    i32x4 kr = {(int)(uint32_t)ka, (int)((uint32_t)(ka >> 32) & 0xffffu), UNIT * D * 2, 0x00020000};
    i32x4 vr = {(int)(uint32_t)va, (int)((uint32_t)(va >> 32) & 0xffffu), UNIT * D * 2, 0x00020000};
    uint32_t dst = ring + (uint32_t)((it % DEPTH) * SH::unitElems) * 2;
    settle_sgprs(kr, vr, dst);
#pragma unroll
    for (int i = 0; i < RPW; ++i) {
      const uint32_t region = (uint32_t)((rt * RPW + i) * 1024);
      const int row = min(dma_row[i], keys - 1) * (2 * D);
      dma16(kr, dst + region, row + dma_kc[i]);
      dma16(vr, dst + UNIT * D * 2 + region, row + dma_vc[i]);
    }
  };

  // ---- LDS offsets of the operands (elements inside a unit)
  int kread[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) kread[kk] = col * D + (((2 * kk + half) ^ SH::kswz(col)) * 8);
  const int tr_g1 = (lane >> 4) & 1, tr_k = (lane >> 2) & 3, tr_m = lane & 3;
  const int vsw = SH::vswz(4 * half + tr_k);
  int vread[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb)
    vread[mb] = (4 * half + tr_k) * D + (((4 * mb + 2 * tr_g1 + (tr_m >> 1)) ^ vsw) * 8) + (tr_m & 1) * 4;

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

  auto compute = [&](int it) {
    const int u = it * KS + ks;
    const uint16_t* ku = smem + (ks * DEPTH + it % DEPTH) * SH::unitElems;
    const uint16_t* vu = ku + UNIT * D;
    f32x16 sc[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) sc[nb] = nref;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        sc[nb] = mfma32(*(const bf16x8*)(ku + kread[kk] + nb * 32 * D), qf[kk], sc[nb]);
    if (NB == 2) {
      // K reads four MFMAs ahead of their use
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int i = 0; i < D / 8 - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    }
    // mask the units that some row does not see whole
    const int at = p0 + u / UPP;
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
    // Weights are rounded to bf16 for the second product; the normaliser sums the
    // rounded ones, so that the rounding cancels where one key dominates.
    bf16x8 pf[2 * NB];
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
#pragma unroll
    for (int f = 0; f < 2 * NB; ++f)
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        const i16x4 lo = lds_read_tr(vu + vread[mb] + (16 * f) * D);
        const i16x4 hi = lds_read_tr(vu + vread[mb] + (16 * f + 8) * D);
        const i16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        o[mb] = mfma32(__builtin_bit_cast(bf16x8, both), pf[f], o[mb]);
      }
    if (NB == 2) {
      // V^T reads (two per MFMA) four MFMAs ahead of their use
      __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
      for (int i = 0; i < D / 8 - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    }
  };

  // ---- the loop.  Streams of one wave need no barrier: a stage is filled again when
  // the wave's own reads of it are done.  Waves that share a unit publish its parts
  // with one barrier per unit, which also says that the unit before it is read.  Page
  // ids are read one unit ahead of the transfers that need them.
  int e[DEPTH];  // ids of the units in flight, the next to compute first
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d) {
    e[d] = page_of(d);
    dma(d, e[d]);
  }
  e[DEPTH - 1] = page_of(DEPTH - 1);
  for (int it = 0; it < n_it; ++it) {
    if (RT == 1) {
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the reads of the stage that fills next
      asm volatile("" ::: "memory");
      dma(it + DEPTH - 1, e[DEPTH - 1]);
      wait_vm<(DEPTH - 1) * 2 * RPW>();
      asm volatile("" ::: "memory");
    } else {
      wait_vm<(DEPTH - 2) * 2 * RPW>();
      __syncthreads();
      dma(it + DEPTH - 1, e[DEPTH - 1]);
    }
    const int now = e[0];
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d) e[d] = e[d + 1];
    e[DEPTH - 1] = page_of(it + DEPTH);
    if (now >= 0) compute(it);
  }
  wait_vm<0>();
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
  if (r >= n_rows) return;
  const int64_t orow = t * a.Hq + h;
  if (n_eff <= 1) {
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
  } else {
    const int64_t prow = (((int64_t)b * a.N + i_tok) * a.Hq + h) * a.n_split + split;
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
}

// Merge of the splits' partial results, one workgroup per row: every wave finds the
// largest reference with a split per lane, then groups of D/4 lanes take splits in
// turn, four loads in flight each, and meet in LDS.
constexpr int kMergeThreads = 256;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void paged_merge_kernel(PagedArgs a) {
  constexpr int kLanes = D / 4, kGroups = kMergeThreads / kLanes, kFlight = 4;
  __shared__ f32x4 xo[kGroups][kLanes];
  __shared__ float xl[kGroups];
  const int tid = threadIdx.x, grp = tid / kLanes, c = tid % kLanes;
  const int h = blockIdx.x % (unsigned)a.Hq;
  const unsigned item = blockIdx.x / (unsigned)a.Hq;
  const int b = item / (unsigned)a.N, i = item % (unsigned)a.N;
  const int64_t base = a.cu ? a.cu[b] : (int64_t)b * a.N;
  const int m = min(a.cu ? a.cu[b + 1] - a.cu[b] : a.N, a.N);
  if (i >= m) return;
  const Span sp = span_of(a, b, m, i);
  const int n = splits_of(sp);
  if (n <= 1) return;  // written by its one split
  const int64_t orow = (base + i) * a.Hq + h;
  const int64_t prow = (int64_t)blockIdx.x * a.n_split;
  const float* po = a.part_o + prow * D + c * 4;
  const f32x2* ml = (const f32x2*)a.part_ml + prow;
  float top = -1e30f;
  for (int s = tid & 63; s < n; s += 64) top = fmaxf(top, ml[s][0]);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
  f32x4 acc = f32x4{};
  float l = 0.f;
  for (int s0 = grp; s0 < n; s0 += kGroups * kFlight) {
    f32x2 x[kFlight];
    f32x4 y[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {  // (past the last split: that one again, unused)
      const int s = min(s0 + u * kGroups, n - 1);
      x[u] = ml[s];
      y[u] = *(const f32x4*)(po + (int64_t)s * D);
    }
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const float f = s0 + u * kGroups < n ? fast_exp2(x[u][0] - top) : 0.f;
      l += f * x[u][1];
      acc += f * y[u];
    }
  }
  xo[grp][c] = acc;
  if (c == 0) xl[grp] = l;
  __syncthreads();
  if (grp) return;
#pragma unroll
  for (int w = 1; w < kGroups; ++w) {
    acc += xo[w][c];
    l += xl[w];
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *(bf16x4*)(a.out + orow * D + c * 4) = __builtin_convertvector(acc * inv, bf16x4);
  if (a.lse && c == 0) a.lse[orow] = l > 0.f ? (top + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace

hipError_t launch_paged_attn(const PagedArgs& a, int row_tiles, hipStream_t s) {
  const int64_t groups = a.lists ? (int64_t)a.B * a.N : a.B;
  const uint32_t items = (uint32_t)(groups * a.Hkv * a.n_split);
  const dim3 grid((items + 7) / 8 * 8 * (uint32_t)a.n_rowgroups);
#define DA_PAGED(DD, RT, LS)                                                                       \
  hipLaunchKernelGGL((paged_attn_kernel<DD, RT, LS>), grid, dim3(64 * Shape<DD, RT>::NW),          \
                     (Shape<DD, RT>::ldsBytes), s, a, items)
#define DA_PAGED_RT(DD, LS)                                                                        \
  switch (row_tiles) {                                                                             \
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
    if (row_tiles == 8)
      DA_PAGED(128, 8, false);
    else
      DA_PAGED_RT(128, false)
  } else {
    DA_PAGED_RT(64, false)
  }
#undef DA_PAGED_RT
#undef DA_PAGED
  if (a.n_split > 1) {
    const dim3 g((unsigned)((int64_t)a.B * a.N * a.Hq));
    if (a.d == 128)
      hipLaunchKernelGGL(paged_merge_kernel<128>, g, dim3(kMergeThreads), 0, s, a);
    else
      hipLaunchKernelGGL(paged_merge_kernel<64>, g, dim3(kMergeThreads), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace da
