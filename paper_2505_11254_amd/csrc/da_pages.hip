// da_pages.hip -- the pages of a key/value cache: forking, resizing with copy on
// write, appending and compacting (gfx950).
//
// A sequence ("slot") owns a row of the page table, whose first entries name its
// pages; refs[p] counts the slots that name page p.  Every call takes a list of
// requests and behaves as if they were served in the order of the list, so that
// tables, lengths and counts come out the same on every run: ranks come from
// prefix sums over the list, never from the order in which atomics land (they only
// add to counters).  What bounds these kernels is latency where they touch
// integers only, and HBM where they move rows (16 bytes per lane, whole rows).
//
// Nothing on the device is taken on trust that would lead out of bounds: slots,
// lengths and page ids are checked before use, and a request that does not fit is
// refused (its result says so) and leaves its sequence as it was.
#include "da_device.hpp"
#include "da_paged.hpp"

namespace da {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ bool page_ok(int e, int P) { return (unsigned)e < (unsigned)P; }

// Whether request i is the first of the list to name slot s (all threads of the
// workgroup together).
template <int NT>
__device__ __forceinline__ bool first_to_name(const int32_t* list, int i, int s) {
  int seen = 0;
  for (int j = threadIdx.x; j < i; j += NT) seen |= list[j] == s;
  return !__syncthreads_or(seen);
}

__device__ __forceinline__ int pages_of(int tokens) { return (tokens + kPage - 1) / kPage; }

// A count that atomics of this kernel may have changed (they act past the L1 cache).
__device__ __forceinline__ int load_count(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Thread i of n gives back its share of the pages in entries [c0, c1) of slot s.
__device__ __forceinline__ void give_back(const Table& t, int s, int c0, int c1, int i = threadIdx.x,
                                          int n = kThreads) {
  int32_t* const row = t.table + (int64_t)s * t.M;
  for (int c = c0 + i; c < c1; c += n) {
    const int e = row[c];
    if (page_ok(e, t.P)) atomicSub(t.refs + e, 1);
    row[c] = -1;
  }
}

// One request per workgroup: slot dst shares every page of slot src.  Four reads one after
// the other, then all entries at once: 4.8 us for 256 forks of up to 30 pages.
__global__ __launch_bounds__(kThreads) void fork_kernel(Table t, const int32_t* __restrict__ src,
                                                       const int32_t* __restrict__ dst, int n,
                                                       int32_t* __restrict__ result) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int from = src[i], to = dst[i];
  bool ok = (unsigned)from < (unsigned)t.S && (unsigned)to < (unsigned)t.S;
  // (a slot that some request fills is no source, whatever their order: its row
  // is being written)
  int bad = 0;
  for (int j = tid; j < n; j += kThreads) bad |= dst[j] == from || (j < i && dst[j] == to);
  ok = !__syncthreads_or(bad) && ok;
  if (ok) ok = t.lens[to] == 0 && (t.M == 0 || t.table[(int64_t)to * t.M] < 0);
  if (!ok) {
    if (tid == 0) result[i] = -1;
    return;
  }
  const int L = min(max(t.lens[from], 0), t.M * kPage);
  const int pages = pages_of(L);
  const int32_t* a = t.table + (int64_t)from * t.M;
  int32_t* b = t.table + (int64_t)to * t.M;
  __syncthreads();  // (b[0] was read above, by every thread)
  for (int c = tid; c < pages; c += kThreads) {
    const int e = a[c];
    if (page_ok(e, t.P)) {
      atomicAdd(t.refs + e, 1);
      b[c] = e;
    }
  }
  if (tid == 0) {
    t.lens[to] = L;
    result[i] = L;
  }
}

// Freeing, one request per workgroup.
__global__ __launch_bounds__(kThreads) void free_kernel(Table t, const int32_t* __restrict__ slots,
                                                       int32_t* __restrict__ result) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int s = slots[i];
  bool ok = (unsigned)s < (unsigned)t.S;
  ok = first_to_name<kThreads>(slots, i, s) && ok;
  if (ok) {
    const int old = min(max(t.lens[s], 0), t.M * kPage);
    give_back(t, s, 0, pages_of(old));
    __syncthreads();  // (every thread has read the old length)
    if (tid == 0) t.lens[s] = 0;
  }
  if (tid == 0) ((int4*)result)[i] = int4{ok ? 0 : -1, -1, -1, 0};
}

// Inclusive sum over the threads of a workgroup of NT (at most 1024).
template <int NT>
__device__ __forceinline__ int block_scan(int x, int* lds, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_scan_add(x);
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const int y = lds[w];
    before += w < wave ? y : 0;
    all += y;
  }
  *total = all;
  return x + before;
}

// Resizing, one workgroup, a thread per request.  Slots that shrink give back their
// pages first: a thread its own few, the waves those of longer rests.  A thread whose
// slot grows then finds whether the page holding its last token has to be copied (other
// slots hold it too) and how many pages it lacks; a prefix sum over the list gives each
// its ranks among the free pages, which a scan of the reference counts hands out in
// ascending order.  Of the holders of one page that all grow in this call, as many
// copy as there are others left: the last one keeps the page.  Bound by latency, its
// barriers and dependent reads: 5 to 6 us for one or two requests, 11 for 64 that take up to
// a page each, 32 for 256 that copy one (the thread that owns sixteen counts hands out its free
// pages one after the other).
constexpr int kPlanThreads = 1024;
constexpr int kRefsPerThread = 16;
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(Table t, const int32_t* __restrict__ slots,
                                                           const int32_t* __restrict__ new_lens, int n, int32_t* __restrict__ result) {
  __shared__ __attribute__((aligned(16))) int named[kMaxRequests];  // the slots of the requests
  __shared__ __attribute__((aligned(16))) int part[kMaxRequests];   // the page a request would write into, or -1
  __shared__ int cum[kMaxRequests];    // pages that the requests up to this one ask for
  __shared__ int entry[kMaxRequests];  // the entries it holds
  __shared__ int copied[kMaxRequests];  // 1: the last of them is copied, before new ones follow
  __shared__ int scan[kPlanThreads / 64];
  const int i = threadIdx.x;
  int4* const r = (int4*)result + i;
  // Free pages: a bit each for sixteen counts per thread and step.  The first step's are
  // loaded ahead (again after shrinking), all that a pool of 16384 pages needs.
  constexpr int kStep = kPlanThreads * kRefsPerThread;
  // (Plain loads: whether a count is 0 changes by atomics only where slots shrink, and the
  // L1 cache holds no count from before that but the first step's, which an atomic
  // load then fetches again.)
  auto load = [&](int64_t base) -> unsigned {
    typedef int i32x4u __attribute__((ext_vector_type(4), aligned(4)));
    unsigned bits = 0;
    const int64_t p0 = base + i * kRefsPerThread;
    if (p0 + kRefsPerThread <= t.P) {
#pragma unroll
      for (int j = 0; j < kRefsPerThread; j += 4) {
        const i32x4u x = *(const i32x4u*)(t.refs + p0 + j);
        bits |= (unsigned)(x[0] == 0) << j | (unsigned)(x[1] == 0) << (j + 1) | (unsigned)(x[2] == 0) << (j + 2) |
                (unsigned)(x[3] == 0) << (j + 3);
      }
    } else {
      for (int j = 0; j < kRefsPerThread; ++j)
        if (p0 + j < t.P && t.refs[p0 + j] == 0) bits |= 1u << j;
    }
    return bits;
  };
  unsigned bits0 = load(0);
  int s = -1, old = 0, want = -1, pg = -1, holders = 0;
  if (i < n) {
    s = slots[i];
    want = new_lens[i];
  }
  named[i] = s;
  bool valid = (unsigned)s < (unsigned)t.S && want >= 0 && want <= t.M * kPage;
  if (valid) old = min(max(t.lens[s], 0), t.M * kPage);
  __syncthreads();
  // (a wave compares with the requests before its own last; names past n are -1)
  const int n4 = (i & ~63) < n ? min((n + 3) / 4 * 4, (i & ~63) + 64) : 0;
  for (int j = 0; j < n4; j += 4) {
    const int4 x = *(const int4*)(named + j);
    valid &= !((x.x == s && j < i) || (x.y == s && j + 1 < i) || (x.z == s && j + 2 < i) || (x.w == s && j + 3 < i));
  }
  if (i < n && !valid) *r = int4{-1, -1, -1, 0};

  // ---- shrinking
  const bool shrink = valid && want < old;
  const bool shrunk = __syncthreads_or(shrink);
  if (shrunk) {
    constexpr int kOwn = 4;  // pages that a thread gives back itself
    const int c0 = pages_of(want), c1 = pages_of(old);
    if (shrink) t.lens[s] = want;
    if (shrink && c1 - c0 <= kOwn) give_back(t, s, c0, c1, 0, 1);
    entry[i] = c0;
    cum[i] = shrink && c1 - c0 > kOwn ? c1 : 0;
    __syncthreads();
    for (int j = i >> 6; j < n; j += kPlanThreads / 64)
      if (cum[j]) give_back(t, named[j], entry[j], cum[j], i & 63, 64);
    // (counts given back are counts handed out below: by atomics, past this L1)
    __threadfence();
    __syncthreads();
  }

  // ---- growing
  const bool grow = valid && want > old;
  if (grow && old % kPage) {
    pg = t.table[(int64_t)s * t.M + old / kPage];
    if (page_ok(pg, t.P)) holders = load_count(t.refs + pg);
    else pg = -1;
  }
  part[i] = pg;
  int rank = 0;
  if (__syncthreads_or(holders > 1)) {
    for (int j = 0; j < n4; j += 4) {
      const int4 x = *(const int4*)(part + j);
      rank += (x.x == pg && j < i) + (x.y == pg && j + 1 < i) + (x.z == pg && j + 2 < i) + (x.w == pg && j + 3 < i);
    }
  }
  const bool copy = pg >= 0 && holders - rank > 1;
  const int ask = grow ? (copy ? 1 : 0) + pages_of(want) - pages_of(old) : 0;
  // (sums are held at the pool's size: one more page than that is refused anyway)
  int total, upto;
  {
    // a sum of n requests of up to M pages each may pass 31 bits: each is held at the
    // pool's size + 1, in 64-bit sums across the waves (64 of them fit 32 bits inside one
    // where the pool is below 2^25 pages, beyond which a page's bytes pass all memory)
    const int lane = i & 63, wave = i >> 6;
    const int cap = min(t.P, (1 << 25) - 2) + 1;
    const int x = wave_scan_add(min(ask, cap));
    if (lane == 63) scan[wave] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      before += w < wave ? scan[w] : 0;
      all += scan[w];
    }
    upto = (int)min(before + x, (int64_t)cap);
    total = (int)min(all, (int64_t)cap);
    __syncthreads();
  }
  cum[i] = upto;
  entry[i] = pages_of(old);
  copied[i] = copy;

  int avail = 0;
  if (shrunk) {
    bits0 = 0;
    for (int j = 0; j < kRefsPerThread; ++j) {
      const int p = i * kRefsPerThread + j;
      if (p < t.P && load_count(t.refs + p) == 0) bits0 |= 1u << j;
    }
  }
  for (int64_t base = 0; base < t.P && avail < total; base += kStep) {
    int all;
    block_scan<kPlanThreads>(__popc(base ? load(base) : bits0), scan, &all);
    avail += all;
  }
  // Served in order until one does not fit; that one and every later one that
  // grows are refused.
  const bool served = grow && upto <= avail;
  if (i < n) {
    if (served) {
      t.lens[s] = want;
      if (copy) atomicSub(t.refs + pg, 1);
    }
    // (of a copy, the source and its rows; its new page follows below)
    if (valid) *r = int4{grow && !served ? -1 : want, served && copy ? pg : -1, -1, served && copy ? old % kPage : 0};
  }
  __syncthreads();
  int seen = 0;
  // the pages handed out: those asked for by the requests that are served
  int granted;
  {
    const int x = wave_reduce(served ? upto : 0, 0, [](int p, int q) { return max(p, q); });
    __syncthreads();
    if ((i & 63) == 0) scan[i >> 6] = x;
    __syncthreads();
    granted = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) granted = max(granted, scan[w]);
  }
  for (int64_t base = 0; base < t.P && seen < granted; base += kStep) {
    const unsigned bits = base ? load(base) : bits0;
    int all;
    int k = seen + block_scan<kPlanThreads>(__popc(bits), scan, &all) - __popc(bits);
    for (unsigned b = bits; b && k < granted; b &= b - 1, ++k) {
      const int p = (int)base + i * kRefsPerThread + __ffs(b) - 1;
      // the request that rank k falls to: the first whose sum exceeds it
      int lo = 0, hi = n - 1;
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (cum[mid] > k) hi = mid;
        else lo = mid + 1;
      }
      const int before = lo ? cum[lo - 1] : 0;
      int32_t* const row = t.table + (int64_t)slots[lo] * t.M + entry[lo] - copied[lo];
      row[k - before] = p;
      if (copied[lo] && k == before) result[4 * lo + 2] = p;
      t.refs[p] = 1;
    }
    seen += all;
  }
}

// Second launch: the rows of the copied pages, a workgroup per (request, layer, keys
// or values, `heads` kv heads), and of codes their scales.  Bound by HBM: 256 pages of 16 layers, 8 kv heads, d 128,
// 1.18 GB read and written in 190 to 208 us, 5.7 to 6.2 TB/s.
__global__ __launch_bounds__(kThreads) void copy_kernel(Pages p, int P, const int32_t* __restrict__ result,
                                                       int n, int heads) {
  unsigned b = blockIdx.x;
  const int i = b % (unsigned)n;
  const int4 r = ((const int4*)result)[i];
  if (r.y < 0 || r.z < 0) return;
  b /= (unsigned)n;
  const int groups = p.Hkv / heads, h0 = b % (unsigned)groups * heads;
  b /= (unsigned)groups;
  uint16_t* const base = (b & 1) ? p.v : p.k;
  const int64_t layer = b >> 1;
  const int64_t head = (int64_t)kPage * p.d;
  const int chunks = r.w * (p.d / 8);
  for (int h = h0; h < h0 + heads; ++h) {
    const u32x4* const from = (const u32x4*)(base + ((layer * P + r.y) * p.Hkv + h) * head);
    u32x4* const to = (u32x4*)(base + ((layer * P + r.z) * p.Hkv + h) * head);
    for (int c = threadIdx.x; c < chunks; c += kThreads) to[c] = from[c];
  }
  if (p.k_scales && (int)threadIdx.x < heads) {
    float* const s = ((b & 1) ? p.v_scales : p.k_scales) + h0 + threadIdx.x;
    s[(layer * P + r.z) * p.Hkv] = s[(layer * P + r.y) * p.Hkv];
  }
}

// New tokens become the last ones of their sequences: each thread moves 16 bytes
// of keys or values.  A workgroup takes kAppendChunks of one sequence, if its slot has the length
// asked for (one that did not get it holds old tokens where the new ones belong).  Bound by HBM: 87302
// tokens of 8 kv heads, d 128, 0.72 GB read and written in 122 us, 5.9 TB/s.
constexpr int kAppendPer = 4;
constexpr int kAppendChunks = kThreads * kAppendPer;
__global__ __launch_bounds__(kThreads) void append_kernel(Table t, Pages p, const uint16_t* __restrict__ k,
                                                         const uint16_t* __restrict__ v, int64_t T,
                                                         const int32_t* __restrict__ slots,
                                                         const int32_t* __restrict__ cu, int B, int N,
                                                         const int32_t* __restrict__ new_lens) {
  const int b = blockIdx.x % (unsigned)B;
  const unsigned part = blockIdx.x / (unsigned)B;
  const int64_t layer = blockIdx.y >> 1;
  const uint16_t* const src = ((blockIdx.y & 1) ? v : k) + layer * T * p.Hkv * p.d;
  uint16_t* const dst = ((blockIdx.y & 1) ? p.v : p.k) + layer * t.P * p.Hkv * (int64_t)kPage * p.d;
  const int64_t base = cu ? cu[b] : (int64_t)b * N;
  const int m = min(cu ? cu[b + 1] - cu[b] : N, N);
  const int s = slots ? slots[b] : b;
  if ((unsigned)s >= (unsigned)t.S || m <= 0 || base < 0 || base + m > T) return;
  const int per_head = p.d / 8;
  const int row = p.Hkv * per_head;  // chunks per token
  const unsigned chunks = (unsigned)m * row;  // (the host has checked that N tokens' fit)
  if (part * kAppendChunks >= chunks) return;
  const int len = t.lens[s], pos0 = len - m;
  if (new_lens && len != new_lens[b]) return;
  // (in phases, so that the loads of a thread's chunks are under way together)
  int64_t at[kAppendPer];  // (a page of 2^18 kv heads passes 2^31 elements)
  int e[kAppendPer];
  u32x4 x[kAppendPer];
#pragma unroll
  for (int j = 0; j < kAppendPer; ++j) {
    const unsigned c = part * kAppendChunks + j * kThreads + threadIdx.x;
    const int i = min(c, chunks - 1) / (unsigned)row, w = min(c, chunks - 1) % (unsigned)row;
    const int pos = pos0 + i;
    const bool inside = c < chunks && pos >= 0 && pos < t.M * kPage;
    e[j] = inside ? t.table[(int64_t)s * t.M + pos / kPage] : -1;
    x[j] = *(const u32x4*)(src + (base + i) * (int64_t)p.Hkv * p.d + w * 8);
    at[j] = (int64_t)(w / per_head * kPage + pos % kPage) * p.d + w % per_head * 8;
  }
#pragma unroll
  for (int j = 0; j < kAppendPer; ++j)
    if (page_ok(e[j], t.P)) *(u32x4*)(dst + (int64_t)e[j] * p.Hkv * kPage * p.d + at[j]) = x[j];
}

// Compacting, first launch, one request per workgroup: checks the kept places
// (ascending, inside the sequence, no shared page to be written) and sets the new
// length.  result[i] = {tokens kept, or -1: refused; the first that moves; the old
// length; 0}.
__global__ __launch_bounds__(kThreads) void compact_check_kernel(
    Table t, const int32_t* __restrict__ slots, const int32_t* __restrict__ start,
    const int32_t* __restrict__ keep, int64_t n_keep, const int32_t* __restrict__ cu_keep,
    int32_t* __restrict__ result) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int s = slots[i], st = start[i];
  const int64_t k0 = cu_keep[i], k1 = cu_keep[i + 1];
  int4* const r = (int4*)result + i;
  bool ok = (unsigned)s < (unsigned)t.S && st >= 0 && k0 >= 0 && k1 >= k0 && k1 <= n_keep;
  ok = first_to_name<kThreads>(slots, i, s) && ok;
  int len = 0;
  if (ok) {
    len = min(max(t.lens[s], 0), t.M * kPage);
    ok = st <= len && k1 - k0 <= len - st;
  }
  if (!ok) {
    if (tid == 0) *r = int4{-1, 0, 0, 0};
    return;
  }
  const int m = (int)(k1 - k0);
  int bad = 0, moved = m;  // the first place of this thread's that moves
  for (int j = tid; j < m; j += kThreads) {
    const int x = keep[k0 + j];
    bad |= x < j || x >= len - st || (j > 0 && keep[k0 + j - 1] >= x);
    if (x != j) moved = min(moved, j);
  }
  __shared__ int least;
  if (tid == 0) least = m;
  bad = __syncthreads_or(bad);
  if (!bad && moved < m) atomicMin(&least, moved);
  __syncthreads();
  const int j0 = least;
  if (!bad && j0 < m) {
    const int32_t* row = t.table + (int64_t)s * t.M;
    for (int c = (st + j0) / kPage + tid; c <= (st + m - 1) / kPage; c += kThreads) {
      const int e = row[c];
      bad |= !page_ok(e, t.P) || t.refs[e] > 1;
    }
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    *r = bad ? int4{-1, 0, 0, 0} : int4{m, j0, len, 0};
    if (!bad) t.lens[s] = st + m;
  }
}

// Second launch: a workgroup per (request, layer, keys or values, HB kv heads) moves
// its rows up, kSteps steps at a time, each of the rows that the workgroup holds.
// Kept places ascend, so a row never moves down and a batch's rows are all read before
// any of them, or of a later batch's sources, can be written over.  Bound by latency where
// a few tokens move: 64 requests of 16 drafts, 4 layers, 8 kv heads 7 us, and 4 for the check.
constexpr int kMoveSteps = 8;
template <int HB>
__global__ __launch_bounds__(kThreads) void compact_kernel(Table t, Pages p, const int32_t* __restrict__ slots,
                                                          const int32_t* __restrict__ start,
                                                          const int32_t* __restrict__ keep,
                                                          const int32_t* __restrict__ cu_keep, int n,
                                                          int32_t* __restrict__ result) {
  unsigned b = blockIdx.x;
  const int i = b % (unsigned)n;
  b /= (unsigned)n;
  const int4 r = ((const int4*)result)[i];
  const int st = start[i], slot = slots[i];
  const int32_t* const kp = keep + cu_keep[i];
  if (r.x < 0) return;  // refused
  const int32_t* const row = t.table + (int64_t)slot * t.M;
  const int per = p.d / 8;                // 16-byte chunks per row
  const int rows = kThreads / per / HB;   // rows per step of the workgroup
  const int j_in = threadIdx.x / (per * HB), c = threadIdx.x % per;
  const int groups = p.Hkv / HB, h = b % (unsigned)groups * HB + threadIdx.x / per % HB;
  b /= (unsigned)groups;
  const int64_t layer = b >> 1;
  uint16_t* const base = ((b & 1) ? p.v : p.k) + (layer * t.P * p.Hkv + h) * (int64_t)kPage * p.d + c * 8;
  const int64_t page = (int64_t)p.Hkv * kPage * p.d;
  for (int j0 = r.y; j0 < r.x; j0 += kMoveSteps * rows) {
    u32x4 x[kMoveSteps];
    int from[kMoveSteps], e[kMoveSteps], to[kMoveSteps];
    // (in phases, so that the loads of a thread's rows are under way together; whole steps
    // past the last row are left out)
#pragma unroll
    for (int u = 0; u < kMoveSteps; ++u) {
      if (j0 + u * rows >= r.x) break;
      const int j = min(j0 + u * rows + j_in, r.x - 1);
      from[u] = st + kp[j];
      to[u] = row[(st + j) / kPage];
    }
#pragma unroll
    for (int u = 0; u < kMoveSteps; ++u) {
      if (j0 + u * rows >= r.x) break;
      e[u] = row[from[u] / kPage];
    }
#pragma unroll
    for (int u = 0; u < kMoveSteps; ++u) {
      if (j0 + u * rows >= r.x) break;
      x[u] = page_ok(e[u], t.P) ? *(const u32x4*)(base + e[u] * page + (from[u] % kPage) * p.d) : u32x4{};
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMoveSteps; ++u) {
      const int j = j0 + u * rows + j_in;
      if (j < r.x) *(u32x4*)(base + to[u] * page + ((st + j) % kPage) * p.d) = x[u];
    }
    __syncthreads();
  }
  // The last of a request's workgroups, which all have read the table by then, gives
  // back the pages past the new end (result[i].w counts them from 0).
  const int c0 = pages_of(st + r.x), c1 = pages_of(r.z);
  if (c0 >= c1) return;
  __shared__ int left;
  __syncthreads();
  if (threadIdx.x == 0) left = p.layers * 2 * groups - 1 - atomicAdd(result + 4 * i + 3, 1);
  __syncthreads();
  if (left == 0) give_back(t, slot, c0, c1);
}

// Kv heads that a workgroup takes: one where that makes few workgroups, up to four where
// it makes more than a few per CU, most of which would come and go without work.
int heads_together(int n, const Pages& p) {
  const int64_t wgs = (int64_t)n * p.layers * 2 * p.Hkv;
  return wgs > 4096 && p.Hkv % 4 == 0 ? 4 : wgs > 2048 && p.Hkv % 2 == 0 ? 2 : 1;
}

}  // namespace

hipError_t launch_pages_fork(const Table& t, const int32_t* src, const int32_t* dst, int n,
                             int32_t* result, hipStream_t s) {
  hipLaunchKernelGGL(fork_kernel, dim3(n), dim3(kThreads), 0, s, t, src, dst, n, result);
  return hipGetLastError();
}

hipError_t launch_pages_resize(const Table& t, const Pages& p, const int32_t* slots,
                               const int32_t* new_lens, int n, int32_t* result, hipStream_t s) {
  if (!new_lens) {
    hipLaunchKernelGGL(free_kernel, dim3(n), dim3(kThreads), 0, s, t, slots, result);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, t, slots, new_lens, n, result);
  const int heads = heads_together(n, p);
  hipLaunchKernelGGL(copy_kernel, dim3((unsigned)(n * p.layers * 2 * (p.Hkv / heads))), dim3(kThreads), 0, s, p,
                     t.P, result, n, heads);
  return hipGetLastError();
}

hipError_t launch_pages_append(const Table& t, const Pages& p, const uint16_t* k,
                               const uint16_t* v, int64_t T, const int32_t* slots,
                               const int32_t* cu, int B, int N, const int32_t* new_lens, hipStream_t s) {
  const int64_t chunks = (int64_t)N * p.Hkv * (p.d / 8);
  const int64_t parts = (chunks + kAppendChunks - 1) / kAppendChunks;
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)(parts * B), p.layers * 2), dim3(kThreads), 0, s, t, p, k,
                     v, T, slots, cu, B, N, new_lens);
  return hipGetLastError();
}

hipError_t launch_compact_check(const Table& t, const int32_t* slots, const int32_t* start, const int32_t* keep,
                                int64_t n_keep, const int32_t* cu_keep, int n, int32_t* result, hipStream_t s) {
  hipLaunchKernelGGL(compact_check_kernel, dim3(n), dim3(kThreads), 0, s, t, slots, start, keep, n_keep,
                     cu_keep, result);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const Table& t, const Pages& p, const int32_t* slots,
                                const int32_t* start, const int32_t* keep, int64_t n_keep,
                                const int32_t* cu_keep, int n, int32_t* result, hipStream_t s) {
  const hipError_t e = launch_compact_check(t, slots, start, keep, n_keep, cu_keep, n, result, s);
  if (e != hipSuccess) return e;
  const int heads = heads_together(n, p);
  const dim3 grid((unsigned)(n * p.layers * 2 * (p.Hkv / heads)));
#define DA_COMPACT(HB)                                                                             \
  hipLaunchKernelGGL(compact_kernel<HB>, grid, dim3(kThreads), 0, s, t, p, slots, start, keep,     \
                     cu_keep, n, result)
  if (heads == 4)
    DA_COMPACT(4);
  else if (heads == 2)
    DA_COMPACT(2);
  else
    DA_COMPACT(1);
#undef DA_COMPACT
  return hipGetLastError();
}

}  // namespace da
