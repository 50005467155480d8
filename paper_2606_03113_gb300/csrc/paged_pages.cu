// paged_pages.cu -- the pages of a paged KV cache: reserved, copied on write, forked, given back,
// compacted, and rows appended to them.
//
// us on the GPU: a reserve that finds its pages there 4.2 (two launches), a fork 1.5 to 3.6, a step of
// 64 sequences with 24 copies of 5.2 MB 39.6 (6.2 TB/s), 100 pages of 5.2 MB moved by a compaction 172
// (6.1 TB/s), 2047 rows of 40 heads appended 14.6 a call (5.8 TB/s), 16 rows of 8 heads 2.2.
//
// Which page goes where is whole-number work on a table and a few counts, bound by round trips of
// memory (a table entry, its page's count) and not by bytes; what is moved is bound by bytes. So one
// block plans (its barriers order the steps that have to see each other's counts) and
// leaves a list of copies in the workspace, and all SMs carry it out in a second launch, which
// is resident by then (programmatic dependence). Every result is independent of the order in which
// threads run: sums of whole numbers, maxima, and ranks counted in the order of ids or of
// (sequence, position).
#include "paged.cuh"

#include <cuda_runtime.h>

namespace ssd {

namespace {

constexpr int kScan = 16;    // counts of a thread in a pass over refs
constexpr int kHeld = 2048;  // entries of a reserve that stay in registers
constexpr int kClaim = 1 << 16;  // refs while a reserve looks: entries below, claims above
constexpr int kCopyThreads = 256;
constexpr int kForkCols = 8;     // entries of a sequence that a fork's block looks at: a sector

// The plan's scratch: what the second launch does.
struct __align__(16) Copy {
  int32_t src, dst, rows, pad;  // the first `rows` positions of every slab
};
struct PlanHead {
  int32_t copies, low;  // entries of the list; (compact) pages in use
};
struct PlanWork {
  PlanHead* head;
  Copy* list;                // [n_pages]
  int32_t *a, *fresh, *old;  // [n_pages] each
};
constexpr size_t kHeadBytes = 256;
size_t plan_bytes(int n_pages) { return kHeadBytes + (size_t)n_pages * (sizeof(Copy) + 3 * 4); }
PlanWork plan_work(void* p, int n_pages) {
  char* c = static_cast<char*>(p);
  PlanWork w;
  w.head = reinterpret_cast<PlanHead*>(c);
  w.list = reinterpret_cast<Copy*>(c + kHeadBytes);
  w.a = reinterpret_cast<int32_t*>(w.list + n_pages);
  w.fresh = w.a + n_pages;
  w.old = w.fresh + n_pages;
  return w;
}

struct PlanSmem {
  int warp[32];
};

// Sum of v over the threads before this one, of WARPS warps; `total` of all. Two barriers.
template <int WARPS>
__device__ __forceinline__ int before_me(int v, PlanSmem& sm, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  __syncthreads();  // the sums of the call before have been read
  if (lane == 31) sm.warp[warp] = inc;
  __syncthreads();
  int sums = lane < WARPS ? sm.warp[lane] : 0;  // every warp adds up the warps' sums
#pragma unroll
  for (int o = 1; o < WARPS; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, sums, o);
    if (lane >= o) sums += u;
  }
  total = __shfl_sync(0xffffffffu, sums, WARPS - 1);
  const int base = __shfl_sync(0xffffffffu, sums, warp > 0 ? warp - 1 : 0);
  return (warp > 0 ? base : 0) + inc - v;
}

// The kScan counts from id0 on (1 behind the pool's end: not free).
__device__ __forceinline__ void load_refs(const PagedView& c, int id0, int (&r)[kScan]) {
#pragma unroll
  for (int j = 0; j < kScan; j += 4) {
    int4 v = make_int4(1, 1, 1, 1);
    if (id0 + j + 3 < c.n_pages) {
      v = __ldcg(reinterpret_cast<const int4*>(c.refs + id0 + j));
    } else {
      if (id0 + j < c.n_pages) v.x = __ldcg(c.refs + id0 + j);
      if (id0 + j + 1 < c.n_pages) v.y = __ldcg(c.refs + id0 + j + 1);
      if (id0 + j + 2 < c.n_pages) v.z = __ldcg(c.refs + id0 + j + 2);
    }
    r[j] = v.x, r[j + 1] = v.y, r[j + 2] = v.z, r[j + 3] = v.w;
  }
}

}  // namespace

// Steps of a reserve, each behind a barrier:
//  1 every wanted entry whose page has other names claims it (counted above the names, so that
//    who else has claimed does not matter for who is sharing);
//  2 where all names claim, the largest sequence is found, which keeps the page;
//  3 the entries that need a page are counted and as many free pages found, lowest first;
//  4 (too few: the claims are taken back) entries get theirs by rank, the list of copies is written,
//    the counts follow.
// One block, bound by round trips to L2: three where nothing is needed (positions, entries, counts), a pass
// over the counts for free pages, two more for shared ones. Up to kHeld wanted entries, as a decode step
// has them, stay in registers from step to step; more are looked at again in each.
template <int TH>
__global__ void __launch_bounds__(TH, 1) k_paged_reserve(const PagedView c, const PlanWork w,
                                                      const int32_t* pos, const int32_t* rows, int M,
                                                      int32_t* err) {
  constexpr int kWarps = TH / 32, kScanStep = TH * kScan;  // counts of a pass
  __shared__ PlanSmem sm;
  __shared__ int s_pre[SSD_KV8_MAX_SEQS + 1];  // wanted entries of the sequences before
  __shared__ int s_pos[SSD_KV8_MAX_SEQS];
  __shared__ int s_fresh[kHeld];
  __shared__ int s_copies;
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x;
  // sequences tid per .. (tid + 1) per - 1 are this thread's
  const int per = (c.n_seq + TH - 1) / TH;
  int sum = 0;
  for (int j = 0; j < per; ++j) {
    const int b = tid * per + j;
    if (b >= c.n_seq) break;
    const int p = pos[b], n = rows ? rows[b] : M;
    int cnt = 0;
    if (p < 0 || n < 0 || n > M || p > c.cap() - n) {
      if (err) atomicOr(err, n < 0 || n > M ? (int)kErrControl : (int)kErrCapacity);
    } else if (n > 0) {
      cnt = ((p + n - 1) >> c.shift) - (p >> c.shift) + 1;
    }
    s_pos[b] = p;
    s_pre[b] = sum;  // (of this thread's, for now)
    sum += cnt;
  }
  if (tid == 0) s_copies = 0;
  int E;
  const int at = before_me<kWarps>(sum, sm, E);
  for (int j = 0; j < per && tid * per + j < c.n_seq; ++j) s_pre[tid * per + j] += at;
  if (tid == 0) s_pre[c.n_seq] = E;
  __syncthreads();
  // wanted entry x: its sequence and place in the table
  auto find = [&](int x, int& b, int& i) {
    int lo = 0, hi = c.n_seq - 1;  // the last sequence that begins at x or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_pre[mid] <= x) lo = mid;
      else hi = mid - 1;
    }
    b = lo;
    i = (s_pos[b] >> c.shift) + x - s_pre[b];
  };
  auto entry = [&](int b, int i) {
    const int e = __ldcg(c.table + (size_t)b * c.max_pages + i);
    return (unsigned)e < (unsigned)c.n_pages ? e : -1;
  };
  auto all_claim = [&](int v) { return (v >> 16) == (v & (kClaim - 1)); };
  // as many free pages as are needed, lowest first; how many were found
  auto find_free = [&](int need, int32_t* fresh) {
    int found = 0;
    for (int id0 = 0; id0 < c.n_pages && found < need; id0 += kScanStep) {
      int r[kScan], n = 0, total;
      load_refs(c, id0 + tid * kScan, r);
#pragma unroll
      for (int j = 0; j < kScan; ++j) n += r[j] == 0;
      int rank = found + before_me<kWarps>(n, sm, total);
#pragma unroll
      for (int j = 0; j < kScan; ++j)
        if (r[j] == 0) {
          if (rank < need) fresh[rank] = id0 + tid * kScan + j;
          ++rank;
        }
      found += total;
    }
    __syncthreads();
    return found;
  };
  // entry i of sequence b gets page `to`; the page that it leaves is `from` (-1: none)
  auto give = [&](int b, int i, int from, int to) {
    c.table[(size_t)b * c.max_pages + i] = to;
    const int kept = s_pos[b] - (i << c.shift);  // positive in a sequence's first entry alone
    if (from >= 0 && kept > 0) w.list[atomicAdd(&s_copies, 1)] = Copy{from, to, kept, 0};
  };

  if (E <= kHeld) {
    constexpr int K = kHeld / TH;
    const int each = (E + TH - 1) / TH;  // entries tid each .. are this thread's
    int eb[K], ei[K], ee[K];
    bool wanted[K], shared[K], all[K];
    int claims = 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int x = tid * each + k;
      eb[k] = ei[k] = 0, ee[k] = -1;
      wanted[k] = k < each && x < E;
      if (!wanted[k]) continue;
      if (k == 0) {
        find(x, eb[0], ei[0]);
      } else {
        eb[k] = eb[k - 1];
        while (s_pre[eb[k] + 1] <= x) ++eb[k];
        ei[k] = (s_pos[eb[k]] >> c.shift) + x - s_pre[eb[k]];
      }
      ee[k] = entry(eb[k], ei[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      shared[k] = ee[k] >= 0 && (__ldcg(c.refs + ee[k]) & (kClaim - 1)) > 1;
      all[k] = false;
      if (shared[k]) {
        atomicAdd(c.refs + ee[k], kClaim);
        w.a[ee[k]] = 0;
        claims = 1;
      }
    }
    if (__syncthreads_or(claims)) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (shared[k]) {
          all[k] = all_claim(__ldcg(c.refs + ee[k]));
          if (all[k]) atomicMax(w.a + ee[k], eb[k] + 1);
        }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k)  // whether the entry keeps a page that all claim
        all[k] = all[k] && __ldcg(w.a + ee[k]) == eb[k] + 1;
    }
    int mine = 0, need;
    bool needs[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      needs[k] = wanted[k] && (ee[k] < 0 || (shared[k] && !all[k]));
      mine += needs[k];
    }
    int rank = before_me<kWarps>(mine, sm, need);
    const bool enough = need == 0 || find_free(need, s_fresh) >= need;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (enough && needs[k]) {
        const int to = s_fresh[rank++];
        give(eb[k], ei[k], shared[k] ? ee[k] : -1, to);
        c.refs[to] = 1;
      }
      if (shared[k]) atomicSub(c.refs + ee[k], kClaim + (enough && needs[k]));
    }
    __syncthreads();
    if (tid == 0) {
      w.head->copies = s_copies;
      if (!enough && err) atomicOr(err, (int)kErrPages);
    }
    return;
  }

  int claims = 0;
  for (int x = tid; x < E; x += TH) {
    int b, i;
    find(x, b, i);
    const int e = entry(b, i);
    if (e >= 0 && (__ldcg(c.refs + e) & (kClaim - 1)) > 1) {
      atomicAdd(c.refs + e, kClaim);
      w.a[e] = 0;
      claims = 1;
    }
  }
  const bool any = __syncthreads_or(claims);
  if (any) {
    for (int x = tid; x < E; x += TH) {
      int b, i;
      find(x, b, i);
      const int e = entry(b, i);
      if (e < 0) continue;
      const int v = __ldcg(c.refs + e);
      if ((v & (kClaim - 1)) > 1 && all_claim(v)) atomicMax(w.a + e, b + 1);
    }
    __syncthreads();
  }
  // whether the entry needs a page; `from`: the page that it leaves, or -1
  auto needs = [&](int b, int e, int& from) {
    from = -1;
    if (e < 0) return true;
    if (!any) return false;
    const int v = __ldcg(c.refs + e);
    if ((v & (kClaim - 1)) <= 1) return false;
    if (all_claim(v) && __ldcg(w.a + e) == b + 1) return false;
    from = e;
    return true;
  };
  int need = 0;
  for (int x0 = 0; x0 < E; x0 += TH) {
    int mine = 0;
    if (x0 + tid < E) {
      int b, i, from;
      find(x0 + tid, b, i);
      mine = needs(b, entry(b, i), from);
    }
    need += __syncthreads_count(mine);
  }
  if (find_free(need, w.fresh) < need) {
    for (int x = tid; x < E; x += TH) {
      int b, i;
      find(x, b, i);
      const int e = entry(b, i);
      // (the names alone tell who claimed: they have not changed)
      if (e >= 0 && (__ldcg(c.refs + e) & (kClaim - 1)) > 1) atomicSub(c.refs + e, kClaim);
    }
    if (tid == 0) {
      w.head->copies = 0;
      if (err) atomicOr(err, (int)kErrPages);
    }
    return;
  }
  int base = 0;
  for (int x0 = 0; x0 < E && need > 0; x0 += TH) {
    int b = 0, i = 0, from = -1, total;
    bool mine = false;
    if (x0 + tid < E) {
      find(x0 + tid, b, i);
      mine = needs(b, entry(b, i), from);
    }
    const int rank = base + before_me<kWarps>(mine, sm, total);
    base += total;
    if (mine) {
      give(b, i, from, __ldcg(w.fresh + rank));
      w.old[rank] = from;
    }
  }
  __syncthreads();
  for (int k = tid; k < need; k += TH) {
    c.refs[__ldcg(w.fresh + k)] = 1;
    const int from = __ldcg(w.old + k);
    if (from >= 0) atomicSub(c.refs + from, kClaim + 1);
  }
  if (any) {  // the claims of those who keep a page, which their entries still name
    __syncthreads();
    for (int x = tid; x < E; x += TH) {
      int b, i;
      find(x, b, i);
      const int e = entry(b, i);
      if (e >= 0 && __ldcg(c.refs + e) >> 16) atomicAnd(c.refs + e, kClaim - 1);
    }
  }
  if (tid == 0) w.head->copies = s_copies;
}

// Carries out a list of copies: a warp a slab, so that all SMs have many lines on their way; the next
// slab's entry of the list is looked up beside the copy.
__device__ __forceinline__ void copy_pages(const PagedView& c, const PlanWork& w, int copies) {
  const int lane = threadIdx.x & 31;
  const int64_t units = (int64_t)copies * c.slabs;
  const int64_t step = (int64_t)gridDim.x * (kCopyThreads / 32);
  const int row_shift = 31 - __clz(c.slab) - c.shift - 4;  // 16-byte chunks of a row
  int64_t u = (int64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5);
  int s = 0;
  int4 next = make_int4(0, 0, 0, 0);
  auto look = [&]() {
    if (u < units) {
      const int k = units <= 0x7fffffff ? (int)((uint32_t)u / (uint32_t)c.slabs) : (int)(u / c.slabs);
      s = (int)(u - (int64_t)k * c.slabs);
      next = __ldcg(reinterpret_cast<const int4*>(w.list + k));
    }
  };
  look();
  while (u < units) {
    const int4 d = next;
    const uint4* src = reinterpret_cast<const uint4*>(c.pages + d.x * c.bytes + (size_t)s * c.slab);
    uint4* dst = reinterpret_cast<uint4*>(c.pages + d.y * c.bytes + (size_t)s * c.slab);
    u += step;
    look();
    const int n = d.z << row_shift;
    for (int x0 = lane; x0 < n; x0 += 8 * 32) {
      uint4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (x0 + j * 32 < n) v[j] = __ldcs(src + x0 + j * 32);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (x0 + j * 32 < n) __stcs(dst + x0 + j * 32, v[j]);
    }
  }
}

__global__ void __launch_bounds__(kCopyThreads) k_paged_copy(const PagedView c, const PlanWork w) {
  pdl_wait();
  copy_pages(c, w, __ldcg(&w.head->copies));
}

// One block: pages in use are counted, then holes below that number and pages above it are
// listed in the order of their ids.
template <int TH>
__global__ void __launch_bounds__(TH, 1) k_paged_compact(const PagedView c, const PlanWork w,
                                                                int32_t* used) {
  constexpr int kWarps = TH / 32, kScanStep = TH * kScan;
  __shared__ PlanSmem sm;
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x;
  int n = 0, low, r[kScan];
  for (int id0 = 0; id0 < c.n_pages; id0 += kScanStep) {
    load_refs(c, id0 + tid * kScan, r);
#pragma unroll
    for (int j = 0; j < kScan; ++j) n += r[j] != 0 && id0 + tid * kScan + j < c.n_pages;
  }
  before_me<kWarps>(n, sm, low);
  int holes = 0, moved = 0;
  for (int id0 = 0; id0 < c.n_pages; id0 += kScanStep) {
    int mine = 0, total;
    const int first = id0 + tid * kScan;
    if (c.n_pages > kScanStep) load_refs(c, first, r);  // (one pass: they are here)
#pragma unroll
    for (int j = 0; j < kScan; ++j) {
      const bool in = first + j < c.n_pages, below = first + j < low;
      mine += in && below && r[j] == 0 ? 1 : 0;
      mine += in && !below && r[j] != 0 ? 1 << 16 : 0;
    }
    const int rank = before_me<kWarps>(mine, sm, total);  // (at most kScanStep of each: 15 bits)
    int h = holes + (rank & 0xffff), m = moved + (rank >> 16);
#pragma unroll
    for (int j = 0; j < kScan; ++j) {
      const bool in = first + j < c.n_pages, below = first + j < low;
      if (in && below && r[j] == 0) w.fresh[h++] = first + j;
      if (in && !below) {
        if (r[j] != 0) w.old[m++] = first + j;
        else w.a[first + j] = -1;
      }
    }
    holes += total & 0xffff;
    moved += total >> 16;
  }
  __syncthreads();
  for (int k = tid; k < moved; k += TH) {
    const int from = __ldcg(w.old + k), to = __ldcg(w.fresh + k);
    w.a[from] = to;
    w.list[k] = Copy{from, to, 1 << c.shift, 0};
    c.refs[to] = __ldcg(c.refs + from);
    c.refs[from] = 0;
  }
  if (tid == 0) {
    w.head->copies = moved;
    w.head->low = low;
    if (used) *used = low;
  }
}

__global__ void __launch_bounds__(kCopyThreads) k_paged_move(const PagedView c, const PlanWork w) {
  pdl_wait();
  const int copies = __ldcg(&w.head->copies), low = __ldcg(&w.head->low);
  if (copies) {
    const int64_t n = (int64_t)c.n_seq * c.max_pages;
    for (int64_t x = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; x < n;
         x += (int64_t)gridDim.x * kCopyThreads) {
      const int e = c.table[x];
      if (e >= low && e < c.n_pages) c.table[x] = __ldcg(w.a + e);
    }
  }
  copy_pages(c, w, copies);
}

// Entry i of the new table depends on the entries i of the old one alone, so a block takes
// kForkCols entries of all sequences, reads them, and writes them behind a barrier: no second table,
// no second launch. Counts change by atomic sums, for entries that change.
__global__ void __launch_bounds__(kCopyThreads) k_paged_fork(const PagedView c,
                                                             const int32_t* parent,
                                                             const int32_t* length, int32_t* err) {
  extern __shared__ int s_old[];  // [n_seq][kForkCols]
  pdl_wait();
  const int c0 = blockIdx.x * kForkCols;
  for (int x = threadIdx.x; x < c.n_seq * kForkCols; x += kCopyThreads) {
    const int b = x / kForkCols, i = c0 + x % kForkCols;
    s_old[x] = i < c.max_pages ? c.table[(size_t)b * c.max_pages + i] : -1;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < c.n_seq * kForkCols; x += kCopyThreads) {
    const int b = x / kForkCols, i = c0 + x % kForkCols;
    if (i >= c.max_pages) continue;
    const int p = parent ? parent[b] : b, n = length ? length[b] : 0x7fffffff;
    if (p < -1 || p >= c.n_seq || n < 0) {
      if (i == 0 && err) atomicOr(err, (int)kErrControl);
      continue;
    }
    const int was = s_old[x];
    int now = p >= 0 && ((int64_t)i << c.shift) < n ? s_old[p * kForkCols + x % kForkCols] : -1;
    if ((unsigned)now >= (unsigned)c.n_pages) now = -1;
    if (now == was) continue;
    c.table[(size_t)b * c.max_pages + i] = now;
    if (now >= 0) atomicAdd(c.refs + now, 1);
    if ((unsigned)was < (unsigned)c.n_pages) atomicSub(c.refs + was, 1);
  }
}

// ------------------------------------------------------------- append

namespace {

constexpr int kRowThreads = 128;
constexpr int kRowBatch = 5;  // 16-byte chunks of K and of V that a thread has on their way

struct PagedAppend {
  PagedView c;
  const char *k, *v;
  int64_t stride;  // bytes between rows
  size_t to_k, to_v;  // layer's K and V in a page
  int32_t chunks;  // 16-byte chunks of a row
  int32_t head_shift;  // log2 of those of a head
  const int32_t *pos, *rows;
  int32_t* err;
  int32_t M;
};

}  // namespace

// A block a row: its K and V are on their way while the table entry and the page's count are looked up,
// one after the other (a row is not written to a page that others name).
__global__ void __launch_bounds__(kRowThreads) k_paged_append(const PagedAppend a) {
  pdl_wait();
  const int m = blockIdx.x, b = blockIdx.y;
  const uint4* xk = reinterpret_cast<const uint4*>(a.k + ((int64_t)b * a.M + m) * a.stride);
  const uint4* xv = reinterpret_cast<const uint4*>(a.v + ((int64_t)b * a.M + m) * a.stride);
  const int p0 = a.pos[b], n = a.rows ? a.rows[b] : a.M;
  uint4 uk[kRowBatch], uv[kRowBatch];
  auto load = [&](int x0) {
#pragma unroll
    for (int j = 0; j < kRowBatch; ++j) {
      const int x = x0 + j * kRowThreads;
      if (x < a.chunks) {
        uk[j] = __ldcs(xk + x);
        uv[j] = __ldcs(xv + x);
      }
    }
  };
  if (p0 < 0 || n < 0 || n > a.M || p0 > a.c.cap() - n) {
    if (threadIdx.x == 0 && m == 0 && a.err)
      atomicOr(a.err, n < 0 || n > a.M ? (int)kErrControl : (int)kErrCapacity);
    return;
  }
  if (m >= n) return;
  load(threadIdx.x);
  const int p = p0 + m, e = a.c.entry(b, p >> a.c.shift);
  if (e < 0 || a.c.refs[e] > 1) {
    if (threadIdx.x == 0 && a.err) atomicOr(a.err, (int)kErrTable);
    return;
  }
  const int slot = p & ((1 << a.c.shift) - 1);
  char* const page = a.c.pages + e * a.c.bytes;
  for (int x0 = threadIdx.x;;) {
#pragma unroll
    for (int j = 0; j < kRowBatch; ++j) {
      const int x = x0 + j * kRowThreads, h = x >> a.head_shift;
      if (x < a.chunks) {
        const size_t off = h * a.c.head() +
                           ((size_t)((slot << a.head_shift) + (x - (h << a.head_shift))) << 4);
        *reinterpret_cast<uint4*>(page + a.to_k + off) = uk[j];
        *reinterpret_cast<uint4*>(page + a.to_v + off) = uv[j];
      }
    }
    x0 += kRowBatch * kRowThreads;
    if (x0 >= a.chunks) break;
    load(x0);
  }
}

// ------------------------------------------------------------- host side

const char* check_paged(const ssd_paged_cache* c, ssd_status* status) noexcept {
  *status = SSD_ERR_INVALID_ARG;
  if (!c) return "cache is NULL";
  if (c->n_seq < 1 || c->n_seq > SSD_KV8_MAX_SEQS) return "cache: n_seq must be in 1..4096";
  if (c->n_layers < 1 || c->n_layers > 1024) return "cache: n_layers must be in 1..1024";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return "cache: n_kv_heads must be in 1..1024";
  if (c->dtype != SSD_DTYPE_F32 && c->dtype != SSD_DTYPE_BF16)
    return "cache: dtype must be fp32 or bf16";
  if (c->n_pages < 1 || c->n_pages > (1 << 24)) return "cache: n_pages must be in 1..2^24";
  *status = SSD_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return "cache: head_dim must be 64 or 128";
  if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1)))
    return "cache: page must be 16, 32, 64, 128 or 256";
  *status = SSD_ERR_INVALID_ARG;
  if (c->max_pages < 1 || c->max_pages > (1 << 30) / c->page)
    return "cache: max_pages x page must be in 1..2^30";
  if ((int64_t)c->n_seq * c->max_pages > 0x7fffffffll)
    return "cache: n_seq x max_pages must be below 2^31";
  if (!c->pages || !c->table || !c->refs || ((uintptr_t)c->pages & 15u) ||
      ((uintptr_t)c->table & 3u) || ((uintptr_t)c->refs & 15u))
    return "cache: NULL or unaligned pointer";
  *status = SSD_OK;
  return nullptr;
}

PagedView paged_view(const ssd_paged_cache* c) noexcept {
  PagedView v{};
  v.pages = static_cast<char*>(c->pages);
  v.table = c->table;
  v.refs = c->refs;
  v.n_seq = c->n_seq;
  v.n_pages = c->n_pages;
  v.max_pages = c->max_pages;
  while ((1 << v.shift) < c->page) ++v.shift;
  v.n_kv_heads = c->n_kv_heads;
  v.slab = c->page * c->head_dim * (c->dtype == SSD_DTYPE_BF16 ? 2 : 4);
  v.slabs = c->n_layers * 2 * c->n_kv_heads;
  v.bytes = (size_t)v.slabs * v.slab;
  return v;
}

namespace {

const char* check_work(const ssd_paged_cache* c, const void* workspace, size_t bytes,
                       ssd_status* status) {
  *status = SSD_ERR_INVALID_ARG;
  if (!workspace || ((uintptr_t)workspace & 255u))
    return "workspace must be non-NULL and 256-byte aligned";
  *status = SSD_ERR_CAPACITY;
  if (bytes < plan_bytes(c->n_pages)) return "workspace too small";
  *status = SSD_OK;
  return nullptr;
}

// Pools for which the planning block has 256 threads, whose barriers cost less, and above which 1024,
// which look at more counts at once. us, fork and reserve, 256 / 1024 threads: 4 sequences and 12 pages
// 8.7 / 10.7, 64 sequences with 24 copies of 5 MB and 146 pages 39.6 / 40.4, 192 sequences with 1548
// new pages of 30961 28.6 / 17.9.
constexpr int kSmallPool = 8192;

// The launch that carries a plan out: up to four blocks an SM.
template <typename Kern>
cudaError_t carry_out(Kern k, const PagedView& v, const PlanWork& w, int most, int64_t more,
                      cudaStream_t st) {
  int64_t blocks = ((int64_t)most * v.slabs + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  if (blocks < more) blocks = more;
  if (blocks > 608) blocks = 608;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kCopyThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = g_pdl_enabled ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, v, w);
}

}  // namespace
}  // namespace ssd

extern "C" size_t ssd_paged_workspace_bytes(const ssd_paged_cache* c) {
  using namespace ssd;
  ssd_status status;
  if (const char* why = check_paged(c, &status)) {
    fail_op(status, why);
    return 0;
  }
  return plan_bytes(c->n_pages);
}

extern "C" ssd_status ssd_paged_reserve(const ssd_paged_cache* c, const int32_t* pos,
                                        const int32_t* rows, int32_t M, void* workspace,
                                        size_t workspace_bytes, int32_t* err_dev, void* stream) {
  using namespace ssd;
  ssd_status status;
  if (const char* why = check_paged(c, &status)) return fail_op(status, why);
  if (!pos) return fail_op(SSD_ERR_INVALID_ARG, "pos: NULL pointer");
  if (M < 1) return fail_op(SSD_ERR_INVALID_ARG, "M must be at least 1");
  if (M > c->max_pages * c->page)
    return fail_op(SSD_ERR_CAPACITY, "more rows than the cache has positions");
  if (const char* why = check_work(c, workspace, workspace_bytes, &status))
    return fail_op(status, why);
  const PagedView v = paged_view(c);
  const PlanWork w = plan_work(workspace, c->n_pages);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool small = c->n_pages <= kSmallPool;
  cudaError_t e = launch_first(small ? k_paged_reserve<256> : k_paged_reserve<1024>, dim3(1),
                               small ? 256 : 1024, 0, 1, st, v, w, pos, rows, M, err_dev);
  if (e == cudaSuccess)
    e = carry_out(k_paged_copy, v, w, c->n_seq < c->n_pages ? c->n_seq : c->n_pages, 1, st);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_paged_reserve", e);
}

extern "C" ssd_status ssd_paged_fork(const ssd_paged_cache* c, const int32_t* parent,
                                     const int32_t* length, int32_t* err_dev, void* stream) {
  using namespace ssd;
  ssd_status status;
  if (const char* why = check_paged(c, &status)) return fail_op(status, why);
  if (!parent && !length) return fail_op(SSD_ERR_INVALID_ARG, "neither parent nor length");
  const PagedView v = paged_view(c);
  const size_t smem = (size_t)c->n_seq * kForkCols * sizeof(int);
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024)
    e = cudaFuncSetAttribute(k_paged_fork, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             SSD_KV8_MAX_SEQS * kForkCols * (int)sizeof(int));
  if (e == cudaSuccess)
    e = launch_first(k_paged_fork, dim3((c->max_pages + kForkCols - 1) / kForkCols), kCopyThreads, smem, 1,
                     static_cast<cudaStream_t>(stream), v, parent, length, err_dev);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_paged_fork", e);
}

extern "C" ssd_status ssd_paged_compact(const ssd_paged_cache* c, int32_t* used, void* workspace,
                                        size_t workspace_bytes, int32_t* err_dev, void* stream) {
  using namespace ssd;
  (void)err_dev;  // nothing that only the device can see goes wrong here
  ssd_status status;
  if (const char* why = check_paged(c, &status)) return fail_op(status, why);
  if (const char* why = check_work(c, workspace, workspace_bytes, &status))
    return fail_op(status, why);
  const PagedView v = paged_view(c);
  const PlanWork w = plan_work(workspace, c->n_pages);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = c->n_pages <= kSmallPool
                      ? launch_first(k_paged_compact<256>, dim3(1), 256, 0, 1, st, v, w, used)
                      : launch_first(k_paged_compact<1024>, dim3(1), 1024, 0, 1, st, v, w, used);
  if (e == cudaSuccess)
    e = carry_out(k_paged_move, v, w, c->n_pages / 2,
                  ((int64_t)c->n_seq * c->max_pages + kCopyThreads - 1) / kCopyThreads, st);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_paged_compact", e);
}

extern "C" ssd_status ssd_paged_append(const ssd_paged_cache* c, int32_t layer, const void* k,
                                       const void* v, int64_t row_stride, int32_t M,
                                       const int32_t* pos, const int32_t* rows, int32_t* err_dev,
                                       void* stream) {
  using namespace ssd;
  ssd_status status;
  if (const char* why = check_paged(c, &status)) return fail_op(status, why);
  if (layer < 0 || layer >= c->n_layers)
    return fail_op(SSD_ERR_INVALID_ARG, "layer must be in 0..n_layers - 1");
  const int elt = c->dtype == SSD_DTYPE_BF16 ? 2 : 4;
  if (!k || !v || !pos || ((uintptr_t)k & 15u) || ((uintptr_t)v & 15u))
    return fail_op(SSD_ERR_INVALID_ARG, "k, v or pos: NULL or unaligned pointer");
  if (M < 1) return fail_op(SSD_ERR_INVALID_ARG, "M must be at least 1");
  if (M > c->max_pages * c->page)
    return fail_op(SSD_ERR_CAPACITY, "more rows than the cache has positions");
  if (row_stride < (int64_t)c->n_kv_heads * c->head_dim || row_stride > (1ll << 40) ||
      (row_stride * elt) % 16)
    return fail_op(SSD_ERR_INVALID_ARG,
                   "row_stride: below a row's length, or not a multiple of 16 bytes");
  PagedAppend a{};
  a.c = paged_view(c);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.stride = row_stride * elt;
  a.to_k = a.c.side(layer, 0);
  a.to_v = a.c.side(layer, 1);
  a.chunks = c->n_kv_heads * c->head_dim * elt / 16;
  while ((16 << a.head_shift) < c->head_dim * elt) ++a.head_shift;
  a.pos = pos;
  a.rows = rows;
  a.err = err_dev;
  a.M = M;
  const cudaError_t e = launch_first(k_paged_append, dim3(M, c->n_seq), kRowThreads, 0, 1,
                                     static_cast<cudaStream_t>(stream), a);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_paged_append", e);
}
