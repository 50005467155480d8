// paged.cuh -- the paged KV cache of the kernel-level entry points: where things stand in it.
//
// pages [n_pages][n_layers][n_kv_heads][2][page][head_dim]: a page is one piece of memory, so that
// copying or moving one is a single long copy. What an attention reads of a page, a head's keys (a slab)
// and its values, lies in one piece, too.
#pragma once

#include "kv8.cuh"
#include "mma.cuh"

namespace ssd {

struct PagedView {
  char* pages;
  int32_t* table;
  int32_t* refs;
  int32_t n_seq, n_pages, max_pages, shift;  // page = 1 << shift
  int32_t n_kv_heads, slab, slabs;           // bytes of a slab, slabs of a page
  size_t bytes;                              // of a page
  __host__ __device__ __forceinline__ int cap() const { return max_pages << shift; }
  // The page of entry i of sequence b, or -1.
  __device__ __forceinline__ int entry(int b, int i) const {
    const int e = table[(size_t)b * max_pages + i];
    return (unsigned)e < (unsigned)n_pages ? e : -1;
  }
  // Layer `layer`, side 0 (K) or 1 (V) of page 0, head 0; bytes to the next head.
  __host__ __device__ __forceinline__ size_t side(int layer, int side) const {
    return ((size_t)layer * n_kv_heads * 2 + side) * slab;
  }
  __host__ __device__ __forceinline__ size_t head() const { return (size_t)2 * slab; }
};

// The pages of a sequence's entries in order, for a warp that walks keys kb .. ke - 1: a lane holds one
// of 32 entries, and the next 32 are on their way meanwhile. (Looked up a stage of 64 keys ahead, an
// entry that had to come from memory held the copies up: pages of 16, 64 and 256 positions were read at
// 5.6, 6.4 and 6.7 TB/s, now at 6.5, 7.2 and 7.4.)
struct PageWalk {
  const PagedView* view;
  int32_t* err;
  int b, from, to, base, now, then;  // entries from .. to are there; `now` are those from base on
  __device__ __forceinline__ PageWalk(const PagedView& v, int32_t* e)
      : view(&v), err(e), b(0), from(0), to(-1), base(0), now(0), then(0) {}
  __device__ __forceinline__ int load(int i) const {
    i += threadIdx.x & 31;
    return i < from || i > to ? 0 : view->entry(b, i);
  }
  // key0: where the walk begins, kb or in front of it
  __device__ __forceinline__ void start(int seq, int key0, int kb, int ke) {
    b = seq;
    from = kb >> view->shift;
    to = kb < ke ? (ke - 1) >> view->shift : -1;
    base = key0 >> view->shift;
    now = load(base);
    then = load(base + 32);
  }
  // The page of the entry that holds `key` (one for the whole warp, none in front of the last one's).
  __device__ __forceinline__ int page(int key) {
    const int i = key >> view->shift;
    if (i >= base + 32) {
      base += 32;
      now = then;
      then = load(base + 32);
    }
    const int e = __shfl_sync(0xffffffffu, now, i - base);
    if (e < 0 && (threadIdx.x & 31) == 0 && err) atomicOr(err, (int)kErrTable);
    return max(e, 0);
  }
};

// Where keys k0 .. k0 + KEYS - 1 stand, by sixteens, which lie in one page each: bytes from position 0
// of page 0.
template <int KEYS, int ROW_BYTES>
__device__ __forceinline__ void find_keys(PageWalk& walk, int k0, size_t (&off)[KEYS / 16]) {
#pragma unroll
  for (int j = 0; j < KEYS / 16; ++j)
    off[j] = (size_t)walk.page(k0 + 16 * j) * walk.view->bytes +
             (size_t)((k0 + 16 * j) & ((1 << walk.view->shift) - 1)) * ROW_BYTES;
}
// Copies them (or their values) to shared memory, zeros for those outside of kb .. ke - 1, as one of
// the threads that hold PASS rows at a time: p at its chunk of its row (r0, below PASS) of position 0
// of page 0, to(r) where that chunk of row r0 + r goes.
template <int KEYS, int ROW_BYTES, int PASS, typename To>
__device__ __forceinline__ void copy_keys(const size_t (&off)[KEYS / 16], const char* p, int r0, int k0,
                                          int kb, int ke, To to) {
  static_assert(16 % PASS == 0, "whole passes of sixteen rows");
  const bool all = k0 >= kb && k0 + KEYS <= ke;
#pragma unroll
  for (int j = 0; j < KEYS; j += PASS) {
    const int key = k0 + j + r0;
    cp_async16(to(j), p + off[j / 16] + j % 16 * ROW_BYTES, all || (key >= kb && key < ke));
  }
}

// Launches a call's first kernel, which begins with pdl_wait(): its blocks take their places while the
// kernel before it in the stream ends (a call of 9 us takes 12 otherwise; not while a graph is
// captured, where what comes before need not be a kernel). What that kernel may have written is read by
// plain loads, not as read-only data, which has to be constant while a kernel is resident. cluster:
// blocks of a cluster, or 1.
template <typename Kern, typename... Args>
cudaError_t launch_first(Kern k, dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st,
                         Args... args) {
  cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
  const bool early = g_pdl_enabled && cudaStreamIsCapturing(st, &capturing) == cudaSuccess &&
                     capturing == cudaStreamCaptureStatusNone;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = early ? 1 : 0;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k, args...);
}

// Checks of a cache that every entry point makes; null: fine.
const char* check_paged(const ssd_paged_cache* c, ssd_status* status) noexcept;
PagedView paged_view(const ssd_paged_cache* c) noexcept;

}  // namespace ssd
