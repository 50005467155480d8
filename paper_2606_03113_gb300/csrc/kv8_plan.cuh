// kv8_plan.cuh -- how the attention over the 8-bit cache is dealt out.
//
// The query rows of one sequence and KV head are the M new rows times the G
// query heads of the group, row r = m G + h, cut into tiles of RT rows.  An entry
// is a (sequence, row tile) pair, an item an entry with a KV head, and an item's
// work is counted in units of one cache block (kKv8Block keys) that some row of
// the tile sees, at least one.  The units of all items stand in one line (entries,
// then heads, then keys) that a grid of P blocks shares evenly, whatever
// the lengths are; they are read from device memory, so a captured launch serves
// growing sequences.  A block's stretch of the line can begin and end inside an
// item: it then leaves the item's partial sums in the workspace, and k_kv8_merge
// joins them.
#pragma once

#include "kv8.cuh"

namespace ssd {

struct Kv8Attn {
  const uint8_t *k, *v;
  const float *ks, *vs;
  const void* q;
  void* out;
  const int32_t *pos, *rows, *first;
  int32_t* err;
  int64_t q_stride, out_stride;  // elements between rows
  int32_t n_seq, Hkv, G, M, max_seq, window, n_rt, entries;
  float scale;  // log2(e) / sqrt(head_dim)
  struct Kv8Desc* desc;
  float* part;  // [2 P][RT][hd] normalised partial outputs
  float2* ml;   // [2 P][RT] their (max, sum), max in powers of two
};

// What block i of the attention left to be joined: the item that begins in its
// stretch and ends in that of block `last`; nr: its rows (0: nothing here).
struct __align__(32) Kv8Desc {
  int32_t nr, b, r0, g, last, total, pos, first;
};

struct Kv8Item {
  int b, rt, r0, nr;   // sequence, tile, first row, rows
  int pos, first;      // position of the sequence's first new row; first visible key
  int lo, hi;          // keys that some row sees: lo .. hi (none when lo > hi)
  int unit0, units;    // first unit of KU keys, number of them (0: no rows here)
};

__device__ __forceinline__ int kv8_row_pos(const Kv8Item& it, int r, int G) { return it.pos + r / G; }
// First key that the row at position p sees.
__device__ __forceinline__ int kv8_row_lo(const Kv8Item& it, int p, int window) {
  return window > 0 ? max(it.first, p - window + 1) : it.first;
}

template <int RT, int KU>
__device__ __forceinline__ Kv8Item kv8_entry(const Kv8Attn& a, int e) {
  Kv8Item it;
  it.b = e / a.n_rt;
  it.rt = e - it.b * a.n_rt;
  it.pos = __ldg(a.pos + it.b);
  const int n = a.rows ? __ldg(a.rows + it.b) : a.M;
  it.first = a.first ? max(__ldg(a.first + it.b), 0) : 0;
  it.r0 = it.rt * RT;
  it.nr = 0;
  it.units = it.unit0 = it.lo = it.hi = 0;
  if (it.pos < 0 || n < 0 || n > a.M || it.pos > a.max_seq - n) {
    if (it.rt == 0 && blockIdx.x == 0 && a.err)
      atomicOr(a.err, n < 0 || n > a.M ? (int)kErrControl : (int)kErrCapacity);
    return it;
  }
  it.nr = min(RT, n * a.G - it.r0);
  if (it.nr <= 0) return it;
  it.lo = kv8_row_lo(it, kv8_row_pos(it, it.r0, a.G), a.window);
  it.hi = kv8_row_pos(it, it.r0 + it.nr - 1, a.G);
  it.unit0 = min(it.lo, it.hi) / KU;
  it.units = it.hi / KU - it.unit0 + 1;
  return it;
}

// First unit of block i's stretch.
__device__ __forceinline__ int kv8_start(int i, int P, int total) {
  return (int)((long long)i * total / P);
}

// The block's part of an item: units u0 .. u0 + nu - 1.
struct Kv8Seg {
  Kv8Item it;
  int g, u0, nu;
  __device__ __forceinline__ bool whole() const { return nu == it.units; }
};

struct Kv8Cursor {
  int w0, w1, total;  // the block's stretch, all units
  int e, off;         // entry that holds w0, units of that entry before w0
};

// Every thread of the block gets the block's stretch; sm: THREADS / 32 + 2 ints.
template <int RT, int KU, int THREADS>
__device__ __forceinline__ Kv8Cursor kv8_plan(const Kv8Attn& a, int* sm) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.entries + THREADS - 1) / THREADS;
  const int e0 = min(tid * per, a.entries), e1 = min(e0 + per, a.entries);
  int sum = 0;
  for (int e = e0; e < e1; ++e) sum += kv8_entry<RT, KU>(a, e).units * a.Hkv;
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  if (lane == 31) sm[warp] = inc;
  __syncthreads();
  int before = inc - sum, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += sm[w];
    total += sm[w];
  }
  Kv8Cursor c;
  c.total = total;
  c.w0 = kv8_start(blockIdx.x, gridDim.x, total);
  c.w1 = kv8_start(blockIdx.x + 1, gridDim.x, total);
  if (c.w0 < c.w1 && before <= c.w0 && c.w0 < before + sum) {  // one thread
    int off = c.w0 - before, e = e0;
    for (;; ++e) {
      const int u = kv8_entry<RT, KU>(a, e).units * a.Hkv;
      if (off < u) break;
      off -= u;
    }
    sm[THREADS / 32] = e;
    sm[THREADS / 32 + 1] = off;
  }
  __syncthreads();
  c.e = sm[THREADS / 32];
  c.off = sm[THREADS / 32 + 1];
  return c;
}

// The next segment of the block's stretch; false at its end.
template <int RT, int KU>
__device__ __forceinline__ bool kv8_next(const Kv8Attn& a, Kv8Cursor& c, Kv8Seg& s) {
  while (c.w0 < c.w1) {
    s.it = kv8_entry<RT, KU>(a, c.e);
    if (c.off >= s.it.units * a.Hkv) {
      c.off = 0;
      ++c.e;
      continue;
    }
    s.g = c.off / s.it.units;
    s.u0 = c.off - s.g * s.it.units;
    s.nu = min(s.it.units - s.u0, c.w1 - c.w0);
    c.w0 += s.nu;
    c.off += s.nu;
    return true;
  }
  return false;
}

// The segment as the merge finds it, where it begins an item that goes on in
// the next block.  c: the cursor behind the segment.
__device__ __forceinline__ Kv8Desc kv8_desc(const Kv8Cursor& c, const Kv8Seg& s) {
  const long long end = (long long)c.w0 - s.nu + s.it.units;  // the unit behind the item
  return Kv8Desc{s.it.nr, s.it.b, s.it.r0, s.g, (int)((end * gridDim.x - 1) / c.total), c.total,
                 s.it.pos, s.it.first};
}

}  // namespace ssd
