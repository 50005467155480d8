// kv8_plan.cuh -- how the attention over the 8-bit cache, or over pages, is dealt out.
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
// joins them.  Short caches have a cluster of blocks for each item instead, which joins its
// sums itself.
#pragma once

#include "kv8.cuh"

namespace ssd {

// n / d for 0 <= n < 2^31 by a product: m = ceil(2^(31 + s) / d), 2^(s - 1) < d <= 2^s.
struct Kv8Div {
  uint32_t d, m, s;
  static Kv8Div of(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return Kv8Div{d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
  }
  __device__ __forceinline__ int operator()(int n) const {
    return (int)((((uint64_t)(uint32_t)n * m) >> 31) >> s);
  }
};

// What an item costs beside its units (queries, the join of the warps or of the
// parts), in units.  Tiles of 16 and 128 rows: 2 to 3 us against 0.7 a unit; without it 24
// ragged sequences of 32 heads kept the last block busy for 90 us and the first for 59.
// Tiles of 256: 8 us against 1 (512 rows of 32 heads over 8 x 7936 keys: 2 % slower at 5, the
// same at 11).
template <int RT>
constexpr int kKv8ItemCost = RT > 128 ? 8 : 3;

// What the plan, the join of parts and the kernels of both caches (8 bits, pages) share.
struct AttnArgs {
  Kv8Div byG, byRt, byP;
  const void* q;
  void* out;
  const int32_t *pos, *rows, *first;
  int32_t* err;
  int64_t q_stride, out_stride;  // elements between rows
  int32_t n_seq, Hkv, G, M, max_seq, window, n_rt, entries;
  int32_t part_rows;  // rows of a tile, at most
  int32_t split;  // 0: the line; else each item's own blocks, a cluster: no parts
  float scale;  // log2(e) / sqrt(head_dim)
  struct Kv8Desc* desc;
  float* part;  // [2 P][part_rows][hd] normalised partial outputs
  float2* ml;   // [2 P][part_rows] their (max, sum), max in powers of two
};

struct Kv8Attn : AttnArgs {
  const uint8_t *k, *v;
  const float *ks, *vs;
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

__device__ __forceinline__ int kv8_row_pos(const AttnArgs& a, const Kv8Item& it, int r) {
  return it.pos + a.byG(r);
}
// First key that the row at position p sees.
__device__ __forceinline__ int kv8_row_lo(const Kv8Item& it, int p, int window) {
  return window > 0 ? max(it.first, p - window + 1) : it.first;
}

template <int RT, int KU>
__device__ __forceinline__ Kv8Item kv8_entry(const AttnArgs& a, int e) {
  Kv8Item it;
  it.b = a.byRt(e);
  it.rt = e - it.b * a.n_rt;
  it.pos = a.pos[it.b];
  const int n = a.rows ? a.rows[it.b] : a.M;
  it.first = a.first ? max(a.first[it.b], 0) : 0;
  it.r0 = it.rt * RT;
  it.nr = 0;
  it.units = it.unit0 = it.lo = it.hi = 0;
  if (it.pos < 0 || n < 0 || n > a.M || it.pos > a.max_seq - n) {
    if (it.rt == 0 && (blockIdx.x == 0 || a.split) && a.err)
      atomicOr(a.err, n < 0 || n > a.M ? (int)kErrControl : (int)kErrCapacity);
    return it;
  }
  it.nr = min(RT, n * a.G - it.r0);
  if (it.nr <= 0) return it;
  it.lo = kv8_row_lo(it, kv8_row_pos(a, it, it.r0), a.window);
  it.hi = kv8_row_pos(a, it, it.r0 + it.nr - 1);
  it.unit0 = min(it.lo, it.hi) / KU;
  it.units = it.hi / KU - it.unit0 + 1;
  return it;
}

// The line as the blocks share it: block i's stretch begins at i total / P.
struct Kv8Line {
  int total, q, r;  // total = q P + r
  __device__ __forceinline__ Kv8Line(const AttnArgs& a, int t) : total(t) {
    q = a.byP(t);
    r = t - q * (int)a.byP.d;
  }
  __device__ __forceinline__ int start(const AttnArgs& a, int i) const { return i * q + a.byP(i * r); }
  // The block whose stretch holds unit x.
  __device__ __forceinline__ int block(const AttnArgs& a, int x) const {
    int j = min((int)((float)x * (float)a.byP.d / (float)total), (int)a.byP.d - 1);
    while (j > 0 && start(a, j) > x) --j;
    while (start(a, j + 1) <= x) ++j;
    return j;
  }
};

// The line's places that an item takes.
template <int RT, int KU>
__device__ __forceinline__ int kv8_len(const Kv8Item& it) {
  return it.units ? it.units + kKv8ItemCost<RT> : 0;
}

// The block's part of an item: units u0 .. u0 + nu - 1.
struct Kv8Seg {
  Kv8Item it;
  int g, u0, nu;
  __device__ __forceinline__ bool whole() const { return nu == it.units; }
};

struct Kv8Cursor {
  int w0, w1, total;  // the block's stretch that is left, the whole line
  int e, off;         // entry that holds w0, its places before w0
};

struct Kv8PlanSmem {
  int warp[32];
  Kv8Cursor c;
};

// Every thread of the block gets the block's stretch.
template <int RT, int KU, int THREADS>
__device__ __forceinline__ Kv8Cursor kv8_plan(const AttnArgs& a, Kv8PlanSmem& sm) {
  static_assert(THREADS / 32 <= 32, "a sum for each warp");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (a.split) {
    const int i = (int)blockIdx.x / a.split, rank = (int)blockIdx.x - i * a.split;
    const int e = i / a.Hkv, g = i - e * a.Hkv;
    const Kv8Item own = kv8_entry<RT, KU>(a, e);
    const int w0 = own.units * rank / a.split, w1 = own.units * (rank + 1) / a.split;
    return Kv8Cursor{w0, w1, 0, e, g * kv8_len<RT, KU>(own) + w0};
  }
  const int per = (a.entries + THREADS - 1) / THREADS;
  const int e0 = min(tid * per, a.entries), e1 = min(e0 + per, a.entries);
  int sum = 0;
  Kv8Item it;
  for (int e = e0; e < e1; ++e) {
    it = kv8_entry<RT, KU>(a, e);
    sum += kv8_len<RT, KU>(it) * a.Hkv;
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  if (lane == 31) sm.warp[warp] = inc;
  if (tid == 0) sm.c.w0 = sm.c.w1 = 0;
  __syncthreads();
  int before = inc - sum, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += sm.warp[w];
    total += sm.warp[w];
  }
  const Kv8Line line(a, total);
  const int w0 = line.start(a, blockIdx.x), w1 = line.start(a, blockIdx.x + 1);
  if (w0 < w1 && before <= w0 && w0 < before + sum) {  // one thread
    int off = w0 - before, e = e0;
    for (;; ++e) {
      if (per > 1) it = kv8_entry<RT, KU>(a, e);
      const int u = kv8_len<RT, KU>(it) * a.Hkv;
      if (off < u) break;
      off -= u;
    }
    sm.c = Kv8Cursor{w0, w1, total, e, off};
  }
  __syncthreads();
  return sm.c;
}

// The next segment of the block's stretch; false at its end.
template <int RT, int KU>
__device__ __forceinline__ bool kv8_next(const AttnArgs& a, Kv8Cursor& c, Kv8Seg& s) {
  while (c.w0 < c.w1) {
    s.it = kv8_entry<RT, KU>(a, c.e);
    const int len = kv8_len<RT, KU>(s.it);
    if (c.off >= len * a.Hkv) {
      c.off = 0;
      ++c.e;
      continue;
    }
    s.g = c.off / len;
    s.u0 = c.off - s.g * len;
    if (s.u0 >= s.it.units) {  // the item's cost
      const int n = min(len - s.u0, c.w1 - c.w0);
      c.w0 += n;
      c.off += n;
      continue;
    }
    s.nu = min(s.it.units - s.u0, c.w1 - c.w0);
    c.w0 += s.nu;
    c.off += s.nu;
    return true;
  }
  return false;
}

// The segment as the merge finds it, where it begins an item that goes on in
// the next block.  c: the cursor behind the segment.
__device__ __forceinline__ Kv8Desc kv8_desc(const AttnArgs& a, const Kv8Cursor& c, const Kv8Seg& s) {
  const int last = c.w0 - s.nu + s.it.units - 1;  // the item's last unit
  return Kv8Desc{s.it.nr, s.it.b, s.it.r0, s.g, Kv8Line(a, c.total).block(a, last), c.total,
                 s.it.pos, s.it.first};
}

}  // namespace ssd
