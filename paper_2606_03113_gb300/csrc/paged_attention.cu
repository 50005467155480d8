// paged_attention.cu -- attention of new rows over the pages of a layer (paged.cuh):
//   o_r = sum_j p_rj v_j / sum_j p_rj,  p_rj = e^(q_r . k_j / sqrt(hd) - max),
// over the keys j that row r sees: first .. its own position, at most `window`.
//
// Work is dealt out as in the 8-bit attention (kv8_plan.cuh): items of a sequence, tile of query rows
// and KV head, their keys in units of 64 on a line that all blocks share, parts joined by k_kv8_merge;
// or, where sequences are short, a cluster of blocks for each item. The kernels, chosen by the rules in
// front of plan_of:
// - k_paged_rows: 8 to 64 rows a block, two blocks an SM, clusters; for short sequences, for fp32, and
//   for more than 16 rows of head_dim 64;
// - k_paged_stream (paged_stream.cuh): up to 16 rows over long sequences, one block an SM;
// - k_paged_wide (paged_wide.cuh): more rows, on tcgen05.
//
// k_paged_rows: stages of 32 or 64 keys and values come by cp.async, kNst - 1 of them on their way. A
// warp has a tile of the item's rows and, of each stage, the keys of its group; it keeps a running
// maximum, sum and output of its own, and the block joins the groups once per item. bf16: mma.sync on
// the rows as they are, probabilities in two bf16 parts (16 bits), so that the output's own rounding is
// what remains. fp32: fused multiply-adds. Scores, sums and outputs are fp32. A cluster's blocks write
// their parts to the shared memory of the block that joins the row, so one barrier lies between them
// and its sums.
//
// Bound by bytes for long sequences: 1 row of 32 heads over 8 KV heads x 131072 keys in pages of 64,
// 83.9 us = 6.4 TB/s (7.2 once it runs; 5 us are the start, 4 the join), fp32 1 row over 4 x 100000
// keys of head_dim 64 40 us = 5.1 TB/s. By round trips of memory for short ones: 1 row at 1100 keys 8.9
// us, of which 1.0 are positions, 1.3 table and queries, 0.7 the first keys, 1.8 three stages, 3.6 the
// joins of warps and blocks.
//
// A key that some row of the tile does not see can hold anything: its scores are dropped by
// position, and a value there that is no number is zeroed before the product. A row that sees one
// gets it back at the end of the item: rows with such a value are summed again, key by key.
#include <math.h>

#include <mutex>
#include <type_traits>

#include "kv8_merge.cuh"
#include "mma.cuh"
#include "paged.cuh"

namespace ssd {

namespace {

constexpr int kUnit = kKv8Block;  // keys of a unit of the plan
constexpr int kTile = 16;         // query rows of a warp, at most
constexpr int kSplitMax = 8;      // blocks of a short sequence's item, a cluster, at most

// The cluster's barrier in two halves (a warp's lanes can come apart), and writes to another block's
// shared memory.
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ void st_cluster_f32x2(uint32_t at, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void st_cluster_f32x4(uint32_t at, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z),
               "f"(v.w)
               : "memory");
}

struct PagedAttn : AttnArgs {
  PagedView c;
  const char *k, *v;  // the layer's K and V in page 0
};

// Where things stand in a block's shared memory.
template <typename T, int HD, int R, int NB>
struct PL {
  static constexpr int NW = sizeof(T) == 4 && NB == 1 ? 8 : 4;  // warps
  static constexpr int kRowBytes = HD * (int)sizeof(T);
  static constexpr int kChunks = kRowBytes / 16;           // 16-byte chunks of a row
  static constexpr int kKeys = kRowBytes > 256 ? 32 : 64;  // of a stage
  static constexpr uint32_t kSide = kKeys * kRowBytes;
  static constexpr uint32_t kStage = 2 * kSide;
  static constexpr int kNst = 96 * 1024 / (int)kStage;
  static constexpr uint32_t kRing = kNst * kStage;
  static constexpr int kGroups = NW / R;               // of warps, with keys of their own each
  static constexpr int kGroupKeys = kKeys / kGroups;
  static constexpr int kThreads = NW * 32;
  static constexpr int kWarpRows = 8 * NB, kRows = R * kWarpRows;
  static constexpr int kOPad = HD + 4;  // floats of a row in the exchange
  static constexpr uint32_t kQ = sizeof(T) == 4 ? kRows * kOPad * 4 : 0;  // fp32 queries
  static constexpr uint32_t kSmem = kRing + kQ;
  static constexpr uint32_t kExchange = kGroups * kRows * kOPad * 4;
  static_assert(kExchange + kRows * HD * 4 <= kRing, "the exchange and the part fit the ring");
  static_assert(kRows % kSplitMax == 0, "a cluster's blocks have as many rows each");
  static_assert(kKeys * kChunks % kThreads == 0 && kThreads % kChunks == 0, "whole rows a pass");
  // Chunk ch of row r: bf16 rows as ldmatrix wants them; fp32 rows such that eight lanes meet
  // all banks, as two keys x four chunks and as four keys of one parity x two.
  __device__ static __forceinline__ uint32_t place(int r, int ch) {
    const int x = sizeof(T) == 2 ? r & 7 : (r & 6) ^ ((r & 1) << 2);
    return (uint32_t)(r * kRowBytes + ((ch ^ x) << 4));
  }
  // The same for row r0 + r, with at0 = place(r0, ch), r a multiple of PASS and r0 below it.
  template <int PASS>
  __device__ static __forceinline__ uint32_t place_from(uint32_t at0, int r) {
    return PASS % 8 == 0 ? at0 + (uint32_t)(r * kRowBytes)
                         : (at0 ^ (uint32_t)((r & 4) << 4)) + (uint32_t)(r * kRowBytes);
  }
};

__device__ __forceinline__ bool no_number(float x) {
  return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u;
}
// The bf16 pair without what is no number; `any` where there was one.
__device__ __forceinline__ uint32_t numbers(uint32_t u, uint32_t& any) {
  const uint32_t lo = (u & 0x7f80u) == 0x7f80u ? 0xffffu : 0u;
  const uint32_t hi = (u & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
  any |= lo | hi;
  return u & ~(lo | hi);
}
__device__ __forceinline__ float4 lds4(const unsigned char* p) {
  return *reinterpret_cast<const float4*>(p);
}

// What a warp holds of up to 8 query rows, fp32: every lane has all rows, HD / 32 columns of each; a
// step is of KEYS keys, a key's score the sum of 32 / KEYS lanes.
template <int HD, int KEYS>
struct FewTile {
  static constexpr int kRows = 8, C = HD / 32, SUB = 32 / KEYS;
  float o[kRows][C], mx[kRows], ls[kRows];
  __device__ __forceinline__ void start(const AttnArgs&, const Kv8Item&, int) {
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      mx[r] = -INFINITY;
      ls[r] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[r][c] = 0.f;
    }
  }
  // Keys kk0 .. kk0 + KEYS - 1 of a stage, of them key k0 the first.
  template <typename L>
  __device__ __forceinline__ uint32_t step(const AttnArgs& a, const Kv8Item& it, const float* Qs,
                                           const unsigned char* sk, const unsigned char* sv, int kk0,
                                           int k0, bool full) {
    const int lane = threadIdx.x & 31, kk = lane / SUB, q = lane % SUB;
    float4 k4[L::kChunks / SUB];
#pragma unroll
    for (int i = 0; i < L::kChunks / SUB; ++i) k4[i] = lds4(sk + L::place(kk0 + kk, i * SUB + q));
    float p[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      p[r] = 0.f;
      if (r >= it.nr) break;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < L::kChunks / SUB; ++i) {
        const float4 u = *reinterpret_cast<const float4*>(Qs + r * L::kOPad + (i * SUB + q) * 4);
        s = fmaf(u.x, k4[i].x, s);
        s = fmaf(u.y, k4[i].y, s);
        s = fmaf(u.z, k4[i].z, s);
        s = fmaf(u.w, k4[i].w, s);
      }
#pragma unroll
      for (int y = 1; y < SUB; y <<= 1) s += __shfl_xor_sync(0xffffffffu, s, y);
      float z = __fmul_rn(s, a.scale);  // (not contracted: the maximum is one of these)
      if (!full) {
        const int at = kv8_row_pos(a, it, it.r0 + r);
        if (k0 + kk > at || k0 + kk < kv8_row_lo(it, at, a.window)) z = -INFINITY;
      }
      float nm = z;
#pragma unroll
      for (int y = SUB; y < 32; y <<= 1) nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, y));
      nm = fmaxf(nm, mx[r]);
      if (nm != mx[r]) {  // (the same in all lanes)
        const float f = exp2f(mx[r] - nm);
        ls[r] *= f;
#pragma unroll
        for (int c = 0; c < C; ++c) o[r][c] *= f;
        mx[r] = nm;
      }
      p[r] = exp2f(z - (nm == -INFINITY ? 0.f : nm));
      ls[r] += p[r];
    }
    uint32_t any = 0;
    float v[KEYS][C];
#pragma unroll
    for (int x = 0; x < KEYS; ++x) {
      const unsigned char* const at = sv + L::place(kk0 + x, lane * C / 4) + (lane * C % 4) * 4;
      if constexpr (C == 4) {
        const float4 u = *reinterpret_cast<const float4*>(at);
        v[x][0] = u.x, v[x][1] = u.y, v[x][2] = u.z, v[x][3] = u.w;
      } else {
        const float2 u = *reinterpret_cast<const float2*>(at);
        v[x][0] = u.x, v[x][1] = u.y;
      }
      if (!full) {
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (no_number(v[x][c])) v[x][c] = 0.f, any = 1;
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (r >= it.nr) break;
#pragma unroll
      for (int x = 0; x < KEYS; ++x) {
        const float w = __shfl_sync(0xffffffffu, p[r], x * SUB);
#pragma unroll
        for (int c = 0; c < C; ++c) o[r][c] = fmaf(w, v[x][c], o[r][c]);
      }
    }
    return any;
  }
  // The rows' sums, of all lanes.
  __device__ __forceinline__ void sum_up() {
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int y = SUB; y < 32; y <<= 1) ls[r] += __shfl_xor_sync(0xffffffffu, ls[r], y);
  }
};

// What a warp holds of 16 query rows, fp32: lane n8, t has rows n8 and n8 + 8.
template <int HD>
struct RowTile {
  float o[HD / 8][4], mx[2], ls[2];  // outputs, running maxima (in powers of two) and sums
  int plo[2], phi[2];                // the rows see keys plo .. phi
  __device__ __forceinline__ void start(const AttnArgs& a, const Kv8Item& it, int row0) {
    const int n8 = (threadIdx.x & 31) >> 2;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = row0 + n8 + 8 * i;
      phi[i] = row < it.nr ? kv8_row_pos(a, it, it.r0 + row) : -1;  // no row here: sees none
      plo[i] = row < it.nr ? kv8_row_lo(it, phi[i], a.window) : 0;
      mx[i] = -INFINITY;
      ls[i] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < HD / 8; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j][i] = 0.f;
  }
  // Scores sc of 8 N keys from k0 on (lane: keys 8 n + 2 t and 8 n + 2 t + 1) become
  // probabilities; maxima, sums and outputs follow.
  template <int N>
  __device__ __forceinline__ void weigh(float (&sc)[2][4], int k0, bool full, float scale) {
    const int t = threadIdx.x & 3;
    float nm[2] = {-INFINITY, -INFINITY}, f[2], top[2];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        sc[n][x] = __fmul_rn(sc[n][x], scale);  // (not contracted: the maximum is one of these)
        if (!full) {
          const int key = k0 + 8 * n + 2 * t + (x & 1);
          if (key < plo[x >> 1] || key > phi[x >> 1]) sc[n][x] = -INFINITY;
        }
        nm[x >> 1] = fmaxf(nm[x >> 1], sc[n][x]);
      }
    bool moved = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      nm[i] = fmaxf(nm[i], __shfl_xor_sync(0xffffffffu, nm[i], 1));
      nm[i] = fmaxf(nm[i], __shfl_xor_sync(0xffffffffu, nm[i], 2));
      nm[i] = fmaxf(nm[i], mx[i]);
      top[i] = nm[i] == -INFINITY ? 0.f : nm[i];
      f[i] = nm[i] == mx[i] ? 1.f : exp2f(mx[i] - nm[i]);
      moved |= nm[i] != mx[i];
      mx[i] = nm[i];
      ls[i] *= f[i];
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int j = 0; j < HD / 8; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[j][x] *= f[x >> 1];
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        sc[n][x] = exp2f(sc[n][x] - top[x >> 1]);
        ls[x >> 1] += sc[n][x];
      }
  }
  // The rows' sums, of all lanes.
  __device__ __forceinline__ void sum_up() {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ls[i] += __shfl_xor_sync(0xffffffffu, ls[i], 1);
      ls[i] += __shfl_xor_sync(0xffffffffu, ls[i], 2);
    }
  }
};

// The rows and columns of an 8 x 8 matrix of 16-bit values, two a lane, exchanged.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// What a warp holds of 8 NB query rows, bf16. Keys are the matrix rows of its products (S^T = K Q^T, 16
// keys x 8 query rows an instruction, and O^T = V^T P^T), so that the few rows of a decode step take
// half of the instructions that a tile of 16 would: mma.sync is what a step of 16 keys takes longest
// for (24 of them for 8 rows, 48 for 16; about 19 cycles each of a quarter of an SM). Lane n8, t has
// keys n8 and n8 + 8, rows 8 b + 2 t and + 1.
template <int HD, int NB>
struct ColTile {
  float o[HD / 16][NB][4], mx[NB][2], ls[NB][2];  // outputs (columns 16 j + n8, + 8), maxima, sums
  int plo[NB][2], phi[NB][2];                     // the rows see keys plo .. phi
  __device__ __forceinline__ void start(const AttnArgs& a, const Kv8Item& it, int row0) {
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = row0 + 8 * b + 2 * t + i;
        phi[b][i] = row < it.nr ? kv8_row_pos(a, it, it.r0 + row) : -1;  // no row here: sees none
        plo[b][i] = row < it.nr ? kv8_row_lo(it, phi[b][i], a.window) : 0;
        mx[b][i] = -INFINITY;
        ls[b][i] = 0.f;
      }
#pragma unroll
    for (int j = 0; j < HD / 16; ++j)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[j][b][x] = 0.f;
  }
  // 16 keys from row kk0 of a stage on: keys at sk, values at sv (shared memory), places by L. qf: the rows
  // as an operand. Nonzero where a value that is no number was zeroed.
  template <typename L>
  __device__ __forceinline__ uint32_t step(const uint32_t (&qf)[HD / 16][NB][2], uint32_t sk, uint32_t sv,
                                           int kk0, int k0, bool full, float scale) {
    const int lane = threadIdx.x & 31, n8 = lane >> 2;
    float s2[2][NB][4];  // even and odd 16-column steps summed apart
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x) s2[i][b][x] = 0.f;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
      uint32_t u[4];
      ldsm4(sk + L::place(kk0 + (lane & 15), 2 * k + (lane >> 4)), u);
#pragma unroll
      for (int b = 0; b < NB; ++b) mma16816(s2[k & 1][b], u, qf[k][b][0], qf[k][b][1]);
    }
    float z[NB][4], f[NB][2], top[NB][2];
    bool moved = false;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float nm[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        // (not contracted with what follows: the maximum is one of these)
        z[b][x] = __fmul_rn(s2[0][b][x] + s2[1][b][x], scale);
        if (!full) {
          const int key = k0 + n8 + 8 * (x >> 1);
          if (key < plo[b][x & 1] || key > phi[b][x & 1]) z[b][x] = -INFINITY;
        }
        nm[x & 1] = fmaxf(nm[x & 1], z[b][x]);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int y = 4; y < 32; y <<= 1) nm[i] = fmaxf(nm[i], __shfl_xor_sync(0xffffffffu, nm[i], y));
        nm[i] = fmaxf(nm[i], mx[b][i]);
        top[b][i] = nm[i] == -INFINITY ? 0.f : nm[i];
        f[b][i] = nm[i] == mx[b][i] ? 1.f : exp2f(mx[b][i] - nm[i]);
        moved |= nm[i] != mx[b][i];
        mx[b][i] = nm[i];
        ls[b][i] *= f[b][i];
      }
    }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int j = 0; j < HD / 16; ++j)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[j][b][x] *= f[b][x & 1];
    }
    uint32_t any = 0, hi[NB][2], lo[NB][2];  // probabilities in two parts, keys n8 and n8 + 8
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = exp2f(z[b][2 * h] - top[b][0]), p1 = exp2f(z[b][2 * h + 1] - top[b][1]);
        ls[b][0] += p0;
        ls[b][1] += p1;
        split2(p0, p1, hi[b][h], lo[b][h]);
        hi[b][h] = transpose8(hi[b][h]);
        lo[b][h] = transpose8(lo[b][h]);
      }
#pragma unroll
    for (int j = 0; j < HD / 16; ++j) {
      uint32_t u[4];
      ldsm4t(sv + L::place(kk0 + (lane & 7) + ((lane >> 4) << 3), 2 * j + (lane >> 3 & 1)), u);
      if (!full) {
#pragma unroll
        for (int x = 0; x < 4; ++x) u[x] = numbers(u[x], any);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) mma16816(o[j][b], u, lo[b][0], lo[b][1]);
#pragma unroll
      for (int b = 0; b < NB; ++b) mma16816(o[j][b], u, hi[b][0], hi[b][1]);
    }
    return any;
  }
  // The rows' sums, of all lanes.
  __device__ __forceinline__ void sum_up() {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int y = 4; y < 32; y <<= 1) ls[b][i] += __shfl_xor_sync(0xffffffffu, ls[b][i], y);
  }
};

// The rows of a block's part of an item, from what GROUPS groups of warps left: outputs in Ox
// [GROUPS][ROWS][HD + 4], weights s_w (NULL: 1), the rows' maxima and sums. Of keys kb .. ke - 1. To
// the output, to the workspace, or, for a cluster's join, where `put` says.
template <typename T, int HD, int GROUPS, int ROWS, int THREADS, typename Put>
__device__ __forceinline__ void finish_rows(const PagedAttn& a, const Kv8Seg& sg, int kb, int ke,
                                            const float* Ox, const float (*s_w)[ROWS],
                                            const float* s_gm, const float* s_sum, bool bad, int tid,
                                            Put put) {
  constexpr int NT = HD / 8, kOPad = HD + 4;
  const Kv8Item& it = sg.it;
  const bool whole = sg.whole();
  const int slot = 2 * blockIdx.x + (sg.u0 == 0), g = sg.g, pmask = (1 << a.c.shift) - 1;
  const char* const vp = a.v + g * a.c.head();
#pragma unroll 1
  for (int x0 = 0; x0 < ROWS * NT; x0 += THREADS) {
    const int row = (x0 + tid) / NT, c8 = (tid % NT) * 8;
    if (row >= it.nr) continue;
    const int r = it.r0 + row, m = a.byG(r), h = g * a.G + r - m * a.G;
    const int p = kv8_row_pos(a, it, r), lo = kv8_row_lo(it, p, a.window);
    const float gm = s_gm[row], Ls = s_sum[row];
    float acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = 0.f;
    bool nan = false;
#pragma unroll
    for (int x = 0; x < GROUPS; ++x) {
      const float wt = s_w ? s_w[x][row] : 1.f;
      const float4* ox = reinterpret_cast<const float4*>(Ox + (size_t)(x * ROWS + row) * kOPad + c8);
      const float4 u = ox[0], w = ox[1];
      acc[0] = fmaf(u.x, wt, acc[0]);
      acc[1] = fmaf(u.y, wt, acc[1]);
      acc[2] = fmaf(u.z, wt, acc[2]);
      acc[3] = fmaf(u.w, wt, acc[3]);
      acc[4] = fmaf(w.x, wt, acc[4]);
      acc[5] = fmaf(w.y, wt, acc[5]);
      acc[6] = fmaf(w.z, wt, acc[6]);
      acc[7] = fmaf(w.w, wt, acc[7]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) nan |= acc[j] != acc[j];
    // values that are no numbers belong to the rows that see them (a part of a probability times
    // infinity may have made NaN of one); where the scores are NaN, so is everything
    if ((bad || nan) && Ls == Ls) {
      float sum[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] = 0.f;
      for (int key = max(kb, lo); key < min(ke, p + 1); ++key) {
        const int e = max(a.c.entry(it.b, key >> a.c.shift), 0);
        const T* v = reinterpret_cast<const T*>(vp + (size_t)e * a.c.bytes) +
                     (size_t)(key & pmask) * HD + c8;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = Elem<T>::to_f(v[j]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (no_number(f[j])) sum[j] += f[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (sum[j] != 0.f) acc[j] = sum[j];
    }
    if (a.split > 1) {
      put(row, c8, acc);
    } else if (whole) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        acc[j] = p < lo ? 0.f : Ls == 0.f ? __uint_as_float(0x7fffffffu) : acc[j];
      store_out8(static_cast<T*>(a.out) + ((int64_t)it.b * a.M + m) * a.out_stride + (int64_t)h * HD +
                     c8,
                 acc);
    } else {
      store_out8(a.part + ((size_t)slot * a.part_rows + row) * HD + c8, acc);
      if (c8 == 0) a.ml[(size_t)slot * a.part_rows + row] = make_float2(gm, Ls);
    }
  }
}

}  // namespace

template <typename T, int HD, int R, int NB>
__global__ void __launch_bounds__(PL<T, HD, R, NB>::kThreads, 2) k_paged_rows(const PagedAttn a) {
  using L = PL<T, HD, R, NB>;
  constexpr bool BF = sizeof(T) == 2, FEW = !BF && NB == 1;
  constexpr int NT = HD / 8;   // 8-column tiles of the output
  constexpr int KS = HD / 16;  // 16-column steps of a score
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ Kv8PlanSmem s_plan;
  __shared__ float s_m[L::kGroups][L::kRows], s_l[L::kGroups][L::kRows], s_w[L::kGroups][L::kRows];
  __shared__ float s_gm[L::kRows], s_sum[L::kRows];
  __shared__ float2 s_in[kSplitMax][L::kRows];  // of a cluster's join: (max, sum) of the blocks' parts
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t = lane & 3, n8 = lane >> 2;
  const int rt = warp % R, grp = warp / R;
  float* const Ox = reinterpret_cast<float*>(smem);
  // a cluster's join: block `row % split` takes the row, [its rows][HD] of each block's part
  float* const parts = Ox + L::kExchange / 4;
  constexpr int kPass = L::kThreads / L::kChunks;  // rows of a pass of copies
  const int ch = tid % L::kChunks, r0 = tid / L::kChunks;
  const uint32_t at0 = L::place(r0, ch);

  pdl_wait();
  Kv8Cursor cur;
  Kv8Seg sg;
  bool more;
  const int rank = a.split > 1 ? (int)blockIdx.x % a.split : 0;
  if (a.split) {  // the block's share of its cluster's item
    const int i = (int)blockIdx.x / a.split, e = i / a.Hkv;
    sg.it = kv8_entry<L::kRows, kUnit>(a, e);
    sg.g = i - e * a.Hkv;
    sg.u0 = sg.it.units * rank / a.split;
    sg.nu = sg.it.units * (rank + 1) / a.split - sg.u0;
    more = sg.nu > 0;
  } else {
    cur = kv8_plan<L::kRows, kUnit, L::kThreads>(a, s_plan);
    pdl_launch_dependents();
    if (tid == 0) a.desc[blockIdx.x].nr = 0;
    more = kv8_next<L::kRows, kUnit>(a, cur, sg);
  }
  while (more) {
    const Kv8Item& it = sg.it;
    const int g = sg.g;
    const int seg0 = (it.unit0 + sg.u0) * kUnit;
    const int kb = max(it.lo, seg0), ke = min(it.hi + 1, seg0 + sg.nu * kUnit);
    const int nst = ke > kb ? (ke - seg0 + L::kKeys - 1) / L::kKeys : 0;
    const int st0 = ke > kb ? (kb - seg0) / L::kKeys : 0;
    const char* const kp = a.k + g * a.c.head() + r0 * L::kRowBytes + ch * 16;
    const char* const vp = kp + (a.v - a.k);

    // ---- stages
    PageWalk walk(a.c, a.err);
    auto issue = [&](int s) {
      if (s < nst) {
        const uint32_t dst = smem_u32(smem) + (uint32_t)(s % L::kNst) * L::kStage + at0;
        const int k0 = seg0 + s * L::kKeys;
        size_t off[L::kKeys / 16];
        find_keys<L::kKeys, L::kRowBytes>(walk, k0, off);
        copy_keys<L::kKeys, L::kRowBytes, kPass>(
            off, kp, r0, k0, kb, ke, [&](int r) { return L::template place_from<kPass>(dst, r); });
        copy_keys<L::kKeys, L::kRowBytes, kPass>(off, vp, r0, k0, kb, ke, [&](int r) {
          return L::template place_from<kPass>(dst, r) + L::kSide;
        });
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    walk.start(it.b, seg0 + st0 * L::kKeys, kb, ke);
#pragma unroll
    for (int i = 0; i < L::kNst - 1; ++i) issue(st0 + i);

    // ---- queries of the warp's tile
    uint32_t qf[BF ? KS : 1][NB][2];
    float* const Qs = reinterpret_cast<float*>(smem + L::kRing);
    if (tid == 0) s_bad = 0;
    if constexpr (BF) {
      const T* qp[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int r = it.r0 + min(rt * L::kWarpRows + 8 * b + n8, it.nr - 1);
        const int m = a.byG(r), h = g * a.G + r - m * a.G;
        qp[b] = static_cast<const T*>(a.q) + ((int64_t)it.b * a.M + m) * a.q_stride +
                (int64_t)h * HD + 2 * t;
      }
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            qf[k][b][x] = *reinterpret_cast<const uint32_t*>(qp[b] + 16 * k + 8 * x);
    } else {
      for (int x = tid; x < L::kRows * (HD / 4); x += L::kThreads) {
        const int row = x / (HD / 4), c4 = x % (HD / 4);
        float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < it.nr) {
          const int r = it.r0 + row, m = a.byG(r), h = g * a.G + r - m * a.G;
          u = *(reinterpret_cast<const float4*>(static_cast<const T*>(a.q) +
                                                ((int64_t)it.b * a.M + m) * a.q_stride +
                                                (int64_t)h * HD) +
                c4);
        }
        *reinterpret_cast<float4*>(Qs + row * L::kOPad + c4 * 4) = u;
      }
    }
    typename std::conditional<
        BF, ColTile<HD, NB>,
        typename std::conditional<FEW, FewTile<HD, L::kGroupKeys>, RowTile<HD>>::type>::type w;
    w.start(a, it, rt * L::kWarpRows);
    // every row of the item sees keys full_lo .. full_hi
    const int full_lo = kv8_row_lo(it, it.hi, a.window);
    const int full_hi = kv8_row_pos(a, it, it.r0);
    const bool some = rt * L::kWarpRows < it.nr;  // a tile without rows only helps to copy
    const bool two = rt * kTile + 8 < it.nr;      // fp32: rows n8 + 8 are there

    for (int s = st0; s < nst; ++s) {
      asm volatile("cp.async.wait_group %0;" ::"n"(L::kNst - 2) : "memory");
      __syncthreads();  // the stage is there, and everybody has read the one that is filled next
      issue(s + L::kNst - 1);
      const unsigned char* const sk = smem + (uint32_t)(s % L::kNst) * L::kStage;
      const unsigned char* const sv = sk + L::kSide;
#pragma unroll 1
      for (int x0 = 0; x0 < L::kGroupKeys; x0 += 16) {
        // the warp's 16 keys, or 8 kN, or as many as its group has
        constexpr int kN = L::kGroupKeys < 16 ? 1 : 2, kStep = FEW ? L::kGroupKeys : 8 * kN;
        const int kk0 = grp * L::kGroupKeys + x0, k0 = seg0 + s * L::kKeys + kk0;
        if (!some || k0 >= ke || k0 + kStep <= kb) continue;
        const bool full = k0 >= full_lo && k0 + kStep - 1 <= full_hi;
        uint32_t any = 0;
        if constexpr (BF) {
          any = w.template step<L>(qf, smem_u32(sk), smem_u32(sv), kk0, k0, full, a.scale);
        } else if constexpr (FEW) {
          any = w.template step<L>(a, it, Qs, sk, sv, kk0, k0, full);
        } else {
          float p[2][4];  // lane n8, t: rows n8 and n8 + 8, keys 8 n + 2 t and 8 n + 2 t + 1
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) p[n][x] = 0.f;
#pragma unroll 4
          for (int c4 = 0; c4 < L::kChunks; ++c4) {
            float4 kq[kN][2];
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
              for (int x = 0; x < 2; ++x) kq[n][x] = lds4(sk + L::place(kk0 + 8 * n + 2 * t + x, c4));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              if (i == 1 && !two) continue;
              const float4 q = lds4(reinterpret_cast<const unsigned char*>(
                  Qs + (rt * kTile + n8 + 8 * i) * L::kOPad + c4 * 4));
#pragma unroll
              for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  float& d = p[n][2 * i + x];
                  d = fmaf(q.x, kq[n][x].x, d);
                  d = fmaf(q.y, kq[n][x].y, d);
                  d = fmaf(q.z, kq[n][x].z, d);
                  d = fmaf(q.w, kq[n][x].w, d);
                }
            }
          }
          w.template weigh<kN>(p, k0, full, a.scale);
          // o[j][2 i + ..]: row n8 + 8 i; columns 16 (j / 2) + 4 t + 2 (j % 2) + ..
#pragma unroll
          for (int kk = 0; kk < 8 * kN; ++kk) {
            float pw[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
              pw[i] = __shfl_sync(0xffffffffu, p[kk >> 3][2 * i + (kk & 1)], (lane & 28) + (kk >> 1 & 3));
#pragma unroll
            for (int j = 0; j < NT; j += 2) {
              float4 u = lds4(sv + L::place(kk0 + kk, 2 * j + t));
              if (!full) {
                float* e = &u.x;
#pragma unroll
                for (int x = 0; x < 4; ++x)
                  if (no_number(e[x])) e[x] = 0.f, any = 1;
              }
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                if (i == 1 && !two) continue;
                w.o[j][2 * i] = fmaf(pw[i], u.x, w.o[j][2 * i]);
                w.o[j][2 * i + 1] = fmaf(pw[i], u.y, w.o[j][2 * i + 1]);
                w.o[j + 1][2 * i] = fmaf(pw[i], u.z, w.o[j + 1][2 * i]);
                w.o[j + 1][2 * i + 1] = fmaf(pw[i], u.w, w.o[j + 1][2 * i + 1]);
              }
            }
          }
        }
        if (any) s_bad = 1;
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");

    // ---- the groups' parts together
    w.sum_up();
    if constexpr (BF) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (n8 == 0) {
            s_m[grp][rt * L::kWarpRows + 8 * b + 2 * t + i] = w.mx[b][i];
            s_l[grp][rt * L::kWarpRows + 8 * b + 2 * t + i] = w.ls[b][i];
          }
    } else if constexpr (FEW) {
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (lane == 0) {
          s_m[grp][r] = w.mx[r];
          s_l[grp][r] = w.ls[r];
        }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (t == 0) {
          s_m[grp][rt * kTile + n8 + 8 * i] = w.mx[i];
          s_l[grp][rt * kTile + n8 + 8 * i] = w.ls[i];
        }
    }
    __syncthreads();  // nobody reads the ring any more
    if (a.split > 1) cluster_arrive();
    if (tid < L::kRows) {
      float gm = -INFINITY, sum = 0.f;
#pragma unroll
      for (int x = 0; x < L::kGroups; ++x) gm = fmaxf(gm, s_m[x][tid]);
#pragma unroll
      for (int x = 0; x < L::kGroups; ++x) sum = fmaf(part_weight(s_m[x][tid], gm), s_l[x][tid], sum);
#pragma unroll
      for (int x = 0; x < L::kGroups; ++x)
        s_w[x][tid] = sum != 0.f ? part_weight(s_m[x][tid], gm) / sum : 0.f;
      s_gm[tid] = gm;
      s_sum[tid] = sum;
    }
    if constexpr (BF) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = rt * L::kWarpRows + 8 * b + 2 * t + i;
          float* p = Ox + (size_t)(grp * L::kRows + row) * L::kOPad + n8;
          if (row < it.nr)
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) {
              p[16 * j] = w.o[j][b][i];
              p[16 * j + 8] = w.o[j][b][2 + i];
            }
        }
    } else if constexpr (FEW) {
      constexpr int C = HD / 32;
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < it.nr)
#pragma unroll
          for (int c = 0; c < C; ++c)
            Ox[(size_t)(grp * L::kRows + r) * L::kOPad + lane * C + c] = w.o[r][c];
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = rt * kTile + n8 + 8 * i;
        float* p = Ox + (size_t)(grp * L::kRows + row) * L::kOPad;
        if (row < it.nr)
#pragma unroll
          for (int j = 0; j < NT; j += 2)
            *reinterpret_cast<float4*>(p + 8 * j + 4 * t) =
                make_float4(w.o[j][2 * i], w.o[j][2 * i + 1], w.o[j + 1][2 * i], w.o[j + 1][2 * i + 1]);
      }
    }
    __syncthreads();
    if (a.split > 1) {
      cluster_wait();  // nobody reads its ring any more
      if (tid < it.nr) {
        const float2 v = make_float2(s_gm[tid], s_sum[tid]);
        st_cluster_f32x2(in_block(&s_in[rank][tid], tid % a.split), v);
      }
    }
    finish_rows<T, HD, L::kGroups, L::kRows, L::kThreads>(
        a, sg, kb, ke, Ox, s_w, s_gm, s_sum, s_bad, tid, [&](int row, int c8, const float (&acc)[8]) {
          float* const p = parts + ((size_t)rank * (L::kRows / a.split) + row / a.split) * HD + c8;
          const uint32_t at = in_block(p, row % a.split);
          st_cluster_f32x4(at, make_float4(acc[0], acc[1], acc[2], acc[3]));
          st_cluster_f32x4(at + 16, make_float4(acc[4], acc[5], acc[6], acc[7]));
        });
    if (a.split) break;
    if (!sg.whole() && sg.u0 == 0 && tid == 0) a.desc[blockIdx.x] = kv8_desc(a, cur, sg);
    __syncthreads();
    more = kv8_next<L::kRows, kUnit>(a, cur, sg);
  }
  if (a.split > 1) {
    const Kv8Item& it = sg.it;
    if (!more) {  // no keys for this block: a sum of 0
      cluster_arrive();
      cluster_wait();
      if (tid < it.nr)
        st_cluster_f32x2(in_block(&s_in[rank][tid], tid % a.split), make_float2(-INFINITY, 0.f));
    }
    cluster_arrive();
    cluster_wait();  // every block's parts of this one's rows are here
    for (int x = tid; x < (it.nr + a.split - 1 - rank) / a.split * NT; x += L::kThreads) {
      const int mine = x / NT, row = mine * a.split + rank, c8 = (x % NT) * 8;
      float w[kSplitMax], gm = -INFINITY, sum = 0.f, acc[8];
      uint32_t has = 0;  // parts whose keys the row sees (of the others there may be nothing to read)
#pragma unroll
      for (int y = 0; y < kSplitMax; ++y) {
        if (y >= a.split) break;
        const float2 v = s_in[y][row];
        w[y] = v.y;
        if (v.y != 0.f) {
          has |= 1u << y;
          gm = fmaxf(gm, v.x);
        }
      }
#pragma unroll
      for (int y = 0; y < kSplitMax; ++y)
        if (has >> y & 1) {
          w[y] *= part_weight(s_in[y][row].x, gm);
          sum += w[y];
        }
      // (the parts are weighed by w / sum: w times a large value can be out of range; a row whose
      // every score is -inf has no sum)
      const float inv = 1.f / sum, none = sum == 0.f ? __uint_as_float(0x7fffffffu) : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = none;
#pragma unroll
      for (int y = 0; y < kSplitMax; ++y) {
        if (!(has >> y & 1)) continue;
        const float4* u = reinterpret_cast<const float4*>(
            parts + ((size_t)y * (L::kRows / a.split) + mine) * HD + c8);
        const float4 lo = u[0], hi = u[1];
        const float wt = w[y] * inv;
        acc[0] = fmaf(wt, lo.x, acc[0]);
        acc[1] = fmaf(wt, lo.y, acc[1]);
        acc[2] = fmaf(wt, lo.z, acc[2]);
        acc[3] = fmaf(wt, lo.w, acc[3]);
        acc[4] = fmaf(wt, hi.x, acc[4]);
        acc[5] = fmaf(wt, hi.y, acc[5]);
        acc[6] = fmaf(wt, hi.z, acc[6]);
        acc[7] = fmaf(wt, hi.w, acc[7]);
      }
      const int r = it.r0 + row, mr = a.byG(r), h = sg.g * a.G + r - mr * a.G;
      const int p = kv8_row_pos(a, it, r);
      const bool sees = kv8_row_lo(it, p, a.window) <= p;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = sees ? acc[j] : 0.f;
      store_out8(static_cast<T*>(a.out) + ((int64_t)it.b * a.M + mr) * a.out_stride +
                     (int64_t)h * HD + c8,
                 acc);
    }
  }
}

}  // namespace ssd

#include "paged_stream.cuh"
#include "paged_wide.cuh"

namespace ssd {

// ------------------------------------------------------------- host side

namespace {

struct PagedDevice {
  bool ready = false;
  int sms = 0;
};
std::mutex g_paged_mu;
PagedDevice g_paged_dev[64];

template <typename T, int HD, int R, int NB>
cudaError_t prep() {
  return cudaFuncSetAttribute(k_paged_rows<T, HD, R, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)PL<T, HD, R, NB>::kSmem);
}
template <int TILES>
cudaError_t prep_wide() {
  return cudaFuncSetAttribute(k_paged_wide<TILES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)PWideL<TILES>::kSmem);
}
template <int HD, int NB>
cudaError_t prep_stream() {
  return cudaFuncSetAttribute(k_paged_stream<HD, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)SL<HD, NB>::kSmem);
}
template <int HD>
cudaError_t prep_hd() {
  cudaError_t e = prep<float, HD, 1, 1>();
  if (e == cudaSuccess) e = prep<float, HD, 1, 2>();
  if (e == cudaSuccess) e = prep<__nv_bfloat16, HD, 1, 1>();
  if (e == cudaSuccess) e = prep<__nv_bfloat16, HD, 1, 2>();
  if (e == cudaSuccess) e = prep<__nv_bfloat16, HD, 2, 2>();
  if constexpr (HD == 64)
    if (e == cudaSuccess) e = prep<__nv_bfloat16, HD, 4, 2>();
  if (e == cudaSuccess) e = prep_stream<HD, 1>();
  if (e == cudaSuccess) e = prep_stream<HD, 2>();
  return e;
}

// SMs of the current device; its kernels' limits of shared memory are set on the first call
// there.
cudaError_t paged_device(int* sms) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_paged_mu);
  PagedDevice& d = g_paged_dev[dev];
  if (!d.ready) {
    if ((e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess ||
        (e = prep_hd<64>()) != cudaSuccess || (e = prep_hd<128>()) != cudaSuccess ||
        (e = prep_wide<1>()) != cudaSuccess || (e = prep_wide<2>()) != cudaSuccess)
      return e;
    d.ready = true;
  }
  *sms = d.sms;
  return cudaSuccess;
}

// Short sequences: a cluster of blocks for each item, which joins its parts itself (no workspace, no
// second launch): 1, 2, 4 or 8 blocks with 128 keys or more each, as long as there is room for all, two
// on each of 152 SMs; up to 512 keys a block and 2048 in all (fp32 1024, and 512 for more than 8 rows,
// whose blocks are bound by their multiply-adds). What counts is how many keys an item's rows can see:
// what the caller says of the lengths, or the window. us on the GPU, line / clusters, all sequences of
//                                   128       512        1024       2048       4096 positions
//   1 x 8 KV heads, 4 rows       9.5/5.1    9.5/7.2    9.9/7.9  10.2/10.0  11.3/14.3
//   1 x 8, 16 rows              12.5/6.6   13.2/8.7   13.6/9.5  13.8/11.7  15.0/16.4
//   1 x 40, 2 rows              10.2/5.5   10.6/7.8  12.8/10.3  15.4/15.3  20.8/25.1
//   16 x 8, 4 rows              12.9/5.6  16.6/10.5  21.7/15.3  32.3/27.4  51.3/46.9
//   1 x 8, 32 rows              11.6/8.3  12.5/10.6  13.5/11.2  14.8/15.1  15.8/23.0
//   fp32, 1 x 4, 1 row           8.5/6.1    8.7/7.8    8.9/8.4   8.7/10.6   9.7/14.6
//   fp32, 1 x 4, 12 rows       12.4/11.4  12.8/13.1  12.8/14.2  12.9/21.1  15.4/35.5
// (sequences of one length, for which clusters are at their best.)
// More than 16 rows a KV head, bf16 and head_dim 128: tcgen05 tiles, but for 17 to 32 rows where there are
// clusters. us, k_paged_rows / k_paged_wide, 8 KV heads, sequences x keys:
//                   17 rows       32         33         64
//   1 x 250       10.5/11.8  10.9/11.8  14.5/12.1  15.9/12.2
//   1 x 1000      10.7/14.2  11.2/14.2  13.8/14.3  14.7/14.7
//   1 x 4000      18.0/15.9  18.9/16.2  22.2/16.2  23.9/16.7
//   16 x 250      12.4/20.3  13.0/20.5  16.9/20.6  18.7/21.4
//   16 x 1000     26.5/28.7  27.6/29.0  39.9/29.4  42.4/30.8
//   16 x 16000     269/179    271/182    426/183    436/187
constexpr int kSplitKeys = 128, kSplitBlocks = 304, kSplitSeq = 512;

struct PagedPlan {
  int wide;   // accumulators of a tile on tcgen05, 0: mma.sync
  bool stream;  // k_paged_stream
  int tiles;  // warps of a block that have rows of their own each
  int eights;  // a warp's rows by eights
  int split;  // blocks of an item's own, 0: the line
  int max_blocks, part_rows;
  long long n_rt, units;  // tiles of a sequence; the line's places, at most
};
PagedPlan plan_of(const ssd_paged_cache* c, int n_heads, int M, int longest, int window) {
  PagedPlan p;
  const long long rows = (long long)M * (n_heads / c->n_kv_heads);
  const long long heads = (long long)c->n_seq * c->n_kv_heads;
  p.tiles = c->dtype == SSD_DTYPE_F32 || rows <= kTile ? 1 : rows <= 2 * kTile ? 2 : 4;
  p.eights = rows > 8 ? 2 : 1;
  int rt = p.tiles * p.eights * 8;
  p.n_rt = (rows + rt - 1) / rt;
  long long items = p.n_rt * heads;
  // keys that an item's rows see, at most
  const int span = window > 0 && window < longest - M ? window + M : longest;
  p.split = 1;
  while (p.split < kSplitMax && span > kSplitKeys * p.split && items * p.split * 2 <= kSplitBlocks)
    p.split *= 2;
  const int most = c->dtype == SSD_DTYPE_BF16 ? 2048 : rows > 8 ? 512 : 1024;
  if (span > kSplitSeq * p.split || span > most) p.split = 0;
  p.wide = 0;
  if (c->dtype == SSD_DTYPE_BF16 && c->head_dim == kWHd && rows > (p.split ? 2 * kTile : kTile)) {
    p.wide = rows > kWRows ? 2 : 1;
    p.split = 0;
    rt = p.wide * kWRows;
    p.n_rt = (rows + rt - 1) / rt;
    items = p.n_rt * heads;
  }
  p.stream = !p.wide && !p.split && c->dtype == SSD_DTYPE_BF16 && rows <= kTile;
  p.part_rows = rows < rt ? (int)rows : rt;
  p.units = items * ((span + 2 * kUnit - 2) / kUnit +
                     (p.wide == 2 ? kKv8ItemCost<256> : kKv8ItemCost<kTile>));
  p.max_blocks = p.wide || p.stream ? kKv8MaxBlocks / 2 : kKv8MaxBlocks;
  if (p.units < p.max_blocks) p.max_blocks = (int)p.units;
  return p;
}

const char* check_attention(const ssd_paged_cache* c, int32_t n_heads, int32_t M, int32_t window,
                            int32_t longest, PagedPlan* plan, ssd_status* status) {
  if (const char* why = check_paged(c, status)) return why;
  *status = SSD_ERR_INVALID_ARG;
  if (n_heads < c->n_kv_heads || n_heads % c->n_kv_heads || n_heads > 65536)
    return "n_heads must be a multiple of the cache's n_kv_heads";
  if (M < 1) return "M must be at least 1";
  if (window < 0) return "window must be 0 (none) or positive";
  if (longest < 0) return "longest must be 0 (the cache's positions) or positive";
  *status = SSD_ERR_CAPACITY;
  const int cap = c->max_pages * c->page;
  if (M > cap) return "more rows than the cache has positions";
  if (longest > cap) return "longest: more than the cache has positions";
  // (a tile's first row is an int, also of those behind the rows that a short `longest` leaves)
  if ((long long)M * (n_heads / c->n_kv_heads) > 0x7fffffffll - 256)
    return "M x n_heads / n_kv_heads: more than 2^31 rows of a KV head";
  *plan = plan_of(c, n_heads, M, longest ? longest : cap, window);
  if (plan->units > 0x7fffffffll) return "n_seq x M x longest: more than 2^31 units of work";
  *status = SSD_OK;
  return nullptr;
}

template <typename T, int HD, int R, int NB>
cudaError_t rows_launch(const PagedAttn& a, int P, cudaStream_t st) {
  using L = PL<T, HD, R, NB>;
  const cudaError_t e = launch_first(k_paged_rows<T, HD, R, NB>, dim3(P), L::kThreads, L::kSmem,
                                     a.split > 1 ? a.split : 1, st, a);
  if (e != cudaSuccess || a.split) return e;
  return R == 1 ? merge_launch<T, HD, kMWarps>(a, P, st) : merge_launch<T, HD, 1>(a, P, st);
}
template <int HD, int NB>
cudaError_t stream_launch(const PagedAttn& a, int P, cudaStream_t st) {
  using L = SL<HD, NB>;
  const cudaError_t e = launch_first(k_paged_stream<HD, NB>, dim3(P), L::kThreads, L::kSmem, 1, st, a);
  return e != cudaSuccess ? e : merge_launch<__nv_bfloat16, HD, kMWarps>(a, P, st);
}
template <int TILES>
cudaError_t wide_launch(const PagedAttn& a, int P, cudaStream_t st) {
  using L = PWideL<TILES>;
  const cudaError_t e = launch_first(k_paged_wide<TILES>, dim3(P), L::kThreads, L::kSmem, 1, st, a);
  return e != cudaSuccess ? e : merge_launch<__nv_bfloat16, kWHd, 1>(a, P, st);
}
template <int HD>
cudaError_t launch(const PagedAttn& a, int dtype, const PagedPlan& p, int P, cudaStream_t st) {
  using B = __nv_bfloat16;
  if (dtype == SSD_DTYPE_F32)
    return p.eights == 1 ? rows_launch<float, HD, 1, 1>(a, P, st) : rows_launch<float, HD, 1, 2>(a, P, st);
  if (p.wide) return p.wide == 2 ? wide_launch<2>(a, P, st) : wide_launch<1>(a, P, st);
  if (p.stream) return p.eights == 1 ? stream_launch<HD, 1>(a, P, st) : stream_launch<HD, 2>(a, P, st);
  if (p.eights == 1) return rows_launch<B, HD, 1, 1>(a, P, st);
  if (p.tiles == 1) return rows_launch<B, HD, 1, 2>(a, P, st);
  if constexpr (HD == 64)
    if (p.tiles == 4) return rows_launch<B, HD, 4, 2>(a, P, st);
  return rows_launch<B, HD, 2, 2>(a, P, st);
}

}  // namespace
}  // namespace ssd

extern "C" size_t ssd_paged_attention_bytes(const ssd_paged_cache* c, int32_t n_heads, int32_t M,
                                            int32_t window, int32_t longest) {
  using namespace ssd;
  ssd_status status;
  PagedPlan p;
  if (const char* why = check_attention(c, n_heads, M, window, longest, &p, &status)) {
    fail_op(status, why);
    return 0;
  }
  return p.split ? 256 : kv8_work(p.max_blocks, p.part_rows, c->head_dim).total;
}

extern "C" ssd_status ssd_paged_attention(const ssd_paged_cache* c, int32_t layer, const void* q,
                                          int32_t n_heads, int64_t q_stride, int32_t M,
                                          const int32_t* pos, const int32_t* rows,
                                          const int32_t* first, int32_t window, int32_t longest,
                                          void* out, int64_t out_stride, void* workspace,
                                          size_t workspace_bytes, int32_t* err_dev, void* stream) {
  using namespace ssd;
  ssd_status status;
  PagedPlan plan;
  if (const char* why = check_attention(c, n_heads, M, window, longest, &plan, &status))
    return fail_op(status, why);
  if (layer < 0 || layer >= c->n_layers)
    return fail_op(SSD_ERR_INVALID_ARG, "layer must be in 0..n_layers - 1");
  const int elt = c->dtype == SSD_DTYPE_BF16 ? 2 : 4;
  const int64_t len = (int64_t)n_heads * c->head_dim;
  if (!q || !out || !pos || ((uintptr_t)q & 15u) || ((uintptr_t)out & 15u))
    return fail_op(SSD_ERR_INVALID_ARG, "q, out or pos: NULL or unaligned pointer");
  if (q_stride < len || out_stride < len || q_stride > (1ll << 40) || out_stride > (1ll << 40) ||
      (q_stride * elt) % 16 || (out_stride * elt) % 16)
    return fail_op(SSD_ERR_INVALID_ARG,
                   "q_stride or out_stride: below a row's length, or not a multiple of 16 bytes");
  if (out == q && out_stride != q_stride)
    return fail_op(SSD_ERR_INVALID_ARG, "out is q, but their strides differ");
  const Kv8Work lay = kv8_work(plan.max_blocks, plan.part_rows, c->head_dim);
  if (!plan.split) {
    if (!workspace || ((uintptr_t)workspace & 255u))
      return fail_op(SSD_ERR_INVALID_ARG, "workspace must be non-NULL and 256-byte aligned");
    if (workspace_bytes < lay.total) return fail_op(SSD_ERR_CAPACITY, "workspace too small");
  }
  int sms = 0;
  cudaError_t e = paged_device(&sms);
  if (e != cudaSuccess) return fail_op_cuda("ssd_paged_attention", e);
  PagedAttn a{};
  a.c = paged_view(c);
  a.k = a.c.pages + a.c.side(layer, 0);
  a.v = a.c.pages + a.c.side(layer, 1);
  a.q = q;
  a.out = out;
  a.pos = pos;
  a.rows = rows;
  a.first = first;
  a.err = err_dev;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.n_seq = c->n_seq;
  a.Hkv = c->n_kv_heads;
  a.G = n_heads / c->n_kv_heads;
  a.M = M;
  a.max_seq = longest ? longest : c->max_pages * c->page;
  a.window = window;
  a.n_rt = (int)plan.n_rt;
  a.entries = (int)plan.n_rt * c->n_seq;
  a.scale = (float)(1.4426950408889634 / sqrt((double)c->head_dim));
  char* ws = static_cast<char*>(workspace);
  a.desc = reinterpret_cast<Kv8Desc*>(ws);
  a.ml = reinterpret_cast<float2*>(ws + lay.ml);
  a.part = reinterpret_cast<float*>(ws + lay.part);
  a.byG = Kv8Div::of((uint32_t)a.G);
  a.byRt = Kv8Div::of((uint32_t)plan.n_rt);
  int P = sms * (plan.wide || plan.stream ? 1 : 2);  // blocks of an SM
  if (P > plan.max_blocks) P = plan.max_blocks;
  a.part_rows = plan.part_rows;
  a.split = plan.split;
  if (plan.split) P = a.entries * a.Hkv * plan.split;
  a.byP = Kv8Div::of((uint32_t)P);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  e = c->head_dim == 128 ? launch<128>(a, c->dtype, plan, P, st) : launch<64>(a, c->dtype, plan, P, st);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_paged_attention", e);
}
