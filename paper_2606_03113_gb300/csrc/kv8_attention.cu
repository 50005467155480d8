// kv8_attention.cu -- attention of new rows over the 8-bit cache (kv8.cuh), for
// 1 row a sequence (decoding) up to prompt chunks, with grouped queries:
//   o_r = sum_j p_rj v_j / sum_j p_rj,  p_rj = e^(q_r . k_j / sqrt(hd) - max),
// over the keys j that row r sees: first .. its own position, at most `window`.
//
// k_kv8_rows: a block takes a stretch of the plan's units (kv8_plan.cuh), or, for short
// caches, a cluster of blocks an item; its four warps take the 16-key steps of an item
// in turn, each with its own running maximum, sum and output, and the block joins the
// warps once per item.  Queries
// and probabilities are f16 operands of mma.sync against the codes, which f16
// holds exactly; a row of queries is first brought near f16's upper end by a
// power of two, so a bf16 query is exact down to 2^-28 of its row's largest, and
// the probabilities are scaled by 2^15, so those above 2^-29 of the running
// maximum keep f16's 11 bits.  fp32 queries and probabilities enter as two f16
// parts, 22 bits.  Scores, sums and outputs are fp32.
//
// The places of a lane in the matrix fragments can be any as long as both
// operands agree, so they are chosen such that a lane's codes lie in 16
// consecutive bytes of a key.  Each warp copies its own steps to shared memory,
// whole lines at a time (cp.async, kRing steps ahead; lane by lane, as the
// fragments read them, the same copies reach 4.9 TB/s and not 6.3), and waits for no
// other warp until the end of an item.
//
// Bound by bytes for long caches, with the latencies of two warps a scheduler close
// behind (issue slots 49 %, ALU 45 % in use): 32 heads over 8 KV heads x 131072 keys 54 us
// = 4.95 TB/s, 24 ragged sequences of 32 heads, 5 rows, window 2500,
// 85 us = 4.4 TB/s.  Two blocks of four warps an SM, 244 registers a thread; three
// of 168 take 59 us for those 54.
//
// A key that some row of the tile does not see can hold anything: its scores are
// dropped by position, and a NaN code of such a value row is zeroed before the
// product and put back, row by row, for the rows that see it.
#include <math.h>

#include <mutex>
#include <type_traits>

#include "kv8_plan.cuh"
#include "mma.cuh"
#include "tc.cuh"

namespace ssd {

namespace {

constexpr int kRT = 16;       // query rows of a tile
constexpr int kStep = 16;     // keys of a warp's step
constexpr int kRing = 5;      // steps in flight per warp
constexpr int kVWarps = 4;
constexpr int kVBlocks = 2;   // blocks of an SM
constexpr int kVThreads = kVWarps * 32;
constexpr int kKv8MaxBlocks = 320;
constexpr int kSplitMax = 8;  // blocks of a short cache's item, a cluster, at most

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t half2_bits(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 half2_floats(uint32_t u) {
  return __half22float2(*reinterpret_cast<const __half2*>(&u));
}
// The ring of a warp: steps of 16 keys, then their values, rows of HD bytes.
template <int HD>
struct RowsL {
  static constexpr int kCpr = HD / 16;                  // 16-byte chunks of a row
  static constexpr int kCopies = kStep * kCpr / 32;     // a lane's copies of a step's keys
  static constexpr uint32_t kKBytes = kStep * HD;
  static constexpr uint32_t kStepBytes = 2 * kKBytes;
  static constexpr uint32_t kWarpBytes = kRing * kStepBytes;
  static constexpr int kOPad = HD + 4;            // floats of a row in the warps' exchange
  static constexpr uint32_t kQOff = kVWarps * kWarpBytes;
  template <int PARTS>
  static constexpr uint32_t total() {
    return kQOff + PARTS * kRT * HD * 2;
  }
  // Where chunk ch of key kk stands: its place in the row is moved by the key, so
  // that eight lanes meet all banks, both as two keys x four chunks (scores) and
  // as four keys of one parity x two chunks (values; two by two at HD 64).
  __device__ static __forceinline__ uint32_t place(int kk, int ch) {
    const int x = HD == 128 ? ((kk >> 1 & 3) << 1) ^ ((kk & 1) << 2) : kk >> 1 & 3;
    return (uint32_t)(kk * HD + ((ch ^ x) << 4));
  }
  static_assert(kVWarps * kRT * kOPad * 4 + kRT * HD * 4 <= kVWarps * kWarpBytes,
                "the exchange and the part fit the ring");
};

__device__ __forceinline__ void load_query8(const float* p, float (&f)[8]) {
  const float4 x = __ldg(reinterpret_cast<const float4*>(p));
  const float4 y = __ldg(reinterpret_cast<const float4*>(p) + 1);
  f[0] = x.x, f[1] = x.y, f[2] = x.z, f[3] = x.w;
  f[4] = y.x, f[5] = y.y, f[6] = y.z, f[7] = y.w;
}
__device__ __forceinline__ void load_query8(const __nv_bfloat16* p, float (&f)[8]) {
  Elem<__nv_bfloat16>::unpack(__ldg(reinterpret_cast<const uint4*>(p)), f);
}
__device__ __forceinline__ void store_out8(float* p, const float (&f)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  *(reinterpret_cast<float4*>(p) + 1) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store_out8(__nv_bfloat16* p, const float (&f)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
    u[j] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}
// 2^(m - max), the weight of a part whose maximum is m; 0 for a part without keys.
__device__ __forceinline__ float part_weight(float m, float mx) {
  return exp2f(m - (mx == -INFINITY ? 0.f : mx));
}

}  // namespace

template <typename T, int HD>
__global__ void __launch_bounds__(kVThreads, kVBlocks) k_kv8_rows(const Kv8Attn a) {
  using L = RowsL<HD>;
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  constexpr int NT = HD / 8;   // 8-column tiles of the output
  constexpr int KS = HD / 16;  // 16-column steps of a score
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ Kv8PlanSmem s_plan;
  __shared__ float s_qs[kRT];  // scores = dot * s_qs * key scale
  __shared__ float s_m[kVWarps][kRT], s_l[kVWarps][kRT], s_ref[kVWarps][kRT];
  __shared__ float s_w[kVWarps][kRT], s_gm[kRT], s_sum[kRT];  // the warps' weights, the row's (max, sum)
  __shared__ int s_nan;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t = lane & 3, n8 = lane >> 2;
  unsigned char* const wring = smem + warp * L::kWarpBytes;
  unsigned char* const Qs = smem + L::kQOff;
  float* const Ox = reinterpret_cast<float*>(smem);
  float* const part = Ox + kVWarps * kRT * L::kOPad;  // [kRT][HD]: the block's part of a cluster's item

  Kv8Cursor cur = kv8_plan<kRT, kKv8Block, kVThreads>(a, s_plan);
  pdl_launch_dependents();
  if (tid == 0 && !a.split) a.desc[blockIdx.x].nr = 0;
  if (tid < kRT) s_sum[tid] = 0.f;
  Kv8Seg sg;
  while (kv8_next<kRT, kKv8Block>(a, cur, sg)) {
    const Kv8Item& it = sg.it;
    const int g = sg.g;

    // ---- queries of the tile: read before the keys, whose copies they would wait behind
    constexpr int kLanes = HD / 8;  // lanes of a row
    constexpr int kQPasses = (kRT * kLanes + kVThreads - 1) / kVThreads;
    float fq[kQPasses][8];
#pragma unroll
    for (int x = 0; x < kQPasses; ++x) {
      const int row = (x * kVThreads + tid) / kLanes, ch = tid % kLanes;
#pragma unroll
      for (int j = 0; j < 8; ++j) fq[x][j] = 0.f;
      if (row < it.nr) {
        const int r = it.r0 + row, m = a.byG(r), h = g * a.G + r - m * a.G;
        load_query8(static_cast<const T*>(a.q) + ((int64_t)it.b * a.M + m) * a.q_stride +
                        (int64_t)h * HD + ch * 8,
                    fq[x]);
      }
    }

    // ---- keys of the segment, by 16-key steps
    const int seg0 = (it.unit0 + sg.u0) * kKv8Block;
    const int kb = max(it.lo & ~(kStep - 1), seg0);
    const int ke = min(it.hi + 1, seg0 + sg.nu * kKv8Block);
    const int nsteps = ke > kb ? (ke - kb + kStep - 1) / kStep : 0;
    const size_t slab = (size_t)it.b * a.Hkv + g;
    const uint8_t* kp = a.k + slab * a.max_seq * HD;
    const uint8_t* vp = a.v + slab * a.max_seq * HD;
    const float* ksp = a.ks + slab * (a.max_seq / kKv8Block);
    const float* vsp = a.vs + slab * (a.max_seq / kKv8Block);
    // every row sees keys full_lo .. full_hi
    const int full_lo = kv8_row_lo(it, it.hi, a.window);
    const int full_hi = kv8_row_pos(a, it, it.r0);
    auto issue = [&](int s) {  // the warp's codes of step s, whole lines at a time
      if (s < nsteps) {
        const int k0 = kb + s * kStep;
        const uint32_t dst = smem_u32(wring) + (uint32_t)((s / kVWarps) % kRing) * L::kStepBytes;
#pragma unroll
        for (int i = 0; i < L::kCopies; ++i) {
          const int kk = i * (32 / L::kCpr) + lane / L::kCpr, ch = lane % L::kCpr;
          const bool in = k0 + kk >= it.lo && k0 + kk <= it.hi;
          const size_t off = (size_t)(in ? k0 + kk : it.hi) * HD + ch * 16;
          const uint32_t at = dst + L::place(kk, ch);
          cp_async16(at, kp + off, in);
          cp_async16(at + L::kKBytes, vp + off, in);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };

#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) issue(warp + i * kVWarps);
    float nks = 0.f, nvs = 0.f;
    if (warp < nsteps) {
      nks = __ldg(ksp + (kb + warp * kStep) / kKv8Block);
      nvs = __ldg(vsp + (kb + warp * kStep) / kKv8Block);
    }

    // the queries in the order of the matrix fragments
    if (tid == 0) s_nan = 0;
#pragma unroll
    for (int x = 0; x < kQPasses; ++x) {
      const int row = (x * kVThreads + tid) / kLanes, ch = tid % kLanes;
      float (&f)[8] = fq[x];
      float amax = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(f[j]));
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1)
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      // the row's largest magnitude to [2^13, 2^14)
      const int ex = min(max((int)(__float_as_uint(amax) >> 23) - 127 - 13, -100), 115);
      const float inv = pow2i(-ex);
      if (row < kRT) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float u = f[j] * inv, w = f[j + 1] * inv;
          const uint32_t hi = half2_bits(u, w);
          const int c = ch * 8 + j;  // lane c / 16 % 4 of the row, its step c / 64 * 4 + c / 4 % 4
          unsigned char* p = Qs + (((c / 64 * 4 + c / 4 % 4) * 32 + (row & 7) * 4 + c / 16 % 4) * 4 +
                                   (c % 4) + (row >> 3)) *
                                      4;
          *reinterpret_cast<uint32_t*>(p) = hi;
          if constexpr (PARTS == 2) {
            const float2 v = half2_floats(hi);
            *reinterpret_cast<uint32_t*>(p + kRT * HD * 2) = half2_bits(u - v.x, w - v.y);
          }
        }
        if (ch == 0) s_qs[row] = pow2i(ex) * a.scale;
      }
    }
    __syncthreads();

    int plo[2], phi[2];
    float qs[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = n8 + 8 * i;
      phi[i] = row < it.nr ? kv8_row_pos(a, it, it.r0 + row) : -1;  // no row here: sees none
      plo[i] = row < it.nr ? kv8_row_lo(it, phi[i], a.window) : 0;
      qs[i] = s_qs[row];
    }
    uint32_t qf[PARTS == 1 ? KS : 1][4];
    if constexpr (PARTS == 1)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const uint4 u = *reinterpret_cast<const uint4*>(Qs + (k * 32 + lane) * 16);
        qf[k][0] = u.x, qf[k][1] = u.y, qf[k][2] = u.z, qf[k][3] = u.w;
      }

    float o[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[j][i] = 0.f;
    // running maximum and sum of the lane's rows; a row's output stands in units of
    // the largest value scale that it has seen, rref is one over that
    float mx[2] = {-INFINITY, -INFINITY}, ls[2] = {0.f, 0.f}, rref[2] = {pow2i(126), pow2i(126)};
    for (int s = warp; s < nsteps; s += kVWarps) {
      __syncwarp();  // every lane has read the step whose place is filled now
      issue(s + (kRing - 1) * kVWarps);
      const float ks = nks, vs = nvs;
      if (s + kVWarps < nsteps) {
        nks = __ldg(ksp + (kb + (s + kVWarps) * kStep) / kKv8Block);
        nvs = __ldg(vsp + (kb + (s + kVWarps) * kStep) / kKv8Block);
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
      __syncwarp();
      const int k0 = kb + s * kStep;
      const unsigned char* sp = wring + (uint32_t)((s / kVWarps) % kRing) * L::kStepBytes;

      // scores: 2 tiles of 8 keys, even and odd 16-column steps summed apart
      float sc[2][2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) sc[i][n][x] = 0.f;
#pragma unroll
      for (int hf = 0; hf < HD / 64; ++hf) {
        uint4 kw[2];
#pragma unroll
        for (int n = 0; n < 2; ++n)
          kw[n] = *reinterpret_cast<const uint4*>(sp + L::place(8 * n + n8, hf * 4 + t));
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int k = hf * 4 + q4;
          uint32_t kf[2][2];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const uint32_t x = q4 == 0 ? kw[n].x : q4 == 1 ? kw[n].y : q4 == 2 ? kw[n].z : kw[n].w;
            kf[n][0] = e4m3_to_half2(x);
            kf[n][1] = e4m3_to_half2(x >> 16);
          }
          if constexpr (PARTS == 1) {
            mma_f16(sc[q4 & 1][0], qf[k], kf[0][0], kf[0][1]);
            mma_f16(sc[q4 & 1][1], qf[k], kf[1][0], kf[1][1]);
          } else {
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) {
              const uint4 u =
                  *reinterpret_cast<const uint4*>(Qs + p * kRT * HD * 2 + (k * 32 + lane) * 16);
              const uint32_t qa[4] = {u.x, u.y, u.z, u.w};
              mma_f16(sc[q4 & 1][0], qa, kf[0][0], kf[0][1]);
              mma_f16(sc[q4 & 1][1], qa, kf[1][0], kf[1][1]);
            }
          }
        }
      }
      const bool full = k0 >= full_lo && k0 + kStep - 1 <= full_hi;
      float z[2][4], nm[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          z[n][x] = (sc[0][n][x] + sc[1][n][x]) * kv8_factor(qs[x >> 1], ks);
          if (!full) {
            const int key = k0 + 8 * n + 2 * t + (x & 1);
            if (key < plo[x >> 1] || key > phi[x >> 1]) z[n][x] = -INFINITY;
          }
          nm[x >> 1] = fmaxf(nm[x >> 1], z[n][x]);
        }
      float f[2];
      bool moved = false, up[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        nm[i] = fmaxf(nm[i], __shfl_xor_sync(0xffffffffu, nm[i], 1));
        nm[i] = fmaxf(nm[i], __shfl_xor_sync(0xffffffffu, nm[i], 2));
        up[i] = vs * rref[i] > 1.f && nm[i] > -INFINITY;
        nm[i] = fmaxf(nm[i], mx[i]);
        f[i] = nm[i] == mx[i] ? 1.f : exp2f(mx[i] - nm[i]);
        moved |= nm[i] != mx[i] || up[i];
        mx[i] = nm[i];
        ls[i] *= f[i];
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (up[i]) {
            f[i] *= 1.f / (vs * rref[i]);
            rref[i] = 1.f / vs;
          }
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[j][x] *= f[x >> 1];
      }
      uint32_t pf[PARTS][4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          // (rounded up: no probability passes 2^15 where the maximum's unit is above 1)
          const float top = mx[i] == -INFINITY ? 0.f : __fadd_ru(mx[i], -15.f);
          const float vrel = fminf(vs * rref[i], 1.f);  // (above 1: a row that sees no key here)
          const float x = exp2f(z[n][2 * i] - top), y = exp2f(z[n][2 * i + 1] - top);
          ls[i] += x + y;
          pf[0][2 * n + i] = half2_bits(x * vrel, y * vrel);
          if constexpr (PARTS == 2) {
            const float2 v = half2_floats(pf[0][2 * n + i]);
            pf[1][2 * n + i] = half2_bits(x * vrel - v.x, y * vrel - v.y);
          }
        }
      // values: words of the lane's four keys
      uint32_t vw[4][NT / 4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int kk = 2 * t + (c & 1) + 8 * (c >> 1);
        const unsigned char* p = sp + L::kKBytes + (HD == 128 ? L::place(kk, n8)
                                                              : L::place(kk, n8 >> 1) + 8 * (n8 & 1));
        if constexpr (HD == 128) {
          const uint4 u = *reinterpret_cast<const uint4*>(p);
          vw[c][0] = u.x, vw[c][1] = u.y, vw[c][2] = u.z, vw[c][3] = u.w;
        } else {
          const uint2 u = *reinterpret_cast<const uint2*>(p);
          vw[c][0] = u.x, vw[c][1] = u.y;
        }
      }
      if (!full) {
        uint32_t any = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int j = 0; j < NT / 4; ++j) {
            const uint32_t m = e4m3_nan_mask(vw[c][j]);
            any |= m;
            vw[c][j] &= ~((m >> 7) * 0xffu);
          }
        if (any) s_nan = 1;
      }
#pragma unroll
      for (int j4 = 0; j4 < NT / 4; ++j4) {
        // bytes (key, key + 1) of columns j4 * 4 .. + 3
        const uint32_t a01 = __byte_perm(vw[0][j4], vw[1][j4], 0x5140);
        const uint32_t a23 = __byte_perm(vw[0][j4], vw[1][j4], 0x7362);
        const uint32_t b01 = __byte_perm(vw[2][j4], vw[3][j4], 0x5140);
        const uint32_t b23 = __byte_perm(vw[2][j4], vw[3][j4], 0x7362);
        const uint32_t lo[4] = {e4m3_to_half2(a01), e4m3_to_half2(a01 >> 16), e4m3_to_half2(a23),
                                e4m3_to_half2(a23 >> 16)};
        const uint32_t hi[4] = {e4m3_to_half2(b01), e4m3_to_half2(b01 >> 16), e4m3_to_half2(b23),
                                e4m3_to_half2(b23 >> 16)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p) mma_f16(o[j4 * 4 + j], pf[p], lo[j], hi[j]);
        }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");

    // ---- the warps' parts together
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ls[i] += __shfl_xor_sync(0xffffffffu, ls[i], 1);
      ls[i] += __shfl_xor_sync(0xffffffffu, ls[i], 2);
      if (t == 0) {
        s_m[warp][n8 + 8 * i] = mx[i];
        s_l[warp][n8 + 8 * i] = ls[i];
        s_ref[warp][n8 + 8 * i] = 1.f / rref[i];
      }
    }
    __syncthreads();  // nobody reads the ring any more
    const int nw = min(nsteps, kVWarps);
    if (tid < kRT) {
      float gm = -INFINITY, sum = 0.f;
      for (int x = 0; x < nw; ++x) gm = fmaxf(gm, s_m[x][tid]);
      for (int x = 0; x < nw; ++x) sum = fmaf(part_weight(s_m[x][tid], gm), s_l[x][tid], sum);
      for (int x = 0; x < nw; ++x)
        s_w[x][tid] = sum != 0.f ? part_weight(s_m[x][tid], gm) / sum : 0.f;
      s_gm[tid] = gm;
      s_sum[tid] = sum;
    }
    if (warp < nw) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = n8 + 8 * (i >> 1);
        if (row < it.nr) {
          float* p = Ox + (size_t)(warp * kRT + row) * L::kOPad + (2 * t + (i & 1)) * NT;
#pragma unroll
          for (int j = 0; j < NT; j += 4)
            *reinterpret_cast<float4*>(p + j) =
                make_float4(o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]);
        }
      }
    }
    __syncthreads();
    const bool whole = sg.whole();
    const int slot = 2 * blockIdx.x + (sg.u0 == 0);
#pragma unroll 1
    for (int x0 = 0; x0 < kRT * NT; x0 += kVThreads) {
      const int row = (x0 + tid) / NT, c8 = (tid % NT) * 8;
      if (row < it.nr) {
        const int r = it.r0 + row, m = a.byG(r), h = g * a.G + r - m * a.G;
        const int p = kv8_row_pos(a, it, r), lo = kv8_row_lo(it, p, a.window);
        const float gm = s_gm[row], Ls = s_sum[row];
        float acc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        for (int x = 0; x < nw; ++x) {
          const float wt = s_w[x][row], rf = s_ref[x][row];
          const float4* ox = reinterpret_cast<const float4*>(Ox + (size_t)(x * kRT + row) * L::kOPad + c8);
          const float4 u = ox[0], w = ox[1];
          // (the weight before the unit: their product can be out of range)
          acc[0] = fmaf(u.x * wt, rf, acc[0]);
          acc[1] = fmaf(u.y * wt, rf, acc[1]);
          acc[2] = fmaf(u.z * wt, rf, acc[2]);
          acc[3] = fmaf(u.w * wt, rf, acc[3]);
          acc[4] = fmaf(w.x * wt, rf, acc[4]);
          acc[5] = fmaf(w.y * wt, rf, acc[5]);
          acc[6] = fmaf(w.z * wt, rf, acc[6]);
          acc[7] = fmaf(w.w * wt, rf, acc[7]);
        }
        if (s_nan) {  // a NaN value belongs to the rows that see its key
          for (int key = kb; key < ke; ++key) {
            const int k0 = key & ~(kStep - 1);  // the key's step (kb is one's first key)
            if (k0 >= full_lo && k0 + kStep - 1 <= full_hi) continue;  // nothing was zeroed there
            if (key < lo || key > p) continue;
            const uint2 u = *reinterpret_cast<const uint2*>(vp + (size_t)key * HD + c8);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t code = ((j < 4 ? u.x : u.y) >> (8 * (j & 3))) & 0x7fu;
              if (code == 0x7fu) acc[j] = __uint_as_float(0x7fffffffu);
            }
          }
        }
        if (a.split > 1) {
          store_out8(part + row * HD + c8, acc);
        } else if (whole) {
          if (p < lo) {  // sees no key
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = 0.f;
          } else if (Ls == 0.f) {
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = __uint_as_float(0x7fffffffu);
          }
          store_out8(static_cast<T*>(a.out) + ((int64_t)it.b * a.M + m) * a.out_stride +
                         (int64_t)h * HD + c8,
                     acc);
        } else {
          store_out8(a.part + ((size_t)slot * a.part_rows + row) * HD + c8, acc);
          if (c8 == 0) a.ml[(size_t)slot * a.part_rows + row] = make_float2(gm, Ls);
        }
      }
    }
    if (!a.split && !whole && sg.u0 == 0 && tid == 0) a.desc[blockIdx.x] = kv8_desc(a, cur, sg);
    __syncthreads();
  }
  if (a.split > 1) {  // the cluster's parts together, each block some of the columns
    const int i = (int)blockIdx.x / a.split, rank = (int)blockIdx.x - i * a.split;
    const int e = i / a.Hkv, g = i - e * a.Hkv;
    const Kv8Item it = kv8_entry<kRT, kKv8Block>(a, e);
    cluster_sync();
    for (int x = rank * kVThreads + tid; x < it.nr * NT; x += a.split * kVThreads) {
      const int row = x / NT, c8 = (x % NT) * 8;
      float w[kSplitMax], m[kSplitMax], gm = -INFINITY, sum = 0.f, acc[8];
#pragma unroll
      for (int y = 0; y < kSplitMax; ++y) {
        w[y] = y < a.split ? ld_cluster_f32(in_block(&s_sum[row], y)) : 0.f;
        m[y] = y < a.split ? ld_cluster_f32(in_block(&s_gm[row], y)) : 0.f;
      }
#pragma unroll
      for (int y = 0; y < kSplitMax; ++y)  // (a sum of 0: the row sees none of the part's keys)
        gm = fmaxf(gm, w[y] != 0.f ? m[y] : -INFINITY);
#pragma unroll
      for (int y = 0; y < kSplitMax; ++y) {
        if (w[y] != 0.f) w[y] *= part_weight(m[y], gm);
        sum += w[y];
      }
      // (the parts are weighed by w / sum: w times a large value can be out of range; a row whose
      // every score is -inf has no sum)
      const float inv = 1.f / sum, none = sum == 0.f ? __uint_as_float(0x7fffffffu) : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = none;
#pragma unroll
      for (int y = 0; y < kSplitMax; ++y) {
        if (w[y] == 0.f) continue;
        const uint32_t at = in_block(part + row * HD + c8, y);
        const float4 u = ld_cluster_f32x4(at), v = ld_cluster_f32x4(at + 16);
        const float wt = w[y] * inv;
        acc[0] = fmaf(wt, u.x, acc[0]);
        acc[1] = fmaf(wt, u.y, acc[1]);
        acc[2] = fmaf(wt, u.z, acc[2]);
        acc[3] = fmaf(wt, u.w, acc[3]);
        acc[4] = fmaf(wt, v.x, acc[4]);
        acc[5] = fmaf(wt, v.y, acc[5]);
        acc[6] = fmaf(wt, v.z, acc[6]);
        acc[7] = fmaf(wt, v.w, acc[7]);
      }
      const int r = it.r0 + row, mr = a.byG(r), h = g * a.G + r - mr * a.G;
      const int p = kv8_row_pos(a, it, r);
      const bool sees = kv8_row_lo(it, p, a.window) <= p;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = sees ? acc[j] : 0.f;
      store_out8(static_cast<T*>(a.out) + ((int64_t)it.b * a.M + mr) * a.out_stride +
                     (int64_t)h * HD + c8,
                 acc);
    }
    cluster_sync();  // everybody has read this block's part
  }
}

}  // namespace ssd

#include "kv8_wide.cuh"

namespace ssd {

// Joins the parts of the items that several blocks shared: blocks (i, *) those of
// the item that begins in block i's stretch.  WPR warps share a row: warp w of them
// takes parts w, w + WPR, ..; their sums are added in order.
// Bound by round trips to L2: a part's place depends on the item alone, so the
// first parts are on their way while the weights are worked out.  Few rows have many
// parts and get a block a row; many rows have few and get a warp.  About 6 of
// the 75 us of 512 rows of 32 heads over 7936 keys.
constexpr int kMWarps = 8;
// Blocks that share an item's rows, at most; parts of a warp on their way; blocks of an SM.
// A warp a row: 17 rows of 64 heads over 8 x 16000 keys, 512 of 32 over 8 x 7936: 33.8 and 77.3 us
// as for few rows, 30.6 and 75.5 so; two warps a row 32.0 and 84.8.
template <int WPR>
constexpr int kMRowBlocks = WPR == kMWarps ? 8 : 32;
template <int WPR>
constexpr int kMBatch = WPR == kMWarps ? 6 : 4;
template <int WPR>
constexpr int kMBlocks = WPR == kMWarps ? 3 : 4;

template <typename T, int HD, int RT, int WPR>
__global__ void __launch_bounds__(kMWarps * 32, kMBlocks<WPR>) k_kv8_merge(const Kv8Attn a) {
  constexpr int kC = HD / 32;  // columns of a lane
  constexpr int kBatch = kMBatch<WPR>;
  constexpr int kRows = kMWarps / WPR;
  using Vec = typename std::conditional<HD == 128, float4, float2>::type;
  __shared__ float2 s_ml[kRows][kKv8MaxBlocks + 1];
  __shared__ int s_slot[kKv8MaxBlocks + 1];
  __shared__ float s_red[kMWarps][HD];
  __shared__ float s_gm[kMWarps], s_sum[kMWarps];
  pdl_wait();
  const int i = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rl = warp / WPR, w = warp % WPR;
  const int4 d0 = __ldcg(reinterpret_cast<const int4*>(a.desc + i));
  const int4 d1 = __ldcg(reinterpret_cast<const int4*>(a.desc + i) + 1);
  if ((int)blockIdx.y * kRows >= d0.x) return;
  // its parts: one of each block i .. last, or, with fewer units than blocks, one
  // of each unit's block
  const Kv8Line line(a, d1.y);
  const int last = d1.x, u0 = line.start(a, i);
  const bool dense = line.q > 0;
  const int n = dense ? last - i + 1 : line.start(a, last) - u0 + 1;
  for (int x = threadIdx.x; x < n; x += kMWarps * 32)
    s_slot[x] = 2 * (dense ? i + x : line.block(a, u0 + x)) + (x == 0);
  __syncthreads();
  for (int row0 = blockIdx.y * kRows; row0 < d0.x; row0 += gridDim.y * kRows) {
    const int row = min(row0 + rl, d0.x - 1);
    auto slot = [&](int x) -> size_t { return (size_t)s_slot[x] * a.part_rows + row; };
    auto part = [&](int x) -> Vec {
      return __ldcg(reinterpret_cast<const Vec*>(a.part + slot(x) * HD) + lane);
    };
    Vec pre[kBatch];
#pragma unroll
    for (int x = 0; x < kBatch; ++x)
      if (w + x * WPR < n) pre[x] = part(w + x * WPR);
    // the row's weights: its first warp's lanes, or all of its warps'
    float gm = -INFINITY, Ls = 0.f;
    for (int x = w * 32 + lane; x < n; x += WPR * 32) {
      const float2 v = __ldcg(&a.ml[slot(x)]);
      s_ml[rl][x] = v;
      gm = fmaxf(gm, v.x);
    }
    gm = warp_max(gm);
    if constexpr (WPR > 1) {
      if (lane == 0) s_gm[warp] = gm;
      __syncthreads();
#pragma unroll
      for (int y = 0; y < WPR; ++y) gm = fmaxf(gm, s_gm[rl * WPR + y]);
    }
    for (int x = w * 32 + lane; x < n; x += WPR * 32) {
      const float2 v = s_ml[rl][x];
      const float wt = part_weight(v.x, gm) * v.y;
      s_ml[rl][x].y = wt;
      Ls += wt;
    }
    Ls = warp_sum(Ls);
    if constexpr (WPR > 1) {
      if (lane == 0) s_sum[warp] = Ls;
      __syncthreads();
      Ls = 0.f;
#pragma unroll
      for (int y = 0; y < WPR; ++y) Ls += s_sum[rl * WPR + y];
    } else {
      __syncwarp();
    }
    const float inv = 1.f / Ls;
    float acc[kC];
#pragma unroll
    for (int j = 0; j < kC; ++j) acc[j] = 0.f;
    for (int x0 = w; x0 < n; x0 += kBatch * WPR) {
      if (x0 != w)
#pragma unroll
        for (int x = 0; x < kBatch; ++x)
          if (x0 + x * WPR < n) pre[x] = part(x0 + x * WPR);
#pragma unroll
      for (int x = 0; x < kBatch; ++x)
        if (x0 + x * WPR < n) {
          const float wt = s_ml[rl][x0 + x * WPR].y * inv;
          const float* f = reinterpret_cast<const float*>(&pre[x]);
#pragma unroll
          for (int j = 0; j < kC; ++j) acc[j] = fmaf(wt, f[j], acc[j]);
        }
    }
    if constexpr (WPR > 1) {
#pragma unroll
      for (int j = 0; j < kC; ++j) s_red[warp][lane * kC + j] = acc[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kC; ++j) {
        acc[j] = 0.f;
#pragma unroll
        for (int y = 0; y < WPR; ++y) acc[j] += s_red[rl * WPR + y][lane * kC + j];
      }
    }
    if (w == 0 && row0 + rl < d0.x) {
      const int r = d0.z + row, m = a.byG(r), h = d0.w * a.G + r - m * a.G;
      const int p = d1.z + m;
      const int lo = a.window > 0 ? max(d1.w, p - a.window + 1) : d1.w;
      if (p < lo)  // sees no key
#pragma unroll
        for (int j = 0; j < kC; ++j) acc[j] = 0.f;
      T* out = static_cast<T*>(a.out) + ((int64_t)d0.y * a.M + m) * a.out_stride + (int64_t)h * HD +
               lane * kC;
      if constexpr (sizeof(T) == 4) {
        Vec v;
#pragma unroll
        for (int j = 0; j < kC; ++j) reinterpret_cast<float*>(&v)[j] = acc[j];
        *reinterpret_cast<Vec*>(out) = v;
      } else {
        uint32_t u[kC / 2];
#pragma unroll
        for (int j = 0; j < kC; j += 2) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(acc[j], acc[j + 1]);
          u[j / 2] = *reinterpret_cast<const uint32_t*>(&b);
        }
        if constexpr (HD == 128)
          *reinterpret_cast<uint2*>(out) = make_uint2(u[0], u[1]);
        else
          *reinterpret_cast<uint32_t*>(out) = u[0];
      }
    }
    if constexpr (WPR > 1) __syncthreads();
    else __syncwarp();  // every lane has read the weights
  }
}

// ------------------------------------------------------------- host side

namespace {

struct Kv8Device {
  bool ready = false;
  int sms = 0;
};
std::mutex g_kv8_mu;
Kv8Device g_kv8_dev[64];

template <typename T, int HD>
cudaError_t prep_rows() {
  return cudaFuncSetAttribute(k_kv8_rows<T, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)RowsL<HD>::template total<sizeof(T) == 4 ? 2 : 1>());
}

template <int TILES>
cudaError_t prep_wide() {
  return cudaFuncSetAttribute(k_kv8_wide<TILES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)WideL<TILES>::kSmem);
}

// SMs of the current device; its kernels' limits of shared memory are set on
// the first call there.
cudaError_t kv8_device(int* sms) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_kv8_mu);
  Kv8Device& d = g_kv8_dev[dev];
  if (!d.ready) {
    if ((e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess ||
        (e = prep_rows<float, 64>()) != cudaSuccess || (e = prep_rows<float, 128>()) != cudaSuccess ||
        (e = prep_rows<__nv_bfloat16, 64>()) != cudaSuccess ||
        (e = prep_rows<__nv_bfloat16, 128>()) != cudaSuccess ||
        (e = prep_wide<1>()) != cudaSuccess || (e = prep_wide<2>()) != cudaSuccess)
      return e;
    d.ready = true;
  }
  *sms = d.sms;
  return cudaSuccess;
}

// Workspace of an attention call: descriptors, (max, sum) pairs, parts.
struct Kv8Work {
  size_t ml, part, total;
};
Kv8Work kv8_work(int blocks, int rows, int hd) {
  Kv8Work w;
  w.ml = ((size_t)blocks * sizeof(Kv8Desc) + 255) / 256 * 256;
  w.part = w.ml + ((size_t)2 * blocks * rows * sizeof(float2) + 255) / 256 * 256;
  w.total = w.part + (size_t)2 * blocks * rows * hd * sizeof(float);
  return w;
}

template <typename T, int HD, int RT>
cudaError_t merge_launch(const Kv8Attn& a, int P, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  constexpr int kWpr = RT == kRT ? kMWarps : 1;  // warps of a row
  const int ny = (a.part_rows * kWpr + kMWarps - 1) / kMWarps;
  cfg.gridDim = dim3(P, ny < kMRowBlocks<kWpr> ? ny : kMRowBlocks<kWpr>);
  cfg.blockDim = dim3(kMWarps * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = g_pdl_enabled ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_kv8_merge<T, HD, RT, kWpr>, a);
}

template <typename T, int HD>
cudaError_t rows_launch(const Kv8Attn& a, int P, cudaStream_t st) {
  const size_t smem = RowsL<HD>::template total<sizeof(T) == 4 ? 2 : 1>();
  if (a.split > 1) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(P);
    cfg.blockDim = dim3(kVThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_kv8_rows<T, HD>, a);
  }
  k_kv8_rows<T, HD><<<P, kVThreads, smem, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess || a.split ? e : merge_launch<T, HD, kRT>(a, P, st);
}

template <int TILES>
cudaError_t wide_launch(const Kv8Attn& a, int P, cudaStream_t st) {
  using L = WideL<TILES>;
  k_kv8_wide<TILES><<<P, L::kThreads, L::kSmem, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : merge_launch<__nv_bfloat16, kWHd, L::kRows>(a, P, st);
}

// The kernel of a call.  Tiles on tcgen05 where a KV head has more than 16 query rows,
// the type is bf16 and head_dim 128, with one accumulator of 128 rows, or two where there
// are more; tiles of 16 on mma.sync otherwise, and where these form clusters (below) that
// have room all at once.  us a call, mma.sync / tcgen05, by rows of 8 KV heads (of 32 in the
// third line):
//                     16           17           32           48          128
//   16000         19.6/23.8    24.4/24.4    25.7/25.0    33.2/25.8    63.3/29.9
//   100000        51.1/66.2    81.8/66.8    82.7/67.4     121/68.5     281/75.9
//   16 x 1000     60.6/62.6    86.9/64.0    97.8/69.0     130/71.9     304/90.8
// clusters / tcgen05 (one accumulator):
//   240 keys                    8.9/13.0     8.9/13.7     8.9/13.9    11.0/14.6
//   1000                        9.8/14.7    11.8/15.7    12.2/16.2    13.8/18.6
//   2000                       11.5/17.3    13.6/18.1    13.9/18.9
// and one / two accumulators, 8 KV heads:
//                    129          256          300          512         1024
//   500 keys      17.4/17.6    19.5/20.3    20.5/22.1    21.9/22.8    30.1/28.2
//   16000         32.5/30.6    41.3/33.3    48.9/48.2    58.5/50.3    94.1/76.6
//   100000         113/93.0     125/95.6     184/172      232/175      449/326
//   16 x 1000     51.7/42.2    58.8/51.8    72.9/79.2    91.5/83.0     174/155
constexpr int kWideFrom = 16;
// Short caches: a cluster of blocks for each item, which joins its parts itself (mma.sync
// kernel): of 1, 2, 4 or 8 blocks with 128 keys or more each, as long as there is room for
// all, two on each of 152 SMs; up to 512 keys a block and 2048 in all.  us, line / clusters,
// at full caches of 128, 512, 1024, 2048 and 4096 positions:
//   1 sequence, 8 KV heads, 4 rows each     8.5/6.0   8.7/7.6   8.9/8.0   9.8/9.6   10.8/12.1
//   1, 40 heads, 2 rows                     9.2/6.3  10.1/8.4  11.1/10.3 12.8/13.7  17.5/19.6
//   4, 8 heads, 4 rows                      9.2/6.3  10.5/8.1  11.0/9.5  12.9/11.4  16.2/14.8
//   16, 8 heads, 4 rows                    10.7/6.3  15.4/10.8 18.5/14.4 24.4/20.5  38.0/34.9
// (sequences of one length, for which clusters are at their best), and a launch and a
// workspace less, which the host takes 6 to 8 us for.  The capacity is what the host knows: 1 row of 32
// heads over 8 KV heads x 1100 keys takes 8.7 us in a cache of 1216 positions and, on the line, 10.1 in one
// of 2112 to 131072.
constexpr int kSplitKeys = 128, kSplitBlocks = 304, kSplitSeq = 512, kSplitMost = 2048;

struct Kv8Plan {
  int wide;  // accumulators of a wide tile, 0: not wide
  int split;     // blocks of an item's own, 0: the line
  int rt, ku;
  int max_blocks, part_rows;
  long long n_rt, units;  // tiles of a sequence; the line's places, at most
};
Kv8Plan plan_of(const ssd_kv8_cache* c, int dtype, int n_heads, int M) {
  Kv8Plan p;
  const long long rows = (long long)M * (n_heads / c->n_kv_heads);
  const long long heads = (long long)c->n_seq * c->n_kv_heads;
  const long long small = (rows + kRT - 1) / kRT * heads;  // items of 16 rows
  p.split = 1;
  while (p.split < kSplitMax && c->max_seq > kSplitKeys * p.split &&
         small * p.split * 2 <= kSplitBlocks)
    p.split *= 2;
  if (c->max_seq > kSplitSeq * p.split || c->max_seq > kSplitMost) p.split = 0;
  p.wide = 0;
  if (dtype == SSD_DTYPE_BF16 && c->head_dim == kWHd && rows > kWideFrom &&
      !(p.split && small * p.split <= kSplitBlocks)) {
    p.wide = rows > kWRows ? 2 : 1;
    p.split = 0;
  }
  p.rt = p.wide ? p.wide * kWRows : kRT;
  p.part_rows = rows < p.rt ? (int)rows : p.rt;
  p.ku = p.wide ? kWKeys : kKv8Block;
  p.n_rt = (rows + p.rt - 1) / p.rt;
  p.units = p.n_rt * heads * ((c->max_seq + p.ku - 1) / p.ku +
                              (p.wide == 2 ? kKv8ItemCost<256> : kKv8ItemCost<kRT>));
  p.max_blocks = p.wide == 2 ? kKv8MaxBlocks / 2 : kKv8MaxBlocks;
  if (p.units < p.max_blocks) p.max_blocks = (int)p.units;
  return p;
}

// What both attention entry points check of the sizes, and their plan; null: fine.
const char* check_attention(const ssd_kv8_cache* c, int32_t dtype, int32_t n_heads, int32_t M,
                            Kv8Plan* plan, ssd_status* status) {
  *status = c && c->head_dim != 64 && c->head_dim != 128 ? SSD_ERR_UNSUPPORTED : SSD_ERR_INVALID_ARG;
  if (const char* why = check_kv8(c)) return why;
  if (dtype != SSD_DTYPE_F32 && dtype != SSD_DTYPE_BF16) return "dtype must be fp32 or bf16";
  if (n_heads < c->n_kv_heads || n_heads % c->n_kv_heads || n_heads > 65536)
    return "n_heads must be a multiple of the cache's n_kv_heads";
  if (M < 1) return "M must be at least 1";
  *status = SSD_ERR_CAPACITY;
  if (M > c->max_seq) return "more rows than the cache has positions";
  *plan = plan_of(c, dtype, n_heads, M);
  if (plan->units > 0x7fffffffll) return "n_seq x M x max_seq: more than 2^31 units of work";
  *status = SSD_OK;
  return nullptr;
}

}  // namespace
}  // namespace ssd

extern "C" size_t ssd_kv8_attention_bytes(const ssd_kv8_cache* c, int32_t dtype, int32_t n_heads,
                                          int32_t M) {
  using namespace ssd;
  Kv8Plan p;
  ssd_status status;
  if (const char* why = check_attention(c, dtype, n_heads, M, &p, &status)) {
    fail_op(status, why);
    return 0;
  }
  return p.split ? 256 : kv8_work(p.max_blocks, p.part_rows, c->head_dim).total;
}

extern "C" ssd_status ssd_kv8_attention(const ssd_kv8_cache* c, const void* q, int32_t dtype,
                                        int32_t n_heads, int64_t q_stride, int32_t M,
                                        const int32_t* pos, const int32_t* rows,
                                        const int32_t* first, int32_t window, void* out,
                                        int64_t out_stride, void* workspace,
                                        size_t workspace_bytes, int32_t* err_dev, void* stream) {
  using namespace ssd;
  Kv8Plan plan;
  ssd_status status;
  if (const char* why = check_attention(c, dtype, n_heads, M, &plan, &status))
    return fail_op(status, why);
  const int elt = dtype == SSD_DTYPE_BF16 ? 2 : 4;
  const int64_t len = (int64_t)n_heads * c->head_dim;
  if (!q || !out || !pos || ((uintptr_t)q & 15u) || ((uintptr_t)out & 15u))
    return fail_op(SSD_ERR_INVALID_ARG, "q, out or pos: NULL or unaligned pointer");
  if (q_stride < len || out_stride < len || q_stride > (1ll << 40) || out_stride > (1ll << 40) ||
      (q_stride * elt) % 16 || (out_stride * elt) % 16)
    return fail_op(SSD_ERR_INVALID_ARG,
                   "q_stride or out_stride: below a row's length, or not a multiple of 16 bytes");
  if (out == q && out_stride != q_stride)
    return fail_op(SSD_ERR_INVALID_ARG, "out is q, but their strides differ");
  if (window < 0) return fail_op(SSD_ERR_INVALID_ARG, "window must be 0 (none) or positive");
  const int G = n_heads / c->n_kv_heads;
  const Kv8Work lay = kv8_work(plan.max_blocks, plan.part_rows, c->head_dim);
  if (!plan.split) {
    if (!workspace || ((uintptr_t)workspace & 255u))
      return fail_op(SSD_ERR_INVALID_ARG, "workspace must be non-NULL and 256-byte aligned");
    if (workspace_bytes < lay.total) return fail_op(SSD_ERR_CAPACITY, "workspace too small");
  }
  int sms = 0;
  cudaError_t e = kv8_device(&sms);
  if (e != cudaSuccess) return fail_op_cuda("ssd_kv8_attention", e);
  Kv8Attn a{};
  a.k = static_cast<const uint8_t*>(c->k);
  a.v = static_cast<const uint8_t*>(c->v);
  a.ks = c->k_scale;
  a.vs = c->v_scale;
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
  a.G = G;
  a.M = M;
  a.max_seq = c->max_seq;
  a.window = window;
  a.n_rt = (int)plan.n_rt;
  a.entries = (int)plan.n_rt * c->n_seq;
  a.scale = (float)(1.4426950408889634 / sqrt((double)c->head_dim));
  char* ws = static_cast<char*>(workspace);
  a.desc = reinterpret_cast<Kv8Desc*>(ws);
  a.ml = reinterpret_cast<float2*>(ws + lay.ml);
  a.part = reinterpret_cast<float*>(ws + lay.part);
  a.byG = Kv8Div::of((uint32_t)G);
  a.byRt = Kv8Div::of((uint32_t)plan.n_rt);
  int P = sms * (plan.wide == 2 ? 1 : 2);  // blocks of an SM
  if (P > plan.max_blocks) P = plan.max_blocks;
  a.part_rows = plan.part_rows;
  a.split = plan.split;
  if (plan.split) P = a.entries * a.Hkv * plan.split;
  a.byP = Kv8Div::of((uint32_t)P);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = c->head_dim == 128;
  if (plan.wide)
    e = plan.wide == 2 ? wide_launch<2>(a, P, st) : wide_launch<1>(a, P, st);
  else if (dtype == SSD_DTYPE_BF16)
    e = wide ? rows_launch<__nv_bfloat16, 128>(a, P, st) : rows_launch<__nv_bfloat16, 64>(a, P, st);
  else
    e = wide ? rows_launch<float, 128>(a, P, st) : rows_launch<float, 64>(a, P, st);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_kv8_attention", e);
}
