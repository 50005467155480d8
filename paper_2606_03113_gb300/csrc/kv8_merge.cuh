// kv8_merge.cuh -- the join of the parts that the blocks of an attention left (kv8_plan.cuh), and what
// its kernels have in common: rows of queries and outputs, the weight of a part, the workspace.
#pragma once

#include <math.h>

#include <type_traits>

#include "kv8_plan.cuh"

namespace ssd {
namespace {

constexpr int kKv8MaxBlocks = 320;

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

template <typename T, int HD, int WPR>
__global__ void __launch_bounds__(kMWarps * 32, kMBlocks<WPR>) k_kv8_merge(const AttnArgs a) {
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

// kWpr: warps of a row.
template <typename T, int HD, int kWpr>
cudaError_t merge_launch(const AttnArgs& a, int P, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  const int ny = (a.part_rows * kWpr + kMWarps - 1) / kMWarps;
  cfg.gridDim = dim3(P, ny < kMRowBlocks<kWpr> ? ny : kMRowBlocks<kWpr>);
  cfg.blockDim = dim3(kMWarps * 32);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = g_pdl_enabled ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_kv8_merge<T, HD, kWpr>, a);
}

}  // namespace
}  // namespace ssd
