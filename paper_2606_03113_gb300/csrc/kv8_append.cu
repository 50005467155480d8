// kv8_append.cu -- new K and V rows into the 8-bit cache.
//
// A block of threads owns one cache block (kKv8Block positions) of one
// sequence, KV head and side (K or V): it reads the rows that fall there, finds
// their largest magnitude, sets the scale, rounds the rows to codes, and, where
// the scale grew, rounds the codes of the positions in front of them again.
// Nothing else writes a cache block in the same call, so there is no order
// between blocks.
//
// Bound by bytes for prompts (a value is read once and its code written once): 2047
// bf16 rows of 40 heads x 128, K and V, 12.8 us = 4.9 TB/s, the rows kept in
// registers as they stand in memory.  By the launch and one round trip of memory for a few
// rows: 16 sequences x 1 row of 8 heads 2.3 us.
#include "kv8.cuh"

namespace ssd {

namespace {

// 2047 rows of 40 heads: 64 threads 14.1 us, 128 12.8, 256 14.0, 512 19.7; one row of 16
// sequences: 2.9, 2.3, 2.2, 2.8.
constexpr int kApThreads = 128;

struct AppendArgs {
  uint8_t* code[2];
  float* scale[2];
  const void* x[2];
  int64_t stride;  // elements between rows
  const int32_t *pos, *rows;
  int32_t* err;
  int32_t M, heads, max_seq;
};

// Eight values of a row as they stand in memory.
template <typename T>
struct Eight {
  static constexpr int kWords = sizeof(T) / 2;  // 16-byte words
  uint4 w[kWords];
  __device__ __forceinline__ void load(const T* p) {  // 16-byte aligned
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void values(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      float x[Elem<T>::kPerChunk];
      Elem<T>::unpack(w[i], x);
#pragma unroll
      for (int j = 0; j < Elem<T>::kPerChunk; ++j) f[i * Elem<T>::kPerChunk + j] = x[j];
    }
  }
  // Largest magnitude, NaN aside.
  __device__ __forceinline__ float amax() const;
};
template <>
__device__ __forceinline__ float Eight<float>::amax() const {
  float f[8], m = 0.f;
  values(f);
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(f[j]));
  return m;
}
template <>
__device__ __forceinline__ float Eight<__nv_bfloat16>::amax() const {
  const uint32_t u[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
  __nv_bfloat162 m = __float2bfloat162_rn(0.f);
#pragma unroll
  for (int j = 0; j < 4; ++j) m = __hmax2(m, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&u[j])));
  return fmaxf(__low2float(m), __high2float(m));
}

constexpr float kMaxFloat = 3.4028235e38f;

__device__ __forceinline__ uint2 codes8(const float (&f)[8]) {
  uint2 r;
  r.x = e4m3_pair(f[0], f[1]) | e4m3_pair(f[2], f[3]) << 16;
  r.y = e4m3_pair(f[4], f[5]) | e4m3_pair(f[6], f[7]) << 16;
  return r;
}

}  // namespace

// Grid (cache blocks that M rows can touch, 2 x KV heads, sequences).
template <typename T, int HD>
__global__ void __launch_bounds__(kApThreads) k_kv8_append(const AppendArgs a) {
  constexpr int kCpr = HD / 8;                            // chunks of 8 per row
  constexpr int kPer = kKv8Block * kCpr / kApThreads;     // chunks per thread
  const int b = blockIdx.z, h = blockIdx.y >> 1, side = blockIdx.y & 1;
  const int tid = threadIdx.x;
  const int p0 = __ldg(a.pos + b), n = a.rows ? __ldg(a.rows + b) : a.M;
  if (p0 < 0 || n < 0 || n > a.M || p0 > a.max_seq - n) {
    if (tid == 0 && blockIdx.x == 0 && blockIdx.y == 0 && a.err)
      atomicOr(a.err, n < 0 || n > a.M ? (int)kErrControl : (int)kErrCapacity);
    return;
  }
  const int blk = p0 / kKv8Block + (int)blockIdx.x, k0 = blk * kKv8Block;
  if (n == 0 || k0 >= p0 + n) return;
  const int lo = max(p0 - k0, 0), hi = min(p0 + n - k0, kKv8Block);  // new rows of the block
  const T* x = static_cast<const T*>(side ? a.x[1] : a.x[0]) + (int64_t)h * HD;
  const int64_t row0 = (int64_t)b * a.M + (k0 - p0);  // input row of position k0

  Eight<T> f[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int c = tid + i * kApThreads, r = c / kCpr, off = (c % kCpr) * 8;
    if (r >= lo && r < hi) f[i].load(x + (row0 + r) * a.stride + off);
    else f[i].zero();
  }
  const size_t slab = (size_t)b * a.heads + h;
  float* sp = (side ? a.scale[1] : a.scale[0]) + slab * (a.max_seq / kKv8Block) + blk;
  const float old = lo > 0 ? *sp : 0.f;  // positions in front of lo hold codes at this scale
  __shared__ float warp_amax[2][kApThreads / 32];
  // the block's largest of m
  auto block_amax = [&](float m, int at) {
    m = warp_max(m);
    if ((tid & 31) == 0) warp_amax[at][tid >> 5] = m;
    __syncthreads();  // (every thread has read the old scale)
#pragma unroll
    for (int w = 0; w < kApThreads / 32; ++w) m = fmaxf(m, warp_amax[at][w]);
    return m;
  };
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) amax = fmaxf(amax, f[i].amax());
  amax = block_amax(amax, 0);
  // an infinity has no code: it is kept as NaN, and takes no part in the scale
  const bool infinite = amax > kMaxFloat;
  if (infinite) {
    amax = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float v[8];
      f[i].values(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(v[j]) <= kMaxFloat ? fabsf(v[j]) : 0.f);
    }
    amax = block_amax(amax, 1);
  }

  const int e = kv8_scale_exp(amax);
  const float s = fmaxf(pow2i(e), old);
  const float inv = 1.0f / s;  // a power of two: exact
  uint8_t* code = (side ? a.code[1] : a.code[0]) + (slab * a.max_seq + k0) * HD;
  if (s > old && lo > 0) {
    const float ratio = old / s;
    for (int c = tid; c < lo * kCpr; c += kApThreads) {
      uint2* p = reinterpret_cast<uint2*>(code + (size_t)c * 8);
      const uint2 u = *p;
      float g[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = j < 2 ? u.x : u.y;
        const uint32_t hb = e4m3_to_half2(j & 1 ? w >> 16 : w);
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&hb));
        g[2 * j] = v.x * ratio;
        g[2 * j + 1] = v.y * ratio;
      }
      *p = codes8(g);
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int c = tid + i * kApThreads, r = c / kCpr, off = (c % kCpr) * 8;
    if (r < lo || r >= hi) continue;
    float v[8];
    f[i].values(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (infinite && !(fabsf(v[j]) <= kMaxFloat)) v[j] = __uint_as_float(0x7fffffffu);
      v[j] *= inv;
    }
    *reinterpret_cast<uint2*>(code + (size_t)r * HD + off) = codes8(v);
  }
  if (tid == 0) *sp = s;
}

template <typename T, int HD>
static cudaError_t append(const AppendArgs& a, int n_seq, cudaStream_t st) {
  const dim3 grid((a.M + kKv8Block - 2) / kKv8Block + 1, 2 * a.heads, n_seq);
  k_kv8_append<T, HD><<<grid, kApThreads, 0, st>>>(a);
  return cudaGetLastError();
}

const char* check_kv8(const ssd_kv8_cache* c) noexcept {
  if (!c) return "cache is NULL";
  if (c->n_seq < 1 || c->n_seq > SSD_KV8_MAX_SEQS) return "cache: n_seq must be in 1..4096";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return "cache: n_kv_heads must be in 1..1024";
  if (c->head_dim != 64 && c->head_dim != 128) return "cache: head_dim must be 64 or 128";
  if (c->max_seq < kKv8Block || c->max_seq % kKv8Block || c->max_seq > (1 << 30))
    return "cache: max_seq must be a multiple of 64, at most 2^30";
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || ((uintptr_t)c->k & 15u) ||
      ((uintptr_t)c->v & 15u) || ((uintptr_t)c->k_scale & 3u) || ((uintptr_t)c->v_scale & 3u))
    return "cache: NULL or unaligned pointer";
  return nullptr;
}

}  // namespace ssd

extern "C" ssd_status ssd_kv8_append(const ssd_kv8_cache* c, const void* k, const void* v,
                                     int32_t dtype, int64_t row_stride, int32_t M,
                                     const int32_t* pos, const int32_t* rows, int32_t* err_dev,
                                     void* stream) {
  using namespace ssd;
  if (const char* why = check_kv8(c))
    return fail_op(c && c->head_dim != 64 && c->head_dim != 128 ? SSD_ERR_UNSUPPORTED
                                                                : SSD_ERR_INVALID_ARG, why);
  if (dtype != SSD_DTYPE_F32 && dtype != SSD_DTYPE_BF16)
    return fail_op(SSD_ERR_INVALID_ARG, "dtype must be fp32 or bf16");
  const int elt = dtype == SSD_DTYPE_BF16 ? 2 : 4;
  if (!k || !v || !pos || ((uintptr_t)k & 15u) || ((uintptr_t)v & 15u))
    return fail_op(SSD_ERR_INVALID_ARG, "k, v or pos: NULL or unaligned pointer");
  if (M < 1) return fail_op(SSD_ERR_INVALID_ARG, "M must be at least 1");
  if (M > c->max_seq) return fail_op(SSD_ERR_CAPACITY, "more rows than the cache has positions");
  if (row_stride < (int64_t)c->n_kv_heads * c->head_dim || row_stride > (1ll << 40) ||
      (row_stride * elt) % 16)
    return fail_op(SSD_ERR_INVALID_ARG,
                   "row_stride: below a row's length, or not a multiple of 16 bytes");
  AppendArgs a{};
  a.code[0] = static_cast<uint8_t*>(c->k);
  a.code[1] = static_cast<uint8_t*>(c->v);
  a.scale[0] = c->k_scale;
  a.scale[1] = c->v_scale;
  a.x[0] = k;
  a.x[1] = v;
  a.stride = row_stride;
  a.pos = pos;
  a.rows = rows;
  a.err = err_dev;
  a.M = M;
  a.heads = c->n_kv_heads;
  a.max_seq = c->max_seq;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = c->head_dim == 128;
  cudaError_t e;
  if (dtype == SSD_DTYPE_BF16)
    e = wide ? append<__nv_bfloat16, 128>(a, c->n_seq, st) : append<__nv_bfloat16, 64>(a, c->n_seq, st);
  else
    e = wide ? append<float, 128>(a, c->n_seq, st) : append<float, 64>(a, c->n_seq, st);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_kv8_append", e);
}
