// paged_attention.cu -- attention of new rows over the pages of a layer (paged.cuh):
//   o_r = sum_j p_rj v_j / sum_j p_rj,  p_rj = e^(q_r . k_j / sqrt(hd) - max),
// over the keys j that row r sees: first .. its own position, at most `window`.
//
// k_paged_plain: a block a row and head, its warps take the keys in turn.
#include <math.h>

#include "paged.cuh"

namespace ssd {

namespace {

constexpr int kPlainWarps = 8;

struct PagedAttn {
  PagedView c;
  const char *k, *v;  // the layer's K and V of page 0
  const void* q;
  void* out;
  const int32_t *pos, *rows, *first;
  int32_t* err;
  int64_t q_stride, out_stride;
  int32_t G, M, longest, window;
  float scale;  // log2(e) / sqrt(head_dim)
};

}  // namespace

template <typename T, int HD>
__global__ void __launch_bounds__(kPlainWarps * 32) k_paged_plain(const PagedAttn a) {
  constexpr int C = HD / 32;
  __shared__ float s_o[kPlainWarps][HD], s_m[kPlainWarps], s_l[kPlainWarps];
  const int h = blockIdx.x, b = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int p0 = __ldg(a.pos + b), n = a.rows ? __ldg(a.rows + b) : a.M;
  if (p0 < 0 || n < 0 || n > a.M || p0 > a.longest - n) {
    if (threadIdx.x == 0 && h == 0 && blockIdx.y == 0 && a.err)
      atomicOr(a.err, n < 0 || n > a.M ? (int)kErrControl : (int)kErrCapacity);
    return;
  }
  const int first = a.first ? max(__ldg(a.first + b), 0) : 0;
  const size_t head = (size_t)(h / a.G) * a.c.slab;
  const int mask = (1 << a.c.shift) - 1;
  for (int m = blockIdx.y; m < n; m += gridDim.y) {
    const int p = p0 + m, lo = a.window > 0 ? max(first, p - a.window + 1) : first;
    const T* q = static_cast<const T*>(a.q) + ((int64_t)b * a.M + m) * a.q_stride + (int64_t)h * HD;
    float fq[C], o[C], mx = -INFINITY, sum = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) fq[j] = Elem<T>::to_f(q[lane + 32 * j]) * a.scale, o[j] = 0.f;
    for (int key = lo + warp; key <= p; key += kPlainWarps) {
      const int e = a.c.entry(b, key >> a.c.shift);
      if (e < 0) {
        if (lane == 0 && a.err) atomicOr(a.err, (int)kErrTable);
        continue;
      }
      const size_t at = e * a.c.bytes + head + (size_t)(key & mask) * HD * sizeof(T);
      const T* kr = reinterpret_cast<const T*>(a.k + at);
      const T* vr = reinterpret_cast<const T*>(a.v + at);
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < C; ++j) s = fmaf(fq[j], Elem<T>::to_f(kr[lane + 32 * j]), s);
      s = warp_sum(s);
      const float nm = fmaxf(mx, s), top = nm == -INFINITY ? 0.f : nm;
      const float f = exp2f(mx - top), w = exp2f(s - top);
      sum = sum * f + w;
#pragma unroll
      for (int j = 0; j < C; ++j) o[j] = fmaf(w, Elem<T>::to_f(vr[lane + 32 * j]), o[j] * f);
      mx = nm;
    }
#pragma unroll
    for (int j = 0; j < C; ++j) s_o[warp][lane + 32 * j] = o[j];
    if (lane == 0) s_m[warp] = mx, s_l[warp] = sum;
    __syncthreads();
    if (threadIdx.x < HD) {
      float gm = -INFINITY, L = 0.f, acc = 0.f;
      for (int w = 0; w < kPlainWarps; ++w) gm = fmaxf(gm, s_m[w]);
      for (int w = 0; w < kPlainWarps; ++w) {
        const float f = exp2f(s_m[w] - (gm == -INFINITY ? 0.f : gm));
        L = fmaf(f, s_l[w], L);
        acc = fmaf(f, s_o[w][threadIdx.x], acc);
      }
      static_cast<T*>(a.out)[((int64_t)b * a.M + m) * a.out_stride + (int64_t)h * HD + threadIdx.x] =
          Elem<T>::from_f(lo <= p ? acc / L : 0.f);
    }
    __syncthreads();
  }
}

namespace {

const char* check_attention(const ssd_paged_cache* c, int32_t n_heads, int32_t M, int32_t longest,
                            ssd_status* status) {
  if (const char* why = check_paged(c, status)) return why;
  *status = SSD_ERR_INVALID_ARG;
  if (n_heads < c->n_kv_heads || n_heads % c->n_kv_heads || n_heads > 65536)
    return "n_heads must be a multiple of the cache's n_kv_heads";
  if (M < 1) return "M must be at least 1";
  if (longest < 0) return "longest must be 0 (the cache's positions) or positive";
  *status = SSD_ERR_CAPACITY;
  if (M > c->max_pages * c->page) return "more rows than the cache has positions";
  if (longest > c->max_pages * c->page) return "longest: more than the cache has positions";
  *status = SSD_OK;
  return nullptr;
}

template <typename T, int HD>
cudaError_t plain_launch(const PagedAttn& a, int heads, int n_seq, cudaStream_t st) {
  k_paged_plain<T, HD><<<dim3(heads, a.M < 65535 ? a.M : 65535, n_seq), kPlainWarps * 32, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace
}  // namespace ssd

extern "C" size_t ssd_paged_attention_bytes(const ssd_paged_cache* c, int32_t n_heads, int32_t M,
                                            int32_t longest) {
  using namespace ssd;
  ssd_status status;
  if (const char* why = check_attention(c, n_heads, M, longest, &status)) {
    fail_op(status, why);
    return 0;
  }
  return 256;
}

extern "C" ssd_status ssd_paged_attention(const ssd_paged_cache* c, int32_t layer, const void* q,
                                          int32_t n_heads, int64_t q_stride, int32_t M,
                                          const int32_t* pos, const int32_t* rows,
                                          const int32_t* first, int32_t window, int32_t longest,
                                          void* out, int64_t out_stride, void* workspace,
                                          size_t workspace_bytes, int32_t* err_dev, void* stream) {
  using namespace ssd;
  (void)workspace;
  (void)workspace_bytes;
  ssd_status status;
  if (const char* why = check_attention(c, n_heads, M, longest, &status)) return fail_op(status, why);
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
  if (window < 0) return fail_op(SSD_ERR_INVALID_ARG, "window must be 0 (none) or positive");
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
  a.G = n_heads / c->n_kv_heads;
  a.M = M;
  a.longest = longest ? longest : c->max_pages * c->page;
  a.window = window;
  a.scale = (float)(1.4426950408889634 / sqrt((double)c->head_dim));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool wide = c->head_dim == 128;
  cudaError_t e;
  if (c->dtype == SSD_DTYPE_BF16)
    e = wide ? plain_launch<__nv_bfloat16, 128>(a, n_heads, c->n_seq, st)
             : plain_launch<__nv_bfloat16, 64>(a, n_heads, c->n_seq, st);
  else
    e = wide ? plain_launch<float, 128>(a, n_heads, c->n_seq, st)
             : plain_launch<float, 64>(a, n_heads, c->n_seq, st);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_paged_attention", e);
}
