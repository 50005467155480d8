// logprobs.cu -- log-probabilities of given tokens over rows of logits, with
// the row's log-sum-exp, entropy and most probable tokens, at a temperature t:
//   lse = ln sum_v e^(z_v / t),  logp_v = z_v / t - lse,
//   H = -sum_v p_v ln p_v = ln S - T / S,
// with S = sum e^(d_v), T = sum e^(d_v) d_v, d_v = z_v / t - max.
//
// k_logprobs: one pass over a row or a chunk of it.  A thread keeps a running
// maximum, S and T (in powers of two) of the vectors it reads, and nothing else: its
// maximum is also what the most probable tokens are found by.  The n-th largest
// of the maxima of kGroups groups of threads is not above the row's n-th
// largest logit, so only the few threads with a maximum that high can hold one of
// the n; their vectors are read again (from L2), by all threads together, and the
// logits not below that bound are ranked by (value, lower id).  Where that gives
// more than kCand logits (ties, a spread that the threads' stride meets), the bound
// is raised by bisection first.
//
// Bound by issue slots beside the loads: 1023 rows of 128256 bf16 logits, top 8, 58 us = 4.5
// TB/s; in fp32 106 us = 5.0 TB/s; 13 rows in fp32, top 20, 9.0 us.
//
// Few rows are cut into chunks, one for each block of a cluster; the first block reads
// the others' parts from their shared memory and joins them in order.
//
// A logit of -inf has probability 0 and is none of the most probable; a NaN
// takes no place among them either, and it or +inf make the row's lse, entropy
// and log-probabilities NaN.
#include <math.h>

#include <atomic>

#include "kv8.cuh"

namespace ssd {

namespace {

constexpr int kLThreads = 256;
constexpr int kLWarps = kLThreads / 32;
constexpr int kUnroll = 4;       // 16-byte vectors of a thread in flight
constexpr int kGroups = 64;      // groups of threads whose maxima bound the top
constexpr int kCand = 1024;      // candidates that are ranked
constexpr int kMaxTop = SSD_MAX_TOP;
constexpr int kMaxChunks = 16;   // chunks of a row: blocks of a cluster
static_assert(kMaxTop <= kGroups, "a group for each of the most probable");
static_assert(kMaxChunks <= 32, "a lane for each chunk");
static_assert(kMaxChunks * kMaxTop <= kCand, "the chunks' lists fit the candidates' place");

struct LogpArgs {
  const void* z;
  const int32_t* tok;
  int64_t stride;
  int32_t rows, vocab, ntok, top, chunks;
  int32_t vec_per_chunk;
  float inv_t;   // 1 / t
  float* logprob;
  float* lse;
  float* entropy;
  int32_t* top_id;
  float* top_logprob;
  int32_t* err;
};

// (value, id) as one key: larger values first, then lower ids; 0: none.
__device__ __forceinline__ uint64_t logit_key(float z, int id) {
  if (!(z > -INFINITY)) return 0ull;
  const uint32_t b = __float_as_uint(z + 0.f);
  return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~id;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t h = (uint32_t)(k >> 32);
  return __uint_as_float(h & 0x80000000u ? h ^ 0x80000000u : ~h);
}
__device__ __forceinline__ int key_id(uint64_t k) { return (int)~(uint32_t)k; }

template <typename T>
__device__ __forceinline__ float logit(const T* row, int v) { return Elem<T>::to_f(row[v]); }

// Maximum (a logit), S and T of a set of logits; S = 0: an empty set.
struct Stat {
  float m, S, T;
};
// Two sets together; c: log2(e) / t.
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b, float c) {
  if (a.S == 0.f) return b;
  if (b.S == 0.f) return a;
  const float m = fmaxf(a.m, b.m);
  const float da = (a.m - m) * c, db = (b.m - m) * c;
  const float ea = ex2_approx(da), eb = ex2_approx(db);
  Stat r;
  r.m = m;
  r.S = a.S * ea + b.S * eb;
  // (a set 2^126 below the other adds nothing, even where its distance is infinite)
  r.T = (ea > 0.f || ea != ea ? ea * (a.T + da * a.S) : 0.f) +
        (eb > 0.f || eb != eb ? eb * (b.T + db * b.S) : 0.f);
  return r;
}

struct LogpSmem {
  Stat stat[kLWarps];
  float group[kGroups];
  float bound;
  int nthreads, ncand, count;
  int list[kLThreads];
  int scan[kLWarps];
  uint64_t cand[kCand];
  uint64_t top[kMaxTop];
  uint64_t best[kMaxTop];  // of all chunks
  Stat all;                // of the block's chunk; in the first block then of all
};

// A row's vectors: the 16-byte aligned places that hold its elements, the first
// and last of them perhaps in part.
template <typename T>
struct Row {
  static constexpr int kE = 16 / sizeof(T);
  const T* base;  // aligned down
  int skip, n;    // elements of the first vector before the row; of the row
  __device__ __forceinline__ int vectors() const { return (skip + n + kE - 1) / kE; }
  // vector i as it stands in memory, -inf in places outside the row
  __device__ __forceinline__ uint4 raw(int i) const {
    const int id0 = i * kE - skip;
    if (id0 >= 0 && id0 + kE <= n) return __ldg(reinterpret_cast<const uint4*>(base) + i);
    union {
      T e[kE];
      uint4 u;
    } x{};
#pragma unroll
    for (int j = 0; j < kE; ++j) {
      const int id = id0 + j;
      x.e[j] = id >= 0 && id < n ? base[skip + id] : Elem<T>::from_f(-INFINITY);
    }
    return x.u;
  }
  // its elements; returns the first one's id
  __device__ __forceinline__ int load(int i, float (&f)[kE]) const {
    Elem<T>::unpack(raw(i), f);
    return i * kE - skip;
  }
};

// The larger of packed logits, NaN aside, and the largest of a word's.
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b, float) {
  return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
}
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b, __nv_bfloat16) {
  const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a),
                                   *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ float max_of_word(uint32_t a, float) { return __uint_as_float(a); }
__device__ __forceinline__ float max_of_word(uint32_t a, __nv_bfloat16) {
  return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
}

// The chunk's `top` largest keys in order into sm.top; tmax: the thread's largest
// logit (-inf: none).  v0, v1: the chunk's vectors.
template <typename T>
__device__ void chunk_top(const Row<T>& row, int v0, int v1, int top, float tmax, LogpSmem& sm) {
  constexpr int kE = Row<T>::kE;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // bound: the top-th largest of the groups' maxima
  float gm = tmax;
#pragma unroll
  for (int o = 1; o < kLThreads / kGroups; o <<= 1) gm = fmaxf(gm, __shfl_xor_sync(0xffffffffu, gm, o));
  if (tid % (kLThreads / kGroups) == 0) sm.group[tid / (kLThreads / kGroups)] = gm;
  if (tid == 0) sm.nthreads = sm.ncand = 0;
  if (tid < top) sm.top[tid] = 0ull;
  __syncthreads();
  if (tid < kGroups) {
    const float g = sm.group[tid];
    int rank = 0;
    for (int i = 0; i < kGroups; ++i) {
      const float x = sm.group[i];
      rank += x > g || (x == g && i < tid);
    }
    if (rank == top - 1) sm.bound = g;  // exactly one
  }
  __syncthreads();
  float bound = sm.bound;
  // threads that can hold one of them
  if (tmax >= bound && tmax > -INFINITY) sm.list[atomicAdd(&sm.nthreads, 1)] = tid;
  __syncthreads();
  const int nt = sm.nthreads, per = (v1 - v0 + kLThreads - 1) / kLThreads;
  auto scan = [&](auto&& f) {  // every element of those threads
    for (int i = tid; i < nt * per; i += kLThreads) {
      const int v = v0 + sm.list[i % nt] + (i / nt) * kLThreads;
      if (v >= v1) continue;
      float x[kE];
      const int id0 = row.load(v, x);
#pragma unroll
      for (int j = 0; j < kE; ++j) f(x[j], id0 + j);
    }
  };
  scan([&](float x, int id) {
    if (x >= bound && x > -INFINITY) {
      const int at = atomicAdd(&sm.ncand, 1);
      if (at < kCand) sm.cand[at] = logit_key(x, id);
    }
  });
  __syncthreads();
  int n = sm.ncand;
  if (n > kCand) {
    // raise the bound to the top-th largest value itself: the largest key half
    // with at least `top` elements at or above it
    uint32_t lo = (uint32_t)(logit_key(bound > -INFINITY ? bound : -3.4028235e38f, 0) >> 32);
    uint32_t hi = 0xff800000u;  // +inf
    // (mostly the bound is that value itself, the one that so many logits have: one scan)
    for (bool first = true; lo < hi; first = false) {
      const uint32_t mid = first ? lo + 1 : lo + (hi - lo + 1) / 2;
      __syncthreads();
      if (tid == 0) sm.count = 0;
      __syncthreads();
      int c = 0;
      scan([&](float x, int id) { c += (uint32_t)(logit_key(x, id) >> 32) >= mid; });
      c = __reduce_add_sync(0xffffffffu, c);
      if (lane == 0) atomicAdd(&sm.count, c);
      __syncthreads();
      if (sm.count >= top) lo = mid;
      else hi = mid - 1;
    }
    __syncthreads();
    if (tid == 0) sm.ncand = 0;
    __syncthreads();
    // those above it are fewer than top; of those at it the lowest ids are taken
    scan([&](float x, int id) {
      const uint64_t k = logit_key(x, id);
      if ((uint32_t)(k >> 32) > lo) sm.cand[atomicAdd(&sm.ncand, 1)] = k;
    });
    __syncthreads();
    const int above = sm.ncand;
    int have = above;
    for (int b0 = v0; b0 < v1 && have < top; b0 += kLThreads) {
      const int v = b0 + tid;
      float x[kE];
      int id0 = 0, c = 0;
      if (v < v1) {
        id0 = row.load(v, x);
#pragma unroll
        for (int j = 0; j < kE; ++j) c += (uint32_t)(logit_key(x[j], id0 + j) >> 32) == lo;
      }
      int inc = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += u;
      }
      if (lane == 31) sm.scan[warp] = inc;
      __syncthreads();
      int at = have + inc - c, all = 0;
#pragma unroll
      for (int w = 0; w < kLWarps; ++w) {
        if (w < warp) at += sm.scan[w];
        all += sm.scan[w];
      }
      if (c)
#pragma unroll
        for (int j = 0; j < kE; ++j) {
          const uint64_t k = logit_key(x[j], id0 + j);
          if ((uint32_t)(k >> 32) == lo) {
            if (at < top) sm.cand[at] = k;
            ++at;
          }
        }
      have = min(have + all, top);
      __syncthreads();
    }
    n = have;
  }
  for (int i = tid; i < n; i += kLThreads) {
    const uint64_t k = sm.cand[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += sm.cand[j] > k;
    if (rank < top) sm.top[rank] = k;
  }
  __syncthreads();
}

// What a finished row puts out: x: its statistics, keys: its top.
template <typename T>
__device__ __forceinline__ void finish_row(const LogpArgs& a, int r, const T* row, const Stat& x,
                                           const uint64_t* keys, int threads) {
  constexpr float kLn2 = 0.6931471805599453f;
  // a row of -inf alone: lse is -inf, the rest NaN
  const bool none = x.S == 0.f;
  const float log_s = none ? __uint_as_float(0x7fffffffu) : logf(x.S);
  const int tid = threadIdx.x;
  if (tid == 0) {
    if (a.lse) a.lse[r] = none ? -INFINITY : fmaf(x.m, a.inv_t, log_s);
    if (a.entropy) a.entropy[r] = log_s - x.T / x.S * kLn2;
  }
  for (int i = tid; i < a.ntok; i += threads) {
    const int v = __ldg(a.tok + (int64_t)r * a.ntok + i);
    float lp = 0.f;
    if (v >= 0 && v < a.vocab) {
      lp = fmaf(logit<T>(row, v) - x.m, a.inv_t, -log_s);
    } else if (v != -1) {
      lp = __uint_as_float(0x7fffffffu);
      if (a.err) atomicOr(a.err, (int)kErrToken);
    }
    a.logprob[(int64_t)r * a.ntok + i] = lp;
  }
  for (int i = tid; i < a.top; i += threads) {
    const uint64_t k = keys[i];
    a.top_id[(int64_t)r * a.top + i] = k ? key_id(k) : -1;
    a.top_logprob[(int64_t)r * a.top + i] =
        k ? fmaf(key_value(k) - x.m, a.inv_t, -log_s) : -INFINITY;
  }
}

}  // namespace

// fp32 rows wait for memory: a thread has the next step's vectors on their way, at
// three blocks an SM (1023 rows of 128256 without a top: 82 us, 144 without that).  bf16 rows
// have twice the arithmetic a byte and run better as four blocks without (53, 62).
template <typename T>
constexpr bool kAhead = sizeof(T) == 4;

// Grid (chunks, rows).
template <typename T>
__global__ void __launch_bounds__(kLThreads, kAhead<T> ? 3 : 4) k_logprobs(const LogpArgs a) {
  constexpr int kE = Row<T>::kE;
  __shared__ LogpSmem sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float c = a.inv_t * 1.4426950408889634f;  // to powers of two
  for (int64_t r64 = blockIdx.y; r64 < a.rows; r64 += gridDim.y) {
    const int r = (int)r64;
    const T* zr = static_cast<const T*>(a.z) + r64 * a.stride;
    Row<T> row;
    row.skip = (int)(((uintptr_t)zr & 15u) / sizeof(T));
    row.base = zr - row.skip;
    row.n = a.vocab;
    const int nv = row.vectors();
    const int v0 = min((int)blockIdx.x * a.vec_per_chunk, nv);
    const int v1 = blockIdx.x + 1 == gridDim.x ? nv : min(v0 + a.vec_per_chunk, nv);

    // running statistics of the thread's vectors v0 + tid, + kLThreads, ..., kUnroll of
    // them a step
    float tmax = -INFINITY;  // largest logit
    float m = 0.f;           // what the sums stand against: tmax once there is one
    uint64_t S2 = 0, T2 = 0, nm2 = 0;
    const uint64_t c2 = pack2(c, c);
    const int whole0 = row.skip > 0, whole1 = min(v1, (row.skip + row.n) / kE);
    auto load = [&](int vb, uint4 (&x)[kUnroll]) {
      if (vb >= whole0 && vb + (kUnroll - 1) * kLThreads < whole1) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          x[u] = __ldg(reinterpret_cast<const uint4*>(row.base) + vb + u * kLThreads);
      } else {
        constexpr uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;  // -inf
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int v = vb + u * kLThreads;
          x[u] = v < v1 ? row.raw(v) : make_uint4(none, none, none, none);
        }
      }
    };
    auto add = [&](const uint4 (&x)[kUnroll]) {
      uint32_t bw = x[0].x;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        bw = max_word(max_word(bw, x[u].x, T()), x[u].y, T());
        bw = max_word(max_word(bw, x[u].z, T()), x[u].w, T());
      }
      const float bm = max_of_word(bw, T());
      if (bm > tmax) {
        if (tmax > -INFINITY) {
          const float d = (tmax - bm) * c, f = ex2_approx(d);
          const uint64_t f2 = pack2(f, f);
          T2 = f > 0.f ? mul2(f2, fma2(pack2(d, d), S2, T2)) : 0ull;
          S2 = mul2(f2, S2);
        }
        tmax = m = bm;
        nm2 = pack2(-m, -m);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
        for (int j = 0; j < kE; j += 2) {
          const uint64_t z2 = sizeof(T) == 4
                                  ? pack2(__uint_as_float(w[j]), __uint_as_float(w[j + 1 < 4 ? j + 1 : 3]))
                                  : pack2(__uint_as_float(w[j / 2] << 16),
                                          __uint_as_float(w[j / 2] & 0xffff0000u));
          // (differences first: a row of the type's lowest value is a row of equal logits)
          const float2 d = unpack2(mul2(add2(z2, nm2), c2));
          const uint64_t e2 = pack2(ex2_approx(d.x), ex2_approx(d.y));
          S2 = add2(S2, e2);
          // (a logit of -inf adds 0)
          T2 = fma2(e2, pack2(fmaxf(d.x, -1e30f), fmaxf(d.y, -1e30f)), T2);
        }
      }
    };
    constexpr int kStep = kLThreads * kUnroll;
    if constexpr (kAhead<T>) {
      uint4 xa[kUnroll], xb[kUnroll];
      int vb = v0 + tid;
      if (vb < v1) load(vb, xa);
      while (vb < v1) {
        if (vb + kStep < v1) load(vb + kStep, xb);
        add(xa);
        vb += kStep;
        if (vb >= v1) break;
        if (vb + kStep < v1) load(vb + kStep, xa);
        add(xb);
        vb += kStep;
      }
    } else {
      for (int vb = v0 + tid; vb < v1; vb += kStep) {
        uint4 x[kUnroll];
        load(vb, x);
        add(x);
      }
    }
    const float2 Sv = unpack2(S2), Tv = unpack2(T2);
    Stat st{m, Sv.x + Sv.y, Tv.x + Tv.y};
    // (a thread whose logits are all -inf has S = 0, with a NaN among them NaN)
    if (a.top > 0) chunk_top<T>(row, v0, v1, a.top, tmax, sm);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Stat b;
      b.m = __shfl_down_sync(0xffffffffu, st.m, o);
      b.S = __shfl_down_sync(0xffffffffu, st.S, o);
      b.T = __shfl_down_sync(0xffffffffu, st.T, o);
      st = join(st, b, c);
    }
    if (lane == 0) sm.stat[warp] = st;
    __syncthreads();
    st = sm.stat[0];
#pragma unroll
    for (int w = 1; w < kLWarps; ++w) st = join(st, sm.stat[w], c);
    const uint64_t* top = sm.top;
    if (a.chunks > 1) {
      if (tid == 0) sm.all = st;
      cluster_sync();
      if (blockIdx.x == 0) {
        for (int i = tid; i < a.chunks * a.top; i += kLThreads)
          sm.cand[i] = ld_cluster_u64(in_block(&sm.top[i % a.top], i / a.top));
        if (warp == 0) {
          st = Stat{0.f, 0.f, 0.f};
          if (lane < a.chunks)
            st = Stat{ld_cluster_f32(in_block(&sm.all.m, lane)),
                      ld_cluster_f32(in_block(&sm.all.S, lane)),
                      ld_cluster_f32(in_block(&sm.all.T, lane))};
#pragma unroll
          for (int o = kMaxChunks / 2; o > 0; o >>= 1) {
            Stat b;
            b.m = __shfl_down_sync(0xffffffffu, st.m, o);
            b.S = __shfl_down_sync(0xffffffffu, st.S, o);
            b.T = __shfl_down_sync(0xffffffffu, st.T, o);
            st = join(st, b, c);
          }
          if (lane == 0) sm.all = st;
        }
        __syncthreads();
        if (warp == 0) {  // the largest of the lists' heads, a.top times
          int at = 0;
          uint64_t head = a.top > 0 && lane < a.chunks ? sm.cand[lane * a.top] : 0ull;
          for (int i = 0; i < a.top; ++i) {
            const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(head >> 32));
            const uint32_t lo =
                __reduce_max_sync(0xffffffffu, (uint32_t)(head >> 32) == hi ? (uint32_t)head : 0u);
            const uint64_t best = (uint64_t)hi << 32 | lo;
            if (lane == 0) sm.best[i] = best;
            if (best && head == best) head = ++at < a.top ? sm.cand[lane * a.top + at] : 0ull;
          }
        }
        __syncthreads();
        st = sm.all;
        top = sm.best;
      }
    }
    if (blockIdx.x == 0) finish_row<T>(a, r, zr, st, top, kLThreads);
    if (a.chunks > 1) cluster_sync();  // the first block has read the others'
    else __syncthreads();
  }
}

namespace {

// Chunks of a row: blocks enough for four on each of 152 SMs, a power of two of them, and
// no chunk below 4096 logits (one step of a block for fp32, half of one for bf16).
int logp_chunks(int rows, int vocab) {
  constexpr int per = kLThreads * kUnroll * 4;
  const int want = (152 * 4 + rows - 1) / rows, most = (vocab + per - 1) / per;
  int n = 1;
  while (n < kMaxChunks && n < want && 2 * n <= most) n *= 2;
  return n;
}

const char* check_logp(int32_t rows, int32_t vocab, int32_t ntok, int32_t top) {
  if (rows < 1) return "n_rows must be at least 1";
  if (vocab < 1 || vocab > (1 << 30)) return "vocab must be in 1..2^30";
  if (ntok < 0 || ntok > (1 << 20)) return "n_tokens must be in 0..2^20";
  if (top < 0 || top > kMaxTop || top > vocab) return "top_n must be in 0..32 and at most vocab";
  return nullptr;
}

// More than eight blocks in a cluster have to be allowed, once a device.
template <typename T>
cudaError_t allow_clusters() {
  static std::atomic<bool> done[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (done[dev].load(std::memory_order_acquire)) return cudaSuccess;
  e = cudaFuncSetAttribute(k_logprobs<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) done[dev].store(true, std::memory_order_release);
  return e;
}

template <typename T>
cudaError_t logp_launch(const LogpArgs& a, cudaStream_t st) {
  const int gy = a.rows < 32768 ? a.rows : 32768;
  if (a.chunks == 1) {
    k_logprobs<T><<<dim3(1, gy), kLThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  const cudaError_t e = allow_clusters<T>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.chunks, gy);
  cfg.blockDim = dim3(kLThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = a.chunks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_logprobs<T>, a);
}

}  // namespace
}  // namespace ssd

extern "C" ssd_status ssd_token_logprobs(const void* logits, int32_t dtype, int32_t n_rows,
                                         int32_t vocab, int64_t row_stride, const int32_t* tokens,
                                         int32_t n_tokens, float temperature, int32_t top_n,
                                         float* logprob, float* lse, float* entropy,
                                         int32_t* top_id, float* top_logprob, int32_t* err_dev,
                                         void* stream) {
  using namespace ssd;
  if (const char* why = check_logp(n_rows, vocab, n_tokens, top_n))
    return fail_op(SSD_ERR_INVALID_ARG, why);
  if (dtype != SSD_DTYPE_F32 && dtype != SSD_DTYPE_BF16)
    return fail_op(SSD_ERR_INVALID_ARG, "dtype must be fp32 or bf16");
  const int elt = dtype == SSD_DTYPE_BF16 ? 2 : 4;
  if (!logits || (uintptr_t)logits % elt || row_stride < vocab || row_stride > (1ll << 40))
    return fail_op(SSD_ERR_INVALID_ARG, "logits NULL or unaligned, or row_stride below vocab");
  if ((n_tokens > 0 && (!tokens || !logprob)) || (top_n > 0 && (!top_id || !top_logprob)))
    return fail_op(SSD_ERR_INVALID_ARG, "NULL buffer of tokens or of the most probable");
  if (!(temperature >= 1e-3f && temperature <= 1e3f))
    return fail_op(SSD_ERR_INVALID_ARG, "temperature must be in 0.001..1000");
  const int chunks = logp_chunks(n_rows, vocab);
  LogpArgs a{};
  a.z = logits;
  a.tok = tokens;
  a.stride = row_stride;
  a.rows = n_rows;
  a.vocab = vocab;
  a.ntok = n_tokens;
  a.top = top_n;
  a.chunks = chunks;
  const int e16 = 16 / elt;
  const int nv = (vocab + e16 - 1) / e16;
  a.vec_per_chunk = (nv + chunks - 1) / chunks;
  a.inv_t = 1.0f / temperature;
  a.logprob = logprob;
  a.lse = lse;
  a.entropy = entropy;
  a.top_id = top_id;
  a.top_logprob = top_logprob;
  a.err = err_dev;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e =
      dtype == SSD_DTYPE_BF16 ? logp_launch<__nv_bfloat16>(a, st) : logp_launch<float>(a, st);
  return e == cudaSuccess ? SSD_OK : fail_op_cuda("ssd_token_logprobs", e);
}
