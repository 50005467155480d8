// paged_stream.cuh -- attention over pages for up to 16 query rows a KV head (decoding, narrow
// verifications; bf16) over long sequences. Included by paged_attention.cu.
//
// One block an SM, so that its stretch of the plan's line is one stream of stages (64 keys, K and V)
// through a ring of 160 KB: four warps copy (cp.async), across items, and never wait for their end;
// eight take every other stage by fours, 16 keys each, and at an item's end join what they have while the
// ring fills with the next one's.
#pragma once

#include "attn_wide.cuh"

namespace ssd {

namespace {

template <int HD>
struct SL {
  using P = PL<__nv_bfloat16, HD, 1, 4>;  // its stages and places
  static constexpr int kKeys = P::kKeys, kChunks = P::kChunks;
  static constexpr uint32_t kStage = P::kStage, kSide = P::kSide;
  static constexpr int kNst = 160 * 1024 / (int)kStage;
  static constexpr uint32_t kExchange = kNst * kStage;                 // where it begins
  static constexpr uint32_t kQ = kExchange + 4 * kTile * (HD + 4) * 4;  // two items' queries
  static constexpr uint32_t kQBytes = kTile * HD * 2;
  static constexpr uint32_t kSmem = kQ + 2 * kQBytes;
  static constexpr int kUse = 8, kCopy = 4;  // warps
  static constexpr int kThreads = (kUse + kCopy) * 32;
};

template <int HD>
struct StreamBars {
  uint64_t full[SL<HD>::kNst], empty[SL<HD>::kNst];  // a stage is there; is read
  uint64_t q_full[2], q_free[2];
};

}  // namespace

template <int HD>
__global__ void __launch_bounds__(SL<HD>::kThreads, 1) k_paged_stream(const PagedAttn a) {
  using L = SL<HD>;
  using T = __nv_bfloat16;
  constexpr int NT = HD / 8;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ Kv8PlanSmem s_plan;
  __shared__ StreamBars<HD> bar;
  __shared__ float s_m[L::kUse][kTile], s_l[L::kUse][kTile], s_gm[kTile], s_sum[kTile];
  __shared__ int s_bad[2], s_fail;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t = lane & 3, n8 = lane >> 2;
  const int pmask = (1 << a.c.shift) - 1;
  if (tid == 0) {
    for (int i = 0; i < L::kNst; ++i) {
      mbar_init(&bar.full[i], L::kCopy * 32);
      mbar_init(&bar.empty[i], L::kUse / 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar.q_full[i], L::kCopy * 32);
      mbar_init(&bar.q_free[i], L::kUse);
    }
    mbar_init_fence();
    s_bad[0] = s_bad[1] = s_fail = 0;
    a.desc[blockIdx.x].nr = 0;
  }
  Kv8Cursor cur = kv8_plan<kTile, kUnit, L::kThreads>(a, s_plan);  // (with block barriers)
  pdl_launch_dependents();
  uint32_t n = 0;  // stages so far
  Ring<L::kNst> ring;
  bool bad = false;
  Kv8Seg sg;
  // stages of a segment: first .. last - 1, of keys kb .. ke - 1, counted from seg0
  int seg0, kb, ke, first, last;
  auto stages = [&]() {
    const Kv8Item& it = sg.it;
    seg0 = (it.unit0 + sg.u0) * kUnit;
    kb = max(it.lo, seg0);
    ke = min(it.hi + 1, seg0 + sg.nu * kUnit);
    last = ke > kb ? (ke - seg0 + L::kKeys - 1) / L::kKeys : 0;
    first = ke > kb ? (kb - seg0) / L::kKeys : 0;
  };

  if (warp >= L::kUse) {
    // ------------------------------------------------------------ copies
    const int ct = tid - L::kUse * 32;
    const int ch = ct % L::kChunks, r0 = ct / L::kChunks;
    constexpr int kPass = L::kCopy * 32 / L::kChunks;  // rows of a pass
    for (uint32_t i = 0; kv8_next<kTile, kUnit>(a, cur, sg); ++i) {
      const Kv8Item& it = sg.it;
      stages();
      PageWalk walk(a.c, a.err);
      walk.start(it.b, seg0 + first * L::kKeys, kb, ke);
      if (i >= 2) p_wait(&bar.q_free[i & 1], ((i >> 1) - 1) & 1, bad);
      for (int x = ct; x < kTile * L::kChunks; x += L::kCopy * 32) {
        const int row = x / L::kChunks, r = it.r0 + min(row, it.nr - 1), m = a.byG(r);
        cp_async16(smem_u32(smem) + L::kQ + (i & 1) * L::kQBytes + L::P::place(row, ch),
                   static_cast<const T*>(a.q) + ((int64_t)it.b * a.M + m) * a.q_stride +
                       (int64_t)(sg.g * a.G + r - m * a.G) * HD + ch * 8,
                   true);
      }
      p_arrive(&bar.q_full[i & 1]);
      const char* const kp = a.k + sg.g * a.c.head() + ch * 16;
      const char* const vp = a.v + sg.g * a.c.head() + ch * 16;
      for (int s = first; s < last; ++s, ++n, ring.next()) {
        if (n >= (uint32_t)L::kNst) p_wait(&bar.empty[ring.at], ring.phase ^ 1, bad);
        const uint32_t dst = smem_u32(smem) + ring.at * L::kStage;
        int look[L::kKeys / 16];
#pragma unroll
        for (int j = 0; j < L::kKeys / 16; ++j) look[j] = walk.page(seg0 + s * L::kKeys + 16 * j);
#pragma unroll
        for (int j = 0; j < L::kKeys / kPass; ++j) {
          const int r = r0 + j * kPass, key = seg0 + s * L::kKeys + r;
          const bool in = key >= kb && key < ke;
          const size_t off =
              (size_t)look[j * kPass / 16] * a.c.bytes + (size_t)(key & pmask) * (HD * 2);
          const uint32_t at = dst + L::P::place(r, ch);
          cp_async16(at, kp + (in ? off : 0), in);
          cp_async16(at + L::kSide, vp + (in ? off : 0), in);
        }
        p_arrive(&bar.full[ring.at]);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    // ------------------------------------------------------------ products
    const int grp = warp & 3, team = warp >> 2;
    float* const Ox = reinterpret_cast<float*>(smem + L::kExchange);
    for (uint32_t i = 0; kv8_next<kTile, kUnit>(a, cur, sg); ++i) {
      const Kv8Item& it = sg.it;
      stages();
      uint32_t qf[HD / 16][4];
      p_wait(&bar.q_full[i & 1], (i >> 1) & 1, bad);
#pragma unroll
      for (int k = 0; k < HD / 16; ++k)
        ldsm4(smem_u32(smem) + L::kQ + (i & 1) * L::kQBytes + L::P::place(lane & 15, 2 * k + (lane >> 4)),
              qf[k]);
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar.q_free[i & 1]);
      RowTile<HD> w;
      w.start(a, it, 0);
      const int full_lo = kv8_row_lo(it, it.hi, a.window), full_hi = kv8_row_pos(a, it, it.r0);
      for (int s = first; s < last; ++s, ++n, ring.next()) {
        if ((int)(n & 1) != team) continue;
        p_wait(&bar.full[ring.at], ring.phase, bad);
        const int kk0 = grp * 16, k0 = seg0 + s * L::kKeys + kk0;
        if (k0 < ke && k0 + 16 > kb) {
          const uint32_t sk = smem_u32(smem) + ring.at * L::kStage;
          const bool full = k0 >= full_lo && k0 + 15 <= full_hi;
          if (bf16_step<typename L::P, HD>(w, qf, sk, sk + L::kSide, kk0, k0, full, a.scale))
            s_bad[i & 1] = 1;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar.empty[ring.at]);
      }
      // ---- the warps' parts together: weights from all maxima and sums, then the second team's
      // outputs by way of shared memory into the first's
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        w.ls[x] += __shfl_xor_sync(0xffffffffu, w.ls[x], 1);
        w.ls[x] += __shfl_xor_sync(0xffffffffu, w.ls[x], 2);
        if (t == 0) {
          s_m[warp][n8 + 8 * x] = w.mx[x];
          s_l[warp][n8 + 8 * x] = w.ls[x];
        }
      }
      named_sync(1, L::kUse * 32);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int row = n8 + 8 * x;
        float gm = -INFINITY, sum = 0.f;
#pragma unroll
        for (int y = 0; y < L::kUse; ++y) gm = fmaxf(gm, s_m[y][row]);
#pragma unroll
        for (int y = 0; y < L::kUse; ++y) sum = fmaf(part_weight(s_m[y][row], gm), s_l[y][row], sum);
        const float wt = sum != 0.f ? part_weight(w.mx[x], gm) / sum : 0.f;
        if (warp == 0 && t == 0) s_gm[row] = gm, s_sum[row] = sum;
        float* p = Ox + (size_t)(grp * kTile + row) * (HD + 4) + 2 * t;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          w.o[j][2 * x] *= wt, w.o[j][2 * x + 1] *= wt;
          if (team == 1)
            *reinterpret_cast<float2*>(p + 8 * j) = make_float2(w.o[j][2 * x], w.o[j][2 * x + 1]);
        }
      }
      named_sync(1, L::kUse * 32);
      if (team == 0) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float* p = Ox + (size_t)(grp * kTile + n8 + 8 * x) * (HD + 4) + 2 * t;
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const float2 u = *reinterpret_cast<const float2*>(p + 8 * j);
            *reinterpret_cast<float2*>(p + 8 * j) =
                make_float2(w.o[j][2 * x] + u.x, w.o[j][2 * x + 1] + u.y);
          }
        }
      }
      if (tid == 0) s_bad[(i + 1) & 1] = 0;
      named_sync(1, L::kUse * 32);
      finish_rows<T, HD, 4, kTile, L::kUse * 32>(a, sg, kb, ke, Ox, nullptr, s_gm, s_sum, s_bad[i & 1],
                                                 nullptr, tid);
      if (!sg.whole() && sg.u0 == 0 && tid == 0) a.desc[blockIdx.x] = kv8_desc(a, cur, sg);
      named_sync(1, L::kUse * 32);  // the exchange is read
    }
  }
  if (bad) s_fail = 1;
  __syncthreads();
  if (tid == 0 && s_fail && a.err) atomicOr(a.err, (int)kErrTimeout);
}

}  // namespace ssd
