// paged_stream.cuh -- attention over pages for up to 16 query rows a KV head (decoding, narrow
// verifications; bf16) over long sequences. Included by paged_attention.cu.
//
// One block an SM, so that its stretch of the plan's line is one stream of stages (64 keys, K and V)
// through a ring of 160 KB: four warps copy (cp.async), across items, and never wait for their end;
// eight take every other stage by fours, 16 keys each, and at an item's end join what they have while the
// ring fills with the next one's.
//
// Bound by bytes: pages of 16, 64 and 256 positions are read at 6.5, 7.2 and 7.4 TB/s (262144 keys more
// of 8 KV heads); 24 ragged sequences of 32 heads, 5 rows each, window 2500, pages of 16: 117 us = 5.8
// TB/s, where an item of 20 stages takes 2 us longer than its bytes, since the copying warps' 160 KB do
// not last for the joins of eight warps. mma.sync is the next bound: 24 instructions of about 19 cycles
// a warp's step (9 to 16 rows: 48), two warps a quarter of an SM, are 0.25 of the 0.7 us that a stage's
// bytes take.
#pragma once

#include "attn_wide.cuh"

namespace ssd {

namespace {

template <int HD, int NB>
struct SL {
  using P = PL<__nv_bfloat16, HD, 1, NB>;  // its stages and places
  static constexpr int kRows = 8 * NB;
  static constexpr int kKeys = P::kKeys, kChunks = P::kChunks;
  static constexpr uint32_t kStage = P::kStage, kSide = P::kSide;
  static constexpr int kNst = 160 * 1024 / (int)kStage;
  static constexpr uint32_t kExchange = kNst * kStage;                 // where it begins
  static constexpr uint32_t kQ = kExchange + 4 * kRows * (HD + 4) * 4;  // two items' queries
  static constexpr uint32_t kQBytes = kRows * HD * 2;
  static constexpr uint32_t kSmem = kQ + 2 * kQBytes;
  static constexpr int kUse = 8, kCopy = 4;  // warps
  static constexpr int kThreads = (kUse + kCopy) * 32;
};

template <int NST>
struct StreamBars {
  uint64_t full[NST], empty[NST];  // a stage is there; is read
  uint64_t q_full[2], q_free[2];
};

// Named barrier over the first `threads` threads; whether x holds for one of them.
__device__ __forceinline__ bool named_or(int id, int threads, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %3, 0;\n\t"
      "bar.red.or.pred q, %1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(id), "r"(threads), "r"((uint32_t)x)
      : "memory");
  return r != 0;
}

}  // namespace

template <int HD, int NB>
__global__ void __launch_bounds__(SL<HD, NB>::kThreads, 1) k_paged_stream(const PagedAttn a) {
  using L = SL<HD, NB>;
  using T = __nv_bfloat16;
  constexpr int kRows = L::kRows;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ Kv8PlanSmem s_plan;
  __shared__ StreamBars<L::kNst> bar;
  __shared__ float s_m[L::kUse][kRows], s_l[L::kUse][kRows], s_gm[kRows], s_sum[kRows];
  __shared__ int s_bad[2], s_fail, s_more[2];
  __shared__ Kv8Seg s_seg[2];  // the items under way, as the copying warps hand them on
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t = lane & 3, n8 = lane >> 2;
  pdl_wait();
  if (tid == 0) {
    for (int i = 0; i < L::kNst; ++i) {
      mbar_init(&bar.full[i], L::kCopy * 32);
      mbar_init(&bar.empty[i], L::kUse / 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar.q_full[i], L::kCopy * 32 + 1);
      mbar_init(&bar.q_free[i], L::kUse);
    }
    mbar_init_fence();
    s_bad[0] = s_bad[1] = s_fail = 0;
    a.desc[blockIdx.x].nr = 0;
  }
  Kv8Cursor cur = kv8_plan<kRows, kUnit, L::kThreads>(a, s_plan);  // (with block barriers)
  pdl_launch_dependents();
  uint32_t n = 0;  // stages so far
  Ring<L::kNst> ring;
  bool bad = false;
  // stages of a segment: first .. last - 1, of keys kb .. ke - 1, counted from seg0
  struct Span {
    int seg0, kb, ke, first, last;
    __device__ __forceinline__ Span(const Kv8Seg& s) {
      seg0 = (s.it.unit0 + s.u0) * kUnit;
      kb = max(s.it.lo, seg0);
      ke = min(s.it.hi + 1, seg0 + s.nu * kUnit);
      last = ke > kb ? (ke - seg0 + L::kKeys - 1) / L::kKeys : 0;
      first = ke > kb ? (kb - seg0) / L::kKeys : 0;
    }
  };

  if (warp >= L::kUse) {
    // ------------------------------------------------------------ copies
    const int ct = tid - L::kUse * 32;
    const int ch = ct % L::kChunks, r0 = ct / L::kChunks;
    constexpr int kPass = L::kCopy * 32 / L::kChunks;  // rows of a pass
    const uint32_t at0 = L::P::place(r0, ch);
    // the next segment is found, and its first pages are looked up, while the last stage of the one
    // before waits for its place
    Kv8Seg next;
    PageWalk ahead(a.c, a.err);
    auto look = [&]() -> bool {
      if (!kv8_next<kRows, kUnit>(a, cur, next)) return false;
      const Span n(next);
      ahead.start(next.it.b, n.seg0 + n.first * L::kKeys, n.kb, n.ke);
      if (ct == 0 && !next.whole() && next.u0 == 0) a.desc[blockIdx.x] = kv8_desc(a, cur, next);
      return true;
    };
    bool more = look();
    for (uint32_t i = 0;; ++i) {
      if (i >= 2) p_wait(&bar.q_free[i & 1], ((i >> 1) - 1) & 1, bad);
      const Kv8Seg sg = next;
      const Kv8Item& it = sg.it;
      if (ct == 0) {
        s_more[i & 1] = more;
        s_seg[i & 1] = sg;
        mbar_arrive(&bar.q_full[i & 1]);
      }
      if (!more) {
        mbar_arrive(&bar.q_full[i & 1]);
        break;
      }
      for (int x = ct; x < kRows * L::kChunks; x += L::kCopy * 32) {
        const int row = x / L::kChunks, r = it.r0 + min(row, it.nr - 1), m = a.byG(r);
        cp_async16(smem_u32(smem) + L::kQ + (i & 1) * L::kQBytes + L::P::place(row, ch),
                   static_cast<const T*>(a.q) + ((int64_t)it.b * a.M + m) * a.q_stride +
                       (int64_t)(sg.g * a.G + r - m * a.G) * HD + ch * 8,
                   true);
      }
      p_arrive(&bar.q_full[i & 1]);
      const Span sp(sg);
      const int seg0 = sp.seg0, kb = sp.kb, ke = sp.ke, last = sp.last;
      PageWalk walk = ahead;
      if (sp.first >= last) more = look();
      const char* const kp = a.k + sg.g * a.c.head() + r0 * HD * 2 + ch * 16;
      const char* const vp = kp + (a.v - a.k);
      for (int s = sp.first; s < last; ++s, ++n, ring.next()) {
        if (s == last - 1) more = look();
        const int k0 = seg0 + s * L::kKeys;
        size_t off[L::kKeys / 16];
        find_keys<L::kKeys, HD * 2>(walk, k0, off);
        if (n >= (uint32_t)L::kNst) p_wait(&bar.empty[ring.at], ring.phase ^ 1, bad);
        const uint32_t dst = smem_u32(smem) + ring.at * L::kStage + at0;
        copy_keys<L::kKeys, HD * 2, kPass>(
            off, kp, r0, k0, kb, ke, [&](int r) { return L::P::template place_from<kPass>(dst, r); });
        copy_keys<L::kKeys, HD * 2, kPass>(off, vp, r0, k0, kb, ke, [&](int r) {
          return L::P::template place_from<kPass>(dst, r) + L::kSide;
        });
        p_arrive(&bar.full[ring.at]);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    // ------------------------------------------------------------ products
    const int grp = warp & 3, team = warp >> 2;
    float* const Ox = reinterpret_cast<float*>(smem + L::kExchange);
    for (uint32_t i = 0;; ++i) {
      p_wait(&bar.q_full[i & 1], (i >> 1) & 1, bad);
      // (all or none go on: a wait that gave up leaves nobody alone at a barrier)
      if (named_or(1, L::kUse * 32, bad || !s_more[i & 1])) break;
      const Kv8Seg sg = s_seg[i & 1];
      const Kv8Item& it = sg.it;
      const Span sp(sg);
      const int seg0 = sp.seg0, kb = sp.kb, ke = sp.ke;
      uint32_t qf[HD / 16][NB][2];
      const uint32_t sq = smem_u32(smem) + L::kQ + (i & 1) * L::kQBytes;
#pragma unroll
      for (int k = 0; k < HD / 16; k += 3 - NB) {  // 8 rows x 32 columns, or 16 x 16
        uint32_t u[4];
        ldsm4(sq + (NB == 1 ? L::P::place(lane & 7, 2 * k + (lane >> 3))
                            : L::P::place((lane & 7) + ((lane >> 4) << 3), 2 * k + (lane >> 3 & 1))),
              u);
#pragma unroll
        for (int x = 0; x < 4; ++x) qf[NB == 1 ? k + (x >> 1) : k][NB == 1 ? 0 : x >> 1][x & 1] = u[x];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar.q_free[i & 1]);
      ColTile<HD, NB> w;
      w.start(a, it, 0);
      const int full_lo = kv8_row_lo(it, it.hi, a.window), full_hi = kv8_row_pos(a, it, it.r0);
      for (int s = sp.first; s < sp.last; ++s, ++n, ring.next()) {
        if ((int)(n & 1) != team) continue;
        p_wait(&bar.full[ring.at], ring.phase, bad);
        const int kk0 = grp * 16, k0 = seg0 + s * L::kKeys + kk0;
        if (k0 < ke && k0 + 16 > kb) {
          const uint32_t sk = smem_u32(smem) + ring.at * L::kStage;
          const bool full = k0 >= full_lo && k0 + 15 <= full_hi;
          if (w.template step<typename L::P>(qf, sk, sk + L::kSide, kk0, k0, full, a.scale))
            s_bad[i & 1] = 1;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar.empty[ring.at]);
      }
      // ---- the warps' parts together: weights from all maxima and sums, then the second team's
      // outputs by way of shared memory into the first's
      w.sum_up();
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (n8 == 0) {
            s_m[warp][8 * b + 2 * t + x] = w.mx[b][x];
            s_l[warp][8 * b + 2 * t + x] = w.ls[b][x];
          }
      named_sync(1, L::kUse * 32);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int row = 8 * b + 2 * t + x;
          float gm = -INFINITY, sum = 0.f;
#pragma unroll
          for (int y = 0; y < L::kUse; ++y) gm = fmaxf(gm, s_m[y][row]);
#pragma unroll
          for (int y = 0; y < L::kUse; ++y) sum = fmaf(part_weight(s_m[y][row], gm), s_l[y][row], sum);
          const float wt = sum != 0.f ? part_weight(w.mx[b][x], gm) / sum : 0.f;
          if (warp == 0 && n8 == 0) s_gm[row] = gm, s_sum[row] = sum;
          float* p = Ox + (size_t)(grp * kRows + row) * (HD + 4) + n8;
#pragma unroll
          for (int j = 0; j < HD / 16; ++j) {
            w.o[j][b][x] *= wt, w.o[j][b][2 + x] *= wt;
            if (team == 1) p[16 * j] = w.o[j][b][x], p[16 * j + 8] = w.o[j][b][2 + x];
          }
        }
      named_sync(1, L::kUse * 32);
      if (team == 0) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float* p = Ox + (size_t)(grp * kRows + 8 * b + 2 * t + x) * (HD + 4) + n8;
#pragma unroll
            for (int j = 0; j < HD / 16; ++j) {
              p[16 * j] += w.o[j][b][x];
              p[16 * j + 8] += w.o[j][b][2 + x];
            }
          }
      }
      if (tid == 0) s_bad[(i + 1) & 1] = 0;
      named_sync(1, L::kUse * 32);
      finish_rows<T, HD, 4, kRows, L::kUse * 32>(a, sg, kb, ke, Ox, nullptr, s_gm, s_sum, s_bad[i & 1],
                                                 tid, [](int, int, const float (&)[8]) {});
      named_sync(1, L::kUse * 32);  // the exchange is read
    }
  }
  if (bad) s_fail = 1;
  __syncthreads();
  if (tid == 0 && s_fail && a.err) atomicOr(a.err, (int)kErrTimeout);
}

}  // namespace ssd
