// paged_wide.cuh -- attention over pages for many query rows a KV head (wide verifications, grouped
// queries, prompt chunks; bf16, head_dim 128), on the 5th-generation tensor cores. Included by
// paged_attention.cu.
//
// A tile (the plan's items) has one or two accumulators of 128 query rows each; a block, one an SM,
// walks its keys 64 at a time. Its warps work side by side:
//  - four copy keys and values as they are (cp.async) to a ring of steps in shared memory, rows of
//    128 bytes with the 128-byte swizzle; keys are a K-major operand, values, whose columns lie one
//    behind the other, an MN-major one;
//  - one an accumulator issues S = Q K^T (tcgen05.mma, 128 x 64 x 128, fp32 in tensor memory, two
//    buffers) for a step while the softmax of the step before is at work, another one O += P V,
//    P read from tensor memory, as soon as a softmax is done;
//  - four an accumulator do the softmax, a thread per row: the row's 64 scores into registers, their
//    maximum, p = 2^(s - ref) as two bf16 parts, which take the place of S. ref lies 8 (in powers of
//    two) above what the row's maximum was the last time it passed ref, so O is rescaled in tensor
//    memory only then, and no p is above 1: sums stay as far from fp32's end as in the other kernels.
// A probability's two parts keep 16 bits of it, as in the kernels for fewer rows. One part is not enough:
// an error of 2^-8 of each weight is one of up to 2^-8 sum w |v|, many units of an output whose values
// cancel (17 rows of 64 heads over 16000 keys were 0.0022 off for 0.0017 with fp32 weights, which two
// parts give back). The second part is half as many products again, conversions and stores: 28 -> 31 us,
// 73 -> 78, 98 -> 118 and 174 -> 210 for the sizes below.
//
// 17 rows of 64 heads over 8 x 16000 keys: 31 us; 8 x 100000 keys, 64 rows a KV head 78 us (5.3 TB/s),
// 256 rows 118, 512 rows 210 (1.0 PFLOP/s, the second parts' products not counted). Of the 31, 6.4 lie in
// front of the first scores (the plan 1.8, the next item's look-up, the first pages and keys), 15 are
// 13 steps of 64 keys, 3 the outputs, 4 the join. A step of two accumulators takes 1.1 us with 136 rows,
// 1.27 with 256, where 0.7 would be its bytes and 0.85 the products of 256 rows at the nominal rate: the
// softmax's warps, two a quarter of an SM. (With one part and two threads a row, which halve a row's chain
// but add instructions and barriers, 17 to 128 rows were no faster, 136 and more 10 to 15 % slower.)
#pragma once

#include "attn_wide.cuh"

namespace ssd {

namespace {

// A block's tile of TILES accumulators.
template <int TILES>
struct PWideL {
  static constexpr int kRows = TILES * kWRows;
  // warps: 4 TILES softmax, 4 copies, then the accumulators' scores and outputs
  static constexpr int kSoft = 4 * TILES, kQk = kSoft + 4, kPv = kQk + TILES;
  static constexpr int kThreads = (kPv + TILES) * 32;
  static constexpr int kNst = 6 - TILES;  // steps of the ring (five for two accumulators: no faster)
  static constexpr uint32_t kStep = 2 * kWKTile;
  static constexpr uint32_t kSmem = 2 * TILES * kWQHalf + kNst * kStep + 1024;  // queries, ring; alignment
  static constexpr uint32_t kCols = 256 * TILES;  // tensor memory: S and P (2 x 64 each), O
};
constexpr float kPGrow = 8.f;
constexpr float kPFar = 1048576.f;  // 2^20: half a unit there is 2^-4, and ref is rounded twice

// Instruction descriptors: bf16 operands, fp32 accumulator, M = 128; values are MN-major (bit 16).
constexpr uint32_t kPIdesc = idesc_bf16_f32(128, kWKeys);
constexpr uint32_t kPIdescV = idesc_bf16_f32(128, kWHd) | 1u << 16;

// Barriers: a ring step's keys and values stored, and free again (one each for both: with barriers of
// their own, which 128 threads arrive at, 8 x 100000 keys took 78 us where they took 72 so, a
// probability in one part); of the two buffers of S: scores there, probabilities there, output added;
// queries of the segment stored.
template <int TILES>
struct PWideBars {
  uint64_t full[PWideL<TILES>::kNst], free[PWideL<TILES>::kNst];
  uint64_t s_done[TILES][2], p_full[TILES][2], o_done[TILES][2], q_full[TILES];
  uint64_t drained;  // after a wait that gave up: the products still in flight are done
};

// The phase that step n completes on its buffer's barrier; after a wait that gave up, no thread of
// this role waits again: it runs through its steps, meets its barriers and reports.
__device__ __forceinline__ void p_wait2(uint64_t (&b)[2], uint32_t n, bool& bad) {
  if (!bad) bad = !w_sleep(&b[n & 1], (n >> 1) & 1);
}
}  // namespace

template <int TILES>
__global__ void __launch_bounds__(PWideL<TILES>::kThreads, 1) k_paged_wide(const PagedAttn a) {
  using L = PWideL<TILES>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ Kv8PlanSmem s_plan;
  __shared__ PWideBars<TILES> bar;
  __shared__ uint32_t s_tmem;
  __shared__ int s_fail, s_more[TILES];
  // i + 1 at i % 8 where a value of the block's segment i was zeroed. Segments have a step or more, so the
  // copies are at most kNst segments ahead of a softmax that has not begun its next one.
  __shared__ uint32_t s_odd[8];
  static_assert(L::kNst < 8, "a place for each segment under way");
  __shared__ Kv8Cursor s_cur[TILES];  // of the softmax warps
  __shared__ Kv8Seg s_seg[TILES];
  unsigned char* const smem =
      reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char* const Qs = smem;
  unsigned char* const Ks = Qs + 2 * TILES * kWQHalf;  // [kNst] keys, then values
  const int tid = threadIdx.x, warp = tid >> 5;
  const int pmask = (1 << a.c.shift) - 1;

  pdl_wait();
  if (tid == 0) {
    for (int i = 0; i < L::kNst; ++i) {
      mbar_init(&bar.full[i], 128);
      mbar_init(&bar.free[i], TILES);
    }
    for (int t = 0; t < TILES; ++t) {
      for (int i = 0; i < 2; ++i) {
        mbar_init(&bar.p_full[t][i], 128);
        mbar_init(&bar.s_done[t][i], 1);
        mbar_init(&bar.o_done[t][i], 1);
      }
      mbar_init(&bar.q_full[t], 128);
    }
    mbar_init(&bar.drained, 2 * TILES);
    mbar_init_fence();
    for (int i = 0; i < 8; ++i) s_odd[i] = 0;
    s_fail = 0;
    a.desc[blockIdx.x].nr = 0;
  }
  if (warp == L::kQk) tc_alloc(&s_tmem, L::kCols);
  tc_fence_before();
  Kv8Cursor cur = kv8_plan<L::kRows, kWKeys, L::kThreads>(a, s_plan);  // (with block barriers)
  tc_fence_after();
  pdl_launch_dependents();
  // tensor memory: the accumulators' scores, two buffers each, then their outputs
  const uint32_t tm = s_tmem;
  constexpr uint32_t kS = 2 * kWKeys, kO = TILES * kS;
  if (warp < L::kSoft && (tid & 127) == 0) s_cur[tid >> 7] = cur;
  uint32_t n = 0;  // steps so far: the phases of the two buffers
  Ring<L::kNst> ring;
  bool bad = false;

  if (warp >= L::kQk && warp < L::kPv) {
    // ------------------------------------------------------------ scores
    Kv8Seg sg;
    const uint32_t one = w_elect();
    const int t = warp - L::kQk;
    const uint32_t tmS = tm + t * kS;
    const uint64_t dq = sdesc_k128(smem_u32(Qs)) + (2 * t * kWQHalf >> 4);
    const uint64_t dk = sdesc_k128(smem_u32(Ks));
    for (uint32_t seg = 0; kv8_next<L::kRows, kWKeys>(a, cur, sg); ++seg) {
      p_wait(&bar.q_full[t], seg & 1, bad);
      for (int i = 0; i < sg.nu; ++i, ++n, ring.next()) {
        p_wait(&bar.full[ring.at], ring.phase, bad);
        if (n >= 2) p_wait2(bar.o_done[t], n - 2, bad);  // P of that step was read there
        w_smem_fence();
        __syncwarp();
        tc_fence_after();
        const uint32_t buf = n & 1;
        if (t == 0 || sg.it.nr > t * kWRows)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            w_mma(tmS + buf * kWKeys, dq + (((k >> 2) * kWQHalf + (k & 3) * 32) >> 4),
                  dk + ((ring.at * L::kStep + (k >> 2) * kWKHalf + (k & 3) * 32) >> 4), kPIdesc, k > 0,
                  one);
        if (one) tc_commit(&bar.s_done[t][buf]);
      }
    }
  } else if (warp >= L::kPv) {
    // ------------------------------------------------------------ outputs
    Kv8Seg sg;
    const uint32_t one = w_elect();
    const int t = warp - L::kPv;
    const uint32_t tmS = tm + t * kS, tmO = tm + kO + t * kWHd;
    const uint64_t dv = w_desc_mn(smem_u32(Ks + kWKTile));
    while (kv8_next<L::kRows, kWKeys>(a, cur, sg))
      for (int i = 0; i < sg.nu; ++i, ++n, ring.next()) {
        p_wait(&bar.full[ring.at], ring.phase, bad);
        p_wait2(bar.p_full[t], n, bad);
        w_smem_fence();
        __syncwarp();
        tc_fence_after();
        const uint32_t buf = n & 1;
        if (t == 0 || sg.it.nr > t * kWRows)
#pragma unroll
          for (int k = 0; k < kWKeys / 16; ++k)  // 16 keys: 8 words of a part of P, two 8-row groups of V
#pragma unroll
            for (int x = 1; x >= 0; --x)  // (second parts first, as the small ones)
              w_mma_ts(tmO, tmS + buf * kWKeys + x * (kWKeys / 2) + 8 * k,
                       dv + ((ring.at * L::kStep + k * 2048) >> 4), kPIdescV, i > 0 || k > 0 || x == 0,
                       one);
        if (one) {
          tc_commit(&bar.o_done[t][buf]);
          tc_commit(&bar.free[ring.at]);
        }
      }
  } else if (warp >= L::kSoft) {
    // ------------------------------------------------------------ copies
    const int ct = tid - L::kSoft * 32;
    const int ch = ct & 15, r0 = ct >> 4;  // chunk of rows r0 + 8 j
    const uint32_t to = (ch >> 3) * kWKHalf;
    // values that are no numbers to zero, in a step that not every row sees whole (each thread in the
    // chunks that it copied)
    uint32_t seg = 0;
    auto clean = [&]() {
      unsigned char* const st = Ks + ring.at * L::kStep + kWKTile + to;
      uint32_t any = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint4* p = reinterpret_cast<uint4*>(st + w_place(r0 + 8 * j, ch & 7));
        uint4 u = *p;
        u.x = numbers(u.x, any), u.y = numbers(u.y, any);
        u.z = numbers(u.z, any), u.w = numbers(u.w, any);
        *p = u;
      }
      if (any) s_odd[seg & 7] = seg + 1;  // (published by the arrival that follows)
    };
    Kv8Seg sg;
    for (; kv8_next<L::kRows, kWKeys>(a, cur, sg); ++seg) {
      const Kv8Item& it = sg.it;
      const int k00 = (it.unit0 + sg.u0) * kWKeys;
      const int full_lo = kv8_row_lo(it, it.hi, a.window), full_hi = kv8_row_pos(a, it, it.r0);
      const char* const kp = a.k + sg.g * a.c.head() + r0 * kWHd * 2 + ch * 16;
      const char* const vp = kp + (a.v - a.k);
      PageWalk walk(a.c, a.err);
      walk.start(it.b, k00, max(k00, it.lo), min(k00 + sg.nu * kWKeys, it.hi + 1));
      for (int i = 0; i < sg.nu; ++i, ++n, ring.next()) {
        const int k0 = k00 + i * kWKeys;
        const uint32_t dst = smem_u32(Ks) + ring.at * L::kStep + to + w_place(r0, ch & 7);
        size_t off[kWKeys / 16];
        find_keys<kWKeys, kWHd * 2>(walk, k0, off);
        if (n >= (uint32_t)L::kNst) p_wait(&bar.free[ring.at], ring.phase ^ 1, bad);
        copy_keys<kWKeys, kWHd * 2, 8>(off, kp, r0, k0, it.lo, it.hi + 1,
                                       [&](int r) { return dst + (uint32_t)(r * 128); });
        copy_keys<kWKeys, kWHd * 2, 8>(off, vp, r0, k0, it.lo, it.hi + 1,
                                       [&](int r) { return dst + kWKTile + (uint32_t)(r * 128); });
        if (k0 >= full_lo && k0 + kWKeys - 1 <= full_hi) {
          p_arrive(&bar.full[ring.at]);
        } else {
          asm volatile("cp.async.wait_all;" ::: "memory");
          clean();
          mbar_arrive(&bar.full[ring.at]);
        }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    // ------------------------------------------------------------ softmax
    const int t = TILES == 1 ? 0 : warp >> 2, ttid = tid & 127;  // the accumulator, its thread
    const int row = tid;  // of the tile
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tmS = tm + t * kS + lanes, tmO = tm + kO + t * kWHd + lanes;
    for (uint32_t seg = 0;; ++seg) {
      // the segment stands in shared memory: the steps need the registers
      if (ttid == 0) s_more[t] = kv8_next<L::kRows, kWKeys>(a, s_cur[t], s_seg[t]);
      named_sync(1 + t, 128);
      if (!s_more[t]) break;
      const Kv8Seg& sg = s_seg[t];
      const Kv8Item& it = sg.it;
      // queries, sixteen lanes a row (rows past the last: the last one's, not used); the products
      // of the segment before are done with theirs
      {
        const int ch = tid % 16;
        const __nv_bfloat16* const q0 = static_cast<const __nv_bfloat16*>(a.q) + ch * 8 +
                                        (int64_t)it.b * a.M * a.q_stride + (int64_t)sg.g * a.G * kWHd;
        unsigned char* const own = Qs + (2 * t + (ch >> 3)) * kWQHalf;
        uint4 u[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int r = it.r0 + min(t * kWRows + j * 8 + ttid / 16, it.nr - 1), m = a.byG(r);
          u[j] = *reinterpret_cast<const uint4*>(q0 + m * a.q_stride + (r - m * a.G) * kWHd);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j)
          *reinterpret_cast<uint4*>(own + w_place(j * 8 + ttid / 16, ch & 7)) = u[j];
      }
      w_smem_fence();
      tc_fence_before();
      mbar_arrive(&bar.q_full[t]);
      const bool live = warp * 32 < it.nr;  // the warp has rows
      const int k00 = (it.unit0 + sg.u0) * kWKeys;
      const int full_lo = kv8_row_lo(it, it.hi, a.window);
      const int full_hi = kv8_row_pos(a, it, it.r0);
      const int phi = row < it.nr ? kv8_row_pos(a, it, it.r0 + row) : -1;
      const int plo = row < it.nr ? kv8_row_lo(it, phi, a.window) : 0;
      float ref = -INFINITY, ls = 0.f;  // of the row
      // Some row of the warp has a ref whose rounding is more than a small part of a power of two: the
      // product in the exponent is not rounded, so such a row's scores are, beforehand, and taken from
      // ref (in the branch below, which every step then takes).
      bool far = false;
      for (int i = 0; i < sg.nu; ++i, ++n) {
        p_wait2(bar.s_done[t], n, bad);
        __syncwarp();
        tc_fence_after();
        if (live) {
          const int k0 = k00 + i * kWKeys;
          const bool full = k0 >= full_lo && k0 + kWKeys - 1 <= full_hi;
          const uint32_t at = tmS + (n & 1) * kWKeys;
          uint32_t r[64];
          w_ld64(at, r);
          if (!full) {
            const int lo = plo - k0, hi = phi - k0;
#pragma unroll
            for (int x = 0; x < 64; ++x)
              if (x < lo || x > hi) r[x] = 0xff800000u;  // -inf
          }
          float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int x = 0; x < 64; x += 8)
#pragma unroll
            for (int y = 0; y < 4; ++y)
              m[y] = w_max3(m[y], __uint_as_float(r[x + 2 * y]), __uint_as_float(r[x + 2 * y + 1]));
          const float mx = fmaxf(w_max3(m[0], m[1], m[2]), m[3]) * a.scale;
          const bool grow = mx > ref;
          float c = a.scale, base = ref;  // what the exponents below are taken from
          if (__any_sync(0xffffffffu, grow || far)) {
            float f = 1.f;
            if (grow) {
              const float up = mx + kPGrow;
              f = ref == -INFINITY ? 0.f : exp2f(ref - up);
              ref = up;
              ls *= f;
            }
            if (i > 0) {
              p_wait2(bar.o_done[t], n - 1, bad);
              __syncwarp();
              tc_fence_after();
              if (__any_sync(0xffffffffu, grow)) {
#pragma unroll 1
                for (int q = 0; q < 8; ++q) {
                  uint32_t o[16];
                  w_ld16(tmO + 16 * q, o);
#pragma unroll
                  for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
                  w_st16(tmO + 16 * q, o);
                }
              }
            }
            base = ref;
            const bool own = ref > -INFINITY && fabsf(ref) >= kPFar;
            far = __any_sync(0xffffffffu, own);
            if (far) {
              const float by = own ? c : 1.f, off = own ? ref : 0.f;
#pragma unroll
              for (int x = 0; x < 64; ++x)
                r[x] = __float_as_uint(__fsub_rn(__fmul_rn(__uint_as_float(r[x]), by), off));
              if (own) c = 1.f, base = 0.f;
            }
          }
          const float top = base == -INFINITY ? 0.f : base;
          const uint64_t c2 = pack2(c, c), t2 = pack2(-top, -top);
          uint64_t sum2 = 0;
          uint32_t lo[32];  // the probabilities' second parts
#pragma unroll
          for (int x = 0; x < 64; x += 2) {
            const float2 z =
                unpack2(fma2(pack2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), c2, t2));
            const float p0 = ex2_approx(z.x), p1 = ex2_approx(z.y);
            sum2 = add2(sum2, pack2(p0, p1));
            split2(p0, p1, r[x / 2], lo[x / 2]);
          }
          const float2 sum = unpack2(sum2);
          ls += sum.x + sum.y;
          w_st32(at, r);
          w_st32(at + kWKeys / 2, lo);
          w_st_wait();
        }
        tc_fence_before();
        mbar_arrive(&bar.p_full[t][n & 1]);
      }
      p_wait2(bar.o_done[t], n - 1, bad);
      __syncwarp();
      tc_fence_after();
      // ---- the rows' outputs, or the block's part of them
      if (live) {
        const bool whole = sg.whole(), odd = *(volatile uint32_t*)&s_odd[seg & 7] == seg + 1;
        const int slot = 2 * blockIdx.x + (sg.u0 == 0);
        const bool in = row < it.nr, sees = plo <= phi;
        const float unit = ls == 0.f ? 0.f : 1.f / ls;
        // 64 columns at a time through the warp's part of the queries' place, which is free now, so
        // that a row is stored in one piece
        unsigned char* const xs = Qs + warp * 8192;
        const int lane = tid & 31, c4 = lane & 15;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          uint32_t o[32];
          w_ld32(tmO + 32 * q, o);
          float f[32];
          bool nan = false;
#pragma unroll
          for (int x = 0; x < 32; ++x) {
            f[x] = ls == 0.f ? 0.f : __uint_as_float(o[x]) * unit;
            nan |= f[x] != f[x];
          }
          const bool mend = (odd || nan) && in && ls == ls;  // as in k_paged_rows
          if (__any_sync(0xffffffffu, mend)) {
            uint32_t seen = 0;  // columns with such a value: their sum takes the column's place
            const int last = min(k00 + sg.nu * kWKeys - 1, it.hi);
            const int kb = max(k00, plo), ke = min(last, phi);
            const char* const v0 = a.v + sg.g * a.c.head() + 64 * q;
            auto at = [&](int key) -> const char* {
              const int e = max(a.c.entry(it.b, key >> a.c.shift), 0);
              return v0 + (size_t)e * a.c.bytes + (size_t)(key & pmask) * (kWHd * 2);
            };
            // a lane a key looks for them (an exponent of ones and one more is a carry), each row takes
            // what it sees (a thread a row that walked 3000 keys by itself took 25 ms)
            for (int k1 = max(k00, it.lo); k1 <= last; k1 += 32) {
              uint32_t carry = 0;
              if (k1 + lane <= last) {
                const uint4* v = reinterpret_cast<const uint4*>(at(k1 + lane));
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  const uint4 u = v[x];
                  carry |= (u.x & 0x7f807f80u) + 0x00800080u;
                  carry |= (u.y & 0x7f807f80u) + 0x00800080u;
                  carry |= (u.z & 0x7f807f80u) + 0x00800080u;
                  carry |= (u.w & 0x7f807f80u) + 0x00800080u;
                }
              }
              uint32_t hits = __ballot_sync(0xffffffffu, (carry & 0x80008000u) != 0);
              for (; hits; hits &= hits - 1) {
                const int key = k1 + __ffs(hits) - 1;
                if (!mend || key < kb || key > ke) continue;
                const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(at(key));
#pragma unroll 1
                for (int x = 0; x < 32; ++x) {
                  const float y = __bfloat162float(v[x]);
                  if (!no_number(y)) continue;
#pragma unroll
                  for (int z = 0; z < 32; ++z)
                    if (z == x) f[z] = seen >> x & 1 ? f[z] + y : y;
                  seen |= 1u << x;
                }
              }
            }
          }
          if (whole && (!sees || ls == 0.f)) {
#pragma unroll
            for (int x = 0; x < 32; ++x) f[x] = sees ? __uint_as_float(0x7fffffffu) : 0.f;
          }
#pragma unroll
          for (int x = 0; x < 8; ++x)
            *reinterpret_cast<float4*>(xs + lane * 256 + ((((q & 1) * 8 + x) ^ (lane & 15)) << 4)) =
                make_float4(f[4 * x], f[4 * x + 1], f[4 * x + 2], f[4 * x + 3]);
          if (!(q & 1)) continue;
          __syncwarp();
          const int rows = min(32, it.nr - warp * 32), col = (q >> 1) * 64 + c4 * 4;
          auto from = [&](int y) -> float4 {
            return *reinterpret_cast<const float4*>(xs + y * 256 + ((c4 ^ (y & 15)) << 4));
          };
          if (whole) {
#pragma unroll 4
            for (int y = lane >> 4; y < rows; y += 2) {
              const float4 v = from(y);
              const int r = it.r0 + warp * 32 + y, m = a.byG(r), h = sg.g * a.G + r - m * a.G;
              const __nv_bfloat162 b0 = __floats2bfloat162_rn(v.x, v.y);
              const __nv_bfloat162 b1 = __floats2bfloat162_rn(v.z, v.w);
              *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) +
                                        ((int64_t)it.b * a.M + m) * a.out_stride + (int64_t)h * kWHd +
                                        col) =
                  make_uint2(*reinterpret_cast<const uint32_t*>(&b0),
                             *reinterpret_cast<const uint32_t*>(&b1));
            }
          } else {
            float* const to = a.part + ((size_t)slot * a.part_rows + warp * 32) * kWHd + col;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int y = (lane >> 4) + 2 * i;
              if (y < rows) *reinterpret_cast<float4*>(to + y * kWHd) = from(y);
            }
          }
          __syncwarp();
        }
        if (in && !whole) a.ml[(size_t)slot * a.part_rows + row] = make_float2(ref, ls);
      }
      if (row == 0 && !sg.whole() && sg.u0 == 0) a.desc[blockIdx.x] = kv8_desc(a, s_cur[0], sg);
      named_sync(1 + t, 128);  // the next segment's queries go where outputs were exchanged
      tc_fence_before();  // the next segment's products overwrite O, behind its p_full
    }
  }
  if (bad) s_fail = 1;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (__builtin_expect(s_fail, 0)) {  // products may still be at work in this block's memory
    if (tid == 0 && a.err) atomicOr(a.err, (int)kErrTimeout);
    if (warp >= L::kQk) {  // the warps that issue them, 2 TILES
      if (w_elect()) tc_commit(&bar.drained);
      w_sleep(&bar.drained, 0);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  }
  if (warp == L::kQk) tc_dealloc(tm, L::kCols);
}

}  // namespace ssd
