// kv8_wide.cuh -- attention over the 8-bit cache for many query rows a KV head
// (wide verifications, grouped queries, prompt chunks; bf16, head_dim 128), on
// the 5th-generation tensor cores.  Included by kv8_attention.cu.
//
// A tile (the plan's items) has one or two accumulators of 128 query rows each.  A block
// walks its keys a cache block (64) at a time; two blocks share an SM, of two
// accumulators one has it alone.  Its warps work side by side:
//  - four convert: they read the codes a step ahead into registers and write them to
//    shared memory as f16, exact, rows of 128 bytes with the 128-byte swizzle, two
//    steps deep: keys as a K-major operand, values, whose columns lie one behind
//    the other, as an MN-major one (two accumulators: four for keys and four for values,
//    which both then use);
//  - one an accumulator issues S = Q K^T (tcgen05.mma, 128 x 64 x 128, fp32 in tensor memory,
//    two buffers) for a step while the softmax of the step before is at work, another
//    one O += P V, P read from tensor memory, as soon as a softmax is done;
//  - four an accumulator do the softmax, a thread per row: the row's 64 scores into
//    registers, their maximum, p = 2^(s - ref + 7) as f16, which takes the place of S.  ref is
//    the row's maximum as of the last time it grew by more than 8 (in powers of two), so
//    O is rescaled in tensor memory only then, and p stays below 2^15.
// Queries are scaled to f16 and value scales moved into p as in k_kv8_rows.
//
// Bound, per 64 keys and accumulator: 640 cycles of tensor pipe (8 instructions of
// 48 cycles for S, whose operands come from shared memory, 4 of 64 for O) and as much of
// shared memory; 256 of code conversions (half with two accumulators), 256 of
// exponentials; 700 of a scheduler's issue slots with two softmax warps there.  What it
// takes is about 1050 (1200 with one accumulator), the rest waits of one role for another.
// 512 rows of 32 heads over 8 KV heads x 7936 keys: 76 us = 876 TFLOP/s, of which 6 are
// the start (the plan, the queries), 4 the last outputs and 6 the join; a floor of 34 at
// the library's bf16 rate.  17 rows of 64 heads over 8 x 16000
// keys: 31 us.
#pragma once

namespace ssd {

namespace {

constexpr int kWRows = 128;   // query rows of an accumulator
constexpr int kWKeys = kKv8Block;  // keys of a step: one scale
constexpr int kWHd = 128;
constexpr uint32_t kWQHalf = kWRows * 128;       // bytes of 64 f16 columns of the queries
constexpr uint32_t kWKHalf = kWKeys * 128;       // of a step's keys or values
constexpr uint32_t kWKTile = 2 * kWKHalf;
// A block's tile of TILES accumulators.
template <int TILES>
struct WideL {
  static constexpr int kRows = TILES * kWRows;
  // warps: 4 TILES softmax, 4 TILES conversion (two: keys, then values), then the
  // accumulators' scores and outputs
  static constexpr int kSoft = 4 * TILES, kQk = 2 * kSoft, kPv = kQk + TILES;
  static constexpr int kThreads = 320 * TILES;
  static constexpr int kBlocks = 3 - TILES;  // of an SM
  static constexpr uint32_t kSmem = 2 * TILES * kWQHalf + 4 * kWKTile + 1024;  // queries, keys and values; alignment
  static constexpr uint32_t kCols = 256 * TILES;  // tensor memory: S and P (2 x 64 each), O
};
constexpr float kWBase = 7.f, kWGrow = 8.f;
constexpr float kWFar = 1048576.f;  // 2^20: half a unit there is 2^-4

// Byte of 16-byte chunk ch (0..7, eight f16 each) of row r in 64 columns.
__device__ __forceinline__ uint32_t w_place(int r, int ch) {
  return (uint32_t)(r * 128 + ((ch ^ (r & 7)) << 4));
}

// Instruction descriptors: f16 operands, fp32 accumulator, M = 128, N = the keys of a
// step or the columns of the output; bit 16: B is MN-major.
constexpr uint32_t kWIdesc = (1u << 4) | ((uint32_t)(kWKeys >> 3) << 17) | ((128u >> 4) << 24);
constexpr uint32_t kWIdescV = (1u << 4) | (1u << 16) | ((128u >> 3) << 17) | ((128u >> 4) << 24);

// MN-major operand of 128-byte rows (64 columns) with the 128-byte swizzle: the
// leading offset leads to the next 64 columns, the stride offset to the next 8 rows.
__device__ __forceinline__ uint64_t w_desc_mn(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(kWKHalf >> 4) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// A whole warp comes here, and the lane with `one` issues: where a branch leaves one lane
// alone, the operands have to be brought into the warp's registers for each instruction,
// and it took up to 125 cycles to issue what the tensor cores need 48 for.
__device__ __forceinline__ void w_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc,
                                      uint32_t one) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc), "r"(one)
      : "memory");
}
// A from tensor memory.
__device__ __forceinline__ void w_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                         bool acc, uint32_t one) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc), "r"(one)
      : "memory");
}
// 1 in one lane of the warp.
__device__ __forceinline__ uint32_t w_elect() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r;
}

// Columns of the thread's lane, there on return.
__device__ __forceinline__ void w_ld16(uint32_t t, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
      "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15"
      "}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
        "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(t)
      : "memory");
}
__device__ __forceinline__ void w_ld32(uint32_t t, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
      "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31"
      "}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
        "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
        "=r"(r[30]), "=r"(r[31])
      : "r"(t)
      : "memory");
}
__device__ __forceinline__ void w_ld64(uint32_t t, uint32_t (&r)[64]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,"
      "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
      "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63"
      "}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
        "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
        "=r"(r[30]), "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]),
        "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]), "=r"(r[41]),
        "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
        "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]),
        "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]),
        "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
      : "r"(t)
      : "memory");
}
__device__ __forceinline__ void w_st16(uint32_t t, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(t),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void w_st32(uint32_t t, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(t),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void w_st_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// Writes of this thread to shared memory, for the tensor cores to read.
__device__ __forceinline__ void w_smem_fence() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// Codes that are read once, a step ahead of their use (volatile: the load stays
// where it is issued).
__device__ __forceinline__ uint4 w_load16(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}

// The larger of three.
__device__ __forceinline__ float w_max3(float x, float y, float z) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}
// Barriers of the two buffers: keys and values stored, scores there (and the keys'
// place free), probabilities there, output added (the values' and their place
// free); queries of the segment stored.
template <int TILES>
struct WideBars {
  uint64_t k_full[2], v_full[2], s_done[TILES][2], p_full[TILES][2], o_done[TILES][2], q_full[TILES];
  uint64_t drained;  // after a wait that gave up: the products still in flight are done
};

// Keys of step i of a segment.
__device__ __forceinline__ int w_key0(const Kv8Seg& s, int i) {
  return (s.it.unit0 + s.u0 + i) * kWKeys;
}

// Waits for a barrier's phase, asleep for up to a millisecond at a time (a
// poll without that hint comes back at once, and the polls of nine waiting warps take
// the issue slots of those at work); false after a few seconds.
__device__ __forceinline__ bool w_sleep(uint64_t* b, uint32_t parity) {
  for (int i = 0; i < 4096; ++i) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_u32(b)), "r"(parity), "r"(1000000u)
        : "memory");
    if (done) return true;
  }
  return false;
}
// The phase that step n completes on its buffer's barrier; after a wait that gave
// up, no thread of this role waits again: it runs through its steps, meets its
// barriers and reports.
__device__ __forceinline__ void w_wait(uint64_t (&b)[2], uint32_t n, bool& bad) {
  if (!bad) bad = !w_sleep(&b[n & 1], (n >> 1) & 1);
}

}  // namespace

template <int TILES>
__global__ void __launch_bounds__(WideL<TILES>::kThreads, WideL<TILES>::kBlocks)
    k_kv8_wide(const Kv8Attn a) {
  using L = WideL<TILES>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ Kv8PlanSmem s_plan;
  __shared__ WideBars<TILES> bar;
  __shared__ uint32_t s_tmem;
  __shared__ int s_nan, s_fail, s_more[TILES];
  __shared__ Kv8Cursor s_cur[TILES];  // of the softmax warps
  __shared__ Kv8Seg s_seg[TILES];
  __shared__ float s_qs[L::kRows];
  unsigned char* const smem =
      reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  unsigned char* const Qs = smem;
  unsigned char* const Ks = Qs + 2 * TILES * kWQHalf;   // [2 buffers]
  unsigned char* const Vs = Ks + 2 * kWKTile;
  const int tid = threadIdx.x, warp = tid >> 5;

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar.k_full[i], 128);
      mbar_init(&bar.v_full[i], 128);
      for (int t = 0; t < TILES; ++t) {
        mbar_init(&bar.p_full[t][i], 128);
        mbar_init(&bar.s_done[t][i], 1);
        mbar_init(&bar.o_done[t][i], 1);
      }
    }
    for (int t = 0; t < TILES; ++t) mbar_init(&bar.q_full[t], 128);
    mbar_init(&bar.drained, 2 * TILES);
    mbar_init_fence();
    s_nan = s_fail = 0;
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
  uint32_t n = 0;  // steps so far: the barriers' phases
  bool bad = false;

  // registers: 128 x 112 + 128 x 80 + 64 x 96 = 320 x 96, what the block was launched with;
  // two accumulators: 256 x 136 + 256 x 72 + 128 x 64 = 640 x 96
  if (TILES == 2 && warp >= L::kQk) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  if (warp >= L::kQk && warp < L::kPv) {
    // ------------------------------------------------------------ scores
    Kv8Seg sg;
    const uint32_t one = w_elect();
    const int t = warp - L::kQk;
    const uint32_t tmS = tm + t * kS;
    const uint64_t dq = sdesc_k128(smem_u32(Qs)) + (2 * t * kWQHalf >> 4);
    const uint64_t dk = sdesc_k128(smem_u32(Ks));
    for (uint32_t seg = 0; kv8_next<L::kRows, kWKeys>(a, cur, sg); ++seg) {
      if (!bad) bad = !w_sleep(&bar.q_full[t], seg & 1);
      for (int i = 0; i < sg.nu; ++i, ++n) {
        w_wait(bar.k_full, n, bad);
        if (n >= 2) w_wait(bar.o_done[t], n - 2, bad);  // P of that step was read there
        __syncwarp();
        tc_fence_after();
        const uint32_t buf = n & 1;
        if (t == 0 || sg.it.nr > t * kWRows)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            w_mma(tmS + buf * kWKeys, dq + (((k >> 2) * kWQHalf + (k & 3) * 32) >> 4),
                  dk + ((buf * kWKTile + (k >> 2) * kWKHalf + (k & 3) * 32) >> 4), kWIdesc, k > 0,
                  one);
        if (one) tc_commit(&bar.s_done[t][buf]);
      }
    }
  } else if (warp >= L::kPv && warp < L::kPv + TILES) {
    // ------------------------------------------------------------ outputs
    Kv8Seg sg;
    const uint32_t one = w_elect();
    const int t = warp - L::kPv;
    const uint32_t tmS = tm + t * kS, tmO = tm + kO + t * kWHd;
    const uint64_t dv = w_desc_mn(smem_u32(Vs));
    while (kv8_next<L::kRows, kWKeys>(a, cur, sg))
      for (int i = 0; i < sg.nu; ++i, ++n) {
        w_wait(bar.v_full, n, bad);
        w_wait(bar.p_full[t], n, bad);
        __syncwarp();
        tc_fence_after();
        const uint32_t buf = n & 1;
        if (t == 0 || sg.it.nr > t * kWRows)
#pragma unroll
          for (int k = 0; k < kWKeys / 16; ++k)  // 16 keys: 8 words of P, two 8-row groups of V
            w_mma_ts(tmO, tmS + buf * kWKeys + 8 * k, dv + ((buf * kWKTile + k * 2048) >> 4),
                     kWIdescV, i > 0 || k > 0, one);
        if (one) tc_commit(&bar.o_done[t][buf]);
      }
  } else if (warp >= L::kSoft && warp < L::kQk) {
    // ------------------------------------------------------------ codes to f16
    // (too few here spill: one accumulator 31 us with 72 for 26 over 16000 keys and 40 rows, two
    // 88 us with 64 for 77)
    if constexpr (TILES == 1) asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    const int ct = tid & 127;
    // the step that is loaded next: its first row in the cache, the keys (counted from
    // it) that some row sees, those that every row sees, steps left in the segment
    int64_t off = 0;
    int lo = 0, hi = 0, flo = 0, fhi = 0, left = 0;
    auto advance = [&]() -> bool {
      if (--left > 0) {
        off += kWKeys * kWHd;
        lo -= kWKeys, hi -= kWKeys, flo -= kWKeys, fhi -= kWKeys;
        return true;
      }
      Kv8Seg sg;
      if (!kv8_next<L::kRows, kWKeys>(a, cur, sg)) return false;
      const int k0 = w_key0(sg, 0);
      off = (((int64_t)sg.it.b * a.Hkv + sg.g) * a.max_seq + k0) * kWHd;
      lo = sg.it.lo - k0, hi = sg.it.hi - k0;
      flo = kv8_row_lo(sg.it, sg.it.hi, a.window) - k0;
      fhi = kv8_row_pos(a, sg.it, sg.it.r0) - k0;
      left = sg.nu;
      return true;
    };
    // rows ct / 8 + 16 j of a step, 16 codes each
    auto load = [&](const uint8_t* base, uint4 (&c)[4]) {
      const uint8_t* p = base + off + ct * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        c[j] = ct / 8 + 16 * j >= lo && ct / 8 + 16 * j <= hi ? w_load16(p + 16 * j * kWHd)
                                                              : make_uint4(0, 0, 0, 0);
    };
    // eight lanes hold a row, 128 bytes of each half; the upper four store their two
    // chunks the other way round, so that all eight meet different banks
    const bool up = ct & 4;
    const uint32_t row0 = (ct & 4 ? kWKHalf : 0) + (ct / 8) * 128;
    const uint32_t at0 = row0 + (((2 * (ct & 3) + up) ^ (ct / 8 & 7)) << 4);
    const uint32_t at1 = row0 + (((2 * (ct & 3) + !up) ^ (ct / 8 & 7)) << 4);
    auto store = [&](unsigned char* tile, const uint4 (&c)[4]) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w0 = up ? c[j].z : c[j].x, w1 = up ? c[j].w : c[j].y;
        const uint32_t w2 = up ? c[j].x : c[j].z, w3 = up ? c[j].y : c[j].w;
        *reinterpret_cast<uint4*>(tile + at0 + j * 2048) =
            make_uint4(e4m3_to_half2(w0), e4m3_to_half2(w0 >> 16), e4m3_to_half2(w1),
                       e4m3_to_half2(w1 >> 16));
        *reinterpret_cast<uint4*>(tile + at1 + j * 2048) =
            make_uint4(e4m3_to_half2(w2), e4m3_to_half2(w2 >> 16), e4m3_to_half2(w3),
                       e4m3_to_half2(w3 >> 16));
      }
      w_smem_fence();
    };
    // NaN codes of values to zero, in a step that not every row sees whole
    auto zero_nan = [&](uint4 (&c)[4]) {
      uint32_t any = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&c[j]);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t m = e4m3_nan_mask(w[x]);
          any |= m;
          w[x] &= ~((m >> 7) * 0xffu);
        }
      }
      // (published by the arrival that follows; it stays set for the block's later tiles, which
      // then look at the values of their own steps of this kind again, byte by byte)
      if (any) s_nan = 1;
    };
    bool more = advance();
    if constexpr (TILES == 1) {  // keys and values in turn, a step ahead
      uint4 kc[4], vc[4];
      if (more) {
        load(a.k, kc);
        load(a.v, vc);
      }
      for (; more; ++n) {
        const uint32_t buf = (n & 1) * kWKTile;
        if (n >= 2) w_wait(bar.s_done[0], n - 2, bad);
        store(Ks + buf, kc);
        mbar_arrive(&bar.k_full[n & 1]);
        if (0 < flo || kWKeys - 1 > fhi) zero_nan(vc);
        more = advance();
        if (more) load(a.k, kc);
        if (n >= 2) w_wait(bar.o_done[0], n - 2, bad);
        store(Vs + buf, vc);
        mbar_arrive(&bar.v_full[n & 1]);
        if (more) load(a.v, vc);
      }
    } else {  // four warps each
      const bool values = warp >= L::kSoft + 4;
      const uint8_t* const base = values ? a.v : a.k;
      unsigned char* const tile = values ? Vs : Ks;
      uint4 c[4];
      if (more) load(base, c);
      for (; more; ++n) {
        if (values && (0 < flo || kWKeys - 1 > fhi)) zero_nan(c);
        if (n >= 2)
#pragma unroll
          for (int t = 0; t < TILES; ++t) w_wait(values ? bar.o_done[t] : bar.s_done[t], n - 2, bad);
        store(tile + (n & 1) * kWKTile, c);
        mbar_arrive(values ? &bar.v_full[n & 1] : &bar.k_full[n & 1]);
        more = advance();
        if (more) load(base, c);
      }
    }
  } else if (warp < L::kSoft) {
    // ------------------------------------------------------------ softmax
    if constexpr (TILES == 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
    const int t = TILES == 1 ? 0 : warp >> 2, ttid = tid & 127;  // the accumulator, its thread
    const int row = tid;  // of the tile
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tmS = tm + t * kS + lanes, tmO = tm + kO + t * kWHd + lanes;
    for (;;) {
      // the segment stands in shared memory: the steps need the registers
      if (ttid == 0) s_more[t] = kv8_next<L::kRows, kWKeys>(a, s_cur[t], s_seg[t]);
      named_sync(1 + t, 128);
      if (!s_more[t]) break;
      const Kv8Seg& sg = s_seg[t];
      const Kv8Item& it = sg.it;
      // queries as f16, sixteen lanes a row (rows past the last: the last one's, not
      // used); the products of the segment before are done with theirs
      {
        const int ch = tid % 16;
        const __nv_bfloat16* const q0 = static_cast<const __nv_bfloat16*>(a.q) + ch * 8 +
                                        (int64_t)it.b * a.M * a.q_stride + (int64_t)sg.g * a.G * kWHd;
        unsigned char* const own = Qs + (2 * t + (ch >> 3)) * kWQHalf;
        uint4 u[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int r = it.r0 + min(t * kWRows + j * 8 + ttid / 16, it.nr - 1), m = a.byG(r);
          u[j] = w_load16(q0 + m * a.q_stride + (r - m * a.G) * kWHd);
        }
#pragma unroll
        for (int j0 = 0; j0 < 16; j0 += 4) {
          float amax[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162* w = reinterpret_cast<const __nv_bfloat162*>(&u[j0 + j]);
            const __nv_bfloat162 am = __hmax2(__hmax2(__habs2(w[0]), __habs2(w[1])),
                                              __hmax2(__habs2(w[2]), __habs2(w[3])));
            amax[j] = fmaxf(__low2float(am), __high2float(am));
          }
#pragma unroll
          for (int o = 8; o > 0; o >>= 1)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              amax[j] = fmaxf(amax[j], __shfl_xor_sync(0xffffffffu, amax[j], o));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int qr = (j0 + j) * 8 + ttid / 16;
            const int ex = min(max((int)(__float_as_uint(amax[j]) >> 23) - 127 - 13, -100), 115);
            const float inv = pow2i(-ex);
            float f[8];
            Elem<__nv_bfloat16>::unpack(u[j0 + j], f);
            *reinterpret_cast<uint4*>(own + w_place(qr, ch & 7)) =
                make_uint4(half2_bits(f[0] * inv, f[1] * inv), half2_bits(f[2] * inv, f[3] * inv),
                           half2_bits(f[4] * inv, f[5] * inv), half2_bits(f[6] * inv, f[7] * inv));
            if (ch == 0) s_qs[t * kWRows + qr] = pow2i(ex) * a.scale;
          }
        }
      }
      w_smem_fence();
      tc_fence_before();
      mbar_arrive(&bar.q_full[t]);
      named_sync(1 + t, 128);
      const float qs = s_qs[row];  // scores = products * qs * key scale
      const bool live = warp * 32 < it.nr;  // the warp has rows
      const size_t slab = (size_t)it.b * a.Hkv + sg.g;
      const int b0 = it.unit0 + sg.u0;
      const float* ksp = a.ks + slab * (a.max_seq / kKv8Block) + b0;
      const float* vsp = a.vs + slab * (a.max_seq / kKv8Block) + b0;
      const int full_lo = kv8_row_lo(it, it.hi, a.window);
      const int full_hi = kv8_row_pos(a, it, it.r0);
      const int phi = row < it.nr ? kv8_row_pos(a, it, it.r0 + row) : -1;
      const int plo = row < it.nr ? kv8_row_lo(it, phi, a.window) : 0;
      float ref = -INFINITY, ls = 0.f;   // of the row
      float vref = pow2i(-126);          // the output's unit, as in k_kv8_rows
      // Some row of the warp has a ref whose rounding is more than a small part of a power of two:
      // the product in the exponent is not rounded, so such a row's scores are, beforehand, and
      // taken from ref (in the branch below, which every step then takes: a branch of its own
      // costs the others 0.5 %).
      bool far = false;
      // (rows that see nothing have no block whose scale means something)
      const bool any = it.lo <= it.hi;
      float nks = any ? __ldg(ksp) : 0.f, nvs = any ? __ldg(vsp) : 0.f;
      for (int i = 0; i < sg.nu; ++i, ++n) {
        const float ks = nks, vs = nvs;
        if (i + 1 < sg.nu) {
          nks = __ldg(ksp + i + 1);
          nvs = __ldg(vsp + i + 1);
        }
        w_wait(bar.s_done[t], n, bad);
        __syncwarp();
        tc_fence_after();
        if (live) {
          const int k0 = w_key0(sg, i);
          const bool full = k0 >= full_lo && k0 + kWKeys - 1 <= full_hi;
          const uint32_t at = tmS + (n & 1) * kWKeys;
          // (never 0, as it is for small queries over a block of zero keys: the -inf of a key
          // out of sight stays -inf in a product with it)
          float c = fmaxf(kv8_factor(qs, ks), pow2i(-126));
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
          float mx = fmaxf(w_max3(m[0], m[1], m[2]), m[3]);
          if (mx > -INFINITY) mx *= c;
          // (rounded down: what stays is not above ref + 8, whatever ref's unit is)
          const bool grow = mx > __fadd_rd(ref, kWGrow) || (ref == -INFINITY && mx > ref);
          const bool up = vs > vref && mx > -INFINITY;
          float base = ref;  // what the exponents below are taken from
          if (__any_sync(0xffffffffu, grow || up || far)) {
            float f = 1.f;
            if (grow) {
              f = ref == -INFINITY ? 0.f : exp2f(ref - mx);
              ref = mx;
              ls *= f;
            }
            if (up) {
              f *= vref / vs;
              vref = vs;
            }
            if (i > 0) {
              w_wait(bar.o_done[t], n - 1, bad);
              __syncwarp();
              tc_fence_after();
#pragma unroll 1
              for (int q = 0; q < 8; ++q) {
                uint32_t o[16];
                w_ld16(tmO + 16 * q, o);
#pragma unroll
                for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
                w_st16(tmO + 16 * q, o);
              }
            }
            base = ref;
            const bool own = ref > -INFINITY && fabsf(ref) >= kWFar;
            far = __any_sync(0xffffffffu, own);
            if (far) {
              const float by = own ? c : 1.f, off = own ? ref : 0.f;
#pragma unroll
              for (int x = 0; x < 64; ++x)
                r[x] = __float_as_uint(__fsub_rn(__fmul_rn(__uint_as_float(r[x]), by), off));
              if (own) c = 1.f, base = 0.f;
            }
          }
          const float top = base == -INFINITY ? 0.f : base - kWBase;
          const float rel = fminf(vs / vref, 1.f);  // (above 1: a row that sees no key here)
          const uint64_t c2 = pack2(c, c), t2 = pack2(-top, -top);
          uint64_t sum2 = 0;
#pragma unroll
          for (int x = 0; x < 64; x += 2) {
            const float2 z =
                unpack2(fma2(pack2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), c2, t2));
            const float e0 = ex2_approx(z.x), e1 = ex2_approx(z.y);
            sum2 = add2(sum2, pack2(e0, e1));
            r[x / 2] = half2_bits(e0 * rel, e1 * rel);
          }
          const float2 sum = unpack2(sum2);
          ls += sum.x + sum.y;
          w_st32(at, r);
          w_st_wait();
        }
        tc_fence_before();
        mbar_arrive(&bar.p_full[t][n & 1]);
      }
      w_wait(bar.o_done[t], n - 1, bad);
      __syncwarp();
      tc_fence_after();
      // ---- the rows' outputs, or the block's part of them
      if (live) {
        const bool whole = sg.whole(), nan = *(volatile int*)&s_nan;
        const int slot = 2 * blockIdx.x + (sg.u0 == 0);
        const bool in = row < it.nr, sees = plo <= phi;
        const float unit = ls == 0.f ? 0.f : 1.f / ls;
        // 64 columns at a time through the warp's part of the queries' place, which
        // is free now, so that a row is stored in one piece
        unsigned char* const xs = Qs + warp * 8192;
        const int lane = tid & 31, c4 = lane & 15;
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          uint32_t o[32];
          w_ld32(tmO + 32 * q, o);
          float f[32];
#pragma unroll
          for (int x = 0; x < 32; ++x) f[x] = ls == 0.f ? 0.f : __uint_as_float(o[x]) * unit * vref;
          if (nan && in) {
            // a NaN value belongs to the rows that see its key (zeroed in steps that not
            // every row sees whole)
            const uint8_t* vp = a.v + slab * a.max_seq * kWHd + 32 * q;
            const int kb = max(w_key0(sg, 0), plo), ke = min(w_key0(sg, sg.nu) - 1, phi);
            for (int key = kb; key <= ke; ++key) {
              const int s0 = key & ~(kWKeys - 1);
              if (s0 >= full_lo && s0 + kWKeys - 1 <= full_hi) continue;
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if ((vp[(size_t)key * kWHd + x] & 0x7f) == 0x7f) f[x] = __uint_as_float(0x7fffffffu);
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
          const int rows = min(32, it.nr - warp * 32);
          for (int y = lane >> 4; y < rows; y += 2) {
            const float4 v = *reinterpret_cast<const float4*>(xs + y * 256 + ((c4 ^ (y & 15)) << 4));
            const int col = (q >> 1) * 64 + c4 * 4;
            if (whole) {
              const int r = it.r0 + warp * 32 + y, m = a.byG(r), h = sg.g * a.G + r - m * a.G;
              const __nv_bfloat162 b0 = __floats2bfloat162_rn(v.x, v.y);
              const __nv_bfloat162 b1 = __floats2bfloat162_rn(v.z, v.w);
              *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) +
                                        ((int64_t)it.b * a.M + m) * a.out_stride +
                                        (int64_t)h * kWHd + col) =
                  make_uint2(*reinterpret_cast<const uint32_t*>(&b0),
                             *reinterpret_cast<const uint32_t*>(&b1));
            } else {
              *reinterpret_cast<float4*>(
                  a.part + ((size_t)slot * a.part_rows + warp * 32 + y) * kWHd + col) = v;
            }
          }
          __syncwarp();
        }
        // (max, sum) as the merge weighs parts: p stands against 2^(ref - kWBase)
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
