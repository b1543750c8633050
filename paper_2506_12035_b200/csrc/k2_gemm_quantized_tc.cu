// K2 on weights held in 4 bits, large matrices: the products on the 5th-generation tensor cores, the weights converted straight into tensor memory.
//
// out^T = w a^T: 128 outputs are the rows of the A operand, which tcgen05.mma reads from tensor memory, 16 or 32 rows of a the columns of B (shared
// memory, as TMA brings them).  A thread owns an output: it takes the output's 64 codes of a chunk (32 bytes) from shared memory, makes fp16
// (bf16) numbers of them (exact, see k2_gemm_quantized.cu), and stores them to its tensor-memory lane.  Sums of a group (32, 64 or 128 inputs)
// accumulate in tensor memory in fp32; four other warps, a thread per output again, read them, multiply by the group's scale and add them up in
// fp32 registers, which are stored as whole lines at the end.
// Persistent CTAs, one per SM, or pairs (a cluster) that split K where that divides the units more evenly: the halves' sums meet by st.async in the
// CTA that owns the row (31 x 24576 x 12288, 192 units: 61 and 52 us).  Stages of 256 inputs; warps: 0-3 convert the even stages, 4-7 the odd ones, 8-11 add
// up, 12 fetches, 13 and 14 issue MMAs of even and odd stages.  All waits are bounded and report through the status word (all but the allocation of tensor
// memory, for which no cluster of another kernel can make a pair wait for good: kPairSmem).
// What bounds it: the conversion's instructions (per 64 inputs of 32 outputs 48 integer ones at two cycles each and 32 packed FMAs), 1200 cycles a stage
// where its bytes would take 700; half of the issue slots, 40 % of the integer pipe, and 72 stages on the busiest SM for 62 on average.
// 31 x 24576 x 12288, group 128: 52 us of 25 for the bytes (3.0 TB/s); group 64 59 us, group 32 79 us (sums twice and four times as often).
// On the way: stages of 128 inputs 104 us; residual rows loaded one after the other in the epilogue 80; one MMA warp, one lane's branch 55.
#include <cuda.h>

#include "kernels.h"
#include "launch_pdl.h"
#include "sm100_ptx.cuh"
#include "tma_host.h"

namespace marche {

namespace {

constexpr int kChunk = 64;                 // inputs
constexpr int kOut = 128;                  // outputs of a unit
constexpr int SC = 4;                      // chunks of a stage
constexpr int kThreads = 15 * 32;
constexpr int NST = 6;                     // stages (even: a stage and its slot are of one parity)
// A pair waits for its partner with all tensor memory allocated: the other kernel whose clusters do such a thing is kept off its SM (kernels.h), in the
// narrow forms by shared memory that is not used.
constexpr int kPairSmem = 212 * 1024;
enum { W_ACC = 8, W_PROD = 12, W_MMA = 13 };   // (and W_MMA + 1)
enum { ST_GEMM_QUANTIZED_TC = 0x67 };
enum { B_FULL = 0, B_EMPTY = B_FULL + NST, B_A_FULL = B_EMPTY + NST, B_A_EMPTY = B_A_FULL + 2, B_D_FULL = B_A_EMPTY + 2, B_D_EMPTY = B_D_FULL + 4, B_RECV = B_D_EMPTY + 4, NB = B_RECV + 2 };

template <int NR, int G> struct Cfg {
  static constexpr int GROUPS = SC * kChunk / G;           // of a stage
  static constexpr int DG = 2;                             // whose sums one of the four D buffers (two for the even stages, two for the odd) holds
  static constexpr int ROWS = SC * NR * 128, CODES = 8 * SC * 512, SCALES = 8 * GROUPS * 32;
  static constexpr int STAGE = (ROWS + CODES + SCALES + 1023) / 1024 * 1024, FILL = ROWS + CODES + SCALES;
  static constexpr int RECV = 2 * (NR / 2) * kOut * 4;     // two units' halves
  static constexpr int SMEM = 1024 + NST * STAGE + RECV;
  static constexpr int SMEM_PAIR = SMEM > kPairSmem ? SMEM : kPairSmem;
  static constexpr uint32_t COL_A = 0, COL_D = 2 * SC * 32, COLS = 512;   // A: two buffers of SC chunks, 32 columns each; D: four of DG groups of NR
};

MARCHE_DEVINL void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
MARCHE_DEVINL void tmem_ld_32x16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
MARCHE_DEVINL void tmem_st_32x16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
MARCHE_DEVINL void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Two pairs of an output's codes (each + 8) in a word: nibbles h and 4 + h, 2 + h and 6 + h (h 0 or 1: output g or g + 8 of a tile).
template <bool BF> struct Nibbles {
  uint32_t shift, mask, factor, offset;
  MARCHE_DEVINL explicit Nibbles(int h) : shift(BF ? 4 * h : 0), mask(BF || !h ? 0x000f000fu : 0x00f000f0u), factor(h ? 0x2c002c00u : 0x3c003c00u), offset(h ? 0xd480d480u : 0xe408e408u) {}
  MARCHE_DEVINL void numbers(uint32_t w, uint32_t& lo, uint32_t& hi) const {
    const uint32_t u = BF ? w >> shift : w;
    lo = pair(u);
    hi = pair(u >> 8);
  }
  // fp16: 1024 + c, or 1024 + 16 c for the odd nibble, times 1 or 1/16, minus 1032 or 72.  bf16, whose 7 bits hold no 16 c: 128 + c, shifted before.
  MARCHE_DEVINL uint32_t pair(uint32_t u) const {
    uint32_t x, r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(x) : "r"(u), "r"(mask), "r"(BF ? 0x43004300u : 0x64006400u));
    if (BF) asm("sub.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0x43084308u));
    else asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(factor), "r"(offset));
    return r;
  }
};

struct Shape { int M, N, chunks, n_rb, units, cs, epi, out_bf16; };

template <int NR, int G, bool BF>
__global__ void __launch_bounds__(kThreads, 1)
gemm_quantized_tc_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_codes, const __grid_constant__ CUtensorMap tmap_scales,
                         const float* __restrict__ bias, void* __restrict__ out, const Shape sh, int* __restrict__ status) {
  using C = Cfg<NR, G>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[NB];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flags[2];
  volatile int* abort_flag = abort_flags;
  const uint32_t raw = ptx::smem_u32(smem_raw), ring = (raw + 1023u) & ~1023u, bar0 = ptx::smem_u32(bars);
  const uint8_t* smem = smem_raw + (ring - raw);
  auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rank = sh.cs > 1 ? (int)ptx::cluster_ctarank() : 0, first = (int)blockIdx.x / sh.cs, step = (int)gridDim.x / sh.cs;
  const int stages = (sh.chunks + SC - 1) / SC, s0 = rank * stages / sh.cs, n_stages = (rank + 1) * stages / sh.cs - s0;   // of a unit, this CTA's
  const int all_stages = first < sh.units ? ((sh.units - 1 - first) / step + 1) * n_stages : 0;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NB; ++i)
      ptx::mbar_init(bar(i), i >= B_EMPTY && i < B_A_FULL ? 4 + 1 + 4 : (i >= B_A_FULL && i < B_A_EMPTY) || (i >= B_D_EMPTY && i < B_RECV) ? 4 : 1);
    abort_flags[0] = abort_flags[1] = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
    ptx::prefetch_tensormap(&tmap_codes);
    ptx::prefetch_tensormap(&tmap_scales);
    ptx::prefetch_tensormap(&tmap_a);
  }
  if (warp == W_MMA) {
    ptx::tmem_alloc(ptx::smem_u32(&tmem_slot), C::COLS);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (sh.cs > 1) ptx::cluster_sync_all();                  // the partner's barriers exist
  ptx::tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)&tmem_slot;
  bool ok = true;

  if (warp == W_PROD) {
    // ---------------------------------------------------------------- producer (what lies outside the matrices comes as zeros)
    if (ptx::elect_one()) {
      // codes and scales, which no kernel writes, and rows, apart so that the first ones' codes can go ahead of the dependency wait
      auto load_codes = [&](int slot, int tile0, int s) {
        const uint32_t dst = ring + (uint32_t)(slot * C::STAGE), b = bar(B_FULL + slot);
        ptx::mbar_expect_tx(b, C::FILL);
        ptx::tma_load_4d(dst + C::ROWS, &tmap_codes, 0, 0, s * SC, tile0, b);
        ptx::tma_load_3d(dst + C::ROWS + C::CODES, &tmap_scales, 0, s * C::GROUPS, tile0, b);
      };
      auto load_rows = [&](int slot, int row0, int s) { ptx::tma_load_3d(ring + (uint32_t)(slot * C::STAGE), &tmap_a, 0, row0, s * SC, bar(B_FULL + slot)); };
      const int ahead = first < sh.units ? min(NST, n_stages) : 0;
      {
        const int tile0 = first / sh.n_rb * 8, row0 = first % sh.n_rb * NR;
        for (int i = 0; i < ahead; ++i) load_codes(i, tile0, s0 + i);
        pdl_wait();
        for (int i = 0; i < ahead; ++i) load_rows(i, row0, s0 + i);
      }
      int slot = ahead == NST ? 0 : ahead, phase = ahead == NST ? 0 : 1, filled = ahead;
      for (int unit = first, from = ahead; unit < sh.units && ok; unit += step, from = 0) {
        const int tile0 = unit / sh.n_rb * 8, row0 = unit % sh.n_rb * NR;
        for (int s = from; s < n_stages; ++s) {
          if (!ptx::mbar_wait(bar(B_EMPTY + slot), (uint32_t)phase, abort_flag)) { ok = false; break; }
          load_codes(slot, tile0, s0 + s);
          load_rows(slot, row0, s0 + s);
          ++filled;
          if (++slot == NST) { slot = 0; phase ^= 1; }
        }
      }
      if (!ok) {                                           // let copies already issued land before the CTA's shared memory is released
        *(volatile int*)status = ST_GEMM_QUANTIZED_TC;
        for (int k = filled > NST ? filled - NST : 0; k < filled; ++k)
          ptx::mbar_wait(bar(B_FULL + k % NST), (uint32_t)(k / NST) & 1u, abort_flag + 1, 20000000LL);
      }
    }
    __syncwarp();
  } else {
    pdl_sync();
    if (warp >= W_MMA) {
      // ---------------------------------------------------------------- MMA issuers: one warp for the even stages, one for the odd.  The whole warp
      // runs the loop and one lane issues, so that descriptors can stay in uniform registers (in a branch of one lane an MMA took 70 cycles to issue,
      // four times what it takes to run; so, with one warp, 50)
      constexpr uint32_t idesc = ptx::idesc_16_f32(kOut, NR, BF);
      const bool issuer = ptx::elect_one();
      const int set = warp - W_MMA;
      const uint32_t a0 = tmem + C::COL_A + (uint32_t)(set * SC * 32), d0 = tmem + C::COL_D + (uint32_t)(set * 2 * C::DG * NR);
      int slot = set, full_phase = 0, a_phase = 0, d = 0, d_phase = 1;   // d_phase: an empty buffer's first wait passes at once
      for (int i = set; i < all_stages; i += 2) {
        ok = ptx::mbar_wait(bar(B_FULL + slot), (uint32_t)full_phase, abort_flag) && ptx::mbar_wait(bar(B_A_FULL + set), (uint32_t)a_phase, abort_flag);
        const uint64_t dx = ptx::smem_desc_k_sw128(ring + (uint32_t)(slot * C::STAGE));
#pragma unroll
        for (int part = 0; part < C::GROUPS / C::DG; ++part) {
          ok = __all_sync(0xffffffffu, ok && ptx::mbar_wait(bar(B_D_EMPTY + 2 * set + d), (uint32_t)d_phase, abort_flag));
          if (!ok) break;
          ptx::tc_fence_after();
          const uint32_t dd = d0 + (uint32_t)(d * C::DG * NR);
#pragma unroll
          for (int j = 0; j < C::DG * G; j += 16) {
            const int k = part * C::DG * G + j;
            if (issuer) umma_f16_ts(dd + (uint32_t)(j / G * NR), a0 + k / 2, dx + (uint32_t)(k / kChunk * (NR * 8) + k % kChunk / 8), idesc, j % G ? 1u : 0u);
          }
          if (issuer) ptx::umma_commit(bar(B_D_FULL + 2 * set + d));
          d ^= 1;
          d_phase ^= d ^ 1;
        }
        if (!ok) break;
        if (issuer) {
          ptx::umma_commit(bar(B_A_EMPTY + set));
          ptx::umma_commit(bar(B_EMPTY + slot));
        }
        __syncwarp();
        a_phase ^= 1;
        if ((slot += 2) >= NST) { slot = set; full_phase ^= 1; }
      }
      if (!ok && lane == 0) *(volatile int*)status = ST_GEMM_QUANTIZED_TC;
    } else if (warp < W_ACC) {
      // ---------------------------------------------------------------- converters: four warps take the even stages, four the odd ones, so that one
      // four's stores and waits lie under the other's arithmetic (both on every stage: 55 us for 31 x 24576 x 12288); lane = output
      const int set = warp >> 2, r = (warp & 3) * 32 + lane, g = r & 7, h = (r >> 3) & 1;
      const uint32_t codes_at = (uint32_t)(C::ROWS + (r >> 4) * (SC * 512) + g * 64), a_at = tmem + C::COL_A + ((uint32_t)((warp & 3) * 32) << 16) + 32u * SC * set;
      const Nibbles<BF> nibbles(h);
      int slot = set, full_phase = 0, a_phase = 1;
      for (int i = set; i < all_stages; i += 2) {
        if (!__all_sync(0xffffffffu, ptx::mbar_wait(bar(B_FULL + slot), (uint32_t)full_phase, abort_flag))) { ok = false; break; }
        const uint8_t* from = smem + slot * C::STAGE + codes_at;
#pragma unroll 1
        for (int j = 0; j < SC; j += 2) {                  // (unrolled, the roles' code does not fit the instruction caches, 52 -> 55 us; by one chunk 57)
          uint32_t a[2][32];                               // column k / 2: word q of lane t holds inputs 32 (q / 2) + 8 t + 4 (q % 2) .. + 3
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint4 v[4];                                    // (64-byte rows under TMA's 64-byte swizzle)
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] = *reinterpret_cast<const uint4*>(from + (j + c) * 512 + ((t ^ (g >> 1)) << 4));
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const uint32_t w[4] = {v[t].x, v[t].y, v[t].z, v[t].w};
#pragma unroll
              for (int q = 0; q < 4; ++q) nibbles.numbers(w[q], a[c][16 * (q >> 1) + 4 * t + 2 * (q & 1)], a[c][16 * (q >> 1) + 4 * t + 2 * (q & 1) + 1]);
            }
          }
          if (j == 0) {
            if (!__all_sync(0xffffffffu, ptx::mbar_wait(bar(B_A_EMPTY + set), (uint32_t)a_phase, abort_flag))) { ok = false; break; }
            ptx::tc_fence_after();
          } else {
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(B_EMPTY + slot));
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            tmem_st_32x16(a_at + 32u * (uint32_t)(j + c), a[c]);
            tmem_st_32x16(a_at + 32u * (uint32_t)(j + c) + 16u, a[c] + 16);
          }
        }
        if (!ok) break;
        tmem_st_wait();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B_A_FULL + set));
        a_phase ^= 1;
        if ((slot += 2) >= NST) { slot = set; full_phase ^= 1; }
      }
      if (!ok && lane == 0) *(volatile int*)status = ST_GEMM_QUANTIZED_TC;
    } else {
      // ---------------------------------------------------------------- sums: lane = output
      const int quarter = warp & 3, r = quarter * 32 + lane;
      const uint32_t d_at = tmem + C::COL_D + ((uint32_t)(quarter * 32) << 16);
      const uint32_t scale_at = (uint32_t)(C::ROWS + C::CODES + (r >> 4) * (C::GROUPS * 32) + (2 * (r & 7) + ((r >> 3) & 1)) * 2);
      float* recv = reinterpret_cast<float*>(smem_raw + (ring - raw) + NST * C::STAGE);
      int slot = 0, full_phase = 0, d = 0, d_phase = 0, parity = 0, turn = 0;   // d, d_phase: a bit for each parity of the stages
      for (int unit = first; unit < sh.units && ok; unit += step, ++turn) {
        float acc[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) acc[i] = 0.f;
        if (sh.cs > 1 && threadIdx.x == W_ACC * 32) ptx::mbar_expect_tx(bar(B_RECV + (turn & 1)), (NR / 2) * kOut * 4);
        for (int s = 0; s < n_stages && ok; ++s) {
          if (!__all_sync(0xffffffffu, ptx::mbar_wait(bar(B_FULL + slot), (uint32_t)full_phase, abort_flag))) { ok = false; break; }
#pragma unroll 1
          for (int part = 0; part < C::GROUPS / C::DG; ++part) {
            float scale[C::DG];
#pragma unroll
            for (int i = 0; i < C::DG; ++i)
              scale[i] = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(smem + slot * C::STAGE + scale_at + (part * C::DG + i) * 32) << 16);
            if (part == C::GROUPS / C::DG - 1) {
              __syncwarp();
              if (lane == 0) ptx::mbar_arrive(bar(B_EMPTY + slot));
            }
            const int e = 2 * parity + (d >> parity & 1);
            if (!__all_sync(0xffffffffu, ptx::mbar_wait(bar(B_D_FULL + e), (uint32_t)(d_phase >> parity) & 1u, abort_flag))) { ok = false; break; }
            ptx::tc_fence_after();
            uint32_t x[C::DG][NR];
#pragma unroll
            for (int i = 0; i < C::DG; ++i)
#pragma unroll
              for (int q = 0; q < NR; q += 16) tmem_ld_32x16(d_at + (uint32_t)((e * C::DG + i) * NR + q), x[i] + q);
#pragma unroll
            for (int i = 0; i < C::DG; ++i) ptx::tmem_ld_wait(x[i]);
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(B_D_EMPTY + e));
#pragma unroll
            for (int i = 0; i < C::DG; ++i)
#pragma unroll
              for (int q = 0; q < NR; ++q) acc[q] = fmaf(__uint_as_float(x[i][q]), scale[i], acc[q]);
            d ^= 1 << parity;
            d_phase ^= ~d & (1 << parity);
          }
          parity ^= 1;
          if (++slot == NST) { slot = 0; full_phase ^= 1; }
        }
        if (!ok) break;
        const int n = unit / sh.n_rb * kOut + r, row0 = unit % sh.n_rb * NR;
        int from = 0, to = NR;                             // the rows that this CTA finishes
        if (sh.cs > 1) {
          // the other half's sums go to the partner, [row pair][output][2]; two buffers: who sends for the unit after next has received what the partner
          // sent after it had read the buffer
          const int own = rank * (NR / 2), other = NR / 2 - own;
          const uint32_t dst = ptx::mapa(ptx::smem_u32(recv) + (uint32_t)((turn & 1) * (NR / 2) * kOut * 4), (uint32_t)(rank ^ 1)), b = ptx::mapa(bar(B_RECV + (turn & 1)), (uint32_t)(rank ^ 1));
#pragma unroll
          for (int i = 0; i < NR / 4; ++i) {
            const float lo = other ? acc[NR / 2 + 2 * i] : acc[2 * i], hi = other ? acc[NR / 2 + 2 * i + 1] : acc[2 * i + 1];
            ptx::st_async_v2(dst + (uint32_t)((i * kOut + r) * 8), lo, hi, b);
          }
          if (!__all_sync(0xffffffffu, ptx::mbar_wait_cluster(bar(B_RECV + (turn & 1)), (uint32_t)(turn >> 1) & 1u, abort_flag))) { ok = false; break; }
          const float2* in = reinterpret_cast<const float2*>(recv + (turn & 1) * (NR / 2) * kOut);
#pragma unroll
          for (int i = 0; i < NR / 4; ++i) {
            const float2 v = in[i * kOut + r];
            // (rank order: the first half of K first)
            if (rank == 0) { acc[2 * i] += v.x; acc[2 * i + 1] += v.y; }
            else { acc[NR / 2 + 2 * i] = v.x + acc[NR / 2 + 2 * i]; acc[NR / 2 + 2 * i + 1] = v.y + acc[NR / 2 + 2 * i + 1]; }
          }
          from = own;
          to = own + NR / 2;
        }
        if (n < sh.N) {
          const float bn = __ldg(bias + n);
          const int rows = min(to, sh.M - row0);
          const size_t at = (size_t)row0 * sh.N + n;
          if (sh.epi == 1) {                               // (all loads ahead of the stores: one after the other took 16 kcycles a unit)
            float* o = reinterpret_cast<float*>(out) + at;
#pragma unroll
            for (int q = 0; q < NR; q += 16) {
              float res[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) res[i] = q + i >= from && q + i < rows ? o[(size_t)(q + i) * sh.N] : 0.f;
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (q + i >= from && q + i < rows) o[(size_t)(q + i) * sh.N] = res[i] + (acc[q + i] + bn);
            }
          } else {
            uint16_t* o = reinterpret_cast<uint16_t*>(out) + at;
#pragma unroll
            for (int i = 0; i < NR; ++i)
              if (i >= from && i < rows) {
                const float y = acc[i] + bn;
                o[(size_t)i * sh.N] = (uint16_t)(pack_a16x2(sh.epi == 2 ? gelu_erf(y) : y, 0.f, sh.out_bf16 != 0) & 0xffffu);
              }
          }
        }
      }
      if (!ok && lane == 0) *(volatile int*)status = ST_GEMM_QUANTIZED_TC;
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == W_MMA) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, C::COLS);
  }
  if (sh.cs > 1) {
    __syncwarp();
    ptx::cluster_sync_all();                               // nobody leaves while a partner may still send to it
  }
}

template <int NR, int G, bool BF>
cudaError_t launch(const void* a, int lda, int M, const void* codes, const void* scales, const float* bias, int N, int K, int epi, void* out, int out_bf16, int cs,
                   int* status, cudaStream_t st) {
  using C = Cfg<NR, G>;
  static_assert(C::SMEM_PAIR <= 226 * 1024 && keeps_clusters_out(C::SMEM_PAIR), "shared memory of one CTA");
  const size_t smem = cs > 1 ? C::SMEM_PAIR : C::SMEM;
  CUtensorMap ta, tc, ts;
  EncodeTiledFn fn = tma_encode_fn();
  if (!fn) return cudaErrorInvalidValue;
  const cuuint64_t chunks = K / kChunk, groups = K / G, tiles = N / 16;
  const cuuint32_t unit[4] = {1, 1, 1, 1};
  const cuuint64_t da[3] = {kChunk, (cuuint64_t)M, chunks}, sa[2] = {(cuuint64_t)lda * 2, kChunk * 2};
  const cuuint32_t ba[3] = {kChunk, NR, SC};
  const cuuint64_t dc[4] = {16, 8, chunks, tiles}, sc[3] = {64, 512, chunks * 512};
  const cuuint32_t bc[4] = {16, 8, SC, 8};
  const cuuint64_t ds[3] = {8, groups, tiles}, ss[2] = {32, groups * 32};
  const cuuint32_t bs[3] = {8, C::GROUPS, 8};
  auto make = [&](CUtensorMap* map, CUtensorMapDataType type, int rank, const void* p, const cuuint64_t* d, const cuuint64_t* s, const cuuint32_t* b, CUtensorMapSwizzle sw) {
    return fn(map, type, (cuuint32_t)rank, const_cast<void*>(p), d, s, b, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (!make(&ta, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, a, da, sa, ba, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !make(&tc, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, codes, dc, sc, bc, CU_TENSOR_MAP_SWIZZLE_64B) ||
      !make(&ts, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, scales, ds, ss, bs, CU_TENSOR_MAP_SWIZZLE_NONE))
    return cudaErrorInvalidValue;
  static size_t smem_set[kMaxDevices] = {};
  cudaError_t e = ensure_dynamic_smem(gemm_quantized_tc_kernel<NR, G, BF>, smem, smem_set);
  if (e != cudaSuccess) return e;
  Shape sh = {M, N, (int)chunks, (M + NR - 1) / NR, 0, cs, epi, out_bf16};
  sh.units = (N + kOut - 1) / kOut * sh.n_rb;
  const int most = device_sm_count() / cs, clusters = sh.units < most ? sh.units : most;
  return launch_pdl_cluster(gemm_quantized_tc_kernel<NR, G, BF>, dim3((unsigned)(clusters * cs)), dim3(kThreads), smem, cs, st, ta, tc, ts, bias, out, sh, status);
}

template <int NR, bool BF>
cudaError_t by_group(const void* a, int lda, int M, const void* codes, const void* scales, const float* bias, int N, int K, int group, int epi, void* out, int ob, int cs,
                     int* status, cudaStream_t st) {
  return group == 32   ? launch<NR, 32, BF>(a, lda, M, codes, scales, bias, N, K, epi, out, ob, cs, status, st)
         : group == 64 ? launch<NR, 64, BF>(a, lda, M, codes, scales, bias, N, K, epi, out, ob, cs, status, st)
                       : launch<NR, 128, BF>(a, lda, M, codes, scales, bias, N, K, epi, out, ob, cs, status, st);
}

}  // namespace

size_t gemm_quantized_tc_smem(int M, int group, int cs) {
  auto of = [&](auto c) { return (size_t)(cs > 1 ? decltype(c)::SMEM_PAIR : decltype(c)::SMEM); };
  if (M <= 16) return group == 32 ? of(Cfg<16, 32>()) : group == 64 ? of(Cfg<16, 64>()) : of(Cfg<16, 128>());
  return group == 32 ? of(Cfg<32, 32>()) : group == 64 ? of(Cfg<32, 64>()) : of(Cfg<32, 128>());
}

cudaError_t launch_gemm_quantized_tc(const void* a, int lda, int M, const void* codes, const void* scales, const float* bias, int N, int K, int group, int epilogue,
                                     void* out, bool a_bf16, int cs, int* status, cudaStream_t st) {
  const int ob = epilogue == 0 || a_bf16;                  // (the bias epilogue's output is bf16 in every 16-bit context)
  if (M <= 16)
    return a_bf16 ? by_group<16, true>(a, lda, M, codes, scales, bias, N, K, group, epilogue, out, ob, cs, status, st)
                  : by_group<16, false>(a, lda, M, codes, scales, bias, N, K, group, epilogue, out, ob, cs, status, st);
  return a_bf16 ? by_group<32, true>(a, lda, M, codes, scales, bias, N, K, group, epilogue, out, ob, cs, status, st)
                : by_group<32, false>(a, lda, M, codes, scales, bias, N, K, group, epilogue, out, ob, cs, status, st);
}

}  // namespace marche
