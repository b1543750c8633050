// K2 on weights held in 4 bits: out = epilogue(a * w^T + bias) for a few rows, w[n][k] = code * scale[n][k / group], code -8 .. 7.
//
// What bounds it: HBM for large matrices (N K / 2 bytes), the launch for small ones.  The products are mma.sync m16n8k16 with the
// WEIGHTS as the 16-row operand and up to eight rows of a as the 8-column one, so that a single row wastes seven eighths of a tensor
// operation that costs next to nothing and no bandwidth.  The matrix is laid out once (marche_quantize_weights) in the order in
// which lanes multiply: [N / 16][K / 64][lane][16 bytes], a warp's load is 512 contiguous bytes, 16 outputs by 64 inputs, and each of a lane's
// four words is one operand: output lane / 4 (and + 8), inputs of k16 step s.  A dot product does not mind the order in which
// k is taken: step s of lane t = lane % 4 holds inputs 32 (s / 2) + 8 t + 4 (s % 2) .. + 3, so that eight consecutive values of a row
// of a serve two steps by one 16-byte load.  (A step stays within 32 inputs, the smallest group.)
// Codes become numbers without conversion instructions: a nibble c under the exponent of 1024 (fp16; 128 for bf16) is 1024 + c, or
// 1024 + 16 c for the nibble above it; one packed subtraction or FMA takes 1032 (or 64 + 8 after the division by 16) off, exactly.
// Products of a group add up in fp32 in the tensor core, are scaled once per group and output in fp32 and added in fp32; the warps of a
// CTA take the inputs in turn and their sums meet in shared memory in a fixed order (bit-reproducible).  No other rounding before the last.
// Three kernels: this file's two, for small matrices and for up to eight rows of large ones, and k2_gemm_quantized_tc.cu for more rows.  With
// 9 to 32 rows of a large matrix the work of a warp here (90 to 110 instructions for 16 outputs x 64 inputs x 32 rows: operands, conversion, sums of a
// group, barriers) exceeded the bytes' time four times: 31 x 24576 x 12288 97 us.
#include "common.cuh"
#include "kernels.h"
#include "launch_pdl.h"
#include "sm100_ptx.cuh"
#include "tma_host.h"

namespace marche {

namespace {

constexpr int kChunk = 64;                 // inputs of a warp's load
constexpr int kMaxRows = 32;               // of a CTA

template <bool BF>
MARCHE_DEVINL void mma_weights(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The same into a fresh accumulator.
template <bool BF>
MARCHE_DEVINL void mma_weights_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// (w & mask) | magic in one instruction
template <uint32_t MASK, uint32_t MAGIC>
MARCHE_DEVINL uint32_t and_or(uint32_t w) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "n"(MASK), "n"(MAGIC));
  return r;
}

// The eight codes of a word (each + 8 in its nibble) as four packed pairs of numbers.
template <bool BF>
MARCHE_DEVINL void numbers_of(uint32_t w, uint32_t (&a)[4]) {
  if (BF) {
    const uint32_t off = 0x43084308u;                      // 136 = 128 + 8
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = and_or<0x000f000fu, 0x43004300u>(w >> (4 * i));
      asm("sub.bf16x2 %0, %1, %2;" : "=r"(a[i]) : "r"(x), "r"(off));
    }
  } else {
    const uint32_t off = 0x64086408u, sixteenth = 0x2c002c00u, off_hi = 0xd480d480u;   // 1032, 1 / 16, -72
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const uint32_t v = w >> (4 * i);
      const uint32_t lo = and_or<0x000f000fu, 0x64006400u>(v), hi = and_or<0x00f000f0u, 0x64006400u>(v);
      asm("sub.f16x2 %0, %1, %2;" : "=r"(a[i]) : "r"(lo), "r"(off));
      asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(a[i + 1]) : "r"(hi), "r"(sixteenth), "r"(off_hi));
    }
  }
}

MARCHE_DEVINL uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// Two neighbouring outputs n, n + 1 of a row: bias, epilogue, store.
MARCHE_DEVINL void finish(float2 y, const float* __restrict__ bias, int row, int n, int N, int epi, void* __restrict__ out, int out_bf16) {
  const float2 b = __ldg(reinterpret_cast<const float2*>(bias + n));
  const size_t at = (size_t)row * N + n;
  y.x += b.x;
  y.y += b.y;
  if (epi == 1) {
    float2* o = reinterpret_cast<float2*>((float*)out + at);
    const float2 r = *o;
    *o = make_float2(r.x + y.x, r.y + y.y);
  } else {
    if (epi == 2) { y.x = gelu_erf(y.x); y.y = gelu_erf(y.y); }
    reinterpret_cast<uint32_t*>(out)[at >> 1] = pack_a16x2(y.x, y.y, out_bf16 != 0);
  }
}

// A chunk of a tile (a lane's 16 bytes of codes; G / 32 groups, or part of one) times 8 MT rows (a lane's 16 values of each eight), scaled and added up.
// both(k): scales of the chunk's k-th group for outputs g and g + 8.
template <int MT, bool BF, int G, typename Both>
MARCHE_DEVINL void multiply_chunk(float (&acc)[MT][4], const uint4& w, const uint4 (&x)[MT][2], Both both) {
  const uint32_t words[4] = {w.x, w.y, w.z, w.w};
  float part[MT][4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    uint32_t f[4];
    numbers_of<BF>(words[s], f);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const uint4& v = x[m][s >> 1];
      if (s == 0 || (G == 32 && s == 2)) mma_weights_first<BF>(part[m], f, s & 1 ? v.z : v.x, s & 1 ? v.w : v.y);
      else mma_weights<BF>(part[m], f, s & 1 ? v.z : v.x, s & 1 ? v.w : v.y);
    }
    if (s == 3 || (G == 32 && s == 1)) {
      const uint32_t sc = both(s >> 1);
      const float s0 = __uint_as_float(sc << 16), s1 = __uint_as_float(sc & 0xffff0000u);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        acc[m][0] = fmaf(part[m][0], s0, acc[m][0]);
        acc[m][1] = fmaf(part[m][1], s0, acc[m][1]);
        acc[m][2] = fmaf(part[m][2], s1, acc[m][2]);
        acc[m][3] = fmaf(part[m][3], s1, acc[m][3]);
      }
    }
  }
}

// Small matrices: a CTA per tile of 16 outputs and 8 MT rows, whose warps take the chunks of K in turn, straight from global memory to registers
// PF chunks ahead; the first of them before the dependency wait.
template <int MT, bool BF, int G>
__global__ void __launch_bounds__(512)
gemm_quantized_small_kernel(const uint16_t* __restrict__ a, int lda, int M, const uint4* __restrict__ codes, const uint32_t* __restrict__ scales,
                            const float* __restrict__ bias, int N, int K, int epi, void* __restrict__ out, int out_bf16) {
  constexpr int PF = 4, SC = G == 32 ? 2 : 1;
  extern __shared__ float sums[];                          // [warp][8 MT rows][16]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, g = lane >> 2, t = lane & 3;
  const int chunks = K / kChunk, row0 = blockIdx.y * (8 * MT);
  const uint4* src = codes + (size_t)blockIdx.x * chunks * 32 + lane;
  const uint32_t* sc = scales + (size_t)blockIdx.x * (K / G) * 8 + g;
  uint4 w[PF];
  uint32_t ws[PF][SC];
  auto fetch = [&](int p, int c) {
    w[p] = ld_stream(src + (size_t)c * 32);
#pragma unroll
    for (int k = 0; k < SC; ++k) ws[p][k] = __ldg(sc + (size_t)(G == 32 ? 2 * c + k : c * kChunk / G) * 8);
  };
#pragma unroll
  for (int p = 0; p < PF; ++p)
    if (warp + p * warps < chunks) fetch(p, warp + p * warps);
  pdl_sync();                                              // the weights are on their way while the previous kernel drains

  float acc[MT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m][0] = acc[m][1] = acc[m][2] = acc[m][3] = 0.f;
  const uint4* row[MT];                                    // (rows behind the last are the last one again: what they give is not stored)
#pragma unroll
  for (int m = 0; m < MT; ++m) row[m] = reinterpret_cast<const uint4*>(a + (size_t)min(row0 + 8 * m + g, M - 1) * lda + 8 * t);
  for (int c0 = warp; c0 < chunks; c0 += PF * warps) {
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      const int c = c0 + p * warps;
      if (c < chunks) {
        uint4 x[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          x[m][0] = row[m][c * 8];
          x[m][1] = row[m][c * 8 + 4];
        }
        multiply_chunk<MT, BF, G>(acc, w[p], x, [&](int k) { return ws[p][G == 32 ? k : 0]; });
        if (c + PF * warps < chunks) fetch(p, c + PF * warps);
      }
    }
  }
  // accumulator: outputs g and g + 8, rows 2 t and 2 t + 1 of an eight
  float* mine = sums + warp * (8 * MT * 16);
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) mine[(8 * m + 2 * t + (e & 1)) * 16 + g + 8 * (e >> 1)] = acc[m][e];
  __syncthreads();
  const int all = min(8 * MT, M - row0) * 8;               // two neighbouring outputs of a row each
  for (int q = threadIdx.x; q < all; q += blockDim.x) {
    float2 y = make_float2(0.f, 0.f);
    for (int k = 0; k < warps; ++k) {                      // over the warps, in their order
      const float2 v = *reinterpret_cast<const float2*>(sums + k * (8 * MT * 16) + 2 * q);
      y.x += v.x;
      y.y += v.y;
    }
    finish(y, bias, row0 + (q >> 3), blockIdx.x * 16 + 2 * (q & 7), N, epi, out, out_bf16);
  }
}

constexpr int kMaxStages = 16;
enum { ST_GEMM_QUANTIZED = 0x66 };

// Of a stage: WK CW chunks of the eight rows (a chunk's 128 bytes under TMA's 128-byte swizzle), of the unit's tiles, and their scales.
constexpr int WK = 4, CW = 2, kStageChunks = WK * CW, kMaxTiles = 7;
template <int G> struct Stage {
  static constexpr int GROUPS = kStageChunks * kChunk / G, ROWS = kStageChunks * 1024, CODES = kStageChunks * 512, SCALES = GROUPS * 32;
};
inline size_t stage_bytes_of(int group, int tiles) {
  return ((size_t)kStageChunks * 1024 + (size_t)tiles * (kStageChunks * 512 + kStageChunks * kChunk / group * 32) + 1023) / 1024 * 1024;
}

// Large matrices, up to eight rows: persistent CTAs, one per SM.  A unit is wn tiles of 16 outputs, units are dealt in turn; warp (iw, ik) has one
// of the tiles and the ik-th CW chunks of every stage.  Codes, scales and rows of a stage come by one TMA box each (bulk copies of a tile's or a
// row's part alone take 40 ns apiece: 31 x 24576 x 12288 211 us for the copies) into a ring that all warps share and that a warp of its own fills, over
// the borders of units, too: the matrix flows in without a pause.  (A consumer that fills slots on the way, with divisions for the slot and its
// phase, took 860 cycles for every stage, whatever it loaded.)  1 x 16384 x 8192: two warps along K 22.7 us, four 20.9, of 11.0 for the bytes; the
// launch and the first stage's way take 4.
template <bool BF, int G>
__global__ void __launch_bounds__(32 * (WK * kMaxTiles + 1))
gemm_quantized_stream_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_codes,
                             const __grid_constant__ CUtensorMap tmap_scales, int M, const float* __restrict__ bias, int N, int K, int epi,
                             void* __restrict__ out, int out_bf16, int wn, int nst, uint32_t stage_bytes, int* __restrict__ status) {
  using St = Stage<G>;
  extern __shared__ uint8_t smem_raw[];                    // stages (1 KB aligned): [chunk][rows] | [tile][chunk] codes | [tile][group] scales; sums [WK][8 rows][cols]
  __shared__ __align__(8) uint64_t bars[2 * kMaxStages];   // full, empty
  __shared__ int abort_flags[2];
  volatile int* abort_flag = abort_flags;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, iw = warp / WK, ik = warp % WK, g = lane >> 2, t = lane & 3;
  const int chunks = K / kChunk, cols = 16 * wn, units = (N / 16 + wn - 1) / wn, per_unit = (chunks + kStageChunks - 1) / kStageChunks;
  const uint32_t scales_at = (uint32_t)(St::ROWS + wn * St::CODES), filling = scales_at + (uint32_t)(wn * St::SCALES);
  const uint32_t raw = ptx::smem_u32(smem_raw), ring = (raw + 1023u) & ~1023u, full0 = ptx::smem_u32(bars), empty0 = full0 + 8u * kMaxStages;
  const uint8_t* smem = smem_raw + (ring - raw);
  float* sums = reinterpret_cast<float*>(smem_raw + (ring - raw) + (size_t)nst * stage_bytes);

  if (threadIdx.x == 0) {
    abort_flags[0] = abort_flags[1] = 0;
    for (int i = 0; i < nst; ++i) {
      ptx::mbar_init(full0 + 8u * i, 1);
      ptx::mbar_init(empty0 + 8u * i, WK * wn);
    }
    ptx::fence_barrier_init();
    ptx::prefetch_tensormap(&tmap_codes);
    ptx::prefetch_tensormap(&tmap_scales);
    ptx::prefetch_tensormap(&tmap_a);
  }
  __syncthreads();
  bool ok = true;
  if (warp == WK * wn) {
    // ---------------------------------------------------------------- producer (what lies outside the matrices comes as zeros)
    if (ptx::elect_one()) {
      // codes and scales, which no kernel writes, and rows, apart so that the first ones' codes can go ahead of the dependency wait
      auto load_codes = [&](int slot, int tile0, int piece) {
        const uint32_t dst = ring + (uint32_t)slot * stage_bytes, bar = full0 + 8u * slot;
        ptx::mbar_expect_tx(bar, filling);
        ptx::tma_load_3d(dst + St::ROWS, &tmap_codes, 0, piece * kStageChunks, tile0, bar);
        ptx::tma_load_3d(dst + scales_at, &tmap_scales, 0, piece * St::GROUPS, tile0, bar);
      };
      auto load_rows = [&](int slot, int piece) {
        ptx::tma_load_3d(ring + (uint32_t)slot * stage_bytes, &tmap_a, 0, 0, piece * kStageChunks, full0 + 8u * slot);
      };
      const int ahead = min(nst, per_unit);                // of the first unit's
      for (int i = 0; i < ahead; ++i) load_codes(i, (int)blockIdx.x * wn, i);
      pdl_wait();
      for (int i = 0; i < ahead; ++i) load_rows(i, i);
      int slot = ahead == nst ? 0 : ahead, phase = ahead == nst ? 0 : 1, filled = ahead;   // phase: parity of the emptying waited for (1: a fresh slot passes)
      for (int unit = blockIdx.x, first = ahead; unit < units && ok; unit += gridDim.x, first = 0) {
        for (int p = first; p < per_unit; ++p) {
          if (!ptx::mbar_wait(empty0 + 8u * slot, (uint32_t)phase, abort_flag)) { ok = false; break; }
          load_codes(slot, unit * wn, p);
          load_rows(slot, p);
          ++filled;
          if (++slot == nst) { slot = 0; phase ^= 1; }
        }
      }
      if (!ok) {                                           // let copies already issued land before the CTA's shared memory is released
        *(volatile int*)status = ST_GEMM_QUANTIZED;
        for (int k = filled > nst ? filled - nst : 0; k < filled; ++k)
          ptx::mbar_wait(full0 + 8u * (k % nst), (uint32_t)(k / nst) & 1u, abort_flag + 1, 20000000LL);
      }
    }
    __syncwarp();
    pdl_launch_dependents();
    return;
  }
  pdl_sync();
  const int consumers = 32 * WK * wn;                      // (their barriers do not wait for the producer, which runs ahead)
  auto sync_consumers = [&]() { asm volatile("bar.sync 1, %0;" ::"r"(consumers) : "memory"); };

  const uint32_t x_lo = (uint32_t)(g * 128 + ((t ^ g) << 4)), x_hi = x_lo ^ 64u;   // a lane's pieces of a row, swizzled
  int slot = 0, phase = 0;
  for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
    float acc[1][4] = {};
    for (int p = 0; p < per_unit && ok; ++p) {
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(full0 + 8u * slot, (uint32_t)phase, abort_flag))) { ok = false; break; }
      const uint8_t* stage = smem + (uint32_t)slot * stage_bytes;
      const uint8_t* w_at = stage + St::ROWS + iw * St::CODES + lane * 16;
      const uint8_t* s_at = stage + scales_at + iw * St::SCALES + g * 4;
      const int left = chunks - p * kStageChunks;
#pragma unroll
      for (int j = 0; j < CW; ++j) {
        const int c = ik * CW + j;                         // of the stage
        if (c < left) {
          uint4 x[1][2];
          x[0][0] = *reinterpret_cast<const uint4*>(stage + x_lo + c * 1024);
          x[0][1] = *reinterpret_cast<const uint4*>(stage + x_hi + c * 1024);
          multiply_chunk<1, BF, G>(acc, *reinterpret_cast<const uint4*>(w_at + c * 512), x, [&](int k) {
            return *reinterpret_cast<const uint32_t*>(s_at + (G == 32 ? 2 * c + k : c * kChunk / G) * 32);
          });
        }
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(empty0 + 8u * slot);
      if (++slot == nst) { slot = 0; phase ^= 1; }
    }
    // accumulator: outputs g and g + 8, rows 2 t and 2 t + 1
    sync_consumers();                                      // the unit before has been stored
    float* mine = sums + ik * (8 * cols) + 16 * iw;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine[(2 * t + (e & 1)) * cols + g + 8 * (e >> 1)] = acc[0][e];
    sync_consumers();
    if (*abort_flag) { ok = false; continue; }             // nothing is stored of what is missing; the barriers stay in step
    const int pairs = cols / 2, all = M * pairs;           // two neighbouring outputs of a row each
    for (int q = threadIdx.x; q < all; q += consumers) {
      const int m = q / pairs, n = unit * cols + 2 * (q - m * pairs);
      if (n >= N) continue;
      float2 y = *reinterpret_cast<const float2*>(sums + 2 * q);
#pragma unroll
      for (int k = 1; k < WK; ++k) {
        const float2 v = *reinterpret_cast<const float2*>(sums + k * (8 * cols) + 2 * q);
        y.x += v.x;
        y.y += v.y;
      }
      finish(y, bias, m, n, N, epi, out, out_bf16);
    }
  }
  if (!ok && lane == 0) *(volatile int*)status = ST_GEMM_QUANTIZED;
}

// One CTA per tile of 16 outputs and span of max(64, group) inputs: eight threads per output find the scales, then every thread packs words.
__global__ void __launch_bounds__(128)
quantize_weights_kernel(const float* __restrict__ w, int N, int K, int group, uint32_t* __restrict__ codes, uint16_t* __restrict__ scales) {
  __shared__ float s_scale[16][2];
  pdl_wait();                                              // (and no early release: see the end)
  const int span = group > kChunk ? group : kChunk, per = span / 8, r = threadIdx.x >> 3, j = threadIdx.x & 7;
  const int tile = blockIdx.x, k0 = blockIdx.y * span;
  const float* src = w + (size_t)(tile * 16 + r) * K + k0 + j * per;
  float amax = 0.f;
  bool finite = true;
  for (int i = 0; i < per; ++i) {
    const float x = fabsf(src[i]);
    finite = finite && x <= 3.402823466e38f;
    amax = fmaxf(amax, x);
  }
  if (!finite) amax = INFINITY;
  for (int d = 1; d < group / per; d *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, d));
  const bf16 rounded = __float2bfloat16_rn(amax == INFINITY ? __int_as_float(0x7fffffff) : __fdiv_rn(amax, 7.0f));
  if (j * per % group == 0) {
    const int in_span = j * per / group;
    s_scale[r][in_span] = __bfloat162float(rounded);
    scales[((size_t)tile * (K / group) + k0 / group + in_span) * 16 + 2 * (r & 7) + (r >> 3)] = __bfloat16_as_ushort(rounded);
  }
  __syncthreads();
  for (int q = threadIdx.x; q < span / kChunk * 128; q += 128) {
    const int c = q >> 7, lane = (q >> 2) & 31, s = q & 3, g = lane >> 2, t = lane & 3;
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {                          // nibble e & 4 ? high half : low half of operand register e & 3
      const int reg = e & 3, row = g + 8 * (reg & 1), k = c * kChunk + 32 * (s >> 1) + 8 * t + 4 * (s & 1) + 2 * (reg >> 1) + (e >> 2);
      const float scale = s_scale[row][k / group];
      const float x = w[(size_t)(tile * 16 + row) * K + k0 + k];
      const float code = scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(x, scale)), -7.f), 7.f) : 0.f;
      word |= (uint32_t)((int)code + 8) << (4 * reg + 16 * (e >> 2));
    }
    codes[(((size_t)tile * (K / kChunk) + k0 / kChunk + c) * 32 + lane) * 4 + s] = word;
  }
  // A projection fetches its first codes ahead of its dependency wait: it may not start before these are written and visible.
  __threadfence();
}

}  // namespace

// How a projection is cut: the kernel for small matrices, with so many warps per CTA; for large ones the one for up to eight rows, with units of wn
// tiles and nst stages, or, for more, the one on tcgen05 by CTAs or pairs of them.
// Large: the matrix is worth a ring and the CTAs are many enough to fill the device, which few outputs with a long K are only as pairs (us, small
// kernel and tcgen05: 31 x 4096 x 11008 20.0, 16.7; 31 x 8192 x 4096 15.0, 11.8; 31 x 16384 x 1024 11.6, 8.4; but 31 x 4096 x 4096 8.7, 9.4;
// 31 x 8192 x 1024 6.8, 7.5; 31 x 1024 x 8192 8.7, 13.1; 1 x 16384 x 8192 on tcgen05 21.3, by the ring 20.9).
QuantizedGemmShape gemm_quantized_pick(int M, int N, int K, int group) {
  const int tiles = N / 16, chunks = K / kChunk, sms = device_sm_count();
  QuantizedGemmShape s = {};
  const long size = (long)tiles * chunks;
  if (M > 8) {
    // a unit is 128 outputs by 16 or 32 rows; pairs where half the stages (of 4 chunks) in more turns are fewer
    const int nr = M <= 16 ? 16 : 32, stages = (chunks + 3) / 4;
    const long units = (long)((N + 127) / 128) * ((M + nr - 1) / nr);
    if (size >= (tiles >= 2 * sms ? 64L : 128L) * sms && 6 * units >= sms)
      s.tc = stages >= 2 && (units + sms / 2 - 1) / (sms / 2) * ((stages + 1) / 2) < (units + sms - 1) / sms * stages ? 2 : 1;
  } else if (tiles >= 2 * sms && size >= 64L * sms) {
    long best = 0;                                         // the fewest tiles in turn on an SM
    for (int wn = 4; wn <= kMaxTiles; ++wn) {
      const long cost = ((tiles + wn - 1) / wn + sms - 1) / sms * wn;
      if (!best || cost <= best) { best = cost; s.wn = wn; }
    }
    while (s.nst < kMaxStages) {
      ++s.nst;
      if (gemm_quantized_smem(M, group, s) > 200 * 1024) { --s.nst; break; }
    }
  }
  if (!s.tc && !s.wn) s.warps = chunks < 8 ? chunks : (tiles <= sms && chunks >= 16 ? 16 : 8);
  return s;
}

size_t gemm_quantized_smem(int M, int group, const QuantizedGemmShape& s) {
  if (s.wn) return 1024 + (size_t)s.nst * stage_bytes_of(group, s.wn) + (size_t)WK * 8 * 16 * s.wn * 4;
  return (size_t)s.warps * 8 * (M > kMaxRows ? kMaxRows / 8 : (M + 7) / 8) * 16 * 4;
}

namespace {

struct Args {
  const void* a; int lda, M; const void* codes; const void* scales; const float* bias; int N, K, group, epi; void* out; int out_bf16, *status; cudaStream_t st;
};

template <int MT, bool BF, int G>
cudaError_t launch_small(const Args& p, const QuantizedGemmShape& s) {
  return launch_pdl(gemm_quantized_small_kernel<MT, BF, G>, dim3(p.N / 16, (p.M + 8 * MT - 1) / (8 * MT)), dim3(32 * s.warps), gemm_quantized_smem(p.M, G, s), p.st,
                    (const uint16_t*)p.a, p.lda, p.M, (const uint4*)p.codes, (const uint32_t*)p.scales, p.bias, p.N, p.K, p.epi, p.out, p.out_bf16);
}

template <bool BF, int G>
cudaError_t launch_stream(const Args& p, const QuantizedGemmShape& s) {
  const size_t smem = gemm_quantized_smem(p.M, G, s);
  if (smem > 220 * 1024 || s.nst < 2 || s.wn > kMaxTiles || p.M > 8) return cudaErrorInvalidValue;
  static size_t smem_set[kMaxDevices] = {};
  cudaError_t e = ensure_dynamic_smem(gemm_quantized_stream_kernel<BF, G>, smem, smem_set);
  if (e != cudaSuccess) return e;
  const int sms = device_sm_count(), units = (p.N / 16 + s.wn - 1) / s.wn;
  // boxes of a stage: [chunk][8 rows][64 values], [tile][chunk][512 bytes], [tile][group][32 bytes]
  CUtensorMap ta, tc, ts;
  EncodeTiledFn fn = tma_encode_fn();
  const cuuint64_t chunks = p.K / kChunk, groups = p.K / G, tiles = p.N / 16;
  auto make = [&](CUtensorMap* map, CUtensorMapDataType type, const void* ptr, cuuint64_t d0, cuuint64_t d1, cuuint64_t d2, cuuint64_t s1, cuuint64_t s2, int b0,
                  int b1, int b2, bool swizzle) {
    const cuuint64_t dims[3] = {d0, d1, d2}, strides[2] = {s1, s2};
    const cuuint32_t box[3] = {(cuuint32_t)b0, (cuuint32_t)b1, (cuuint32_t)b2}, unit[3] = {1, 1, 1};
    return fn && fn(map, type, 3, const_cast<void*>(ptr), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (!make(&ta, CU_TENSOR_MAP_DATA_TYPE_UINT16, p.a, kChunk, p.M, chunks, (cuuint64_t)p.lda * 2, kChunk * 2, kChunk, 8, kStageChunks, true) ||
      !make(&tc, CU_TENSOR_MAP_DATA_TYPE_UINT32, p.codes, 128, chunks, tiles, 512, chunks * 512, 128, kStageChunks, s.wn, false) ||
      !make(&ts, CU_TENSOR_MAP_DATA_TYPE_UINT32, p.scales, 8, groups, tiles, 32, groups * 32, 8, Stage<G>::GROUPS, s.wn, false))
    return cudaErrorInvalidValue;
  return launch_pdl(gemm_quantized_stream_kernel<BF, G>, dim3((unsigned)(units < sms ? units : sms)), dim3(32 * (s.wn * WK + 1)), smem, p.st, ta, tc, ts, p.M, p.bias,
                    p.N, p.K, p.epi, p.out, p.out_bf16, s.wn, s.nst, (uint32_t)stage_bytes_of(G, s.wn), p.status);
}

template <bool BF, int G>
cudaError_t launch(const Args& p, const QuantizedGemmShape& s) {
  if (s.wn) return launch_stream<BF, G>(p, s);
  switch ((p.M + 7) / 8) {
    case 1: return launch_small<1, BF, G>(p, s);
    case 2: return launch_small<2, BF, G>(p, s);
    case 3: return launch_small<3, BF, G>(p, s);
    default: return launch_small<4, BF, G>(p, s);
  }
}

}  // namespace

cudaError_t launch_gemm_quantized(const void* a, int lda, int M, const void* codes, const void* scales, const float* bias, int N, int K, int group,
                                  int epilogue, void* out, bool a_bf16, int* status, cudaStream_t st) {
  const QuantizedGemmShape s = gemm_quantized_pick(M, N, K, group);
  if (s.tc) return launch_gemm_quantized_tc(a, lda, M, codes, scales, bias, N, K, group, epilogue, out, a_bf16, s.tc, status, st);
  // (the bias epilogue's output is bf16 in every 16-bit context)
  const Args p = {a, lda, M, codes, scales, bias, N, K, group, epilogue, out, epilogue == 0 || a_bf16, status, st};
  if (a_bf16) return group == 32 ? launch<true, 32>(p, s) : group == 64 ? launch<true, 64>(p, s) : launch<true, 128>(p, s);
  return group == 32 ? launch<false, 32>(p, s) : group == 64 ? launch<false, 64>(p, s) : launch<false, 128>(p, s);
}

cudaError_t launch_quantize_weights(const float* w, int N, int K, int group, void* codes, void* scales, cudaStream_t st) {
  const int span = group > kChunk ? group : kChunk;
  return launch_pdl(quantize_weights_kernel, dim3(N / 16, K / span), dim3(128), 0, st, w, N, K, group, (uint32_t*)codes, (uint16_t*)scales);
}

}  // namespace marche
