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
#include "common.cuh"
#include "kernels.h"
#include "launch_pdl.h"
#include "tma_host.h"

namespace marche {

namespace {

constexpr int kChunk = 64;                 // inputs of a warp's load
constexpr int kMaxRows = 32;               // of a CTA

template <bool BF>
MARCHE_DEVINL void mma_weights(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

// blockIdx.x: NT tiles of 16 outputs; blockIdx.y: 8 MT rows.  The CTA's warps take the 64-wide chunks of K in turn, PF chunks ahead of
// themselves.  G32: k16 steps of a group of 32 inputs (2), else a group is one or two whole chunks.
template <int NT, int MT, bool BF, bool G32>
__global__ void __launch_bounds__(NT == 1 ? 512 : 256)
gemm_quantized_kernel(const uint16_t* __restrict__ a, int lda, int M, const uint4* __restrict__ codes, const uint16_t* __restrict__ scales,
                      const float* __restrict__ bias, int N, int K, int group, int epi, void* __restrict__ out, int out_bf16) {
  constexpr int PF = NT == 1 ? 4 : 3;
  extern __shared__ float parts[];                         // [warp][8 MT rows][16 NT outputs]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, g = lane >> 2, t = lane & 3;
  const int chunks = K / kChunk, tile0 = blockIdx.x * NT, tiles = N / 16, row0 = blockIdx.y * (8 * MT);
  const int n_groups = K / group;
  const uint4* src[NT];
  const uint16_t* sc[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int tile = min(tile0 + i, tiles - 1);            // (the last CTA's surplus tile is computed and not stored)
    src[i] = codes + (size_t)tile * chunks * 32 + lane;
    sc[i] = scales + (size_t)tile * n_groups * 16 + g;
  }
  uint4 w[PF][NT];
#pragma unroll
  for (int p = 0; p < PF; ++p) {
    const int c = warp + p * warps;
#pragma unroll
    for (int i = 0; i < NT; ++i) w[p][i] = c < chunks ? ld_stream(src[i] + (size_t)c * 32) : make_uint4(0, 0, 0, 0);
  }
  pdl_sync();                                              // the weights are on their way while the previous kernel drains

  float acc[NT][MT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[i][m][0] = acc[i][m][1] = acc[i][m][2] = acc[i][m][3] = 0.f;
  const uint16_t* rows[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) rows[m] = a + (size_t)(row0 + 8 * m + g) * lda + 8 * t;

  for (int c0 = warp; c0 < chunks; c0 += PF * warps) {
#pragma unroll
    for (int p = 0; p < PF; ++p) {
      const int c = c0 + p * warps;
      if (c < chunks) {
        uint4 x[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            x[m][hf] = row0 + 8 * m + g < M ? *reinterpret_cast<const uint4*>(rows[m] + (size_t)c * kChunk + 32 * hf) : make_uint4(0, 0, 0, 0);
        const int next = c + PF * warps;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const uint32_t words[4] = {w[p][i].x, w[p][i].y, w[p][i].z, w[p][i].w};
          float part[MT][4];
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            if (s == 0 || (G32 && s == 2)) {
#pragma unroll
              for (int m = 0; m < MT; ++m) part[m][0] = part[m][1] = part[m][2] = part[m][3] = 0.f;
            }
            uint32_t f[4];
            numbers_of<BF>(words[s], f);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const uint4& v = x[m][s >> 1];
              mma_weights<BF>(part[m], f, s & 1 ? v.z : v.x, s & 1 ? v.w : v.y);
            }
            if (s == 3 || (G32 && s == 1)) {
              const uint16_t* at = sc[i] + (size_t)(G32 ? 2 * c + (s >> 1) : c * kChunk / group) * 16;
              const float s0 = __uint_as_float((uint32_t)__ldg(at) << 16), s1 = __uint_as_float((uint32_t)__ldg(at + 8) << 16);
#pragma unroll
              for (int m = 0; m < MT; ++m) {
                acc[i][m][0] = fmaf(part[m][0], s0, acc[i][m][0]);
                acc[i][m][1] = fmaf(part[m][1], s0, acc[i][m][1]);
                acc[i][m][2] = fmaf(part[m][2], s1, acc[i][m][2]);
                acc[i][m][3] = fmaf(part[m][3], s1, acc[i][m][3]);
              }
            }
          }
          if (next < chunks) w[p][i] = ld_stream(src[i] + (size_t)next * 32);
        }
      }
    }
  }
  // accumulator: outputs g and g + 8, rows 2 t and 2 t + 1 of an eight
  float* mine = parts + warp * (8 * MT * 16 * NT);
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[(8 * m + 2 * t + (e & 1)) * (16 * NT) + 16 * i + g + 8 * (e >> 1)] = acc[i][m][e];
  __syncthreads();
  for (int q = threadIdx.x; q < 8 * MT * 8 * NT; q += blockDim.x) {      // two neighbouring outputs
    const int m = q / (8 * NT), col = 2 * (q - m * (8 * NT)), row = row0 + m, n = tile0 * 16 + col;
    if (row >= M || n >= N) continue;
    float2 y = __ldg(reinterpret_cast<const float2*>(bias + n));
    for (int k = 0; k < warps; ++k) {
      const float2 v = *reinterpret_cast<const float2*>(parts + k * (8 * MT * 16 * NT) + m * (16 * NT) + col);
      y.x += v.x;
      y.y += v.y;
    }
    if (epi == 1) {
      float2* o = reinterpret_cast<float2*>((float*)out + (size_t)row * N + n);
      const float2 r = *o;
      *o = make_float2(r.x + y.x, r.y + y.y);
    } else {
      if (epi == 2) { y.x = gelu_erf(y.x); y.y = gelu_erf(y.y); }
      reinterpret_cast<uint32_t*>(out)[((size_t)row * N + n) >> 1] = pack_a16x2(y.x, y.y, out_bf16 != 0);
    }
  }
}

// One CTA per tile of 16 outputs and span of max(64, group) inputs: eight threads per output find the scales, then every thread packs words.
__global__ void __launch_bounds__(128)
quantize_weights_kernel(const float* __restrict__ w, int N, int K, int group, uint32_t* __restrict__ codes, uint16_t* __restrict__ scales) {
  __shared__ float s_scale[16][2];
  pdl_sync();
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
    scales[((size_t)tile * (K / group) + k0 / group + in_span) * 16 + r] = __bfloat16_as_ushort(rounded);
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
}

struct Shape { int nt, warps; };

// Tiles of a warp and warps of a CTA.  Two tiles share what is read of the rows, one gives twice the CTAs.
Shape pick(int M, int N, int K) {
  const int tiles = N / 16, chunks = K / kChunk, sms = device_sm_count();
  Shape s;
  s.nt = tiles >= 4 * sms ? 2 : 1;
  s.warps = chunks < 8 ? chunks : 8;
  const int ctas = (tiles + s.nt - 1) / s.nt;
  if (ctas <= sms) s.warps = chunks < 16 ? chunks : 16;
  return s;
}

template <int NT, int MT, bool BF, bool G32>
cudaError_t launch(const void* a, int lda, int M, const void* codes, const void* scales, const float* bias, int N, int K, int group, int epi,
                   void* out, int out_bf16, int warps, cudaStream_t st) {
  const size_t smem = (size_t)warps * (8 * MT * 16 * NT) * 4;
  static size_t smem_set[kMaxDevices] = {};
  cudaError_t e = smem > 48 * 1024 ? ensure_dynamic_smem(gemm_quantized_kernel<NT, MT, BF, G32>, smem, smem_set) : cudaSuccess;
  if (e != cudaSuccess) return e;
  return launch_pdl(gemm_quantized_kernel<NT, MT, BF, G32>, dim3((N / 16 + NT - 1) / NT, (M + 8 * MT - 1) / (8 * MT)), dim3(32 * warps), smem, st,
                    (const uint16_t*)a, lda, M, (const uint4*)codes, (const uint16_t*)scales, bias, N, K, group, epi, out, out_bf16);
}

}  // namespace

cudaError_t launch_gemm_quantized(const void* a, int lda, int M, const void* codes, const void* scales, const float* bias, int N, int K, int group,
                                  int epilogue, void* out, bool a_bf16, cudaStream_t st) {
  const Shape s = pick(M, N, K);
  const int mt = M > kMaxRows ? kMaxRows / 8 : (M + 7) / 8, ob = epilogue == 0 || a_bf16;   // (the bias epilogue's output is bf16)
#define MARCHE_Q_LAUNCH(NT_, MT_, BF_, G_) \
  return launch<NT_, MT_, BF_, G_>(a, lda, M, codes, scales, bias, N, K, group, epilogue, out, ob, s.warps, st)
#define MARCHE_Q_TYPE(NT_, MT_)                                                     \
  do {                                                                              \
    if (a_bf16) { if (group == 32) MARCHE_Q_LAUNCH(NT_, MT_, true, true); MARCHE_Q_LAUNCH(NT_, MT_, true, false); } \
    if (group == 32) MARCHE_Q_LAUNCH(NT_, MT_, false, true);                        \
    MARCHE_Q_LAUNCH(NT_, MT_, false, false);                                        \
  } while (0)
#define MARCHE_Q_ROWS(NT_)                     \
  do {                                         \
    if (mt == 1) MARCHE_Q_TYPE(NT_, 1);        \
    if (mt == 2) MARCHE_Q_TYPE(NT_, 2);        \
    if (mt == 3) MARCHE_Q_TYPE(NT_, 3);        \
    MARCHE_Q_TYPE(NT_, 4);                     \
  } while (0)
  if (s.nt == 2) MARCHE_Q_ROWS(2);
  MARCHE_Q_ROWS(1);
#undef MARCHE_Q_ROWS
#undef MARCHE_Q_TYPE
#undef MARCHE_Q_LAUNCH
}

cudaError_t launch_quantize_weights(const float* w, int N, int K, int group, void* codes, void* scales, cudaStream_t st) {
  const int span = group > kChunk ? group : kChunk;
  return launch_pdl(quantize_weights_kernel, dim3(N / 16, K / span), dim3(128), 0, st, w, N, K, group, (uint32_t*)codes, (uint16_t*)scales);
}

}  // namespace marche
