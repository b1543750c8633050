// K3 over a cache held in 8 bits: attention of n query rows per sample over the sample's keys, values code * scale.
//
// o = softmax(q K^T / sqrt(dh)) V with K[s] = ks[s] ck[s], V[s] = vs[s] cv[s], codes c in -127 .. 127 and one scale per key and head.
// The scales are kept out of the products: the logit of a key is ks[s] (q . ck[s]), and vs[s] goes into the weight, so the tensor
// cores multiply the codes themselves, which are exact in fp16.  q (bf16) is exact in fp16 after a power of two of its row is taken off; what
// is rounded is the weight: p vs / 2^e to fp16 (11 bits), where 2^e bounds the largest value scale met so far and the whole is
// lifted by 2^14, so that a weight 2^-28 of the largest possible keeps all its bits (scales far apart: attention_quantized.cuh).  Maxima, sums and
// accumulators are fp32, and the running exponent e moves with the running maximum (one factor for both).
// Where the output is fp16, what that rounding left off follows as a second operand (FINE): with one rounding of as many bits as the output's own the
// error is 1.4 times the output's, 1.55 over few keys.  A bf16 output, eight times coarser, does not need it (128 x 43 rows over 320 keys of 16
// heads of 80: 66 us without, 77 with it).
// Query heads that share a cached head are rows of one item: row r is token r / G, head r % G of the group.
//
// mma.sync m16n8k16 on the transposed products, S^T = K q^T and O^T = V^T P^T: keys (then columns of V) are the 16-row operand and the
// query rows come in eights, so one token costs half of what a 16-row tile of queries would, and the codes, converted once, serve all
// NB eights of a warp.  K: a dot product does not mind the order of its terms, so a lane's 16 consecutive bytes of a key serve as its
// operands of four k16 steps (bytes 0 and 2 of a word, then 1 and 3): no transposition and one shared-memory load.  V: ldmatrix.trans on
// pairs of bytes, whose even and odd bytes are rows g and g + 8 of the operand.  Codes become numbers (1024 + code + 128, minus 1152); as they
// stand, code + 128 is a fp16 subnormal, which the tensor cores multiply exactly, but 128 times the sum of the other operand would
// have to come off, and where that is of one sign the result loses as many bits as it is smaller (logits are then off by 2^-16 of the sum of
// magnitudes, where fp32 sums are by 2^-23; it would save 2 % at 128 x 43 rows, 3 % at one token over 65521 keys).  P: the accumulator's layout is turned by movmatrix.
// nr warps take 8 NB rows each; nk groups of them take the tiles of 32 or 64 keys (K, V and both scales, by TMA) in turn, each group with a
// ring of nst stages that its first warp fills (slot and phase are stepped: a division in that place cost more than the tile); a cluster of cs
// CTAs splits a long sequence.  (CTA, group) pairs merge in rank order in the CTA that owns the row: bit-reproducible.  A sample without
// keys gives zeros.
// What bounds it: with a row or a few, one warp's chain through a tile (2500 cycles for 32 keys of 128 values: wait, products, maxima over lanes,
// exponentials, products, refill), and the cut by sample: at most eight CTAs work on a (sample, head), so the longest sample's finish alone: 4 x 65521
// keys at most, 8 cached heads of 128, one token: 90 us of 42 for the bytes.  With more rows its instructions, a third of them conversions that the
// warps of a tile repeat: the 128 x 43 rows above 66 us of 21, 54 % of the issue slots (16 warps on an SM instead of 12, at 128 registers, spill: slower).
#include <cuda.h>

#include "attention_common.cuh"
#include "attention_quantized.cuh"
#include "kernels.h"
#include "launch_pdl.h"
#include "sm100_ptx.cuh"
#include "tma_host.h"

namespace marche {

namespace {

using att::ex2_approx;
using att::ldsm_x4_trans;
using attq::pow2;

constexpr int kMaxStages = 16;             // of a CTA
constexpr int kThreadsMax = 256;
constexpr int kSpread = 16;                // a row's largest product is at least 2^(14 - 1 - 16) before its sample counts as wide
enum { ST_ATTENTION_QUANTIZED = 0x25 };

// Keys per tile: 64 where shared memory holds two tiles for each of eight warps.
constexpr int tile_keys(int dh) { return dh == 128 ? 32 : 64; }

template <int DH, int NB> struct Cfg {
  static constexpr int KT = tile_keys(DH), NM = KT / 16;
  static constexpr int TILE = KT * DH;                     // K or V of a stage
  static constexpr int STAGE = 2 * TILE;
  static constexpr int SCALES = 2 * KT * 4;                // of a stage: K's, V's
  static constexpr int STEPS = DH / 16, CHUNKS = DH / 16;  // k16 steps of q . k; 16-byte pieces of a row
  static constexpr int ROW = DH + 4;                       // floats of a partial result: sums, maximum, sum of weights
};

// Byte offset of 16-byte piece c of key r in a tile, as TMA wrote it (64- and 128-byte rows swizzled, 80-byte rows as they are: eight
// consecutive rows' pieces lie on different banks in all three).
template <int DH> MARCHE_DEVINL uint32_t piece(int r, int c) {
  if (DH == 64) return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
  if (DH == 128) return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4));
  return (uint32_t)(r * DH + (c << 4));
}
// First of the four values that lane t of a quad holds in k16 step s (the first and third for the step's lower, the others for its upper half).
template <int DH> MARCHE_DEVINL int value_of(int s, int t) { return DH == 80 ? 16 * s + 4 * t : 16 * (4 * (s / 4) + t) + 4 * (s % 4); }

MARCHE_DEVINL void ldsm_x2_trans(uint32_t addr, uint32_t& r0, uint32_t& r1) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(r0), "=r"(r1) : "r"(addr));
}
MARCHE_DEVINL void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two of the four bytes of a word of codes + 128 (SEL picks them and puts 0x64 above each) as fp16: 1024 + (code + 128) - 1152.
template <uint32_t SEL> MARCHE_DEVINL uint32_t two_of(uint32_t biased) {
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(__byte_perm(biased, 0x64646464u, SEL)), "r"(0x64806480u));
  return r;
}
MARCHE_DEVINL uint32_t pack_weights(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
MARCHE_DEVINL float2 unpack_f16x2(uint32_t u) {
  __half2 h = *reinterpret_cast<__half2*>(&u);
  return __half22float2(h);
}
// Packed fp32 pairs, one instruction for two values.
MARCHE_DEVINL void mul2(float& a, float& b, float x, float y) {
  const float2 r = __fmul2_rn(make_float2(a, b), make_float2(x, y));
  a = r.x;
  b = r.y;
}
MARCHE_DEVINL void add2(float& a, float& b, float x, float y) {
  const float2 r = __fadd2_rn(make_float2(a, b), make_float2(x, y));
  a = r.x;
  b = r.y;
}
MARCHE_DEVINL float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
MARCHE_DEVINL uint32_t turn8x8(uint32_t x) {               // an 8 x 8 matrix of 16-bit values, spread over the warp as fragments are
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// Grid: B * H * n_rb * cs CTAs, the cs of a cluster next to one another.  (At head_dim 80 the bound of 384 threads, which no launch has, keeps the
// registers to 168, with which four CTAs of three warps fit on an SM: 128 x 43 rows with fp16 outputs 109 us with 174 registers, 78 with 168.)
template <int DH, int NB, bool FINE>
__global__ void __launch_bounds__(DH == 80 && NB == 2 ? 384 : kThreadsMax)
attention_quantized_kernel(const __grid_constant__ CUtensorMap tmap, const __grid_constant__ CUtensorMap tmap_scales, const bf16* __restrict__ q, int ld_q, int n, int heads, int H, int G, int B, int S,
                           const int32_t* __restrict__ kv_len, uint16_t* __restrict__ o, int o_bf16,
                           const QuantizedSplit sp, int* __restrict__ status) {
  using C = Cfg<DH, NB>;
  constexpr int RPW = 8 * NB, KT = C::KT, NM = C::NM;      // rows of a warp
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t scale_base = base + (uint32_t)(sp.nk * sp.nst * C::STAGE), recv = scale_base + (uint32_t)(sp.nk * sp.nst * C::SCALES);
  uint8_t* gen = smem_raw + (base - raw);
  const float* recv_gen = reinterpret_cast<const float*>(smem_raw + (recv - raw));
  __shared__ __align__(8) uint64_t bars[2 * kMaxStages];   // full, empty
  __shared__ int abort_flags[2];
  volatile int* abort_flag = abort_flags;
  const uint32_t full0 = ptx::smem_u32(bars), empty0 = full0 + 8u * kMaxStages;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int wk = warp / sp.nr, wr = warp - wk * sp.nr;
  const int rank = sp.cs > 1 ? (int)ptx::cluster_ctarank() : 0;
  const int block = (int)blockIdx.x / sp.cs, item = block / sp.n_rb, b = item / H, h = item - b * H;
  const int R = n * G, row_block = (block - item * sp.n_rb) * (sp.nr * RPW), row_w = row_block + wr * RPW;
  if (threadIdx.x == 0) {
    for (int i = 0; i < sp.nk * sp.nst; ++i) {
      ptx::mbar_init(full0 + 8u * i, 1);
      ptx::mbar_init(empty0 + 8u * i, (uint32_t)sp.nr);
    }
    abort_flags[0] = abort_flags[1] = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
    ptx::prefetch_tensormap(&tmap);
    ptx::prefetch_tensormap(&tmap_scales);
  }
  __syncwarp();
  if (sp.cs > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  __syncthreads();
  pdl_sync();

  int len = S;
  if (kv_len) len = min(max(kv_len[b], 0), S);
  const int tiles = (len + KT - 1) / KT;
  const int kt0 = (int)((long long)rank * tiles / sp.cs), n_tiles = (int)((long long)(rank + 1) * tiles / sp.cs) - kt0;
  const int mine = (n_tiles - wk + sp.nk - 1) / sp.nk, stage0 = wk * sp.nst;   // tiles wk, wk + nk, .. of the CTA's; the group's first stage
  // The group's next tile into its next stage (lane 0 of its first warp): K and V by one copy, both scales by another (four copies took 88 -> 94 us
  // for 4 x 65521 keys; a warp of its own for the refills costs registers, that is CTAs on an SM, and ties the groups to one another: 112).
  int f_slot = 0, issued = 0;
  auto load = [&]() {
    const int s = stage0 + f_slot, kt = kt0 + wk + issued * sp.nk;
    const uint32_t bar = full0 + 8u * s, dst = base + (uint32_t)(s * C::STAGE), dst_s = scale_base + (uint32_t)(s * C::SCALES);
    ptx::mbar_expect_tx(bar, C::STAGE + C::SCALES);
    ptx::tma_load_4d(dst, &tmap, h * DH, kt * KT, b, 0, bar);
    ptx::tma_load_3d(dst_s, &tmap_scales, kt * KT, b * H + h, 0, bar);
    ++issued;
    if (++f_slot == sp.nst) f_slot = 0;
  };
  if (wr == 0 && lane == 0)
    while (issued < mine && issued < sp.nst) load();
  __syncwarp();

  // Rows 2 t and 2 t + 1 of each eight: running maximum (of the logits in units of log2), this lane's part of the sum of weights; O^T: columns 16 c + 2 g (entries
  // 0, 1 for the two rows) and 16 c + 2 g + 1 (2, 3).
  bool ok = true;
  const bool active = row_w < R;
  float m_run[NB][2], l_run[NB][2], oacc[NB][C::CHUNKS][4];
  attq::Units units;
#pragma unroll
  for (int m = 0; m < NB; ++m) {
    m_run[m][0] = m_run[m][1] = -INFINITY;
    l_run[m][0] = l_run[m][1] = 0.f;
#pragma unroll
    for (int c = 0; c < C::CHUNKS; ++c) oacc[m][c][0] = oacc[m][c][1] = oacc[m][c][2] = oacc[m][c][3] = 0.f;
  }
  // ---- the warp's query rows as the operand of eight columns: lane (g, t) holds row g's values 0, 2 and 1, 3 of each step's four
  uint32_t qf[NB][C::STEPS][2];
  float c_log2[NB][2];                                     // of rows 2 t and 2 t + 1 of each eight
  if (active) {
    uint2 x[NB][C::STEPS];
#pragma unroll
    for (int m = 0; m < NB; ++m) {
      const int row = min(row_w + 8 * m + g, R - 1), token = row / G;       // (rows behind the last are the last one again: not stored)
      const bf16* src = q + ((size_t)b * n + token) * ld_q + (h * G + row - token * G) * DH;
#pragma unroll
      for (int s = 0; s < C::STEPS; ++s) x[m][s] = *reinterpret_cast<const uint2*>(src + value_of<DH>(s, t));
    }
    const float scale_log2 = rsqrtf((float)DH) * 1.4426950408889634f;
#pragma unroll
    for (int m = 0; m < NB; ++m) {
      uint32_t both = 0;
#pragma unroll
      for (int s = 0; s < C::STEPS; ++s) both = attq::larger2(both, attq::larger2(x[m][s].x & 0x7fff7fffu, x[m][s].y & 0x7fff7fffu));
      uint32_t top = max(both & 0xffffu, both >> 16);
      if (top >= 0x7f80u) {                                // (infinities and NaN stay what they are)
        top = 0;
#pragma unroll
        for (int s = 0; s < C::STEPS; ++s) top = max(top, max(attq::finite_of(x[m][s].x), attq::finite_of(x[m][s].y)));
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));   // of row g
      // The row divided by its largest value's power of two and lifted by 2^15, fp16's largest (a bf16 number below 2 stays below 65504): exact
      // down to 2^-32 of the largest value, and no logit is off by more than 2^-40 of its row's largest ones'.  Each row by its own: a row of padding
      // may hold numbers of any size.
      const int e = min(max((int)(top >> 7), 16), 254);
      const float f = pow2(269 - e), c = scale_log2 * pow2(e - 15);
#pragma unroll
      for (int s = 0; s < C::STEPS; ++s) {
        const float2 lo = unpack_bf16x2(x[m][s].x), hi = unpack_bf16x2(x[m][s].y);
        qf[m][s][0] = pack_weights(lo.x * f, hi.x * f);
        qf[m][s][1] = pack_weights(lo.y * f, hi.y * f);
      }
      c_log2[m][0] = __shfl_sync(0xffffffffu, c, 8 * t);
      c_log2[m][1] = __shfl_sync(0xffffffffu, c, 8 * t + 4);
    }
  }
  int turn = 0, phase = 0, turn_before = 0, phase_before = 0;   // stage of tile u in the group's ring, its fill's parity; the tile's before it
  for (int u = 0; u < mine; ++u) {
    const int s = stage0 + turn;
    if (!__all_sync(0xffffffffu, ptx::mbar_wait(full0 + 8u * s, (uint32_t)phase, abort_flag))) { ok = false; break; }
    if (active) {
      const uint8_t* k_tile = gen + s * C::STAGE;
      const uint32_t v_tile = base + (uint32_t)(s * C::STAGE + C::TILE);
      float* ks = reinterpret_cast<float*>(gen + (scale_base - base) + s * C::SCALES);
      float* vs = ks + KT;
      const int left = len - (kt0 + wk + u * sp.nk) * KT;  // keys of this tile that count
      if (left < KT) {                                     // scales behind the last key may be anything
        for (int k = lane; k < KT; k += 32)
          if (k >= left) ks[k] = vs[k] = 0.f;
        __syncwarp();
      }
      // ---- S^T: lane (g, t) gets keys 16 i + g (entries 0, 1: rows 2 t, 2 t + 1) and 16 i + g + 8 (2, 3)
      float sacc[NB][NM][4];
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        uint32_t w0[C::STEPS], w1[C::STEPS];
        const int key = 16 * i + g;
        if (DH == 80) {
#pragma unroll
          for (int k = 0; k < C::STEPS; ++k) {
            w0[k] = *reinterpret_cast<const uint32_t*>(k_tile + key * DH + 16 * k + 4 * t);
            w1[k] = *reinterpret_cast<const uint32_t*>(k_tile + (key + 8) * DH + 16 * k + 4 * t);
          }
        } else {
#pragma unroll
          for (int k = 0; k < C::STEPS / 4; ++k) {
            const uint4 u0 = *reinterpret_cast<const uint4*>(k_tile + piece<DH>(key, 4 * k + t));
            const uint4 u1 = *reinterpret_cast<const uint4*>(k_tile + piece<DH>(key + 8, 4 * k + t));
            w0[4 * k] = u0.x; w0[4 * k + 1] = u0.y; w0[4 * k + 2] = u0.z; w0[4 * k + 3] = u0.w;
            w1[4 * k] = u1.x; w1[4 * k + 1] = u1.y; w1[4 * k + 2] = u1.z; w1[4 * k + 3] = u1.w;
          }
        }
#pragma unroll
        for (int m = 0; m < NB; ++m) sacc[m][i][0] = sacc[m][i][1] = sacc[m][i][2] = sacc[m][i][3] = 0.f;
#pragma unroll
        for (int k = 0; k < C::STEPS; ++k) {
          const uint32_t lo = w0[k] ^ 0x80808080u, hi = w1[k] ^ 0x80808080u;
          const uint32_t a[4] = {two_of<0x4240>(lo), two_of<0x4240>(hi), two_of<0x4341>(lo), two_of<0x4341>(hi)};
#pragma unroll
          for (int m = 0; m < NB; ++m) mma_f16(sacc[m][i], a, qf[m][k][0], qf[m][k][1]);
        }
        const float f0 = ks[key], f1 = ks[key + 8];
#pragma unroll
        for (int m = 0; m < NB; ++m) {                     // in units of log2
          mul2(sacc[m][i][0], sacc[m][i][1], f0 * c_log2[m][0], f0 * c_log2[m][1]);
          mul2(sacc[m][i][2], sacc[m][i][3], f1 * c_log2[m][0], f1 * c_log2[m][1]);
        }
      }
      if (left < KT) {
#pragma unroll
        for (int m = 0; m < NB; ++m)
#pragma unroll
          for (int i = 0; i < NM; ++i) {
            if (16 * i + g >= left) sacc[m][i][0] = sacc[m][i][1] = -INFINITY;
            if (16 * i + g + 8 >= left) sacc[m][i][2] = sacc[m][i][3] = -INFINITY;
          }
      }
      // ---- references: the unit above the value scales, the rows' maxima
      const uint32_t v0 = attq::magnitude(vs[lane]), v1 = KT == 64 ? attq::magnitude(vs[lane + KT / 2]) : v0;
      units.see(__reduce_max_sync(0xffffffffu, max(v0, v1)), min(v0 - 1u, v1 - 1u));
      const bool apart = units.apart<kSpread>();
      bool moved = apart || units.top != units.unit;
      float most[NB][2], neg[NB][2];
      auto over_lanes = [&](float& mx) {
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
      };
#pragma unroll
      for (int m = 0; m < NB; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          most[m][r] = m_run[m][r];
#pragma unroll
          for (int i = 0; i < NM; ++i) most[m][r] = max3(most[m][r], sacc[m][i][r], sacc[m][i][2 + r]);
          over_lanes(most[m][r]);
          moved = moved || most[m][r] != m_run[m][r];
        }
      if (__any_sync(0xffffffffu, moved)) {
        const int d = units.move(__any_sync(0xffffffffu, apart), u == 0);
        float step_l = 1.f;
        if (__builtin_expect(units.wide, 0)) {             // other references than the rows' largest logits
          const float over_unit = pow2(max(253 - units.unit, 1));
          step_l = pow2(127 + d);
#pragma unroll
          for (int m = 0; m < NB; ++m) most[m][0] = m_run[m][0] -= (float)d, most[m][1] = m_run[m][1] -= (float)d;
#pragma unroll
          for (int i = 0; i < NM; ++i) {
            const float a0 = attq::counts(vs[16 * i + g] * over_unit), a1 = attq::counts(vs[16 * i + g + 8] * over_unit);
#pragma unroll
            for (int m = 0; m < NB; ++m)
#pragma unroll
              for (int r = 0; r < 2; ++r) most[m][r] = max3(most[m][r], sacc[m][i][r] + a0, sacc[m][i][2 + r] + a1);
          }
#pragma unroll
          for (int m = 0; m < NB; ++m) {
            over_lanes(most[m][0]);
            over_lanes(most[m][1]);
          }
        }
        const float step = units.wide ? 1.f : attq::step_of(d);
#pragma unroll
        for (int m = 0; m < NB; ++m) {
          float corr[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            corr[r] = ex2_approx(m_run[m][r] - (most[m][r] == -INFINITY ? 0.f : most[m][r]));
            m_run[m][r] = most[m][r];
          }
          mul2(l_run[m][0], l_run[m][1], corr[0], corr[1]);
          mul2(l_run[m][0], l_run[m][1], step_l, step_l);
          mul2(corr[0], corr[1], step, step);
#pragma unroll
          for (int c = 0; c < C::CHUNKS; ++c) {
            mul2(oacc[m][c][0], oacc[m][c][1], corr[0], corr[1]);
            mul2(oacc[m][c][2], oacc[m][c][3], corr[0], corr[1]);
          }
        }
      }
      const float lift = pow2(267 - units.unit);           // 2^14 over the power of two above the scale
#pragma unroll
      for (int m = 0; m < NB; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) neg[m][r] = m_run[m][r] == -INFINITY ? 0.f : -m_run[m][r];
      // ---- weights, turned, and O^T += V^T P^T
      float ls[NB][2];
#pragma unroll
      for (int m = 0; m < NB; ++m) ls[m][0] = ls[m][1] = 0.f;
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        uint32_t pb[NB][2], pl[NB][2];
        float f0 = vs[16 * i + g], f1 = vs[16 * i + g + 8];
        mul2(f0, f1, lift, lift);
#pragma unroll
        for (int m = 0; m < NB; ++m)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            float p0 = sacc[m][i][2 * hf], p1 = sacc[m][i][2 * hf + 1];
            add2(p0, p1, neg[m][0], neg[m][1]);
            p0 = ex2_approx(p0);
            p1 = ex2_approx(p1);
            add2(ls[m][0], ls[m][1], p0, p1);
            mul2(p0, p1, hf ? f1 : f0, hf ? f1 : f0);
            const uint32_t w = pack_weights(p0, p1);
            pb[m][hf] = turn8x8(w);
            if (FINE) {
              const float2 hi = unpack_f16x2(w);
              pl[m][hf] = turn8x8(pack_weights(p0 - hi.x, p1 - hi.y));
            }
          }
        const int key = 16 * i + 8 * ((lane >> 3) & 1) + (lane & 7);
#pragma unroll
        for (int c = 0; c < C::CHUNKS; c += 2) {
          uint32_t w[4];
          if (c + 1 < C::CHUNKS) ldsm_x4_trans(v_tile + piece<DH>(key, c + (lane >> 4)), w[0], w[1], w[2], w[3]);
          else ldsm_x2_trans(v_tile + piece<DH>(key, c), w[0], w[1]);
#pragma unroll
          for (int d = 0; d < 2 && c + d < C::CHUNKS; ++d) {
            const uint32_t lo = w[2 * d] ^ 0x80808080u, hi = w[2 * d + 1] ^ 0x80808080u;
            const uint32_t a[4] = {two_of<0x4240>(lo), two_of<0x4341>(lo), two_of<0x4240>(hi), two_of<0x4341>(hi)};
#pragma unroll
            for (int m = 0; m < NB; ++m) {
              mma_f16(oacc[m][c + d], a, pb[m][0], pb[m][1]);
              if (FINE) mma_f16(oacc[m][c + d], a, pl[m][0], pl[m][1]);
            }
          }
        }
      }
#pragma unroll
      for (int m = 0; m < NB; ++m) add2(l_run[m][0], l_run[m][1], ls[m][0], ls[m][1]);
    }
    __syncwarp();
    if (lane == 0) {
      ptx::mbar_arrive(empty0 + 8u * s);
      // The stage of the tile before this one (of this one where no other warp reads it) is free, or nearly: its next tile.
      if (wr == 0 && issued < mine && (sp.nr == 1 || u > 0)) {
        const int f = stage0 + (sp.nr == 1 ? turn : turn_before);
        if (ptx::mbar_wait(empty0 + 8u * f, (uint32_t)(sp.nr == 1 ? phase : phase_before), abort_flag)) load();
        else ok = false;
      }
    }
    ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
    if (!ok) break;
    turn_before = turn;
    phase_before = phase;
    if (++turn == sp.nst) { turn = 0; phase ^= 1; }
  }
  if (!ok && wr == 0 && lane == 0) {                       // let copies already issued land before the CTA's shared memory is released
    for (int u = issued > sp.nst ? issued - sp.nst : 0; u < issued; ++u)
      ptx::mbar_wait(full0 + 8u * (stage0 + u % sp.nst), (uint32_t)(u / sp.nst) & 1u, abort_flag + 1, 20000000LL);
  }
  if (!ok && lane == 0) *(volatile int*)status = ST_ATTENTION_QUANTIZED;
#pragma unroll
  for (int m = 0; m < NB; ++m)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l_run[m][r] += __shfl_xor_sync(0xffffffffu, l_run[m][r], 4);
      l_run[m][r] += __shfl_xor_sync(0xffffffffu, l_run[m][r], 8);
      l_run[m][r] += __shfl_xor_sync(0xffffffffu, l_run[m][r], 16);
    }
  auto row_out = [&](int row) {                            // of the item's rows
    const int token = row / G;
    return o + (((size_t)b * n + token) * heads + h * G + row - token * G) * DH;
  };
  const int n_parts = sp.cs * sp.nk;
  if (n_parts == 1) {
    if (active && ok) {
#pragma unroll
      for (int m = 0; m < NB; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = row_w + 8 * m + 2 * t + r;
          if (row < R) {
            uint16_t* to = row_out(row) + 2 * g;
            const float2 f = attq::unit_over(l_run[m][r], units.unit - 13);
#pragma unroll
            for (int c = 0; c < C::CHUNKS; ++c)
              *reinterpret_cast<uint32_t*>(to + 16 * c) = pack_a16x2(oacc[m][c][r] * f.x * f.y, oacc[m][c][2 + r] * f.x * f.y, o_bf16 != 0);
          }
        }
    }
    return;
  }
  // ---- partial results, means of values already (their sums could leave the format), to the owners of the rows, then the merge
  const int rows_cta = sp.nr * RPW, own = (rows_cta + sp.cs - 1) / sp.cs;
  if (sp.cs > 1) {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");                  // every CTA of the cluster has started
    if (!ok) ptx::cluster_raise(ptx::smem_u32(abort_flags), sp.cs);                      // nobody merges what is missing
  }
  if (active && ok) {
#pragma unroll
    for (int m = 0; m < NB; ++m)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int in = wr * RPW + 8 * m + 2 * t + r, owner = in / own;
        if (row_block + in < R) {
          uint32_t dst = recv + 4u * (uint32_t)(((rank * sp.nk + wk) * own + in - owner * own) * C::ROW);
          if (sp.cs > 1) dst = ptx::mapa(dst, (uint32_t)owner);
          const float2 f = attq::unit_over(l_run[m][r], units.unit - 13);
#pragma unroll
          for (int c = 0; c < C::CHUNKS; ++c)
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(dst + 4u * (16 * c + 2 * g)), "f"(oacc[m][c][r] * f.x * f.y),
                         "f"(oacc[m][c][2 + r] * f.x * f.y) : "memory");
          if (g == 0) {
            float ref = m_run[m][r], l = l_run[m][r];
            if (__builtin_expect(units.wide, 0) && l > 0.f) {                   // (references and sums far from the logits: the power of two belongs to the reference)
              ref += (float)((int)(__float_as_uint(l) >> 23) - 127);
              l = __int_as_float((__float_as_int(l) & 0x7fffff) | 0x3f800000);
            }
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(dst + 4u * DH), "f"(ref), "f"(l * 0x1p-24f) : "memory");   // (below 1: no sum leaves the format)
          }
        }
      }
  }
  if (sp.cs > 1) {
    __syncwarp();
    ptx::cluster_sync_all();
  } else {
    __syncthreads();
  }
  if (*abort_flag) return;
  const int stride = own * C::ROW;
  for (int e = threadIdx.x; e < own * (DH / 4); e += (int)blockDim.x) {
    const int j = e / (DH / 4), c = e % (DH / 4) * 4, in = rank * own + j, row = row_block + in;
    if (in >= rows_cta || row >= R) continue;
    const float* p = recv_gen + j * C::ROW;
    float mx = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < n_parts; ++s) mx = fmaxf(mx, p[s * stride + DH]);
    if (mx == -INFINITY) mx = 0.f;
    for (int s = 0; s < n_parts; ++s) {
      const float w = ex2_approx(p[s * stride + DH] - mx) * p[s * stride + DH + 1];
      const float4 v = *reinterpret_cast<const float4*>(p + s * stride + c);
      l += w;
      acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y);
      acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
    }
    const float f = l > 0.f ? 1.0f / l : l;                // (no key: zeros; NaN stays)
    uint2 v;
    v.x = pack_a16x2(acc.x * f, acc.y * f, o_bf16 != 0);
    v.y = pack_a16x2(acc.z * f, acc.w * f, o_bf16 != 0);
    *reinterpret_cast<uint2*>(row_out(row) + c) = v;
  }
}

template <int DH, int NB, bool FINE>
cudaError_t launch(const void* q, int ld_q, int n, int heads, const QuantizedKv& c, const int32_t* kv_len, void* o, bool o_bf16, const QuantizedSplit& s,
                   int* status, cudaStream_t st) {
  using C = Cfg<DH, NB>;
  const size_t smem = attention_quantized_smem(DH, s);
  if (smem > 226 * 1024) return cudaErrorInvalidValue;
  // boxes of a tile: K and V [2][keys][dh], their scales [2][keys]
  CUtensorMap tm, ts;
  EncodeTiledFn fn = tma_encode_fn();
  const cuuint64_t D = (cuuint64_t)c.H * DH, dims[4] = {D, (cuuint64_t)c.S, (cuuint64_t)c.B, 2}, strides[3] = {D, D * c.S, D * c.S * c.B};
  const cuuint64_t dims_s[3] = {(cuuint64_t)c.pad, (cuuint64_t)c.B * c.H, 2}, strides_s[2] = {(cuuint64_t)c.pad * 4, (cuuint64_t)c.pad * 4 * c.B * c.H};
  const cuuint32_t box[4] = {DH, C::KT, 1, 2}, box_s[3] = {C::KT, 1, 2}, unit[4] = {1, 1, 1, 1};
  const CUtensorMapSwizzle sw = DH == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : DH == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE;
  if (!fn || fn(&tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, c.codes, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS ||
      fn(&ts, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, c.scales, dims_s, strides_s, box_s, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  static size_t smem_set[kMaxDevices] = {};
  cudaError_t e = ensure_dynamic_smem(attention_quantized_kernel<DH, NB, FINE>, smem, smem_set);
  if (e != cudaSuccess) return e;
  const int G = heads / c.H;
  return launch_pdl_cluster(attention_quantized_kernel<DH, NB, FINE>, dim3((unsigned)((long)c.B * c.H * s.n_rb * s.cs)), dim3(s.nr * s.nk * 32), smem, s.cs, st, tm, ts,
                            (const bf16*)q, ld_q, n, heads, c.H, G, c.B, c.S, kv_len, (uint16_t*)o, o_bf16 ? 1 : 0, s, status);
}

}  // namespace

// Which kernel: by estimated time (us).  This one: a warp of 16 rows takes a tile of 64 keys in 0.3 us of an SM's time where the SMs are full (0.4 where
// a warp or two are on each), and splits long sequences; the tcgen05 one 0.8 us for 128 rows, but not less than 1.3 us a tile in turn.  Measured, this
// one and tcgen05, us: head_dim 64, 2048 items, S 320: 43 rows 61 and 63, 64 rows 76 and 66, 128 rows 156 and 81; 512 items, S 1088: 32 rows 42.4
// and 42.9, 43 rows 52 and 44, 200 rows 191 and 97; 128 items 43 rows 22.4 and 22.2, 64 rows 27.6 and 22.4; 32 items 128 rows 21.5 and 21.6;
// 24 items, S 5000, 200 rows 58 and 81; head_dim 80, 2048 items, S 320, 43 rows 66 and 70; head_dim 128, 512 items, S 1088, 32 rows 74 and 91, 64
// rows 122 and 94.  The choice costs 3 % at most at 20 measured shapes.
bool attention_quantized_tc_wins(int R, int S, int dh, int items) {
  if (R <= 16) return false;
  const double sms = device_sm_count(), tiles = (S + 63) / 64, warp_tiles = (double)items * ((R + 15) / 16) * tiles / sms, units = (double)items * ((R + 127) / 128);
  const double mma = 5.0 + warp_tiles * ((dh == 64 ? 0.3 : (dh == 80 ? 0.325 : 0.65)) + (warp_tiles < 100 ? 0.1 : 0.0));
  const double a_tile = dh == 64 ? 0.8 : (dh == 80 ? 0.88 : 1.55), a_unit = dh == 128 ? 3.5 : 0.7, busy = units / sms * (tiles * a_tile + a_unit);
  return 4.0 + (busy > tiles * 1.3 ? busy : tiles * 1.3) < mma;
}

QuantizedSplit attention_quantized_plan(int R, int S, int dh, int items) {
  const int sms = device_sm_count(), eights = (R + 7) / 8;
  QuantizedSplit s;
  const int warps = (eights + 1) / 2;                      // along the rows
  s.nb = (eights + warps - 1) / warps;
  s.n_rb = (warps + 2) / 3;
  s.nr = (warps + s.n_rb - 1) / s.n_rb;
  const int kt = tile_keys(dh), tiles = (S + kt - 1) / kt;
  const long blocks = (long)items * s.n_rb;
  s.cs = 1;
  while (s.cs < 8 && blocks * s.cs < 2 * sms && tiles > 4 * s.cs) s.cs *= 2;
  const int per = (tiles + s.cs - 1) / s.cs;
  // (a stage is filled again one tile late where other warps read it, too: three of them)
  const int stage = 2 * kt * dh + 2 * kt * 4, least = s.nr > 1 ? 3 : 2;
  const long want = (6L * sms + blocks * s.cs - 1) / (blocks * s.cs);   // six groups on an SM, if the tiles go round
  s.nk = 8 / s.nr < per ? 8 / s.nr : per;
  if (s.nk > want) s.nk = (int)want;
  while (s.nk > 1 && s.nk * least * stage > 150 * 1024) --s.nk;
  const int mine = (per + s.nk - 1) / s.nk, fit = kMaxStages / s.nk;
  s.nst = mine < least ? mine : least;
  while (s.nst < mine && s.nst < fit && s.nk * (s.nst + 1) * stage <= 40 * 1024) ++s.nst;
  return s;
}

// Shared memory of a CTA: the rings, and the partial results where there are several of a row.
size_t attention_quantized_smem(int dh, const QuantizedSplit& s) {
  const int parts = s.cs * s.nk, own = (s.nr * 8 * s.nb + s.cs - 1) / s.cs, kt = tile_keys(dh);
  return 1024 + (size_t)s.nk * s.nst * (2 * kt * dh + 2 * kt * 4) + (parts > 1 ? (size_t)parts * own * (dh + 4) * 4 : 0);
}

cudaError_t launch_attention_quantized(const void* q, int ld_q, int n, int heads, const QuantizedKv& c, const int32_t* kv_len, void* o, bool o_bf16,
                                       int* status, cudaStream_t st) {
  const QuantizedSplit s = attention_quantized_plan(n * (heads / c.H), c.S, c.dh, c.B * c.H);
#define MARCHE_QA(DH_, NB_) \
  case DH_ * 8 + NB_:                                      \
    return o_bf16 ? launch<DH_, NB_, false>(q, ld_q, n, heads, c, kv_len, o, true, s, status, st) : launch<DH_, NB_, true>(q, ld_q, n, heads, c, kv_len, o, false, s, status, st);
  switch (c.dh * 8 + s.nb) {
    MARCHE_QA(64, 1) MARCHE_QA(64, 2) MARCHE_QA(80, 1) MARCHE_QA(80, 2) MARCHE_QA(128, 1) MARCHE_QA(128, 2)
  }
#undef MARCHE_QA
  return cudaErrorInvalidValue;
}

}  // namespace marche
