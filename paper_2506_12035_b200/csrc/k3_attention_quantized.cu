// K3 over a cache held in 8 bits: attention of n query rows per sample over the sample's keys, values code * scale.
//
// o = softmax(q K^T / sqrt(dh)) V with K[s] = ks[s] ck[s], V[s] = vs[s] cv[s], codes c in -127 .. 127 and one scale per key and head.
// The scales are kept out of the products: the logit of a key is ks[s] (q . ck[s]), and vs[s] goes into the weight, so the tensor
// cores multiply the codes themselves, which are exact in fp16.  q (bf16) is exact in fp16 after its row's power of two is taken off; what
// is rounded is the weight: p vs / 2^e to fp16 (11 bits), where 2^e bounds the largest value scale met so far and the whole is
// lifted by 2^14, so that a weight 2^-28 of the largest possible keeps all its bits.  Maxima, sums and accumulators are fp32, and the running
// exponent e moves with the running maximum (one factor for both).
// Query heads that share a cached head are rows of one item: row r is token r / G, head r % G of the group.
//
// mma.sync m16n8k16; codes become fp16 under the exponent of 1024 (a byte permute and a packed subtraction for two).  K: a dot product
// does not mind the order of its terms, so a lane's 16 consecutive bytes of a key serve as its pairs of four k16 steps, no transposition and
// one shared-memory load; V: ldmatrix.trans on pairs of bytes, whose even and odd bytes are two tiles of eight columns.
// nr warps take 16 or 32 rows each; nk groups of them take the tiles of 64 keys (K, V and both scales, by TMA) in turn, each group with a
// ring of nst stages that its first warp fills (a producer warp of its own would be the ninth: three warps on one quarter of the SM's
// registers, 168 for each); a cluster of cs CTAs splits a long sequence.  (CTA, group) pairs merge in rank order in the CTA that owns
// the row: bit-reproducible.  A sample without keys gives zeros.
#include <cuda.h>

#include "attention_common.cuh"
#include "kernels.h"
#include "launch_pdl.h"
#include "sm100_ptx.cuh"
#include "tma_host.h"

namespace marche {

namespace {

using att::ex2_approx;
using att::ldsm_x4_trans;

constexpr int KT = 64;                     // keys per tile
constexpr int kMaxStages = 16;             // of a CTA
constexpr int kThreadsMax = 256;
enum { ST_ATTENTION_QUANTIZED = 0x25 };

template <int DH> struct Cfg {
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
// First of the four values that lane t of a quad holds in k16 step s (two for the step's lower, two for its upper half).
template <int DH> MARCHE_DEVINL int value_of(int s, int t) { return DH == 80 ? 16 * s + 4 * t : 16 * (4 * (s / 4) + t) + 4 * (s % 4); }

MARCHE_DEVINL uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
MARCHE_DEVINL uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
MARCHE_DEVINL float2 lds_f2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a));
  return v;
}
MARCHE_DEVINL void ldsm_x2_trans(uint32_t addr, uint32_t& r0, uint32_t& r1) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(r0), "=r"(r1) : "r"(addr));
}
MARCHE_DEVINL void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two of the four signed bytes of a word (SEL picks them and puts 0x64 above each) as fp16: 1024 + (byte + 128) - 1152.
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
MARCHE_DEVINL void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
MARCHE_DEVINL float pow2(int biased_exponent) { return __int_as_float(biased_exponent << 23); }

// Grid: B * H * n_rb * cs CTAs, the cs of a cluster next to one another.
template <int DH, int MT>
__global__ void __launch_bounds__(kThreadsMax)
attention_quantized_kernel(const __grid_constant__ CUtensorMap tmap, const bf16* __restrict__ q, int ld_q, int n, int heads, int H, int G, int B, int S,
                           int pad, const float* __restrict__ scales, const int32_t* __restrict__ kv_len, uint16_t* __restrict__ o, int o_bf16,
                           const QuantizedSplit sp, int* __restrict__ status) {
  using C = Cfg<DH>;
  constexpr int RPW = 16 * MT;                             // rows of a warp
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t scale_base = base + (uint32_t)(sp.nk * sp.nst * C::STAGE), recv = scale_base + (uint32_t)(sp.nk * sp.nst * C::SCALES);
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
  }
  __syncwarp();
  if (sp.cs > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  __syncthreads();
  pdl_sync();

  int len = S;
  if (kv_len) len = min(max(kv_len[b], 0), S);
  const int tiles = (len + KT - 1) / KT;
  const int kt0 = (int)((long long)rank * tiles / sp.cs), n_tiles = (int)((long long)(rank + 1) * tiles / sp.cs) - kt0;
  bool ok = true;
  float m_run[MT][2], l_run[MT][2], c_row[MT][2], oacc[MT][C::CHUNKS][2][4];
  int e_run = 14;                                          // biased exponent above every value scale so far (14: the lowest whose factors exist)
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    m_run[m][0] = m_run[m][1] = -INFINITY;
    l_run[m][0] = l_run[m][1] = 0.f;
#pragma unroll
    for (int c = 0; c < C::CHUNKS; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) oacc[m][c][e >> 2][e & 3] = 0.f;
  }
  const bool active = row_w < R;
  const int mine = (n_tiles - wk + sp.nk - 1) / sp.nk, stage0 = wk * sp.nst;   // tiles wk, wk + nk, .. of the CTA's; the group's first stage
  // Tile u of the group into its stage.
  auto load = [&](int u) {
    const int s = stage0 + u % sp.nst, kt = kt0 + wk + u * sp.nk;
    const uint32_t bar = full0 + 8u * s, dst = base + (uint32_t)(s * C::STAGE), dst_s = scale_base + (uint32_t)(s * C::SCALES);
    ptx::mbar_expect_tx(bar, C::STAGE + C::SCALES);
    ptx::tma_load_3d(dst, &tmap, h * DH, kt * KT, b, bar);
    ptx::tma_load_3d(dst + C::TILE, &tmap, h * DH, kt * KT, B + b, bar);
    bulk_load(dst_s, scales + ((size_t)b * H + h) * pad + (size_t)kt * KT, KT * 4, bar);
    bulk_load(dst_s + KT * 4, scales + ((size_t)(B + b) * H + h) * pad + (size_t)kt * KT, KT * 4, bar);
  };
  int issued = 0;                                          // by lane 0 of the group's first warp
  if (wr == 0 && lane == 0)
    for (; issued < mine && issued < sp.nst; ++issued) load(issued);
  __syncwarp();
  {
    uint32_t qf[MT][C::STEPS][4];
    if (active) {
      const float scale_log2 = rsqrtf((float)DH) * 1.4426950408889634f;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = row_w + 16 * m + 8 * r + g, token = row / G;
          const bf16* src = q + ((size_t)b * n + token) * ld_q + (h * G + row - token * G) * DH;
          uint2 x[C::STEPS];
          uint32_t top = 0;
#pragma unroll
          for (int s = 0; s < C::STEPS; ++s) {
            x[s] = row < R ? *reinterpret_cast<const uint2*>(src + value_of<DH>(s, t)) : make_uint2(0, 0);
            top = max(max(top, max(x[s].x & 0x7fffu, (x[s].x >> 16) & 0x7fffu)), max(x[s].y & 0x7fffu, (x[s].y >> 16) & 0x7fffu));
          }
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          // the row divided by its largest power of two: exact in fp16 (2^-24 of the largest value and less goes), and no overflow
          const int e = min(max((int)(top >> 7), 1), 253);
          const float f = pow2(254 - e);
          c_row[m][r] = scale_log2 * pow2(e);
#pragma unroll
          for (int s = 0; s < C::STEPS; ++s) {
            const float2 lo = unpack_bf16x2(x[s].x), hi = unpack_bf16x2(x[s].y);
            qf[m][s][r] = pack_weights(lo.x * f, lo.y * f);
            qf[m][s][2 + r] = pack_weights(hi.x * f, hi.y * f);
          }
        }
    }
    int turn = 0, phase = 0;                               // stage of tile u in the group's ring, its fill's parity
    for (int u = 0; u < mine; ++u) {
      const int s = stage0 + turn;
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(full0 + 8u * s, (uint32_t)phase, abort_flag))) { ok = false; break; }
      if (active) {
        const uint32_t k_tile = base + (uint32_t)(s * C::STAGE), v_tile = k_tile + C::TILE;
        const uint32_t ks = scale_base + (uint32_t)(s * C::SCALES), vs = ks + KT * 4;
        const int left = len - (kt0 + wk + u * sp.nk) * KT;             // keys of this tile that count
        float sacc[MT][8][4];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t w[C::STEPS];
          const int key = 8 * j + g;
          if (DH == 80) {
#pragma unroll
            for (int k = 0; k < C::STEPS; ++k) w[k] = lds32(k_tile + (uint32_t)(key * DH + 16 * k + 4 * t));
          } else {
#pragma unroll
            for (int k = 0; k < C::STEPS / 4; ++k) {
              const uint4 v = lds128(k_tile + piece<DH>(key, 4 * k + t));
              w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
            }
          }
#pragma unroll
          for (int m = 0; m < MT; ++m) sacc[m][j][0] = sacc[m][j][1] = sacc[m][j][2] = sacc[m][j][3] = 0.f;
#pragma unroll
          for (int k = 0; k < C::STEPS; ++k) {
            const uint32_t u = w[k] ^ 0x80808080u, b0 = two_of<0x4140>(u), b1 = two_of<0x4342>(u);
#pragma unroll
            for (int m = 0; m < MT; ++m) mma_f16(sacc[m][j], qf[m][k], b0, b1);
          }
          const float2 f = lds_f2(ks + (uint32_t)(8 * j + 2 * t) * 4u);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            sacc[m][j][0] *= f.x; sacc[m][j][1] *= f.y;
            sacc[m][j][2] *= f.x; sacc[m][j][3] *= f.y;
          }
        }
        if (left < KT) {
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (8 * j + 2 * t + (e & 1) >= left) sacc[m][j][e] = -INFINITY;
        }
        // largest value scale of the tile (they are not negative: they order as integers; NaN counts as the largest number)
        const float2 mine = lds_f2(vs + (uint32_t)lane * 8u);
        uint32_t top = max(2 * lane < left ? __float_as_uint(mine.x) : 0u, 2 * lane + 1 < left ? __float_as_uint(mine.y) : 0u);
        top = __reduce_max_sync(0xffffffffu, top);
        const int e_new = max(e_run, min((int)(top >> 23), 254));
        const float lift = pow2(267 - e_new);              // 2^14 over the power of two above the scale
        float step = e_new == e_run ? 1.f : (e_new - e_run > 120 ? 0.f : pow2(127 - (e_new - e_run)));
        e_run = e_new;
        float neg[MT][2];
        bool moved = step != 1.f;
        float corr[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) mx = fmaxf(mx, fmaxf(sacc[m][j][2 * r], sacc[m][j][2 * r + 1]));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            const float m_new = fmaxf(m_run[m][r], mx), ref = m_new == -INFINITY ? 0.f : m_new;
            corr[m][r] = ex2_approx((m_run[m][r] - ref) * c_row[m][r]);
            moved = moved || m_new != m_run[m][r];
            m_run[m][r] = m_new;
            neg[m][r] = -ref * c_row[m][r];
          }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            l_run[m][0] *= corr[m][0];
            l_run[m][1] *= corr[m][1];
            const float c0 = corr[m][0] * step, c1 = corr[m][1] * step;
#pragma unroll
            for (int c = 0; c < C::CHUNKS; ++c)
#pragma unroll
              for (int p = 0; p < 2; ++p) {
                oacc[m][c][p][0] *= c0; oacc[m][c][p][1] *= c0;
                oacc[m][c][p][2] *= c1; oacc[m][c][p][3] *= c1;
              }
          }
        }
#pragma unroll
        for (int k2 = 0; k2 < KT / 16; ++k2) {
          uint32_t pf[MT][4];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int j = 2 * k2 + hf;
            float2 f = lds_f2(vs + (uint32_t)(8 * j + 2 * t) * 4u);
            f.x = 8 * j + 2 * t < left ? f.x * lift : 0.f;
            f.y = 8 * j + 2 * t + 1 < left ? f.y * lift : 0.f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const float p0 = ex2_approx(fmaf(sacc[m][j][2 * r], c_row[m][r], neg[m][r]));
                const float p1 = ex2_approx(fmaf(sacc[m][j][2 * r + 1], c_row[m][r], neg[m][r]));
                l_run[m][r] += p0 + p1;
                pf[m][2 * hf + r] = pack_weights(p0 * f.x, p1 * f.y);
              }
          }
          const int key = 16 * k2 + 8 * ((lane >> 3) & 1) + (lane & 7);
#pragma unroll
          for (int c = 0; c < C::CHUNKS; c += 2) {
            uint32_t w[4];
            if (c + 1 < C::CHUNKS) ldsm_x4_trans(v_tile + piece<DH>(key, c + (lane >> 4)), w[0], w[1], w[2], w[3]);
            else ldsm_x2_trans(v_tile + piece<DH>(key, c), w[0], w[1]);
#pragma unroll
            for (int d = 0; d < 2 && c + d < C::CHUNKS; ++d) {
              const uint32_t lo = w[2 * d] ^ 0x80808080u, hi = w[2 * d + 1] ^ 0x80808080u;
              const uint32_t e0 = two_of<0x4240>(lo), e1 = two_of<0x4240>(hi), o0 = two_of<0x4341>(lo), o1 = two_of<0x4341>(hi);
#pragma unroll
              for (int m = 0; m < MT; ++m) {
                mma_f16(oacc[m][c + d][0], pf[m], e0, e1);
                mma_f16(oacc[m][c + d][1], pf[m], o0, o1);
              }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) {
        ptx::mbar_arrive(empty0 + 8u * s);
        // The stage of the tile before this one (of this one where no other warp reads it) is free, or nearly: its next tile.
        const int from = sp.nr == 1 ? u : u - 1;
        if (wr == 0 && from >= 0 && from + sp.nst < mine) {
          const int f = stage0 + from % sp.nst;
          if (ptx::mbar_wait(empty0 + 8u * f, (uint32_t)(from / sp.nst) & 1u, abort_flag)) { load(from + sp.nst); ++issued; }
          else ok = false;
        }
      }
      ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
      if (!ok) break;
      if (++turn == sp.nst) { turn = 0; phase ^= 1; }
    }
    if (!ok && wr == 0 && lane == 0) {                     // let copies already issued land before the CTA's shared memory is released
      for (int u = issued > sp.nst ? issued - sp.nst : 0; u < issued; ++u)
        ptx::mbar_wait(full0 + 8u * (stage0 + u % sp.nst), (uint32_t)(u / sp.nst) & 1u, abort_flag + 1, 20000000LL);
    }
    if (!ok && lane == 0) *(volatile int*)status = ST_ATTENTION_QUANTIZED;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l_run[m][r] += __shfl_xor_sync(0xffffffffu, l_run[m][r], 1);
        l_run[m][r] += __shfl_xor_sync(0xffffffffu, l_run[m][r], 2);
        if (!active) m_run[m][r] = -INFINITY;
      }
  }
  const float unlift = pow2(e_run - 13);
  auto row_out = [&](int row) {                            // of the item's rows
    const int token = row / G;
    return o + (((size_t)b * n + token) * heads + h * G + row - token * G) * DH;
  };
  auto inverse = [](float l) { return l > 0.f ? 1.0f / l : l; };   // no key: zeros; NaN stays
  auto store = [&](uint16_t* to, float4 v, float f) {
    uint2 u;
    u.x = pack_a16x2(v.x * f, v.y * f, o_bf16 != 0);
    u.y = pack_a16x2(v.z * f, v.w * f, o_bf16 != 0);
    *reinterpret_cast<uint2*>(to) = u;
  };
  const int n_parts = sp.cs * sp.nk;
  if (n_parts == 1) {
    if (active && ok) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = row_w + 16 * m + 8 * r + g;
          if (row < R) {
            uint16_t* to = row_out(row) + 4 * t;
            const float f = inverse(l_run[m][r]) * unlift;
#pragma unroll
            for (int c = 0; c < C::CHUNKS; ++c)
              store(to + 16 * c, make_float4(oacc[m][c][0][2 * r], oacc[m][c][1][2 * r], oacc[m][c][0][2 * r + 1], oacc[m][c][1][2 * r + 1]), f);
          }
        }
    }
    return;
  }
  // ---- partial results to the owners of the rows, then the merge
  const int rows_cta = sp.nr * RPW, own = (rows_cta + sp.cs - 1) / sp.cs;
  if (sp.cs > 1) {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");                  // every CTA of the cluster has started
    if (!ok) ptx::cluster_raise(ptx::smem_u32(abort_flags), sp.cs);                      // nobody merges what is missing
  }
  if (active && ok) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int in = wr * RPW + 16 * m + 8 * r + g, owner = in / own;
        if (row_block + in < R) {
          uint32_t dst = recv + 4u * (uint32_t)(((rank * sp.nk + wk) * own + in - owner * own) * C::ROW);
          if (sp.cs > 1) dst = ptx::mapa(dst, (uint32_t)owner);
#pragma unroll
          for (int c = 0; c < C::CHUNKS; ++c)
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst + 4u * (16 * c + 4 * t)), "f"(oacc[m][c][0][2 * r] * unlift),
                         "f"(oacc[m][c][1][2 * r] * unlift), "f"(oacc[m][c][0][2 * r + 1] * unlift), "f"(oacc[m][c][1][2 * r + 1] * unlift) : "memory");
          if (t == 0)                                      // the maximum in the exponent's own units
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(dst + 4u * DH), "f"(m_run[m][r] * c_row[m][r]), "f"(l_run[m][r]) : "memory");
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
      const float w = ex2_approx(p[s * stride + DH] - mx);
      const float4 v = *reinterpret_cast<const float4*>(p + s * stride + c);
      l = fmaf(w, p[s * stride + DH + 1], l);
      acc.x = fmaf(w, v.x, acc.x); acc.y = fmaf(w, v.y, acc.y);
      acc.z = fmaf(w, v.z, acc.z); acc.w = fmaf(w, v.w, acc.w);
    }
    store(row_out(row) + c, acc, inverse(l));
  }
}

template <int DH, int MT>
cudaError_t launch(const CUtensorMap& tm, const void* q, int ld_q, int n, int heads, const QuantizedKv& c, const int32_t* kv_len, void* o, bool o_bf16,
                   const QuantizedSplit& s, int* status, cudaStream_t st) {
  const size_t smem = attention_quantized_smem(DH, s);
  if (smem > 226 * 1024) return cudaErrorInvalidValue;
  static size_t smem_set[kMaxDevices] = {};
  cudaError_t e = ensure_dynamic_smem(attention_quantized_kernel<DH, MT>, smem, smem_set);
  if (e != cudaSuccess) return e;
  const int G = heads / c.H;
  return launch_pdl_cluster(attention_quantized_kernel<DH, MT>, dim3((unsigned)((long)c.B * c.H * s.n_rb * s.cs)), dim3(s.nr * s.nk * 32), smem, s.cs, st, tm,
                            (const bf16*)q, ld_q, n, heads, c.H, G, c.B, c.S, c.pad, (const float*)c.scales, kv_len, (uint16_t*)o, o_bf16 ? 1 : 0, s, status);
}

}  // namespace

QuantizedSplit attention_quantized_plan(int R, int S, int dh, int items) {
  const int tiles = (S + KT - 1) / KT, sms = device_sm_count();
  QuantizedSplit s;
  s.mt = R > 16 && dh != 128 ? 2 : 1;
  const int rpw = 16 * s.mt, groups = (R + rpw - 1) / rpw;
  s.n_rb = (groups + 3) / 4;
  s.nr = (groups + s.n_rb - 1) / s.n_rb;
  const long blocks = (long)items * s.n_rb;
  s.cs = 1;
  while (s.cs < 8 && blocks * s.cs < 2 * sms && tiles > 4 * s.cs) s.cs *= 2;
  const int per = (tiles + s.cs - 1) / s.cs;
  // (a stage is filled again one tile late where other warps read it, too: three of them)
  const int stage = 2 * KT * dh + 2 * KT * 4, least = s.nr > 1 ? 3 : 2;
  s.nk = 1;
  while (2 * s.nk * s.nr <= 8 && 2 * s.nk <= per && 2 * s.nk * least * stage <= 150 * 1024 && blocks * s.cs * s.nk < 6 * sms) s.nk *= 2;
  const int mine = (per + s.nk - 1) / s.nk, most = kMaxStages / s.nk;
  s.nst = mine < least ? mine : least;
  while (s.nst < mine && s.nst < most && s.nk * (s.nst + 1) * stage <= 40 * 1024) ++s.nst;
  return s;
}

// Shared memory of a CTA: the rings, and the partial results where there are several of a row.
size_t attention_quantized_smem(int dh, const QuantizedSplit& s) {
  const int parts = s.cs * s.nk, own = (s.nr * 16 * s.mt + s.cs - 1) / s.cs;
  return 1024 + (size_t)s.nk * s.nst * (2 * KT * dh + 2 * KT * 4) + (parts > 1 ? (size_t)parts * own * (dh + 4) * 4 : 0);
}

cudaError_t launch_attention_quantized(const void* q, int ld_q, int n, int heads, const QuantizedKv& c, const int32_t* kv_len, void* o, bool o_bf16,
                                       int* status, cudaStream_t st) {
  CUtensorMap tm;
  EncodeTiledFn fn = tma_encode_fn();
  const cuuint64_t D = (cuuint64_t)c.H * c.dh, dims[3] = {D, (cuuint64_t)c.S, (cuuint64_t)2 * c.B}, strides[2] = {D, D * c.S};
  const cuuint32_t box[3] = {(cuuint32_t)c.dh, KT, 1}, unit[3] = {1, 1, 1};
  const CUtensorMapSwizzle sw = c.dh == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : c.dh == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE;
  if (!fn || fn(&tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, c.codes, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  const QuantizedSplit s = attention_quantized_plan(n * (heads / c.H), c.S, c.dh, c.B * c.H);
  switch (c.dh) {
    case 64:
      return s.mt == 2 ? launch<64, 2>(tm, q, ld_q, n, heads, c, kv_len, o, o_bf16, s, status, st) : launch<64, 1>(tm, q, ld_q, n, heads, c, kv_len, o, o_bf16, s, status, st);
    case 80:
      return s.mt == 2 ? launch<80, 2>(tm, q, ld_q, n, heads, c, kv_len, o, o_bf16, s, status, st) : launch<80, 1>(tm, q, ld_q, n, heads, c, kv_len, o, o_bf16, s, status, st);
    case 128: return launch<128, 1>(tm, q, ld_q, n, heads, c, kv_len, o, o_bf16, s, status, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace marche
