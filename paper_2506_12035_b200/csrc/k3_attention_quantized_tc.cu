// K3 over a cache held in 8 bits, many query rows: the products on the 5th-generation tensor cores, one conversion of the codes for 128 rows.
//
// The mathematics is that of the mma.sync kernel (k3_attention_quantized.cu): codes are multiplied as exact fp16 numbers, a key's scale
// multiplies its logits, its value scale its weight before that is rounded to fp16.  Here weights are lifted by 2^7 only, since the reference lags by up
// to 2^8, and there is no second operand for what the rounding left off (it would take the columns and the instructions of a second P V): the error of
// fp16 outputs is 1.4 times the output's own rounding, where the mma.sync kernel's is that rounding alone.  What that kernel is bound by from some
// 32 rows on is its own instructions (1000 to 1500 of a warp for 64 keys x 32 rows, a third of them conversions that every warp repeats).  Here
// a warp pair converts a tile once for a unit of 128 rows, and a thread owns a row of the softmax.
// Persistent CTAs, one per SM; unit = 128 rows (tokens x query heads of a group) of one (sample, cached head) against all of its
// keys; NS independent streams per CTA take the units, each with (warps)
//   4  softmax, one thread per row: logits from tensor memory times the keys' scales less the running reference (it moves only when a tile
//      exceeds it by 2^8, so that one packed FMA per pair is all before the exponential), weights times value scales packed to fp16 and
//      written back to tensor memory as the A operand of P V
//   2  converters: the unit's query rows (fp16, divided by a power of two), then per tile K and V from bytes to swizzled
//      fp16 operand tiles (two of each), the scales, and the running exponent above all value scales, which the weights are relative
//      to.  (Four of them, or a third stream, take registers from the softmax: 484 and 492 us where two streams of two took 424.)  Every 128 rows
//      of an item convert its tiles again.
//   1  TMA producer: codes and scales of the tiles into a staging ring
//   1  issues tcgen05.mma: S = Q K^T (M128 x N64), O += P V (V as an MN-major operand); S of the next tile runs under the softmax of this one
// What bounds it: the chain of a stream's tile, softmax (of it the exponentials, 16 per clock and SM, 512 cycles for a tile of 64 x 128), conversion and products
// in turn, with two streams to fill the gaps (46 % of the issue slots).  32 samples x 1088 rows over 1088 keys, 16 heads of 64: 405 us, of which the
// exponentials alone 140 and the products 94.  Where rows need powers of two of their own 454, where value scales lie far apart 630.
// All waits are bounded and report through the status word.
#include <cuda.h>

#include "attention_quantized.cuh"
#include "kernels.h"
#include "launch_pdl.h"
#include "sm100_ptx.cuh"
#include "tma_host.h"

namespace marche {

namespace {

using attq::pow2;

constexpr int QT = 128;                    // rows of a unit (= TMEM lanes)
constexpr int KT = 64;                     // keys per tile
constexpr int NSTG = 3, NB2 = 2, NSC = 4;  // staging slots; operand tiles of K and of V; slots of scales (a converter is at most three tiles ahead of a softmax)
enum { ST_ATT_QUANTIZED_TC = 0x53 };
// barriers of one stream
enum { B_STG_FULL = 0, B_STG_EMPTY = B_STG_FULL + NSTG, B_K_FULL = B_STG_EMPTY + NSTG, B_K_EMPTY = B_K_FULL + NB2, B_V_FULL = B_K_EMPTY + NB2,
       B_V_EMPTY = B_V_FULL + NB2, B_SC_FULL = B_V_EMPTY + NB2, B_Q_FULL = B_SC_FULL + NSC, B_TOP, B_Q_EMPTY, B_S_FULL, B_S_FREE, B_P_FULL, B_O_FULL, NB };
constexpr int kScaleSlot = 2 * KT + 4;     // words: ks in units of log2 [64], vs lifted [64], step, unlift, flags, by how much a wide sample's unit rises
enum { F_BUFFER = 1, F_OWN = 2, F_WIDE = 4 };   // which buffer of the rows' own factors, where they have some; value scales far apart
constexpr int kSpread = 10;                // a row's largest product is at least 2^(7 - 1 - 10) before its sample counts as wide

template <int DH, int NS> struct Cfg {
  static constexpr int NC = 2;                             // converters of a stream
  static constexpr int WARPS = 6 + NC, THREADS = NS * WARPS * 32;
  static constexpr int W_CONV = 4 * NS, W_PROD = (4 + NC) * NS, W_MMA = (5 + NC) * NS;   // roles by warp: softmax 0 .. 4 NS - 1, converters, producers, issuers
  static constexpr int BLOCKS = DH / 64, TAIL = DH % 64;   // columns in blocks of 64 (128-byte rows) and a tail of 16 (32-byte rows)
  static constexpr int T_BLOCK = KT * 128, T_BYTES = KT * DH * 2, Q_BLOCK = QT * 128, Q_BYTES = QT * DH * 2;
  static constexpr int STG_BYTES = 2 * KT * DH;
  static constexpr uint32_t COL_P = KT, COL_O = KT + KT / 2, COL_STREAM = KT + KT / 2 + DH;
  static constexpr int TMEM_COLS = NS * COL_STREAM <= 256 ? 256 : 512;
  // shared memory (from a 1024-byte aligned base), [stream][slot]
  static constexpr int OFF_Q = 0, OFF_K = OFF_Q + NS * Q_BYTES, OFF_V = OFF_K + NS * NB2 * T_BYTES, OFF_STG = OFF_V + NS * NB2 * T_BYTES;
  static constexpr int OFF_RAW = OFF_STG + NS * NSTG * STG_BYTES;          // scales as they come: [stream][slot][2 KT]
  static constexpr int OFF_SC = OFF_RAW + NS * NSTG * 2 * KT * 4, OFF_ROW = OFF_SC + NS * NSC * kScaleSlot * 4;
  static constexpr int OFF_FACTOR = OFF_ROW + NS * 32;                     // largest and smallest value of each converter's rows
  static constexpr int OFF_BAR = OFF_FACTOR + NS * 2 * QT * 4;             // the rows' own powers of two: [stream][units in turn][row]
  static constexpr int OFF_MISC = OFF_BAR + 8 * NS * NB, SMEM_BYTES = OFF_MISC + 32 + 1024;
  static_assert(NS * COL_STREAM <= TMEM_COLS && SMEM_BYTES <= 227 * 1024 && OFF_BAR % 8 == 0 && OFF_SC % 16 == 0 && (kScaleSlot * 4) % 16 == 0, "budgets of a CTA");
  static_assert(T_BYTES % 1024 == 0 && Q_BYTES % 1024 == 0 && STG_BYTES % 1024 == 0 && OFF_RAW % 16 == 0, "alignment of operand tiles");
};

MARCHE_DEVINL constexpr uint32_t idesc_f16(int M, int N, bool b_mn_major) {
  return (1u << 4) | (b_mn_major ? (1u << 16) : 0u) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// MN-major operand tile of [k rows][64 elements = 128 bytes] under the 128-byte swizzle: 8 k-rows form a 1024-byte atom.
MARCHE_DEVINL uint64_t smem_desc_mn_sw128(uint32_t addr) {
  const uint32_t lo = ((addr & 0x3FFFFu) >> 4) | ((1024u >> 4) << 16);
  const uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);
  return ((uint64_t)hi << 32) | lo;
}
// The same for tiles of 32-byte rows (16 elements) under the 32-byte swizzle: 8 rows form a 256-byte atom.
MARCHE_DEVINL uint64_t smem_desc_sw32(uint32_t addr) {
  const uint32_t lo = ((addr & 0x3FFFFu) >> 4) | ((256u >> 4) << 16);
  const uint32_t hi = (256u >> 4) | (1u << 14) | (6u << 29);
  return ((uint64_t)hi << 32) | lo;
}
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
// 16 columns of a row in tensor memory times f.
MARCHE_DEVINL void scale_in_place(uint32_t taddr, float f) {
  uint32_t v[16];
  tmem_ld_32x16(taddr, v);
  ptx::tmem_ld_wait(v);
#pragma unroll
  for (int c = 0; c < 16; ++c) v[c] = __float_as_uint(__uint_as_float(v[c]) * f);
  tmem_st_32x16(taddr, v);
}
MARCHE_DEVINL float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
MARCHE_DEVINL float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
MARCHE_DEVINL uint32_t pack_weights(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two neighbouring bytes of a word of codes + 128 as fp16: 1024 + (code + 128) - 1152.
template <uint32_t SEL> MARCHE_DEVINL uint32_t two_of(uint32_t biased) {
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(__byte_perm(biased, 0x64646464u, SEL)), "r"(0x64806480u));
  return r;
}
MARCHE_DEVINL void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Byte offset of 16-byte piece c of key r in a staging tile, as TMA wrote it (64- and 128-byte rows swizzled, 80-byte rows as they are): eight
// consecutive keys' pieces lie on different banks.
template <int DH> MARCHE_DEVINL uint32_t piece(int r, int c) {
  if (DH == 64) return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
  if (DH == 128) return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4));
  return (uint32_t)(r * DH + (c << 4));
}
// Byte offset of 16-byte piece c (8 fp16 values) of row r in an operand tile of `rows` rows: blocks of 64 columns under the 128-byte swizzle, a
// tail of 16 under the 32-byte swizzle.
template <int DH> MARCHE_DEVINL uint32_t operand_off(int rows, int r, int c) {
  if (c < DH / 64 * 8) return (uint32_t)((c >> 3) * rows * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
  return (uint32_t)(DH / 64 * rows * 128 + r * 32 + (((c & 1) ^ ((r >> 2) & 1)) << 4));
}

// Units are dealt to the CTAs in turn, stream j of a CTA takes its units j, j + NS, ..; where there is more than one turn, the places rotate, so that
// the short last tiles of items do not all fall to the same CTAs (the rule of the 16-bit kernel, attention_tc_rotation).
struct Deal {
  int units, grid, rotate, rotate_turn;
  template <int NS> MARCHE_DEVINL int place(int k) const { return ((int)blockIdx.x + k * rotate + k / NS * rotate_turn) % grid; }
};
struct Unit { int b, h, start, row0, n_kv, len; };         // first row; the row on lane 0; key tiles and keys of the sample
struct Shape { int n, G, R, H, B, S, heads, n_qt; };
template <int NS>
MARCHE_DEVINL Unit unit_of(int j, int u, const Deal& deal, const Shape& sh, const int32_t* kv_len) {
  const int k = NS * u + j, i = k * deal.grid + deal.place<NS>(k);
  const int item = i / sh.n_qt, qt = i - item * sh.n_qt;
  Unit r;
  r.b = item / sh.H;
  r.h = item - r.b * sh.H;
  r.start = qt * QT;
  // a tile that needs one, two or three of the four lane quarters starts at another quarter in another stream
  const int quarters = sh.R - r.start >= QT ? 4 : (sh.R - r.start + 31) / 32;
  r.row0 = r.start - 32 * (quarters == 1 ? j : (quarters == 4 ? 0 : (j & 1) * (4 - quarters)));
  r.len = kv_len ? min(max(kv_len[r.b], 0), sh.S) : sh.S;
  r.n_kv = (r.len + KT - 1) / KT;
  return r;
}

template <int DH, int NS>
__global__ void __launch_bounds__(Cfg<DH, NS>::THREADS, 1)
attention_quantized_tc_kernel(const __grid_constant__ CUtensorMap tmap, const bf16* __restrict__ q, int ld_q, const float* __restrict__ scales, int pad,
                              const int32_t* __restrict__ kv_len, uint16_t* __restrict__ o, int o_bf16, const Shape sh, const Deal deal, int* __restrict__ status) {
  using C = Cfg<DH, NS>;
  constexpr int NC = C::NC;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  auto bar = [&](int j, int i) { return base + C::OFF_BAR + 8u * (uint32_t)(j * NB + i); };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + C::OFF_MISC + 8);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int units_cta = deal.units / deal.grid + (deal.place<NS>(deal.units / deal.grid) < deal.units % deal.grid ? 1 : 0);

  if (threadIdx.x == 0) {
    for (int j = 0; j < NS; ++j)
      for (int i = 0; i < NB; ++i)
        ptx::mbar_init(bar(j, i), i == B_P_FULL || i == B_S_FREE ? 4 : (i >= B_STG_EMPTY && i < B_K_FULL) || i == B_Q_FULL || i == B_TOP ? C::NC :
                                  ((i >= B_K_FULL && i < B_K_EMPTY) || (i >= B_V_FULL && i < B_V_EMPTY) || (i >= B_SC_FULL && i < B_Q_FULL) ? 2 : 1));
    abort_flag[0] = 0;
    abort_flag[1] = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
    ptx::prefetch_tensormap(&tmap);
  }
  if (warp == C::W_MMA) {
    ptx::tmem_alloc(ptx::smem_u32((const void*)tmem_slot), C::TMEM_COLS);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_sync();

  if (warp >= C::W_MMA) {
    // ---------------------------------------------------------------- MMA issuer of stream j.  The whole warp runs the loop and one lane issues, so that
    // descriptors can stay in uniform registers (in a branch of one lane an MMA takes 70 cycles to issue, more than to run)
    {
      const bool issuer = ptx::elect_one();
      const int j = warp - C::W_MMA, n_units = (units_cta + NS - 1 - j) / NS;
      constexpr uint32_t idesc_s = idesc_f16(QT, KT, false), idesc_o = idesc_f16(QT, 64, true), idesc_tail = idesc_f16(QT, 16, true);
      const uint32_t d_s = tmem_base + (uint32_t)j * C::COL_STREAM, d_p = d_s + C::COL_P, d_o = d_s + C::COL_O;
      const uint32_t q0 = base + C::OFF_Q + j * C::Q_BYTES, k0 = base + C::OFF_K + j * NB2 * C::T_BYTES, v0 = base + C::OFF_V + j * NB2 * C::T_BYTES;
      // two walks over the (unit, tile) pairs that exist: of the next S and of the next O
      struct Walk { int u, i, n; } ws = {-1, 0, 0}, wo = {-1, 0, 0};
      auto next_unit = [&](Walk& w) {                      // to the next unit with keys; false: none
        for (++w.u; w.u < n_units; ++w.u) {
          w.n = unit_of<NS>(j, w.u, deal, sh, kv_len).n_kv;
          w.i = 0;
          if (w.n > 0) return true;
        }
        return false;
      };
      int s_slot = 0, o_slot = 0;
      uint32_t k_phase = 0, v_phase = 0, q_phase = 0;
      bool ok = true;
      auto wait = [&](int i, uint32_t parity) { return __all_sync(0xffffffffu, ptx::mbar_wait(bar(j, i), parity, abort_flag)) != 0; };
      auto wait_s = [&]() -> bool {
        if (ws.i == 0) {
          if (!wait(B_Q_FULL, q_phase)) return false;
          q_phase ^= 1u;
        }
        return wait(B_K_FULL + s_slot, k_phase);
      };
      auto issue_s = [&]() {
        const uint32_t kt = k0 + (uint32_t)s_slot * C::T_BYTES;
#pragma unroll
        for (int bl = 0; bl < C::BLOCKS; ++bl) {
          const uint64_t dq = ptx::smem_desc_k_sw128(q0 + bl * C::Q_BLOCK), dk = ptx::smem_desc_k_sw128(kt + bl * C::T_BLOCK);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (issuer) ptx::umma_f16(d_s, dq + 2 * k, dk + 2 * k, idesc_s, (bl | k) ? 1u : 0u);
        }
        if (C::TAIL && issuer) ptx::umma_f16(d_s, smem_desc_sw32(q0 + C::BLOCKS * C::Q_BLOCK), smem_desc_sw32(kt + C::BLOCKS * C::T_BLOCK), idesc_s, 1u);
        if (issuer) {
          ptx::umma_commit(bar(j, B_S_FULL));
          ptx::umma_commit(bar(j, B_K_EMPTY + s_slot));
          if (ws.i + 1 == ws.n) ptx::umma_commit(bar(j, B_Q_EMPTY));     // the unit's last: its rows may be overwritten
        }
        __syncwarp();
        if (++s_slot == NB2) { s_slot = 0; k_phase ^= 1u; }
      };
      bool more_s = next_unit(ws), more_o = next_unit(wo);
      if (more_s) {
        ok = wait_s();
        ptx::tc_fence_after();
        if (ok) issue_s();
      }
      for (int t = 0; more_o && ok; ++t) {
        if (more_s && ++ws.i == ws.n) more_s = next_unit(ws);
        if (more_s) {                                      // the logits are in registers: the next ones may come
          if (!wait_s() || !wait(B_S_FREE, (uint32_t)t & 1u)) { ok = false; break; }
          ptx::tc_fence_after();
          issue_s();
        }
        if (!wait(B_V_FULL + o_slot, v_phase) ||
            // (for a unit's first tile the previous output has been read out: every softmax warp did so before it wrote)
            !wait(B_P_FULL, (uint32_t)t & 1u)) { ok = false; break; }
        ptx::tc_fence_after();
        const uint32_t vt = v0 + (uint32_t)o_slot * C::T_BYTES;
#pragma unroll
        for (int k = 0; k < KT / 16; ++k) {
#pragma unroll
          for (int bl = 0; bl < C::BLOCKS; ++bl)
            if (issuer) umma_f16_ts(d_o + 64u * bl, d_p + 8u * k, smem_desc_mn_sw128(vt + bl * C::T_BLOCK) + 128 * k, idesc_o, (wo.i | k) ? 1u : 0u);
          if (C::TAIL && issuer) umma_f16_ts(d_o + 64u * C::BLOCKS, d_p + 8u * k, smem_desc_sw32(vt + C::BLOCKS * C::T_BLOCK) + 32 * k, idesc_tail, (wo.i | k) ? 1u : 0u);
        }
        if (issuer) {
          ptx::umma_commit(bar(j, B_O_FULL));
          ptx::umma_commit(bar(j, B_V_EMPTY + o_slot));
        }
        __syncwarp();
        if (++o_slot == NB2) { o_slot = 0; v_phase ^= 1u; }
        if (++wo.i == wo.n) more_o = next_unit(wo);
      }
      if (!ok && issuer) *(volatile int*)status = ST_ATT_QUANTIZED_TC;
    }
  } else if (warp >= C::W_PROD) {
    // ---------------------------------------------------------------- TMA producer of stream j
    if (ptx::elect_one()) {
      const int j = warp - C::W_PROD, n_units = (units_cta + NS - 1 - j) / NS;
      const uint32_t stg0 = base + C::OFF_STG + j * NSTG * C::STG_BYTES, raw0 = base + C::OFF_RAW + j * NSTG * 2 * KT * 4;
      int slot = 0, issued = 0;
      uint32_t phase = 1;                                  // an empty slot's first wait passes at once
      bool ok = true;
      for (int u = 0; u < n_units && ok; ++u) {
        const Unit un = unit_of<NS>(j, u, deal, sh, kv_len);
        const float* ks = scales + ((size_t)un.b * sh.H + un.h) * pad;
        const float* vs = scales + ((size_t)(sh.B + un.b) * sh.H + un.h) * pad;
        for (int kt = 0; kt < un.n_kv; ++kt) {
          if (!ptx::mbar_wait(bar(j, B_STG_EMPTY + slot), phase, abort_flag)) { ok = false; break; }
          const uint32_t full = bar(j, B_STG_FULL + slot), dst = stg0 + slot * C::STG_BYTES, dst_s = raw0 + slot * 2 * KT * 4;
          ptx::mbar_expect_tx(full, C::STG_BYTES + 2 * KT * 4);
          ptx::tma_load_3d(dst, &tmap, un.h * DH, kt * KT, un.b, full);
          ptx::tma_load_3d(dst + KT * DH, &tmap, un.h * DH, kt * KT, sh.B + un.b, full);
          bulk_load(dst_s, ks + (size_t)kt * KT, KT * 4, full);
          bulk_load(dst_s + KT * 4, vs + (size_t)kt * KT, KT * 4, full);
          ++issued;
          if (++slot == NSTG) { slot = 0; phase ^= 1u; }
        }
      }
      if (!ok) {                                           // let copies already issued land before the CTA's shared memory is released
        *(volatile int*)status = ST_ATT_QUANTIZED_TC;
        for (int k = issued > NSTG ? issued - NSTG : 0; k < issued; ++k)
          ptx::mbar_wait(bar(j, B_STG_FULL + k % NSTG), (uint32_t)(k / NSTG) & 1u, abort_flag + 1, 20000000LL);
      }
    }
  } else if (warp >= C::W_CONV) {
    // ---------------------------------------------------------------- converters of stream j: a quarter of the rows; half of the keys of K or V
    const int j = (warp - C::W_CONV) / NC, part = (warp - C::W_CONV) % NC, n_units = (units_cta + NS - 1 - j) / NS;
    uint8_t* q_tile = gen + C::OFF_Q + j * C::Q_BYTES;
    auto wait = [&](int i, uint32_t parity) { return __all_sync(0xffffffffu, ptx::mbar_wait(bar(j, i), parity, abort_flag)) != 0; };
    auto arrive = [&](int i) { if (lane == 0) ptx::mbar_arrive(bar(j, i)); };
    bool ok = true;
    int stg = 0, slot = 0, sc = 0, qn = 0;
    uint32_t stg_phase = 0, phase = 1;
    for (int u = 0; u < n_units && ok; ++u) {
      const Unit un = unit_of<NS>(j, u, deal, sh, kv_len);
      if (un.n_kv == 0) continue;
      // ---- the unit's rows, one per lane at a time: in fp16, divided by a power of two and lifted by 2^15 (a bf16 number below 2 stays below fp16's
      // end); the loads are under way while the last unit's S is.  The power is that of the unit's largest value where that keeps all bits of
      // all values (down to 2^-32 of it), so that it goes into the keys' scales.  Elsewhere (a row of padding may hold numbers of any size)
      // each row has its own, no logit of it is off by more than 2^-40 of its largest ones', and its softmax thread multiplies its products by
      // it.  Both give the same bits: no row depends on another.
      float c_log2;
      bool own;
      {
        constexpr int ROWS = QT / NC / 32;                 // of a lane
        uint4 x[ROWS][DH / 8];
        uint32_t top[ROWS], low = 0xffffffffu;             // largest finite one of each row; smallest of all that are not 0, less 1 (0xffff: none)
#pragma unroll
        for (int p = 0; p < ROWS; ++p) {
          const int row = un.row0 + part * (QT / NC) + p * 32 + lane, token = row / sh.G;
          const bool there = row >= un.start && row < sh.R;
          const bf16* src = q + ((size_t)un.b * sh.n + token) * ld_q + (un.h * sh.G + row - token * sh.G) * DH;
#pragma unroll
          for (int c = 0; c < DH / 8; ++c) x[p][c] = there ? *reinterpret_cast<const uint4*>(src + 8 * c) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int p = 0; p < ROWS; ++p) {
          uint32_t both = 0;
#pragma unroll
          for (int c = 0; c < DH / 8; ++c) {
            const uint32_t w[4] = {x[p][c].x, x[p][c].y, x[p][c].z, x[p][c].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              both = attq::larger2(both, w[i] & 0x7fff7fffu);
              low = attq::smaller2_less_1(low, w[i] & 0x7fff7fffu);
            }
          }
          top[p] = max(both & 0xffffu, both >> 16);
          if (top[p] >= 0x7f80u) {                         // (infinities and NaN stay what they are, in their row)
            top[p] = 0;
#pragma unroll
            for (int c = 0; c < DH / 8; ++c)
              top[p] = max(max(top[p], max(attq::finite_of(x[p][c].x), attq::finite_of(x[p][c].y))), max(attq::finite_of(x[p][c].z), attq::finite_of(x[p][c].w)));
          }
        }
        low = min(low & 0xffffu, low >> 16);
        uint32_t all = top[0];
#pragma unroll
        for (int p = 1; p < ROWS; ++p) all = max(all, top[p]);
        all = __reduce_max_sync(0xffffffffu, all);
        low = __reduce_min_sync(0xffffffffu, low);
        // (two buffers: who writes a buffer again has passed the barrier of the unit between, which all reach after reading)
        volatile uint32_t* tops = reinterpret_cast<volatile uint32_t*>(gen + C::OFF_ROW) + (j * 2 + (qn & 1)) * 4;
        if (lane == 0) {
          tops[part] = all;
          tops[NC + part] = low;
        }
        __syncwarp();
        arrive(B_TOP);
        if (!wait(B_TOP, (uint32_t)qn & 1u)) { ok = false; break; }
#pragma unroll
        for (int p = 0; p < NC; ++p) {
          all = max(all, tops[p]);
          low = min(low, tops[NC + p]);
        }
        const int e = min(max((int)(all >> 7), 16), 254);
        own = (int)((low + 1u) >> 7) + 32 < e || e > 191;  // (above: the scales' products with it could leave the range for a smaller row)
        c_log2 = rsqrtf((float)DH) * 1.4426950408889634f * (own ? 256.0f : pow2(e - 15));
        float* factors = reinterpret_cast<float*>(gen + C::OFF_FACTOR) + (j * 2 + (qn & 1)) * QT + part * (QT / NC) + lane;
        if (!wait(B_Q_EMPTY, ((uint32_t)qn & 1u) ^ 1u)) { ok = false; break; }
#pragma unroll
        for (int p = 0; p < ROWS; ++p) {
          const int e_row = own ? min(max((int)(top[p] >> 7), 24), 254) : e;
          const float f = pow2(269 - e_row);
          if (own) factors[p * 32] = pow2(e_row - 23);     // (2^8 of it is in the scales: a row's products with its codes stay in range)
#pragma unroll
          for (int c = 0; c < DH / 8; ++c) {
            const uint32_t w[4] = {x[p][c].x, x[p][c].y, x[p][c].z, x[p][c].w};
            uint32_t y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 v = unpack_bf16x2(w[i]);
              y[i] = pack_weights(v.x * f, v.y * f);
            }
            *reinterpret_cast<uint4*>(q_tile + operand_off<DH>(QT, part * (QT / NC) + p * 32 + lane, c)) = make_uint4(y[0], y[1], y[2], y[3]);
          }
        }
      }
      ptx::fence_proxy_async();
      __syncwarp();
      arrive(B_Q_FULL);
      ++qn;
      attq::Units units;
      for (int kt = 0; kt < un.n_kv; ++kt) {
        if (!wait(B_STG_FULL + stg, stg_phase)) { ok = false; break; }
        const int key = part * 32 + lane;
        const uint8_t* codes = gen + C::OFF_STG + (j * NSTG + stg) * C::STG_BYTES;
        // 32 keys of a tile from bytes to an operand tile, a key per lane
        constexpr int PIECES = DH / 16;
        uint4 w[PIECES];
        auto take = [&](const uint8_t* from) {
#pragma unroll
          for (int c = 0; c < PIECES; ++c) w[c] = *reinterpret_cast<const uint4*>(from + piece<DH>(key, c));
        };
        auto give = [&](uint8_t* to, int b_full) {
#pragma unroll
          for (int c = 0; c < PIECES; ++c) {
            const uint32_t b[4] = {w[c].x ^ 0x80808080u, w[c].y ^ 0x80808080u, w[c].z ^ 0x80808080u, w[c].w ^ 0x80808080u};
            *reinterpret_cast<uint4*>(to + operand_off<DH>(KT, key, 2 * c)) =
                make_uint4(two_of<0x4140>(b[0]), two_of<0x4342>(b[0]), two_of<0x4140>(b[1]), two_of<0x4342>(b[1]));
            *reinterpret_cast<uint4*>(to + operand_off<DH>(KT, key, 2 * c + 1)) =
                make_uint4(two_of<0x4140>(b[2]), two_of<0x4342>(b[2]), two_of<0x4140>(b[3]), two_of<0x4342>(b[3]));
          }
          ptx::fence_proxy_async();
          __syncwarp();
          arrive(b_full + slot);
        };
        take(codes);
        float* scale_slot = reinterpret_cast<float*>(gen + C::OFF_SC) + (j * NSC + sc) * kScaleSlot;
        const float* raw_s = reinterpret_cast<const float*>(gen + C::OFF_RAW) + (j * NSTG + stg) * 2 * KT;
        const int left = un.len - kt * KT;               // keys of this tile that count (behind them scales may be anything)
        const float ks = key < left ? raw_s[key] : 0.f, vs = key < left ? raw_s[KT + key] : 0.f;
        const uint32_t other = (key ^ 32) < left ? attq::magnitude(raw_s[KT + (key ^ 32)]) : 0u;
        const uint32_t mine = attq::magnitude(vs);
        units.see(__reduce_max_sync(0xffffffffu, max(mine, other)), min(mine - 1u, other - 1u));
        const int d = units.move(__any_sync(0xffffffffu, units.apart<kSpread>()), kt == 0);
        if (!wait(B_K_EMPTY + slot, phase)) { ok = false; break; }
        scale_slot[key] = ks * c_log2;
        scale_slot[KT + key] = vs * pow2(260 - units.unit);   // below 2^7, so that weights of up to 2^8 stay below fp16's end
        if (part == 0 && lane == 0) {
          scale_slot[2 * KT] = units.wide ? 1.f : attq::step_of(d);
          scale_slot[2 * KT + 1] = pow2(units.unit - 6);
          // (two buffers: who writes a row's factor for the unit after next has seen this unit's S taken out of tensor memory)
          scale_slot[2 * KT + 2] = __int_as_float((units.wide ? F_WIDE : 0) | (own ? F_OWN | ((qn - 1) & 1) : 0));
          scale_slot[2 * KT + 3] = units.wide ? (float)d : 0.f;
        }
        __syncwarp();
        arrive(B_SC_FULL + sc);
        if (++sc == NSC) sc = 0;
        give(gen + C::OFF_K + (j * NB2 + slot) * C::T_BYTES, B_K_FULL);
        take(codes + KT * DH);
        if (!wait(B_V_EMPTY + slot, phase)) { ok = false; break; }
        give(gen + C::OFF_V + (j * NB2 + slot) * C::T_BYTES, B_V_FULL);
        arrive(B_STG_EMPTY + stg);
        if (++slot == NB2) { slot = 0; phase ^= 1u; }
        if (++stg == NSTG) { stg = 0; stg_phase ^= 1u; }
      }
    }
    if (!ok && lane == 0) *(volatile int*)status = ST_ATT_QUANTIZED_TC;
  } else {
    // ---------------------------------------------------------------- softmax streams (one thread per row)
    const int j = warp >> 2, n_units = (units_cta + NS - 1 - j) / NS, quarter = warp & 3;
    const int r = quarter * 32 + lane;                     // row inside the unit = TMEM lane
    const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t t_s = t_lane + (uint32_t)j * C::COL_STREAM, t_p = t_s + C::COL_P, t_o = t_s + C::COL_O;
    auto wait = [&](int i, uint32_t parity) { return __all_sync(0xffffffffu, ptx::mbar_wait(bar(j, i), parity, abort_flag)) != 0; };
    bool ok = true;
    int t = 0, sc = 0;                                     // tiles of this stream so far; slot of scales
    uint32_t sc_phase = 0;
    for (int u = 0; u < n_units && ok; ++u) {
      const Unit un = unit_of<NS>(j, u, deal, sh, kv_len);
      const int row = un.row0 + r, row_w = un.row0 + quarter * 32;   // this thread's row, the warp's first one
      const bool warp_valid = row_w >= un.start && row_w < sh.R, there = row >= un.start && row < sh.R;
      const int token = row / sh.G;
      uint16_t* dst = o + (((size_t)un.b * sh.n + token) * sh.heads + un.h * sh.G + row - token * sh.G) * DH;
      if (un.n_kv == 0) {                                  // no keys: zeros
        if (there)
#pragma unroll
          for (int c = 0; c < DH / 8; ++c) reinterpret_cast<uint4*>(dst)[c] = make_uint4(0, 0, 0, 0);
        continue;
      }
      float m_ref = 0.f, l = 0.f, unlift = 1.f;            // exponent reference (log2), running sum
      for (int i = 0; i < un.n_kv; ++i, ++t) {
        // the tile's scales, and S of this tile
        if (!wait(B_SC_FULL + sc, sc_phase) || !wait(B_S_FULL, (uint32_t)t & 1u)) { ok = false; break; }
        ptx::tc_fence_after();
        const float4* ks4 = reinterpret_cast<const float4*>(gen + C::OFF_SC + (j * NSC + sc) * kScaleSlot * 4);
        const float4* vs4 = ks4 + KT / 4;
        const float4 of_tile = ks4[KT / 2];
        const float step = of_tile.x;
        const int flags = __float_as_int(of_tile.z);
        unlift = of_tile.y;
        if (++sc == NSC) { sc = 0; sc_phase ^= 1u; }
        const int lim = un.len - i * KT;                   // keys of this tile that exist
        // The previous P V of this unit has read its weights and added to O.  (Without it no warp may announce this tile's weights.)
        auto previous_done = [&]() { return i == 0 || wait(B_O_FULL, (uint32_t)(t - 1) & 1u); };
        if (warp_valid) {
          if (__builtin_expect(flags & F_OWN, 0)) {                             // (in place, so that units that need none of it pay a branch)
            const float power = *(reinterpret_cast<const float*>(gen + C::OFF_FACTOR) + (2 * j + (flags & F_BUFFER)) * QT + r);
#pragma unroll 1
            for (int qc = 0; qc < KT / 16; ++qc) scale_in_place(t_s + (uint32_t)(qc * 16), power);
            tmem_st_wait();
          }
          uint32_t va[KT / 2], vb[KT / 2];                 // logits of the first and second 32 keys
          ptx::tmem_ld_32x32(t_s, va);
          ptx::tmem_ld_32x32(t_s + KT / 2, vb);
          ptx::tmem_ld_wait(va);
          ptx::tmem_ld_wait(vb);
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(j, B_S_FREE));
          // log2 of the weights against the reference so far: times the keys' scales (a broadcast: all lanes read the same)
          float* sa = reinterpret_cast<float*>(va);
          float* sb = reinterpret_cast<float*>(vb);
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          const float2 neg = make_float2(-m_ref, -m_ref);
          auto logits = [&](float* s, const float4* ks, float& m0, float& m1, int left) {
#pragma unroll
            for (int c = 0; c < KT / 8; ++c) {
              const float4 k = ks[c];
              const float2 x = __ffma2_rn(make_float2(s[4 * c], s[4 * c + 1]), make_float2(k.x, k.y), neg);
              const float2 y = __ffma2_rn(make_float2(s[4 * c + 2], s[4 * c + 3]), make_float2(k.z, k.w), neg);
              s[4 * c] = x.x; s[4 * c + 1] = x.y; s[4 * c + 2] = y.x; s[4 * c + 3] = y.y;
            }
            if (left < KT / 2) {
#pragma unroll
              for (int c = 0; c < KT / 2; ++c)
                if (c >= left) s[c] = -INFINITY;
            }
#pragma unroll
            for (int c = 0; c < KT / 2; c += 4) {
              m0 = max3(m0, s[c], s[c + 1]);
              m1 = max3(m1, s[c + 2], s[c + 3]);
            }
          };
          logits(sa, ks4, mx[0], mx[1], lim);
          logits(sb, ks4 + KT / 8, mx[2], mx[3], lim - KT / 2);
          float tmax = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), falls = 0.f;
          if (__builtin_expect(flags & F_WIDE, 0)) {                            // what counts for the reference; the reference falls by as much as the unit rises
            tmax = -INFINITY;
            falls = of_tile.w;
#pragma unroll
            for (int c = 0; c < KT / 2; ++c) {
              const float* vs = reinterpret_cast<const float*>(vs4);
              tmax = max3(tmax, sa[c] + attq::counts(vs[c] * 0x1p-7f), sb[c] + attq::counts(vs[KT / 2 + c] * 0x1p-7f));
            }
            tmax += falls;
          }
          // lazy reference: it moves only when this tile exceeds it by more than 2^8 (and to the first tile's maximum)
          const bool move = i == 0 || tmax > 8.0f;
          const bool any_move = __any_sync(0xffffffffu, move || falls != 0.f), rescale = i > 0 && (step != 1.f || any_move);
          float f = 1.0f, f_l = 1.0f;
          if (any_move) {
            const float d = move ? tmax : 0.f;
            f = i > 0 ? ex2_approx(-d) : 0.f;
            f_l = f * ex2_approx(falls);
            m_ref += d - falls;
            const float2 dd = make_float2(falls - d, falls - d);
#pragma unroll
            for (int c = 0; c < KT / 2; c += 2) {
              const float2 x = __fadd2_rn(make_float2(sa[c], sa[c + 1]), dd), y = __fadd2_rn(make_float2(sb[c], sb[c + 1]), dd);
              sa[c] = x.x; sa[c + 1] = x.y; sb[c] = y.x; sb[c + 1] = y.y;
            }
          }
          float2 ls[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          auto weights = [&](uint32_t (&v)[KT / 2], const float4* vs) {
            const float* s = reinterpret_cast<const float*>(v);
#pragma unroll
            for (int c = 0; c < KT / 8; ++c) {
              const float4 x = vs[c];
              float2 p = make_float2(ex2_approx(s[4 * c]), ex2_approx(s[4 * c + 1])), r2 = make_float2(ex2_approx(s[4 * c + 2]), ex2_approx(s[4 * c + 3]));
              ls[0] = __fadd2_rn(ls[0], p);
              ls[1] = __fadd2_rn(ls[1], r2);
              p = __fmul2_rn(p, make_float2(x.x, x.y));
              r2 = __fmul2_rn(r2, make_float2(x.z, x.w));
              v[2 * c] = pack_weights(p.x, p.y);           // pair c -> v[c]
              v[2 * c + 1] = pack_weights(r2.x, r2.y);
            }
          };
          weights(vb, vs4 + KT / 8);
          ok = previous_done();
          ptx::tc_fence_after();
          tmem_st_32x16(t_p + KT / 4, vb);
          weights(va, vs4);
          tmem_st_32x16(t_p, va);
          if (rescale) {
            // this row's accumulator in tensor memory moves to the new references
            const float fo = f * step;
#pragma unroll 1
            for (int qc = 0; qc < DH / 16; ++qc) scale_in_place(t_o + (uint32_t)(qc * 16), fo);
          }
          l = fmaf(l, f_l, (ls[0].x + ls[0].y) + (ls[1].x + ls[1].y));
          tmem_st_wait();
        } else {
          if (lane == 0) ptx::mbar_arrive(bar(j, B_S_FREE));
          ok = previous_done();
        }
        if (!ok) break;
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(j, B_P_FULL));
      }
      if (!ok) break;
      // ---- end of the unit: O / l -> output rows
      if (!wait(B_O_FULL, (uint32_t)(t - 1) & 1u)) { ok = false; break; }
      ptx::tc_fence_after();
      if (warp_valid) {
        const float2 inv = attq::unit_over(l, (int)(__float_as_uint(unlift) >> 23));
#pragma unroll
        for (int qc = 0; qc < DH / 16; ++qc) {
          uint32_t ov[16];
          tmem_ld_32x16(t_o + (uint32_t)(qc * 16), ov);
          ptx::tmem_ld_wait(ov);
          if (there) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = pack_a16x2(__uint_as_float(ov[2 * e]) * inv.x * inv.y, __uint_as_float(ov[2 * e + 1]) * inv.x * inv.y, o_bf16 != 0);
            reinterpret_cast<uint4*>(dst)[2 * qc] = make_uint4(w[0], w[1], w[2], w[3]);
            reinterpret_cast<uint4*>(dst)[2 * qc + 1] = make_uint4(w[4], w[5], w[6], w[7]);
          }
        }
        ptx::tc_fence_before();                            // (the next unit's first P V overwrites what has been read)
      }
    }
    if (!ok && lane == 0) *(volatile int*)status = ST_ATT_QUANTIZED_TC;
  }

  ptx::tc_fence_before();
  __syncthreads();
  if (warp == C::W_MMA) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem_base, C::TMEM_COLS);
  }
}

template <int DH, int NS>
cudaError_t launch(const void* q, int ld_q, int n, int heads, const QuantizedKv& c, const int32_t* kv_len, void* o, bool o_bf16, int* status, cudaStream_t st) {
  using C = Cfg<DH, NS>;
  CUtensorMap tm;
  EncodeTiledFn fn = tma_encode_fn();
  const cuuint64_t D = (cuuint64_t)c.H * DH, dims[3] = {D, (cuuint64_t)c.S, (cuuint64_t)2 * c.B}, strides[2] = {D, D * c.S};
  const cuuint32_t box[3] = {DH, KT, 1}, unit[3] = {1, 1, 1};
  const CUtensorMapSwizzle sw = DH == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : DH == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE;
  if (!fn || fn(&tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, c.codes, dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  static size_t smem_set[kMaxDevices] = {};
  cudaError_t e = ensure_dynamic_smem(attention_quantized_tc_kernel<DH, NS>, (size_t)C::SMEM_BYTES, smem_set);
  if (e != cudaSuccess) return e;
  Shape sh;
  sh.n = n; sh.G = heads / c.H; sh.R = n * sh.G; sh.H = c.H; sh.B = c.B; sh.S = c.S; sh.heads = heads; sh.n_qt = (sh.R + QT - 1) / QT;
  const int sms = device_sm_count();
  Deal deal;
  deal.units = c.B * c.H * sh.n_qt;
  deal.grid = deal.units < sms ? deal.units : sms;
  deal.rotate = attention_tc_rotation(deal.units, sh.n_qt, deal.grid, NS, &deal.rotate_turn);
  return launch_pdl(attention_quantized_tc_kernel<DH, NS>, dim3(deal.grid), dim3(C::THREADS), (size_t)C::SMEM_BYTES, st, tm, (const bf16*)q, ld_q,
                    (const float*)c.scales, c.pad, kv_len, (uint16_t*)o, o_bf16 ? 1 : 0, sh, deal, status);
}

}  // namespace

cudaError_t launch_attention_quantized_tc(const void* q, int ld_q, int n, int heads, const QuantizedKv& c, const int32_t* kv_len, void* o, bool o_bf16,
                                          int* status, cudaStream_t st) {
  switch (c.dh) {
    case 64: return launch<64, 2>(q, ld_q, n, heads, c, kv_len, o, o_bf16, status, st);
    case 80: return launch<80, 2>(q, ld_q, n, heads, c, kv_len, o, o_bf16, status, st);
    case 128: return launch<128, 1>(q, ld_q, n, heads, c, kv_len, o, o_bf16, status, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace marche
