// K7: rows of K and V into a cache held in 8 bits, and rows of that cache back.
//
// A head's dh values of one token share a scale: amax = max |x|, code = round(127 x / amax) (ties to even), scale = amax / 127,
// value = code * scale.  Codes are those of exact arithmetic.  127 / amax is found once per head as the sum of two fp32 numbers, an approximate
// reciprocal's 127 fold and, of the remainder, which is exact (amax has 8 bits, so it has few), the rest: right to 2^-44.  x times the sum by a
// product and an FMA is the quotient rounded once, by at most 2^-18 (it is below 128).  A quotient that is not a half is at least 2^-17 away from one
// (numerator and denominator have few bits), so it stays on its own side; one that is a half (x = amax / 2 is: 63.5) is a fp32 number, and the FMA
// lands on it.  Rounding is the addition of 1.5 * 2^23, whose sum's low byte is the code.  scale comes from amax / 127 by a multiplication and a
// correction by the remainder: a quotient of 8 bits by 127 is at least 2^-32 of itself away from the middle of two fp32 numbers.
// amax comes from the magnitudes, with NaN above infinity above every number: a head that holds one gets codes 0 and a NaN scale, so all of it
// reads back as NaN, and no code is ever anything but a number.
//
// What bounds it: HBM for many rows, the launch for few.  A warp takes a row of K or V, a group of dh / 8 lanes a head of it (16 bytes in, 8 out
// per lane), all loads of up to four heads a group ahead; the row leaves as whole 32-byte sectors; the scales lie key by key (their readers'
// order) and leave as single words.  Rows whose token is outside the cache are skipped: a batch with different numbers of rows is padded with -1.
// 6 x 8191 rows of 16 heads of 64: a division per value and index divisions per head 116 us for the writing (85 % of the issue slots), as it
// stands 65 us (a remainder per quotient 69; more registers than five CTAs on an SM have, at head_dim 80 1 us more for 128 x 43 rows); reading back
// 53 us, 5.8 TB/s.
#include "common.cuh"
#include "kernels.h"
#include "launch_pdl.h"

namespace marche {

namespace {

constexpr int kThreads = 256;

// Maximum over the W lanes of a group (lanes base .. base + W - 1), for W = 8, 10, 16: windows that wrap around inside the group.
template <int W>
MARCHE_DEVINL uint32_t group_max(uint32_t v, int base, int in) {
#pragma unroll
  for (int d = 1; d < W; d *= 2) {
    const int step = 2 * d <= W ? d : W - d;               // W = 10: windows of 1, 2, 4, 8, then 10
    int from = in + step;
    if (from >= W) from -= W;
    const uint32_t other = __shfl_sync(0xffffffffu, v, base + from);
    v = other > v ? other : v;
  }
  return v;
}

MARCHE_DEVINL float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
MARCHE_DEVINL uint32_t max_bf16x2(uint32_t a, uint32_t b) {   // NaN wins
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// blockIdx.y: K or V.  A warp takes a row, U rounds of 32 / W heads at a time.
template <int DH, int U>
__global__ void __launch_bounds__(kThreads, 5)
scatter_kv_quantized_kernel(const bf16* __restrict__ k, const bf16* __restrict__ v, size_t ld, const int32_t* __restrict__ idx, int n, int rows, int B,
                            int S, int H, int pad, int8_t* __restrict__ codes, float* __restrict__ scales) {
  constexpr int W = DH / 8, HPW = 32 / W;
  pdl_sync();
  const int which = blockIdx.y, lane = threadIdx.x & 31, group = lane / W, in = lane - group * W;
  const int row = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int b = row / n, t = idx ? idx[row] : row - b * n;
  if ((uint32_t)t >= (uint32_t)S) return;                  // (the whole warp)
  const bf16* src = (which ? v : k) + row * ld + 8 * in;
  int8_t* to = codes + (((size_t)which * B + b) * S + t) * ((size_t)H * DH) + 8 * in;
  float* to_scale = scales + ((size_t)which * B + b) * H * pad + t;
  for (int h0 = 0; h0 < H; h0 += HPW * U) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * HPW + group;
      x[u] = group < HPW && h < H ? *reinterpret_cast<const uint4*>(src + h * DH) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * HPW + group;
      if (u > 0 && h0 + u * HPW >= H) break;               // (the whole warp)
      uint32_t words[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      const uint32_t both = max_bf16x2(max_bf16x2(words[0] & 0x7fff7fffu, words[1] & 0x7fff7fffu), max_bf16x2(words[2] & 0x7fff7fffu, words[3] & 0x7fff7fffu));
      const uint32_t top = group_max<W>(max(both & 0xffffu, both >> 16), (group < HPW ? group : 0) * W, in);
      // Both sides of the division move to the range's middle by the same power of two near its ends; a head of zeros, or one that is not
      // finite, is divided by 1.
      const bool plain = top != 0 && top < 0x7f80u;
      const float amax = __uint_as_float(top << 16), shift = !plain ? 1.0f : (top >= 0x6000u ? 0x1p-64f : (top < 0x2000u ? 0x1p64f : 1.0f));
      const float d = plain ? amax * shift : 1.0f, inv = rcp_approx(d), r_hi = 127.0f * inv, r_lo = fmaf(-r_hi, d, 127.0f) * inv;
      if (!plain) words[0] = words[1] = words[2] = words[3] = 0;
      if (shift != 1.0f) {                                 // (what gets too small for a bf16 here has code 0)
        const uint32_t both_shifts = __float_as_uint(shift) | (__float_as_uint(shift) >> 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(words[i]) : "r"(both_shifts));
      }
      uint32_t c[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = make_float2(__uint_as_float(words[i] << 16), __uint_as_float(words[i] & 0xffff0000u));
        const float2 q = __ffma2_rn(v, make_float2(r_hi, r_hi), __fmul2_rn(v, make_float2(r_lo, r_lo)));
        const float2 r = __fadd2_rn(q, make_float2(12582912.0f, 12582912.0f));
        c[2 * i] = __float_as_uint(r.x);
        c[2 * i + 1] = __float_as_uint(r.y);
      }
      if (group < HPW && h < H) {
        uint2 out;
        out.x = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
        out.y = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
        *reinterpret_cast<uint2*>(to + (size_t)h * DH) = out;
        if (in == 0) {
          constexpr float r127 = 1.0f / 127.0f;
          const float s = amax * r127;
          float scale = fmaf(fmaf(-s, 127.0f, amax), r127, s);
          if (top < 0x2000u) scale = __fdiv_rn(amax, 127.0f);   // (a remainder could be too small for the format)
          to_scale[(size_t)h * pad] = top >= 0x7f80u ? __int_as_float(0x7fffffff) : scale;
        }
      }
    }
  }
}

// blockIdx.y: K or V.  A thread takes 16 values of a row.
template <int U>
__global__ void __launch_bounds__(kThreads)
gather_kv_quantized_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales, const int32_t* __restrict__ idx, int n, int B,
                           int S, int H, int dh, int pad, bf16* __restrict__ k_out, bf16* __restrict__ v_out, size_t ld) {
  pdl_sync();
  const int which = blockIdx.y;
  const uint32_t per_head = (uint32_t)dh / 16, per_row = per_head * H, total = (uint32_t)B * (uint32_t)n * per_row;   // below 2^31 (launch)
  const uint32_t first = blockIdx.x * (kThreads * U) + threadIdx.x;
  uint4 c[U];
  float s[U];
  bf16* to[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t i = first + u * kThreads;
    to[u] = nullptr;
    if (i < total) {
      const uint32_t row = i / per_row, e = i - row * per_row, h = e / per_head, b = row / (uint32_t)n;
      const int t = idx ? idx[row] : (int)(row - b * n);
      if ((uint32_t)t < (uint32_t)S) {
        c[u] = __ldcg(reinterpret_cast<const uint4*>(codes + (((size_t)which * B + b) * S + t) * ((size_t)H * dh)) + e);
        s[u] = *(scales + (((size_t)which * B + b) * H + h) * pad + t);
        to[u] = (which ? v_out : k_out) + row * ld + 16 * e;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!to[u]) continue;
    const uint32_t words[4] = {c[u].x, c[u].y, c[u].z, c[u].w};
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // code + 128 under the exponent of 2^23, and that off again: no conversion instruction (they run at a quarter of the rate)
      const uint32_t biased = words[i] ^ 0x80808080u;
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = (__uint_as_float(__byte_perm(biased, 0x4b000000u, 0x7540 + j)) - 8388736.0f) * s[u];
      r[2 * i] = pack_bf16x2(f[0], f[1]);
      r[2 * i + 1] = pack_bf16x2(f[2], f[3]);
    }
    reinterpret_cast<uint4*>(to[u])[0] = make_uint4(r[0], r[1], r[2], r[3]);
    reinterpret_cast<uint4*>(to[u])[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
}

template <int DH>
cudaError_t scatter(const void* k, const void* v, int ld, const int32_t* idx, int n, const QuantizedKv& c, cudaStream_t st) {
  constexpr int per_cta = kThreads / 32;
  const int rows = c.B * n;
  return launch_pdl(scatter_kv_quantized_kernel<DH, 4>, dim3((unsigned)((rows + per_cta - 1) / per_cta), 2), dim3(kThreads), 0, st, (const bf16*)k, (const bf16*)v,
                    (size_t)ld, idx, n, rows, c.B, c.S, c.H, c.pad, c.codes, c.scales);
}

}  // namespace

cudaError_t launch_scatter_kv_quantized(const void* k, const void* v, int ld, const int32_t* idx, int n, const QuantizedKv& c, cudaStream_t st) {
  switch (c.dh) {
    case 64: return scatter<64>(k, v, ld, idx, n, c, st);
    case 80: return scatter<80>(k, v, ld, idx, n, c, st);
    case 128: return scatter<128>(k, v, ld, idx, n, c, st);
  }
  return cudaErrorInvalidValue;
}

cudaError_t launch_gather_kv_quantized(const QuantizedKv& c, const int32_t* idx, int n, void* k_out, void* v_out, int ld, cudaStream_t st) {
  constexpr int U = 2;
  const uint32_t total = (uint32_t)c.B * (uint32_t)n * (uint32_t)(c.H * c.dh / 16);
  return launch_pdl(gather_kv_quantized_kernel<U>, dim3((total + kThreads * U - 1) / (kThreads * U), 2), dim3(kThreads), 0, st, (const int8_t*)c.codes,
                    (const float*)c.scales, idx, n, c.B, c.S, c.H, c.dh, c.pad, (bf16*)k_out, (bf16*)v_out, (size_t)ld);
}

}  // namespace marche
