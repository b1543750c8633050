// K7: rows of K and V into a cache held in 8 bits, and rows of that cache back.
//
// A head's dh values of one token share a scale: amax = max |x|, code = round(127 x / amax) (ties to even), scale = amax / 127,
// value = code * scale.  Codes are those of exact arithmetic: 127 x is exact in fp32 for a bf16 x (8 + 7 bits), and the quotient comes from a
// reciprocal of amax (one per head) with one correction by the exact remainder 127 x - t amax (Markstein's), which leaves an error of 2^-46 t
// before the last rounding.  A quotient that is not a half is at least 2^-17 away from one (numerator and denominator have few bits),
// so it rounds to its own side; one that is a half (x = amax / 2 is: 63.5) is a fp32 number, and the correction lands on it.  Rounding is the
// addition of 1.5 * 2^23, whose sum's low byte is the code.  With a division per value (20 instructions and a conversion) the kernel was bound
// by those: 128 x 43 rows of 16 heads of 80, 42.6 us.
// amax comes from the magnitude bits, which order as integers and put infinities and NaN above every number: such a head gets codes 0
// and a NaN scale, so all of it reads back as NaN, and no code is ever anything but a number.
//
// What bounds it: HBM for many rows, the launch for few.  A group of dh / 8 lanes takes a head of a row (16 bytes in, 8 out per
// lane), reduces in shuffles, and the row leaves as whole 32-byte sectors; the scales lie key by key (their readers' order) and leave
// as single words.  Rows whose token is outside the cache are skipped: a batch with different numbers of rows is padded with -1.
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

// blockIdx.y: K or V.  A warp takes 32 / W heads of the [rows][heads] list at a time, U times.
template <int DH, int U>
__global__ void __launch_bounds__(kThreads)
scatter_kv_quantized_kernel(const bf16* __restrict__ k, const bf16* __restrict__ v, size_t ld, const int32_t* __restrict__ idx, int n, int B,
                            int S, int H, int pad, int8_t* __restrict__ codes, float* __restrict__ scales) {
  constexpr int W = DH / 8, HPW = 32 / W;
  pdl_sync();
  const int which = blockIdx.y, lane = threadIdx.x & 31, in_warp = lane / W, in = lane - in_warp * W;
  const uint32_t total = (uint32_t)B * (uint32_t)n * (uint32_t)H;      // below 2^31 (launch)
  const uint32_t first = (blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * (HPW * U) + in_warp;
  const bf16* src = which ? v : k;
  uint4 x[U];
  int8_t* to[U];
  float* to_scale[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t head = first + u * HPW;
    to[u] = nullptr;
    x[u] = make_uint4(0, 0, 0, 0);
    if (in_warp < HPW && head < total) {
      const uint32_t row = head / (uint32_t)H, h = head - row * H, b = row / (uint32_t)n;
      const int t = idx ? idx[row] : (int)(row - b * n);
      if ((uint32_t)t < (uint32_t)S) {
        x[u] = *reinterpret_cast<const uint4*>(src + row * ld + h * DH + 8 * in);
        to[u] = codes + ((((size_t)which * B + b) * S + t) * H + h) * DH + 8 * in;
        to_scale[u] = scales + (((size_t)which * B + b) * H + h) * pad + t;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t words[4] = {x[u].x, x[u].y, x[u].z, x[u].w}, top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = words[i] & 0x7fffu, hi = (words[i] >> 16) & 0x7fffu;
      top = max(top, max(lo, hi));
    }
    top = group_max<W>(top, (lane / W < HPW ? lane / W : 0) * W, in);
    const float amax = __uint_as_float(top << 16);
    const float scale = top >= 0x7f80u ? __int_as_float(0x7fffffff) : __fdiv_rn(amax, 127.0f);
    // Near the ends of the range both sides of the division move to its middle by the same power of two; a head of zeros, or one that is not
    // finite, is multiplied by 0 throughout (and its infinities by none: a remainder that is not a number is not added).
    const bool plain = top != 0 && top < 0x7f80u;
    const float shift = top >= 0x6000u ? 0x1p-64f : (top < 0x2000u ? 0x1p64f : 1.0f), d = amax * shift;
    const float inv = plain ? __frcp_rn(d) : 0.f, times = 127.0f * shift;
    uint32_t packed[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t word = plain ? words[2 * i + (j >> 1)] : 0u;
        const float x = __uint_as_float(j & 1 ? word & 0xffff0000u : word << 16) * times;
        const float t = x * inv;
        c[j] = __float_as_uint(fmaf(plain ? fmaf(-t, d, x) : 0.f, inv, t) + 12582912.0f);
      }
      packed[i] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
    }
    if (to[u]) {
      *reinterpret_cast<uint2*>(to[u]) = make_uint2(packed[0], packed[1]);
      if (in == 0) *to_scale[u] = scale;
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
  constexpr int per_cta = kThreads / 32 * (32 / (DH / 8)), U = 2;
  const uint32_t total = (uint32_t)c.B * (uint32_t)n * (uint32_t)c.H;
  return launch_pdl(scatter_kv_quantized_kernel<DH, U>, dim3((total + per_cta * U - 1) / (per_cta * U), 2), dim3(kThreads), 0, st, (const bf16*)k, (const bf16*)v,
                    (size_t)ld, idx, n, c.B, c.S, c.H, c.pad, c.codes, c.scales);
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
