// A token's keys or values of one head on their way into the cache, for the kernels that write it.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cstdint>

#include "pad_chunk.h"
#include "pad_tc_common.cuh"

namespace pad {

// The 4-bit codes of eight values with scale byte `byte`.  x / s is x times 1 / s, 2^-22 off at most, rounded
// to f16 on the way: x has eight significant bits and s four, so that x / s either is a number half way between two
// codes (three significant bits), which f16 restores, or is 2^-8 of itself away from every one, further than f16 moves it.
__device__ __forceinline__ uint32_t e2m1_codes(const uint32_t (&x)[4], uint32_t byte) {
  const float s = (byte >> 3) ? __uint_as_float((byte + 896u) << 20) : (float)byte * 0x1p-17f;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  if (byte == 0u) inv = 0.f;
  const uint64_t inv2 = tc::f2pack(inv, inv);
  float y[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint64_t p = tc::fmul2(tc::f2pack(__uint_as_float(x[j] << 16), __uint_as_float(x[j] & 0xffff0000u)), inv2);
    const __half2 h = __floats2half2_rn(tc::f2lo(p), tc::f2hi(p));
    y[2 * j] = __low2float(h);
    y[2 * j + 1] = __high2float(h);
  }
  uint32_t r;
  asm("{\n .reg .b8 a, b, c, d;\n"
      " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      " mov.b32 %0, {a, b, c, d};\n}\n"
      : "=r"(r) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return r;
}
// The scale byte of a group whose largest magnitude has this bf16 pattern: max / 6 to the nearest.  The product with 1 / 6,
// which is 2^-25 of itself off as an fp32 number, is enough: a quotient that lies half way between two scales comes out exact
// (2^-25 t is less than half a step of t, t < 2), and any other lies 2^-8 of itself from there (max has eight significant bits).
__device__ __forceinline__ uint32_t e2m1_scale(uint32_t m) {
  if (m >= 0x7f80u) return 255u;
  const float s = __uint_as_float(m << 16) * (1.f / 6.f);
  const uint32_t u = __float_as_uint(s);
  const uint32_t b = s < 0x1p-14f ? (uint32_t)rintf(s * 0x1p17f) : ((u + 0x7ffffu + ((u >> 20) & 1u)) >> 20) - 896u;
  return min(b, 226u);
}

// Eight bf16 values (16-byte chunk c of a row of D / 8 consecutive lanes, all of a warp's rows together) into row `slot` of a
// pool, and the row's scales; `on`: the lane's row is there.
template <int D, int FMT>
__device__ __forceinline__ void store_group(uint4 x, int c, bool on, int64_t slot, void* pool, uint8_t* scales) {
  constexpr int L = D / 8;
  if (FMT == PAD_KV_BF16) {
    if (on) *(reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(pool) + slot * D) + c) = x;
    return;
  }
  // the largest magnitude as a bf16 pattern: integer order is theirs, NaN and infinity on top
  const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
  uint32_t m = __vmaxu2(__vmaxu2(xs[0] & 0x7fff7fffu, xs[1] & 0x7fff7fffu), __vmaxu2(xs[2] & 0x7fff7fffu, xs[3] & 0x7fff7fffu));
  m = max(m & 0xffffu, m >> 16);
#pragma unroll
  for (int o = FMT == PAD_KV_FP4 ? 1 : L / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (FMT == PAD_KV_FP4) {
    const uint32_t byte = e2m1_scale(m);
    if (on) {
      static_cast<uint32_t*>(pool)[slot * L + c] = byte == 255u ? 0u : e2m1_codes(xs, byte);
      if (!(c & 1)) scales[slot * (D / 16) + (c >> 1)] = (uint8_t)byte;
    }
    return;
  }
  // max = f * 2^(e - 127) with f in [1, 2): max <= 448 * 2^k = 1.75 * 2^(k + 8).  (A subnormal's k
  // is below the range in any case.)
  const int e = (int)(m >> 7);
  const int k = min(max(e - 127 - 8 + ((m & 0x7fu) > 0x60u ? 1 : 0), -120), 7);
  const bool bad = m >= 0x7f80u;
  const float inv = __uint_as_float((uint32_t)(127 - k) << 23);  // 2^-k
  uint32_t code[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    uint32_t two[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const uint32_t v = xs[2 * j + q];
      const float2 f = make_float2(__uint_as_float(v << 16) * inv, __uint_as_float(v & 0xffff0000u) * inv);
      two[q] = bad ? 0u : __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);  // (codes are finite, always)
    }
    code[j] = two[0] | (two[1] << 16);
  }
  if (on) {
    *(reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + slot * D) + c) = make_uint2(code[0], code[1]);
    if (c == 0) scales[slot] = (uint8_t)(bad ? 255 : m == 0u ? 0 : k + 127);
  }
}

}  // namespace pad
