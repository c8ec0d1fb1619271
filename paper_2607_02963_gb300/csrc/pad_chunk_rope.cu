// Rotary positions of a step's new queries and keys (pad_chunk_append_rope): q into q_out, k_new into the pools (with
// v_new as it is), in the cache's format.
//
// The angle of pair i at position m is m f_i.  f_i / 2 pi comes as a 64-bit fraction, so that its product with the
// position, the upper bits left out, is the angle in turns: exact to 2^-64 times the position, where a 32-bit angle at
// position 10^6 is off by a tenth of a turn and more.  Its upper 32 bits, as a signed fraction of a turn, go to sincospi.
//
// One pass over the bytes, bound by memory: each token's q, k_new and v_new in, q_out, K and V out (16k tokens of 28 + 8 heads x 128,
// half of the head interleaved: 55 us, 5.4 TB/s, into 8 bits 54, 4 bits 53; the whole head in halves 59, 60, 60; 160 tokens: about
// 8 us in each, the host's call).  A CTA takes a few
// tokens of one page; their cosines and sines, the same for all heads, go to shared memory once.  A warp takes whole
// heads, 16 bytes a lane, and a lane keeps its eight pairs' cosines and sines in registers for all heads of a token.
#include <cuda_bf16.h>
#include <algorithm>
#include <cstdint>

#include "pad_chunk.h"
#include "pad_chunk_quant.cuh"

namespace pad {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// How a lane finds its pairs' other members: in its own 16 bytes, in those of the lane R / 16 further, or, where half of
// the rotary dimensions are no multiple of eight, in the row in shared memory.
enum { kInterleaved, kHalf, kHalfOdd };

struct RopeArgs {
  pad_rope rope;
  int32_t slices, warps_per_token;
  const int32_t* position;
  const __nv_bfloat16* q;
  int64_t q_stride, out_stride, new_stride;
  __nv_bfloat16* q_out;
  const __nv_bfloat16* k_new;
  const __nv_bfloat16* v_new;
  void* k_pool;
  void* v_pool;
  uint8_t* k_scale;
  uint8_t* v_scale;
};

__device__ __forceinline__ uint32_t rounded2(float lo, float hi) {
  const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ float lo_of(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_of(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// The lane's eight values turned.  cs: cosine and signed sine that go with each (kInterleaved: of the pairs); n: how many of
// the eight are turned, an even number (kHalf: 0 or 8); other: the lane (of the warp) or the row in shared memory with the pairs' other members.
template <int LAYOUT>
__device__ __forceinline__ uint4 turned(uint4 x, const float2 (&cs)[8], int n, int other, const uint16_t* row, int d0, int rotary) {
  uint32_t v[4] = {x.x, x.y, x.z, x.w};
  if (LAYOUT == kInterleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = lo_of(v[j]), b = hi_of(v[j]);
      if (2 * j < n) v[j] = rounded2(a * cs[j].x - b * cs[j].y, b * cs[j].x + a * cs[j].y);
    }
  } else if (LAYOUT == kHalf) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = __shfl_sync(0xffffffffu, v[j], other);
      if (n) v[j] = rounded2(lo_of(v[j]) * cs[2 * j].x + lo_of(w) * cs[2 * j].y, hi_of(v[j]) * cs[2 * j + 1].x + hi_of(w) * cs[2 * j + 1].y);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float o[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int d = d0 + 2 * j + u;
        const float a = u ? hi_of(v[j]) : lo_of(v[j]);
        const float b = d < rotary ? lo_of(row[d < rotary / 2 ? d + rotary / 2 : d - rotary / 2]) : 0.f;
        o[u] = a * cs[2 * j + u].x + b * cs[2 * j + u].y;
      }
      const uint32_t w = rounded2(o[0], o[1]);
      if (2 * j < n) v[j] = w;
    }
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

template <int D, int FMT, int LAYOUT>
__global__ void __launch_bounds__(kThreads, 3) chunk_rope_kernel(const __grid_constant__ ChunkParams p,
                                                              const ChunkPages* __restrict__ work,
                                                              const __grid_constant__ RopeArgs a) {
  constexpr int L = D / 8, RPW = 32 / L;              // lanes of a head, heads of a warp at a time
  __shared__ float2 table[kWarps][D / 2];             // of the CTA's tokens
  __shared__ __align__(16) uint16_t rows[LAYOUT == kHalfOdd ? kWarps : 1][LAYOUT == kHalfOdd ? RPW * D : 1];
  const int slice = (int)blockIdx.x % a.slices;
  const ChunkPages w = work[(int)blockIdx.x / a.slices];
  const int per = kWarps / a.warps_per_token, first = slice * per, n = min(per, w.count - first);  // the CTA's tokens
  if (n <= 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane % L, sub = lane / L;
  const int R = a.rope.rotary_dim, H = R / 2;
  int32_t* entry = p.page_table + (int64_t)w.event * p.max_pages + w.column;
  const int page = w.page >= 0 ? w.page : __ldcg(entry);
  const bool there = (unsigned)page < (unsigned)p.n_pages;
  if (slice == 0 && threadIdx.x == 0) {
    if (w.page >= 0) *entry = page;
    if (!there) pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_BOUNDS, w.event, w.column, page);
  }
  // The token's heads in order: of q, of k, of v; a batch of U is on its way while the one before is turned, the first
  // while the cosines and sines are formed.
  constexpr int U = 4;
  const int t = warp / a.warps_per_token, part = warp % a.warps_per_token;
  const int heads = p.h_q + 2 * p.h_kv, step = RPW * a.warps_per_token;
  const int64_t tok = w.tok + first + t;
  const __nv_bfloat16* const q = a.q + tok * a.q_stride + 8 * c;
  const __nv_bfloat16* const kn = a.k_new + tok * a.new_stride - (int64_t)p.h_q * D + 8 * c;
  const __nv_bfloat16* const vn = a.v_new + tok * a.new_stride - (int64_t)(p.h_q + p.h_kv) * D + 8 * c;
  uint4 next[U];
  auto fetch = [&](int h0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + sub + u * step;
      if (h < heads && t < n) next[u] = __ldcs(reinterpret_cast<const uint4*>((h < p.h_q ? q : h < p.h_q + p.h_kv ? kn : vn) + h * D));
    }
  };
  fetch(RPW * part);
  for (int i = threadIdx.x; i < n * H; i += kThreads) {
    const int ti = i / H, k = i % H;
    const uint64_t turn = (uint64_t)(int64_t)a.position[w.tok + first + ti] * a.rope.turn[k];
    float s, co;
    sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &s, &co);
    table[ti][k] = make_float2(co * a.rope.magnitude, s * a.rope.magnitude);
  }
  __syncthreads();
  if (t >= n) return;
  // this lane's cosines and sines, the sine's sign with it
  float2 cs[8];
  const int d0 = 8 * c, turns = min(max(R - d0, 0), 8);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    cs[j] = make_float2(1.f, 0.f);
    if (LAYOUT == kInterleaved) {
      if (j < 4 && 2 * j < turns) cs[j] = table[t][d0 / 2 + j];
    } else if (j < turns) {
      const int d = d0 + j;
      cs[j] = table[t][d < H ? d : d - H];
      if (d < H) cs[j].y = -cs[j].y;
    }
  }
  const int other = LAYOUT == kHalf && turns ? lane + (d0 < H ? H / 8 : -(H / 8)) : lane;
  uint16_t* row = rows[LAYOUT == kHalfOdd ? warp : 0] + (LAYOUT == kHalfOdd ? sub * D : 0);
  auto turn = [&](uint4 x) {
    if (LAYOUT == kHalfOdd) {
      __syncwarp();
      *reinterpret_cast<uint4*>(row + d0) = x;
      __syncwarp();
    }
    return turned<LAYOUT>(x, cs, turns, other, row, d0, R);
  };
  __nv_bfloat16* const out = a.q_out + tok * a.out_stride + d0;
  const int64_t slot = w.slot + first + t;
#pragma unroll 1
  for (int h0 = RPW * part; h0 < heads; h0 += U * step) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = next[u];
    fetch(h0 + U * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h0 + u * step >= heads) break;  // (whole warps)
      const int h = h0 + sub + u * step, kv = h - p.h_q;
      const uint4 o = turn(x[u]);
      if (kv < 0) __stcs(reinterpret_cast<uint4*>(out + h * D), o);
      if (there && h0 + u * step + RPW > p.h_q) {  // (some head of the warp's is the cache's)
        const bool v = kv >= p.h_kv;
        const int hk = max(v ? kv - p.h_kv : kv, 0);
        const uint4 y = v ? x[u] : o;
        store_group<D, FMT>(y, c, kv >= 0 && h < heads, ((int64_t)page * p.h_kv + hk) * p.page_size + slot, v ? a.v_pool : a.k_pool, v ? a.v_scale : a.k_scale);
      }
    }
  }
}

template <int D, int FMT>
cudaError_t launch(const ChunkParams& p, const RopeArgs& a, const ChunkPages* work, int n, cudaStream_t s) {
  const int half = a.rope.rotary_dim / 2;
  auto* f = a.rope.layout == PAD_ROPE_INTERLEAVED ? chunk_rope_kernel<D, FMT, kInterleaved>
            : half % 8 == 0                       ? chunk_rope_kernel<D, FMT, kHalf>
                                                  : chunk_rope_kernel<D, FMT, kHalfOdd>;
  if ((int64_t)n * a.slices > INT32_MAX) return cudaErrorInvalidValue;
  return launch_early(false, f, dim3(n * a.slices), kThreads, 0, s, p, work, a);
}

}  // namespace

cudaError_t launch_chunk_rope(const ChunkParams& p, int head_dim, int kv_format, const pad_rope& rope, const ChunkPages* work,
                              int n_work, int most, int64_t n_tokens, int sms, const int32_t* position, const void* q, int64_t q_stride,
                              void* q_out, int64_t out_stride, const void* k_new, const void* v_new, int64_t new_stride,
                              void* k_pool, void* v_pool, uint8_t* k_scale, uint8_t* v_scale, cudaStream_t s) {
  RopeArgs a{};
  a.rope = rope;
  // warps share a token where there are too few for the GPU
  a.warps_per_token = 1;
  while (a.warps_per_token < kWarps && n_tokens * a.warps_per_token < 32 * (int64_t)sms) a.warps_per_token *= 2;
  const int per = kWarps / a.warps_per_token;
  a.slices = (most + per - 1) / per;
  a.position = position;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.q_out = static_cast<__nv_bfloat16*>(q_out);
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.new_stride = new_stride;
  a.k_new = static_cast<const __nv_bfloat16*>(k_new);
  a.v_new = static_cast<const __nv_bfloat16*>(v_new);
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  auto* f = head_dim == 128 ? (kv_format == PAD_KV_FP4 ? launch<128, PAD_KV_FP4> : kv_format == PAD_KV_FP8 ? launch<128, PAD_KV_FP8> : launch<128, PAD_KV_BF16>)
                            : (kv_format == PAD_KV_FP4 ? launch<64, PAD_KV_FP4> : kv_format == PAD_KV_FP8 ? launch<64, PAD_KV_FP8> : launch<64, PAD_KV_BF16>);
  return f(p, a, work, n_work, s);
}

}  // namespace pad
