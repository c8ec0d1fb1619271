// The private paged cache of the multi-token step: pad_chunk_append writes the new tokens of every
// branch, in bf16 or as 8-bit groups, and pad_chunk_read copies cached tokens out as bf16.
//
// An 8-bit group (the head_dim values of one token and kv-head): k is the smallest integer with
// max|x| <= 448 * 2^k, kept in [-120, 7]; codes are e4m3 of x / 2^k to nearest even.  Both sides of
// that division are powers of two apart, so nothing is rounded but the code, and the code times 2^k
// is exact in bf16 again (three bits of mantissa).  Above 57344 = 448 * 2^7 values saturate: k ends
// there because the readers undo the format's exponent offset and the scale in one bf16 product,
// 2^(120 + k), which has to be finite.
//
// Bound by memory, one pass each; short ones by the launch.  32768 tokens of 4 heads x 128 written and read back
// (two calls of 101 MB): 45 us, 4.5 TB/s; 32 branches x 5 tokens written and 9000 read: 12 us.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <algorithm>
#include <cstdint>

#include "pad_chunk.h"

namespace pad {

namespace {

constexpr int kThreads = 256;
constexpr int kReadTokens = 32;  // of a span

// 16 lanes of 8 bf16 values (8 at head_dim 64) hold one group.
template <int D, bool FP8>
__global__ void __launch_bounds__(kThreads) chunk_append_kernel(const __grid_constant__ ChunkParams p,
                                                                const ChunkPages* __restrict__ work,
                                                                const __nv_bfloat16* __restrict__ k_new,
                                                                const __nv_bfloat16* __restrict__ v_new, int64_t stride,
                                                                void* __restrict__ k_pool, void* __restrict__ v_pool,
                                                                uint8_t* __restrict__ k_scale, uint8_t* __restrict__ v_scale) {
  constexpr int L = D / 8;  // lanes of a group
  const ChunkPages w = work[blockIdx.x];
  int32_t* entry = p.page_table + (int64_t)w.event * p.max_pages + w.column;
  const int page = w.page >= 0 ? w.page : __ldcg(entry);
  const int groups = w.count * p.h_kv * 2, lanes = (groups * L + 31) / 32 * 32, c = threadIdx.x % L;
  constexpr int U = 4;  // groups of a thread under way together
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < lanes; i0 += U * kThreads) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int g = (i0 + u * kThreads) / L, tok = g / (2 * p.h_kv), r = g % (2 * p.h_kv);
      x[u] = make_uint4(0u, 0u, 0u, 0u);
      if (g < groups) x[u] = __ldcs(reinterpret_cast<const uint4*>(((r & 1) ? v_new : k_new) + (w.tok + tok) * stride + (r >> 1) * D) + c);
    }
    // (the data is on its way while the page is looked up)
    if (i0 == (int)threadIdx.x) {
      if (w.page >= 0 && threadIdx.x == 0) *entry = page;
      if ((unsigned)page >= (unsigned)p.n_pages) {
        if (threadIdx.x == 0) pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_BOUNDS, w.event, w.column, page);
        return;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * kThreads >= lanes) break;  // (whole warps)
      const int g = (i0 + u * kThreads) / L, tok = g / (2 * p.h_kv), r = g % (2 * p.h_kv), h = r >> 1;
      const bool on = g < groups;
      const int64_t slot = ((int64_t)page * p.h_kv + h) * p.page_size + w.slot + tok;
      if (!FP8) {
        if (on) *(reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>((r & 1) ? v_pool : k_pool) + slot * D) + c) = x[u];
        continue;
      }
      // the largest magnitude as a bf16 pattern: integer order is theirs, NaN and infinity on top
      uint32_t m = 0u;
      const uint32_t xs[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) m = max(m, max(xs[j] & 0x7fffu, (xs[j] >> 16) & 0x7fffu));
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
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
        *(reinterpret_cast<uint2*>(static_cast<uint8_t*>((r & 1) ? v_pool : k_pool) + slot * D) + c) = make_uint2(code[0], code[1]);
        if (c == 0) ((r & 1) ? v_scale : k_scale)[slot] = (uint8_t)(bad ? 255 : m == 0u ? 0 : k + 127);
      }
    }
  }
}

// One span: up to kReadTokens consecutive tokens of an event, all heads, K and V.  A thread moves 16
// bytes in bf16, or 8 codes to 16 bytes.
template <int D, bool FP8>
__global__ void __launch_bounds__(kThreads) chunk_read_kernel(const __grid_constant__ ChunkParams p,
                                                              const ChunkRead* __restrict__ work, int n_events,
                                                              __nv_bfloat16* __restrict__ k_out,
                                                              __nv_bfloat16* __restrict__ v_out) {
  constexpr int L = D / 8;
  __shared__ int pages[kReadTokens];
  __shared__ ChunkRead mine;
  __shared__ int event;
  const int b = (int)blockIdx.x;
  for (int e = threadIdx.x; e < n_events; e += kThreads) {
    const ChunkRead w = work[e];
    if (b >= w.span0 && b < w.span0 + (w.count + kReadTokens - 1) / kReadTokens) mine = w, event = e;  // (one event holds it)
  }
  __syncthreads();
  const int pos = (b - mine.span0) * kReadTokens, count = min(kReadTokens, mine.count - pos);
  if ((int)threadIdx.x < count) {
    const int col = (pos + (int)threadIdx.x) >> p.page_shift, pg = __ldcg(p.page_table + (int64_t)event * p.max_pages + col);
    pages[threadIdx.x] = pg;
    if ((unsigned)pg >= (unsigned)p.n_pages) pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_BOUNDS, event, col, pg);
  }
  __syncthreads();
  const int n = count * p.h_kv * L, c = threadIdx.x % L;
  constexpr int U = 4;  // rows of a thread under way together, K and V
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < n; i0 += U * kThreads) {
    uint4 x[U][2];
    uint32_t sc[U][2];
    int64_t to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kThreads, g = i / L, h = g % p.h_kv, t = g / p.h_kv;
      to[u] = i < n ? ((mine.out + pos + t) * p.h_kv + h) * D + 8 * c : -1;
      x[u][0] = x[u][1] = make_uint4(0u, 0u, 0u, 0u);
      sc[u][0] = sc[u][1] = 0u;
      const int pg = i < n ? pages[t] : -1;
      if ((unsigned)pg >= (unsigned)p.n_pages) continue;  // (its tokens are zeros)
      const int64_t slot = ((int64_t)pg * p.h_kv + h) * p.page_size + ((pos + t) & (p.page_size - 1));
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const void* pool = kv ? p.v_pool : p.k_pool;
        if (FP8) {
          const uint2 v = __ldcg(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pool) + slot * D) + c);
          x[u][kv].x = v.x;
          x[u][kv].y = v.y;
          sc[u][kv] = __ldcg((kv ? p.v_scale : p.k_scale) + slot);
        } else {
          x[u][kv] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(pool) + slot * D) + c);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (to[u] < 0) continue;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        uint4 o = x[u][kv];
        if (FP8) {
          uint32_t m = scale_mult(sc[u][kv]);
          m |= m << 16;
          o = make_uint4(e4m3_pair(__byte_perm(x[u][kv].x, 0u, 0x1404), m), e4m3_pair(__byte_perm(x[u][kv].x, 0u, 0x3424), m),
                         e4m3_pair(__byte_perm(x[u][kv].y, 0u, 0x1404), m), e4m3_pair(__byte_perm(x[u][kv].y, 0u, 0x3424), m));
        }
        __stcs(reinterpret_cast<uint4*>((kv ? v_out : k_out) + to[u]), o);
      }
    }
  }
}

template <int D, bool FP8>
cudaError_t append(const ChunkParams& p, const ChunkPages* work, int n, const void* k_new, const void* v_new,
                   int64_t stride, void* k_pool, void* v_pool, uint8_t* ks, uint8_t* vs, cudaStream_t s) {
  return launch_early(false, chunk_append_kernel<D, FP8>, dim3(n), kThreads, 0, s, p, work, static_cast<const __nv_bfloat16*>(k_new),
                      static_cast<const __nv_bfloat16*>(v_new), stride, k_pool, v_pool, ks, vs);
}
template <int D, bool FP8>
cudaError_t read(const ChunkParams& p, const ChunkRead* work, int n_events, int n, void* k_out, void* v_out, cudaStream_t s) {
  return launch_early(false, chunk_read_kernel<D, FP8>, dim3(n), kThreads, 0, s, p, work, n_events, static_cast<__nv_bfloat16*>(k_out),
                      static_cast<__nv_bfloat16*>(v_out));
}

}  // namespace

int chunk_read_tokens() { return kReadTokens; }

cudaError_t launch_chunk_append(const ChunkParams& p, int head_dim, bool fp8, const ChunkPages* work, int n_work,
                                const void* k_new, const void* v_new, int64_t stride, void* k_pool, void* v_pool,
                                uint8_t* k_scale, uint8_t* v_scale, cudaStream_t s) {
  auto* f = head_dim == 128 ? (fp8 ? append<128, true> : append<128, false>) : (fp8 ? append<64, true> : append<64, false>);
  return f(p, work, n_work, k_new, v_new, stride, k_pool, v_pool, k_scale, v_scale, s);
}

cudaError_t launch_chunk_read(const ChunkParams& p, int head_dim, bool fp8, const ChunkRead* work, int n_events,
                              int n_spans, void* k_out, void* v_out, cudaStream_t s) {
  auto* f = head_dim == 128 ? (fp8 ? read<128, true> : read<128, false>) : (fp8 ? read<64, true> : read<64, false>);
  return f(p, work, n_events, n_spans, k_out, v_out, s);
}

}  // namespace pad
