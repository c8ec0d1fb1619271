// The private paged cache of the multi-token step: pad_chunk_append writes the new tokens of every
// branch, in bf16 or as 8-bit or 4-bit groups, and pad_chunk_read copies cached tokens out as bf16.
//
// An 8-bit group (the head_dim values of one token and kv-head): k is the smallest integer with
// max|x| <= 448 * 2^k, kept in [-120, 7]; codes are e4m3 of x / 2^k to nearest even.  Both sides of
// that division are powers of two apart, so nothing is rounded but the code, and the code times 2^k
// is exact in bf16 again (three bits of mantissa).  Above 57344 = 448 * 2^7 values saturate: k ends
// there because the readers undo the format's exponent offset and the scale in one bf16 product,
// 2^(120 + k), which has to be finite.
//
// A 4-bit group (16 consecutive values of one token and kv-head): the scale s is max|x| / 6 rounded to 5 exponent
// and 3 mantissa bits, the upper byte of its f16 pattern without the sign, 10240 at most; codes are e2m1 of x / s to
// nearest even.  Code times scale has six significant bits at most and is exact in bf16 and in f16 (up to 6 x 10240 = 61440).
//
// Bound by memory, one pass each; short ones by the launch.  32768 tokens of 4 heads x 128 written and read back
// (two calls of 101 MB): 45 us, 4.5 TB/s; 32 branches x 5 tokens written and 9000 read: 12 us.  In 4 bits the same (two calls
// of 86 MB) 43 us, 4 TB/s, where writing is bound by its instructions (140 for a warp's 256 values); 9000 read 12 us.
#include <cuda_bf16.h>
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "pad_chunk.h"
#include "pad_chunk_quant.cuh"

namespace pad {

namespace {

constexpr int kThreads = 256;
constexpr int kReadTokens = 32;  // of a span

// Division by a count that the launch brings, as a product with 2^32 / d rounded up: the quotient, or one more where n d is
// above 2^32.
struct Divisor {
  uint32_t d, inv;
  __device__ explicit Divisor(int by) : d((uint32_t)by), inv(0xffffffffu / (uint32_t)by + 1u) {}
  __device__ int operator()(int n) const {
    if (d == 1u) return n;
    const uint32_t q = __umulhi((uint32_t)n, inv);
    return (int)(q * d > (uint32_t)n ? q - 1u : q);
  }
};

// 16 lanes of 8 bf16 values (8 at head_dim 64) hold a token and head: one 8-bit group, or a 4-bit one for two lanes.
template <int D, int FMT>
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
  const Divisor rows(2 * p.h_kv);
  const int groups = w.count * p.h_kv * 2, lanes = (groups * L + 31) / 32 * 32, c = threadIdx.x % L;
  constexpr int U = 4;  // groups of a thread under way together
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < lanes; i0 += U * kThreads) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int g = (i0 + u * kThreads) / L, tok = rows(g), r = g - tok * 2 * p.h_kv;
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
      const int g = (i0 + u * kThreads) / L, tok = rows(g), r = g - tok * 2 * p.h_kv, h = r >> 1;
      const bool on = g < groups;
      const int64_t slot = ((int64_t)page * p.h_kv + h) * p.page_size + w.slot + tok;
      store_group<D, FMT>(x[u], c, on, slot, (r & 1) ? v_pool : k_pool, (r & 1) ? v_scale : k_scale);
    }
  }
}

// One span: up to kReadTokens consecutive tokens of an event, all heads, K and V.  A thread moves 16
// bytes in bf16, or 8 codes to 16 bytes.  Work: ChunkRead for tokens copied out, ChunkWiden for pages in bf16.
template <int D, int FMT, class Work>
__global__ void __launch_bounds__(kThreads) chunk_read_kernel(const __grid_constant__ ChunkParams p,
                                                              const Work* __restrict__ work, int n_events,
                                                              __nv_bfloat16* __restrict__ k_out,
                                                              __nv_bfloat16* __restrict__ v_out,
                                                              int32_t* __restrict__ table, int columns) {
  constexpr int L = D / 8;
  constexpr bool kWiden = std::is_same<Work, ChunkWiden>::value;
  __shared__ int pages[kReadTokens];
  __shared__ Work mine;
  __shared__ int row;
  const int b = (int)blockIdx.x;
  for (int e = threadIdx.x; e < n_events; e += kThreads) {
    const Work w = work[e];
    if (b >= w.span0 && b < w.span0 + (w.count + kReadTokens - 1) / kReadTokens) mine = w, row = e;  // (one event holds it)
  }
  __syncthreads();
  int event = row;
  if constexpr (kWiden) event = mine.event;
  const int pos = (b - mine.span0) * kReadTokens, count = min(kReadTokens, mine.count - pos);
  if ((int)threadIdx.x < count) {
    const int col = (pos + (int)threadIdx.x) >> p.page_shift, pg = __ldcg(p.page_table + (int64_t)event * p.max_pages + col);
    pages[threadIdx.x] = pg;
    const bool there = (unsigned)pg < (unsigned)p.n_pages;
    if (!there) pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_BOUNDS, event, col, pg);
    if constexpr (kWiden)
      if (((pos + (int)threadIdx.x) & (p.page_size - 1)) == 0) table[(int64_t)row * columns + col] = there ? mine.page0 + col : -1;
  }
  __syncthreads();
  const int n = count * p.h_kv * L, c = threadIdx.x % L;
  const Divisor heads(p.h_kv);
  constexpr int U = 4;  // rows of a thread under way together, K and V
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < n; i0 += U * kThreads) {
    uint4 x[U][2];
    uint32_t sc[U][2];
    int64_t to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kThreads, g = i / L, t = heads(g), h = g - t * p.h_kv;
      if constexpr (kWiden)
        to[u] = i < n ? ((((int64_t)mine.page0 + ((pos + t) >> p.page_shift)) * p.h_kv + h) * p.page_size + ((pos + t) & (p.page_size - 1))) * D + 8 * c : -1;
      else
        to[u] = i < n ? ((mine.out + pos + t) * p.h_kv + h) * D + 8 * c : -1;
      x[u][0] = x[u][1] = make_uint4(0u, 0u, 0u, 0u);
      sc[u][0] = sc[u][1] = 0u;
      const int pg = i < n ? pages[t] : -1;
      if ((unsigned)pg >= (unsigned)p.n_pages) continue;  // (its tokens are zeros)
      const int64_t slot = ((int64_t)pg * p.h_kv + h) * p.page_size + ((pos + t) & (p.page_size - 1));
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const void* pool = kv ? p.v_pool : p.k_pool;
        if (FMT == PAD_KV_FP4) {
          x[u][kv].x = __ldcg(static_cast<const uint32_t*>(pool) + slot * L + c);
          sc[u][kv] = __ldcg((kv ? p.v_scale : p.k_scale) + slot * (D / 16) + (c >> 1));
        } else if (FMT == PAD_KV_FP8) {
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
        if (FMT == PAD_KV_FP4) {
          const uint32_t m = (sc[u][kv] << 7) * 0x10001u;  // the scale as f16, twice
          uint32_t h[4];
          f16_of_e2m1(x[u][kv].x, h);
#pragma unroll
          for (int j = 0; j < 4; ++j) h[j] = bf16_of_f16(f16_times(h[j], m));
          o = make_uint4(h[0], h[1], h[2], h[3]);
        } else if (FMT == PAD_KV_FP8) {
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

template <int D, int FMT>
cudaError_t append(const ChunkParams& p, const ChunkPages* work, int n, const void* k_new, const void* v_new,
                   int64_t stride, void* k_pool, void* v_pool, uint8_t* ks, uint8_t* vs, cudaStream_t s) {
  return launch_early(false, chunk_append_kernel<D, FMT>, dim3(n), kThreads, 0, s, p, work, static_cast<const __nv_bfloat16*>(k_new),
                      static_cast<const __nv_bfloat16*>(v_new), stride, k_pool, v_pool, ks, vs);
}
template <int D, int FMT>
cudaError_t read(const ChunkParams& p, const ChunkRead* work, int n_events, int n, void* k_out, void* v_out, cudaStream_t s) {
  return launch_early(false, chunk_read_kernel<D, FMT, ChunkRead>, dim3(n), kThreads, 0, s, p, work, n_events,
                      static_cast<__nv_bfloat16*>(k_out), static_cast<__nv_bfloat16*>(v_out), nullptr, 0);
}

}  // namespace

int chunk_read_tokens() { return kReadTokens; }

cudaError_t launch_chunk_append(const ChunkParams& p, int head_dim, int kv_format, const ChunkPages* work, int n_work,
                                const void* k_new, const void* v_new, int64_t stride, void* k_pool, void* v_pool,
                                uint8_t* k_scale, uint8_t* v_scale, cudaStream_t s) {
  auto* f = head_dim == 128 ? (kv_format == PAD_KV_FP4 ? append<128, PAD_KV_FP4> : kv_format == PAD_KV_FP8 ? append<128, PAD_KV_FP8> : append<128, PAD_KV_BF16>)
                            : (kv_format == PAD_KV_FP4 ? append<64, PAD_KV_FP4> : kv_format == PAD_KV_FP8 ? append<64, PAD_KV_FP8> : append<64, PAD_KV_BF16>);
  return f(p, work, n_work, k_new, v_new, stride, k_pool, v_pool, k_scale, v_scale, s);
}

cudaError_t launch_chunk_read(const ChunkParams& p, int head_dim, int kv_format, const ChunkRead* work, int n_events,
                              int n_spans, void* k_out, void* v_out, cudaStream_t s) {
  auto* f = head_dim == 128 ? (kv_format == PAD_KV_FP4 ? read<128, PAD_KV_FP4> : kv_format == PAD_KV_FP8 ? read<128, PAD_KV_FP8> : read<128, PAD_KV_BF16>)
                            : (kv_format == PAD_KV_FP4 ? read<64, PAD_KV_FP4> : kv_format == PAD_KV_FP8 ? read<64, PAD_KV_FP8> : read<64, PAD_KV_BF16>);
  return f(p, work, n_events, n_spans, k_out, v_out, s);
}

cudaError_t launch_chunk_widen(const ChunkParams& p, int head_dim, const ChunkWiden* work, int n_events, int n_spans,
                               void* k_out, void* v_out, int32_t* table, int columns, cudaStream_t s) {
  auto* f = head_dim == 128 ? chunk_read_kernel<128, PAD_KV_FP4, ChunkWiden> : chunk_read_kernel<64, PAD_KV_FP4, ChunkWiden>;
  return launch_early(false, f, dim3(n_spans), kThreads, 0, s, p, work, n_events, static_cast<__nv_bfloat16*>(k_out),
                      static_cast<__nv_bfloat16*>(v_out), table, columns);
}

}  // namespace pad
