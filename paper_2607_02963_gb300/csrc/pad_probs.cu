// Logits of a step's new tokens turned into probabilities (pad_chunk_probs): penalties for tokens that the row's context
// holds, biases, a mask, temperature, softmax.
//
// p = softmax(x / T) wants the row twice, for its maximum and sum and for the result.  A cluster takes a row, each CTA a
// slice of it that stays in shared memory in fp32 between the two: a row is read once and written once, whatever its
// length, and what is done to it in between (penalties and biases at a few hundred places, the mask) costs no memory
// traffic.  Bound by those bytes; short ones by the chain of a CTA's steps.
//
// How often a token occurs in the context is counted in a plane of integers over the slice: additions of whole numbers,
// whose order does not matter; the pass for the maximum reads the counts beside the logits and changes each token once,
// by its whole count.  Biases use the plane to find tokens that occur once (added at once) and those that occur again
// (their first entry adds all, in order).
// Sums are in fp32: a thread's terms, the warps', the slices', each in a fixed order.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <algorithm>
#include <cstdint>

#include "pad_chunk.h"
#include "pad_tc_common.cuh"

namespace pad {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCtas = 16;       // of a row
constexpr int kMaxSlice = 24576;   // entries of a CTA: 4 bytes each of logits and of counts
constexpr int kSlack = 16;          // entries of the buffers beyond a slice
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f;

struct Part {
  float m, l;    // maximum, sum of 2^(..) on it
  int32_t at;    // first place of the maximum
  int32_t nan;
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// Joined with another part, lower places first among equals.
__device__ __forceinline__ void join_max(Part& a, const Part& b) {
  if (b.m > a.m || (b.m == a.m && b.at < a.at)) a.at = b.at;
  a.m = fmaxf(a.m, b.m);
  a.nan |= b.nan;
}

// WIDE: 32-bit counts.
template <class TL, class TP, bool WIDE>
__global__ void __launch_bounds__(kThreads) probs_kernel(const __grid_constant__ ChunkProbs a, const ChunkVerify* __restrict__ work, int slice) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Part warp_part[kWarps];
  __shared__ Part parts[kMaxCtas];
  __shared__ ChunkVerify mine;
  __shared__ int event;
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), ctas = (int)cl.num_blocks();
  const int row = (int)blockIdx.x / ctas, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lo = min(a.vocab, rank * slice), n = min(slice, a.vocab - lo);
  cl.barrier_arrive();  // (every CTA of the cluster runs before one writes into another's memory)

  // The slice, entry i at x[shift + i] with its count at the same place of the plane: shared memory is as far from a
  // 16-byte boundary as the row's memory is.  What lies before and behind it in the same 16 bytes is -infinity.
  constexpr int VL = 16 / (int)sizeof(TL), VP = 16 / (int)sizeof(TP);
  const TL* src = static_cast<const TL*>(a.logits) + row * a.logits_stride + lo;
  const int shift = (int)((reinterpret_cast<uintptr_t>(src) / sizeof(TL)) % VL);
  float* x = reinterpret_cast<float*>(smem);
  uint32_t* plane = reinterpret_cast<uint32_t*>(smem + (size_t)(slice + kSlack) * 4);
  const int fours = (shift + n + 3) / 4;
  if (threadIdx.x < 8) {
    if ((int)threadIdx.x < shift) x[threadIdx.x] = kNegInf;
    x[shift + n + threadIdx.x] = kNegInf;
  }
  // whole pieces of 16 bytes [v0, v1), and what is left before and behind them
  const int v0 = shift > 0 ? 1 : 0, v1 = max(v0, (shift + n) / VL);
  const int head = min(n, v0 * VL - shift), tail = max(head, v1 * VL - shift);
  if constexpr (sizeof(TL) == 4) {
    const uint32_t at = tc::smem_u32(x);
#pragma unroll 4
    for (int v = v0 + threadIdx.x; v < v1; v += kThreads) cp16(at + 16 * v, src + v * VL - shift);
    if ((int)threadIdx.x < head) cp4(at + 4 * (shift + threadIdx.x), src + threadIdx.x);
    if ((int)threadIdx.x < n - tail) cp4(at + 4 * (shift + tail + threadIdx.x), src + tail + threadIdx.x);
  }
  // which event and place in its chunk the row has
  for (int e = threadIdx.x; e < a.n_events; e += kThreads) {
    const ChunkVerify w = work[e];
    if (w.n_draft >= 0 && row >= w.tok0 && row <= w.tok0 + w.n_draft) mine = w, event = e;
  }
  const bool counts = a.history != nullptr || a.tokens != nullptr, plane_used = counts || a.bias_token != nullptr;
  if (plane_used)
    for (int i = threadIdx.x; i < (slice + kSlack) / (WIDE ? 4 : 8); i += kThreads) reinterpret_cast<uint4*>(plane)[i] = make_uint4(0u, 0u, 0u, 0u);
  if constexpr (sizeof(TL) == 2) {
    constexpr int U = 4;
    for (int w = v0 + threadIdx.x; w < v1; w += U * kThreads) {
      uint4 r[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (w + u * kThreads < v1) r[u] = *reinterpret_cast<const uint4*>(src + (w + u * kThreads) * VL - shift);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (w + u * kThreads >= v1) break;
        float4* d = reinterpret_cast<float4*>(x + (w + u * kThreads) * VL);
        d[0] = make_float4(__uint_as_float(r[u].x << 16), __uint_as_float(r[u].x & 0xffff0000u), __uint_as_float(r[u].y << 16), __uint_as_float(r[u].y & 0xffff0000u));
        d[1] = make_float4(__uint_as_float(r[u].z << 16), __uint_as_float(r[u].z & 0xffff0000u), __uint_as_float(r[u].w << 16), __uint_as_float(r[u].w & 0xffff0000u));
      }
    }
    if ((int)threadIdx.x < head) x[shift + threadIdx.x] = __bfloat162float(src[threadIdx.x]);
    if ((int)threadIdx.x < n - tail) x[shift + tail + threadIdx.x] = __bfloat162float(src[tail + threadIdx.x]);
  }
  __syncthreads();
  const int e = event;
  float temperature = 1.f, repetition = 1.f, frequency = 0.f, presence = 0.f;
  if (a.params != nullptr) {
    const float* q = a.params + 4 * (int64_t)e;
    temperature = q[0], repetition = q[1], frequency = q[2], presence = q[3];
  }
  const int32_t* history = a.history != nullptr ? a.history + (int64_t)e * a.history_width : nullptr;
  const int past = history != nullptr ? min(max(a.history_len[e], 0), a.history_width) : 0;
  const int chunk = a.tokens != nullptr ? row - mine.tok0 + 1 : 0;
  // adds one for each of a list's tokens that lie in the slice
  auto count = [&](const int32_t* list, int len) {
    constexpr int U = 8;
    for (int i0 = threadIdx.x; i0 < len; i0 += U * kThreads) {
      int32_t t[U];
#pragma unroll
      for (int u = 0; u < U; ++u) t[u] = i0 + u * kThreads < len ? __ldg(list + i0 + u * kThreads) : -1;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t k = (uint32_t)t[u] - (uint32_t)lo;
        if (t[u] >= 0 && k < (uint32_t)n) {
          const uint32_t at = shift + k;
          atomicAdd(plane + (WIDE ? at : at >> 1), WIDE ? 1u : 1u << (16 * (at & 1)));
        }
      }
    }
  };
  if (counts) {
    count(history, past);
    count(a.tokens + mine.tok0, chunk);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  // the counts of the four entries from 4 v on
  auto counts_of = [&](int v, uint32_t (&c)[4]) -> bool {
    if (WIDE) {
      const uint4 w = reinterpret_cast<const uint4*>(plane)[v];
      c[0] = w.x, c[1] = w.y, c[2] = w.z, c[3] = w.w;
    } else {
      const uint2 w = reinterpret_cast<const uint2*>(plane)[v];
      c[0] = w.x & 0xffffu, c[1] = w.x >> 16, c[2] = w.y & 0xffffu, c[3] = w.y >> 16;
    }
    return (c[0] | c[1] | c[2] | c[3]) != 0u;
  };
  // (a product with the rounded 1 / r: entries that occur are few, but hardly a warp's pass is without one)
  const float up = __fdiv_rn(1.f, repetition);
  auto penalised = [&](float v, uint32_t c) {
    const float y = v * (v > 0.f ? up : repetition) - fmaf(frequency, (float)c, presence);
    return c == 0u ? v : y;
  };
  if (a.bias_token != nullptr) {
    if (counts) {
      for (int v = threadIdx.x; v < fours; v += kThreads) {
        uint32_t c[4];
        if (!counts_of(v, c)) continue;
#pragma unroll
        for (int u = 0; u < 4; ++u) x[4 * v + u] = penalised(x[4 * v + u], c[u]);
        if (WIDE) reinterpret_cast<uint4*>(plane)[v] = make_uint4(0u, 0u, 0u, 0u);
        else reinterpret_cast<uint2*>(plane)[v] = make_uint2(0u, 0u);
      }
      __syncthreads();
    }
    const int64_t first = (int64_t)e * a.bias_width;
    const int32_t* tok = a.bias_token + first;
    const float* value = a.bias_value + first;
    const int len = min(max(a.bias_len[e], 0), a.bias_width);
    count(tok, len);
    __syncthreads();
    for (int i = threadIdx.x; i < len; i += kThreads) {
      const int32_t me = tok[i];
      const uint32_t k = (uint32_t)me - (uint32_t)lo, at = shift + k;
      if (me < 0 || k >= (uint32_t)n) continue;
      float sum = value[i];
      if ((WIDE ? plane[at] : (plane[at >> 1] >> (16 * (at & 1))) & 0xffffu) > 1u) {
        bool before = false;
        for (int j = 0; j < i && !before; ++j) before = tok[j] == me;
        if (before) continue;
        for (int j = i + 1; j < len; ++j)
          if (tok[j] == me) sum += value[j];
      }
      x[at] += sum;
    }
    __syncthreads();
  }
  // Penalties (where biases did not want them first) and the mask, and the slice's maximum.
  const bool apply = counts && a.bias_token == nullptr;
  const bool greedy = !(temperature > 0.f);
  const uint32_t* words = a.mask != nullptr ? a.mask + row * a.mask_stride + lo / 32 : nullptr;  // (slices start at whole words)
  const int n_words = (n + 31) / 32;
  Part q{kNegInf, 0.f, 0x7fffffff, 0};
#pragma unroll 2
  for (int v = threadIdx.x; v < fours; v += kThreads) {
    float4 f = reinterpret_cast<const float4*>(x)[v];
    float y[4] = {f.x, f.y, f.z, f.w};
    bool changed = false;
    uint32_t c[4];
    if (apply && counts_of(v, c)) {
      changed = true;
#pragma unroll
      for (int u = 0; u < 4; ++u) y[u] = penalised(y[u], c[u]);
    }
    if (words != nullptr) {
      const int i0 = 4 * v - shift, w0 = i0 >> 5;  // (of a first place before the slice: -1)
      const uint32_t bits = __funnelshift_r(w0 >= 0 ? __ldg(words + w0) : 0u, w0 + 1 < n_words ? __ldg(words + w0 + 1) : 0u, i0 & 31);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (!((bits >> u) & 1u)) y[u] = kNegInf, changed = true;
    }
    if (changed) reinterpret_cast<float4*>(x)[v] = make_float4(y[0], y[1], y[2], y[3]);
    if (greedy) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (y[u] > q.m) q.m = y[u], q.at = lo + 4 * v + u - shift;
        q.nan |= y[u] != y[u];
      }
    } else {
      q.m = fmaxf(tc::max3f(y[0], y[1], y[2]), fmaxf(y[3], q.m));
    }
  }

  // the maximum's first place, then (T > 0) the sum of 2^((x - m) log2(e) / T), which takes x's place
  auto block_join = [&](Part& q, bool sum) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const Part b{__shfl_xor_sync(0xffffffffu, q.m, o), 0.f, __shfl_xor_sync(0xffffffffu, q.at, o), __shfl_xor_sync(0xffffffffu, q.nan, o)};
      const float l = __shfl_xor_sync(0xffffffffu, q.l, o);
      if (sum) q.l += l;
      else join_max(q, b);
    }
    if (lane == 0) warp_part[warp] = q;
    __syncthreads();
    Part r = warp_part[0];
#pragma unroll
    for (int k = 1; k < kWarps; ++k) {
      if (sum) r.l += warp_part[k].l;
      else join_max(r, warp_part[k]);
    }
    __syncthreads();
    q = r;
  };
  block_join(q, false);
  const float c = fminf(__fdiv_rn(kLog2e, temperature), 3.402823466e38f);  // (0 times it is 0 however small T)
  if (!greedy) {
    const float m = q.m == kNegInf ? 0.f : q.m;
    // (by places from the slice's start: the sum does not depend on where in memory the row begins)
#pragma unroll 4
    for (int i = shift + threadIdx.x; i < shift + n; i += kThreads) {
      const float v = tc::ex2((x[i] - m) * c);
      x[i] = v;
      q.l += v;
    }
    block_join(q, true);
  }
  cl.barrier_wait();
  if ((int)threadIdx.x < ctas) *cl.map_shared_rank(&parts[rank], threadIdx.x) = q;
  cl.sync();  // (nobody reads or writes another CTA's memory after this)
  Part all{kNegInf, 0.f, 0x7fffffff, 0};
  if (lane < ctas) all = parts[lane];
  const float part_m = all.m;
#pragma unroll
  for (int o = kMaxCtas / 2; o > 0; o >>= 1)
    join_max(all, {__shfl_xor_sync(0xffffffffu, all.m, o), 0.f, __shfl_xor_sync(0xffffffffu, all.at, o), __shfl_xor_sync(0xffffffffu, all.nan, o)});
  // (lanes of the upper half repeat nothing: their parts are empty, and only the lower half is read)
  float scale = 0.f;
  if (!greedy) {
    float l = all.l == 0.f ? 0.f : all.l * (part_m == kNegInf ? 1.f : tc::ex2((part_m - all.m) * c));  // (a NaN counts)
#pragma unroll
    for (int o = kMaxCtas / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    scale = l == 0.f ? 0.f : __fdiv_rn(q.m == kNegInf ? 1.f : tc::ex2((q.m - all.m) * c), l);
  } else if (all.nan || all.m == kNegInf) {
    all.at = -1;
  }
  scale = __shfl_sync(0xffffffffu, scale, 0);
  all.at = __shfl_sync(0xffffffffu, all.at, 0);
  TP* dst = static_cast<TP*>(a.p) + row * a.p_stride + lo;
  auto value_at = [&](int i) { return greedy ? (lo + i == all.at ? 1.f : 0.f) : x[shift + i] * scale; };
  const int skew = (int)((reinterpret_cast<uintptr_t>(dst) / sizeof(TP)) % VP);
  if (((shift - skew) & 3) == 0) {
    const int o0 = skew > 0 ? 1 : 0, o1 = max(o0, (skew + n) / VP), front = min(n, o0 * VP - skew), back = max(front, o1 * VP - skew);
#pragma unroll 2
    for (int v = o0 + threadIdx.x; v < o1; v += kThreads) {
      const int i0 = v * VP - skew;
      float y[VP];
#pragma unroll
      for (int u = 0; u < VP; u += 4) {
        const float4 f = *reinterpret_cast<const float4*>(x + shift + i0 + u);
        y[u] = f.x * scale, y[u + 1] = f.y * scale, y[u + 2] = f.z * scale, y[u + 3] = f.w * scale;
      }
      if (greedy) {
#pragma unroll
        for (int u = 0; u < VP; ++u) y[u] = lo + i0 + u == all.at ? 1.f : 0.f;
      }
      if constexpr (sizeof(TP) == 4)
        __stcs(reinterpret_cast<float4*>(dst + i0), make_float4(y[0], y[1], y[2], y[3]));
      else
        __stcs(reinterpret_cast<uint4*>(dst + i0), make_uint4(tc::pack_bf16(y[0], y[1]), tc::pack_bf16(y[2], y[3]), tc::pack_bf16(y[4], y[5]), tc::pack_bf16(y[6], y[7])));
    }
    if ((int)threadIdx.x < front) dst[threadIdx.x] = TP(value_at(threadIdx.x));
    if ((int)threadIdx.x < n - back) dst[back + threadIdx.x] = TP(value_at(back + threadIdx.x));
  } else {
    for (int i = threadIdx.x; i < n; i += kThreads) dst[i] = TP(value_at(i));
  }
}

template <class TL, class TP, bool WIDE>
cudaError_t launch(const ChunkProbs& a, const ChunkVerify* work, int rows, int ctas, int slice, cudaStream_t s) {
  auto* kernel = probs_kernel<TL, TP, WIDE>;
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMaxSlice + kSlack) * (WIDE ? 8 : 6));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  const bool plane = a.history != nullptr || a.tokens != nullptr || a.bias_token != nullptr;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)(slice + kSlack) * (plane ? (WIDE ? 8 : 6) : 4);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, work, slice);
}

}  // namespace

int chunk_probs_max_vocab() { return kMaxCtas * kMaxSlice; }

cudaError_t launch_chunk_probs(const ChunkProbs& a, const ChunkVerify* work, int n_tokens, cudaStream_t s) {
  // a row over as many CTAs as leave each 2048 entries
  int ctas = 1;
  while (ctas < kMaxCtas && a.vocab > ctas * 2048) ctas *= 2;
  const int slice = (a.vocab + 32 * ctas - 1) / (32 * ctas) * 32;
  if ((int64_t)n_tokens * ctas > INT32_MAX) return cudaErrorInvalidValue;
  // (a count is at most the context's length)
  const bool wide = (int64_t)a.history_width + a.longest > 65535 || a.bias_width > 65535;
  if (a.logits_bf16) {
    if (a.p_bf16) return wide ? launch<__nv_bfloat16, __nv_bfloat16, true>(a, work, n_tokens, ctas, slice, s) : launch<__nv_bfloat16, __nv_bfloat16, false>(a, work, n_tokens, ctas, slice, s);
    return wide ? launch<__nv_bfloat16, float, true>(a, work, n_tokens, ctas, slice, s) : launch<__nv_bfloat16, float, false>(a, work, n_tokens, ctas, slice, s);
  }
  if (a.p_bf16) return wide ? launch<float, __nv_bfloat16, true>(a, work, n_tokens, ctas, slice, s) : launch<float, __nv_bfloat16, false>(a, work, n_tokens, ctas, slice, s);
  return wide ? launch<float, float, true>(a, work, n_tokens, ctas, slice, s) : launch<float, float, false>(a, work, n_tokens, ctas, slice, s);
}

}  // namespace pad
