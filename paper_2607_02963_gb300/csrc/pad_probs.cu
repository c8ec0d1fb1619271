// Logits of a step's new tokens turned into probabilities (pad_chunk_probs): penalties for tokens that the row's context
// holds, biases, a mask, temperature, softmax.
//
// p = softmax(x / T) wants the row twice, for its maximum and sum and for the result.  A cluster takes a row, each CTA a
// slice of it that stays in shared memory in fp32 between the two: a row is read once and written once, whatever its
// length, and what is done to it in between (penalties and biases at a few hundred places, the mask) costs no memory
// traffic.  Bound by those bytes; short ones by the chain of a CTA's steps.
//
// How often a token occurs in the context is counted in a plane of integers over the slice: additions of whole numbers,
// whose order does not matter.  Going through the context again, whoever takes a token's count out of the plane first
// applies it, so that each token is changed once, by its whole count.  Biases use the plane to find tokens that occur
// once (added at once) and those that occur again (their first entry adds all, in order).
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

  // The slice, entry i at x[shift + i]: shared memory is as far from a 16-byte boundary as the row's memory is.
  constexpr int VL = 16 / (int)sizeof(TL), VP = 16 / (int)sizeof(TP);
  const TL* src = static_cast<const TL*>(a.logits) + row * a.logits_stride + lo;
  const int shift = (int)((reinterpret_cast<uintptr_t>(src) / sizeof(TL)) % VL);
  float* x = reinterpret_cast<float*>(smem);
  uint32_t* plane = reinterpret_cast<uint32_t*>(smem + (size_t)(slice + 8) * 4);
  const int vecs = n > 0 ? (shift + n + VL - 1) / VL : 0;
  if constexpr (sizeof(TL) == 4) {
    const uint32_t at = tc::smem_u32(x);
    for (int v = threadIdx.x; v < vecs; v += kThreads) {
      const int i0 = v * VL - shift;
      if (i0 >= 0 && i0 + VL <= n) {
        cp16(at + 16 * v, src + i0);
      } else {
#pragma unroll
        for (int u = 0; u < VL; ++u)
          if (i0 + u >= 0 && i0 + u < n) cp4(at + 16 * v + 4 * u, src + i0 + u);
      }
    }
  }
  // which event and place in its chunk the row has
  for (int e = threadIdx.x; e < a.n_events; e += kThreads) {
    const ChunkVerify w = work[e];
    if (w.n_draft >= 0 && row >= w.tok0 && row <= w.tok0 + w.n_draft) mine = w, event = e;
  }
  const bool counts = a.history != nullptr || a.tokens != nullptr, plane_used = counts || a.bias_token != nullptr;
  if (plane_used)
    for (int i = threadIdx.x; i < slice / (WIDE ? 1 : 2); i += kThreads) plane[i] = 0u;
  if constexpr (sizeof(TL) == 2) {
    constexpr int U = 4;
    for (int v0 = threadIdx.x; v0 < vecs; v0 += U * kThreads) {
      uint4 r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i0 = (v0 + u * kThreads) * VL - shift;
        if (i0 >= 0 && i0 + VL <= n) r[u] = *reinterpret_cast<const uint4*>(src + i0);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = v0 + u * kThreads, i0 = v * VL - shift;
        if (i0 >= 0 && i0 + VL <= n) {
          float4* d = reinterpret_cast<float4*>(x + v * VL);
          d[0] = make_float4(__uint_as_float(r[u].x << 16), __uint_as_float(r[u].x & 0xffff0000u), __uint_as_float(r[u].y << 16), __uint_as_float(r[u].y & 0xffff0000u));
          d[1] = make_float4(__uint_as_float(r[u].z << 16), __uint_as_float(r[u].z & 0xffff0000u), __uint_as_float(r[u].w << 16), __uint_as_float(r[u].w & 0xffff0000u));
        } else {
          for (int k = 0; k < VL; ++k)
            if (i0 + k >= 0 && i0 + k < n) x[v * VL + k] = __bfloat162float(src[i0 + k]);
        }
      }
    }
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
  auto token = [&](int i) { return i < past ? history[i] : a.tokens[mine.tok0 + (i - past)]; };
  if (counts) {
    for (int i = threadIdx.x; i < past + chunk; i += kThreads) {
      const int64_t k = (int64_t)token(i) - lo;
      if (k >= 0 && k < n) atomicAdd(plane + (WIDE ? k : k >> 1), WIDE ? 1u : 1u << (16 * (k & 1)));
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  if (counts) {
    for (int i = threadIdx.x; i < past + chunk; i += kThreads) {
      const int64_t k = (int64_t)token(i) - lo;
      if (k < 0 || k >= n) continue;
      uint32_t c;
      if (WIDE) c = atomicExch(plane + k, 0u);
      else c = (atomicAnd(plane + (k >> 1), (k & 1) ? 0xffffu : 0xffff0000u) >> (16 * (k & 1))) & 0xffffu;
      if (c == 0u) continue;
      const float v = x[shift + k];
      x[shift + k] = (v > 0.f ? __fdiv_rn(v, repetition) : v * repetition) - fmaf(frequency, (float)c, presence);
    }
    __syncthreads();
  }
  if (a.bias_token != nullptr) {
    const int64_t first = (int64_t)e * a.bias_width;
    const int32_t* tok = a.bias_token + first;
    const float* value = a.bias_value + first;
    const int len = min(max(a.bias_len[e], 0), a.bias_width);
    for (int i = threadIdx.x; i < len; i += kThreads) {
      const int64_t k = (int64_t)tok[i] - lo;
      if (k >= 0 && k < n) atomicAdd(plane + (WIDE ? k : k >> 1), WIDE ? 1u : 1u << (16 * (k & 1)));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < len; i += kThreads) {
      const int32_t me = tok[i];
      const int64_t k = (int64_t)me - lo;
      if (k < 0 || k >= n) continue;
      float sum = value[i];
      if ((WIDE ? plane[k] : (plane[k >> 1] >> (16 * (k & 1))) & 0xffffu) > 1u) {
        bool before = false;
        for (int j = 0; j < i && !before; ++j) before = tok[j] == me;
        if (before) continue;
        for (int j = i + 1; j < len; ++j)
          if (tok[j] == me) sum += value[j];
      }
      x[shift + k] += sum;
    }
    __syncthreads();
  }
  if (a.mask != nullptr) {  // (slices start at whole words)
    const uint32_t* word = a.mask + row * a.mask_stride + lo / 32;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += kThreads)
      if (!((word[i >> 5] >> lane) & 1u)) x[shift + i] = kNegInf;
    __syncthreads();
  }

  // the slice's maximum and its first place, then (T > 0) the sum of 2^((x - m) log2(e) / T), which takes x's place
  const bool greedy = !(temperature > 0.f);
  const int end = shift + n;
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
  Part q{kNegInf, 0.f, 0x7fffffff, 0};
  if (greedy) {
    for (int i = shift + threadIdx.x; i < end; i += kThreads) {
      const float v = x[i];
      if (v > q.m) q.m = v, q.at = lo + i - shift;
      q.nan |= v != v;
    }
  } else {
    for (int i = shift + threadIdx.x; i < end; i += kThreads) q.m = fmaxf(q.m, x[i]);
  }
  block_join(q, false);
  const float c = fminf(__fdiv_rn(kLog2e, temperature), 3.402823466e38f);  // (0 times it is 0 however small T)
  if (!greedy) {
    const float m = q.m == kNegInf ? 0.f : q.m;
    for (int i = shift + threadIdx.x; i < end; i += kThreads) {
      const float v = tc::ex2((x[i] - m) * c);
      x[i] = v;
      q.l += v;
    }
    block_join(q, true);
  }
  cl.barrier_wait();
  if ((int)threadIdx.x < ctas) *cl.map_shared_rank(&parts[rank], threadIdx.x) = q;
  cl.sync();  // (nobody reads or writes another CTA's memory after this)
  Part all = parts[0];
  for (int k = 1; k < ctas; ++k) join_max(all, parts[k]);
  float scale = 0.f;
  if (!greedy) {
    float l = 0.f;
    for (int k = 0; k < ctas; ++k)
      if (parts[k].l != 0.f) l += parts[k].l * (parts[k].m == kNegInf ? 1.f : tc::ex2((parts[k].m - all.m) * c));  // (a NaN counts)
    scale = l == 0.f ? 0.f : __fdiv_rn(q.m == kNegInf ? 1.f : tc::ex2((q.m - all.m) * c), l);
  } else if (all.nan || all.m == kNegInf) {
    all.at = -1;
  }
  TP* dst = static_cast<TP*>(a.p) + row * a.p_stride + lo;
  auto value_at = [&](int i) { return greedy ? (lo + i == all.at ? 1.f : 0.f) : x[shift + i] * scale; };
  const int skew = (int)((reinterpret_cast<uintptr_t>(dst) / sizeof(TP)) % VP);
  if (((shift - skew) & 3) == 0) {
    const int outs = n > 0 ? (skew + n + VP - 1) / VP : 0;
    for (int v = threadIdx.x; v < outs; v += kThreads) {
      const int i0 = v * VP - skew;
      if (i0 >= 0 && i0 + VP <= n) {
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
      } else {
#pragma unroll
        for (int u = 0; u < VP; ++u)
          if (i0 + u >= 0 && i0 + u < n) dst[i0 + u] = TP(value_at(i0 + u));
      }
    }
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
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMaxSlice + 8) * 4 + kMaxSlice * (WIDE ? 4 : 2));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  const bool plane = a.history != nullptr || a.tokens != nullptr || a.bias_token != nullptr;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)(slice + 8) * 4 + (plane ? (size_t)slice * (WIDE ? 4 : 2) : 0);
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
