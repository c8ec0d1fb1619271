// Logits of a step's new tokens turned into probabilities (pad_chunk_probs): penalties for tokens that the row's context
// holds, biases, a mask, temperature, softmax.
//
// p = softmax(x / T) wants the row twice, for its maximum and sum and for the result.  A cluster takes a row, each CTA a
// slice of it that stays in its threads' registers between the two: a row is read once and written once, whatever its
// length, and what is done to it in between (penalties and biases at a few hundred places, the mask) costs no memory
// traffic.  As many clusters as the GPU holds take rows in turn.  Bound by the chain that a row is to its CTAs, 10 to 14 us
// (event, context, slice, maximum, sum, the cluster's meeting, the way out), and by the 36 rows that are under way
// together: 180 rows of 150001 in fp32 take 71 us, contexts of 2048 tokens on average, 57 without contexts; 64 rows of 131072
// in bf16 with a mask and biases 31 us; 5 rows of 32768 under 9 us, the host's call.  Where biases come with contexts, their
// planes take six bytes an entry of shared memory and bound the CTAs of an SM beside the registers: to two at 131072 entries, to
// one at 150001 (64 rows of it in bf16: 27 us without biases, 69 with 100 of them and a mask).
// (A cluster launched for each row: 77 us, a third of the GPU waiting for a whole cluster's room.  Two passes without
// clusters, the second joining the slices of the first: 74 us, 33 and 12.  The slice in shared memory instead of
// registers: 77, 35 and 9.  The next row's slice fetched to L2 ahead, its event looked up ahead: no gain.  Rows of one event
// one after the other, sharing what is counted: 70 where their length is a multiple of 16 bytes, 76 where it is not.)
//
// How often a token occurs in the context is counted in a plane of integers over the slice in shared memory: additions of
// whole numbers, whose order does not matter.  The pass for the maximum reads the counts beside the logits, where a
// context's token is among a warp's vectors at all, and changes each token once, by its whole count.  Biases are laid out
// the same way; a bitmap finds those of one token, whose first entry adds all, in order.
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

constexpr int kMaxCtas = 16;       // of a row
constexpr int kSlack = 16;         // entries of the planes beyond a slice
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f;

// A CTA's threads hold its slice in registers, kEach entries each; E: entries of a vector, 8 where logits or results are in
// 16 bits.  (us, 192 threads of 104 entries and 256 of 80.  64 rows of 131072: bf16 24.9 and 29.4, with biases and a mask 31.1 and
// 35.2; bf16 to fp32 31.0 and 36.1, 37.1 and 41.4; fp32 to bf16 24.7 and 24.1, 33.2 and 32.6.  180 rows of 150001: 61.7 and 76.2,
// 77.8 and 95.5, 60.3 and 60.2; in fp32 78 and 72.)
template <bool LONG, int E>
struct Shape {
  static constexpr int kThreads = !LONG && E == 8 ? 192 : 256, kEach = LONG ? 96 : E == 8 ? 104 : 80, kWarps = kThreads / 32;
  static constexpr int kSlice = kThreads * kEach / 32 * 32;
};
template <class TL, class TP>
constexpr int vector_entries() { return sizeof(TL) == 2 || sizeof(TP) == 2 ? 8 : 4; }
// Bytes of shared memory: counts (16 or 32 bits an entry), sums of biases and which entries have one or more than one,
// results on their way out where p's rows are not as far from 16-byte boundaries as the logits'.
__host__ __device__ inline size_t count_bytes(int slice, bool wide) { return (size_t)(slice + kSlack) * (wide ? 4 : 2); }
__host__ __device__ inline size_t bias_bytes(int slice) { return (size_t)(slice + kSlack) * 4 + (size_t)(slice / 32 + 1) * 8 / 16 * 16 + 16; }
__host__ __device__ inline size_t stage_bytes(int slice) { return (size_t)(slice + kSlack) * 4; }

struct Part {
  float m, l;    // maximum, sum of 2^(..) on it
  int32_t at;    // first place of the maximum
  int32_t nan;
};

// Joined with another part, lower places first among equals.
__device__ __forceinline__ void join_max(Part& a, const Part& b) {
  if (b.m > a.m || (b.m == a.m && b.at < a.at)) a.at = b.at;
  a.m = fmaxf(a.m, b.m);
  a.nan |= b.nan;
}

// The entries of a vector changed by what the context, the biases and the mask say of them.  at: place in the planes.
struct Change {
  const uint32_t* plane;
  const float* bias;
  const uint32_t* words;
  float up, repetition, frequency, presence;
};
template <int E, bool WIDE>
__device__ __forceinline__ void penalise(float (&y)[E], const Change& h, int at) {
  uint32_t c[E];
#pragma unroll
  for (int u = 0; u < E; u += 4) {
    if (WIDE) {
      const uint4 w = *reinterpret_cast<const uint4*>(h.plane + at + u);
      c[u] = w.x, c[u + 1] = w.y, c[u + 2] = w.z, c[u + 3] = w.w;
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(h.plane + (at + u) / 2);
      c[u] = w.x & 0xffffu, c[u + 1] = w.x >> 16, c[u + 2] = w.y & 0xffffu, c[u + 3] = w.y >> 16;
    }
  }
#pragma unroll
  for (int u = 0; u < E; ++u) {
    const float v = y[u] * (y[u] > 0.f ? h.up : h.repetition) - fmaf(h.frequency, (float)c[u], h.presence);
    if (c[u]) y[u] = v;
  }
}
template <int E>
__device__ __forceinline__ void add_bias(float (&y)[E], const Change& h, int at) {
#pragma unroll
  for (int u = 0; u < E; u += 4) {
    const float4 f = *reinterpret_cast<const float4*>(h.bias + at + u);
    y[u] += f.x, y[u + 1] += f.y, y[u + 2] += f.z, y[u + 3] += f.w;
  }
}
template <int E>
__device__ __forceinline__ void keep_allowed(float (&y)[E], const Change& h, int token, int n_words) {
  const int w0 = token >> 5;  // (of a row's first vector: -1 where it begins before the row)
  const uint32_t bits = __funnelshift_r(w0 >= 0 ? __ldg(h.words + w0) : 0u, w0 + 1 < n_words ? __ldg(h.words + w0 + 1) : 0u, token & 31);
#pragma unroll
  for (int u = 0; u < E; ++u)
    if (!((bits >> u) & 1u)) y[u] = kNegInf;
}

// WIDE: 32-bit counts.
template <class TL, class TP, bool LONG, bool WIDE>
__global__ void __launch_bounds__((Shape<LONG, vector_entries<TL, TP>()>::kThreads), LONG ? 1 : 2)
    probs_kernel(const __grid_constant__ ChunkProbs a, const ChunkVerify* __restrict__ work, int rows, int slice, int staged) {
  constexpr int E = vector_entries<TL, TP>();
  using S = Shape<LONG, E>;
  constexpr int T = S::kThreads, K = S::kEach / E;  // entries of a vector, vectors of a thread
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ Part warp_part[S::kWarps];
  __shared__ Part both[2][kMaxCtas];  // of the row at hand and the one before
  __shared__ ChunkVerify mine;
  __shared__ int event;
  __shared__ uint32_t touched[S::kWarps];  // bit k: a context's token is in the warp's k-th vectors
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), ctas = (int)cl.num_blocks();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  cl.barrier_arrive();  // (every CTA of the cluster runs before one writes into another's memory)
  const int stride = (int)gridDim.x / ctas;
  const int first_row = (int)blockIdx.x / ctas;
#pragma unroll 1
  for (int row = first_row, turn = 0; row < rows; row += stride, turn ^= 1) {
  Part* const parts = both[turn];
  // which event and place in its chunk the row has
  for (int e = threadIdx.x; e < a.n_events; e += T) {
    const ChunkVerify w = work[e];
    if (w.n_draft >= 0 && row >= w.tok0 && row <= w.tok0 + w.n_draft) mine = w, event = e;
  }

  // The row is cut into vectors such that the logits' 16-byte pieces are whole, and p's where that agrees: vector v of the
  // slice holds the tokens from lo + v E on.  Those that are not whole are the row's first and last alone.
  const TL* src = static_cast<const TL*>(a.logits) + row * a.logits_stride;
  TP* dst = static_cast<TP*>(a.p) + row * a.p_stride;
  const int from = (int)((reinterpret_cast<uintptr_t>(src) / sizeof(TL)) % (16 / sizeof(TL)));
  const int to = (int)((reinterpret_cast<uintptr_t>(dst) / sizeof(TP)) % (16 / sizeof(TP)));
  const int shift = E == 8 && sizeof(TL) == 4 && ((to - from) & 3) == 0 ? to : from;
  const int lo = rank * slice - shift, hi = min(lo + slice, a.vocab);  // (the first slice begins before the row)
  const int v0 = lo < 0 ? 1 : 0, v1 = hi > lo ? (hi - lo) / E : 0;     // whole vectors
  // the row's first or last vector, thread 0 of its slice has it beside its own (a row of one vector: as its last)
  const bool ragged_end = hi > lo && (hi - lo) % E != 0;
  float y[K][E], z[2][E];
  const int kf = v1 / T;  // vectors that every thread has
  if (v0 > 0) {           // (thread 0's first is no whole one)
#pragma unroll
    for (int u = 0; u < E; ++u) y[0][u] = kNegInf;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int v = threadIdx.x + k * T;
    if (k >= kf) {
#pragma unroll
      for (int u = 0; u < E; ++u) y[k][u] = kNegInf;
    }
    if (v >= v0 && v < v1) {
      const TL* at = src + (lo + v * E);
      if constexpr (sizeof(TL) == 4) {
#pragma unroll
        for (int u = 0; u < E; u += 4) {
          const float4 f = __ldcs(reinterpret_cast<const float4*>(at + u));
          y[k][u] = f.x, y[k][u + 1] = f.y, y[k][u + 2] = f.z, y[k][u + 3] = f.w;
        }
      } else {
        const uint4 r = __ldcs(reinterpret_cast<const uint4*>(at));
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int u = 0; u < E; ++u) y[k][u] = __uint_as_float(u & 1 ? w[u >> 1] & 0xffff0000u : w[u >> 1] << 16);
      }
    }
  }
  const bool edges = (v0 > 0 || ragged_end) && threadIdx.x == 0;
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int u = 0; u < E; ++u) {
      const int t = s == 0 ? lo + u : lo + v1 * E + u;
      z[s][u] = edges && (s == 0 ? v0 > 0 && v1 > 0 : ragged_end) && t >= 0 && t < hi ? (float)src[t] : kNegInf;
    }
  const bool counts = a.history != nullptr || a.tokens != nullptr, biases = a.bias_token != nullptr;
  uint32_t* plane = reinterpret_cast<uint32_t*>(smem);
  float* bias = reinterpret_cast<float*>(smem + (counts ? count_bytes(slice, WIDE) : 0));
  uint32_t* has = reinterpret_cast<uint32_t*>(bias + slice + kSlack);  // bit of entry k: in word k / 32, and whether again in the next row
  uint32_t* again = has + slice / 32 + 1;
  const int zeros = (int)(((counts ? count_bytes(slice, WIDE) : 0) + (biases ? bias_bytes(slice) : 0)) / 16);
  for (int i = threadIdx.x; i < zeros; i += T) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
  if (threadIdx.x < S::kWarps) touched[threadIdx.x] = 0u;
  __syncthreads();
  const int e = event;
  float temperature = 1.f;
  Change h{plane, bias, a.mask != nullptr ? a.mask + row * a.mask_stride : nullptr, 1.f, 1.f, 0.f, 0.f};
  if (a.params != nullptr) {
    const float* q = a.params + 4 * (int64_t)e;
    temperature = q[0], h.repetition = q[1], h.frequency = q[2], h.presence = q[3];
    h.up = __fdiv_rn(1.f, h.repetition);  // (a product with the rounded 1 / r: a warp's vectors are hardly without a token that occurs)
  }
  const uint32_t width = (uint32_t)max(hi - lo, 0);
  if (counts) {
    // adds one for each of a list's tokens that lie in the slice
    auto count = [&](const int32_t* list, int len) {
      constexpr int U = 8;
      for (int i0 = threadIdx.x; i0 < len; i0 += U * T) {
        int32_t t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) t[u] = i0 + u * T < len ? __ldg(list + i0 + u * T) : -1;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t at = (uint32_t)(t[u] - lo);
          if (t[u] >= 0 && at < width) {
            atomicAdd(plane + (WIDE ? at : at >> 1), WIDE ? 1u : 1u << (16 * (at & 1)));
            const uint32_t v = at / E;
            const uint32_t bit = 1u << (v / T);
            volatile uint32_t* const mark = touched + v % T / 32;
            if (!(*mark & bit)) atomicOr(touched + v % T / 32, bit);  // (contexts repeat themselves: few get here)
          }
        }
      }
    };
    const int past = a.history != nullptr ? min(max(a.history_len[e], 0), a.history_width) : 0;
    if (a.tokens != nullptr) count(a.tokens + mine.tok0, row - mine.tok0 + 1);
    count(a.history + (int64_t)e * a.history_width, past);
  }
  if (biases) {
    const int64_t first = (int64_t)e * a.bias_width;
    const int32_t* tok = a.bias_token + first;
    const float* value = a.bias_value + first;
    const int len = min(max(a.bias_len[e], 0), a.bias_width);
    for (int i = threadIdx.x; i < len; i += T) {
      const uint32_t at = (uint32_t)(tok[i] - lo);
      if (tok[i] < 0 || at >= width) continue;
      const uint32_t bit = 1u << (at & 31);
      if (atomicOr(has + (at >> 5), bit) & bit) atomicOr(again + (at >> 5), bit);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < len; i += T) {
      const int32_t me = tok[i];
      const uint32_t at = (uint32_t)(me - lo);
      if (me < 0 || at >= width) continue;
      float sum = value[i];
      if ((again[at >> 5] >> (at & 31)) & 1u) {
        bool before = false;
        for (int j = 0; j < i && !before; ++j) before = tok[j] == me;
        if (before) continue;
        for (int j = i + 1; j < len; ++j)
          if (tok[j] == me) sum += value[j];
      }
      bias[at] = sum;
    }
  }
  if (counts || biases) __syncthreads();

  // Penalties, biases, the mask, and the slice's maximum.
  const bool greedy = !(temperature > 0.f);
  const uint32_t hits = touched[warp];
  const int n_words = (a.vocab + 31) / 32;
  Part q{kNegInf, 0.f, 0x7fffffff, 0};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int v = threadIdx.x + k * T;
    if (k > kf) break;
    if ((k > 0 || v >= v0) && (k < kf || v < v1)) {
      if ((hits >> k) & 1u) penalise<E, WIDE>(y[k], h, v * E);
      if (biases) add_bias(y[k], h, v * E);
      if (h.words != nullptr) keep_allowed(y[k], h, lo + v * E, n_words);
    }
#pragma unroll
    for (int u = 0; u < E; u += 2) q.m = tc::max3f(q.m, y[k][u], y[k][u + 1]);
  }
  if (edges) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int v = s == 0 ? 0 : v1;
      if (s == 0 ? v0 == 0 || v1 == 0 : !ragged_end) continue;
      if (counts) penalise<E, WIDE>(z[s], h, v * E);
      if (biases) add_bias(z[s], h, v * E);
      if (h.words != nullptr) keep_allowed(z[s], h, lo + v * E, n_words);
#pragma unroll
      for (int u = 0; u < E; ++u) q.m = fmaxf(q.m, z[s][u]);
    }
  }
  auto block_join = [&](bool sum) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      if (sum) q.l += __shfl_xor_sync(0xffffffffu, q.l, o);
      else q.m = fmaxf(q.m, __shfl_xor_sync(0xffffffffu, q.m, o));
    }
    if (lane == 0) warp_part[warp] = q;
    __syncthreads();
    Part r = warp_part[0];
#pragma unroll
    for (int k = 1; k < S::kWarps; ++k) {
      if (sum) r.l += warp_part[k].l;
      else r.m = fmaxf(r.m, warp_part[k].m);
    }
    if (!sum) __syncthreads();
    q.m = r.m, q.l = r.l;
  };
  block_join(false);
  // (0 times it is 0 however small T, -infinity times it -infinity however large)
  const float c = fminf(fmaxf(__fdiv_rn(kLog2e, temperature), 0x1p-149f), 3.402823466e38f);
  if (greedy) {
    // the maximum's first place, and NaNs
    auto look = [&](float f, int token) {
      if (f == q.m) q.at = min(q.at, token);
      q.nan |= f != f;
    };
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int u = 0; u < E; ++u) look(y[k][u], lo + (int)(threadIdx.x + k * T) * E + u);
#pragma unroll
    for (int u = 0; u < E; ++u) look(z[0][u], lo + u), look(z[1][u], lo + v1 * E + u);
    q.at = __reduce_min_sync(0xffffffffu, q.at);
    q.nan = __any_sync(0xffffffffu, q.nan);
    if (lane == 0) warp_part[warp] = q;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < S::kWarps; ++k) {
      q.at = min(q.at, warp_part[k].at);
      q.nan |= warp_part[k].nan;
    }
  } else {
    // 2^((x - m) log2(e) / T) and their sum
    const float m = q.m == kNegInf ? 0.f : q.m;
    uint64_t l[2] = {0ull, 0ull};
    const uint64_t m2 = tc::f2pack(-m, -m), c2 = tc::f2pack(c, c);
    auto exps = [&](float (&f)[E]) {
#pragma unroll
      for (int u = 0; u < E; u += 2) {
        const uint64_t d = tc::fmul2(tc::fadd2(tc::f2pack(f[u], f[u + 1]), m2), c2);
        f[u] = tc::ex2(tc::f2lo(d)), f[u + 1] = tc::ex2(tc::f2hi(d));
        l[(u >> 1) & 1] = tc::fadd2(l[(u >> 1) & 1], tc::f2pack(f[u], f[u + 1]));
      }
    };
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (k > kf) break;
      exps(y[k]);
    }
    if (edges) exps(z[0]), exps(z[1]);
    l[0] = tc::fadd2(l[0], l[1]);
    q.l = tc::f2lo(l[0]) + tc::f2hi(l[0]);
    block_join(true);
  }
  if (row == first_row) cl.barrier_wait();
  if ((int)threadIdx.x < ctas) *cl.map_shared_rank(&parts[rank], threadIdx.x) = q;
  cl.sync();  // (another CTA writes to `parts` next two rows on, after it has met this one again)
  Part all{kNegInf, 0.f, 0x7fffffff, 0};
  if (lane < ctas) all = parts[lane];
  const float part_m = all.m;
#pragma unroll
  for (int o = kMaxCtas / 2; o > 0; o >>= 1)
    join_max(all, {__shfl_xor_sync(0xffffffffu, all.m, o), 0.f, __shfl_xor_sync(0xffffffffu, all.at, o), __shfl_xor_sync(0xffffffffu, all.nan, o)});
  float scale = 0.f;
  if (!greedy) {
    float l = all.l == 0.f ? 0.f : all.l * (part_m == kNegInf ? 1.f : tc::ex2((part_m - all.m) * c));  // (a NaN counts)
#pragma unroll
    for (int o = kMaxCtas / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    scale = l == 0.f ? 0.f : __fdiv_rn(q.m == kNegInf ? 1.f : tc::ex2((q.m - all.m) * c), l);
  } else if (all.nan || all.m == kNegInf) {
    all.at = -1;
  }
  // (the lower half of a warp has joined the parts, the upper half nothing)
  scale = __shfl_sync(0xffffffffu, scale, 0);
  const int one = __shfl_sync(0xffffffffu, all.at, 0);
  if (greedy) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int u = 0; u < E; ++u) y[k][u] = lo + (int)(threadIdx.x + k * T) * E + u == one ? 1.f : 0.f;
#pragma unroll
    for (int u = 0; u < E; ++u) z[0][u] = lo + u == one ? 1.f : 0.f, z[1][u] = lo + v1 * E + u == one ? 1.f : 0.f;
    scale = 1.f;
  }
  if (!staged) {
    const uint64_t scale2 = tc::f2pack(scale, scale);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int v = threadIdx.x + k * T;
      if (k > kf) break;
#pragma unroll
      for (int u = 0; u < E; u += 2) {
        const uint64_t d = tc::fmul2(tc::f2pack(y[k][u], y[k][u + 1]), scale2);
        y[k][u] = tc::f2lo(d), y[k][u + 1] = tc::f2hi(d);
      }
      if (v >= v0 && v < v1) {
        TP* at = dst + (lo + v * E);
        if constexpr (sizeof(TP) == 4) {
#pragma unroll
          for (int u = 0; u < E; u += 4) __stcs(reinterpret_cast<float4*>(at + u), make_float4(y[k][u], y[k][u + 1], y[k][u + 2], y[k][u + 3]));
        } else {
          __stcs(reinterpret_cast<uint4*>(at), make_uint4(tc::pack_bf16(y[k][0], y[k][1]), tc::pack_bf16(y[k][2], y[k][3]),
                                                          tc::pack_bf16(y[k][4 % E], y[k][5 % E]), tc::pack_bf16(y[k][6 % E], y[k][7 % E])));
        }
      }
    }
  } else {
    // through shared memory, so that the stores of a warp lie together
    float* out = reinterpret_cast<float*>(smem);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int v = threadIdx.x + k * T;
      if (v >= v0 && v < v1) {
#pragma unroll
        for (int u = 0; u < E; u += 4)
          *reinterpret_cast<float4*>(out + v * E + u) = make_float4(y[k][u] * scale, y[k][u + 1] * scale, y[k][u + 2] * scale, y[k][u + 3] * scale);
      }
    }
    __syncthreads();
#pragma unroll 4
    for (int i = v0 * E + threadIdx.x; i < v1 * E; i += T) dst[lo + i] = TP(out[i]);
  }
  if (edges) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int u = 0; u < E; ++u) {
        const int t = s == 0 ? lo + u : lo + v1 * E + u;
        if ((s == 0 ? v0 > 0 && v1 > 0 : ragged_end) && t >= 0 && t < hi) dst[t] = TP(z[s][u] * scale);
      }
  }
  __syncthreads();  // (shared memory is the next row's)
  }
}

template <class TL, class TP, bool LONG, bool WIDE>
cudaError_t launch(const ChunkProbs& a, const ChunkVerify* work, int rows, int ctas, int slice, bool staged, cudaStream_t s) {
  auto* kernel = probs_kernel<TL, TP, LONG, WIDE>;
  using S = Shape<LONG, vector_entries<TL, TP>()>;
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(count_bytes(S::kSlice, WIDE) + bias_bytes(S::kSlice)));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  const size_t planes = (a.history != nullptr || a.tokens != nullptr ? count_bytes(slice, WIDE) : 0) + (a.bias_token != nullptr ? bias_bytes(slice) : 0);
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(S::kThreads);
  cfg.dynamicSmemBytes = std::max(planes, staged ? stage_bytes(slice) : 0);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  // as many clusters as the GPU holds, each taking rows in turn: with one for each row, the 16 or eight CTAs' room comes free
  // piece by piece, and a third of the GPU waits for the rest of it
  static thread_local size_t known_smem[64];
  static thread_local int known_ctas[64], known[64];
  const bool keep = dev >= 0 && dev < 64;
  int most = keep && known[dev] > 0 && known_smem[dev] == cfg.dynamicSmemBytes && known_ctas[dev] == ctas ? known[dev] : 0;
  if (most == 0) {
    cfg.gridDim = dim3((unsigned)ctas);
    e = cudaOccupancyMaxActiveClusters(&most, kernel, &cfg);
    if (e != cudaSuccess) return e;
    if (most < 1) return cudaErrorLaunchOutOfResources;
    if (keep) known_smem[dev] = cfg.dynamicSmemBytes, known_ctas[dev] = ctas, known[dev] = most;
  }
  cfg.gridDim = dim3((unsigned)(std::min(rows, most) * ctas));
  return cudaLaunchKernelEx(&cfg, kernel, a, work, rows, slice, staged ? 1 : 0);
}

template <class TL, class TP>
cudaError_t launch(const ChunkProbs& a, const ChunkVerify* work, int rows, int ctas, int slice, cudaStream_t s) {
  // whether p's rows ever lie differently from the logits' within the entries that move together
  constexpr int64_t unit = sizeof(TL) == 2 && sizeof(TP) == 2 ? 8 : 4;
  const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(a.p) / sizeof(TP)) - (int64_t)(reinterpret_cast<uintptr_t>(a.logits) / sizeof(TL));
  const bool staged = apart % unit != 0 || (rows > 1 && (a.p_stride - a.logits_stride) % unit != 0);
  // (a count is at most the context's length)
  const bool wide = (int64_t)a.history_width + a.longest > 65535;
  if (slice <= Shape<false, vector_entries<TL, TP>()>::kSlice)
    return wide ? launch<TL, TP, false, true>(a, work, rows, ctas, slice, staged, s) : launch<TL, TP, false, false>(a, work, rows, ctas, slice, staged, s);
  return wide ? launch<TL, TP, true, true>(a, work, rows, ctas, slice, staged, s) : launch<TL, TP, true, false>(a, work, rows, ctas, slice, staged, s);
}

}  // namespace

int chunk_probs_max_vocab() { return kMaxCtas * Shape<true, 4>::kSlice - 64; }

cudaError_t launch_chunk_probs(const ChunkProbs& a, const ChunkVerify* work, int n_tokens, cudaStream_t s) {
  // a row over as many CTAs as leave each 2048 entries, eight where they hold it in 16 bits, up to 159232 entries (with 16 of half
  // as many threads 180 rows of 150001 take 82 us, not 71)
  int ctas = 1;
  while (ctas < kMaxCtas && a.vocab > ctas * (ctas < 8 ? 2048 : Shape<false, 8>::kSlice - 64)) ctas *= 2;
  const int slice = (a.vocab + 7 + 32 * ctas - 1) / (32 * ctas) * 32;  // (the first begins up to seven entries before the row)
  if ((int64_t)n_tokens * ctas > INT32_MAX) return cudaErrorInvalidValue;
  if (a.logits_bf16)
    return a.p_bf16 ? launch<__nv_bfloat16, __nv_bfloat16>(a, work, n_tokens, ctas, slice, s) : launch<__nv_bfloat16, float>(a, work, n_tokens, ctas, slice, s);
  return a.p_bf16 ? launch<float, __nv_bfloat16>(a, work, n_tokens, ctas, slice, s) : launch<float, float>(a, work, n_tokens, ctas, slice, s);
}

}  // namespace pad
