// Verification of drafted tokens (pad_draft_verify): drafted token i, x_i, is kept while
// u_i q_i(x_i) < p_i(x_i); at the first position a that fails the next token is drawn from
// max(p_a - q_a, 0), after a whole accepted draft from p itself.  Together these give tokens
// distributed as p.
//
// The draw needs the sum over the vocabulary and the place where the running sum passes a point of it.
// The weights are integers, floor(2^38 min(r, 1)), and sums of integers do not depend on their order:
// any split over threads gives the token that one running sum would.  2^38 keeps what fp32 has of
// a probability down to 4e-12, and leaves 25 bits for the number of terms.
//
// Bound by bytes: one row of p and one of q per event.  A cluster of eight CTAs takes an event; each sums
// an eighth of the rows, warp by warp over consecutive entries, hands its sum to the others through
// distributed shared memory, and the CTA that holds the point goes through the one warp's part it lies
// in again (a 128th of the row, from L2).  32 branches, vocabulary 150001, fp32: 12 us, 3.2 TB/s; one branch,
// vocabulary 32768: 7 us, which is the launch and the chain ahead of the row's loads (work entry, draft, its probabilities).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <algorithm>
#include <cstdint>

#include "pad_chunk.h"

namespace pad {

namespace {

namespace cg = cooperative_groups;

constexpr int kCtas = 8;       // of an event
constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }

// floor(2^38 min(r, 1)), 0 for a NaN, as its upper and lower 19 bits, each in the low bits of a float's pattern
// (above those of 2^23): adding 2^23 with rounding down leaves the floor there, and what it cuts off is
// exact in fp32.  (Patterns are added as they are; 64-bit shifts or conversions take twice the instructions.)
struct Halves {
  uint32_t hi, lo;
};
constexpr uint32_t kBase = 0x4b000000u;  // the pattern of 2^23
__device__ __forceinline__ Halves halves(float r) {
  const float x = fminf(fmaxf(r, 0.f), 1.f) * 524288.f;  // 2^19; fmaxf(NaN, 0) = 0
  const float t = __fadd_rd(x, 8388608.f);
  const float rest = x - (t - 8388608.f);
  return {__float_as_uint(t), __float_as_uint(__fmaf_rd(rest, 524288.f, 8388608.f))};
}
__device__ __forceinline__ int64_t weight(float r) {
  const Halves h = halves(r);
  return ((int64_t)(h.hi - kBase) << 19) + (int64_t)(h.lo - kBase);
}

__device__ __forceinline__ int64_t warp_sum(int64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <class T>
__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads)
    draft_verify_kernel(const __grid_constant__ ChunkParams pr, const ChunkVerify* __restrict__ work, int vocab,
                        const T* p, int64_t p_stride, const T* q, int64_t q_stride,
                        const int32_t* draft, const float* u_accept, const float* u_pick, int32_t* __restrict__ accepted, int32_t* __restrict__ token) {
  __shared__ int first_bad;
  __shared__ int64_t part[kWarps];       // sums of each warp's entries
  __shared__ int64_t sums[2][kCtas];     // of each CTA's: first round, second round
  __shared__ int64_t scan[kWarps];
  cg::cluster_group cl = cg::this_cluster();
  const int rank = (int)cl.block_rank(), e = (int)blockIdx.x / kCtas;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const ChunkVerify w = work[e];
  if (w.n_draft < 0) {  // (the whole cluster)
    if (rank == 0 && threadIdx.x == 0) accepted[e] = 0, token[e] = -1;
    return;
  }
  cl.barrier_arrive();  // (every CTA of the cluster runs before one writes into another's memory)
  if (threadIdx.x == 0) first_bad = w.n_draft;
  __syncthreads();
  for (int i = threadIdx.x; i < w.n_draft; i += kThreads) {
    const int x = draft[w.draft0 + i];
    bool ok = (unsigned)x < (unsigned)vocab;
    if (!ok && rank == 0) pad_set_error(pr.header, pr.gen, PAD_ERR_DEVICE_BOUNDS, e, i, x);
    if (ok)
      ok = __fmul_rn(u_accept[w.draft0 + i], value(q[(int64_t)(w.draft0 + i) * q_stride + x])) <
           value(p[(int64_t)(w.tok0 + i) * p_stride + x]);
    if (!ok) atomicMin(&first_bad, i);
  }
  __syncthreads();
  const int a = first_bad;
  const bool sub = a < w.n_draft;
  const T* pa = p + (int64_t)(w.tok0 + a) * p_stride;
  const T* qa = q + (sub ? (int64_t)(w.draft0 + a) * q_stride : 0);
  // this warp's entries: consecutive, the same number for every warp of the cluster
  const int per = (vocab + kCtas * kWarps - 1) / (kCtas * kWarps);
  auto begin_of = [&](int wp) { return (int)min((int64_t)vocab, (int64_t)(rank * kWarps + wp) * per); };
  const int lo = begin_of(warp), hi = min(vocab, lo + per);
  // first of the difference, where there is one; of p itself if it has no weight (or there is none)
  bool take = sub;
  int64_t total = 0, before = 0, mine = 0;
  for (int round = 0;; ++round) {
    uint32_t hi32 = 0, lo32 = 0, n = 0;  // (a thread adds up at most 2^12 + 8 entries: its sums stay below 2^32)
    constexpr int U = 8;
    for (int i0 = lo + lane; i0 < hi; i0 += 32 * U) {
      float x[U], y[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        x[j] = y[j] = 0.f;
        if (i0 + 32 * j < hi) {
          x[j] = value(pa[i0 + 32 * j]);
          if (take) y[j] = value(qa[i0 + 32 * j]);
        }
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const Halves h = halves(x[j] - y[j]);
        hi32 += h.hi;
        lo32 += h.lo;
      }
      n += U;
    }
    const int64_t s = warp_sum(((int64_t)(hi32 - n * kBase) << 19) + (int64_t)(lo32 - n * kBase));
    if (lane == 0) part[warp] = s;
    __syncthreads();
    if (round == 0) cl.barrier_wait();
    if (threadIdx.x < kCtas) {
      int64_t t = 0;
      for (int k = 0; k < kWarps; ++k) t += part[k];
      *cl.map_shared_rank(&sums[round][rank], threadIdx.x) = t;
    }
    cl.sync();  // (nobody reads another CTA's memory after this)
    total = before = 0;
#pragma unroll
    for (int k = 0; k < kCtas; ++k) {
      const int64_t v = sums[round][k];
      if (k < rank) before += v;
      total += v;
    }
    mine = sums[round][rank];
    if (total > 0 || !take) break;
    take = false;
  }
  if (rank == 0 && threadIdx.x == 0) {
    accepted[e] = a;
    if (total == 0) token[e] = -1;
  }
  if (total == 0) return;
  const float u = u_pick[e];
  const int64_t m = (int64_t)fminf(fmaxf(floorf(u * 16777216.f), 0.f), 16777215.f);  // (a NaN: 0)
  const int64_t goal = m * (total >> 24) + ((m * (total & 0xffffff)) >> 24) - before;
  if (goal < 0 || goal >= mine) return;  // (the whole CTA)
  int wp = 0;
  int64_t base = 0;
  while (wp < kWarps - 1 && base + part[wp] <= goal) base += part[wp++];
  // that warp's entries again, a few consecutive ones per thread
  const int wlo = begin_of(wp), whi = min(vocab, wlo + per);
  const int c = (whi - wlo + kThreads - 1) / kThreads, tlo = min(whi, wlo + (int)threadIdx.x * c), thi = min(whi, tlo + c);
  auto weight_of = [&](int i) { return weight(take ? value(pa[i]) - value(qa[i]) : value(pa[i])); };
  int64_t t = 0;
  for (int i = tlo; i < thi; ++i) t += weight_of(i);
  int64_t inc = t;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) scan[warp] = inc;
  __syncthreads();
  int64_t at = base + inc - t;
  for (int k = 0; k < warp; ++k) at += scan[k];
  if (at <= goal && goal < at + t) {
    int i = tlo;
    for (;; ++i) {
      at += weight_of(i);
      if (at > goal || i + 1 >= thi) break;
    }
    token[e] = i;
  }
}

template <class T>
cudaError_t launch(const ChunkParams& p, const ChunkVerify* work, int n, int vocab, const void* tp, int64_t ps,
                   const void* dq, int64_t qs, const int32_t* draft, const float* ua, const float* up, int32_t* acc,
                   int32_t* tok, cudaStream_t s) {
  return launch_early(false, draft_verify_kernel<T>, dim3(n * kCtas), kThreads, 0, s, p, work, vocab, static_cast<const T*>(tp), ps,
                      static_cast<const T*>(dq), qs, draft, ua, up, acc, tok);
}

}  // namespace

cudaError_t launch_draft_verify(const ChunkParams& p, const ChunkVerify* work, int n_events, int vocab, bool bf16,
                                const void* tp, int64_t p_stride, const void* dq, int64_t q_stride,
                                const int32_t* draft, const float* u_accept, const float* u_pick, int32_t* accepted,
                                int32_t* token, cudaStream_t s) {
  return bf16 ? launch<__nv_bfloat16>(p, work, n_events, vocab, tp, p_stride, dq, q_stride, draft, u_accept, u_pick, accepted, token, s)
              : launch<float>(p, work, n_events, vocab, tp, p_stride, dq, q_stride, draft, u_accept, u_pick, accepted, token, s);
}

}  // namespace pad
