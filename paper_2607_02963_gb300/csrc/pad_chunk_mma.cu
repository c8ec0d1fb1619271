// Attention of a step's chunk tokens on the warp-level tensor-core path (mma.sync): for few query rows
// per (event, kv-head), and the join of split key ranges for both paths.
//
// o_t = sum_j softmax_j(scale q_t . k_j) v_j over the keys j that token t sees.  An item is a range of
// keys for up to 32 rows (chunk tokens x the G query heads of a kv-head); a CTA of four warps takes an
// item and a kv-head.  Each warp takes every fourth block of 16 keys with rows of its own running
// maximum, sum and O (no meeting inside the loop), brought in by cp.async through a ring of its own;
// the four states are joined through shared memory at the end, and written to out, or to the partial
// states that chunk_merge_kernel joins, when the item is one of several of its rows.
//
// 8-bit caches: the codes are staged as they are (half the bytes in flight buys twice the keys) and
// widened in the fragments to f16, which holds every e4m3 value exactly, two codes an instruction; the
// scales of K multiply the scores, those of V the weights.  A K word holds four dimensions of a key
// (which Q's fragments follow: the order of a sum's terms is free), a V word four columns of a key, so
// that words of two keys give the pairs P.V wants without a transpose.  Range: Q rows are scaled by a
// power of two to below 2^15 (exact down to 2^-29 of their largest value), weights go in as p 2^(k - r + 15)
// with r the largest V scale so far; where a block's scales lie more than 2^12 below that, they go in as
// bf16, whose range is fp32's, and so do the codes.
// (Widened to bf16 throughout, four to five integer instructions a pair: 129 us for 333k cached tokens, 28/4 heads,
// no faster than the bf16 cache.)
//
// P goes into P.V rounded to bf16 (2^-8 of each weight at most; f16, 2^-11, with 8-bit keys, unless their scales lie far
// apart), at head_dim 64 too, where the one-token step's kernels keep more of it (two bf16 parts, or 32 bits up to 8
// rows); the row sum is that of the unrounded fp32 weights, and all states are fp32.
//
// 16 sequences x 1 token over 333k cached tokens, 28/4 heads: bf16 120 us, 5.6 TB/s, bound by memory; 8 bits 90 us,
// 3.8 TB/s, bound by the instructions that widen the codes and their latency.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <algorithm>
#include <cstdint>

#include "pad_chunk.h"
#include "pad_tc_common.cuh"

namespace pad {

namespace {

using tc::ex2;
using tc::pack_bf16;
using tc::smem_u32;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLn2 = 0.69314718055994531f;

// A warp's stages.  NB: 16-key groups of a block; two where the registers allow it (8 bits, 16 rows): the
// look-ups, the maximum and the waits are per block.
template <int D, bool FP8, int MT>
struct Ring {
  static constexpr int NB = FP8 && MT == 1 ? 2 : 1;
  static constexpr int kBlk = 16 * NB;                    // keys of a block
  static constexpr int kRow = FP8 ? D : 2 * D;            // bytes of a key
  static constexpr int kPitch = FP8 ? D + 16 : 2 * D;     // (8 bits: rows 4 banks apart; bf16: swizzled)
  static constexpr int kV = kBlk * kPitch;
  static constexpr int kScale = 2 * kBlk * kPitch;        // scale bytes: of K, then of V
  static constexpr int kMask = kScale + 2 * kBlk;         // which keys are there
  static constexpr int kStage = kMask + 16;
  // (three CTAs per SM at 16 rows, two at 32: 16 sequences x 1 token over 333k cached tokens, 28/4 heads, take 106 us
  // in 8 bits with two CTAs of three stages, 91 with three of two; bf16 122 and 119)
  static constexpr int kStages = MT == 1 ? 2 : FP8 ? 4 : 3;
  static constexpr int kWarpBytes = kStages * kStage;
};

template <int D, bool FP8, int MT>
constexpr int smem_bytes() {
  constexpr int ring = kWarps * Ring<D, FP8, MT>::kWarpBytes;
  constexpr int join = kWarps * 16 * MT * (D + 2) * 4;
  return ring > join ? ring : join;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, uint32_t n) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The two e4m3 codes in the lower half of x as f16, exactly.
__device__ __forceinline__ uint32_t f16_of_e4m3(uint32_t x) {
  uint32_t r;
  asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n}\n" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t f16_of_e4m3_hi(uint32_t x) {
  uint32_t r;
  asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, hi;\n}\n" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// A scale byte as a number: 2^(byte - 127), 0 for a group of zeros, and for one that holds a NaN (whose codes
// are 0) an infinity, which makes a NaN of them.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ bool not_finite2(uint32_t v) {  // either half's exponent is all ones
  return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
}

// FP8: of paged items; items of the prefix take the bf16 instance.
template <int D, bool FP8, int MT>
__global__ void __launch_bounds__(kThreads, MT == 1 ? 3 : 2) chunk_mma_kernel(const __grid_constant__ ChunkParams p,
                                                             const ChunkItem* __restrict__ items) {
  using R = Ring<D, FP8, MT>;
  constexpr int kRows = 16 * MT, NB = R::NB, kBlk = R::kBlk;
  constexpr uint32_t kEvery = kBlk == 32 ? 0xffffffffu : 0xffffu;
  extern __shared__ __align__(128) uint8_t smem[];
  const ChunkItem it = items[blockIdx.x / p.h_kv];
  const int h = (int)blockIdx.x % p.h_kv, G = p.group;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  uint8_t* ring = smem + warp * R::kWarpBytes;
  const uint32_t ring_at = smem_u32(ring);
  const int n_rows = it.ntok * G;

  grid_wait();
  grid_release();

  const int n_blocks = it.key1 > it.key0 ? (it.key1 - it.key0 + kBlk - 1) / kBlk : 0;
  const int mine = n_blocks > warp ? (n_blocks - warp + kWarps - 1) / kWarps : 0;
  const int32_t* table = p.page_table + (it.paged ? it.src * p.max_pages : 0);
  const uint32_t mul = (uint32_t)(p.h_kv * R::kRow * (it.paged ? p.page_size : 1));
  const uint32_t in_page = it.paged ? (uint32_t)(p.page_size - 1) : 0u;
  const int64_t base = (it.paged ? (int64_t)h * p.page_size : it.src * p.h_kv + h) * R::kRow + 16 * (lane % (R::kRow / 16));
  const uint8_t* kb = static_cast<const uint8_t*>(it.paged ? p.k_pool : p.k_prefix) + base;
  const uint8_t* vb = static_cast<const uint8_t*>(it.paged ? p.v_pool : p.v_prefix) + base;

  // page of this lane's key (one lane each) of the warp's i-th block
  auto page_of = [&](int i) -> int {
    const int key = it.key0 + (warp + kWarps * i) * kBlk + lane;
    return it.paged && i < mine && lane < kBlk && key < it.key1 ? __ldcg(table + (key >> p.page_shift)) : 0;
  };
  auto issue = [&](int i, int page, int stage) {
    if (i >= mine) return;
    const uint32_t st = ring_at + stage * R::kStage;
    const int k0 = it.key0 + (warp + kWarps * i) * kBlk, key = k0 + (lane & (kBlk - 1));
    bool ok = key < it.key1;
    if (it.paged && ok && lane < kBlk && (unsigned)page >= (unsigned)p.n_pages) {
      ok = false;
      pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_BOUNDS, (int)it.src, key >> p.page_shift, page);
    }
    const uint32_t there = __ballot_sync(0xffffffffu, ok) & kEvery;
    // a key lies index x mul (+ its slot within the page) from the base: its page, or of a prefix its token
    const uint32_t index = !ok ? 0u : (uint32_t)(it.paged ? page : key);
    constexpr int CH = R::kRow / 16, kIter = kBlk * CH / 32, RPI = 32 / CH;
    const int r0 = lane / CH, c = lane % CH;
#pragma unroll
    for (int j = 0; j < kIter; ++j) {
      const int row = j * RPI + r0;
      const uint32_t on = (there >> row) & 1u;
      const uint64_t off = (uint64_t)__shfl_sync(0xffffffffu, index, row) * mul + (on ? ((uint32_t)(k0 + row) & in_page) * R::kRow : 0u);
      const uint32_t dst = st + row * R::kPitch + 16 * (FP8 ? c : c ^ (row & 7));
      cp16(dst, kb + off, on * 16u);
      cp16(dst + R::kV, vb + off, on * 16u);
    }
    if (FP8) {  // four keys' scale bytes each (they share a page)
      const uint32_t four = (4 * lane) & (kBlk - 1), on = (there >> four) & 1u;
      const uint64_t at = (uint64_t)__shfl_sync(0xffffffffu, index, four) * (uint32_t)(p.h_kv * p.page_size) +
                          (on ? (uint32_t)(h * p.page_size) + ((uint32_t)(k0 + four) & in_page) : 0u);
      if (lane < kBlk / 2) cp4(st + R::kScale + 4 * lane, (lane < kBlk / 4 ? p.k_scale : p.v_scale) + at, on * 4u);
    }
    if (lane == 0) *reinterpret_cast<uint32_t*>(ring + stage * R::kStage + R::kMask) = there;
  };

  int page = page_of(0);
#pragma unroll
  for (int i = 0; i < R::kStages - 1; ++i) {
    const int next = page_of(i + 1);
    issue(i, page, i);
    asm volatile("cp.async.commit_group;" ::: "memory");
    page = next;
  }

  // Q fragments (rows g and g + 8 of each 16-row group), in the order of K's; 8 bits: as f16 of the row
  // times 2^-e, e such that its largest value lies in [2^14, 2^15), and what a score is to be multiplied by
  uint32_t qf[MT][D / 16][4];
  float qs[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = 16 * m + 8 * u + g;
      const bool on = r < n_rows;
      const __nv_bfloat16* src = p.q + (on ? (it.tok0 + r / G) * p.q_stride + (int64_t)(h * G + r % G) * D : 0);
      if (FP8) {
        uint2 x[D / 16];
        uint32_t top = 0u;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          x[j] = on ? __ldcg(reinterpret_cast<const uint2*>(src + 16 * j + 4 * t4)) : make_uint2(0u, 0u);
          top = max(max(max(top, x[j].x & 0x7fffu), max((x[j].x >> 16) & 0x7fffu, x[j].y & 0x7fffu)), (x[j].y >> 16) & 0x7fffu);
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // (the exponent kept where both powers of two are normal numbers; a row with a NaN or an infinity
        // keeps it whatever the scale)
        const int e = min(max((int)(top >> 7) - 127 - 14, -120), 113);
        const float down = __uint_as_float((uint32_t)(127 - e) << 23);
        qs[m][u] = p.scale_log2 * __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          qf[m][j][u] = pack_f16(__uint_as_float(x[j].x << 16) * down, __uint_as_float(x[j].x & 0xffff0000u) * down);
          qf[m][j][2 + u] = pack_f16(__uint_as_float(x[j].y << 16) * down, __uint_as_float(x[j].y & 0xffff0000u) * down);
        }
      } else {
        qs[m][u] = p.scale_log2;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          qf[m][j][u] = on ? __ldcg(reinterpret_cast<const uint32_t*>(src + 16 * j + 2 * t4)) : 0u;
          qf[m][j][2 + u] = on ? __ldcg(reinterpret_cast<const uint32_t*>(src + 16 * j + 2 * t4 + 8)) : 0u;
        }
      }
    }
  // keys that each of the thread's rows sees, and that all rows see
  int lim[MT][2], lim_all = 0x7fffffff;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = 16 * m + 8 * u + g;
      lim[m][u] = r < n_rows ? min(it.lim0 + (it.paged ? r / G : 0), it.key1) : 0;
      if (r < n_rows) lim_all = min(lim_all, lim[m][u]);
    }
  lim_all = __reduce_min_sync(0xffffffffu, lim_all);

  float o[MT][D / 8][4], mx[MT][2], l[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) o[m][i][u] = 0.f;
    mx[m][0] = mx[m][1] = kNegInf;
    l[m][0] = l[m][1] = 0.f;
  }
  // 8 bits: the largest V scale so far (a byte, 0: none), and 2^unit, which V scales are multiplied by: O is in
  // units of 2^-unit
  int ref = 0, unit = 0;

  int s_use = 0, s_fill = R::kStages - 1;  // the stages of this block and of the one being fetched
#pragma unroll 1
  for (int i = 0; i < mine; ++i) {
    {
      const int next = page_of(i + R::kStages);
      issue(i + R::kStages - 1, page, s_fill);
      asm volatile("cp.async.commit_group;" ::: "memory");
      page = next;
      s_fill = s_fill == R::kStages - 1 ? 0 : s_fill + 1;
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(R::kStages - 1) : "memory");
    __syncwarp();
    const uint8_t* st = ring + s_use * R::kStage;
    const uint32_t st_at = ring_at + s_use * R::kStage;
    const uint8_t* sv = st + R::kV;
    s_use = s_use == R::kStages - 1 ? 0 : s_use + 1;
    const uint32_t there = *reinterpret_cast<const uint32_t*>(st + R::kMask);
    const int k0 = it.key0 + (warp + kWarps * i) * kBlk;
    auto word = [](const uint8_t* a) { return *reinterpret_cast<const uint32_t*>(a); };

    float s[MT][2 * NB][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int b = 0; b < 2 * NB; ++b)
#pragma unroll
        for (int u = 0; u < 4; ++u) s[m][b][u] = 0.f;
    if (FP8) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int b = 0; b < 2 * NB; ++b) {
          const uint32_t w = word(st + (8 * b + g) * R::kPitch + 16 * j + 4 * t4);
          const uint32_t b0 = f16_of_e4m3(w), b1 = f16_of_e4m3_hi(w);
#pragma unroll
          for (int m = 0; m < MT; ++m) mma_f16(s[m][b], qf[m][j], b0, b1);
        }
    } else {
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          uint32_t kf[4];
          const int row = 16 * nb + (lane & 7) + ((lane >> 4) << 3), c = 2 * j + ((lane >> 3) & 1);
          ldsm4(kf, st_at + row * R::kPitch + 16 * (c ^ (row & 7)));
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            mma(s[m][2 * nb], qf[m][j], kf[0], kf[1]);
            mma(s[m][2 * nb + 1], qf[m][j], kf[2], kf[3]);
          }
        }
    }

    // a block that every row sees in full needs no mask
    const bool full = there == kEvery && k0 + kBlk <= lim_all;
    float kf4[2 * NB][2], vf4[2 * NB][2];  // 8 bits: the scales of the thread's keys
    bool far = false;                      // V scales too far apart for f16
    if (FP8) {
      const uint32_t byte = st[R::kScale + kBlk + (lane & (kBlk - 1))];
      const bool counts = ((there >> (lane & (kBlk - 1))) & 1u) && byte != 0u && byte != 255u;
      const int hi = (int)__reduce_max_sync(0xffffffffu, counts ? byte : 0u);
      const int lo = (int)__reduce_min_sync(0xffffffffu, counts ? byte : 255u);
      if (hi > ref) {
        const int now = min(142 - hi, 127);  // 2^15 for the largest scale (less where that is no fp32 number)
        const float down = ref == 0 ? 1.f : __uint_as_float((uint32_t)max(127 + now - unit, 0) << 23);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int c = 0; c < D / 8; ++c)
#pragma unroll
            for (int u = 0; u < 4; ++u) o[m][c][u] *= down;
        ref = hi;
        unit = now;
      }
      far = lo < ref - 12;
      const float up = __uint_as_float((uint32_t)(127 + unit) << 23);
#pragma unroll
      for (int b = 0; b < 2 * NB; ++b) {
        const uint32_t k2 = *reinterpret_cast<const uint16_t*>(st + R::kScale + 8 * b + 2 * t4);
        const uint32_t v2 = *reinterpret_cast<const uint16_t*>(st + R::kScale + kBlk + 8 * b + 2 * t4);
        kf4[b][0] = scale_value(k2 & 255u);
        kf4[b][1] = scale_value(k2 >> 8);
        vf4[b][0] = scale_value(v2 & 255u) * up;
        vf4[b][1] = scale_value(v2 >> 8) * up;
      }
    }

    uint32_t pf[MT][NB][4];
    bool hidden = false;  // some row here does not see some key of the block
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t see = kEvery;
        if (!full) {
          const int n = lim[m][u] - k0;  // keys of the block that the row sees, if they are there
          see = n >= kBlk ? kEvery : n <= 0 ? 0u : (1u << n) - 1u;
          hidden |= see != kEvery && 16 * m + 8 * u + g < n_rows;
          see &= there;
        }
        float top = kNegInf;
#pragma unroll
        for (int b = 0; b < 2 * NB; ++b)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            float& x = s[m][b][2 * u + v];
            x *= FP8 ? qs[m][u] * kf4[b][v] : qs[m][u];
            if (!full && !((see >> (8 * b + 2 * t4 + v)) & 1u)) x = kNegInf;
            top = fmaxf(top, x);
          }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float m_new = fmaxf(mx[m][u], top), base = m_new == kNegInf ? 0.f : m_new;
        // (the maximum of few blocks is above all before them)
        if (__any_sync(0xffffffffu, m_new > mx[m][u])) {
          const float alpha = ex2(mx[m][u] - base);
          l[m][u] *= alpha;
#pragma unroll
          for (int c = 0; c < D / 8; ++c) {
            o[m][c][2 * u] *= alpha;
            o[m][c][2 * u + 1] *= alpha;
          }
          mx[m][u] = m_new;
        }
#pragma unroll
        for (int b = 0; b < 2 * NB; ++b) {
          float a = ex2(s[m][b][2 * u] - base), c = ex2(s[m][b][2 * u + 1] - base);
          l[m][u] += a + c;
          if (FP8) {
            // (a NaN scale reaches the rows that see its key alone)
            a *= full || ((see >> (8 * b + 2 * t4)) & 1u) ? vf4[b][0] : 0.f;
            c *= full || ((see >> (8 * b + 2 * t4 + 1)) & 1u) ? vf4[b][1] : 0.f;
            pf[m][b >> 1][2 * (b & 1) + u] = far ? pack_bf16(a, c) : pack_f16(a, c);
          } else {
            pf[m][b >> 1][2 * (b & 1) + u] = pack_bf16(a, c);
          }
        }
      }

    // P.V.  A weight of 0 times a NaN or an infinity is not 0: where a row does not see all of the block
    // and its values are not all finite, the products are formed one by one instead.  (8-bit codes are
    // finite; a group's NaN is in its scale, and so in the weights of the rows that see it.)
    if (FP8) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int q = 0; q < D / 32; ++q) {
          const uint8_t* a = sv + (16 * nb + 2 * t4) * R::kPitch + 32 * q + 4 * g;
          const uint32_t w0 = word(a), w1 = word(a + R::kPitch), w2 = word(a + 8 * R::kPitch), w3 = word(a + 9 * R::kPitch);
          // column 32 q + 4 g + r of two keys each: column g of O tile 4 q + r
          const uint32_t x01 = __byte_perm(w0, w1, 0x5140), x23 = __byte_perm(w0, w1, 0x7362);
          const uint32_t y01 = __byte_perm(w2, w3, 0x5140), y23 = __byte_perm(w2, w3, 0x7362);
          if (!far) {
            const uint32_t b0[4] = {f16_of_e4m3(x01), f16_of_e4m3_hi(x01), f16_of_e4m3(x23), f16_of_e4m3_hi(x23)};
            const uint32_t b1[4] = {f16_of_e4m3(y01), f16_of_e4m3_hi(y01), f16_of_e4m3(y23), f16_of_e4m3_hi(y23)};
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int m = 0; m < MT; ++m) mma_f16(o[m][4 * q + r], pf[m][nb], b0[r], b1[r]);
          } else {
            // weights of any size: the codes as bf16
            const uint32_t one = 0x7b807b80u;  // 2^120 twice
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const uint32_t b0 = e4m3_pair(__byte_perm(r < 2 ? x01 : x23, 0u, r & 1 ? 0x3424u : 0x1404u), one);
              const uint32_t b1 = e4m3_pair(__byte_perm(r < 2 ? y01 : y23, 0u, r & 1 ? 0x3424u : 0x1404u), one);
#pragma unroll
              for (int m = 0; m < MT; ++m) mma(o[m][4 * q + r], pf[m][nb], b0, b1);
            }
          }
        }
    } else {
      const bool any_hidden = !full && __any_sync(0xffffffffu, hidden);
      auto load_v = [&](uint32_t (&vf)[4], int nb, int c) {  // O tiles c and c + 1
        const int row = 16 * nb + (lane & 7) + (((lane >> 3) & 1) << 3), ch = c + (lane >> 4);
        ldsm4t(vf, st_at + R::kV + row * R::kPitch + 16 * (ch ^ (row & 7)));
      };
      bool bad = false;
      if (any_hidden) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int c = 0; c < D / 8; c += 2) {
            uint32_t vf[4];
            load_v(vf, nb, c);
            bad |= not_finite2(vf[0]) | not_finite2(vf[1]) | not_finite2(vf[2]) | not_finite2(vf[3]);
          }
        bad = __any_sync(0xffffffffu, bad);
      }
      if (!bad) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int c = 0; c < D / 8; c += 2) {
            uint32_t vf[4];
            load_v(vf, nb, c);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              mma(o[m][c], pf[m][nb], vf[0], vf[1]);
              mma(o[m][c + 1], pf[m][nb], vf[2], vf[3]);
            }
          }
      } else {
        static_assert(FP8 || NB == 1, "the keys below are those of one group");
#pragma unroll 1
        for (int key = 0; key < 16; ++key) {
          const int src = 4 * g + ((key & 7) >> 1);
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint32_t w = __shfl_sync(0xffffffffu, key < 8 ? pf[m][0][u] : pf[m][0][2 + u], src);
              const float pw = __uint_as_float(key & 1 ? w & 0xffff0000u : w << 16);
              if (k0 + key >= lim[m][u] || !((there >> key) & 1u)) continue;
#pragma unroll
              for (int c = 0; c < D / 8; ++c) {
                const uint32_t v2 = word(sv + key * R::kPitch + 16 * (c ^ (key & 7)) + 4 * t4);
                o[m][c][2 * u] = fmaf(pw, __uint_as_float(v2 << 16), o[m][c][2 * u]);
                o[m][c][2 * u + 1] = fmaf(pw, __uint_as_float(v2 & 0xffff0000u), o[m][c][2 * u + 1]);
              }
            }
        }
      }
    }
    __syncwarp();
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // The four warps' states through shared memory: O rows, then (m, l).
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      l[m][u] += __shfl_xor_sync(0xffffffffu, l[m][u], 1);
      l[m][u] += __shfl_xor_sync(0xffffffffu, l[m][u], 2);
    }
  // (2^-unit in two factors: the whole may lie below fp32's normal numbers)
  const float unit_lo = __uint_as_float((uint32_t)(127 - unit / 2) << 23), unit_hi = __uint_as_float((uint32_t)(127 - (unit - unit / 2)) << 23);
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);
  float2* sml = reinterpret_cast<float2*>(so + kWarps * kRows * D);
  auto swap = [](int r) { return FP8 ? 4 * (r & 7) : 8 * (r & 3); };
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = 16 * m + 8 * u + g;
      float* dst = so + (warp * kRows + r) * D;
      // (a store's lanes touch distinct banks: the rows' columns are exchanged by groups of four or eight)
      if (FP8) {
#pragma unroll
        for (int q = 0; q < D / 32; ++q)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            float4 x;
            x.x = (o[m][4 * q][2 * u + v] * unit_lo) * unit_hi;
            x.y = (o[m][4 * q + 1][2 * u + v] * unit_lo) * unit_hi;
            x.z = (o[m][4 * q + 2][2 * u + v] * unit_lo) * unit_hi;
            x.w = (o[m][4 * q + 3][2 * u + v] * unit_lo) * unit_hi;
            *reinterpret_cast<float4*>(dst + ((32 * q + 4 * (2 * t4 + v)) ^ swap(r))) = x;
          }
      } else {
#pragma unroll
        for (int c = 0; c < D / 8; ++c)
          *reinterpret_cast<float2*>(dst + ((8 * c + 2 * t4) ^ swap(r))) = make_float2(o[m][c][2 * u], o[m][c][2 * u + 1]);
      }
      if (t4 == 0) sml[warp * kRows + r] = make_float2(mx[m][u], l[m][u]);
    }
  __syncthreads();
  constexpr int C4 = D / 4;  // float4 columns
  for (int i = threadIdx.x; i < n_rows * C4; i += kThreads) {
    const int r = i / C4, c = i % C4;
    float m_all = kNegInf, w[kWarps], l_all = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) m_all = fmaxf(m_all, sml[k * kRows + r].x);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float2 ml = sml[k * kRows + r];
      w[k] = ml.y == 0.f ? 0.f : ex2(ml.x - m_all);  // (l = 0: it saw nothing; a NaN passes)
      l_all += w[k] * ml.y;
    }
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      if (sml[k * kRows + r].y == 0.f) continue;
      const float4 x = *reinterpret_cast<const float4*>(so + (k * kRows + r) * D + ((4 * c) ^ swap(r)));
      a.x += w[k] * x.x;
      a.y += w[k] * x.y;
      a.z += w[k] * x.z;
      a.w += w[k] * x.w;
    }
    const int tok = r / G, head = h * G + r % G;
    if (it.part_row >= 0) {
      const int64_t row = it.part_row + (int64_t)tok * p.h_q + head;
      *reinterpret_cast<float4*>(p.part_o + row * D + 4 * c) = a;
      if (c == 0) p.part_ml[row] = make_float2(m_all, l_all);
    } else {
      const int64_t row = (int64_t)(it.tok0 + tok) * p.h_q + head;
      const float inv = l_all == 0.f ? 0.f : 1.f / l_all;
      if (p.out_bf16)
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + row * D + 4 * c) =
            make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
      else
        *reinterpret_cast<float4*>(static_cast<float*>(p.out) + row * D + 4 * c) =
            make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
      if (c == 0 && p.lse != nullptr) p.lse[row] = l_all == 0.f ? kNegInf : (m_all + log2f(l_all)) * kLn2;
    }
  }
}

// The split key ranges of one (token, query head) joined: weights 2^(m_s - max m), O and l added up in a fixed
// order.  WARPS warps share a row's splits (every WARPS-th each, eight under way at a time), and
// their sums are added through shared memory.
template <int D, int WARPS>
__global__ void __launch_bounds__(128) chunk_merge_kernel(const __grid_constant__ ChunkParams p,
                                                          const ChunkMerge* __restrict__ work) {
  constexpr int V = D / 32, ROWS = 4 / WARPS;  // columns of a lane, rows of a CTA
  __shared__ float red[4][D + 1];
  const ChunkMerge w = work[blockIdx.x];
  grid_wait();
  grid_release();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % WARPS;
  const int head = min((int)blockIdx.y * ROWS + warp / WARPS, p.h_q - 1);  // (a row too many is done twice)
  const int n = w.pre_n + w.page_n;
  auto row_of = [&](int s) {
    return (s < w.pre_n ? w.pre_row + s * w.pre_stride : w.page_row + (s - w.pre_n) * w.page_stride) + head;
  };
  float m_all = kNegInf;
  for (int s = lane; s < n; s += 32) m_all = fmaxf(m_all, p.part_ml[row_of(s)].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m_all = fmaxf(m_all, __shfl_xor_sync(0xffffffffu, m_all, o));
  float acc[V], l = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = 0.f;
  constexpr int U = 8;
  for (int s0 = part; s0 < n; s0 += U * WARPS) {
    float x[U][V], ws[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u * WARPS;
      ws[u] = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) x[u][v] = 0.f;
      if (s < n) {
        const int64_t row = row_of(s);
        const float2 ml = p.part_ml[row];
        const float* src = p.part_o + row * D + V * lane;
        // (l = 0: nothing was visible there, and its O may not have been written; a NaN passes.  A weight that
        // underflows to 0 multiplies all the same: what is not finite in its O stays so.)
        const bool seen = ml.y != 0.f;
        if (seen) {
          ws[u] = ex2(ml.x - m_all);
          l += ws[u] * ml.y;
        }
        if constexpr (V == 4) {
          const float4 t = *reinterpret_cast<const float4*>(src);
          x[u][0] = seen ? t.x : 0.f, x[u][1] = seen ? t.y : 0.f, x[u][2] = seen ? t.z : 0.f, x[u][3] = seen ? t.w : 0.f;
        } else {
          const float2 t = *reinterpret_cast<const float2*>(src);
          x[u][0] = seen ? t.x : 0.f, x[u][1] = seen ? t.y : 0.f;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] += ws[u] * x[u][v];
  }
  if constexpr (WARPS > 1) {
#pragma unroll
    for (int v = 0; v < V; ++v) red[warp][V * lane + v] = acc[v];
    if (lane == 0) red[warp][D] = l;
    __syncthreads();
    if (part != 0) return;
    for (int k = 1; k < WARPS; ++k) {
#pragma unroll
      for (int v = 0; v < V; ++v) acc[v] += red[warp + k][V * lane + v];
      l += red[warp + k][D];
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int64_t row = (int64_t)w.tok * p.h_q + head;
  if (p.out_bf16) {
    uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.out) + row * D) + (V / 2) * lane;
    if constexpr (V == 4)
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
    else
      *dst = pack_bf16(acc[0] * inv, acc[1] * inv);
  } else {
    float* dst = static_cast<float*>(p.out) + row * D + V * lane;
    if constexpr (V == 4)
      *reinterpret_cast<float4*>(dst) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    else
      *reinterpret_cast<float2*>(dst) = make_float2(acc[0] * inv, acc[1] * inv);
  }
  if (lane == 0 && p.lse != nullptr) p.lse[row] = l == 0.f ? kNegInf : (m_all + log2f(l)) * kLn2;
}

template <int D, bool FP8, int MT>
cudaError_t launch(const ChunkParams& p, bool early, const ChunkItem* items, int n, cudaStream_t s) {
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    e = cudaFuncSetAttribute(chunk_mma_kernel<D, FP8, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D, FP8, MT>());
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  if ((int64_t)n * p.h_kv > INT32_MAX) return cudaErrorInvalidValue;
  return launch_early(early, chunk_mma_kernel<D, FP8, MT>, dim3(n * p.h_kv), kThreads, smem_bytes<D, FP8, MT>(), s, p, items);
}

}  // namespace

cudaError_t launch_chunk_mma(const ChunkParams& p, int head_dim, bool fp8, int rows16, bool early, const ChunkItem* items,
                             int n_items, cudaStream_t s) {
  if (head_dim == 128) {
    if (rows16 == 1) return fp8 ? launch<128, true, 1>(p, early, items, n_items, s) : launch<128, false, 1>(p, early, items, n_items, s);
    return fp8 ? launch<128, true, 2>(p, early, items, n_items, s) : launch<128, false, 2>(p, early, items, n_items, s);
  }
  if (rows16 == 1) return fp8 ? launch<64, true, 1>(p, early, items, n_items, s) : launch<64, false, 1>(p, early, items, n_items, s);
  return fp8 ? launch<64, true, 2>(p, early, items, n_items, s) : launch<64, false, 2>(p, early, items, n_items, s);
}

cudaError_t launch_chunk_merge(const ChunkParams& p, int head_dim, int most, const ChunkMerge* work, int n_work, cudaStream_t s) {
  // four warps to a row where it has more splits than one of them keeps under way
  const bool many = most > 8;
  const dim3 grid(n_work, many ? p.h_q : (p.h_q + 3) / 4);
  auto* kernel = head_dim == 128 ? (many ? chunk_merge_kernel<128, 4> : chunk_merge_kernel<128, 1>)
                                 : (many ? chunk_merge_kernel<64, 4> : chunk_merge_kernel<64, 1>);
  return launch_early(true, kernel, grid, 128, 0, s, p, work);
}

}  // namespace pad
