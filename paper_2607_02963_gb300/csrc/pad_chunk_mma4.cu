// Attention of a step's chunk tokens over pages held in 4 bits, on the warp-level tensor-core path (mma.sync).
//
// o_t = sum_j softmax_j(scale q_t . k_j) v_j over the keys j that token t sees.  An item is a range of keys for up to 24
// rows (chunk tokens x the G query heads of a kv-head); a CTA of four warps takes an item and a kv-head, each warp every
// fourth block of 32 keys with states of its own, joined through shared memory at the end.
//
// The codes are widened in the fragments: a pair of codes to f16 (one conversion), times the group's scale (one product;
// code times scale is exact in f16, six significant bits up to 61440 and down to 2^-18).  That is most of the work, so
// everything else is laid out around it: keys are the M side of both products (S^T = K Q^T, O^T = V^T P^T), rows the N
// side in groups of eight, so that few rows leave no half of a 16-row tile empty, and a lane takes the words of whole
// groups (the order of the dimensions in a product is free, Q follows it), so that a scale is fetched once for 16 codes.
//   K: lane (g, t) widens the dimensions D/4 t .. of keys g and g + 8 of 16.
//   V: lane (g, t) widens the columns D/8 g .. of keys 2t, 2t + 1, 2t + 8, 2t + 9: two keys' nibbles are interleaved
//      first, so that a converted byte is a pair of keys.
//   P^T goes from the layout of S^T to that of an operand by a transposition of 8 x 8 halves (movmatrix).
// Q rows are scaled by a power of two to below 2^15 (exact down to 2^-29 of their largest value).
//
// P goes into P.V in f16 as 2^15 times the weight: 2^-11 of itself off at most, and 2^-40 where it is below 2^-29; the
// row sum is that of the unrounded fp32 weights, and all states are fp32.
//
// Bound by the products by the scales, which share a pipe with the MMAs (a scheduler's cycles for one A fragment, in registers
// alone: conversions and MMA 11, with the products 17), and by the issue slots, 62 % of them used: 16 sequences x 1 token
// over 350k cached tokens, 28/4 heads: 49 us, 4.1 TB/s (8 bits 91, bf16 121 over 333k).
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
constexpr int kBlk = 32;          // keys of a block
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kUp = 15.f;       // weights are held as 2^15 times themselves
// Scores (in powers of two) from which on one rounding of a score and of its row's maximum each, 2^-24 of them, may move a weight
// by more than 2^(1/8): 2^15 times it would leave f16 from 2^23 on.
constexpr float kFar = 0x1p20f;

// A warp's stages: the codes and scales of a block as they lie in the pages.
template <int D, int NT>
struct Ring {
  static constexpr int kRow = D / 2;                        // bytes of a key's codes,
  static constexpr int kScales = D / 16;                    // and of its scales
  static constexpr int kV = kBlk * kRow;
  static constexpr int kSK = 2 * kV;
  static constexpr int kSV = kSK + kBlk * kScales;
  static constexpr int kStage = kSV + kBlk * kScales;
  static constexpr int kStages = 3;  // (four CTAs of two stages take 55 us where four of three take 51: 350k tokens as above)
  static constexpr int kWarpBytes = kStages * kStage;
};

template <int D, int NT>
constexpr int smem_bytes() {
  constexpr int ring = kWarps * Ring<D, NT>::kWarpBytes;
  constexpr int join = kWarps * 8 * NT * (D + 2) * 4;
  return ring > join ? ring : join;
}
template <int D, int NT>
constexpr int ctas_per_sm() { return D == 128 ? (NT == 1 ? 4 : NT == 2 ? 3 : 2) : (NT <= 2 ? 4 : 2); }

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
// The key of a 16-key group that row r of S^T stands for: two keys apart lie on the same banks, and the lanes that read
// K rows together differ in g, those that read V rows together in t.
__device__ __forceinline__ int key_of(int r) { return r ^ ((r >> 1) & 1); }
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Of the keys of a block that are there, the first `keys`.
__device__ __forceinline__ uint32_t seen(uint32_t there, int keys) {
  return there & (keys >= kBlk ? 0xffffffffu : keys <= 0 ? 0u : (1u << keys) - 1u);
}
// A scale byte as f16 in both halves, and two of them.
__device__ __forceinline__ uint32_t scale2(uint32_t byte) { return byte * 0x800080u; }
__device__ __forceinline__ uint32_t scale_pair(uint32_t lo, uint32_t hi) { return (lo << 7) | (hi << 23); }
// 16-byte column c of a joined row, by which the stores of a warp touch distinct banks.
template <int D>
__device__ __forceinline__ int swap(int row) {
  const int t = (row >> 1) & 3;
  return D == 128 ? t : (t & 1) | ((t & 2) << 1);
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, (ctas_per_sm<D, NT>())) chunk_mma4_kernel(const __grid_constant__ ChunkParams p,
                                                                                 const ChunkItem* __restrict__ items) {
  using R = Ring<D, NT>;
  constexpr int kRows = 8 * NT, W = D / 32, MT = D / 16;  // words of a lane's K, 16-column tiles of O
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
  const int32_t* table = p.page_table + it.src * p.max_pages;
  // (rows of a pool are counted in 32 bits; the launcher sees to it)
  const uint32_t per_page = (uint32_t)(p.h_kv * p.page_size), row0 = (uint32_t)(h * p.page_size);
  const uint32_t some = p.n_pages > 0 ? 16u : 0u;  // (keys that are not there come as whatever row 0 holds)
  constexpr int CH = R::kRow / 16, RPI = 32 / CH, kIter = kBlk / RPI;   // 16-byte pieces of a row, rows of an instruction
  constexpr int kPer = 16 / R::kScales, kLanes = kBlk / kPer;           // keys whose scales make 16 bytes (they share a page)
  const uint8_t* kb = static_cast<const uint8_t*>(p.k_pool) + 16 * (lane % CH);
  const uint8_t* vb = static_cast<const uint8_t*>(p.v_pool) + 16 * (lane % CH);
  const uint8_t* sb = lane < kLanes ? p.k_scale : p.v_scale;
  const uint32_t to = ring_at + 16 * lane, sto = ring_at + (lane < kLanes ? R::kSK : R::kSV) + 16 * (lane % kLanes);

  // page of this lane's key of the warp's i-th block
  auto page_of = [&](int i) -> int {
    const int key = it.key0 + (warp + kWarps * i) * kBlk + lane;
    return i < mine && key < it.key1 ? __ldcg(table + (key >> p.page_shift)) : -1;
  };
  // Fetches the block; returns which of its keys are there.
  auto issue = [&](int i, int page, int stage) -> uint32_t {
    if (i >= mine) return 0u;
    const int key = it.key0 + (warp + kWarps * i) * kBlk + lane;
    const bool ok = (unsigned)page < (unsigned)p.n_pages;
    if (!ok && key < it.key1) pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_BOUNDS, (int)it.src, key >> p.page_shift, page);
    const uint32_t row = ok ? row0 + (uint32_t)page * per_page + (uint32_t)(key & (p.page_size - 1)) : 0u;
    const uint32_t at = stage * R::kStage;
#pragma unroll
    for (int j = 0; j < kIter; ++j) {
      const uint64_t off = (uint64_t)__shfl_sync(0xffffffffu, row, j * RPI + lane / CH) * R::kRow;
      cp16(to + at + 512 * j, kb + off, some);
      cp16(to + at + R::kV + 512 * j, vb + off, some);
    }
    const uint64_t off = (uint64_t)__shfl_sync(0xffffffffu, row, (lane % kLanes) * kPer) * R::kScales;
    if (lane < 2 * kLanes) cp16(sto + at, sb + off, some);
    return __ballot_sync(0xffffffffu, ok);
  };

  uint32_t keys_in[R::kStages];  // of the blocks under way, the next one's first
  int page = page_of(0);
#pragma unroll
  for (int i = 0; i < R::kStages - 1; ++i) {
    const int next = page_of(i + 1);
    keys_in[i] = issue(i, page, i);
    asm volatile("cp.async.commit_group;" ::: "memory");
    page = next;
  }

  // Q fragments: row 8 n + g, step s of the dimensions D/4 t + 4 s .., as f16 of the row times 2^-e, e such that its
  // largest value lies in [2^14, 2^15); and what the scores of rows 8 n + 2t, + 1 are to be multiplied by
  uint32_t qf[NT][2 * W][2];
  float qs[NT][2];
  int lim[NT][2], lim_all = 0x7fffffff;  // keys that those rows see, and that all rows see
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = 8 * n + g;
    const bool on = r < n_rows;
    const __nv_bfloat16* src = p.q + (on ? (it.tok0 + r / G) * p.q_stride + (int64_t)(h * G + r % G) * D : 0) + D / 4 * t4;
    uint4 x[W];
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      x[j] = on ? __ldcg(reinterpret_cast<const uint4*>(src) + j) : make_uint4(0u, 0u, 0u, 0u);
      const uint32_t xs[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
      for (int u = 0; u < 4; ++u) top = max(top, max(xs[u] & 0x7fffu, (xs[u] >> 16) & 0x7fffu));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // (the exponent kept where both powers of two are normal numbers; a row with a NaN or an infinity keeps it
    // whatever the scale)
    const int e = min(max((int)(top >> 7) - 127 - 14, -120), 113);
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    const float back = fmaxf(p.scale_log2 * __uint_as_float((uint32_t)(127 + e) << 23), 1e-45f);  // (0 would make a NaN of -inf)
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const uint32_t xs[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
      for (int u = 0; u < 4; ++u)
        qf[n][2 * j + (u >> 1)][u & 1] = pack_f16(__uint_as_float(xs[u] << 16) * down, __uint_as_float(xs[u] & 0xffff0000u) * down);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      qs[n][u] = __shfl_sync(0xffffffffu, back, 4 * (2 * t4 + u));
      const int rr = 8 * n + 2 * t4 + u;
      lim[n][u] = rr < n_rows ? min(it.lim0 + rr / G, it.key1) : 0;
      if (rr < n_rows) lim_all = min(lim_all, lim[n][u]);
    }
  }
  lim_all = __reduce_min_sync(0xffffffffu, lim_all);

  float o[NT][MT][4], mx[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) o[n][i][u] = 0.f;
    mx[n][0] = mx[n][1] = kNegInf;
    l[n][0] = l[n][1] = 0.f;
  }

  int s_use = 0, s_fill = R::kStages - 1;  // the stages of this block and of the one being fetched
  bool far = false;                        // some row's maximum is beyond kFar (the same in all lanes)
  const int kg = key_of(g);
#pragma unroll 1
  for (int i = 0; i < mine; ++i) {
    {
      const int next = page_of(i + R::kStages);
      keys_in[R::kStages - 1] = issue(i + R::kStages - 1, page, s_fill);
      asm volatile("cp.async.commit_group;" ::: "memory");
      page = next;
      s_fill = s_fill == R::kStages - 1 ? 0 : s_fill + 1;
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(R::kStages - 1) : "memory");
    __syncwarp();
    uint8_t* st = ring + s_use * R::kStage;
    s_use = s_use == R::kStages - 1 ? 0 : s_use + 1;
    const uint32_t there = keys_in[0];
#pragma unroll
    for (int j = 0; j + 1 < R::kStages; ++j) keys_in[j] = keys_in[j + 1];
    const int k0 = it.key0 + (warp + kWarps * i) * kBlk;

    // S^T: keys 16 m + key_of(g) (and + 8) of the block, rows 8 n + 2 t4 (and + 1)
    // (NT 1: two sums each, of every other step, so that four chains of products are under way)
    constexpr int CHAINS = NT == 1 ? 2 : 1;
    float s[NT][2][4], s2[CHAINS][NT][2][4];
    uint32_t kw[2][2][W], ks[2][2][W / 2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int c = 0; c < CHAINS; ++c)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int u = 0; u < 4; ++u) s2[c][n][m][u] = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int key = 16 * m + 8 * u + kg;
        const uint8_t* a = st + key * R::kRow + 4 * W * t4;
        const uint8_t* b = st + R::kSK + key * R::kScales + (W / 2) * t4;
        if constexpr (W == 4) {
          const uint4 v = *reinterpret_cast<const uint4*>(a);
          kw[m][u][0] = v.x, kw[m][u][1] = v.y, kw[m][u][2] = v.z, kw[m][u][3] = v.w;
          const uint32_t two = *reinterpret_cast<const uint16_t*>(b);
          ks[m][u][0] = scale2(two & 255u), ks[m][u][1] = scale2(two >> 8);
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(a);
          kw[m][u][0] = v.x, kw[m][u][1] = v.y;
          ks[m][u][0] = scale2(*b);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        uint32_t x[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f16_of_e2m1(kw[m][u][j], x[u]);
#pragma unroll
          for (int q = 0; q < 4; ++q) x[u][q] = f16_times(x[u][q], ks[m][u][j / 2]);
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint32_t a[4] = {x[0][2 * q], x[1][2 * q], x[0][2 * q + 1], x[1][2 * q + 1]};
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_f16(s2[q % CHAINS][n][m], a, qf[n][2 * j + q][0], qf[n][2 * j + q][1]);
        }
      }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int u = 0; u < 4; ++u) s[n][m][u] = CHAINS == 2 ? s2[0][n][m][u] + s2[CHAINS - 1][n][m][u] : s2[0][n][m][u];

    // A block that some row does not see in full: hidden scores are replaced.  A weight of 0 times a scale that is not finite is
    // not 0: in such a block those scales become 0, as those of keys that are not there, and the rows that see
    // them get their NaN at the end of it.
    uint32_t nan_keys = 0u;  // of the lane's column group
    if (there != 0xffffffffu || k0 + kBlk > lim_all) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t sees = seen(there, lim[n][u] - k0);
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int v = 0; v < 2; ++v)
              if (!((sees >> (16 * m + 8 * v + kg)) & 1u)) s[n][m][2 * v + u] = kNegInf;
        }
      const bool in = (there >> lane) & 1u;
#pragma unroll
      for (int j = 0; j < R::kScales; ++j) {
        uint8_t* b = st + R::kSV + R::kScales * lane + j;
        const bool odd = in && *b > 226u;
        const uint32_t which = __ballot_sync(0xffffffffu, odd);
        if ((W == 4 ? g : g >> 1) == j) nan_keys = which;
        if (!in || odd) *b = 0;
      }
      __syncwarp();
    }
    bool grow = false;
    float top[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        top[n][u] = fmaxf(tc::max3f(s[n][0][u], s[n][0][2 + u], s[n][1][u]), s[n][1][2 + u]) * qs[n][u];
        grow |= top[n][u] > mx[n][u];
      }
    // (the maximum of few blocks is above all before them)
    if (__any_sync(0xffffffffu, grow)) {
      bool beyond = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float m_new = fmaxf(mx[n][u], top[n][u]);
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) m_new = fmaxf(m_new, __shfl_xor_sync(0xffffffffu, m_new, x));
          const float alpha = m_new == kNegInf ? 1.f : ex2(mx[n][u] - m_new);
          l[n][u] *= alpha;
#pragma unroll
          for (int c = 0; c < MT; ++c) {
            o[n][c][u] *= alpha;
            o[n][c][2 + u] *= alpha;
          }
          mx[n][u] = m_new;
          beyond |= m_new != kNegInf && fabsf(m_new) > kFar;
        }
      far = __any_sync(0xffffffffu, beyond);
    }
    uint32_t pf[NT][2][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float up[2] = {mx[n][0] == kNegInf ? 0.f : kUp - mx[n][0], mx[n][1] == kNegInf ? 0.f : kUp - mx[n][1]};
      float by[2] = {qs[n][0], qs[n][1]};
      if (far) {
        // scores rounded as their maximum was, whose difference from it is then never above 0
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float m0 = mx[n][u] == kNegInf ? 0.f : mx[n][u];
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int v = 0; v < 2; ++v) s[n][m][2 * v + u] = __fsub_rn(__fmul_rn(s[n][m][2 * v + u], by[u]), m0);
          by[u] = 1.f;
          up[u] = kUp;
        }
      }
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const float a = ex2(fmaf(s[n][m][2 * v], by[0], up[0])), b = ex2(fmaf(s[n][m][2 * v + 1], by[1], up[1]));
          l[n][0] += a;
          l[n][1] += b;
          pf[n][m][v] = transposed(pack_f16(a, b));
        }
    }

    // O^T: columns D/8 g + 2 i (and + 1), rows as those of S^T
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      uint32_t w[4][W / 2], b[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int key = 16 * m + 8 * (u >> 1) + key_of(2 * t4 + (u & 1));
        const uint8_t* a = st + R::kV + key * R::kRow + 2 * W * g;
        if constexpr (W == 4) {
          const uint2 v = *reinterpret_cast<const uint2*>(a);
          w[u][0] = v.x, w[u][1] = v.y;
        } else {
          w[u][0] = *reinterpret_cast<const uint32_t*>(a);
        }
        b[u] = st[R::kSV + key * R::kScales + (W == 4 ? g : g >> 1)];
      }
      const uint32_t lo = scale_pair(b[0], b[1]), hi = scale_pair(b[2], b[3]);
#pragma unroll
      for (int j = 0; j < W / 2; ++j) {
        uint32_t x[4][4];  // even columns of the lower and upper keys, odd columns
        f16_of_e2m1((w[0][j] & 0x0f0f0f0fu) | ((w[1][j] << 4) & 0xf0f0f0f0u), x[0]);
        f16_of_e2m1(((w[0][j] >> 4) & 0x0f0f0f0fu) | (w[1][j] & 0xf0f0f0f0u), x[1]);
        f16_of_e2m1((w[2][j] & 0x0f0f0f0fu) | ((w[3][j] << 4) & 0xf0f0f0f0u), x[2]);
        f16_of_e2m1(((w[2][j] >> 4) & 0x0f0f0f0fu) | (w[3][j] & 0xf0f0f0f0u), x[3]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t a[4] = {f16_times(x[0][q], lo), f16_times(x[1][q], lo), f16_times(x[2][q], hi), f16_times(x[3][q], hi)};
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_f16(o[n][4 * j + q], a, pf[n][m][0], pf[n][m][1]);
        }
      }
    }
    if (__any_sync(0xffffffffu, nan_keys != 0u)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (nan_keys & seen(there, lim[n][u] - k0)) {
#pragma unroll
            for (int c = 0; c < MT; ++c) o[n][c][u] = o[n][c][2 + u] = __uint_as_float(0x7fc00000u);
          }
    }
    __syncwarp();
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // The four warps' states through shared memory: O rows, then (m, l).
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l[n][u] += __shfl_xor_sync(0xffffffffu, l[n][u], x);
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);
  float2* sml = reinterpret_cast<float2*>(so + kWarps * kRows * D);
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = 8 * n + 2 * t4 + u;
      float* dst = so + (warp * kRows + r) * D;
#pragma unroll
      for (int c = 0; c < MT / 2; ++c)
        *reinterpret_cast<float4*>(dst + 4 * ((MT / 2 * g + c) ^ swap<D>(r))) =
            make_float4(o[n][2 * c][u], o[n][2 * c][2 + u], o[n][2 * c + 1][u], o[n][2 * c + 1][2 + u]);
      // (weights are on the maximum less kUp)
      if (g == 0) sml[warp * kRows + r] = make_float2(mx[n][u] - kUp, l[n][u]);
    }
  __syncthreads();
  constexpr int C4 = D / 4;  // float4 columns
  for (int i = threadIdx.x; i < n_rows * C4; i += kThreads) {
    const int r = i / C4, c = i % C4;
    float m_all = kNegInf, l_all = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) m_all = fmaxf(m_all, sml[k * kRows + r].x);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float2 ml = sml[k * kRows + r];
      if (ml.y == 0.f) continue;  // (it saw nothing; a NaN passes)
      const float w = ex2(ml.x - m_all);
      const float4 x = *reinterpret_cast<const float4*>(so + (k * kRows + r) * D + 4 * (c ^ swap<D>(r)));
      l_all += w * ml.y;
      a.x += w * x.x;
      a.y += w * x.y;
      a.z += w * x.z;
      a.w += w * x.w;
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

template <int D, int NT>
cudaError_t launch(const ChunkParams& p, bool early, const ChunkItem* items, int n, cudaStream_t s) {
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    e = cudaFuncSetAttribute(chunk_mma4_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D, NT>());
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  if ((int64_t)n * p.h_kv > INT32_MAX || (int64_t)p.n_pages * p.h_kv * p.page_size > UINT32_MAX) return cudaErrorInvalidValue;
  return launch_early(early, chunk_mma4_kernel<D, NT>, dim3(n * p.h_kv), kThreads, smem_bytes<D, NT>(), s, p, items);
}

}  // namespace

int chunk_mma4_ctas(int head_dim, int rows8) {
  static constexpr int kCtas[2][3] = {{ctas_per_sm<64, 1>(), ctas_per_sm<64, 2>(), ctas_per_sm<64, 3>()},
                                      {ctas_per_sm<128, 1>(), ctas_per_sm<128, 2>(), ctas_per_sm<128, 3>()}};
  return kCtas[head_dim == 128][rows8 - 1];
}

cudaError_t launch_chunk_mma4(const ChunkParams& p, int head_dim, int rows8, bool early, const ChunkItem* items, int n_items,
                              cudaStream_t s) {
  static constexpr decltype(&launch<128, 1>) kForms[2][3] = {{launch<64, 1>, launch<64, 2>, launch<64, 3>},
                                                             {launch<128, 1>, launch<128, 2>, launch<128, 3>}};
  return kForms[head_dim == 128][rows8 - 1](p, early, items, n_items, s);
}

}  // namespace pad
