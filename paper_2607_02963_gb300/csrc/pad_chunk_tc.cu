// Attention of a step's chunk tokens on the 5th-generation tensor cores: for many query rows per
// (sequence of keys, kv-head), the drafted tokens of all branches against their video's prefix and a
// prompt's chunk against its pages.
//
// An item is a range of keys for consecutive chunk tokens; a CTA takes an item and a kv-head.  Rows are
// tokens x the G query heads of the kv-head, in slots of 128 / G tokens (126 rows at G = 7).  PAIR: two slots
// of tokens share each tile of 128 keys, one slot's softmax under the other's MMAs.  SPLIT: one
// slot, whose tiles two halves of the softmax warps take in turn, each with an S buffer, a maximum and an O
// of its own, joined at the end: the shorter chain where there are few rows.
//
//   warps 12-15  bring the tiles in.  bf16: TMA boxes of a page (of 128 tokens of a prefix) and 64 columns,
//                128-byte swizzle, warp 12 those of K, warp 13 of V, a lane looking up and fetching one page;
//                V tiles that some row does not see in full are looked over before they count as loaded
//                (warps 13-15): slots past the last token hold anything.  Pages of four tokens, which are half a
//                swizzle atom: 16-byte cp.async, 32 rows a warp, arrival left to the hardware (the mask's
//                word by an arrival of its own), the issuers fence the proxies.  8 bits: codes by cp.async, each thread widening those it has
//                copied itself.  (Through registers instead, the fence behind a tile's stores waited for
//                the next tile's loads: 2300 cycles per K or V tile.  bf16 by cp.async throughout:
//                838 us for 2048 new tokens over 30720, 28/4 heads, where the pages' boxes took 701.)
//   warp 0       S issuer: S_g(k) = Q_g K(k)^T
//   warp 1       TMEM allocation (512 columns) and deallocation, P.V issuer: O_g += P_g(k) V(k), P read
//                back from TMEM, 96 keys and then the last 32
//   warps 4-11   softmax: one row per thread, online in base 2 on a maximum that follows lazily (P's sum
//                tells whether the running one still bounds the scores)
//
// TMEM columns: S_0 at 0, S_1 at 128, O_g at 256 + D g; P_g goes over S_g.
//
// P goes into P.V rounded to bf16, one number each at either head_dim (2^-8 of a weight at most); the row sum is that of
// the unrounded fp32 weights.
//
// What is not finite stays with the rows that see it: scores of hidden keys are replaced, whatever they
// are; a hidden V value would meet a weight of 0, which is not enough for a NaN, so in the tiles that some
// row does not see in full the values past the first row's last key are looked at, and those that are not
// finite are left out of P.V and added to the rows that see them at the end.
//
// Bound by the chain S -> softmax -> P.V of a slot where the other slot's MMAs do not cover it; over pages one
// slot alone by the boxes of a tile, in 8 bits by the warps that widen (one per scheduler: 1.1 us per K or V
// tile at head_dim 128, 0.7 at 64).  2048 new tokens over 30720, 28/4 heads, bf16: 640 to 673 us, 1385 to
// 1456 TFLOP/s; 129 over a prefix of 32768: 74 us; 6 chunks of 130 to 1501 tokens over up to 7001, 14/2 heads,
// head_dim 64, 8 bits: 178 us, 620 TFLOP/s.
//
// Every wait is bounded (about one second); one that runs out records PAD_ERR_DEVICE_TIMEOUT, raises
// a CTA-wide flag, lets what was started drain, frees TMEM and returns.
#include <cuda.h>
#include <cuda_bf16.h>
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "pad_chunk.h"
#include "pad_tc_common.cuh"

namespace pad {

namespace {

using namespace tc;

constexpr int kBN = 128;        // keys per tile
constexpr int kThreads = 512;
constexpr int kLoGroups = 3;    // 32-key groups of a tile whose P is released first
constexpr float kRescaleSum = 256.0f;  // a part of a row whose P sum to more is redone on a new maximum
constexpr float kNegInf = -__builtin_huge_valf();
constexpr int kMasks = 8;       // tiles whose key masks are kept (as many can be between loader and softmax: 8 bits, D 64, one slot)

template <int D, bool FP8>
struct Cfg {
  static constexpr int kHalves = D / 64;                      // 64-column boxes of a row
  static constexpr uint32_t kBoxBytes = kBN * 128;
  static constexpr uint32_t kTileBytes = kHalves * kBoxBytes;
  static constexpr int kKS = D == 128 ? (FP8 ? 2 : 3) : 4;    // (8 bits: a K stage's room for the codes)
  static constexpr int kVS = D == 128 ? 2 : 4;
  static constexpr uint32_t kOffK = 2 * kTileBytes;           // Q_0, Q_1 first
  static constexpr uint32_t kOffV = kOffK + kKS * kTileBytes;
  // 8 bits: K or V tiles of codes on their way, with a word per row that holds its scale byte
  static constexpr int kRaw = FP8 ? (D == 128 ? 2 : 4) : 0;
  static constexpr uint32_t kRawBytes = kBN * (D + 4);
  static constexpr uint32_t kOffRaw = kOffV + kVS * kTileBytes;
  static constexpr uint32_t kOffBar = kOffRaw + kRaw * kRawBytes;
  static constexpr uint32_t kSmemBytes = kOffBar + 512;
  static constexpr uint32_t kColO = 256;
  static constexpr uint32_t kIdescS = make_idesc(128, kBN, false);
  static constexpr uint32_t kIdescPV = make_idesc(128, D, true);
  static_assert(kSmemBytes <= 232448, "fits the 227 KB opt-in shared memory");
};

// Registers per thread after setmaxnreg: 512 x 128 at launch; 128 x 48 + 256 x 184 + 128 x 96 = 65536.
constexpr int kRegsIssue = 48, kRegsSoftmax = 184, kRegsLoad = 96;

struct ChunkMaps {
  CUtensorMap k_pool, v_pool;      // rows of (page, head, slot), boxes of a page x 64 columns
  CUtensorMap k_prefix, v_prefix;  // (column, head, token), boxes of 128 tokens x 64 columns
  int32_t pages;                   // the pools' maps are there
};

struct Bars {
  // (full: one arrival with the bytes; by cp.async one of every loader thread, and for bf16 K tiles one of every warp,
  // which publishes the tile's mask: the arrivals of copies order no other store)
  uint64_t kfull[4], kfree[4];
  uint64_t vfull[4], vfree[4];
  uint64_t sfull[2];
  uint64_t plo[2], phi[2];
  uint64_t pvlo[2];
  uint64_t pvdone[2];
  uint64_t drain_s, drain_pv;
  uint64_t tdone;
  uint64_t vraw, vbad, vlooked; // V tiles that are looked over once they have landed (by three warps together, by one)
  alignas(16) uint32_t mask[kMasks][4];  // which keys of the tile are there
  uint32_t tmem_base;
  int32_t abort;
  int32_t dirty;                // V values that are not finite were left out
  ChunkItem item;               // (read back where its fields are needed late: they would take registers)
};
static_assert(sizeof(Bars) <= 512, "barrier block fits its slot");

__device__ __forceinline__ bool cwait(uint64_t* bar, uint32_t parity, Bars* bars, const ChunkParams& p, int where) {
  unsigned long long t0 = 0;
  for (uint32_t i = 1;; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 255u) == 0) {
      if (*reinterpret_cast<volatile int32_t*>(&bars->abort)) return false;
      const unsigned long long now = globaltimer();
      if (t0 == 0) t0 = now;
      if (now - t0 > kWaitNs) {
        pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_TIMEOUT, (int)blockIdx.x, where, (int)threadIdx.x);
        *reinterpret_cast<volatile int32_t*>(&bars->abort) = 1;
        return false;
      }
    }
  }
}
__device__ __forceinline__ bool cwait_warp(uint64_t* bar, uint32_t parity, Bars* bars, const ChunkParams& p, int where) {
  return __all_sync(0xffffffffu, cwait(bar, parity, bars, p, where)) != 0;
}

template <int N>
__device__ __forceinline__ float row_max(const uint32_t (&s)[kLoGroups][32]) {
  float m[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) m[u] = kNegInf;
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const int u = (i >> 1) & 7;
      m[u] = max3f(m[u], __uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1]));
    }
  return fmaxf(max3f(m[0], m[1], m[2]), max3f(max3f(m[3], m[4], m[5]), m[6], m[7]));
}

// P = 2^(s * sl2 - m) of N 32-score groups of a row, as packed bf16 to TMEM columns taddr ..; returns
// their fp32 sums as four pairs.
template <int N>
__device__ __forceinline__ void part_exp(const uint32_t (&s)[kLoGroups][32], uint64_t sc2, float m, uint32_t taddr, uint64_t (&sum)[4]) {
  const uint64_t nm2 = f2pack(-m, -m);
#pragma unroll
  for (int u = 0; u < 4; ++u) sum[u] = 0ull;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    uint32_t pk[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint64_t x = ffma2(f2pack(__uint_as_float(s[c][2 * i]), __uint_as_float(s[c][2 * i + 1])), sc2, nm2);
      const float a = ex2(f2lo(x)), b = ex2(f2hi(x));
      sum[i & 3] = fadd2(sum[i & 3], f2pack(a, b));
      pk[i] = pack_bf16(a, b);
    }
    tmem_st16(taddr + 16 * c, pk);
  }
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ bool odd2(uint32_t v) {  // a half that is not finite
  return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
}
// The halves that are not finite set to 0.
__device__ __forceinline__ uint32_t clean2(uint32_t v) {
  if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
  if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
  return v;
}
// This thread's arrival, once all of its cp.async so far have completed.
__device__ __forceinline__ void mbar_arrive_copies(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int D, bool FP8, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1)
    chunk_tc_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ ChunkMaps maps,
                    const ChunkItem* __restrict__ items) {
  using C = Cfg<D, FP8>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  Bars* bars = reinterpret_cast<Bars*>(smem + C::kOffBar);
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const ChunkItem it = items[(int)blockIdx.x / p.h_kv];
  const int kvh = (int)blockIdx.x % p.h_kv, G = p.group, tps = 128 / G;
  const int inv_g = 65536 / G + 1;  // row / G = row * inv_g >> 16 for rows below 128
  // (beside the warp-level grid of the same call, which was launched in plain stream order: what the items here read is
  // complete, and that grid is waited for at the end, so that the join's wait covers both)
  grid_release();
  const int key0 = it.key0, key1 = it.key1;
  // (as a warp-uniform value: the issuers' loops, and with them the MMAs' descriptors, stay in uniform registers)
  const int n_tiles = __shfl_sync(0xffffffffu, key1 > key0 ? (key1 - key0 + kBN - 1) / kBN : 0, 0);

  if (n_tiles == 0 || (sbase & 1023u)) {
    if (p.beside) grid_wait();
    if (sbase & 1023u) {  // the swizzle atoms need 1024-byte alignment (never expected)
      if (threadIdx.x == 0) pad_set_error(p.header, p.gen, PAD_ERR_UNSUPPORTED, (int)blockIdx.x, (int)sbase, 0);
    }
    // no key for any row: say so where the join looks (an item that is its rows' only one has keys)
    if (it.part_row >= 0)
      for (int r = threadIdx.x; r < it.ntok * G; r += kThreads)
        p.part_ml[it.part_row + (int64_t)(r / G) * p.h_q + kvh * G + r % G] = make_float2(kNegInf, 0.f);
    return;
  }

  const bool paged = it.paged != 0;
  const bool wide = FP8 && paged;                     // 8-bit tiles
  const bool bulk = !wide && (!paged || maps.pages);  // tiles by TMA
  if (threadIdx.x == 384) {  // (of the warp that fetches the first tile)
    for (int s = 0; s < 4; ++s) {
      mbar_init(&bars->kfull[s], bulk ? 1 : wide ? 128 : 132);
      mbar_init(&bars->kfree[s], 1);
      mbar_init(&bars->vfull[s], bulk ? 1 : 128);
      mbar_init(&bars->vfree[s], 1);
    }
    for (int g = 0; g < 2; ++g) {
      mbar_init(&bars->sfull[g], 1);
      mbar_init(&bars->plo[g], 4);
      mbar_init(&bars->phi[g], 4);
      mbar_init(&bars->pvlo[g], 1);
      mbar_init(&bars->pvdone[g], 1);
    }
    mbar_init(&bars->drain_s, 1);
    mbar_init(&bars->drain_pv, 1);
    mbar_init(&bars->tdone, 8);
    mbar_init(&bars->vraw, 1);
    mbar_init(&bars->vbad, 1);
    mbar_init(&bars->vlooked, 3);
    bars->abort = 0;
    bars->dirty = 0;
    bars->item = it;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)),
                 "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }

  // What a loader warp needs of its 32 rows of a tile, lane L's being 32 w + L.
  const int w = warp & 3;
  const int32_t* table = p.page_table + (paged ? it.src * p.max_pages : 0);
  auto page_of = [&](int t) -> int {
    const int key = key0 + t * kBN + 32 * w + lane;
    return paged && t < n_tiles && key < key1 ? __ldcg(table + (key >> p.page_shift)) : 0;
  };
  // The rows that are there.  A row lies `idx` x mul (+ its slot within the page) from the base: idx is its
  // page, or of a prefix its token.
  auto rows_of = [&](int t, int page, uint32_t& idx, uint32_t& there) {
    const int key = key0 + t * kBN + 32 * w + lane;
    bool ok = t < n_tiles && key < key1;
    if (paged && ok && (unsigned)page >= (unsigned)p.n_pages) {
      ok = false;
      pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_BOUNDS, (int)it.src, key >> p.page_shift, page);
    }
    there = __ballot_sync(0xffffffffu, ok);
    idx = ok ? (uint32_t)(paged ? page : key) : 0u;
  };
  const int row_bytes = wide ? D : 2 * D;
  const uint32_t mul = (uint32_t)(p.h_kv * row_bytes * (paged ? p.page_size : 1));
  const uint32_t in_page = paged ? (uint32_t)(p.page_size - 1) : 0u;
  const int64_t base0 = (paged ? (int64_t)kvh * p.page_size : it.src * p.h_kv + kvh) * row_bytes;
  const uint8_t* k_base = static_cast<const uint8_t*>(paged ? p.k_pool : p.k_prefix) + base0;
  const uint8_t* v_base = static_cast<const uint8_t*>(paged ? p.v_pool : p.v_prefix) + base0;
  auto issue_bf16 = [&](const uint8_t* base, uint32_t tile, int t, uint32_t idx, uint32_t there) {
    constexpr int CH = D / 8, RPI = 32 / CH;  // 16-byte chunks of a row, rows per instruction
    const int c = lane % CH, r0 = lane / CH;
    const uint8_t* src = base + 16 * c;
    const uint32_t dst = tile + (c >> 3) * C::kBoxBytes;
#pragma unroll
    for (int j = 0; j < 32 / RPI; ++j) {
      const int row = j * RPI + r0, r = 32 * w + row;
      const uint32_t i = __shfl_sync(0xffffffffu, idx, row);
      const uint32_t in = ((uint32_t)(key0 + t * kBN + r) & in_page) * (2 * D);
      const uint32_t on = (there >> row) & 1u;
      cp16(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4), src + (uint64_t)i * mul + (on ? in : 0u), on * 16u);
    }
  };
  // By TMA: lane L's page of a tile holds keys L x page size on; the pages that are there.
  auto tile_page = [&](int t) -> int {
    const int key = key0 + t * kBN + (lane << p.page_shift);
    return paged && t < n_tiles && lane < (kBN >> p.page_shift) && key < key1 ? __ldcg(table + (key >> p.page_shift)) : 0;
  };
  auto tile_pages = [&](int t, int page) -> uint32_t {
    const int key = key0 + t * kBN + (lane << p.page_shift);
    const bool in = paged && lane < (kBN >> p.page_shift) && key < key1, ok = in && (unsigned)page < (unsigned)p.n_pages;
    if (in && !ok && warp == 12) pad_set_error(p.header, p.gen, PAD_ERR_DEVICE_BOUNDS, (int)it.src, key >> p.page_shift, page);
    return __ballot_sync(0xffffffffu, ok);
  };
  auto key_there = [&](int t, int r, uint32_t pages) -> bool {
    return key0 + t * kBN + r < key1 && (!paged || ((pages >> (r >> p.page_shift)) & 1u));
  };
  auto fetch_tile = [&](const CUtensorMap* pool, const CUtensorMap* prefix, uint32_t tile, int t, int page, uint32_t pages,
                        uint64_t* full) {
    if (paged) {
      const uint32_t bytes = (uint32_t)__popc(pages) * (uint32_t)p.page_size * (2 * D);
      if (lane == 0) {
        if (bytes) mbar_expect_tx(full, bytes);
        else mbar_arrive(full);
      }
      __syncwarp();
      if ((pages >> lane) & 1u) {
        const int row = (page * p.h_kv + kvh) << p.page_shift;  // (the map's rows are fewer than 2^31)
#pragma unroll
        for (int h = 0; h < C::kHalves; ++h)
          tma_load_3d(tile + h * C::kBoxBytes + ((uint32_t)lane << p.page_shift) * 128, pool, 64 * h, 0, row, full);
      }
    } else if (lane == 0) {
      mbar_expect_tx(full, C::kTileBytes);
#pragma unroll
      for (int h = 0; h < C::kHalves; ++h)
        tma_load_3d(tile + h * C::kBoxBytes, prefix, 64 * h, kvh, (int)it.src + key0 + t * kBN, full);
    }
    __syncwarp();
  };
  // The tile's mask, before its K is fetched: the softmax reads it once S is there, and all of a warp's lanes have to
  // read the same.
  auto note_tile = [&](int t, uint32_t pages) {
    const bool whole = key0 + (t + 1) * kBN <= key1 && (!paged || pages == (uint32_t)((1ull << (kBN >> p.page_shift)) - 1ull));
    uint32_t mine = 0xffffffffu;  // lane's word
    if (!whole) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t m = __ballot_sync(0xffffffffu, key_there(t, 32 * u + lane, pages));
        if (lane == u) mine = m;
      }
    }
    if (lane < 4) bars->mask[t % kMasks][lane] = mine;
    __syncwarp();
  };
  uint32_t idx = 0, there = 0;
  if (warp >= 12) {
    // the first K tile goes out before the CTA has met (by cp.async: its arrival after)
    if (bulk) {
      if (warp == 12) {
        const int page = tile_page(0);
        there = tile_pages(0, page);
        __syncwarp();
        note_tile(0, there);
        fetch_tile(&maps.k_pool, &maps.k_prefix, sbase + C::kOffK, 0, page, there, &bars->kfull[0]);
      }
    } else {
      rows_of(0, page_of(0), idx, there);
      if (!wide) issue_bf16(k_base, sbase + C::kOffK, 0, idx, there);
    }
  } else {
    // Q of the slots by the others: row = token * G + head; what has no token is zero.  All of a thread's
    // chunks are under way together.
    constexpr int CH = D / 8, N = (SPLIT ? 1 : 2) * 128 * CH, PER = (N + 383) / 384;
    uint4 v[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = (int)threadIdx.x + 384 * k, c = i % CH, r = i / CH, g = r >> 7, row = r & 127;
      const int tl = row * inv_g >> 16, tok = g * tps + tl;
      v[k] = make_uint4(0u, 0u, 0u, 0u);
      if (i < N && tl < tps && tok < it.ntok)
        v[k] = __ldcg(reinterpret_cast<const uint4*>(p.q + (it.tok0 + tok) * p.q_stride + (int64_t)(kvh * G + row - tl * G) * D) + c);
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = (int)threadIdx.x + 384 * k, c = i % CH, r = i / CH, g = r >> 7, row = r & 127;
      if (i < N) sts128(sbase + g * C::kTileBytes + (c >> 3) * C::kBoxBytes + row * 128 + (((c & 7) ^ (row & 7)) << 4), v[k]);
    }
    proxy_fence();
  }
  fence_before();
  __syncthreads();
  fence_after();
  // an allocation of all 512 columns starts at TMEM address 0: an immediate for the MMAs
  constexpr uint32_t tmem = 0;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    bool ok = true;
    if (warp == 0) {
      // ------------------------------------------------------------ S issuer
      const bool el = elect_one();
      const uint64_t dK = sdesc(sbase + C::kOffK, 16, 1024);
      int s = 0, ph = 0;
      for (int t = 0; t < n_tiles && ok; ++t) {
        ok = cwait_warp(&bars->kfull[s], (uint32_t)ph, bars, p, 3);
        if (!bulk) proxy_fence();  // (the loaders' writes, before the MMAs read them)
        const int j = SPLIT ? t >> 1 : t;  // the slot's how-manieth tile
#pragma unroll
        for (int i = 0; i < (SPLIT ? 1 : 2); ++i) {
          const int g = SPLIT ? t & 1 : i;
          // S_g holds P of the slot's previous tile until its P.V has completed
          if (ok && j > 0) ok = cwait_warp(&bars->pvdone[g], (uint32_t)((j - 1) & 1), bars, p, 6);
          if (!ok) break;
          fence_after();
          const uint64_t qd = sdesc(sbase + (SPLIT ? 0u : (uint32_t)g * C::kTileBytes), 16, 1024);
          const uint64_t kd = dK + ((uint32_t)s * C::kTileBytes >> 4);
          if (el) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              const uint32_t off = (uint32_t)(kk >> 2) * C::kBoxBytes + (uint32_t)(kk & 3) * 32;
              mma_ss(tmem + 128u * g, qd + (off >> 4), kd + (off >> 4), C::kIdescS, kk > 0 ? 1u : 0u);
            }
            mma_commit(&bars->sfull[g]);
            if (SPLIT || g == 1) mma_commit(&bars->kfree[s]);
          }
          __syncwarp();
        }
        if (++s == C::kKS) {
          s = 0;
          ph ^= 1;
        }
      }
      if (el) mma_commit(&bars->drain_s);
      __syncwarp();
      drain_wait(&bars->drain_s, 0u);
    } else if (warp == 1) {
      // ------------------------------------------------------------ P.V issuer
      const bool el = elect_one();
      const uint64_t dV = sdesc(sbase + C::kOffV, C::kBoxBytes, 1024);
      int s = 0, ph = 0;
      for (int t = 0; t < n_tiles && ok; ++t) {
        ok = cwait_warp(&bars->vfull[s], (uint32_t)ph, bars, p, 4);
        if (!bulk) proxy_fence();
        const uint64_t vd = dV + ((uint32_t)s * C::kTileBytes >> 4);
        const int j = SPLIT ? t >> 1 : t;
#pragma unroll
        for (int i = 0; i < (SPLIT ? 1 : 2); ++i) {
          const int g = SPLIT ? t & 1 : i;
          const uint32_t a = tmem + 128u * g;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (ok) ok = cwait_warp(h ? &bars->phi[g] : &bars->plo[g], (uint32_t)(j & 1), bars, p, 5);
            if (!ok) break;
            fence_after();
            if (el) {
#pragma unroll
              for (int kk = h ? 2 * kLoGroups : 0; kk < (h ? 8 : 2 * kLoGroups); ++kk)
                mma_ts(tmem + C::kColO + (uint32_t)D * g, a + kk * 8, vd + ((uint32_t)kk * 2048 >> 4), C::kIdescPV,
                       (j > 0 || kk > 0) ? 1u : 0u);
              if (h == 0) mma_commit(&bars->pvlo[g]);
              if (h == 1) {
                mma_commit(&bars->pvdone[g]);
                if (SPLIT || g == 1) mma_commit(&bars->vfree[s]);
              }
            }
            __syncwarp();
          }
        }
        if (++s == C::kVS) {
          s = 0;
          ph ^= 1;
        }
      }
      if (el) mma_commit(&bars->drain_pv);
      __syncwarp();
      drain_wait(&bars->drain_pv, 0u);
      // TMEM is freed only after every softmax warp has arrived
      drain_wait(&bars->tdone, 0u);
      __syncwarp();
      fence_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
      if (p.beside) grid_wait();
    }
  } else if (warp >= 12) {
    // ------------------------------------------------------------ loaders
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLoad));
    bool ok = true;
    // keys from here on are hidden from some row (the item's first token sees the fewest)
    const int all_see = paged ? min(it.lim0, key1) : key1;
    auto note = [&](int t) {
      if (lane == 0) bars->mask[t % kMasks][w] = there;
    };
    int ks = 0, kph = 0, vs = 0, vph = 0;  // a tile's stages, and how often they have been used before
    if (bulk) {
      // the tiles from here on are looked over: not every row sees them in full
      const int t_look = min(n_tiles, max(0, all_see - key0) / kBN);
      const uint32_t every = paged ? (kBN >> p.page_shift) >= 32 ? 0xffffffffu : (1u << (kBN >> p.page_shift)) - 1u : 0u;
      // A landed V tile: keys that are not there become zeros, values that are not finite and that some row
      // does not see are left out.
      auto look = [&](int t, uint32_t tile, uint32_t pages, int r_lo, int thread, int threads) {
        constexpr int CH = D / 8;
        bool bad = false;
#pragma unroll 2
        for (int i = thread; i < (kBN - r_lo) * CH; i += threads) {
          const int r = r_lo + i / CH, c = i % CH;
          const uint32_t a = tile + (c >> 3) * C::kBoxBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4);
          if (!key_there(t, r, pages)) {
            sts128(a, make_uint4(0u, 0u, 0u, 0u));
          } else if (key0 + t * kBN + r >= all_see) {
            const uint4 v = lds128(a);
            if (odd2(v.x) | odd2(v.y) | odd2(v.z) | odd2(v.w)) {
              bad = true;
              sts128(a, make_uint4(clean2(v.x), clean2(v.y), clean2(v.z), clean2(v.w)));
            }
          }
        }
        if (bad) *reinterpret_cast<volatile int32_t*>(&bars->dirty) = 1;
        proxy_fence();
      };
      if (warp == 12) {
        int page = 0, issued = 0;
        for (int t = 0; t < n_tiles; ++t) {
          if (t > 0) {
            there = tile_pages(t, page);
            if (kph > 0) ok = cwait_warp(&bars->kfree[ks], (uint32_t)((kph - 1) & 1), bars, p, 1);
            if (!ok) break;
          }
          if (t > 0) note_tile(t, there);
          if (t > 0) fetch_tile(&maps.k_pool, &maps.k_prefix, sbase + C::kOffK + (uint32_t)ks * C::kTileBytes, t, page, there, &bars->kfull[ks]);
          page = tile_page(t + 1);
          issued = t + 1;
          if (++ks == C::kKS) {
            ks = 0;
            ++kph;
          }
        }
        // given up: the loads under way must land before the CTA leaves
        if (!ok)
          for (int t = max(0, issued - C::kKS); t < issued; ++t) drain_wait(&bars->kfull[t % C::kKS], (uint32_t)((t / C::kKS) & 1));
      } else {
        int page = warp == 13 ? tile_page(0) : 0, issued = 0, gaps = 0;
        if (warp == 13) {
          for (int t = 0; t < t_look; ++t) {
            const uint32_t tile = sbase + C::kOffV + (uint32_t)vs * C::kTileBytes;
            const uint32_t pages = tile_pages(t, page);
            if (vph > 0) ok = cwait_warp(&bars->vfree[vs], (uint32_t)((vph - 1) & 1), bars, p, 2);
            if (!ok) break;
            const bool gap = pages != every;
            fetch_tile(&maps.v_pool, &maps.v_prefix, tile, t, page, pages, gap ? &bars->vbad : &bars->vfull[vs]);
            issued = t + 1;
            page = tile_page(t + 1);
            if (gap) {
              ok = cwait_warp(&bars->vbad, (uint32_t)(gaps++ & 1), bars, p, 13);
              if (!ok) break;
              look(t, tile, pages, 0, lane, 32);
              __syncwarp();
              if (lane == 0) mbar_arrive(&bars->vfull[vs]);
            }
            if (++vs == C::kVS) {
              vs = 0;
              ++vph;
            }
          }
        } else {
          vs = t_look % C::kVS;
        }
        for (int t = t_look; t < n_tiles; ++t) {
          const uint32_t tile = sbase + C::kOffV + (uint32_t)vs * C::kTileBytes;
          if (warp > 13) page = tile_page(t);
          const uint32_t pages = tile_pages(t, page);
          const uint32_t par = (uint32_t)((t - t_look) & 1);
          if (warp == 13) {
            if (ok && vph > 0) ok = cwait_warp(&bars->vfree[vs], (uint32_t)((vph - 1) & 1), bars, p, 2);
            if (!ok) break;
            fetch_tile(&maps.v_pool, &maps.v_prefix, tile, t, page, pages, &bars->vraw);
            issued = t + 1;
            page = tile_page(t + 1);
          }
          ok = cwait_warp(&bars->vraw, par, bars, p, 14);
          if (!ok) break;
          const int keys = min(key1 - key0 - t * kBN, kBN);  // of the tile, if all of their pages are there
          const int n = (keys + p.page_size - 1) >> p.page_shift;
          const bool gap = paged && pages != (n >= 32 ? 0xffffffffu : (1u << n) - 1u);
          look(t, tile, pages, gap ? 0 : paged ? min(max(0, all_see - key0 - t * kBN), kBN) : keys, (int)threadIdx.x - 416, 96);
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->vlooked);
          if (warp == 13) {
            ok = cwait_warp(&bars->vlooked, par, bars, p, 15);
            if (!ok) break;
            if (lane == 0) mbar_arrive(&bars->vfull[vs]);
          }
          if (++vs == C::kVS) {
            vs = 0;
            ++vph;
          }
        }
        if (!ok && warp == 13)
          for (int t = max(0, issued - C::kVS); t < issued; ++t)
            drain_wait(t >= t_look ? &bars->vraw : &bars->vfull[t % C::kVS], (uint32_t)((t >= t_look ? t - t_look : t / C::kVS) & 1));
      }
    } else if (!wide) {
      int page = page_of(1);
      note(0);
      for (int t = 0; t < n_tiles; ++t) {
        if (t > 0) {
          rows_of(t, page, idx, there);
          page = page_of(t + 1);
          if (kph > 0) ok = cwait_warp(&bars->kfree[ks], (uint32_t)((kph - 1) & 1), bars, p, 1);
          if (!ok) break;
          note(t);
          issue_bf16(k_base, sbase + C::kOffK + (uint32_t)ks * C::kTileBytes, t, idx, there);
        }
        if (lane == 0) mbar_arrive(&bars->kfull[ks]);  // (lane 0 wrote the mask's word)
        mbar_arrive_copies(&bars->kfull[ks]);
        const uint32_t vt = C::kOffV + (uint32_t)vs * C::kTileBytes;
        if (vph > 0) ok = cwait_warp(&bars->vfree[vs], (uint32_t)((vph - 1) & 1), bars, p, 2);
        if (!ok) break;
        issue_bf16(v_base, sbase + vt, t, idx, there);
        if (key0 + (t + 1) * kBN <= all_see) {
          mbar_arrive_copies(&bars->vfull[vs]);
        } else {
          // a V tile that some row does not see in full: what is not finite there is left out of it
          asm volatile("cp.async.wait_all;" ::: "memory");
          constexpr int CH = D / 8, RPI = 32 / CH;
          bool bad = false;
#pragma unroll 1
          for (int j = 0; j < 32 / RPI; ++j) {
            const int r = 32 * w + j * RPI + lane / CH, c = lane % CH;
            if (key0 + t * kBN + r < all_see) continue;
            const uint32_t a = sbase + vt + (c >> 3) * C::kBoxBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4);
            uint4 v = lds128(a);
            if (odd2(v.x) | odd2(v.y) | odd2(v.z) | odd2(v.w)) {
              bad = true;
              sts128(a, make_uint4(clean2(v.x), clean2(v.y), clean2(v.z), clean2(v.w)));
            }
          }
          if (bad) *reinterpret_cast<volatile int32_t*>(&bars->dirty) = 1;
          proxy_fence();
          mbar_arrive(&bars->vfull[vs]);
        }
        if (++ks == C::kKS) {
          ks = 0;
          ++kph;
        }
        if (++vs == C::kVS) {
          vs = 0;
          ++vph;
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    } else if constexpr (FP8) {
      // 16 codes per lane and instruction, a matrix's 32 rows in NI of them; matrix m is K (even) or V of tile m / 2
      constexpr int CH = D / 16, RPI = 32 / CH, NI = 32 / RPI;
      const int c = lane % CH, r0 = lane / CH;
      const int64_t scale0 = (int64_t)kvh * p.page_size;
      const uint32_t scale_mul = (uint32_t)(p.h_kv * p.page_size);
      const int n_mats = 2 * n_tiles;
      const uint32_t raw0 = C::kOffRaw + (uint32_t)(32 * w + lane) * 16, word0 = C::kOffRaw + kBN * D + (uint32_t)(32 * w + lane) * 4;
      auto fetch = [&](int m, uint32_t at) {
        const uint8_t* src = m & 1 ? v_base : k_base;
        const int t = m >> 1;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int row = i * RPI + r0;
          const uint32_t pgi = __shfl_sync(0xffffffffu, idx, row);
          const uint32_t in = ((uint32_t)(key0 + t * kBN + 32 * w + row) & in_page) * D, on = (there >> row) & 1u;
          cp16(sbase + raw0 + at + i * 2048, src + 16 * c + (uint64_t)pgi * mul + (on ? in : 0u), on * 16u);
        }
        // (its row's scale byte, within the aligned word that holds it: pages hold four tokens at least)
        const uint32_t in = (uint32_t)(key0 + t * kBN + 32 * w + lane) & in_page & ~3u, on = (there >> lane) & 1u;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(sbase + word0 + at),
                     "l"((m & 1 ? p.v_scale : p.k_scale) + scale0 + (uint64_t)idx * scale_mul + (on ? in : 0u)), "r"(on * 4u)
                     : "memory");
      };
      int page = page_of(1);
      static_assert(C::kRaw == 2 || C::kRaw == 4, "the fetches ahead");
      // the tiles' rows are looked up as their K is fetched
      int fetched = 0;
      uint32_t at_f = 0;
      auto fetch_next = [&]() {
        if (fetched < n_mats) {
          if (!(fetched & 1) && fetched > 0) {
            rows_of(fetched >> 1, page, idx, there);
            page = page_of((fetched >> 1) + 1);
            note(fetched >> 1);
          }
          fetch(fetched, at_f);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ++fetched;
        at_f = at_f + C::kRawBytes == C::kRaw * C::kRawBytes ? 0u : at_f + C::kRawBytes;
      };
      note(0);
#pragma unroll 1
      for (int m = 0; m < C::kRaw; ++m) fetch_next();
      uint32_t at = 0;
      for (int m = 0; m < n_mats; ++m) {
        const bool v = m & 1;
        const int t = m >> 1;
        asm volatile("cp.async.wait_group %0;" ::"n"(C::kRaw - 1) : "memory");
        uint4 x[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) x[i] = *reinterpret_cast<const uint4*>(smem + raw0 + at + i * 2048);
        const int key = key0 + t * kBN + 32 * w + lane;
        uint32_t mult = scale_mult((*reinterpret_cast<const uint32_t*>(smem + word0 + at) >> (8 * (key & 3))) & 255u);
        if (v && mult == 0x7fc0u && key >= all_see) {
          mult = 0u;  // a NaN group that some row does not see: left out
          *reinterpret_cast<volatile int32_t*>(&bars->dirty) = 1;
        }
        mult |= mult << 16;
        if (v ? vph > 0 : kph > 0)
          ok = cwait_warp(v ? &bars->vfree[vs] : &bars->kfree[ks], (uint32_t)(((v ? vph : kph) - 1) & 1), bars, p, 1);
        if (!ok) break;
        const uint32_t tile = v ? C::kOffV + (uint32_t)vs * C::kTileBytes : C::kOffK + (uint32_t)ks * C::kTileBytes;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int row = i * RPI + r0, r = 32 * w + row;
          const uint32_t ml = __shfl_sync(0xffffffffu, mult, row);
          const int flip = D == 128 ? c >> 2 : 0;
          const uint32_t in[4] = {flip ? x[i].z : x[i].x, flip ? x[i].w : x[i].y, flip ? x[i].x : x[i].z, flip ? x[i].y : x[i].w};
          uint4 o[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            o[u].x = e4m3_pair(__byte_perm(in[2 * u], 0u, 0x1404), ml);
            o[u].y = e4m3_pair(__byte_perm(in[2 * u], 0u, 0x3424), ml);
            o[u].z = e4m3_pair(__byte_perm(in[2 * u + 1], 0u, 0x1404), ml);
            o[u].w = e4m3_pair(__byte_perm(in[2 * u + 1], 0u, 0x3424), ml);
          }
          // chunks 2 c and 2 c + 1 of the row: the upper half of the row's lanes writes them in the other
          // order, so that one store's lanes touch distinct banks (the two boxes lie on the same ones)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int ch = 2 * c + (u ^ flip);
            *reinterpret_cast<uint4*>(smem + tile + (ch >> 3) * C::kBoxBytes + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = o[u];
          }
        }
        proxy_fence();
        mbar_arrive(v ? &bars->vfull[vs] : &bars->kfull[ks]);
        fetch_next();  // (into the codes just read)
        at = at + C::kRawBytes == C::kRaw * C::kRawBytes ? 0u : at + C::kRawBytes;
        if (v) {
          if (++vs == C::kVS) {
            vs = 0;
            ++vph;
          }
        } else if (++ks == C::kKS) {
          ks = 0;
          ++kph;
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
  } else {
    // ------------------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int g = (warp - 4) >> 2;             // slot
    const int wrow = 32 * (warp & 3);          // TMEM lanes wrow .. wrow + 31
    const int row = wrow + lane;               // row of the slot: token row / G, head row % G
    const int tl = row * inv_g >> 16;
    const int tok = (SPLIT ? 0 : g * tps) + tl;  // of the item
    const bool active = tl < tps && tok < it.ntok;
    const int lim = active ? min(it.lim0 + (paged ? tok : 0), key1) - key0 : 0x7fffffff;  // keys of the item it sees
    const uint32_t tb = tmem + ((uint32_t)wrow << 16);
    const uint32_t tS = tb + 128u * g;
    const uint32_t tO = tb + C::kColO + (uint32_t)D * g;
    const float sl2 = p.scale_log2;
    const uint64_t sc2 = f2pack(sl2, sl2);
    // an inactive row takes no part in any decision
    float m_run = active ? kNegInf : 0.f;
    uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
    bool ok = true;

    // One tile in its two parts: 96 keys, then 32, whose scores are read only once the first part's are
    // done with (their registers are the same).  P of a part is computed on the running maximum; a sum
    // above 2^8 (and the first of all, which has no maximum yet) finds the part's, rescales O and l to it
    // and redoes the part.
    auto tile = [&](int t, auto masked) -> bool {
      const int j = SPLIT ? t >> 1 : t;        // the slot's how-manieth tile
      uint32_t s[kLoGroups][32];
      auto load = [&](int c0, auto n) {
#pragma unroll
        for (int c = 0; c < decltype(n)::value; ++c) tmem_ld32(tS + 32 * (c0 + c), s[c]);
      };
      auto part = [&](auto which) -> bool {
        constexpr int H = decltype(which)::value, N = H ? 4 - kLoGroups : kLoGroups, C0 = H ? kLoGroups : 0;
#pragma unroll
        for (int c = 0; c < N; ++c) tmem_wait_ld_dep(s[c]);
        if (decltype(masked)::value) {
          const int hi = lim - t * kBN;        // the tile's columns below hi, those of them that are there
#pragma unroll
          for (int c = 0; c < N; ++c) {
            const int n = hi - 32 * (C0 + c);
            const uint32_t see = bars->mask[t % kMasks][C0 + c] & (n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!((see >> i) & 1u)) s[c][i] = 0xff800000u;  // -inf
          }
        }
        uint64_t sum[4];
        part_exp<N>(s, sc2, m_run == kNegInf ? 0.f : m_run, tS + 16 * C0, sum);
        const uint64_t s2 = fadd2(fadd2(sum[0], sum[1]), fadd2(sum[2], sum[3]));
        const bool grow = active && (m_run == kNegInf || f2lo(s2) + f2hi(s2) > kRescaleSum);
        if (__any_sync(0xffffffffu, grow)) {
          if (j > 0 || H == 1) {
            // every P.V issued on O so far has completed: O may be rescaled
            if (!__all_sync(0xffffffffu, H == 1 ? cwait(&bars->pvlo[g], (uint32_t)(j & 1), bars, p, 9)
                                                : cwait(&bars->pvdone[g], (uint32_t)((j - 1) & 1), bars, p, 9)))
              return false;
            fence_after();
          }
          const float m_new = fmaxf(m_run, row_max<N>(s) * sl2);
          const bool need = grow && m_new > m_run;
          const float alpha = need ? ex2(m_run - m_new) : 1.f;
          if (j > 0 || H == 1) {
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t r[16];
              tmem_ld16(tO + 16 * c, r);
              tmem_wait_ld_dep16(r);
#pragma unroll
              for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
              tmem_st16(tO + 16 * c, r);
            }
          }
          const uint64_t al2 = f2pack(alpha, alpha);
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[u] = fmul2(acc[u], al2);
          if (need) m_run = m_new;
          // (a row that has seen no visible key keeps m = -inf; its exponent base is 0)
          part_exp<N>(s, sc2, m_run == kNegInf ? 0.f : m_run, tS + 16 * C0, sum);
        }
        tmem_wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(H ? &bars->phi[g] : &bars->plo[g]);
        __syncwarp();
        if (H == 0) load(kLoGroups, std::integral_constant<int, 4 - kLoGroups>{});
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] = fadd2(acc[u], sum[u]);
        return true;
      };
      load(0, std::integral_constant<int, kLoGroups>{});
      return part(std::integral_constant<int, 0>{}) && part(std::integral_constant<int, 1>{});
    };
    // the leading tiles that every row of the warp sees in full need no mask, unless a page is missing
    int least = lim;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
    const int n_full = min(n_tiles, least / kBN);
    for (int t = SPLIT ? g : 0; t < n_tiles && ok; t += SPLIT ? 2 : 1) {
      if (!__all_sync(0xffffffffu, cwait(&bars->sfull[g], (uint32_t)((SPLIT ? t >> 1 : t) & 1), bars, p, 8))) {
        ok = false;
        break;
      }
      fence_after();
      const uint4 mk = lds128(smem_u32(bars->mask[t % kMasks]));
      // (one decision for the warp: what follows is full of warp-wide instructions)
      const bool plain = __all_sync(0xffffffffu, t < n_full && (mk.x & mk.y & mk.z & mk.w) == 0xffffffffu) != 0;
      ok = plain ? tile(t, std::false_type{}) : tile(t, std::true_type{});
    }
    const volatile ChunkItem& itv = bars->item;
    const int mine = SPLIT ? (n_tiles + 1 - g) >> 1 : n_tiles;  // tiles of this slot
    if (ok && mine > 0) ok = cwait(&bars->pvdone[g], (uint32_t)((mine - 1) & 1), bars, p, 10);
    ok = __all_sync(0xffffffffu, ok);
    const uint64_t a2 = fadd2(fadd2(acc[0], acc[1]), fadd2(acc[2], acc[3]));
    float l = f2lo(a2) + f2hi(a2);
    float wgt = 1.f;                           // of this slot's O in the result
    // SPLIT: slot g writes the columns from D/2 g on, and takes the other's share of them: (m, l) of both
    // through the second Q stage, the O rows on the common maximum through the K stages, idle once both
    // slots' last P.V has completed: fp32, row r's 16-byte chunk c at c ^ (r % 16 or 8).
    constexpr int kCo = D / 4;
    static_assert(128u * 4 * D <= C::kKS * C::kTileBytes, "the slots' O rows fit the K stages");
    float2* sml = reinterpret_cast<float2*>(smem + C::kTileBytes);
    uint8_t* so = smem + C::kOffK + (uint32_t)row * (4 * D);
    if (SPLIT) {
      sml[g * 128 + row] = make_float2(m_run, l);
      __syncwarp();
      asm volatile("bar.sync 1, 256;" ::: "memory");
      const float2 other = sml[(g ^ 1) * 128 + row];
      // (l = 0: that half saw nothing; a NaN counts)
      const bool has = mine > 0 && l != 0.f, other_has = other.y != 0.f;
      const float m = fmaxf(m_run, other.x);
      wgt = has ? ex2(m_run - m) : 0.f;
      l = (has ? l * wgt : 0.f) + (other_has ? other.y * ex2(other.x - m) : 0.f);
      m_run = m;
      if (ok) {
        fence_after();
#pragma unroll 1
        for (int c = (1 - g) * (D / 64); c < (2 - g) * (D / 64); ++c) {
          uint32_t r[32];
          if (mine > 0) {
            tmem_ld32(tO + 32 * c, r);
            tmem_wait_ld_dep(r);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (has)
              v = make_float4(__uint_as_float(r[4 * j]) * wgt, __uint_as_float(r[4 * j + 1]) * wgt,
                              __uint_as_float(r[4 * j + 2]) * wgt, __uint_as_float(r[4 * j + 3]) * wgt);
            *reinterpret_cast<float4*>(so + (((8 * c + j) ^ (lane & (kCo / 2 - 1))) << 4)) = v;
          }
        }
      }
      __syncwarp();
      asm volatile("bar.sync 1, 256;" ::: "memory");
      wgt = has ? wgt : 0.f;
    }
    const bool dirty = *reinterpret_cast<volatile int32_t*>(&bars->dirty) != 0;
    // O of 32 columns of the row, from c0 on
    auto load_o = [&](int c0, uint32_t* r) {
      if (!SPLIT || mine > 0) {
        tmem_ld32(tO + c0, r);
        tmem_wait_ld_dep(r);
      }
      if (SPLIT) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float4 v = *reinterpret_cast<const float4*>(so + (((c0 / 4 + j) ^ (lane & (kCo / 2 - 1))) << 4));
          const float a[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int u = 0; u < 4; ++u)
            r[4 * j + u] = __float_as_uint(mine > 0 ? fmaf(__uint_as_float(r[4 * j + u]), wgt, a[u]) : a[u]);
        }
      }
      if (dirty && active && itv.paged) {
        // the values that were left out, of the keys that this row sees
#pragma unroll 1
        for (int key = max(itv.key0, itv.lim0); key < itv.key0 + lim; ++key) {
          const int pg = __ldcg(p.page_table + itv.src * p.max_pages + (key >> p.page_shift));
          if ((unsigned)pg >= (unsigned)p.n_pages) continue;
          const int64_t slot = ((int64_t)pg * p.h_kv + kvh) * p.page_size + (key & (p.page_size - 1));
          if (FP8) {
            if (__ldcg(p.v_scale + slot) == 255)
#pragma unroll
              for (int i = 0; i < 32; ++i) r[i] = 0x7fc00000u;
          } else {
            const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(p.v_pool) + slot * D + c0);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const uint32_t x = __ldcg(v + i);
              if (!odd2(x)) continue;
              if ((x & 0x7f80u) == 0x7f80u) r[2 * i] = __float_as_uint(__uint_as_float(r[2 * i]) + __uint_as_float(x << 16));
              if ((x & 0x7f800000u) == 0x7f800000u)
                r[2 * i + 1] = __float_as_uint(__uint_as_float(r[2 * i + 1]) + __uint_as_float(x & 0xffff0000u));
            }
          }
        }
      }
    };
    if (ok) {
      fence_after();
      const int64_t part_row = itv.part_row;
      const int tok0 = itv.tok0, ntok = itv.ntok;
      const bool part = part_row >= 0;
      const int head = kvh * G + (row - tl * G);
      const float inv = part ? 1.f : l == 0.f ? 0.f : 1.0f / l;
      if (active && (!SPLIT || g == 0)) {
        if (part)
          p.part_ml[part_row + (int64_t)tok * p.h_q + head] = make_float2(m_run, l);
        else if (p.lse != nullptr)
          p.lse[(int64_t)(tok0 + tok) * p.h_q + head] = l == 0.f ? kNegInf : (m_run + log2f(l)) * 0.69314718055994531f;
      }
      // Rows out through this warp's 32 rows of a Q stage, idle by now (SPLIT: slot 1's through the second):
      // row r's 16-byte chunk c at c ^ (r % chunks); then coalesced rows, half of the columns of an fp32 row
      // at a time.
      const bool bf16 = !part && p.out_bf16;
      constexpr int kCh = 2 * D / 16;           // chunks per staged row
      uint8_t* stg = smem + (uint32_t)g * C::kTileBytes + (uint32_t)wrow * (2 * D);
      const int passes = bf16 ? 1 : 2, esz = bf16 ? 2 : 4;
      uint8_t* base = part ? reinterpret_cast<uint8_t*>(p.part_o) : static_cast<uint8_t*>(p.out);
      const int64_t row0 = part ? part_row : (int64_t)tok0 * p.h_q;
#pragma unroll 1
      for (int ps = SPLIT && passes == 2 ? g : 0; ps < (SPLIT && passes == 2 ? g + 1 : passes); ++ps) {
        if (bf16) {
#pragma unroll 1
          for (int c = SPLIT ? g * (D / 64) : 0; c < (SPLIT ? g + 1 : 2) * (D / 64); ++c) {
            uint32_t r[32];
            load_o(32 * c, r);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t v[4];
#pragma unroll
              for (int u = 0; u < 4; ++u)
                v[u] = pack_bf16(__uint_as_float(r[8 * j + 2 * u]) * inv, __uint_as_float(r[8 * j + 2 * u + 1]) * inv);
              *reinterpret_cast<uint4*>(stg + lane * (2 * D) + (((4 * c + j) ^ (lane & (kCh - 1))) << 4)) =
                  make_uint4(v[0], v[1], v[2], v[3]);
            }
          }
        } else {
#pragma unroll 1
          for (int c = 0; c < D / 64; ++c) {
            uint32_t r[32];
            load_o((D / 2) * ps + 32 * c, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t v[4];
#pragma unroll
              for (int u = 0; u < 4; ++u) v[u] = __float_as_uint(__uint_as_float(r[4 * j + u]) * inv);
              *reinterpret_cast<uint4*>(stg + lane * (2 * D) + (((8 * c + j) ^ (lane & (kCh - 1))) << 4)) =
                  make_uint4(v[0], v[1], v[2], v[3]);
            }
          }
        }
        __syncwarp();
        // (rows of kCh chunks, or of the half that this slot writes: `per` lanes a row)
        const bool half = SPLIT && bf16;
        const int per = half ? kCh / 2 : kCh, cl = (half ? g * (kCh / 2) : 0) + lane % per, rows = 32 / per;
#pragma unroll 4
        for (int k = lane / per; k < 32; k += rows) {
          const int rr = wrow + k, rt = rr * inv_g >> 16, rtok = (SPLIT ? 0 : g * tps) + rt;
          if (rt < tps && rtok < ntok) {
            const uint4 v = *reinterpret_cast<const uint4*>(stg + k * (2 * D) + ((cl ^ (k & (kCh - 1))) << 4));
            const int64_t o = (row0 + (int64_t)rtok * p.h_q + kvh * G + (rr - rt * G)) * D * esz + (int64_t)ps * (2 * D) + 16 * cl;
            *reinterpret_cast<uint4*>(base + o) = v;
          }
        }
        __syncwarp();
      }
    }
    fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars->tdone);
  }
}

template <int D, bool FP8, bool SPLIT>
cudaError_t launch(const ChunkParams& p, int64_t prefix_tokens, const ChunkItem* items, int n, cudaStream_t s) {
  static bool configured[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    e = cudaFuncSetAttribute(chunk_tc_kernel<D, FP8, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<D, FP8>::kSmemBytes);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  if ((int64_t)n * p.h_kv > INT32_MAX) return cudaErrorInvalidValue;
  ChunkMaps maps = {};
  const int64_t rows = (int64_t)p.n_pages * p.h_kv * p.page_size;
  if (!FP8 && p.page_size >= 8 && rows > 0 && rows <= INT32_MAX) {
    if (!tma_map(&maps.k_pool, p.k_pool, D, 1, rows, 1, p.page_size) || !tma_map(&maps.v_pool, p.v_pool, D, 1, rows, 1, p.page_size))
      return cudaErrorInvalidValue;
    maps.pages = 1;
  }
  if (prefix_tokens > 0 && !prefix_tensor_maps(p.k_prefix, p.v_prefix, D, p.h_kv, prefix_tokens, &maps.k_prefix, &maps.v_prefix))
    return cudaErrorInvalidValue;
  return launch_early(p.beside, chunk_tc_kernel<D, FP8, SPLIT>, dim3(n * p.h_kv), kThreads, Cfg<D, FP8>::kSmemBytes, s, p, maps, items);
}

}  // namespace

cudaError_t launch_chunk_tc(const ChunkParams& p, int head_dim, bool fp8, bool split, int64_t prefix_tokens,
                            const ChunkItem* items, int n, cudaStream_t s) {
  if (prefix_tokens > INT32_MAX) return cudaErrorInvalidValue;  // (the maps' token coordinates; checked when planning)
  if (head_dim == 128) {
    if (split) return fp8 ? launch<128, true, true>(p, prefix_tokens, items, n, s) : launch<128, false, true>(p, prefix_tokens, items, n, s);
    return fp8 ? launch<128, true, false>(p, prefix_tokens, items, n, s) : launch<128, false, false>(p, prefix_tokens, items, n, s);
  }
  if (split) return fp8 ? launch<64, true, true>(p, prefix_tokens, items, n, s) : launch<64, false, true>(p, prefix_tokens, items, n, s);
  return fp8 ? launch<64, true, false>(p, prefix_tokens, items, n, s) : launch<64, false, false>(p, prefix_tokens, items, n, s);
}

}  // namespace pad
