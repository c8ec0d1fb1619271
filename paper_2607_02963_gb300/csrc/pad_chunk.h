// Internal declarations of the multi-token step (pad_chunk_*): what its host planner
// (pad_chunk_api.cu) and its kernels share.  The plan's device block, in the caller's workspace:
//
//   [0, 256)     PadDevHeader (status word)
//   work lists   copied once per plan: ChunkItem, ChunkMerge, ChunkPages, ChunkRead, ChunkVerify
//   part_ml      float2[partial_rows]            (m in log2 units, l)
//   part_o       float[partial_rows * head_dim]  (unnormalised O)
#pragma once

#include <cuda_fp16.h>

#include "pad_internal.h"

namespace pad {

// A range of keys for the rows of consecutive chunk tokens; a CTA takes one with a kv-head.
struct ChunkItem {
  int64_t part_row;    // partial row of (token tok0, head 0), rows token-major; -1: written to out directly
  int64_t src;         // prefix: first token of the video in k_prefix; pages: row of the page table
  int32_t key0, key1;  // keys [key0, key1) of that sequence (key0 >= key1: none; its partial rows say so)
  int32_t tok0, ntok;  // packed chunk tokens
  int32_t lim0;        // keys that token tok0 sees, from the sequence's start; pages: one more each token
  int32_t paged;       // 0: prefix, 1: pages
};
static_assert(sizeof(ChunkItem) == 40, "item is 40 bytes");

// The partial states of one chunk token whose keys were split.
struct ChunkMerge {
  int64_t pre_row, page_row;          // partial row of (split 0, this token, head 0)
  int64_t pre_stride, page_stride;    // rows from one split to the next
  int32_t pre_n, page_n;              // splits
  int32_t tok, pad;
};
static_assert(sizeof(ChunkMerge) == 48, "merge entry is 48 bytes");

// New tokens that go into one page.
struct ChunkPages {
  int32_t event, column;  // page-table entry
  int32_t page;           // a page taken this step (this entry's writer puts it there too), or -1: read the entry
  int32_t tok, slot, count;
};

// An event's cached tokens, copied out in spans of chunk_read_tokens() tokens.
struct ChunkRead {
  int64_t out;            // first output token
  int32_t span0;          // spans of the events before it
  int32_t count;          // tokens
};

// A sequence held in 4 bits that is widened to bf16 pages of the plan's own, in spans as above.
struct ChunkWiden {
  int32_t event, page0;   // row of the page table; the first of its pages
  int32_t span0, count;   // spans of the sequences before it; tokens
};

struct ChunkVerify {
  int32_t tok0, n_draft, draft0;  // first row of p, drafted tokens and the first of them; n_draft -1: no new token
};

struct ChunkParams {
  int32_t h_q, h_kv, group, page_size, page_shift, max_pages, n_pages;
  int32_t out_bf16;
  int32_t beside;   // the tcgen05 kernel runs beside the warp-level kernel of the same call
  float scale_log2;
  uint64_t gen;
  PadDevHeader* header;
  int32_t* page_table;
  float2* part_ml;
  float* part_o;
  const __nv_bfloat16* q;
  int64_t q_stride;
  const void* k_prefix;
  const void* v_prefix;
  const void* k_pool;
  const void* v_pool;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  void* out;
  float* lse;
};

// Launchers; they return the launch error.
cudaError_t launch_chunk_append(const ChunkParams& p, int head_dim, int kv_format, const ChunkPages* work, int n_work,
                                const void* k_new, const void* v_new, int64_t stride, void* k_pool, void* v_pool,
                                uint8_t* k_scale, uint8_t* v_scale, cudaStream_t s);
cudaError_t launch_chunk_read(const ChunkParams& p, int head_dim, int kv_format, const ChunkRead* work, int n_events,
                              int n_spans, void* k_out, void* v_out, cudaStream_t s);
int chunk_read_tokens();
// The 4-bit tokens of `n_events` sequences into bf16 pages of the plan's own (row e of `table`, `columns` wide, lists
// them; an entry whose page is not in the pool becomes -1).
cudaError_t launch_chunk_widen(const ChunkParams& p, int head_dim, const ChunkWiden* work, int n_events, int n_spans,
                               void* k_out, void* v_out, int32_t* table, int columns, cudaStream_t s);
// Rotates q into q_out and k_new into the pools, v_new goes with it.  most: new tokens of the page that takes the most.
cudaError_t launch_chunk_rope(const ChunkParams& p, int head_dim, int kv_format, const pad_rope& rope, const ChunkPages* work,
                              int n_work, int most, int64_t n_tokens, int sms, const int32_t* position, const void* q, int64_t q_stride,
                              void* q_out, int64_t out_stride, const void* k_new, const void* v_new, int64_t new_stride,
                              void* k_pool, void* v_pool, uint8_t* k_scale, uint8_t* v_scale, cudaStream_t s);
// rows16: 16-row groups that the items' rows take, 1 or 2.  early: not the call's first kernel.
cudaError_t launch_chunk_mma(const ChunkParams& p, int head_dim, bool fp8, int rows16, bool early, const ChunkItem* items,
                             int n_items, cudaStream_t s);
// The same over 4-bit pages; rows8: groups of eight rows, 1 to 3.
cudaError_t launch_chunk_mma4(const ChunkParams& p, int head_dim, int rows8, bool early, const ChunkItem* items, int n_items,
                              cudaStream_t s);
int chunk_mma4_ctas(int head_dim, int rows8);  // that an SM takes
// split: one slot of 128 / group tokens per CTA, its tiles taken in turn by two halves; else two slots.
// prefix_tokens: tokens of k_prefix up to the last one that an item reads, 0 without prefix items.
cudaError_t launch_chunk_tc(const ChunkParams& p, int head_dim, bool fp8, bool split, int64_t prefix_tokens,
                            const ChunkItem* items, int n_items, cudaStream_t s);
// most: splits of the row that has the most.
cudaError_t launch_chunk_merge(const ChunkParams& p, int head_dim, int most, const ChunkMerge* work, int n_work, cudaStream_t s);
cudaError_t launch_draft_verify(const ChunkParams& p, const ChunkVerify* work, int n_events, int vocab, bool bf16,
                                const void* tp, int64_t p_stride, const void* dq, int64_t q_stride,
                                const int32_t* draft, const float* u_accept, const float* u_pick, int32_t* accepted,
                                int32_t* token, cudaStream_t s);

// The rows of logits of a plan's new tokens turned into probabilities.
struct ChunkProbs {
  const void* logits;
  void* p;
  int64_t logits_stride, p_stride;
  const float* params;         // [n_events][4]: temperature, repetition, frequency, presence; or NULL
  const int32_t* tokens;       // [n_tokens], or NULL
  const int32_t* history;      // [n_events][history_width]
  const int32_t* history_len;
  const int32_t* bias_token;   // [n_events][bias_width]
  const float* bias_value;
  const int32_t* bias_len;
  const uint32_t* mask;        // [n_tokens][mask_stride] words of 32 tokens, or NULL
  int64_t mask_stride;
  int32_t history_width, bias_width, vocab, n_events, longest;  // longest: tokens of the longest chunk
  int32_t logits_bf16, p_bf16;
};
int chunk_probs_max_vocab();
cudaError_t launch_chunk_probs(const ChunkProbs& a, const ChunkVerify* work, int n_tokens, cudaStream_t s);

#ifdef __CUDACC__
// Programmatic dependent launch, within one call: its first kernel is launched in plain stream order (its work
// list may still be on its way when it is enqueued, by a copy, which griddepcontrol.wait does not cover); a
// later one may start early, reads its work list, then waits for the grid ahead, and everything after that
// wait is as in plain stream order.  What a grid ahead may have written is read past L1's read-only path.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <class... KArgs, class... Args>
cudaError_t launch_early(bool early, void (*kernel)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t s,
                         Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// Multiplier that turns an e4m3 code whose bits sit where bf16 has its exponent and upper
// mantissa (so that it reads as value * 2^-120) into code * 2^k, as a bf16 pattern: 2^(120 + k),
// with k = byte - 127.  Byte 0 stands for a group of zeros, 255 for one that holds a NaN.
__device__ __forceinline__ uint32_t scale_mult(uint32_t byte) {
  if (byte == 0u) return 0u;
  if (byte == 255u) return 0x7fc0u;
  return (min(max(byte, 7u), 134u) + 120u) << 7;
}
// Two e4m3 codes, in the upper bytes of x's halves, times a pair of multipliers: bf16 values,
// exactly (three bits of mantissa, and bf16 arithmetic keeps subnormals).
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t x, uint32_t mult) {
  const uint32_t b = ((x >> 4) & 0x07f007f0u) | (x & 0x80008000u);
  const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&b), *reinterpret_cast<const __nv_bfloat162*>(&mult));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// The eight e2m1 codes of x as four f16 pairs, exactly: pair j holds the codes 2 j (its lower half) and 2 j + 1.
__device__ __forceinline__ void f16_of_e2m1(uint32_t x, uint32_t (&h)[4]) {
  asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
      " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}\n"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(x));
}
__device__ __forceinline__ uint32_t f16_times(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// (six significant bits at most: exact)
__device__ __forceinline__ uint32_t bf16_of_f16(uint32_t h) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  const __nv_bfloat162 r = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&r);
}
#endif

}  // namespace pad
