// C ABI of the multi-token step (pad_chunk_*, pad_draft_verify): argument checks, page allocation, the
// work lists and their launches.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <exception>
#include <stdexcept>
#include <vector>

#include <nvtx3/nvToolsExt.h>

#include "pad_chunk.h"
#include "pad_wide.h"

static_assert(sizeof(pad_chunk_info) == 64, "prefix_tokens takes what was padding: the struct keeps its size");

using namespace pad;

namespace {

struct Range {
  explicit Range(const char* name) { nvtxRangePushA(name); }
  ~Range() { nvtxRangePop(); }
  Range(const Range&) = delete;
  Range& operator=(const Range&) = delete;
};

constexpr int64_t kMaxLen = 1 << 30;
constexpr int64_t kMaxTokens = INT32_MAX / 2;  // packed new tokens of a step
constexpr int kSplitUnit = 64;                 // key ranges are multiples of this
constexpr int kMinSplit = 256;
// Rows of a branch (tokens x group) up to which the warp-level kernel takes it: two 16-row groups.  13 branches
// of 35 rows over a prefix of 8219 take 25.4 us with this limit, 29.7 with 48 or 64, where they go in pieces.
constexpr int kMmaRows = 32;
// The same over 4-bit pages, which the warp-level kernel takes in pieces of some 16 rows that each widen the keys again; beyond
// it they are widened once, to bf16 pages in the workspace, for the tcgen05 kernel.  (us; 56, 112, 196 rows, 28/4 heads,
// head_dim 128: 16 sequences of 2048 to 8192 keys, in pieces 60, 109, 170, widened 87, 91, 101; one of 30000, 31, 46, 72 and
// 42, 43, 51.  14/2 heads, head_dim 64: 25, 37, 61 and 35, 36, 45; 21, 25, 31 and 27, 29, 29.)
constexpr int kMma4Rows = 96;

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

pad_status cuda_fail(cudaError_t e, const char* what) { return api_fail(PAD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e)); }

// Runs f; an exception (host memory) becomes a status at the C boundary.
template <class F>
pad_status guarded(F f) noexcept {
  try {
    return f();
  } catch (const std::exception& e) {
    return api_fail(PAD_ERR_UNSUPPORTED, "host planning failed: %s", e.what());
  } catch (...) {
    return api_fail(PAD_ERR_UNSUPPORTED, "host planning failed");
  }
}

struct Batch {
  const pad_problem* prob;
  int32_t kv_format, n_videos;
  const int32_t* prefix_len;
  int32_t n_events;
  const int32_t *event_video, *event_len, *n_new;
};

pad_status check_batch(const Batch& b) {
  pad_status st = api_check_problem(b.prob);
  if (st != PAD_OK) return st;
  if (b.prob->flags & ~(PAD_FLAG_PREFIX_MMA | PAD_FLAG_PREFIX_TC))
    return api_fail(PAD_ERR_UNSUPPORTED, "flags 0x%x: a multi-token step takes PAD_FLAG_PREFIX_MMA or PAD_FLAG_PREFIX_TC", b.prob->flags);
  if (b.kv_format != PAD_KV_BF16 && b.kv_format != PAD_KV_FP8 && b.kv_format != PAD_KV_FP4)
    return api_fail(PAD_ERR_INVALID_ARG, "kv_format=%d (0 = bf16, 1 = 8 bits, 4 = 4 bits)", b.kv_format);
  if (b.n_videos < 0 || b.n_events < 0) return api_fail(PAD_ERR_INVALID_ARG, "negative count");
  if (b.n_events > (1 << 20) || b.n_videos > (1 << 20)) return api_fail(PAD_ERR_UNSUPPORTED, "more than 2^20 events or videos");
  if (b.n_videos > 0 && !b.prefix_len) return api_fail(PAD_ERR_INVALID_ARG, "prefix_len is NULL");
  if (b.n_events > 0 && (!b.event_len || !b.n_new || (b.n_videos > 0 && !b.event_video)))
    return api_fail(PAD_ERR_INVALID_ARG, "an event array is NULL");
  for (int v = 0; v < b.n_videos; ++v)
    if (b.prefix_len[v] < 0 || b.prefix_len[v] > kMaxLen) return api_fail(PAD_ERR_INVALID_ARG, "prefix_len[%d]=%d", v, b.prefix_len[v]);
  int64_t tokens = 0, spans = 0;  // (a read's grid is one CTA per span)
  for (int e = 0; e < b.n_events; ++e) {
    if (b.event_len[e] < 0 || b.n_new[e] < 0 || (int64_t)b.event_len[e] + b.n_new[e] > kMaxLen)
      return api_fail(PAD_ERR_INVALID_ARG, "event_len[%d]=%d, n_new[%d]=%d", e, b.event_len[e], e, b.n_new[e]);
    if (b.n_videos > 0) {
      const int v = b.event_video[e];
      if (v < 0 || v >= b.n_videos || (e > 0 && v < b.event_video[e - 1]))
        return api_fail(PAD_ERR_INVALID_ARG, "event_video[%d]=%d: non-decreasing within [0, %d)", e, v, b.n_videos);
    }
    tokens += b.n_new[e];
    spans += ((int64_t)b.event_len[e] + b.n_new[e] + chunk_read_tokens() - 1) / chunk_read_tokens();
  }
  if (tokens > kMaxTokens || spans > INT32_MAX) return api_fail(PAD_ERR_UNSUPPORTED, "too many tokens");
  return PAD_OK;
}

// The work lists (all but the page ids) and the layout of the workspace.
struct Lists {
  std::vector<ChunkItem> tc;             // items of the tcgen05 kernel
  std::vector<ChunkItem> pre, page;      // items of the warp-level kernel: of the prefixes, of the pages
  bool tc_split = false, has_prefix = false;
  int pre_rows = 1, page_rows = 1;       // rows of the warp-level kernels' tiles, in 16s (4-bit pages: in 8s)
  int pre_tokens = 1, page_tokens = 1;   // tokens of their items
  std::vector<ChunkMerge> merge;
  std::vector<ChunkPages> pages;
  std::vector<ChunkRead> read;
  std::vector<ChunkVerify> verify;
  std::vector<ChunkWiden> widen;
  int64_t n_tokens = 0, n_cached = 0, n_drafts = 0, partial_rows = 0;
  int64_t prefix_tokens = 0;             // of k_prefix, up to the last one read
  int64_t widen_pages = 0;
  int32_t widen_spans = 0, widen_columns = 0;
  int32_t most_in_page = 0, longest = 0;  // new tokens of the page that takes the most, of the branch that brings the most
  int32_t n_spans = 0, pre_splits = 0, page_splits = 0;
  size_t off_tc = 0, off_pre = 0, off_page = 0, off_merge = 0, off_pages = 0, off_read = 0, off_verify = 0, off_widen = 0, image_bytes = 0;
  size_t off_ml = 0, off_o = 0, off_wtable = 0, off_wk = 0, off_wv = 0, total = 0;
};

// Consecutive chunk tokens that attend to one sequence of keys.
struct Segment {
  int64_t src;
  int32_t keys;       // of its last token
  int32_t tok0, ntok;
  int32_t lim0, paged;
  bool tc;            // on the tcgen05 kernel
  int32_t n_splits, split_len;
  int64_t part_row;
};

// Key ranges of about `len` keys, all about as long.
void split_by(Segment& s, int64_t len, int64_t unit) {
  s.n_splits = (int32_t)std::max<int64_t>(1, (s.keys + len - 1) / len);
  const int64_t even = (s.keys + s.n_splits - 1) / s.n_splits;
  s.split_len = (int32_t)align_up((size_t)std::max<int64_t>(1, even), (size_t)unit);
  s.n_splits = std::max(1, (s.keys + s.split_len - 1) / s.split_len);
}

// The warp-level kernel's CTAs take 32 rows at most (16 when no segment has more: twice the CTAs per
// SM), and key ranges are cut so that there are some eight CTAs for each SM, no shorter than
// kMinSplit keys.  (16 x 1 token over 333k cached tokens, 28/4 heads: 121 us in bf16 and 91 in 8 bits; with four CTAs
// for each SM 127 and 98, with sixteen 133 and 110.  128 or 512 keys make no difference beyond a short call's noise.)
// 4-bit pages: tiles of eight rows, up to three; a branch of more rows in pieces of about as many tokens.  The ranges there
// are the shortest that make no more CTAs than fit the GPU at once: a CTA's start and end cost as much as two of
// its blocks, and a few CTAs beyond one wave as much as the wave.
void cut_mma(std::vector<Segment>& segs, int paged, const pad_problem& prob, bool fp4, int sms, int& rows, int& tpt) {
  const int G = prob.h_q / prob.h_kv;
  int longest = 1;
  for (const Segment& s : segs)
    if (!s.tc && s.paged == paged) longest = std::max(longest, s.ntok);
  if (fp4) {
    // (one tile of up to 24 rows takes 29 us where two of 16 take 34, four of 14 take 60 where two of 28 take 65: 21 and
    // 56 rows over 16 sequences as above)
    const int most = longest * (int64_t)G <= 24 ? longest : 16 / G, pieces = (longest + most - 1) / most;
    tpt = (longest + pieces - 1) / pieces;
    rows = (tpt * G + 7) / 8;
  } else {
    rows = (int64_t)longest * G <= 16 ? 1 : 2;
    tpt = 16 * rows / G;
  }
  double work = 0;
  int64_t least = 0, longest_keys = 0;  // CTAs if nothing is cut
  for (const Segment& s : segs)
    if (!s.tc && s.paged == paged) {
      const int64_t n = (int64_t)((s.ntok + tpt - 1) / tpt) * prob.h_kv;
      work += (double)n * s.keys;
      least += n;
      longest_keys = std::max<int64_t>(longest_keys, s.keys);
    }
  double per = work / (8.0 * sms);
  const int64_t slots = fp4 ? (int64_t)chunk_mma4_ctas(prob.head_dim, rows) * sms : 0;
  const bool one_wave = fp4 && least <= slots;
  if (one_wave) per = work / (double)slots;
  int64_t len = std::max<int64_t>(kMinSplit, ((int64_t)(per / kSplitUnit) + 1) * kSplitUnit);
  auto ctas = [&]() {
    int64_t n = 0;
    for (const Segment& s : segs)
      if (!s.tc && s.paged == paged) n += (int64_t)((s.ntok + tpt - 1) / tpt) * prob.h_kv * ((s.keys + len - 1) / len);
    return n;
  };
  if (one_wave)
    while (len < longest_keys && ctas() > slots) len += std::max<int64_t>(1, len / (16 * kSplitUnit)) * kSplitUnit;
  for (Segment& s : segs)
    if (!s.tc && s.paged == paged) split_by(s, len, kSplitUnit);
}

// CTAs of a kernel that runs one per SM, the longest first: the time until the last ends.  Loads are kept as
// (load, SMs that have it); CTAs of one length are dealt out together.
double makespan(std::vector<std::pair<double, int64_t>>& ctas, int sms) {
  std::sort(ctas.begin(), ctas.end(), [](auto& x, auto& y) { return x.first > y.first; });
  std::vector<std::pair<double, int64_t>> load{{0.0, sms}};  // ascending
  double last = 0;
  for (auto [len, n] : ctas) {
    while (n > 0) {
      // (more CTAs of one length than can matter one by one: whole rounds at once)
      const int64_t k = std::min(n, load[0].second);
      const double at = load[0].first + len;
      n -= k;
      load[0].second -= k;
      if (load[0].second == 0) load.erase(load.begin());
      auto it = std::lower_bound(load.begin(), load.end(), at, [](auto& x, double v) { return x.first < v; });
      if (it != load.end() && it->first == at) it->second += k;
      else load.insert(it, {at, k});
      last = std::max(last, at);
    }
  }
  return last;
}

// The tcgen05 kernel: both of its forms and the length of the key ranges (in tiles) are costed with what was
// measured on GB300 (us; 152 CTAs at work, from 4096 and 12288 keys, pages of 16): a CTA's start and end, a tile
// of each form by head_dim and by where its keys are, the partial states' way out and in again.
// With one form for everything (us): 129 tokens over 32768, 28/4 heads, two slots 81.5, one slot 75;
// 2048 tokens over 30720 in pages, 640 and 800; 8-bit chunks of head_dim 64, 177 and 280.
// The costs are those of pages of 16.  Two slots and one on other pages (us, 1024 tokens over 8192, where two are taken;
// head_dim 128, 28/4 heads | 64, 14/2 heads): pages of 4, 148 and 177 | 71 and 72; of 8, 130 and 197 | 69 and 86; of 16,
// 122 and 152 | 71 and 68; of 32, 122 and 132 | 70 and 62; of 64, 120 and 124 | 71 and 58.  In 8 bits the page size makes no
// difference: 175 and 242 to 246 | 77 and 104.
constexpr double kTcCta = 7.0, kPartialRate = 4e6;  // bytes per us
constexpr double kTile[2][2][3] = {  // [one slot per CTA][head_dim 64][prefix, bf16 pages, 8-bit pages]
    {{1.49, 1.53, 2.55}, {1.30, 1.22, 1.60}},
    {{0.69, 1.01, 2.17}, {0.61, 0.78, 1.38}}};
void cut_tc(std::vector<Segment>& segs, const pad_problem& prob, bool fp8, int sms, bool& split) {
  const int tps = 128 / (prob.h_q / prob.h_kv);
  auto tiles_of = [](const Segment& s) { return ((int64_t)s.keys + 127) / 128; };
  int64_t longest = 0;
  double total = 0;
  for (const Segment& s : segs) {
    if (!s.tc) continue;
    longest = std::max(longest, tiles_of(s));
    total += (double)tiles_of(s) * (double)((s.ntok + tps - 1) / tps) * prob.h_kv;
  }
  if (longest == 0) return;
  double best = 1e300;
  int64_t best_len = longest;
  std::vector<std::pair<double, int64_t>> ctas;
  for (int form = 0; form < 2; ++form) {
    const int tpc = form ? tps : 2 * tps;
    const double* tile = kTile[form][prob.head_dim == 64];
    // (ranges much shorter than an SM's share of the work only add starts)
    const int64_t least = std::max<int64_t>(1, (int64_t)(total / sms / 12));
    for (int64_t len = longest;;) {
      ctas.clear();
      double bytes = 0;
      for (const Segment& s : segs) {
        if (!s.tc) continue;
        const int64_t tiles = tiles_of(s), n = (tiles + len - 1) / len, each = (tiles + n - 1) / n;
        ctas.push_back({kTcCta + tile[s.paged + (fp8 && s.paged)] * (double)each, (int64_t)((s.ntok + tpc - 1) / tpc) * prob.h_kv * n});
        if (n > 1 || !s.paged) bytes += 2.0 * (double)n * s.ntok * prob.h_q * (prob.head_dim + 2) * 4;
      }
      const double t = makespan(ctas, sms) + bytes / kPartialRate;
      if (t < best) {
        best = t;
        best_len = len;
        split = form != 0;
      }
      if (len <= least) break;
      // the next length that changes the longest one's count of ranges (in steps of an eighth where that is slow)
      const int64_t n = (longest + len - 1) / len;
      len = std::max<int64_t>(least, std::min(len - 1, std::min((longest + n) / (n + 1), n > 8 ? len * 15 / 16 : len)));
    }
  }
  for (Segment& s : segs)
    if (s.tc) split_by(s, best_len * 128, 128);
}

// tpt: tokens per item.
void items_of(const Segment& s, const pad_problem& prob, int tpt, std::vector<ChunkItem>& out) {
  for (int t = 0; t < s.ntok; t += tpt)
    for (int k = 0; k < s.n_splits; ++k) {
      ChunkItem it;
      it.src = s.src;
      it.tok0 = s.tok0 + t;
      it.ntok = std::min(tpt, s.ntok - t);
      it.lim0 = s.lim0 + (s.paged ? t : 0);
      it.paged = s.paged;
      it.key0 = (int32_t)std::min<int64_t>((int64_t)k * s.split_len, s.keys);
      const int32_t seen = s.paged ? it.lim0 + it.ntok - 1 : s.keys;
      it.key1 = (int32_t)std::min<int64_t>((int64_t)(k + 1) * s.split_len, seen);
      it.part_row = s.part_row < 0 ? -1 : s.part_row + ((int64_t)k * s.ntok + t) * prob.h_q;
      out.push_back(it);
    }
}

void build(const Batch& b, const int64_t* prefix_offset, Lists& L) {
  const pad_problem& prob = *b.prob;
  const int ps = prob.page_size, span = chunk_read_tokens();
  const int sms = prob.num_sms > 0 ? prob.num_sms : api_num_sms();
  const int G = prob.h_q / prob.h_kv;
  const bool fp4 = b.kv_format == PAD_KV_FP4;
  std::vector<Segment> segs;
  std::vector<int32_t> pre_of(b.n_events, -1), own_of(b.n_events, -1);
  int32_t open = -1;  // the video whose prefix segment is growing
  std::vector<int64_t> off(b.n_videos);
  int64_t o = 0;
  for (int v = 0; v < b.n_videos; ++v) {
    off[v] = prefix_offset ? prefix_offset[v] : o;
    o += b.prefix_len[v];
  }
  for (int e = 0; e < b.n_events; ++e) {
    const int n = b.n_new[e], len = b.event_len[e], v = b.n_videos > 0 ? b.event_video[e] : -1;
    const int32_t tok0 = (int32_t)L.n_tokens;
    if (n > 0 && v >= 0 && b.prefix_len[v] > 0) {
      if (open < 0 || segs[open].src != v) {
        open = (int32_t)segs.size();
        segs.push_back({v, b.prefix_len[v], tok0, 0, b.prefix_len[v], 0, false, 0, 0, -1});
      }
      segs[open].ntok += n;
      pre_of[e] = open;
    }
    if (n > 0) {
      own_of[e] = (int32_t)segs.size();
      segs.push_back({e, len + n, tok0, n, len + 1, 1, false, 0, 0, -1});
    }
    for (int i = 0; i < n;) {
      const int pos = len + i, count = std::min(n - i, ps - pos % ps);
      L.pages.push_back({e, pos / ps, -1, tok0 + i, pos % ps, count});
      L.most_in_page = std::max(L.most_in_page, count);
      i += count;
    }
    L.read.push_back({L.n_cached, L.n_spans, len + n});
    L.n_spans += (int32_t)(((int64_t)len + n + span - 1) / span);
    L.longest = std::max(L.longest, n);
    L.verify.push_back({tok0, n - 1, (int32_t)L.n_drafts});
    L.n_tokens += n;
    L.n_cached += (int64_t)len + n;
    L.n_drafts += std::max(0, n - 1);
  }
  for (Segment& s : segs) {
    if (prob.flags & (PAD_FLAG_PREFIX_MMA | PAD_FLAG_PREFIX_TC)) s.tc = (prob.flags & PAD_FLAG_PREFIX_TC) != 0;
    else s.tc = !s.paged || (int64_t)s.ntok * G > (fp4 ? kMma4Rows : kMmaRows);
  }
  cut_tc(segs, prob, b.kv_format == PAD_KV_FP8, sms, L.tc_split);
  cut_mma(segs, 0, prob, false, sms, L.pre_rows, L.pre_tokens);
  cut_mma(segs, 1, prob, fp4, sms, L.page_rows, L.page_tokens);
  for (const Segment& s : segs) {
    int32_t& most = s.paged ? L.page_splits : L.pre_splits;
    most = std::max(most, s.n_splits);
  }
  // a token whose keys are in more than one piece is joined from partial states
  auto partial = [&](Segment& s) {
    s.part_row = L.partial_rows;
    L.partial_rows += (int64_t)s.n_splits * s.ntok * prob.h_q;
  };
  for (Segment& s : segs)
    if (!s.paged) partial(s);  // (the tokens' own keys are a second piece at least)
  for (int e = 0; e < b.n_events; ++e)
    if (own_of[e] >= 0 && (pre_of[e] >= 0 || segs[own_of[e]].n_splits > 1)) {
      Segment& s = segs[own_of[e]];
      partial(s);
      for (int i = 0; i < s.ntok; ++i) {
        ChunkMerge m{};
        m.tok = s.tok0 + i;
        m.page_n = s.n_splits;
        m.page_row = s.part_row + (int64_t)i * prob.h_q;
        m.page_stride = (int64_t)s.ntok * prob.h_q;
        if (pre_of[e] >= 0) {
          const Segment& q = segs[pre_of[e]];
          m.pre_n = q.n_splits;
          m.pre_row = q.part_row + (int64_t)(m.tok - q.tok0) * prob.h_q;
          m.pre_stride = (int64_t)q.ntok * prob.h_q;
        }
        L.merge.push_back(m);
      }
    }
  for (Segment& s : segs) {
    if (s.paged && s.tc && fp4) {
      const int32_t columns = (s.keys + ps - 1) / ps;
      L.widen.push_back({(int32_t)s.src, (int32_t)L.widen_pages, L.widen_spans, s.keys});
      s.src = (int64_t)L.widen.size() - 1;
      L.widen_pages += columns;
      if (L.widen_pages > INT32_MAX) throw std::length_error("too many cached tokens to widen");
      L.widen_spans += (s.keys + span - 1) / span;
      L.widen_columns = std::max(L.widen_columns, columns);
    }
    if (!s.paged) {
      s.src = off[s.src];
      L.has_prefix = true;
      L.prefix_tokens = std::max(L.prefix_tokens, s.src + s.keys);
    }
    if (s.tc) items_of(s, prob, (L.tc_split ? 1 : 2) * (128 / G), L.tc);
    else items_of(s, prob, s.paged ? L.page_tokens : L.pre_tokens, s.paged ? L.page : L.pre);
  }
  // the longest first: what is left at the end of the grid is short
  auto longer = [](const ChunkItem& x, const ChunkItem& y) { return x.key1 - x.key0 > y.key1 - y.key0; };
  std::stable_sort(L.tc.begin(), L.tc.end(), longer);
  std::stable_sort(L.page.begin(), L.page.end(), longer);
  size_t at = sizeof(PadDevHeader);
  auto place = [&](size_t& where, size_t bytes) {
    where = at;
    at = align_up(at + bytes, 16);
  };
  place(L.off_tc, L.tc.size() * sizeof(ChunkItem));
  place(L.off_pre, L.pre.size() * sizeof(ChunkItem));
  place(L.off_page, L.page.size() * sizeof(ChunkItem));
  place(L.off_merge, L.merge.size() * sizeof(ChunkMerge));
  place(L.off_pages, L.pages.size() * sizeof(ChunkPages));
  place(L.off_read, L.read.size() * sizeof(ChunkRead));
  place(L.off_verify, L.verify.size() * sizeof(ChunkVerify));
  place(L.off_widen, L.widen.size() * sizeof(ChunkWiden));
  L.image_bytes = at - sizeof(PadDevHeader);
  at = align_up(at, 256);
  L.off_ml = at;
  at = align_up(at + (size_t)L.partial_rows * sizeof(float2), 256);
  L.off_o = at;
  at = align_up(at + (size_t)L.partial_rows * prob.head_dim * sizeof(float), 256);
  const size_t wide = (size_t)L.widen_pages * prob.h_kv * ps * prob.head_dim * 2;
  L.off_wtable = at;
  at = align_up(at + L.widen.size() * (size_t)L.widen_columns * sizeof(int32_t), 256);
  L.off_wk = at;
  at = align_up(at + wide, 256);
  L.off_wv = at;
  at = align_up(at + wide, 256);
  L.total = at;
}

}  // namespace

struct pad_chunk_t {
  pad_problem prob{};
  int32_t kv_format = 0, n_events = 0, max_pages = 0, n_pages = 0;
  int32_t* page_table = nullptr;
  uint8_t* workspace = nullptr;
  uint64_t gen = 0;
  bool from_cache = false, committed = false;
  Lists L;
  std::vector<int32_t> event_len, n_new;
  std::vector<int32_t> new_event, new_column, new_page;
};

namespace {

ChunkParams params_of(const pad_chunk_t* c) {
  ChunkParams p{};
  p.h_q = c->prob.h_q;
  p.h_kv = c->prob.h_kv;
  p.group = p.h_q / p.h_kv;
  p.page_size = c->prob.page_size;
  while ((1 << p.page_shift) < p.page_size) ++p.page_shift;
  p.max_pages = c->max_pages;
  p.n_pages = c->n_pages;
  p.out_bf16 = c->prob.out_dtype == 1;
  p.scale_log2 = (float)((double)c->prob.scale * 1.4426950408889634);
  p.gen = c->gen;
  p.header = reinterpret_cast<PadDevHeader*>(c->workspace);
  p.page_table = c->page_table;
  p.part_ml = reinterpret_cast<float2*>(c->workspace + c->L.off_ml);
  p.part_o = reinterpret_cast<float*>(c->workspace + c->L.off_o);
  return p;
}

template <class T>
const T* list(const pad_chunk_t* c, size_t off) {
  return reinterpret_cast<const T*>(c->workspace + off);
}

pad_status check_launch(const pad_chunk_t* c, bool pages) {
  if (!c) return api_fail(PAD_ERR_INVALID_ARG, "chunk is NULL");
  if (!c->workspace) return api_fail(PAD_ERR_INVALID_ARG, "a host-only plan cannot be launched");
  if (pages && !c->page_table) return api_fail(PAD_ERR_INVALID_ARG, "the plan has no page table");
  return PAD_OK;
}

pad_status check_pools(const pad_chunk_t* c, const void* k_pool, const void* v_pool, const void* k_scale, const void* v_scale) {
  if (!k_pool || !v_pool) return api_fail(PAD_ERR_INVALID_ARG, "NULL pool");
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16)) return api_fail(PAD_ERR_INVALID_ARG, "pools must be 16-byte aligned");
  if (c->kv_format != PAD_KV_BF16) {
    if (!k_scale || !v_scale)
      return api_fail(PAD_ERR_INVALID_ARG, "%s cache needs its scale pools", c->kv_format == PAD_KV_FP8 ? "an 8-bit" : "a 4-bit");
    if (!aligned(k_scale, 16) || !aligned(v_scale, 16)) return api_fail(PAD_ERR_INVALID_ARG, "scale pools must be 16-byte aligned");
  } else if (k_scale || v_scale) {
    return api_fail(PAD_ERR_INVALID_ARG, "a bf16 cache has no scale pools");
  }
  return PAD_OK;
}

// Elements from one row to the next; 0 = packed.
pad_status check_stride(int64_t& stride, int64_t packed, int64_t unit, const char* what) {
  if (stride == 0) stride = packed;
  if (stride < packed || stride % unit != 0 || stride > ((int64_t)1 << 40))
    return api_fail(PAD_ERR_INVALID_ARG, "%s stride %lld: at least %lld, a multiple of %lld", what, (long long)stride,
                    (long long)packed, (long long)unit);
  return PAD_OK;
}

// Whether `rows` rows of `width` elements at a and of `width_b` at b (of two bytes, strides in elements) share memory.
bool overlap(const void* a, int64_t stride, int64_t width, const void* b, int64_t stride_b, int64_t width_b, int64_t rows) {
  const intptr_t x = reinterpret_cast<intptr_t>(a) / 2, y = reinterpret_cast<intptr_t>(b) / 2;
  if (x + (rows - 1) * stride + width <= y || y + (rows - 1) * stride_b + width_b <= x) return false;
  if (stride != stride_b) return true;
  const int64_t d = ((int64_t)(y - x) % stride + stride) % stride;  // columns of rows that lie one within the other
  return d < width || d > stride - width_b;
}

}  // namespace

extern "C" {

size_t pad_chunk_workspace_size(const pad_problem* prob, int32_t kv_format, int32_t n_videos, const int32_t* prefix_len,
                                int32_t n_events, const int32_t* event_video, const int32_t* event_len,
                                const int32_t* n_new) {
  size_t bytes = 0;
  guarded([&] {
    const Batch b{prob, kv_format, n_videos, prefix_len, n_events, event_video, event_len, n_new};
    pad_status st = check_batch(b);
    if (st != PAD_OK) return st;
    Lists L;
    build(b, nullptr, L);
    bytes = L.total;
    return PAD_OK;
  });
  return bytes;
}

pad_status pad_chunk_plan(const pad_problem* prob, int32_t kv_format, pad_cache_state* cache, int32_t n_videos,
                          const int32_t* prefix_len, const int64_t* prefix_offset, int32_t n_events,
                          const int32_t* event_video, const int32_t* event_len, const int32_t* n_new,
                          int32_t* page_table, int32_t max_pages, int32_t n_pages, void* workspace,
                          size_t workspace_bytes, pad_stream_t stream, pad_chunk_t** out) {
  Range r("pad_chunk_plan");
  if (!out) return api_fail(PAD_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  pad_chunk_t* made = nullptr;
  pad_status st = guarded([&]() -> pad_status {
    const Batch b{prob, kv_format, n_videos, prefix_len, n_events, event_video, event_len, n_new};
    pad_status s = check_batch(b);
    if (s != PAD_OK) return s;
    if (max_pages < 0 || n_pages < 0) return api_fail(PAD_ERR_INVALID_ARG, "negative page count");
    if (cache) {
      const int32_t size = pad_cache_state_num_pages(cache);
      if (n_pages != 0 && n_pages != size) return api_fail(PAD_ERR_INVALID_ARG, "n_pages=%d, the cache has %d", n_pages, size);
      n_pages = size;
    }
    if (kv_format == PAD_KV_FP4 && (int64_t)n_pages * prob->h_kv * prob->page_size > UINT32_MAX)
      return api_fail(PAD_ERR_UNSUPPORTED, "a 4-bit pool of %d pages has more than 2^32 rows", n_pages);
    if (prefix_offset)
      for (int v = 0; v < n_videos; ++v)
        if (prefix_offset[v] < 0 || prefix_offset[v] > ((int64_t)1 << 40)) return api_fail(PAD_ERR_INVALID_ARG, "prefix_offset[%d]", v);
    if (page_table) {
      if (!aligned(page_table, 4)) return api_fail(PAD_ERR_INVALID_ARG, "page_table must be 4-byte aligned");
      for (int e = 0; e < n_events; ++e)
        if (((int64_t)event_len[e] + n_new[e] + prob->page_size - 1) / prob->page_size > max_pages)
          return api_fail(PAD_ERR_INVALID_ARG, "event %d needs more than max_pages=%d pages", e, max_pages);
    } else if (cache) {
      return api_fail(PAD_ERR_INVALID_ARG, "a plan with a cache needs its page table");
    }
    if (workspace && !aligned(workspace, 256)) return api_fail(PAD_ERR_INVALID_ARG, "workspace must be 256-byte aligned");

    made = new pad_chunk_t();
    pad_chunk_t* c = made;
    c->prob = *prob;
    c->kv_format = kv_format;
    c->n_events = n_events;
    c->max_pages = max_pages;
    c->n_pages = n_pages;
    c->page_table = page_table;
    c->gen = api_next_generation();
    c->from_cache = cache != nullptr;
    if (n_events > 0) {
      c->event_len.assign(event_len, event_len + n_events);
      c->n_new.assign(n_new, n_new + n_events);
    }
    build(b, prefix_offset, c->L);
    if (c->L.prefix_tokens > INT32_MAX) return api_fail(PAD_ERR_UNSUPPORTED, "prefixes past 2^31 tokens of k_prefix");
    if (workspace && workspace_bytes < c->L.total)
      return api_fail(PAD_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, the plan needs %zu", workspace_bytes, c->L.total);
    if (cache) {
      // found first, taken last: an error takes no page
      int from = 0;
      for (ChunkPages& w : c->L.pages) {
        if (w.slot != 0) continue;  // (the page that the branch's last cached token is in)
        const int pg = api_next_free_page(cache, from);
        if (pg < 0) return api_fail(PAD_ERR_OUT_OF_PAGES, "%d free pages do not cover the step", pad_cache_state_free_count(cache));
        from = pg + 1;
        w.page = pg;
        c->new_event.push_back(w.event);
        c->new_column.push_back(w.column);
        c->new_page.push_back(pg);
      }
    }
    if (workspace) {
      c->workspace = static_cast<uint8_t*>(workspace);
      std::vector<uint8_t> image(c->L.image_bytes);
      auto put = [&](size_t off, const void* src, size_t n) {
        if (n) memcpy(image.data() + off - sizeof(PadDevHeader), src, n);
      };
      put(c->L.off_tc, c->L.tc.data(), c->L.tc.size() * sizeof(ChunkItem));
      put(c->L.off_pre, c->L.pre.data(), c->L.pre.size() * sizeof(ChunkItem));
      put(c->L.off_page, c->L.page.data(), c->L.page.size() * sizeof(ChunkItem));
      put(c->L.off_merge, c->L.merge.data(), c->L.merge.size() * sizeof(ChunkMerge));
      put(c->L.off_pages, c->L.pages.data(), c->L.pages.size() * sizeof(ChunkPages));
      put(c->L.off_read, c->L.read.data(), c->L.read.size() * sizeof(ChunkRead));
      put(c->L.off_verify, c->L.verify.data(), c->L.verify.size() * sizeof(ChunkVerify));
      put(c->L.off_widen, c->L.widen.data(), c->L.widen.size() * sizeof(ChunkWiden));
      if (!image.empty()) {
        cudaError_t e = api_copy_in(c->workspace + sizeof(PadDevHeader), image.data(), image.size(),
                                    reinterpret_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) return cuda_fail(e, "copying the work lists");
      }
    }
    for (int32_t pg : c->new_page) api_take_page(cache, pg);
    return PAD_OK;
  });
  if (st != PAD_OK) {
    delete made;
    return st;
  }
  *out = made;
  return PAD_OK;
}

pad_status pad_chunk_get_info(const pad_chunk_t* c, pad_chunk_info* info) {
  if (!c || !info) return api_fail(PAD_ERR_INVALID_ARG, "NULL argument");
  *info = pad_chunk_info{};
  info->n_tokens = c->L.n_tokens;
  info->n_cached = c->L.n_cached;
  info->n_drafts = c->L.n_drafts;
  info->workspace_bytes = (int64_t)c->L.total;
  info->partial_rows = c->L.partial_rows;
  info->n_new_pages = (int32_t)c->new_page.size();
  info->prefix_splits = c->L.pre_splits;
  info->page_splits = c->L.page_splits;
  info->tc_items = (int32_t)c->L.tc.size();
  info->mma_items = (int32_t)(c->L.pre.size() + c->L.page.size());
  info->prefix_tokens = (int32_t)c->L.prefix_tokens;
  return PAD_OK;
}

pad_status pad_chunk_new_pages(const pad_chunk_t* c, int32_t* event, int32_t* column, int32_t* page) {
  if (!c) return api_fail(PAD_ERR_INVALID_ARG, "chunk is NULL");
  const size_t n = c->new_page.size();
  if (n > 0 && (!event || !column || !page)) return api_fail(PAD_ERR_INVALID_ARG, "NULL argument");
  std::copy(c->new_event.begin(), c->new_event.end(), event);
  std::copy(c->new_column.begin(), c->new_column.end(), column);
  std::copy(c->new_page.begin(), c->new_page.end(), page);
  return PAD_OK;
}

pad_status pad_chunk_destroy(pad_chunk_t* c) {
  delete c;
  return PAD_OK;
}

pad_status pad_chunk_append(const pad_chunk_t* c, const void* k_new, const void* v_new, int64_t new_stride, void* k_pool,
                            void* v_pool, uint8_t* k_scale, uint8_t* v_scale, pad_stream_t stream) {
  Range r("pad_chunk_append");
  pad_status st = check_launch(c, true);
  if (st != PAD_OK) return st;
  st = check_stride(new_stride, (int64_t)c->prob.h_kv * c->prob.head_dim, 8, "k_new");
  if (st != PAD_OK) return st;
  if (c->L.pages.empty()) return PAD_OK;
  st = check_pools(c, k_pool, v_pool, k_scale, v_scale);
  if (st != PAD_OK) return st;
  if (!k_new || !v_new || !aligned(k_new, 16) || !aligned(v_new, 16))
    return api_fail(PAD_ERR_INVALID_ARG, "k_new and v_new must be 16-byte aligned tensors");
  cudaError_t e = launch_chunk_append(params_of(c), c->prob.head_dim, c->kv_format,
                                      list<ChunkPages>(c, c->L.off_pages), (int)c->L.pages.size(), k_new, v_new, new_stride,
                                      k_pool, v_pool, k_scale, v_scale, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PAD_OK : cuda_fail(e, "chunk append launch");
}

pad_status pad_rope_init(const pad_rope_spec* spec, pad_rope* rope) {
  if (!spec || !rope) return api_fail(PAD_ERR_INVALID_ARG, "NULL argument");
  const pad_rope_spec& s = *spec;
  const double R = s.rotary_dim;
  auto positive = [](double x) { return x > 0 && std::isfinite(x); };
  if (s.head_dim != 64 && s.head_dim != 128) return api_fail(PAD_ERR_UNSUPPORTED, "head_dim=%d (supported: 64, 128)", s.head_dim);
  if (s.rotary_dim < 2 || s.rotary_dim > s.head_dim || s.rotary_dim % 2 != 0)
    return api_fail(PAD_ERR_INVALID_ARG, "rotary_dim=%d: even, 2 to head_dim=%d", s.rotary_dim, s.head_dim);
  if (s.layout != PAD_ROPE_HALF && s.layout != PAD_ROPE_INTERLEAVED) return api_fail(PAD_ERR_INVALID_ARG, "layout=%d", s.layout);
  if (s.scaling < PAD_ROPE_NONE || s.scaling > PAD_ROPE_INDEX) return api_fail(PAD_ERR_INVALID_ARG, "scaling=%d", s.scaling);
  if (!positive(s.theta)) return api_fail(PAD_ERR_INVALID_ARG, "theta must be finite and > 0");
  if (!(std::fabs(s.magnitude) <= FLT_MAX)) return api_fail(PAD_ERR_INVALID_ARG, "magnitude must be finite in 32 bits");
  if (s.scaling != PAD_ROPE_NONE && !positive(s.factor)) return api_fail(PAD_ERR_INVALID_ARG, "factor must be finite and > 0");
  if (s.scaling == PAD_ROPE_BASE && s.rotary_dim < 4) return api_fail(PAD_ERR_INVALID_ARG, "a scaled base needs a rotary_dim of 4 at least");
  if (s.scaling == PAD_ROPE_TURNS || s.scaling == PAD_ROPE_INDEX) {
    if (!positive(s.original_len)) return api_fail(PAD_ERR_INVALID_ARG, "original_len must be finite and > 0");
    if (!(s.low < s.high) || !std::isfinite(s.low) || !std::isfinite(s.high)) return api_fail(PAD_ERR_INVALID_ARG, "low must be below high");
    if (s.scaling == PAD_ROPE_INDEX && (!(s.low > 0) || !(s.theta > 1)))
      return api_fail(PAD_ERR_INVALID_ARG, "a ramp over the index needs low > 0 and theta > 1");
  }
  double a = 0, b = 0;
  const Wide log_theta = wide_log(s.theta);
  if (s.scaling == PAD_ROPE_INDEX) {
    auto index = [&](double n) { return wide_log(Wide(s.original_len) / (wide_two_pi() * n)) * R / (log_theta * 2); };
    a = std::min(std::max(wide_floor(index(s.high)).hi, 0.0), R - 1);
    b = std::min(std::max(-wide_floor(-index(s.low)).hi, 0.0), R - 1);
  }
  const Wide log_base = s.scaling == PAD_ROPE_BASE ? log_theta + wide_log(s.factor) * R / (R - 2) : log_theta;
  pad_rope r{};
  r.head_dim = s.head_dim;
  r.rotary_dim = s.rotary_dim;
  r.layout = s.layout;
  r.magnitude = (float)s.magnitude;
  for (int i = 0; i < s.rotary_dim / 2; ++i) {
    Wide f = wide_exp(log_base * (-2.0 * i) / R), g = 1;
    if (s.scaling == PAD_ROPE_LINEAR) g = 0;
    if (s.scaling == PAD_ROPE_TURNS) g = (f * s.original_len / wide_two_pi() - s.low) / wide_sum(s.high, -s.low);
    if (s.scaling == PAD_ROPE_INDEX) g = Wide(1) - Wide(i - a) / std::max(b - a, 0.001);
    if (g < 0) g = 0;
    if (g < 1) f = f * (g + (Wide(1) - g) / s.factor);
    // as a fraction of a turn, 64 bits of it: whole turns a token make no difference
    const Wide turn = f / wide_two_pi();
    if (!std::isfinite(turn.hi)) return api_fail(PAD_ERR_INVALID_ARG, "the frequency of pair %d is not finite", i);
    const Wide part = turn - wide_floor(turn);
    const double hi = std::ldexp(part.hi, 64), whole = std::floor(hi), rest = std::nearbyint(hi - whole + std::ldexp(part.lo, 64));
    r.turn[i] = (whole < 0x1p64 ? (uint64_t)whole : 0) + (uint64_t)(int64_t)rest;
  }
  *rope = r;
  return PAD_OK;
}

pad_status pad_chunk_append_rope(const pad_chunk_t* c, const pad_rope* rope, const int32_t* position, const void* q,
                                 int64_t q_stride, void* q_out, int64_t out_stride, const void* k_new, const void* v_new,
                                 int64_t new_stride, void* k_pool, void* v_pool, uint8_t* k_scale, uint8_t* v_scale,
                                 pad_stream_t stream) {
  Range r("pad_chunk_append_rope");
  pad_status st = check_launch(c, true);
  if (st != PAD_OK) return st;
  if (!rope) return api_fail(PAD_ERR_INVALID_ARG, "rope is NULL");
  if (rope->head_dim != c->prob.head_dim || rope->rotary_dim < 2 || rope->rotary_dim > rope->head_dim || rope->rotary_dim % 2 != 0 ||
      (rope->layout != PAD_ROPE_HALF && rope->layout != PAD_ROPE_INTERLEAVED))
    return api_fail(PAD_ERR_INVALID_ARG, "rope is not of pad_rope_init for head_dim=%d", c->prob.head_dim);
  const int64_t q_width = (int64_t)c->prob.h_q * c->prob.head_dim, new_width = (int64_t)c->prob.h_kv * c->prob.head_dim;
  st = check_stride(q_stride, q_width, 8, "q");
  if (st == PAD_OK) st = check_stride(out_stride, q_width, 8, "q_out");
  if (st == PAD_OK) st = check_stride(new_stride, new_width, 8, "k_new");
  if (st != PAD_OK) return st;
  const int64_t n = c->L.n_tokens;
  if (n == 0) return PAD_OK;
  st = check_pools(c, k_pool, v_pool, k_scale, v_scale);
  if (st != PAD_OK) return st;
  if (!position || !aligned(position, 4)) return api_fail(PAD_ERR_INVALID_ARG, "position must be a 4-byte aligned tensor");
  for (const void* t : {q, static_cast<const void*>(q_out), k_new, v_new})
    if (!t || !aligned(t, 16)) return api_fail(PAD_ERR_INVALID_ARG, "q, q_out, k_new and v_new must be 16-byte aligned tensors");
  if ((q_out != q || out_stride != q_stride) && overlap(q, q_stride, q_width, q_out, out_stride, q_width, n))
    return api_fail(PAD_ERR_INVALID_ARG, "q_out overlaps q without being q");
  if (overlap(k_new, new_stride, new_width, q_out, out_stride, q_width, n) || overlap(v_new, new_stride, new_width, q_out, out_stride, q_width, n))
    return api_fail(PAD_ERR_INVALID_ARG, "q_out overlaps k_new or v_new");
  const int sms = c->prob.num_sms > 0 ? c->prob.num_sms : api_num_sms();
  cudaError_t e = launch_chunk_rope(params_of(c), c->prob.head_dim, c->kv_format, *rope, list<ChunkPages>(c, c->L.off_pages),
                                    (int)c->L.pages.size(), c->L.most_in_page, n, sms, position, q, q_stride, q_out, out_stride,
                                    k_new, v_new, new_stride, k_pool, v_pool, k_scale, v_scale, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PAD_OK : cuda_fail(e, "chunk append with rotary positions launch");
}

pad_status pad_chunk_probs(const pad_chunk_t* c, int32_t vocab, int32_t logits_dtype, const void* logits, int64_t logits_stride,
                           const float* params, const int32_t* tokens, const int32_t* history, int32_t history_width,
                           const int32_t* history_len, const int32_t* bias_token, const float* bias_value, int32_t bias_width,
                           const int32_t* bias_len, const int32_t* mask, int64_t mask_stride, int32_t p_dtype, void* p,
                           int64_t p_stride, pad_stream_t stream) {
  Range r("pad_chunk_probs");
  pad_status st = check_launch(c, false);
  if (st != PAD_OK) return st;
  if (vocab < 1 || vocab > chunk_probs_max_vocab()) return api_fail(PAD_ERR_UNSUPPORTED, "vocab=%d outside [1, %d]", vocab, chunk_probs_max_vocab());
  if ((logits_dtype != 0 && logits_dtype != 1) || (p_dtype != 0 && p_dtype != 1))
    return api_fail(PAD_ERR_INVALID_ARG, "logits_dtype=%d, p_dtype=%d (0 = fp32, 1 = bf16)", logits_dtype, p_dtype);
  st = check_stride(logits_stride, vocab, 1, "logits");
  if (st == PAD_OK) st = check_stride(p_stride, vocab, 1, "p");
  if (st == PAD_OK) st = check_stride(mask_stride, (vocab + 31) / 32, 1, "mask");
  if (st != PAD_OK) return st;
  if (history_width < 0 || bias_width < 0) return api_fail(PAD_ERR_INVALID_ARG, "negative width");
  if (!history != !history_len) return api_fail(PAD_ERR_INVALID_ARG, "history and history_len come together");
  if (!bias_token != !bias_value || !bias_token != !bias_len) return api_fail(PAD_ERR_INVALID_ARG, "bias_token, bias_value and bias_len come together");
  if (c->L.n_tokens == 0) return PAD_OK;
  if (!logits || !p) return api_fail(PAD_ERR_INVALID_ARG, "NULL tensor");
  for (const void* t : {static_cast<const void*>(params), static_cast<const void*>(tokens), static_cast<const void*>(history),
                        static_cast<const void*>(history_len), static_cast<const void*>(bias_token), static_cast<const void*>(bias_value),
                        static_cast<const void*>(bias_len), static_cast<const void*>(mask)})
    if (!aligned(t, 4)) return api_fail(PAD_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  if (!aligned(logits, logits_dtype ? 2 : 4) || !aligned(p, p_dtype ? 2 : 4))
    return api_fail(PAD_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  const int64_t l2 = logits_dtype ? 1 : 2, p2 = p_dtype ? 1 : 2;
  if ((p != logits || p_dtype != logits_dtype || p_stride != logits_stride) &&
      overlap(logits, logits_stride * l2, vocab * l2, p, p_stride * p2, vocab * p2, c->L.n_tokens))
    return api_fail(PAD_ERR_INVALID_ARG, "p overlaps logits without being logits");
  ChunkProbs a{};
  a.logits = logits;
  a.p = p;
  a.logits_stride = logits_stride;
  a.p_stride = p_stride;
  a.params = params;
  a.tokens = tokens;
  a.history = history;
  a.history_len = history_len;
  a.bias_token = bias_token;
  a.bias_value = bias_value;
  a.bias_len = bias_len;
  a.mask = reinterpret_cast<const uint32_t*>(mask);
  a.mask_stride = mask_stride;
  a.history_width = history_width;
  a.bias_width = bias_width;
  a.vocab = vocab;
  a.n_events = c->n_events;
  a.longest = c->L.longest;
  a.logits_bf16 = logits_dtype;
  a.p_bf16 = p_dtype;
  cudaError_t e = launch_chunk_probs(a, list<ChunkVerify>(c, c->L.off_verify), (int)c->L.n_tokens, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PAD_OK : cuda_fail(e, "logits to probabilities launch");
}

pad_status pad_chunk_read(const pad_chunk_t* c, const void* k_pool, const void* v_pool, const uint8_t* k_scale,
                          const uint8_t* v_scale, void* k_out, void* v_out, pad_stream_t stream) {
  Range r("pad_chunk_read");
  pad_status st = check_launch(c, true);
  if (st != PAD_OK) return st;
  if (c->L.n_spans == 0) return PAD_OK;
  st = check_pools(c, k_pool, v_pool, k_scale, v_scale);
  if (st != PAD_OK) return st;
  if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16))
    return api_fail(PAD_ERR_INVALID_ARG, "k_out and v_out must be 16-byte aligned tensors");
  ChunkParams p = params_of(c);
  p.k_pool = k_pool;
  p.v_pool = v_pool;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  cudaError_t e = launch_chunk_read(p, c->prob.head_dim, c->kv_format, list<ChunkRead>(c, c->L.off_read),
                                    c->n_events, c->L.n_spans, k_out, v_out, reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PAD_OK : cuda_fail(e, "chunk read launch");
}

pad_status pad_chunk_attn(const pad_chunk_t* c, const void* q, int64_t q_stride, const void* k_prefix, const void* v_prefix,
                          const void* k_pool, const void* v_pool, const uint8_t* k_scale, const uint8_t* v_scale,
                          void* out, float* lse, pad_stream_t stream) {
  Range r("pad_chunk_attn");
  pad_status st = check_launch(c, true);
  if (st != PAD_OK) return st;
  st = check_stride(q_stride, (int64_t)c->prob.h_q * c->prob.head_dim, 8, "q");
  if (st != PAD_OK) return st;
  if (c->L.n_tokens == 0) return PAD_OK;
  st = check_pools(c, k_pool, v_pool, k_scale, v_scale);
  if (st != PAD_OK) return st;
  if (!q || !out) return api_fail(PAD_ERR_INVALID_ARG, "NULL tensor");
  if (c->L.has_prefix && (!k_prefix || !v_prefix)) return api_fail(PAD_ERR_INVALID_ARG, "the plan has a prefix, k_prefix or v_prefix is NULL");
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(k_prefix, 16) || !aligned(v_prefix, 16) || !aligned(lse, 4))
    return api_fail(PAD_ERR_INVALID_ARG, "tensors must be 16-byte aligned (lse 4-byte)");
  ChunkParams p = params_of(c);
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.q_stride = q_stride;
  p.k_prefix = k_prefix;
  p.v_prefix = v_prefix;
  p.k_pool = k_pool;
  p.v_pool = v_pool;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  p.out = out;
  p.lse = lse;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  // the warp-level kernel first: its CTAs are short and share an SM, those of the other take one each
  const bool fp8 = c->kv_format == PAD_KV_FP8, fp4 = c->kv_format == PAD_KV_FP4;
  uint8_t* const ws = c->workspace;
  if (!c->L.widen.empty())  // (ahead of them all: what follows starts after it has ended)
    e = launch_chunk_widen(p, c->prob.head_dim, list<ChunkWiden>(c, c->L.off_widen), (int)c->L.widen.size(), c->L.widen_spans,
                           ws + c->L.off_wk, ws + c->L.off_wv, reinterpret_cast<int32_t*>(ws + c->L.off_wtable),
                           c->L.widen_columns, s);
  if (e == cudaSuccess && !c->L.pre.empty())
    e = launch_chunk_mma(p, c->prob.head_dim, false, c->L.pre_rows, false, list<ChunkItem>(c, c->L.off_pre), (int)c->L.pre.size(), s);
  if (e == cudaSuccess && !c->L.page.empty()) {
    const ChunkItem* items = list<ChunkItem>(c, c->L.off_page);
    const int n = (int)c->L.page.size();
    e = fp4 ? launch_chunk_mma4(p, c->prob.head_dim, c->L.page_rows, !c->L.pre.empty(), items, n, s)
            : launch_chunk_mma(p, c->prob.head_dim, fp8, c->L.page_rows, !c->L.pre.empty(), items, n, s);
  }
  if (fp4) {  // (the tcgen05 kernel's pages are the widened ones)
    p.k_pool = ws + c->L.off_wk;
    p.v_pool = ws + c->L.off_wv;
    p.page_table = reinterpret_cast<int32_t*>(ws + c->L.off_wtable);
    p.max_pages = c->L.widen_columns;
    p.n_pages = (int32_t)c->L.widen_pages;
  }
  p.beside = !c->L.pre.empty() || !c->L.page.empty();
  if (e == cudaSuccess && !c->L.tc.empty())
    e = launch_chunk_tc(p, c->prob.head_dim, fp8, c->L.tc_split, c->L.prefix_tokens, list<ChunkItem>(c, c->L.off_tc),
                        (int)c->L.tc.size(), s);
  if (e == cudaSuccess && !c->L.merge.empty())
    e = launch_chunk_merge(p, c->prob.head_dim, c->L.pre_splits + c->L.page_splits, list<ChunkMerge>(c, c->L.off_merge), (int)c->L.merge.size(), s);
  return e == cudaSuccess ? PAD_OK : cuda_fail(e, "chunk attention launch");
}

pad_status pad_draft_verify(const pad_chunk_t* c, int32_t vocab, int32_t dtype, const void* p, int64_t p_stride, const void* q,
                            int64_t q_stride, const int32_t* draft, const float* u_accept, const float* u_pick,
                            int32_t* accepted, int32_t* token, pad_stream_t stream) {
  Range r("pad_draft_verify");
  pad_status st = check_launch(c, false);
  if (st != PAD_OK) return st;
  if (vocab < 1 || vocab > (1 << 24)) return api_fail(PAD_ERR_UNSUPPORTED, "vocab=%d outside [1, 2^24]", vocab);
  if (dtype != 0 && dtype != 1) return api_fail(PAD_ERR_INVALID_ARG, "dtype=%d (0 = fp32, 1 = bf16)", dtype);
  st = check_stride(p_stride, vocab, 1, "p");
  if (st == PAD_OK) st = check_stride(q_stride, vocab, 1, "q");
  if (st != PAD_OK) return st;
  if (c->n_events == 0) return PAD_OK;
  if (!accepted || !token || !u_pick || (c->L.n_tokens > 0 && !p) || (c->L.n_drafts > 0 && (!q || !draft || !u_accept)))
    return api_fail(PAD_ERR_INVALID_ARG, "NULL tensor");
  const size_t el = dtype == 1 ? 2 : 4;
  if (!aligned(p, el) || !aligned(q, el) || !aligned(draft, 4) || !aligned(u_accept, 4) || !aligned(u_pick, 4) ||
      !aligned(accepted, 4) || !aligned(token, 4))
    return api_fail(PAD_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
  cudaError_t e = launch_draft_verify(params_of(c), list<ChunkVerify>(c, c->L.off_verify), c->n_events, vocab, dtype == 1, p,
                                      p_stride, q, q_stride, draft, u_accept, u_pick, accepted, token,
                                      reinterpret_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? PAD_OK : cuda_fail(e, "draft verification launch");
}

pad_status pad_chunk_commit(pad_chunk_t* c, pad_cache_state* cache, const int32_t* accepted, int32_t* event_len) {
  if (!c) return api_fail(PAD_ERR_INVALID_ARG, "chunk is NULL");
  if (c->n_events > 0 && !event_len) return api_fail(PAD_ERR_INVALID_ARG, "event_len is NULL");
  if (c->from_cache && !cache) return api_fail(PAD_ERR_INVALID_ARG, "the plan took pages from a cache, cache is NULL");
  if (c->committed) return api_fail(PAD_ERR_INVALID_ARG, "the plan is committed already");
  return guarded([&]() -> pad_status {
    std::vector<int32_t> len(c->n_events), back;
    for (int e = 0; e < c->n_events; ++e) {
      if (accepted && accepted[e] < 0) return api_fail(PAD_ERR_INVALID_ARG, "accepted[%d]=%d", e, accepted[e]);
      len[e] = c->event_len[e] + (accepted ? (int32_t)std::min<int64_t>((int64_t)accepted[e] + 1, c->n_new[e]) : c->n_new[e]);
    }
    const int ps = c->prob.page_size;
    for (size_t i = 0; i < c->new_page.size(); ++i)
      if ((int64_t)c->new_column[i] * ps >= len[c->new_event[i]]) back.push_back(c->new_page[i]);
    if (!back.empty()) {
      pad_status st = pad_cache_state_release(cache, back.data(), (int32_t)back.size());
      if (st != PAD_OK) return st;
    }
    std::copy(len.begin(), len.end(), event_len);
    c->committed = true;
    return PAD_OK;
  });
}

pad_status pad_chunk_status(const pad_chunk_t* c, pad_stream_t stream) {
  pad_status st = check_launch(c, false);
  if (st != PAD_OK) return st;
  PadDevHeader h;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemcpyAsync(&h, c->workspace, sizeof(h), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return cuda_fail(e, "reading device status");
  const int code = (int)(h.word & 0xffull);
  if ((h.word >> 8) == c->gen && code != PAD_OK)
    return api_fail((pad_status)code, "device reported %s (detail %d %d %d)", pad_status_string((pad_status)code), h.info[0],
                    h.info[1], h.info[2]);
  return PAD_OK;
}

}  // extern "C"
