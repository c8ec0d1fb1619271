"""What is measured of a serving step on a 4-bit cache: the paged cache written and read back in 4 bits (pad_chunk_append,
pad_chunk_read), attention of new tokens over the shared prefix and that cache (pad_chunk_attn), rotary positions of the new
queries and keys on their way into the cache (pad_chunk_append_rope), and logits turned into the probabilities that the
verification of drafted tokens reads (pad_chunk_probs), through the library's public entry points and, with ``own`` false, in
plain torch operations.

A case is a dict of plain values.  Lengths follow from the case alone (``shape_seed``), so that work(case) can count them;
tensors and the page placement follow from the seed given to prepare().

Definitions.
- A 4-bit group is 16 consecutive values of one token and kv-head.  Its scale s is the unsigned number of 5 exponent bits (bias
  15) and 3 mantissa bits nearest to max|x| / 6, ties to the even byte, at most 10240 (byte 226); codes are e2m1 of x / s (0, 0.5, 1, 1.5, 2,
  3, 4, 6 and their negatives), nearest, ties to the even code, saturated.
- The query of chunk token t of an event sees its video's prefix and the event's private tokens up to itself.
- Rotary: pair i of the first R dimensions, (i, i + R/2) or (2i, 2i + 1), is turned by position * f_i, f_i = theta^(-2i/R), scaled
  for long contexts: "linear" f_i / factor; "base" theta replaced by theta * factor^(R/(R-2)); "turns" f_i (g + (1 - g) / factor)
  with g = clamp((n_i - low) / (high - low), 0, 1), n_i = original f_i / 2 pi; "index" the same with g = 1 - clamp((i - a) / (b - a), 0, 1),
  a = floor(I(high)), b = ceil(I(low)), both kept in [0, R - 1], I(n) = R ln(original / (2 pi n)) / (2 ln theta).  Cosine and sine are
  multiplied by ``magnitude``.
- Probabilities: c is how often the token occurs in the event's history and in its chunk's tokens up to the row's.  Where
  c > 0 a logit x becomes x / r if x > 0, else x r, and then x - (frequency c + presence); the event's biases are added; a token whose mask
  bit is 0 is left out; p = softmax(x / T) over what is left, one-hot at the first largest x where T is 0, zeros where nothing is left.
"""
import math

import numpy as np
import torch

own = False

# ------------------------------------------------------------------------------- the cases


def _cache(name, events, lens, news, h_kv, d, page, shape_seed):
    return dict(name=name, kind="cache", events=events, len_lo=lens[0], len_hi=lens[1], new_lo=news[0],
                new_hi=news[1], h_q=h_kv, h_kv=h_kv, d=d, page=page, shape_seed=shape_seed)


def _attn(name, events, lens, news, prefix, shape_seed, h_q=28, h_kv=4, d=128, page=16, videos=1):
    return dict(name=name, kind="attn", events=events, len_lo=lens[0], len_hi=lens[1], new_lo=news[0], new_hi=news[1],
                prefix_lo=prefix[0], prefix_hi=prefix[1], videos=videos, h_q=h_q, h_kv=h_kv, d=d, page=page, shape_seed=shape_seed)


def _rope(name, events, lens, news, far, rotary, layout, scaling, shape_seed, h_q=28, h_kv=4, d=128, page=16):
    return dict(name=name, kind="rope", events=events, len_lo=lens[0], len_hi=lens[1], new_lo=news[0], new_hi=news[1],
                far=far, rotary=rotary, layout=layout, scaling=scaling, h_q=h_q, h_kv=h_kv, d=d, page=page, shape_seed=shape_seed)


def _probs(name, events, drafts, vocab, logits16, probs16, history, biases, allowed, shape_seed):
    return dict(name=name, kind="probs", events=events, draft_lo=drafts[0], draft_hi=drafts[1], vocab=vocab, logits16=logits16,
                probs16=probs16, hist_lo=history[0], hist_hi=history[1], biases=biases, allowed=allowed, shape_seed=shape_seed)


def listed():
    return [
        # one step of 32 event branches with five tokens each, and their captions read back: small pieces
        _cache("cache4_drafts_e32", 32, (0, 549), (5, 5), 4, 128, 16, 1),
        # a prompt written into the cache and read back as the contiguous prefix of a video
        _cache("cache4_prompt_32k", 1, (0, 0), (32768, 32768), 4, 128, 16, 2),
        # the smallest step: four branches, one token each, short captions, no prefix; latency is all of it
        _attn("attn4_token_e4", 4, (0, 100), (1, 1), (0, 0), 3),
        # a serving batch that generates single tokens over long paged caches
        _attn("attn4_token_long", 16, (4096, 32768), (1, 1), (0, 0), 4),
        # the long video: 32 branches, one to eight drafted tokens over its prefix and captions up to their usual length
        _attn("attn4_drafts_e32_32k", 32, (0, 549), (1, 8), (32768, 32768), 5),
        # a prompt's chunk over what is cached of it
        _attn("attn4_chunk_2k_of_32k", 1, (30720, 30720), (2048, 2048), (0, 0), 6),
        # drafted tokens over long captions of a head_dim-64 layer on large pages, odd sizes
        _attn("attn4_ragged_d64", 13, (1, 20001), (0, 9), (0, 0), 7, h_q=14, h_kv=2, d=64, page=64),
        # the drafted tokens of 32 branches, whole head, halves
        _rope("rope_drafts_e32", 32, (0, 549), (5, 5), 32768, 128, "half", "none", 8),
        # a prompt far into a context four times as long as the trained one, part of the head, interleaved
        _rope("rope_prompt_16k", 2, (0, 4097), (8000, 8191), 131072, 64, "interleaved", "turns", 9),
        # one sequence, four drafted tokens, a small vocabulary, a grammar
        _probs("probs_e1_32k", 1, (4, 4), 32768, False, False, (100, 549), 0, 0.02, 10),
        # 32 branches with up to eight drafted tokens over a vocabulary of the backbone's order, odd row length, long histories
        _probs("probs_e32_150k", 32, (1, 8), 150001, False, False, (0, 4096), 0, 0.0, 11),
        # a batch of single tokens, logits and probabilities in 16 bits, biases and a loose grammar
        _probs("probs16_e64_128k", 64, (0, 0), 131072, True, True, (0, 549), 100, 0.6, 12),
    ]


_HEADS = {128: ((28, 4), (28, 4), (32, 8), (16, 1), (8, 2)), 64: ((4, 1), (14, 2), (16, 2), (32, 8))}
_SCALINGS = ("none", "linear", "base", "turns", "index")


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "cache", "rope", "probs", "probs"])
    seed = rng.randrange(1 << 30)
    if kind == "probs":
        lo = rng.randint(0, 4)
        hist, events = _log_int(rng, 1, 4096), _log_int(rng, 1, 32)
        c = _probs("", events, (lo, lo + rng.randint(0, 4)), _log_int(rng, 8000, 150001), rng.random() < 0.4, rng.random() < 0.4,
                   (rng.randint(0, hist), hist), rng.choice([0, rng.randint(1, 300)]), rng.choice([0.0, rng.uniform(0.001, 0.9)]), seed)
        del c["name"]
        return c
    d = 64 if rng.random() < 0.3 else 128
    h_q, h_kv = rng.choice(_HEADS[d])
    page = rng.choice([16, 16, 16, 4, 8, 32, 64])
    if kind in ("cache", "rope"):
        events = _log_int(rng, 1, 64)
        most = 32768 if kind == "cache" else 16384
        new, old = _log_int(rng, 1, max(2, most // events)), _log_int(rng, 1, max(2, most // events))
        lens, news = (rng.randint(0, old), old), (rng.randint(1, new), new)
        if kind == "cache":
            c = _cache("", events, lens, news, h_kv, d, page, seed)
        else:
            c = _rope("", events, lens, news, _log_int(rng, 1, 1 << 20), 2 * rng.randint(2, d // 2) if rng.random() < 0.4 else d,
                      rng.choice(["half", "interleaved"]), rng.choice(_SCALINGS), seed, h_q, h_kv, d, page)
        del c["name"]
        return c
    form = rng.choice(["token", "drafts", "drafts", "chunk"])
    if form == "token":
        events = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 400000 // max(13, events))
        c = _attn("", events, (rng.randint(0, hi), hi), (1, 1), (0, 0), seed, h_q, h_kv, d, page)
    elif form == "drafts":
        videos = rng.choice([1, 1, 1, rng.randint(2, 6)])
        events = _log_int(rng, videos, 48)
        hi, n = _log_int(rng, 1, 549), rng.randint(1, 8)
        p = _log_int(rng, 512, 32768 // videos)
        c = _attn("", events, (rng.randint(0, hi), hi), (rng.randint(0, n), n), (p // rng.randint(1, 3), p), seed, h_q, h_kv, d,
                  page, videos)
    else:
        events = rng.randint(1, 6)
        hi, n = _log_int(rng, 1, 24000 // events), _log_int(rng, 16, 2048 // events)
        c = _attn("", events, (rng.randint(0, hi), hi), (rng.randint(1, n), n), (0, 0), seed, h_q, h_kv, d, page)
    del c["name"]
    return c


# ---------------------------------------------------------------- lengths (from the case alone)


def _shape(c):
    """Private lengths and new tokens per event; for attention also prefix lengths and each event's video."""
    r = np.random.default_rng(c["shape_seed"])
    if c["kind"] == "probs":
        news = 1 + r.integers(c["draft_lo"], c["draft_hi"] + 1, size=c["events"]).astype(np.int32)
        return r.integers(c["hist_lo"], c["hist_hi"] + 1, size=c["events"]).astype(np.int32), news
    lens = r.integers(c["len_lo"], c["len_hi"] + 1, size=c["events"]).astype(np.int32)
    news = r.integers(c["new_lo"], c["new_hi"] + 1, size=c["events"]).astype(np.int32)
    if news.sum() == 0:
        news[0] = 1
    if c["kind"] != "attn":
        return lens, news
    prefix = r.integers(c["prefix_lo"], c["prefix_hi"] + 1, size=c["videos"]).astype(np.int32)
    video = np.sort(np.concatenate([np.arange(c["videos"]), r.integers(0, c["videos"], size=c["events"] - c["videos"])]))
    return lens, news, prefix, video.astype(np.int32)


def work(case):
    """Inputs read once, outputs written once."""
    if case["kind"] == "probs":
        hist, news = (int(x.sum()) for x in _shape(case))
        v = case["vocab"]
        row = v * ((2 if case["logits16"] else 4) + (2 if case["probs16"] else 4)) + (4 * -(-v // 32) if case["allowed"] else 0)
        return {"bytes": float(news * (row + 4) + 4 * hist + case["events"] * (16 + 8 * case["biases"])), "flops": 4.0 * news * v}
    hk, d = case["h_kv"], case["d"]
    packed = d // 2 + d // 16                                               # of a token and head in the cache
    lens, news = _shape(case)[:2]
    if case["kind"] == "cache":
        old, new = int(lens.sum()), int(news.sum())
        # new tokens in, their codes out; older codes in; everything out again in bf16
        return {"bytes": float(2 * hk * (new * (2 * d + packed) + old * packed + (old + new) * 2 * d)), "flops": 0.0}
    if case["kind"] == "rope":
        n = int(news.sum())
        return {"bytes": float(n * (4 * d * case["h_q"] + 8 * d * hk + 4)), "flops": 3.0 * n * (case["h_q"] + hk) * case["rotary"]}
    prefix, video = _shape(case)[2:]
    l, n = lens.astype(np.int64), news.astype(np.int64)
    seen = np.unique(video[n > 0])
    kv = 2 * hk * (int((l + n)[n > 0].sum()) * packed + int(prefix[seen].sum()) * 2 * d)
    pairs = int((n * (prefix[video].astype(np.int64) + l) + n * (n + 1) // 2).sum())
    return {"bytes": float(kv + int(n.sum()) * case["h_q"] * (4 * d + 4)), "flops": 4.0 * case["h_q"] * d * pairs}


# ------------------------------------------------------------------------------ the inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _channels(g, h, d):
    """Per-channel scales of the keys: some channels are much larger than the others."""
    return torch.exp(0.5 * _randn(g, 1, h, d))


def _encode(x):
    """4-bit codes (two a byte, the even value's below) and scale bytes of x [..., d], in 32 bits."""
    g = x.unflatten(-1, (-1, 16))
    s = g.abs().amax(-1) / 6.0
    e = (torch.frexp(s)[1] - 1).clamp_min(-14)
    n = torch.round(torch.ldexp(s, 3 - e))                                  # eighths of the scale's power of two
    byte = torch.where(s > 0, (e + 14) * 8 + n.to(torch.int32), 0).clamp_max(226).to(torch.uint8)
    s = _scale(byte).unsqueeze(-1)
    y = torch.where(s > 0, g / s, 0.0)
    m = y.abs()
    code = ((m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0) + 8 * (y < 0)).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), byte


def _scale(byte):
    b = byte.to(torch.int32)
    e, m = b >> 3, (b & 7).float()
    return torch.where(e > 0, torch.ldexp(8.0 + m, e - 18), torch.ldexp(m, torch.full_like(e, -17)))


def _decode(codes, byte):
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    value = torch.cat([value, -value])
    x = torch.stack([value[(codes & 15).long()], value[(codes >> 4).long()]], -1).flatten(-2)
    return (x.unflatten(-1, (-1, 16)) * _scale(byte).unsqueeze(-1)).flatten(-2)


def _tables(lens, seed, page):
    """A page table [E, max_pages] with pages in random places, and the pool's page count."""
    need = (lens + page - 1) // page
    n_pages = int(need.sum()) + 7
    order = np.random.default_rng(int(seed) & 0x7FFFFFFF).permutation(n_pages)
    table = np.full((len(lens), max(1, int(need.max()))), -1, dtype=np.int32)
    at = 0
    for e, n in enumerate(need):
        table[e, :n] = order[at:at + n]
        at += n
    return table, n_pages


def _index(lens):
    """Event and position of every token of packed sequences."""
    ev = np.repeat(np.arange(len(lens)), lens)
    pos = np.arange(int(lens.sum())) - np.repeat(np.concatenate([[0], np.cumsum(lens)[:-1]]), lens)
    return torch.from_numpy(ev).cuda(), torch.from_numpy(pos).cuda()


def _fill(st, x, page):
    """4-bit pools that hold the packed tokens x [T, h_kv, d] of st's whole sequences; other slots hold NaN."""
    n_pages, (t, h, d) = st["n_pages"], x.shape
    ev, pos = st["all_index"]
    pg, slot = st["table"][ev, pos // page].long(), pos % page
    pool = torch.full((n_pages, h, page, d // 2), 0x77, dtype=torch.uint8, device="cuda")
    scale = torch.full((n_pages, h, page, d // 16), 0xFF, dtype=torch.uint8, device="cuda")
    pool[pg, :, slot], scale[pg, :, slot] = _encode(x.float())
    return pool, scale


def _handle(case, st, lens, news, prefix=None, video=None):
    """The plan that a user's program keeps for the layers of one step."""
    from paper_2607_02963_gb300 import binding as B
    prob = B.make_problem(case.get("h_q", 1), case.get("h_kv", 1), case.get("d", 64), case.get("page", 16), out_dtype=1)
    fmt = B.KV_BF16 if case["kind"] == "rope" else B.KV_FP4
    need = B.pad_chunk_workspace_size(prob, prefix, video, lens, news, kv_format=fmt)
    st["workspace"] = torch.zeros(need, dtype=torch.uint8, device="cuda")
    st["plan"] = B.pad_chunk_plan(prob, None, prefix, video, lens, news, page_table=st.get("table"),
                                  n_pages=st.get("n_pages", 0), kv_format=fmt, workspace=st["workspace"])


def _spec(case):
    """What a program says of its model's rotary positions."""
    return dict(theta=1.0e6, factor=4.0, original=32768, low=1.0, high=4.0 if case["scaling"] == "turns" else 32.0,
                magnitude=1.0 + 0.1 * math.log(4.0) if case["scaling"] == "index" else 1.0)


def _prepare_probs(case, seed, g, st):
    hist, news = _shape(case)
    e, v, rows = case["events"], case["vocab"], int(news.sum())
    st["row_event"], st["row_pos"] = _index(news)
    st["news"] = torch.from_numpy(news).cuda().long()
    st["logits"] = (3.0 * _randn(g, rows, v)).to(torch.bfloat16 if case["logits16"] else torch.float32)
    st["p"] = torch.empty(rows, v, dtype=torch.bfloat16 if case["probs16"] else torch.float32, device="cuda")
    # temperatures from cold to warm, and some events that are greedy
    u = torch.rand(e, 4, generator=g, device="cuda")
    t = torch.where(u[:, 0] < 0.125, 0.0, 0.5 + 0.8 * u[:, 0])
    st["params"] = torch.stack([t, 1.0 + 0.3 * u[:, 1], 0.5 * u[:, 2], 0.5 * u[:, 3]], 1).contiguous()
    # histories repeat themselves, as text does: low tokens far more often than high ones
    most = max(1, int(hist.max()))
    r = torch.rand(e, most, generator=g, device="cuda")
    st["history"] = torch.clamp((r ** 4 * v).int(), max=v - 1)
    st["history_len"] = torch.from_numpy(hist).cuda()
    st["tokens"] = torch.clamp((torch.rand(rows, generator=g, device="cuda") ** 4 * v).int(), max=v - 1)
    st["bias_token"] = st["bias_value"] = st["bias_len"] = st["mask"] = None
    if case["biases"]:
        n = case["biases"]
        order = torch.rand(e, v, generator=g, device="cuda").argsort(1)[:, :n]
        st["bias_token"] = order.sort(1)[0].int().contiguous()
        value = 2.0 * _randn(g, e, n)
        st["bias_value"] = torch.where(torch.rand(e, n, generator=g, device="cuda") < 0.1, -100.0, value)
        st["bias_len"] = torch.randint(0, n + 1, (e,), generator=g, device="cuda", dtype=torch.int32)
    if case["allowed"]:
        bits = torch.rand(rows, -(-v // 32) * 32, generator=g, device="cuda") < case["allowed"]
        if rows > 2:
            bits[rows // 2] = False                                        # a grammar that is at its end
        weight = (torch.ones(32, dtype=torch.int64, device="cuda") << torch.arange(32, device="cuda"))
        words = (bits.unflatten(1, (-1, 32)).long() * weight).sum(-1)
        st["mask"] = torch.where(words >= 1 << 31, words - (1 << 32), words).int().contiguous()
    if own:
        _handle(case, st, np.zeros(e, np.int32), news)
    return st


def prepare(case, seed):
    g = _gen(seed)
    st = {"case": case}
    if case["kind"] == "probs":
        return _prepare_probs(case, seed, g, st)
    hq, hk, d, page = case["h_q"], case["h_kv"], case["d"], case["page"]
    lens, news = _shape(case)[:2]
    tot = lens + news
    table, st["n_pages"] = _tables(tot, seed, page)
    st["table"] = torch.from_numpy(table).cuda()
    st["tot"] = torch.from_numpy(tot).cuda().long()
    st["lens"], st["news"] = torch.from_numpy(lens).cuda().long(), torch.from_numpy(news).cuda().long()
    st["all_index"] = _index(tot)
    st["new_index"] = _index(news)
    t, n = int(tot.sum()), int(news.sum())
    kc = _channels(g, hk, d)
    if case["kind"] == "rope":
        # a pool that holds other tokens already; each sequence starts at a position of its own
        st["k_pool"], st["v_pool"] = (_randn(g, st["n_pages"], hk, page, d).bfloat16() for _ in range(2))
        st["q"], st["q_out"] = _randn(g, n, hq, d).bfloat16(), torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda")
        st["k_new"], st["v_new"] = (_randn(g, n, hk, d) * kc).bfloat16(), _randn(g, n, hk, d).bfloat16()
        ev, pos = st["new_index"]
        start = torch.randint(0, case["far"], (case["events"],), generator=g, device="cuda")
        st["position"] = (start[ev] + st["lens"][ev] + pos).to(torch.int32)
        if own:
            from paper_2607_02963_gb300 import binding as B
            s = _spec(case)
            st["rope"] = B.Rope(d, case["rotary"], s["theta"], layout=case["layout"], scaling=case["scaling"], factor=s["factor"],
                                original_len=s["original"], low=s["low"], high=s["high"], magnitude=s["magnitude"])
            _handle(case, st, lens, news)
        return st
    k_all, v_all = (_randn(g, t, hk, d) * kc).bfloat16(), _randn(g, t, hk, d).bfloat16()
    st["k_pool"], st["k_scale"] = _fill(st, k_all, page)
    st["v_pool"], st["v_scale"] = _fill(st, v_all, page)
    if case["kind"] == "cache":
        st["k_new"], st["v_new"] = (_randn(g, n, hk, d) * kc).bfloat16(), _randn(g, n, hk, d).bfloat16()
        st["k_out"], st["v_out"] = torch.empty_like(k_all), torch.empty_like(v_all)
        if own:
            _handle(case, st, lens, news)
        return st
    prefix, video = _shape(case)[2:]
    p = int(prefix.sum())
    st["k_prefix"], st["v_prefix"] = (_randn(g, p, hk, d) * kc).bfloat16(), _randn(g, p, hk, d).bfloat16()
    st["prefix"], st["video"] = torch.from_numpy(prefix).cuda().long(), torch.from_numpy(video).cuda().long()
    st["q"] = _randn(g, n, hq, d).bfloat16()
    st["out"] = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty(n, hq, dtype=torch.float32, device="cuda")
    if own:
        _handle(case, st, lens, news, prefix, video)
    return st


# ------------------------------------------------------------------------- the plain forms


def _plain_cache(st):
    page = st["case"]["page"]
    ev, pos = st["new_index"]
    at = pos + st["lens"][ev]
    pg, slot = st["table"][ev, at // page].long(), at % page
    st["k_pool"][pg, :, slot], st["k_scale"][pg, :, slot] = _encode(st["k_new"].float())
    st["v_pool"][pg, :, slot], st["v_scale"][pg, :, slot] = _encode(st["v_new"].float())
    ev, pos = st["all_index"]
    pg, slot = st["table"][ev, pos // page].long(), pos % page
    return {"k": _decode(st["k_pool"][pg, :, slot], st["k_scale"][pg, :, slot]).bfloat16(),
            "v": _decode(st["v_pool"][pg, :, slot], st["v_scale"][pg, :, slot]).bfloat16()}


def _padded(st, pool, scale, prefix):
    """Every event's keys or values [E, P + L, h_kv, d] in 32 bits, zero where it has none."""
    page = st["case"]["page"]
    p_most, l_most = int(st["prefix_most"]), int(st["tot_most"])
    pos = torch.arange(l_most, device="cuda")
    pg = st["table"][:, pos // page].long().clamp_min(0)
    x = _decode(st[pool][pg, :, pos % page], st[scale][pg, :, pos % page])
    x = torch.where((pos < st["tot"].unsqueeze(1))[..., None, None], x, 0.0)
    if p_most == 0:
        return x
    pp = torch.arange(p_most, device="cuda")
    first = (torch.cumsum(st["prefix"], 0) - st["prefix"])[st["video"]]
    there = pp < st["prefix"][st["video"]].unsqueeze(1)
    y = st[prefix][torch.where(there, first.unsqueeze(1) + pp, 0)].float()
    return torch.cat([torch.where(there[..., None, None], y, 0.0), x], 1)


def _plain_attn(st):
    c = st["case"]
    hq, hk, d = c["h_q"], c["h_kv"], c["d"]
    grp = hq // hk
    lens, news, prefix, video = _shape(c)
    st["prefix_most"], st["tot_most"] = int(prefix.max()), int((lens + news).max())
    n_most, events, p_most = int(news.max()), len(lens), st["prefix_most"]
    k, v = _padded(st, "k_pool", "k_scale", "k_prefix"), _padded(st, "v_pool", "v_scale", "v_prefix")
    ev, pos = st["new_index"]
    q = torch.zeros(events, n_most, hq, d, device="cuda")
    q[ev, pos] = st["q"].float()
    q = q.view(events, n_most, hk, grp, d).permute(0, 2, 1, 3, 4).reshape(events, hk, n_most * grp, d)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(d)
    s = s.view(events, hk, n_most, grp, -1)
    at = torch.arange(s.shape[-1], device="cuda")
    in_prefix = at < st["prefix"][st["video"]].unsqueeze(1)                                   # [E, K]
    mine = (st["lens"].unsqueeze(1) + torch.arange(n_most, device="cuda")).unsqueeze(2)       # [E, N, 1]
    private = (at >= p_most) & (at - p_most <= mine)                                          # [E, N, K]
    seen = private | (in_prefix & (at < p_most)).unsqueeze(1)
    s = s.masked_fill(~seen[:, None, :, None, :], float("-inf"))
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m)
    l = e.sum(-1, keepdim=True)
    o = torch.matmul((e / l).view(events, hk, n_most * grp, -1), v.permute(0, 2, 1, 3))
    o = o.view(events, hk, n_most, grp, d).permute(0, 2, 1, 3, 4).reshape(events, n_most, hq, d)
    lse = (m + torch.log(l)).squeeze(-1).permute(0, 2, 1, 3).reshape(events, n_most, hq)
    return {"out": o[ev, pos].bfloat16(), "lse": lse[ev, pos]}


def _frequencies(case, device):
    """f_i of the rotary pairs, in 64 bits."""
    s, rd = _spec(case), case["rotary"]
    i = torch.arange(rd // 2, device=device, dtype=torch.float64)
    theta = s["theta"] * (s["factor"] ** (rd / (rd - 2)) if case["scaling"] == "base" else 1.0)
    f = theta ** (-2.0 * i / rd)
    if case["scaling"] == "linear":
        return f / s["factor"]
    if case["scaling"] == "turns":
        ramp = ((s["original"] * f / (2 * math.pi) - s["low"]) / (s["high"] - s["low"])).clamp(0, 1)
        return f * (ramp + (1 - ramp) / s["factor"])
    if case["scaling"] == "index":
        a, b = (rd * math.log(s["original"] / (2 * math.pi * n)) / (2 * math.log(s["theta"])) for n in (s["high"], s["low"]))
        a, b = max(math.floor(a), 0), min(math.ceil(b), rd - 1)
        ramp = 1 - ((i - a) / max(b - a, 0.001)).clamp(0, 1)
        return f * (ramp + (1 - ramp) / s["factor"])
    return f


def _pairs(x, rd, layout):
    """The two members of every pair."""
    return (x[..., :rd // 2], x[..., rd // 2:rd]) if layout == "half" else (x[..., 0:rd:2], x[..., 1:rd:2])


def _joined(a, b, rest, layout):
    x = torch.cat([a, b], -1) if layout == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([x, rest], -1)


def _plain_rope(st):
    c = st["case"]
    rd, page = c["rotary"], c["page"]
    angle = st["position"].double().unsqueeze(1) * _frequencies(c, "cuda")     # (far positions: 32 bits lose the angle)
    mag = _spec(c)["magnitude"]
    cos, sin = (mag * torch.cos(angle)).float().unsqueeze(1), (mag * torch.sin(angle)).float().unsqueeze(1)

    def turned(x):
        x = x.float()
        a, b = _pairs(x, rd, c["layout"])
        return _joined(a * cos - b * sin, b * cos + a * sin, x[..., rd:], c["layout"]).bfloat16()

    ev, pos = st["new_index"]
    at = pos + st["lens"][ev]
    pg, slot = st["table"][ev, at // page].long(), at % page
    st["k_pool"][pg, :, slot] = turned(st["k_new"])
    st["v_pool"][pg, :, slot] = st["v_new"]
    return {"q": turned(st["q"]), "k_pool": st["k_pool"], "v_pool": st["v_pool"]}


def _counts(st):
    """How often each token is in its row's history and chunk [rows, vocab]."""
    c = st["case"]
    e, v, most = c["events"], c["vocab"], st["history"].shape[1]
    there = torch.arange(most, device="cuda") < st["history_len"].unsqueeze(1)
    count = torch.zeros(e, v, dtype=torch.int32, device="cuda")
    count.scatter_add_(1, st["history"].long(), there.int())
    count = count[st["row_event"]]
    rows = torch.arange(count.shape[0], device="cuda")
    longest = int(_shape(c)[1].max())
    back = torch.arange(longest, device="cuda")                                # the row's token, the one before it, ..
    had = back <= st["row_pos"].unsqueeze(1)
    tok = st["tokens"].long()[torch.where(had, rows.unsqueeze(1) - back, 0)]
    return count.scatter_add_(1, tok, had.int())


def _plain_probs(st):
    c = st["case"]
    ev, v = st["row_event"], c["vocab"]
    x = st["logits"].float()
    t, r, freq, pres = (z.unsqueeze(1) for z in st["params"][ev].unbind(1))
    n = _counts(st)
    x = torch.where(n > 0, torch.where(x > 0, x / r, x * r) - (freq * n.float() + pres), x)
    if st["bias_token"] is not None:
        there = torch.arange(c["biases"], device="cuda") < st["bias_len"].unsqueeze(1)
        bias = torch.zeros(c["events"], v, device="cuda").scatter_add_(1, st["bias_token"].long(), torch.where(there, st["bias_value"], 0.0))
        x = x + bias[ev]
    if st["mask"] is not None:
        bits = (st["mask"].unsqueeze(-1) >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(bits.flatten(1)[:, :v] > 0, x, float("-inf"))
    m = x.amax(1, keepdim=True)
    empty = m == float("-inf")
    e = torch.exp((x - torch.where(empty, 0.0, m)) / torch.where(t > 0, t, 1.0))
    p = e / torch.where(empty, 1.0, e.sum(1, keepdim=True))
    at = torch.arange(v, device="cuda")
    first = torch.where(x == m, at, v).amin(1, keepdim=True)
    p = torch.where(t > 0, p, (at == first).float())
    return {"p": torch.where(empty, 0.0, p).to(st["p"].dtype)}


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"cache": _plain_cache, "attn": _plain_attn, "rope": _plain_rope, "probs": _plain_probs}[kind](state)
    from paper_2607_02963_gb300 import binding as B
    st = state
    if kind == "cache":
        B.pad_chunk_append(st["plan"], st["k_new"], st["v_new"], st["k_pool"], st["v_pool"], st["k_scale"], st["v_scale"])
        B.pad_chunk_read(st["plan"], st["k_pool"], st["v_pool"], st["k_out"], st["v_out"], st["k_scale"], st["v_scale"])
        return {"k": st["k_out"], "v": st["v_out"]}
    if kind == "attn":
        B.pad_chunk_attn(st["plan"], st["q"], st["k_prefix"], st["v_prefix"], st["k_pool"], st["v_pool"], st["out"],
                         st["lse"], st["k_scale"], st["v_scale"])
        return {"out": st["out"], "lse": st["lse"]}
    if kind == "rope":
        B.pad_chunk_append_rope(st["plan"], st["rope"], st["position"], st["q"], st["q_out"], st["k_new"], st["v_new"],
                                st["k_pool"], st["v_pool"])
        return {"q": st["q_out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"]}
    B.pad_chunk_probs(st["plan"], st["logits"], st["p"], params=st["params"], history=st["history"], history_len=st["history_len"],
                      tokens=st["tokens"], bias_token=st["bias_token"], bias_value=st["bias_value"], bias_len=st["bias_len"],
                      mask=st["mask"])
    return {"p": st["p"]}


# ------------------------------------------------------------------- the definition in 64 bits


def _grid4(x):
    """x (float64, [..., d]) on its 4-bit grid: groups of 16, the spacing of a value is half of its power of two, half a
    scale at least; that of a scale an eighth of its own, 2^-17 at least."""
    g = x.unflatten(-1, (-1, 16))
    s = g.abs().amax(-1, keepdim=True) / 6
    step = torch.exp2(torch.floor(torch.log2(s.clamp_min(2.0 ** -14))) - 3)
    s = (torch.round(s / step) * step).clamp_max(10240)
    y = g / torch.where(s > 0, s, 1)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(1.0))) - 1)
    return torch.where(s > 0, (torch.round(y / step) * step).clamp(-6, 6) * s, 0).flatten(-2)


def _exact_probs(case, st):
    hist, news = _shape(case)
    v, out, row = case["vocab"], [], 0
    params, tokens, history = st["params"].double().cpu(), st["tokens"].cpu().long(), st["history"].cpu().long()
    for e in range(case["events"]):
        t, r, freq, pres = (float(z) for z in params[e])
        count = torch.bincount(history[e, :int(hist[e])], minlength=v)
        for _ in range(int(news[e])):
            count[tokens[row]] += 1
            n = count.cuda().double()
            x = st["logits"][row].double()
            x = torch.where(n > 0, torch.where(x > 0, x / r, x * r) - freq * n - pres, x)
            if case["biases"]:
                k = int(st["bias_len"][e])
                x.index_add_(0, st["bias_token"][e, :k].long(), st["bias_value"][e, :k].double())
            if case["allowed"]:
                word = st["mask"][row].long() & 0xFFFFFFFF
                i = torch.arange(v, device="cuda")
                x[(word[i // 32] >> (i % 32)) & 1 == 0] = -math.inf
            if float(x.max()) == -math.inf:
                p = torch.zeros_like(x)
            elif t == 0:
                p = torch.zeros_like(x)
                p[torch.nonzero(x == x.max())[0]] = 1
            else:
                p = torch.softmax(x / t, 0)
            out.append(p)
            row += 1
    return {"p": torch.stack(out)}


def _exact_rope(case, st):
    s, rd, lay = _spec(case), case["rotary"], case["layout"]
    f = []
    for i in range(rd // 2):
        theta = s["theta"] * s["factor"] ** (rd / (rd - 2)) if case["scaling"] == "base" else s["theta"]
        a = math.exp(-2 * i / rd * math.log(theta))
        if case["scaling"] == "linear":
            share = 0.0
        elif case["scaling"] == "turns":
            share = (s["original"] * a / (2 * math.pi) - s["low"]) / (s["high"] - s["low"])
        elif case["scaling"] == "index":
            lo, hi = (rd / 2 * (math.log(s["original"]) - math.log(2 * math.pi * n)) / math.log(s["theta"]) for n in (s["high"], s["low"]))
            lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rd - 1)
            share = 1 - (i - lo) / max(hi - lo, 0.001)
        else:
            share = 1.0
        share = min(max(share, 0.0), 1.0)
        f.append(a * share + a / s["factor"] * (1 - share))
    angle = st["position"].double().unsqueeze(1) * torch.tensor(f, dtype=torch.float64, device="cuda")
    c, n = s["magnitude"] * torch.cos(angle).unsqueeze(1), s["magnitude"] * torch.sin(angle).unsqueeze(1)

    def turned(x):
        y = x.double().clone()
        i = torch.arange(rd // 2, device="cuda")
        one, two = (i, i + rd // 2) if lay == "half" else (2 * i, 2 * i + 1)
        a, b = y[..., one].clone(), y[..., two].clone()
        y[..., one], y[..., two] = c * a - n * b, n * a + c * b
        return y

    k_pool, v_pool, page = st["k_pool"].double(), st["v_pool"].double(), case["page"]
    k, v = turned(st["k_new"]), st["v_new"].double()
    lens, news = _shape(case)
    ends = np.cumsum(news)
    table = st["table"].cpu().numpy()
    at = [(table[e, p // page], p % page) for e in range(len(news)) for p in range(lens[e], lens[e] + news[e])]
    pg, slot = (torch.tensor([int(a[j]) for a in at], device="cuda") for j in range(2))
    assert len(at) == ends[-1]
    k_pool[pg, :, slot], v_pool[pg, :, slot] = k, v
    return {"q": turned(st["q"]), "k_pool": k_pool, "v_pool": v_pool}


def exact(case, seed):
    global own
    before, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = before
    if case["kind"] == "probs":
        return _exact_probs(case, st)
    if case["kind"] == "rope":
        return _exact_rope(case, st)
    page, (ev, pos) = case["page"], st["all_index"]
    lens, news = _shape(case)[:2]
    pg, slot = st["table"][ev, pos // page].long(), pos % page

    def stored(pool, scale):
        b, s = st[pool][pg, :, slot].to(torch.int64), st[scale][pg, :, slot].to(torch.int64)
        c = torch.empty(*b.shape[:-1], 2 * b.shape[-1], dtype=torch.int64, device="cuda")
        c[..., 0::2], c[..., 1::2] = b % 16, b // 16
        size, exp = (c & 1).double(), (c >> 1) & 3
        mag = torch.where(exp > 0, (2 + size) * torch.exp2((exp - 2).double()), size / 2)
        top, low = s // 8, (s % 8).double()
        unit = torch.where(top > 0, (1 + low / 8) * torch.exp2(top.double() - 15), low * 2.0 ** -17)
        return torch.where(c > 7, -mag, mag) * unit.repeat_interleave(16, -1)

    k, v = stored("k_pool", "k_scale"), stored("v_pool", "v_scale")
    ends = np.cumsum(lens + news)
    if case["kind"] == "cache":
        at = torch.from_numpy(np.concatenate([np.arange(t - m, t) for t, m in zip(ends, news)])).cuda()
        k[at], v[at] = _grid4(st["k_new"].double()), _grid4(st["v_new"].double())
        return {"k": k, "v": v}
    prefix, video = _shape(case)[2:]
    grp, hk = case["h_q"] // case["h_kv"], case["h_kv"]
    q, p_end, n_end = st["q"].double(), np.cumsum(prefix), np.cumsum(news)
    out = torch.zeros(int(news.sum()), case["h_q"], case["d"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(int(news.sum()), case["h_q"], dtype=torch.float64, device="cuda")
    for e in range(len(lens)):
        if news[e] == 0:
            continue
        a, b, w = ends[e] - lens[e] - news[e], ends[e], video[e]
        pl, nn = int(prefix[w]), int(news[e])
        rows = slice(n_end[e] - nn, n_end[e])
        hidden = torch.ones(nn, pl + b - a, dtype=torch.bool, device="cuda").triu(pl + int(lens[e]) + 1)
        for h in range(hk):
            kk = torch.cat([st["k_prefix"][p_end[w] - pl:p_end[w], h].double(), k[a:b, h]])
            vv = torch.cat([st["v_prefix"][p_end[w] - pl:p_end[w], h].double(), v[a:b, h]])
            for j in range(h * grp, (h + 1) * grp):
                s = (q[rows, j] @ kk.T / math.sqrt(case["d"])).masked_fill(hidden, -math.inf)
                lse[rows, j] = torch.logsumexp(s, -1)
                out[rows, j] = torch.softmax(s, -1) @ vv
    return {"out": out, "lse": lse}
