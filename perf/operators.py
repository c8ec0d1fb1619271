"""What is measured of the multi-token steps of event branches: the private paged cache written and read
back in 8 bits (pad_chunk_append, pad_chunk_read), attention of a chunk of new tokens over the shared prefix
and the paged cache (pad_chunk_attn), and verification of drafted tokens (pad_draft_verify), through the
library's public entry points and, with ``own`` false, in plain torch operations.

A case is a dict of plain values.  Lengths follow from the case alone (``shape_seed``), so that work(case)
can count them; tensors and the page placement follow from the seed given to prepare().

Definitions.  An 8-bit group is the head_dim values of one token and kv-head: codes are e4m3 of x / 2^k,
rounded to nearest even, k the smallest integer with max|x| <= 448 * 2^k, kept in [-120, 7]; the scale is
held as the byte k + 127 (0: a group of zeros).  The query of chunk token t of an event sees its video's
prefix and the event's private tokens up to itself.  Drafted token i, x_i, is accepted while
u_i q_i(x_i) < p_i(x_i); the next token is drawn at the first rejected position a from max(p_a - q_a, 0), or
after a whole accepted draft from p itself: weights floor(2^38 min(r, 1)), the first token whose running sum
exceeds floor(m S / 2^24), S the sum of all weights and m = floor(2^24 u).
"""
import math

import numpy as np
import torch

own = False

# ------------------------------------------------------------------------------- the cases


def _cache(name, events, lens, news, h_kv, d, page, shape_seed):
    return dict(name=name, kind="cache", events=events, len_lo=lens[0], len_hi=lens[1], new_lo=news[0],
                new_hi=news[1], h_q=h_kv, h_kv=h_kv, d=d, page=page, shape_seed=shape_seed)


def _attn(name, events, lens, news, prefix, fp8, shape_seed, h_q=28, h_kv=4, d=128, page=16, videos=1):
    return dict(name=name, kind="attn", events=events, len_lo=lens[0], len_hi=lens[1], new_lo=news[0],
                new_hi=news[1], prefix_lo=prefix[0], prefix_hi=prefix[1], videos=videos, fp8=fp8, h_q=h_q,
                h_kv=h_kv, d=d, page=page, shape_seed=shape_seed)


def _verify(name, events, drafts, vocab, bf16, shape_seed):
    return dict(name=name, kind="verify", events=events, draft_lo=drafts[0], draft_hi=drafts[1], vocab=vocab,
                bf16=bf16, shape_seed=shape_seed)


def listed():
    return [
        # one step of 32 event branches with five tokens each, and their captions read back: small pieces
        _cache("cache_drafts_e32", 32, (0, 549), (5, 5), 4, 128, 16, 1),
        # a prompt written into the cache and read back as the contiguous prefix of a video
        _cache("cache_prompt_32k", 1, (0, 0), (32768, 32768), 4, 128, 16, 2),
        # a handful of ragged sequences of a head_dim-64 layer on small pages
        _cache("cache_ragged_d64", 5, (1, 4097), (1, 1031), 2, 64, 8, 3),
        # the smallest step: four branches, one token each, short captions, no prefix; latency is all of it
        _attn("attn_token_e4", 4, (0, 100), (1, 1), (0, 0), False, 4),
        # drafted tokens of 13 branches (the paper's average) over an 8k prefix
        _attn("attn_drafts_e13_8k", 13, (0, 128), (5, 5), (8219, 8219), False, 5),
        # the long video: 32 branches, one to eight drafted tokens, captions up to their usual length in 8 bits
        _attn("attn_drafts8_e32_32k", 32, (0, 549), (1, 8), (32768, 32768), True, 6),
        # a serving batch that generates single tokens over long paged caches, bf16 and 8 bits
        _attn("attn_token_long", 16, (4096, 32768), (1, 1), (0, 0), False, 7),
        _attn("attn_token8_long", 16, (4096, 32768), (1, 1), (0, 0), True, 7),
        # a prompt's chunk over what is cached of it
        _attn("attn_chunk_2k_of_32k", 1, (30720, 30720), (2048, 2048), (0, 0), False, 8),
        # chunks of several prompts of a head_dim-64 layer, 8 bits, odd sizes
        _attn("attn_chunk8_ragged_d64", 6, (1, 7001), (130, 1501), (0, 0), True, 9, h_q=14, h_kv=2, d=64, page=64),
        # one sequence, four drafted tokens, a small vocabulary
        _verify("verify_e1_32k", 1, (4, 4), 32768, False, 10),
        # 32 branches with up to eight drafted tokens over a vocabulary of the backbone's order, odd row length
        _verify("verify_e32_150k", 32, (1, 8), 150001, False, 11),
    ]


_HEADS = {128: ((28, 4), (28, 4), (32, 8), (16, 1), (8, 2)), 64: ((4, 1), (14, 2), (16, 2), (32, 8))}


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "cache", "verify"])
    seed = rng.randrange(1 << 30)
    if kind == "verify":
        lo = rng.randint(0, 4)
        c = _verify("", _log_int(rng, 1, 64), (lo, lo + rng.randint(0, 4)), _log_int(rng, 8000, 150001),
                    rng.random() < 0.4, seed)
        del c["name"]
        return c
    d = 64 if rng.random() < 0.3 else 128
    h_q, h_kv = rng.choice(_HEADS[d])
    page = rng.choice([16, 16, 16, 4, 8, 32, 64])
    if kind == "cache":
        events = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, max(2, 32768 // events))
        old = _log_int(rng, 1, max(2, 32768 // events))
        c = _cache("", events, (rng.randint(0, old), old), (rng.randint(1, new), new), h_kv, d, page, seed)
        del c["name"]
        return c
    form = rng.choice(["token", "drafts", "drafts", "chunk"])
    fp8 = rng.random() < 0.5
    if form == "token":
        events = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, 400000 // max(13, events))
        c = _attn("", events, (rng.randint(0, hi), hi), (1, 1), (0, 0), fp8, seed, h_q, h_kv, d, page)
    elif form == "drafts":
        videos = rng.choice([1, 1, 1, rng.randint(2, 6)])
        events = _log_int(rng, videos, 48)
        hi, n = _log_int(rng, 1, 549), rng.randint(1, 8)
        p = _log_int(rng, 512, 32768 // videos)
        c = _attn("", events, (rng.randint(0, hi), hi), (rng.randint(0, n), n), (p // rng.randint(1, 3), p), fp8,
                  seed, h_q, h_kv, d, page, videos)
    else:
        events = rng.randint(1, 6)
        hi, n = _log_int(rng, 1, 24000 // events), _log_int(rng, 16, 2048 // events)
        c = _attn("", events, (rng.randint(0, hi), hi), (rng.randint(1, n), n), (0, 0), fp8, seed, h_q, h_kv, d, page)
    del c["name"]
    return c


# ---------------------------------------------------------------- lengths (from the case alone)


def _shape(c):
    """Private lengths and new tokens per event; for attention also prefix lengths and each event's video."""
    r = np.random.default_rng(c["shape_seed"])
    lens = r.integers(c["len_lo"], c["len_hi"] + 1, size=c["events"]).astype(np.int32)
    news = r.integers(c["new_lo"], c["new_hi"] + 1, size=c["events"]).astype(np.int32)
    if news.sum() == 0:
        news[0] = 1
    if c["kind"] == "cache":
        return lens, news
    prefix = r.integers(c["prefix_lo"], c["prefix_hi"] + 1, size=c["videos"]).astype(np.int32)
    video = np.sort(np.concatenate([np.arange(c["videos"]), r.integers(0, c["videos"], size=c["events"] - c["videos"])]))
    return lens, news, prefix, video.astype(np.int32)


def _drafts(c):
    r = np.random.default_rng(c["shape_seed"])
    return r.integers(c["draft_lo"], c["draft_hi"] + 1, size=c["events"]).astype(np.int32)


def work(case):
    """Inputs read once, outputs written once."""
    if case["kind"] == "verify":
        # of the probabilities one row of the target's and one of the draft's per event
        n = _drafts(case)
        el = 2 if case["bf16"] else 4
        return {"bytes": float(2 * case["events"] * case["vocab"] * el + 12 * n.sum() + 12 * case["events"]), "flops": 0.0}
    hk, d = case["h_kv"], case["d"]
    if case["kind"] == "cache":
        lens, news = (int(x.sum()) for x in _shape(case))
        # new tokens in, their codes out; older codes in; everything out again in bf16
        return {"bytes": float(2 * hk * (news * (2 * d + d + 1) + lens * (d + 1) + (lens + news) * 2 * d)), "flops": 0.0}
    lens, news, prefix, video = _shape(case)
    l, n = lens.astype(np.int64), news.astype(np.int64)
    per = (d + 1) if case["fp8"] else 2 * d
    seen = np.unique(video[n > 0])
    kv = 2 * hk * (int((l + n)[n > 0].sum()) * per + int(prefix[seen].sum()) * 2 * d)
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
    """8-bit codes and scale bytes of groups (the last axis), in 32 bits."""
    amax = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)
    k = torch.where(m <= 0.875, e - 9, e - 8).clamp(-120, 7)
    codes = torch.ldexp(x, -k).clamp(-448, 448).to(torch.float8_e4m3fn)
    byte = torch.where(amax > 0, k + 127, torch.zeros_like(k)).to(torch.uint8)
    return codes.view(torch.uint8), byte.squeeze(-1)


def _decode(codes, byte):
    k = byte.to(torch.int32).unsqueeze(-1)
    x = torch.ldexp(codes.view(torch.float8_e4m3fn).float(), k - 127)
    return torch.where(k > 0, x, torch.zeros_like(x))


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


def _fill(st, x, table, page):
    """Pools that hold the packed tokens x [T, h_kv, d] of st's whole sequences; other slots hold NaN."""
    n_pages, (t, h, d) = st["n_pages"], x.shape
    ev, pos = st["all_index"]
    pg, slot = table[ev, pos // page].long(), pos % page
    if st["fp8"]:
        pool = torch.full((n_pages, h, page, d), 0x7F, dtype=torch.uint8, device="cuda")
        scale = torch.full((n_pages, h, page), 0xFF, dtype=torch.uint8, device="cuda")
        pool[pg, :, slot], scale[pg, :, slot] = _encode(x.float())
        return pool, scale
    pool = torch.full((n_pages, h, page, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    pool[pg, :, slot] = x
    return pool, None


def _handle(case, st, lens, news, prefix=None, video=None, bf16_out=False):
    """The plan that a user's program keeps for the layers of one step."""
    from paper_2607_02963_gb300 import binding as B
    prob = B.make_problem(case.get("h_q", 1), case.get("h_kv", 1), case.get("d", 64), case.get("page", 16),
                          out_dtype=1 if bf16_out else 0)
    fmt = B.KV_FP8 if st.get("fp8") else B.KV_BF16
    need = B.pad_chunk_workspace_size(prob, prefix, video, lens, news, kv_format=fmt)
    st["workspace"] = torch.zeros(need, dtype=torch.uint8, device="cuda")
    st["plan"] = B.pad_chunk_plan(prob, None, prefix, video, lens, news, page_table=st.get("table"),
                                  n_pages=st.get("n_pages", 0), kv_format=fmt, workspace=st["workspace"])


def prepare(case, seed):
    g = _gen(seed)
    st = {"case": case}
    if case["kind"] == "verify":
        n, e, v = _drafts(case), case["events"], case["vocab"]
        rows, dt = int(n.sum()) + e, torch.bfloat16 if case["bf16"] else torch.float32
        ev, pos = _index(n + 1)
        st["n"], st["first"] = torch.from_numpy(n).cuda().long(), torch.from_numpy(np.cumsum(n + 1) - n - 1).cuda()
        logits = 3.0 * _randn(g, rows, v)
        st["p"] = torch.softmax(logits, -1).to(dt)
        has = pos < st["n"][ev]                                 # rows that a drafted token follows
        # the draft's distribution: the target's logits with an error of its own
        near = torch.softmax(logits[has] + 0.7 * _randn(g, int(n.sum()), v), -1)
        del logits
        st["q"] = near.to(dt)
        drawn = torch.argmax(near / -torch.log(torch.rand(near.shape, generator=g, device="cuda").clamp_min(1e-12)), -1) \
            if near.shape[0] else torch.zeros(0, dtype=torch.long, device="cuda")
        st["draft"] = drawn.to(torch.int32)
        st["u_accept"] = torch.rand(int(n.sum()), generator=g, device="cuda")
        st["u_pick"] = torch.rand(e, generator=g, device="cuda")
        st["accepted"] = torch.empty(e, dtype=torch.int32, device="cuda")
        st["token"] = torch.empty(e, dtype=torch.int32, device="cuda")
        if own:
            _handle(case, st, np.zeros(e, np.int32), n + 1)
        return st
    hq, hk, d, page = case["h_q"], case["h_kv"], case["d"], case["page"]
    lens, news = _shape(case)[:2]
    tot = lens + news
    st["fp8"] = case["kind"] == "cache" or case["fp8"]
    table, st["n_pages"] = _tables(tot, seed, page)
    st["table"] = torch.from_numpy(table).cuda()
    st["tot"] = torch.from_numpy(tot).cuda().long()
    st["lens"], st["news"] = torch.from_numpy(lens).cuda().long(), torch.from_numpy(news).cuda().long()
    st["all_index"] = _index(tot)
    st["new_index"] = _index(news)
    t, n = int(tot.sum()), int(news.sum())
    kc = _channels(g, hk, d)
    k_all, v_all = (_randn(g, t, hk, d) * kc).bfloat16(), _randn(g, t, hk, d).bfloat16()
    if case["kind"] == "cache":
        st["k_pool"], st["k_scale"] = _fill(st, k_all, st["table"], page)
        st["v_pool"], st["v_scale"] = _fill(st, v_all, st["table"], page)
        st["k_new"], st["v_new"] = (_randn(g, n, hk, d) * kc).bfloat16(), _randn(g, n, hk, d).bfloat16()
        st["k_out"], st["v_out"] = torch.empty_like(k_all), torch.empty_like(v_all)
        if own:
            _handle(case, st, lens, news)
        return st
    prefix, video = _shape(case)[2:]
    st["k_pool"], st["k_scale"] = _fill(st, k_all, st["table"], page)
    st["v_pool"], st["v_scale"] = _fill(st, v_all, st["table"], page)
    p = int(prefix.sum())
    st["k_prefix"], st["v_prefix"] = (_randn(g, p, hk, d) * kc).bfloat16(), _randn(g, p, hk, d).bfloat16()
    st["prefix"], st["video"] = torch.from_numpy(prefix).cuda().long(), torch.from_numpy(video).cuda().long()
    st["q"] = _randn(g, n, hq, d).bfloat16()
    st["out"] = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty(n, hq, dtype=torch.float32, device="cuda")
    if own:
        _handle(case, st, lens, news, prefix, video, bf16_out=True)
    return st


# ------------------------------------------------------------------------- the plain forms


def _plain_cache(st):
    page = st["case"]["page"]
    ev, pos = st["new_index"]
    at = pos + st["lens"][ev]
    pg, slot = st["table"][ev, at // page].long(), at % page
    for x, pool, scale in ((st["k_new"], "k_pool", "k_scale"), (st["v_new"], "v_pool", "v_scale")):
        st[pool][pg, :, slot], st[scale][pg, :, slot] = _encode(x.float())
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
    x = st[pool][pg, :, pos % page]
    x = _decode(x, st[scale][pg, :, pos % page]) if st["fp8"] else x.float()
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


def _plain_verify(st):
    n, first = st["n"], st["first"]
    e, most = n.shape[0], max(1, int(st["case"]["draft_hi"]))
    i = torch.arange(most, device="cuda")
    there = i < n.unsqueeze(1)
    q_first = torch.cumsum(n, 0) - n
    p, q = st["p"], st["q"]
    if q.shape[0]:
        at = torch.where(there, q_first.unsqueeze(1) + i, 0)
        x = st["draft"].long()[at]
        px = p[torch.where(there, first.unsqueeze(1) + i, 0), x].float()
        qx = q[at, x].float()
        good = there & (st["u_accept"][at] * qx < px)
        a = torch.cumprod(good.long(), 1).sum(1)
    else:
        a = torch.zeros_like(n)
    pa = p[first + a].float()
    if q.shape[0]:
        qa = q[torch.where(a < n, q_first + a, 0)].float()
        r = torch.where((a < n).unsqueeze(1), pa - qa, pa)
    else:
        r = pa

    def fixed(w):
        return torch.floor(torch.clamp(torch.where(w > 0, w, 0.0), max=1.0) * 2.0 ** 38).long()

    w, plain = fixed(r), fixed(pa)
    w = torch.where((w.sum(1) > 0).unsqueeze(1), w, plain)
    run_sum = torch.cumsum(w, 1)
    total = run_sum[:, -1]
    m = torch.floor(st["u_pick"] * 2.0 ** 24).long()
    goal = m * (total >> 24) + ((m * (total & ((1 << 24) - 1))) >> 24)
    token = torch.where(total > 0, (run_sum <= goal.unsqueeze(1)).sum(1), -1)
    return {"accepted": a.to(torch.int32), "token": token.to(torch.int32)}


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"cache": _plain_cache, "attn": _plain_attn, "verify": _plain_verify}[kind](state)
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
    B.pad_draft_verify(st["plan"], st["p"], st["q"], st["draft"], st["u_accept"], st["u_pick"], st["accepted"], st["token"])
    return {"accepted": st["accepted"], "token": st["token"]}


# ------------------------------------------------------------------- the definition in 64 bits


def _grid8(x):
    """x (float64, groups along the last axis) on its 8-bit grid: the spacing of a value is an eighth of its
    power of two, 2^-9 scales at least."""
    big = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(big.clamp_min(1e-300) / 448.0))
    k = torch.where(torch.exp2(k - 1) * 448.0 >= big, k - 1, k)            # (log2 just above an integer)
    k = torch.where(torch.exp2(k) * 448.0 < big, k + 1, k).clamp(-120, 7)
    y = x / torch.exp2(k)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448) * torch.exp2(k)


def exact(case, seed):
    global own
    before, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = before
    if case["kind"] == "verify":
        p, q = st["p"].float().cpu().numpy(), st["q"].float().cpu().numpy()
        n, first = st["n"].cpu().numpy(), st["first"].cpu().numpy()
        x, u, v = st["draft"].cpu().numpy(), st["u_accept"].cpu().numpy(), st["u_pick"].cpu().numpy()
        got, tok, at = [], [], 0
        for e in range(len(n)):
            a = 0
            while a < n[e] and np.float32(u[at + a] * q[at + a, x[at + a]]) < p[first[e] + a, x[at + a]]:
                a += 1
            r = p[first[e] + a] - (q[at + a] if a < n[e] else np.float32(0))
            w = [np.floor(np.clip(z, 0, 1).astype(np.float64) * 2.0 ** 38).astype(np.int64) for z in (r, p[first[e] + a])]
            w = w[0] if w[0].any() else w[1]
            total = int(w.sum())
            goal = int(math.floor(float(v[e]) * 2 ** 24)) * total >> 24
            tok.append(int(np.searchsorted(np.cumsum(w), goal, side="right")) if total else -1)
            got.append(a)
            at += int(n[e])
        return {"accepted": np.array(got, np.int32), "token": np.array(tok, np.int32)}
    page, (ev, pos) = case["page"], st["all_index"]
    lens, news = _shape(case)[:2]
    pg, slot = st["table"][ev, pos // page].long(), pos % page

    def stored(pool, scale):
        b = st[pool][pg, :, slot]
        if not st["fp8"]:
            return b.double()
        b = b.to(torch.int64)
        exp, man = (b >> 3) & 15, (b & 7).double()
        mag = torch.where(exp > 0, (8 + man) * torch.exp2((exp - 10).double()), man * 2.0 ** -9)
        return torch.where(b > 127, -mag, mag) * torch.exp2(st[scale][pg, :, slot].double() - 127).unsqueeze(-1)

    k, v = stored("k_pool", "k_scale"), stored("v_pool", "v_scale")
    ends = np.cumsum(lens + news)
    if case["kind"] == "cache":
        at = torch.from_numpy(np.concatenate([np.arange(t - m, t) for t, m in zip(ends, news)])).cuda()
        k[at], v[at] = _grid8(st["k_new"].double()), _grid8(st["v_new"].double())
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
