"""Rotary positions on the way into the cache, and logits turned into probabilities, on the GPU against the fp64 oracle.

Bounds.  Rotary: a value is a cos + b sin, its angle within 2^-24 of a turn, cosine and sine within 2^-22, two products and a sum
in fp32: within 2^-20 magnitude (|a| + |b|) of the exact one, then one rounding to bf16 (2^-8 of the value at most).  Keys in 8 and 4
bits: the codes of the bf16 cache's keys, bit for bit.  Probabilities: with X the largest magnitude that a logit passes through,
an exponent is within 12 roundings of 2^-24 X / T, natural logarithms, in a term and in the sum alike, and 2^-20 covers
the exponentials and the sum: 2^-20 + 2^-19 X / T of p; a bf16 result adds 2^-8 of itself.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_02963_gb300 import binding as B
from paper_2607_02963_gb300.speculative import BranchCache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(padlib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()


def _randn(g, *shape):
    return torch.randn(*shape, generator=g).bfloat16()


class Step:
    """New tokens of a few branches and the pools that they go into."""

    def __init__(self, seed, lens, news, h_q=8, h_kv=2, d=128, page=16, fmt=B.KV_BF16):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.news = np.asarray(lens, np.int32), np.asarray(news, np.int32)
        self.h_q, self.h_kv, self.d, self.page, self.fmt = h_q, h_kv, d, page, fmt
        n = int(self.news.sum())
        self.q, self.k, self.v = _randn(g, n, h_q, d), _randn(g, n, h_kv, d), _randn(g, n, h_kv, d)
        self.cache = BranchCache(h_q, h_kv, d, len(lens), 400, 40, page_size=page, kv_format=fmt)
        self.cache.event_len = self.lens.copy()
        need = [(l + page - 1) // page for l in lens]
        order, at = torch.randperm(400, generator=g), 0
        for e, m in enumerate(need):   # the pages of what is cached already
            self.cache.page_table[e, :m] = order[at:at + m].int()
            at += m
        self.cache.pages = B.CacheState(400, used_pages=order[:at].numpy())
        self.plan = self.cache.plan(self.news)

    def pools(self):
        c = self.cache
        return [x for x in (c.k_pool, c.v_pool, c.k_scale, c.v_scale) if x is not None]


_SPECS = [dict(rotary_dim=None, theta=1e6), dict(rotary_dim=None, theta=1e4, scaling="turns", factor=8.0, original_len=8192.0),
          dict(rotary_dim=32, theta=1e4, scaling="linear", factor=2.0), dict(rotary_dim=52, theta=5e5, scaling="base", factor=4.0),
          dict(rotary_dim=54, theta=1e4, magnitude=0.5), dict(rotary_dim=2, theta=1e4),
          dict(rotary_dim=48, theta=1e6, scaling="index", factor=4.0, original_len=4096.0, low=1.0, high=32.0, magnitude=1.14)]


def _want(spec, d, x, position, layout):
    kw = {k: v for k, v in spec.items() if k not in ("rotary_dim", "theta", "magnitude")}
    f = oracle.rope_frequencies(spec["rotary_dim"] or d, spec["theta"], **kw)
    mag = spec.get("magnitude", 1.0)
    out, size = oracle.rope_turn(x.double().numpy(), position, f, layout, mag)
    return out, 2.0 ** -20 * mag * size, np.arange(d) >= 2 * len(f)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("spec", _SPECS, ids=lambda s: f"{s['rotary_dim']}-{s.get('scaling')}")
@pytest.mark.parametrize("d,h_q,h_kv,page", [(128, 28, 4, 16), (64, 14, 2, 64), (128, 16, 1, 4), (64, 3, 3, 8)])
def test_turned_on_the_way_into_each_cache(d, h_q, h_kv, page, spec, layout):
    lens, news = [0, 5, 33, 16, 7], [1, 40, 0, 3, 25]
    rng = np.random.default_rng(1)
    position = rng.integers(-5, 1 << 20, size=sum(news)).astype(np.int32)
    position[:4] = 0, 1, 2 ** 31 - 1, -2 ** 31
    rope, stored = B.Rope(d, layout=layout, **spec), None
    for fmt in (B.KV_BF16, B.KV_FP8, B.KV_FP4):
        s = Step(3, lens, news, h_q, h_kv, d, page, fmt)
        pos, q, k, v = (x.cuda() for x in (torch.from_numpy(position), s.q, s.k, s.v))
        out = torch.full_like(q, 7.0)
        B.pad_chunk_append_rope(s.plan, rope, pos, q, out, k, v, *s.pools())
        B.pad_chunk_status(s.plan)
        # (the angles of the farthest positions are exact in fp64 to 2^-21 of a radian alone)
        want, tol, still = _want(spec, d, s.q, position, layout)
        tol[2:4] += 2.0 ** -18 * np.abs(want[2:4]).max()
        got = out.double().cpu().numpy()
        assert np.all(np.abs(got - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol))
        assert np.array_equal(got[..., still], s.q.double().numpy()[..., still])
        read = s.cache.read(s.plan)
        new = np.concatenate([np.arange(t - m, t) for t, m in zip(np.cumsum(s.lens + s.news), news)])
        if fmt == B.KV_BF16:
            want, tol, still = _want(spec, d, s.k, position, layout)
            tol[2:4] += 2.0 ** -18 * np.abs(want[2:4]).max()
            got = read[0][new].double().cpu().numpy()
            assert np.all(np.abs(got - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol))
            assert np.array_equal(got[..., still], s.k.double().numpy()[..., still]) and torch.equal(read[1][new].cpu(), s.v)
            stored = read[0][new]
        # the same pools as an append of the turned keys leaves
        other = Step(3, lens, news, h_q, h_kv, d, page, fmt)
        other.cache.append(other.plan, stored.contiguous(), v)
        for a, b in zip(s.pools() + [s.cache.page_table], other.pools() + [other.cache.page_table]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rotary", [128, 54])
def test_in_place_in_a_fused_projection_on_another_stream(rotary, layout):
    s = Step(4, [9, 50], [13, 20])
    n, width = 33, (8 + 2 * 2) * 128 + 8
    pos = torch.arange(1000, 1000 + n, dtype=torch.int32, device="cuda")
    rope = B.Rope(128, rotary, layout=layout)
    out = torch.empty(n, 8, 128, dtype=torch.bfloat16, device="cuda")
    B.pad_chunk_append_rope(s.plan, rope, pos, s.q.cuda(), out, s.k.cuda(), s.v.cuda(), *s.pools())
    want = [x.clone() for x in s.pools()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        fused = torch.full((n, width), float("nan"), dtype=torch.bfloat16, device="cuda")
        q, k, v = (fused[:, a:b].unflatten(1, (-1, 128)) for a, b in ((0, 1024), (1024, 1280), (1280, 1536)))
        for x, y in ((q, s.q), (k, s.k), (v, s.v)):
            x.copy_(y.cuda())
        for x in s.pools():
            x.zero_()
        B.pad_chunk_append_rope(s.plan, rope, pos, q, q, k, v, *s.pools())
    stream.synchronize()
    assert torch.equal(q, out) and torch.equal(k.cpu(), s.k) and torch.isnan(fused[:, 1536:]).all()
    for a, b in zip(s.pools(), want):
        assert torch.equal(a, b)


def test_overlapping_outputs_are_refused():
    s = Step(5, [9], [20])
    rope, pos = B.Rope(128), torch.zeros(20, dtype=torch.int32, device="cuda")
    wide = torch.zeros(21, 1024 + 256, dtype=torch.bfloat16, device="cuda")
    q, k = wide[:20, :1024].unflatten(1, (8, 128)), wide[:20, 1024:].unflatten(1, (2, 128))
    other = torch.zeros(20, 8, 128, dtype=torch.bfloat16, device="cuda")
    def call(q_out):
        B.pad_chunk_append_rope(s.plan, rope, pos, q, q_out, k, k, *s.pools())

    for bad in (wide[1:, :1024], wide[:20, 8:1032], wide.view(-1)[:20 * 1024].view(20, 1024)):
        with pytest.raises(B.PadError, match="overlaps"):
            call(bad.unflatten(1, (8, 128)))
    call(q)
    call(other)
    torch.cuda.synchronize()


def test_a_page_outside_the_pool_keeps_its_keys_out():
    s = Step(6, [5, 20], [7, 3])
    before = [x.clone() for x in s.pools()]
    s.cache.page_table[0, 0] = 400
    out = torch.zeros(10, 8, 128, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(10, dtype=torch.int32, device="cuda")
    B.pad_chunk_append_rope(s.plan, B.Rope(128), pos, s.q.cuda(), out, s.k.cuda(), s.v.cuda(), *s.pools())
    with pytest.raises(B.PadError, match="DEVICE_BOUNDS"):
        B.pad_chunk_status(s.plan)
    page = int(s.cache.page_table[1, 1])
    changed = (s.pools()[0] != before[0]).flatten(1).any(1).nonzero().flatten().tolist()
    assert changed == [page] and (out != 0).flatten(1).any(1).all()


# ------------------------------------------------------------------------- probabilities


def _plan(news):
    prob = B.make_problem(1, 1, 64, 16)
    lens = np.zeros(len(news), np.int32)
    n = B.pad_chunk_workspace_size(prob, None, None, lens, news)
    return B.pad_chunk_plan(prob, None, None, None, lens, news, workspace=torch.zeros(n, dtype=torch.uint8, device="cuda"))


class Rows:
    def __init__(self, seed, news, vocab, hist=40, biases=0, allowed=0.0, bf16=(False, False), scale=3.0):
        r = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        e, n = len(news), int(np.sum(news))
        self.news, self.vocab, self.plan = news, vocab, _plan(news)
        kinds = [torch.bfloat16 if b else torch.float32 for b in bf16]
        self.logits = (scale * torch.randn(n, vocab, generator=g)).to(kinds[0])
        self.kind = kinds[1]
        self.params = torch.from_numpy(np.stack([r.uniform(0.5, 1.5, e), r.uniform(0.8, 1.5, e), r.uniform(-0.2, 0.5, e),
                                                 r.uniform(-0.2, 0.5, e)], 1)).float()
        self.history = torch.from_numpy((r.random((e, max(hist, 1))) ** 3 * vocab).astype(np.int32))
        self.history_len = torch.from_numpy(r.integers(0, hist + 1, e).astype(np.int32))
        self.tokens = torch.from_numpy((r.random(n) ** 3 * vocab).astype(np.int32))
        self.bias = None
        if biases:
            self.bias = [torch.from_numpy(r.integers(0, min(vocab, 2 * biases), (e, biases)).astype(np.int32)),   # (some occur again)
                         torch.from_numpy(r.normal(size=(e, biases))).float(), torch.from_numpy(r.integers(0, biases + 1, e).astype(np.int32))]
        self.allowed = None
        if allowed:
            self.allowed = r.random((n, vocab)) < allowed
            self.allowed[n // 2] = False

    def mask(self):
        if self.allowed is None:
            return None
        words = -(-self.vocab // 32)
        bits = np.ones((len(self.allowed), 32 * words), bool)      # (what lies behind the last token says nothing)
        bits[:, :self.vocab] = self.allowed
        return torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy()).cuda()

    def args(self):
        a = dict(params=self.params.cuda(), history=self.history.cuda(), history_len=self.history_len.cuda(), tokens=self.tokens.cuda(),
                 mask=self.mask())
        if self.bias is not None:
            a |= dict(zip(("bias_token", "bias_value", "bias_len"), (x.cuda() for x in self.bias)))
        return a

    def run(self, logits=None, p=None, **kw):
        logits = self.logits.cuda() if logits is None else logits
        p = torch.full(logits.shape, 7.0, dtype=self.kind, device="cuda") if p is None else p
        B.pad_chunk_probs(self.plan, logits, p, **(self.args() | kw))
        B.pad_chunk_status(self.plan)
        return p

    def check(self, p):
        got, row = p.double().cpu().numpy(), 0
        for e, n in enumerate(self.news):
            past = self.history[e, :int(self.history_len[e])].tolist()
            biases = () if self.bias is None else [(int(t), float(v)) for t, v in zip(*(x[e, :int(self.bias[2][e])] for x in self.bias[:2]))]
            for t in range(n):
                want, size = oracle.logits_to_probs(self.logits[row].double().numpy(), *self.params[e].double().tolist(),
                                                    past + self.tokens[row - t:row + 1].tolist(), biases,
                                                    None if self.allowed is None else self.allowed[row])
                temp = float(self.params[e, 0])
                rel = 2.0 ** -20 + (2.0 ** -19 * size / temp if temp > 0 else 0)
                if self.kind == torch.bfloat16:
                    rel = rel + 2.0 ** -8
                bad = np.abs(got[row] - want) - (rel * want + 1e-37)
                assert not (bad > 0).any(), f"event {e}, token {t}: {bad.max()}"
                row += 1


@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 100, 2047, 2049, 5000, 32768, 50001])
@pytest.mark.parametrize("bf16", [(False, False), (True, True), (True, False), (False, True)])
def test_probabilities(vocab, bf16):
    news = [1, 4, 0, 2]
    for i, (hist, biases, allowed) in enumerate(((40, 0, 0.0), (3000, 30, 0.3), (0, 300, 0.01))):
        r = Rows(vocab + i, news, vocab, hist, biases, allowed, bf16)
        if vocab > 40:
            r.params[1, 0] = 0.02                    # a cold row
        p = r.run()
        r.check(p)
        assert torch.equal(p, r.run())


@pytest.mark.parametrize("bf16", [(False, False), (True, True), (True, False), (False, True)])
@pytest.mark.parametrize("news,vocab", [([90, 1, 0, 130], 20001), ([90, 60, 70], 20000), ([500, 0, 900], 501)])
def test_many_rows_of_an_event(news, vocab, bf16):
    """More rows than are under way together: a cluster takes several of an event's, one after the other."""
    r = Rows(vocab, news, vocab, 200, 20, 0.5, bf16)
    r.params[-1, 0] = 0.0
    r.check(r.run())
    out = torch.full((len(r.logits), vocab + 3), 7.0, dtype=r.kind, device="cuda")   # (rows that lie elsewhere on their way out)
    r.run(p=out[:, 1:1 + vocab])
    r.check(out[:, 1:1 + vocab])
    r.bias = r.allowed = None
    r.check(r.run())


def test_the_largest_vocabulary_and_one_more():
    r = Rows(1, [1, 2], 393152, 100, 10, 0.5)
    r.check(r.run())
    with pytest.raises(B.PadError, match="vocab"):
        x = torch.zeros(3, 393153, device="cuda")
        B.pad_chunk_probs(r.plan, x, x)


def test_probabilities_over_a_part_of_the_logits_are_refused():
    r = Rows(1, [1, 2], 1000)
    x = torch.zeros(7, 1000, device="cuda")
    half = torch.zeros(3, 2000, device="cuda")
    for logits, p in ((x[:3], x[1:4]), (x[0:6:2], x[:3]), (half[:, :1000], half[:, 999:1999]), (x[:3], x.view(torch.bfloat16)[:3, :1000])):
        with pytest.raises(B.PadError, match="overlaps"):
            B.pad_chunk_probs(r.plan, logits, p)
    B.pad_chunk_probs(r.plan, half[:, :1000], half[:, 1000:])
    assert ((half[:, 1000:] - 1e-3).abs() < 1e-8).all() and not half[:, :1000].any()


@pytest.mark.parametrize("vocab", [393152, 165000, 330000])
def test_long_rows_with_long_contexts_and_biases(vocab):
    """32-bit counts and sums of biases beside one another in every form of the kernel."""
    r = Rows(8, [1, 2], vocab, 70000, 3000, 0.9)
    r.params[1, 0] = 0.0
    r.check(r.run())


def test_greedy_rows_that_begin_elsewhere():
    r = Rows(9, [3, 2], 3001, 20, 20, 0.5)
    r.params[:, 0] = 0.0
    r.params[:, 1], r.params[:, 2:] = 1.0, 0.0
    wide = torch.full((5, 3010), 99.0, device="cuda")
    wide[:, 3:3004] = r.logits.cuda()
    for kind, b in ((torch.float32, 1), (torch.float32, 3), (torch.bfloat16, 0), (torch.bfloat16, 7)):
        out = torch.full((5, 3011), 7.0, dtype=kind, device="cuda")
        r.run(wide[:, 3:3004], out[:, b:b + 3001])
        r.check(out[:, b:b + 3001])
        assert (out[:, :b] == 7).all() and (out[:, b + 3001:] == 7).all()


def test_contexts_whose_counts_need_32_bits():
    r = Rows(2, [2, 1], 3000, 70000)
    r.history[0] = 5                                  # 70000 times the same token
    r.history_len[0] = 70000
    r.params[:, 2] = 1e-4
    r.check(r.run())


def test_greedy_rows_take_the_first_largest():
    r = Rows(3, [3, 2], 40000, 10, 0, 0.5)
    r.params[:, 0] = torch.tensor([0.0, -1.0])
    r.params[:, 1], r.params[:, 2:] = 1.0, 0.0
    r.logits[0, [39999, 17, 20000]] = 50.0
    r.allowed[0, [17, 20000, 39999]] = [False, True, True]
    r.logits[1] = 0.0
    r.allowed[1] = True
    p = r.run()
    r.check(p)
    assert p[0, 20000] == 1 and p[1, 0] == 1 and not p[2].any()   # (row 2: nothing allowed)


def test_what_is_not_finite():
    r = Rows(4, [1] * 8, 5000, 0, 0, 0.5)
    r.allowed[:] = True
    nan, inf = float("nan"), float("inf")
    r.logits[0, 7] = nan
    r.logits[1, 7] = nan
    r.allowed[1, 7] = False                           # left out
    r.logits[2, 4999] = inf
    r.logits[3] = -inf
    r.logits[4, 1:] = -inf
    r.logits[5, 9], r.params[5, 0] = nan, 0.0
    r.logits[6, 9], r.params[6, 0] = inf, 0.0
    r.params[7, 0] = 1e-42                            # as cold as can be
    r.params[:, 1], r.params[:, 2:] = 1.0, 0.0
    p = r.run(tokens=None, history=None, history_len=None)
    assert p[0].isnan().all() and p[2].isnan().all()
    assert p[1].isfinite().all() and p[1, 7] == 0 and abs(float(p[1].sum()) - 1) < 1e-4
    assert not p[3].any() and p[4, 0] == 1 and not p[5].any() and p[6, 9] == 1 and p[6].sum() == 1
    assert p[7, int(r.logits[7].argmax())] == 1 and p[7].sum() == 1


def test_an_infinite_temperature_makes_all_that_is_left_alike():
    # (each p is 1 / n to 2^-20: exponents of 0, sums of ones)
    r = Rows(8, [2, 2], 5003, 0, 0, 0.5)
    r.logits[1, ::3] = -float("inf")
    r.params[:, 0] = torch.tensor([float("inf"), 3e38])
    r.params[:, 1], r.params[:, 2:] = 1.0, 0.0
    p = r.run(tokens=None, history=None, history_len=None).double().cpu()
    for row in range(4):
        left = torch.from_numpy(r.allowed[row]) & (r.logits[row] != -float("inf"))
        want = left.double() / left.sum().clamp_min(1)
        assert ((p[row] - want).abs() <= 2.0 ** -20 * want).all()


def test_tokens_outside_the_vocabulary_and_long_lengths_are_passed_over():
    r = Rows(5, [2], 1000, 20, 20)
    r.history[0, ::3], r.bias[0][0, ::4] = -1, 1000
    r.tokens[0] = 2 ** 31 - 1
    r.history_len[0] = 20
    r.bias[2][0] = 20
    p = r.run()
    r.check(p)
    assert torch.equal(p, r.run(history_len=torch.full((1,), 999, dtype=torch.int32, device="cuda")))
    r.history_len[0] = 0
    assert torch.equal(r.run(), r.run(history_len=torch.full((1,), -3, dtype=torch.int32, device="cuda")))


@pytest.mark.parametrize("bf16", [(False, False), (True, True), (True, False), (False, True)])
def test_strides_alignments_and_in_place(bf16):
    r = Rows(6, [3, 2], 3001, 20, 20, 0.5, bf16)
    want = r.run()
    for a, b in ((0, 0), (1, 1), (1, 2), (3, 0), (5, 4)):
        wide = torch.full((5, 3001 + 16), float("nan"), dtype=r.logits.dtype, device="cuda")
        out = torch.full((5, 3001 + 16 + a), 7.0, dtype=r.kind, device="cuda")
        wide[:, a:a + 3001] = r.logits.cuda()
        mask = torch.zeros(5, 97, dtype=torch.int32, device="cuda")
        mask[:, 1:95] = r.mask()
        r.run(wide[:, a:a + 3001], out[:, b:b + 3001], mask=mask[:, 1:95])
        r.check(out[:, b:b + 3001])       # (terms are summed by 16-byte pieces, which begin elsewhere: equal within the bound alone)
        assert (out[:, :b] == 7).all() and (out[:, b + 3001:] == 7).all()
    if bf16[0] == bf16[1]:
        x = r.logits.cuda()
        assert torch.equal(r.run(x, x), want)


def test_nothing_but_a_softmax():
    r = Rows(7, [2, 1], 777)
    x = r.logits.cuda()
    p = torch.empty_like(x)
    B.pad_chunk_probs(r.plan, x, p)
    want = torch.softmax(x.double(), 1)
    assert ((p.double() - want).abs() <= 2.0 ** -19 * 16 * want).all()


# ------------------------------------------------------------- a step's calls in a row


@pytest.mark.parametrize("fmt", [B.KV_BF16, B.KV_FP8, B.KV_FP4])
def test_a_step_captured_and_replayed(fmt):
    """Rotary append, attention, probabilities and verification in one graph, replayed with other contents."""
    news, vocab = [5, 1, 9], 1200
    s = Step(8, [40, 0, 20], news, 28, 4, 128, 16, fmt)
    n, nd = 15, 12
    rope = B.Rope(128, theta=1e6)
    sets = []
    for i in range(3):
        g = torch.Generator().manual_seed(i)
        r = Rows(i, news, vocab, 50, 10, 0.7)
        sets.append([x.cuda() for x in (_randn(g, n, 28, 128), _randn(g, n, 4, 128), _randn(g, n, 4, 128),
                                        torch.randint(0, 9999, (n,), generator=g).int(), r.logits, r.params, r.history, r.history_len,
                                        r.tokens, *r.bias, r.mask(), torch.softmax(r.logits[:nd], 1), r.tokens[:nd],
                                        torch.rand(nd, generator=g), torch.rand(3, generator=g))])
    buf = [x.clone() for x in sets[0]]
    plan, pools = s.plan, s.pools()
    q_out, out = (torch.empty(n, 28, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    p = torch.empty(n, vocab, device="cuda")
    acc, tok = (torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(2))

    def step():
        q, k, v, pos, logits, params, hist, hist_len, tokens, bt, bv, bl, mask, dq, draft, ua, up = buf
        B.pad_chunk_append_rope(plan, rope, pos, q, q_out, k, v, *pools)
        B.pad_chunk_attn(plan, q_out, None, None, *pools[:2], out, None, *pools[2:])
        B.pad_chunk_probs(plan, logits, p, params, hist, hist_len, tokens, bt, bv, bl, mask)
        B.pad_draft_verify(plan, p, dq, draft, ua, up, acc, tok)

    def load(i):
        for b, x in zip(buf, sets[i]):
            b.copy_(x)
        for x in (q_out, out, p, acc, tok):
            x.fill_(3)

    want = []
    for i in range(3):
        load(i)
        step()
        want.append([x.clone() for x in (q_out, out, p, acc, tok, *pools)])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (1, 2, 0, 1):
        load(i)
        graph.replay()
        for x, w in zip((q_out, out, p, acc, tok, *pools), want[i]):
            assert torch.equal(x.view(torch.uint8), w.view(torch.uint8))
    B.pad_chunk_status(plan)


@pytest.mark.parametrize("fmt", [B.KV_BF16, B.KV_FP8, B.KV_FP4])
def test_steps_of_a_loop_against_the_oracle(fmt):
    """Three steps of a loop (rotary append, attention, probabilities, verification, commit) on one cache, each held against the
    oracle: the queries turned, attention over what the cache reads back as (that the cache holds the turned keys is tested
    above), the probabilities, and the drafts that those keep."""
    g = torch.Generator().manual_seed(11)
    events, vocab, h_q, h_kv, d = 3, 700, 14, 2, 64
    cache = BranchCache(h_q, h_kv, d, events, 60, 20, page_size=8, kv_format=fmt, out_dtype=0)
    spec = dict(rotary_dim=48, theta=1e4, scaling="turns", factor=4.0, original_len=512.0)
    rope = B.Rope(d, **spec)
    news = [[5, 1, 9], [40, 3, 0], [2, 8, 4]]
    for i, n_new in enumerate(news):
        plan = cache.plan(n_new)
        n, lens = plan.n_tokens, cache.event_len.copy()
        ev = np.repeat(np.arange(events), n_new)
        pos = np.concatenate([lens[e] + np.arange(m) for e, m in enumerate(n_new)]).astype(np.int32)
        q, k, v = _randn(g, n, h_q, d), _randn(g, n, h_kv, d), _randn(g, n, h_kv, d)
        q_out = cache.append_rope(plan, rope, torch.from_numpy(pos).cuda(), q.cuda(), k.cuda(), v.cuda())
        want, tol, _ = _want(spec, d, q, pos, "half")
        assert np.all(np.abs(q_out.double().cpu().numpy() - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol))
        kk, vv = (x.double().cpu().numpy() for x in cache.read(plan))
        out = cache.attend(plan, q_out).double().cpu().numpy()
        first = np.concatenate([[0], np.cumsum(lens + np.asarray(n_new))])
        for e in range(events):
            mine = slice(first[e], first[e + 1])
            o, _, mag = oracle.chunk_attention(q_out[ev == e].double().cpu().numpy(), kk[mine], vv[mine], int(lens[e]) + 1, d ** -0.5)
            assert np.all(np.abs(out[ev == e] - o) <= (2.0 ** -8 + 1e-4) * mag)
        r = Rows(20 + i, n_new, vocab, 30, 5, 0.6)
        r.plan = plan
        p = r.run()
        r.check(p)
        nd = plan.n_drafts
        drafted = np.concatenate([np.flatnonzero(ev == e)[:-1] for e in range(events)]).astype(int)
        dq = torch.softmax(torch.log(p[drafted].clamp_min(1e-9)) + 0.4 * torch.randn(nd, vocab, generator=g).cuda(), 1)
        draft = dq.argmax(1).int() if nd else torch.empty(0, dtype=torch.int32, device="cuda")
        ua, up = torch.rand(nd, generator=g), torch.rand(events, generator=g)
        accepted, token = cache.verify(plan, p, dq, draft, ua.cuda(), up.cuda())
        B.pad_chunk_status(plan)
        at = 0
        for e, m in enumerate(n_new):
            if m == 0:
                assert int(token[e]) == -1
                continue
            rows = np.flatnonzero(ev == e)
            want = oracle.draft_verify(p[rows].cpu().numpy(), dq[at:at + m - 1].cpu().numpy(), draft[at:at + m - 1].tolist(),
                                       ua[at:at + m - 1].numpy(), float(up[e]))
            assert (int(accepted[e]), int(token[e])) == want
            at += m - 1
        lens = np.where(np.asarray(n_new) > 0, lens + accepted.cpu().numpy() + 1, lens)
        assert np.array_equal(cache.commit(plan, accepted), lens)


@pytest.mark.parametrize("fmt", [B.KV_BF16, B.KV_FP4])
def test_the_example_runs(fmt):
    from paper_2607_02963_gb300 import speculative
    kept, cache = speculative.example(events=3, drafts=3, steps=3, prefix=200, vocab=500, h_q=8, h_kv=2, kv_format=fmt)
    assert len(kept) == 3 and all(1 <= m <= 4 for row in kept for m in row)
    assert cache.event_len.tolist() == np.sum(kept, axis=0).tolist()
