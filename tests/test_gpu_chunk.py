"""The multi-token step on the GPU against its fp64 oracle: the cache written and read back, attention of
chunk tokens, verification of drafted tokens.

Bounds.  The cache: equal, bit for bit (a code is one rounding, whose operand is exact).  Attention: a weight
P is rounded to bf16 (eight significant bits) for P.V, 2^-8 of itself at most, so an output is within
2^-8 sum p |v| of the exact one; 1e-4 sum p |v| more covers scores, exponentials and sums in fp32 (scores below 32 in magnitude, each within
2^-20 of that), and a bf16 output adds 2^-8 of its own magnitude.  The lse: 1e-4.  Verification: equal.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_02963_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(padlib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()


class Case:
    """Random branches: a page table in random order, pools whose other slots hold NaN, whole sequences of
    private tokens (the new ones included) and prefixes."""

    def __init__(self, seed, lens, news, prefix=None, video=None, h_q=8, h_kv=2, d=128, page=16, fp8=False,
                 spare=5, poison=True):
        r = np.random.default_rng(seed)
        self.lens, self.news = np.asarray(lens, np.int32), np.asarray(news, np.int32)
        self.prefix, self.video = prefix, video
        self.h_q, self.h_kv, self.d, self.page, self.fp8 = h_q, h_kv, d, page, fp8
        tot = self.lens + self.news
        need = (tot + page - 1) // page
        self.n_pages = int(need.sum()) + spare
        order = r.permutation(self.n_pages)
        self.table = np.full((len(tot), max(1, int(need.max(initial=0))) + 1), -1, np.int32)
        at = 0
        for e, n in enumerate(need):
            self.table[e, :n] = order[at:at + n]
            at += n
        g = torch.Generator().manual_seed(seed)

        def randn(*shape):
            return torch.randn(*shape, generator=g).bfloat16()

        self.q = randn(int(self.news.sum()), h_q, d)
        self.k = [randn(int(t), h_kv, d) for t in tot]
        self.v = [randn(int(t), h_kv, d) for t in tot]
        n_pre = int(np.sum(prefix)) if prefix is not None else 0
        self.k_pre, self.v_pre = randn(n_pre, h_kv, d), randn(n_pre, h_kv, d)
        shape = (self.n_pages, h_kv, page, d)
        if fp8:
            self.pools = [torch.full(shape, 0x7F if poison else 0, dtype=torch.uint8) for _ in range(2)]
            self.scales = [torch.full(shape[:3], 0xFF if poison else 0, dtype=torch.uint8) for _ in range(2)]
        else:
            self.pools = [torch.full(shape, float("nan") if poison else 0, dtype=torch.bfloat16) for _ in range(2)]
            self.scales = [None, None]

    def store(self, upto=None):
        """Put the sequences (positions below upto[e]) into the host pools."""
        for e in range(len(self.lens)):
            n = int((self.lens + self.news)[e] if upto is None else upto[e])
            if n == 0:
                continue
            pos = np.arange(n)
            pg, slot = self.table[e, pos // self.page].astype(np.int64), pos % self.page
            for i, x in enumerate((self.k[e], self.v[e])):
                if self.fp8:
                    c, b = oracle.kv8_encode(x[:n].double().numpy())
                    self.pools[i][pg, :, slot] = torch.from_numpy(c)
                    self.scales[i][pg, :, slot] = torch.from_numpy(b)
                else:
                    self.pools[i][pg, :, slot] = x[:n]
        return self

    def cached(self, i, e):
        """K (0) or V (1) of event e as the cache holds it, float64."""
        x = (self.k, self.v)[i][e].double().numpy()
        return oracle.kv8_decode(*oracle.kv8_encode(x)) if self.fp8 else x

    def device(self):
        self.dp = [x.cuda() for x in self.pools]
        self.ds = [None if x is None else x.cuda() for x in self.scales]
        self.dt = torch.from_numpy(self.table).cuda()
        return self

    def plan(self, out_dtype=0, flags=0, cache=None, stream=None):
        prob = B.make_problem(self.h_q, self.h_kv, self.d, self.page, out_dtype=out_dtype, flags=flags)
        fmt = B.KV_FP8 if self.fp8 else B.KV_BF16
        n = B.pad_chunk_workspace_size(prob, self.prefix, self.video, self.lens, self.news, kv_format=fmt)
        self.ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
        return B.pad_chunk_plan(prob, cache, self.prefix, self.video, self.lens, self.news, page_table=self.dt,
                                n_pages=self.n_pages, kv_format=fmt, workspace=self.ws, stream=stream)

    def attend(self, plan, q=None, stream=None):
        p = plan.problem
        q = self.q.cuda() if q is None else q
        out = torch.full((plan.n_tokens, self.h_q, self.d), 7.0, device="cuda",
                         dtype=torch.bfloat16 if p.out_dtype == 1 else torch.float32)
        lse = torch.full((plan.n_tokens, self.h_q), 7.0, device="cuda")
        pre = self.k_pre.shape[0] > 0
        B.pad_chunk_attn(plan, q, self.k_pre.cuda() if pre else None, self.v_pre.cuda() if pre else None, *self.dp, out,
                         lse, *self.ds, stream=stream)
        return out, lse

    def want(self, e, k=None, v=None):
        k = self.cached(0, e) if k is None else k
        v = self.cached(1, e) if v is None else v
        pl = 0
        if self.prefix is not None and self.prefix[self.video[e]] > 0:
            pl = int(self.prefix[self.video[e]])
            a = int(np.sum(self.prefix[:self.video[e]]))
            k = np.concatenate([self.k_pre[a:a + pl].double().numpy(), k])
            v = np.concatenate([self.v_pre[a:a + pl].double().numpy(), v])
        at = int(self.news[:e].sum())
        q = self.q[at:at + int(self.news[e])].double().numpy()
        return (at, *oracle.chunk_attention(q, k, v, pl + int(self.lens[e]) + 1, 1.0 / self.d ** 0.5))

    def check(self, out, lse, bf16=False):
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for e in range(len(self.lens)):
            at, o, l, mag = self.want(e)
            n = int(self.news[e])
            tol = (2.0 ** -8 + 1e-4) * mag
            if bf16:
                tol = tol + 2.0 ** -8 * (np.abs(o) + tol)
            assert np.all(np.abs(out[at:at + n] - o) <= tol), f"event {e}: {np.max(np.abs(out[at:at + n] - o) - tol)}"
            assert np.all(np.abs(lse[at:at + n] - l) <= 1e-4)


# ------------------------------------------------------------------------------ attention

_SHAPES = [
    # lens, news, prefix, video: single tokens, lengths of zero and one, page and tile ends, ragged chunks
    ([0], [1], None, None),
    ([0, 1, 15, 16, 17, 255, 256, 257], [1] * 8, None, None),
    ([63, 0, 31, 5], [1, 0, 2, 5], None, None),
    ([0, 0, 40], [3, 8, 1], [77], [0, 0, 0]),
    ([3, 90, 0, 7], [4, 0, 9, 1], [0, 129, 640], [0, 1, 1, 2]),
    ([130], [33], [128], [0]),
    ([700, 2], [70, 150], None, None),
]


@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,h_q,h_kv,page", [(128, 28, 4, 16), (64, 14, 2, 64), (128, 16, 1, 4), (64, 3, 3, 8),
                                             (128, 4, 2, 32)])
def test_attention(d, h_q, h_kv, page, fp8, flags):
    for i, (lens, news, prefix, video) in enumerate(_SHAPES):
        c = Case(100 * i + d + page, lens, news, prefix, video, h_q, h_kv, d, page, fp8).store().device()
        bf16 = (i + page) % 2 == 0
        plan = c.plan(out_dtype=1 if bf16 else 0, flags=flags)
        out, lse = c.attend(plan)
        c.check(out, lse, bf16)
        B.pad_chunk_status(plan)
        out2, lse2 = c.attend(plan)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,lens,news,prefix", [(128, [5000, 3], [1, 1], None), (64, [2500], [17], None),
                                                (128, [64, 10, 0], [5, 2, 8], [3001])])
def test_attention_over_split_keys(d, lens, news, prefix, fp8, flags):
    c = Case(7, lens, news, prefix, None if prefix is None else [0] * len(lens), 8, 2, d, 16, fp8).store().device()
    plan = c.plan(flags=flags)
    i = plan.info()
    assert max(i["page_splits"], i["prefix_splits"]) > 1
    c.check(*c.attend(plan))
    B.pad_chunk_status(plan)


@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC])
@pytest.mark.parametrize("fp8", [False, True])
def test_large_scores_and_a_key_that_dominates(fp8, flags):
    """Scores that span hundreds, rising along the keys: every block moves the running maximum."""
    c = Case(8, [700, 30], [3, 40], [300], [0, 0], 8, 2, 128, 16, fp8)
    c.q = (4.0 * c.q.float()).bfloat16()
    for e in range(2):
        ramp = torch.linspace(0.1, 2.0, c.k[e].shape[0])[:, None, None]
        c.k[e] = (c.k[e].float() * ramp).bfloat16()
    c.store().device()
    out, lse = c.attend(c.plan(flags=flags))
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for e in range(2):
        at, o, l, mag = c.want(e)
        n = int(c.news[e])
        # scores up to 256 in magnitude, each within 2^-20 of that
        assert np.all(np.abs(out[at:at + n] - o) <= (2.0 ** -8 + 1e-3) * mag)
        assert np.all(np.abs(lse[at:at + n] - l) <= 1e-3)


@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_values_of_very_different_size(d, fp8, flags):
    """V whose tokens differ by 2^40 in size, the large ones hardly attended to, Q and K whose channels differ by
    2^20: what is small is as exact as what is large."""
    c = Case(14, [200, 15], [2, 3], None, None, 8, 2, d, 16, fp8)
    wide = torch.where(torch.arange(d) % 8 == 0, 2.0 ** 10, 2.0 ** -10)
    c.q = (c.q.float() * wide * 2.0 ** -3).bfloat16()
    for e in range(2):
        n = c.k[e].shape[0]
        big = torch.arange(n) % 3 == 1
        c.k[e] = (c.k[e].float() / wide).bfloat16()
        c.v[e] = (c.v[e].float() * torch.where(big, 2.0 ** 12, 2.0 ** -28)[:, None, None]).bfloat16()
    # channel 0 of every query is large and positive, and pushes the large tokens' scores 80 and more below
    c.q[:, :, 0] = 2.0 ** 10
    for e in range(2):
        big = torch.arange(c.k[e].shape[0]) % 3 == 1
        c.k[e][:, :, 0] = torch.where(big, -1.0, 0.0)[:, None].bfloat16()
    c.store().device()
    c.check(*c.attend(c.plan(flags=flags)))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_finite_stays_with_the_tokens_that_see_it(what, flags, fp8):
    """A later chunk token's K and V, and another event's, are not finite: earlier tokens do not notice."""
    c = Case(9, [20, 37], [6, 5], None, None, 8, 2, 128, 16, fp8)
    clean = Case(9, [20, 37], [6, 5], None, None, 8, 2, 128, 16, fp8)
    c.k[0][23, 0, 5] = what   # chunk token 3 of event 0, head 0
    c.v[0][24, 1, 9] = what   # chunk token 4, head 1
    c.store().device()
    out, lse = c.attend(c.plan(flags=flags))
    out = out.double().cpu().numpy()
    for e in range(2):
        at, o, l, mag = clean.want(e)
        tol = (2.0 ** -8 + 1e-4) * mag
        good = np.ones(o.shape[:2], bool)
        if e == 0:
            good[3:, :4] = False   # query heads 0-3 read kv-head 0
            good[4:, 4:] = False
        got = out[at:at + len(o)]
        assert np.all((np.abs(got - o) <= tol)[good])
    # and those that do see it notice: a NaN, or where one column of V is infinite that column
    assert not np.all(np.isfinite(out[4:6, 4:]))
    if np.isnan(what):
        assert np.all(np.isnan(out[4:6, 4:, 9]))


@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_TC])
def test_strides_alignment_and_another_stream(flags):
    """q, k_new and v_new as slices of one fused projection, on a stream of their own."""
    c = Case(10, [9, 50], [3, 20], [64], [0, 0], 8, 2, 128, 16, False)
    c.store(c.lens).device()
    n, width = int(c.news.sum()), (8 + 2 * 2) * 128 + 8
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        fused = torch.full((n, width), float("nan"), dtype=torch.bfloat16, device="cuda")
        q, k, v = (fused[:, a:b].unflatten(1, (-1, 128)) for a, b in ((0, 1024), (1024, 1280), (1280, 1536)))
        q.copy_(c.q.cuda())
        new = [slice(int(l), int(l + m)) for l, m in zip(c.lens, c.news)]
        k.copy_(torch.cat([c.k[e][new[e]] for e in range(2)]).cuda())
        v.copy_(torch.cat([c.v[e][new[e]] for e in range(2)]).cuda())
        plan = c.plan(flags=flags)
        B.pad_chunk_append(plan, k, v, *c.dp)
        out, lse = c.attend(plan, q)
    s.synchronize()
    c.check(out, lse)


def test_offsets_past_32_bits():
    """Pools of more than 2^32 bytes, and more than 2^31 elements: the branches' pages lie at their end."""
    for fp8, page_bytes in ((False, 2 * 64 * 4 * 128), (True, 64 * 4 * 128)):
        c = Case(11, [100, 200], [3, 1], None, None, 8, 4, 128, 64, fp8).store()
        extra = (1 << 32) // page_bytes + 3
        total = c.n_pages + extra
        c.dp, c.ds = [], []
        for pool, scale in zip(c.pools, c.scales):
            big = torch.empty((total,) + tuple(pool.shape[1:]), dtype=pool.dtype, device="cuda")
            big[extra:] = pool.cuda()
            c.dp.append(big)
            if scale is None:
                c.ds.append(None)
            else:
                bs = torch.empty((total,) + tuple(scale.shape[1:]), dtype=torch.uint8, device="cuda")
                bs[extra:] = scale.cuda()
                c.ds.append(bs)
        c.n_pages = total
        c.dt = torch.from_numpy(np.where(c.table >= 0, c.table + extra, -1).astype(np.int32)).cuda()
        for flags in (0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC):
            plan = c.plan(flags=flags)
            c.check(*c.attend(plan))
        k, v = (torch.empty((plan.n_cached, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        B.pad_chunk_read(plan, *c.dp, k, v, *c.ds)
        assert np.array_equal(k.double().cpu().numpy(), np.concatenate([c.cached(0, e) for e in range(2)]))
        del c


@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC])
@pytest.mark.parametrize("fp8", [False, True])
def test_pages_outside_the_pool_hide_their_tokens(fp8, flags):
    """A bad page-table entry is reported, and its keys take no part; a row that has no other gets 0."""
    c = Case(12, [40, 3], [2, 2], None, None, 8, 2, 128, 16, fp8).store().device()
    c.dt[0, 1] = c.n_pages
    c.dt[1, 0] = -1
    plan = c.plan(flags=flags)
    out, lse = c.attend(plan)
    with pytest.raises(B.PadError) as err:
        B.pad_chunk_status(plan)
    assert err.value.status == 7
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    keep = [i for i in range(42) if not 16 <= i < 32]
    k, v = c.cached(0, 0)[keep], c.cached(1, 0)[keep]
    o, l, mag = oracle.chunk_attention(c.q[:2].double().numpy(), k, v, 41 - 16, 128 ** -0.5)
    assert np.all(np.abs(out[:2] - o) <= (2.0 ** -8 + 1e-4) * mag) and np.all(np.abs(lse[:2] - l) <= 1e-4)
    assert np.all(out[2:] == 0) and np.all(np.isneginf(lse[2:]))
    # and it is this plan's report alone
    c.dt.copy_(torch.from_numpy(c.table))
    plan = c.plan(flags=flags)
    c.check(*c.attend(plan))
    B.pad_chunk_status(plan)


def test_a_chunk_is_single_token_steps_one_after_the_other():
    """Three tokens at once, and through the one-token step of the library."""
    c = Case(13, [20, 5], [3, 3], [200], [0, 0], 8, 2, 128, 16, False).store().device()
    out, lse = c.attend(c.plan())
    prob = B.make_problem(8, 2, 128, 16)
    used = [int(p) for e in range(2) for p in c.table[e, :(int(c.lens[e]) + 15) // 16]]
    lens = c.lens.copy()
    k_pre, v_pre = c.k_pre.cuda(), c.v_pre.cuda()
    ws = torch.zeros(B.pad_workspace_size(prob, [200], [0, 0]), dtype=torch.uint8, device="cuda")
    table = torch.from_numpy(c.table).cuda()
    cache = B.CacheState(c.n_pages, used_pages=used)
    for t in range(3):
        rows = [t, 3 + t]
        k_new = torch.stack([c.k[e][int(c.lens[e]) + t] for e in range(2)]).cuda()
        v_new = torch.stack([c.v[e][int(c.lens[e]) + t] for e in range(2)]).cuda()
        step = B.pad_plan(prob, cache, [200], [0, 0], lens, page_table=table, workspace=ws)
        o1, l1 = torch.empty(2, 8, 128, device="cuda"), torch.empty(2, 8, device="cuda")
        B.pad_decode_step(step, c.q[rows].cuda(), k_new, v_new, k_pre, v_pre, *c.dp, o1, l1)
        torch.cuda.synchronize()
        assert float((o1 - out[rows]).abs().max()) <= 2e-2 and float((l1 - lse[rows]).abs().max()) <= 2e-4
        lens = lens + 1


# ------------------------------------------------------------------------------ the cache


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,h_kv,page", [(128, 4, 16), (64, 2, 64), (128, 1, 4), (64, 3, 8)])
def test_append_and_read_back(d, h_kv, page, fp8):
    c = Case(20 + page, [0, 1, 17, 64, 5], [1, 0, 30, 129, 3], None, None, h_kv, h_kv, d, page, fp8)
    # magnitudes from the smallest scales to beyond the largest, and special groups
    mag = 2.0 ** np.linspace(-135, 18, c.k[3].shape[0])
    c.k[3] = (c.k[3].double() * torch.from_numpy(mag)[:, None, None]).bfloat16()
    c.k[3][70] = 0
    c.v[3][71, 0, 3] = float("nan")
    c.v[3][72, 0, d - 1] = float("-inf")
    c.v[3][73] = 448.0 * 2.0 ** -3
    c.v[3][74] = 450.0 * 2.0 ** -3
    c.store(c.lens).device()
    used = [int(p) for e in range(5) for p in c.table[e, :(int(c.lens[e]) + page - 1) // page]]
    cache = B.CacheState(c.n_pages, used_pages=used)
    c.dt = torch.where(torch.arange(c.dt.shape[1], device="cuda") < torch.from_numpy((c.lens + page - 1) // page).cuda()[:, None],
                       c.dt, -1).contiguous()
    before = [x.clone() for x in c.dp]
    plan = c.plan(cache=cache)
    new = [slice(int(l), int(l + m)) for l, m in zip(c.lens, c.news)]
    k, v = (torch.cat([x[e][new[e]] for e in range(5)]).cuda() for x in (c.k, c.v))
    B.pad_chunk_append(plan, k, v, *c.dp, *c.ds)
    ko, vo = (torch.full((plan.n_cached, h_kv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.pad_chunk_read(plan, *c.dp, ko, vo, *c.ds)
    B.pad_chunk_status(plan)
    ev, col, pg = plan.new_pages()
    assert np.array_equal(c.dt.cpu().numpy()[ev, col], pg)
    for got, i in ((ko, 0), (vo, 1)):
        want = np.concatenate([c.cached(i, e) for e in range(5)])
        # (what lies below bf16's own grid is rounded to it)
        want = torch.from_numpy(want).bfloat16().double().numpy()
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    # nothing but the new tokens' slots has changed
    table = c.dt.cpu().numpy()
    touched = torch.zeros(c.n_pages, page, dtype=torch.bool)
    for e in range(5):
        for pos in range(int(c.lens[e]), int(c.lens[e] + c.news[e])):
            touched[int(table[e, pos // page]), pos % page] = True
    for a, b in zip(before, c.dp):
        same = (a.view(torch.uint8) == b.view(torch.uint8)).flatten(3).all(-1).all(1).cpu()
        assert bool((same | touched).all())


def test_append_skips_a_page_outside_the_pool():
    c = Case(21, [0, 0], [20, 4], None, None, 2, 2, 64, 16, True, poison=False).device()
    c.dt[0, 1] = 1 << 20
    plan = c.plan()
    k, v = (torch.ones((24, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.pad_chunk_append(plan, k, v, *c.dp, *c.ds)
    with pytest.raises(B.PadError) as err:
        B.pad_chunk_status(plan)
    assert err.value.status == 7
    assert int((c.ds[0] != 0).sum()) == 2 * 20   # 16 tokens of event 0, four of event 1, two heads


# ------------------------------------------------------------------------------ verification


def _verify(n, vocab, p, q, draft, ua, up, stride=None):
    """n: drafted tokens per event, -1 for an event without new tokens."""
    news = np.asarray(n) + 1
    prob = B.make_problem(4, 1, 64)
    ws = torch.zeros(B.pad_chunk_workspace_size(prob, None, None, np.zeros(len(news), np.int32), news), dtype=torch.uint8, device="cuda")
    plan = B.pad_chunk_plan(prob, None, None, None, np.zeros(len(news), np.int32), news, workspace=ws)

    def rows(x):
        if stride is None:
            return x.cuda().contiguous()
        wide = torch.full((x.shape[0], stride), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, :vocab] = x.cuda()
        return wide[:, :vocab]

    acc, tok = (torch.full((len(news),), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    B.pad_draft_verify(plan, rows(p), rows(q), draft.cuda(), ua.cuda(), up.cuda(), acc, tok)
    want, at, row = [], 0, 0
    for e, m in enumerate(n):
        if m < 0:
            want.append((0, -1))
            continue
        want.append(oracle.draft_verify(p[row:row + m + 1].float().numpy(), q[at:at + m].float().numpy(),
                                        draft[at:at + m].tolist(), ua[at:at + m].numpy(), float(up[e])))
        at, row = at + m, row + m + 1
    return plan, list(zip(acc.tolist(), tok.tolist())), want


def _tables(g, rows, vocab, dtype, sharp=2.0):
    return torch.softmax(sharp * torch.randn(rows, vocab, generator=g), -1).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,stride", [(1, None), (2, None), (127, 129), (1000, None), (4096, 4100), (50021, None)])
def test_verify(vocab, stride, dtype):
    g = torch.Generator().manual_seed(vocab)
    n = [0, 1, 3, -1, 8, 2, -1, 5] + [4] * 16
    drafts, rows = sum(max(0, m) for m in n), sum(m + 1 for m in n)
    p = _tables(g, rows, vocab, dtype)
    has = torch.cat([torch.arange(m + 1) < m for m in n if m >= 0])
    q = torch.softmax(torch.log(p[has].float() + 1e-9) + 0.7 * torch.randn(drafts, vocab, generator=g), -1).to(dtype)
    draft = torch.multinomial(q.float() + 1e-12, 1, generator=g)[:, 0].to(torch.int32)
    ua, up = torch.rand(drafts, generator=g), torch.rand(len(n), generator=g)
    plan, got, want = _verify(n, vocab, p, q, draft, ua, up, stride)
    assert got == want
    B.pad_chunk_status(plan)
    if vocab > 1000:
        assert len({a for a, _ in got}) > 2   # (whole drafts, and some cut short)


def test_verify_edges():
    g = torch.Generator().manual_seed(5)
    vocab = 700
    p = _tables(g, 12, vocab, torch.float32)
    q = _tables(g, 6, vocab, torch.float32)
    p[0:2] = q[0]                       # event 0: the draft's own distribution, u near 1: kept
    p[2], p[3] = 0, 0                   # event 1: no weight anywhere
    p[4] = q[2] * 0.5                   # event 2: rejected, and the difference has no weight left: p itself
    p[6, 17] = float("nan")             # event 3: a NaN where the draft is, and others that are masked
    q[3, 17] = 1.0
    p[6, :10] = float("nan")
    p[8, 5] = float("inf")              # event 4: weights are capped
    p[10, :] = 0
    p[10, vocab - 1] = 1e-11            # event 5: the last token alone, close to the smallest weight
    n = [1] * 6
    draft = torch.tensor([3, 4, 5, 17, 5, 6], dtype=torch.int32)
    for up in (0.0, 0.25, 1.0 - 2.0 ** -24):
        ua = torch.tensor([1.0 - 2.0 ** -24, 0.0, 0.75, 0.5, 0.5, 0.9])
        _, got, want = _verify(n, vocab, p, q, draft, ua, torch.full((6,), up))
        assert got == want
        assert got[1] == (0, -1) and got[0][0] == 1 and got[2][0] == 0 and got[3][0] == 0


def test_verify_rejects_tokens_outside_the_vocabulary():
    g = torch.Generator().manual_seed(6)
    p, q = _tables(g, 6, 50, torch.float32), _tables(g, 4, 50, torch.float32)
    draft = torch.tensor([50, 3, -1, 2], dtype=torch.int32)
    plan, got, want = _verify([2, 2], 50, p, q, draft, torch.zeros(4), torch.full((2,), 0.5))
    assert got == want and got[0][0] == 0 and got[1][0] == 0
    with pytest.raises(B.PadError) as err:
        B.pad_chunk_status(plan)
    assert err.value.status == 7


# ------------------------------------------------------------------------------ refusals


def test_refusals():
    c = Case(30, [4], [2], [16], [0], 8, 2, 128, 16, True).store().device()
    plan = c.plan()
    q, out, lse = c.q.cuda(), torch.empty(2, 8, 128, device="cuda"), torch.empty(2, 8, device="cuda")
    pre = (c.k_pre.cuda(), c.v_pre.cuda())
    x = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.PadError):
        B.pad_chunk_attn(plan, q, *pre, *c.dp, out, lse)                       # no scales
    with pytest.raises(B.PadError):
        B.pad_chunk_attn(plan, q, None, None, *c.dp, out, lse, *c.ds)          # no prefix
    with pytest.raises(B.PadError):
        B.pad_chunk_append(plan, x, x, *c.dp)
    for bad in (dict(q=q[:1]), dict(q=q.float()), dict(out=out.bfloat16()), dict(lse=lse[:, :4]), dict(q=q.transpose(0, 1))):
        a = dict(q=q, out=out, lse=lse) | bad
        with pytest.raises(ValueError):
            B.pad_chunk_attn(plan, a["q"], *pre, *c.dp, a["out"], a["lse"], *c.ds)
    with pytest.raises(ValueError):
        B.pad_chunk_append(plan, x, x, c.dp[0][:1], c.dp[1], *c.ds)
    with pytest.raises(B.PadError):
        wide = torch.zeros(2, 2 * 128 + 4, dtype=torch.bfloat16, device="cuda")[:, :256].unflatten(1, (2, 128))
        B.pad_chunk_append(plan, wide, wide, *c.dp, *c.ds)                     # a stride that is no multiple of 8
    with pytest.raises(B.PadError):
        odd = torch.zeros(2 * 8 * 128 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, 8, 128)
        B.pad_chunk_attn(plan, odd, *pre, *c.dp, out, lse, *c.ds)              # alignment
    with pytest.raises(B.PadError):
        B.pad_chunk_plan(plan.problem, None, [16], [0], [4], [2], page_table=c.dt, n_pages=c.n_pages, kv_format=B.KV_FP8,
                         workspace=c.ws[:256])
    with pytest.raises(B.PadError):
        B.pad_chunk_plan(plan.problem, None, [16], [0], [4], [2], page_table=c.dt, n_pages=c.n_pages, kv_format=B.KV_FP8,
                         workspace=c.ws[16:])
    B.pad_chunk_status(plan)


# ------------------------------------------------------------------------------ the steps together


@pytest.mark.parametrize("kv_format", [B.KV_BF16, B.KV_FP8])
def test_speculative_steps_together(kv_format):
    """Drafts written, attended, verified and partly taken back, step after step: the cache holds exactly the kept
    tokens, in the lowest pages, and a step's attention is that over them."""
    from paper_2607_02963_gb300.speculative import BranchCache
    events, page, hq, hk, d, vocab = 3, 4, 8, 2, 64, 50
    g = torch.Generator().manual_seed(3)
    cache = BranchCache(hq, hk, d, events, n_pages=40, max_pages=12, page_size=page, kv_format=kv_format,
                        prefix_len=[20], event_video=[0] * events, out_dtype=0)
    k_pre, v_pre = torch.randn(20, hk, d, generator=g).bfloat16(), torch.randn(20, hk, d, generator=g).bfloat16()
    held = [[np.zeros((0, hk, d))] * 2 for _ in range(events)]

    def stored(x):
        x = x.double().numpy()
        return oracle.kv8_decode(*oracle.kv8_encode(x)) if kv_format == B.KV_FP8 else x

    for step in range(4):
        news = np.array([1 + step, 4, 6 - step])
        plan = cache.plan(news)
        n, nd = int(news.sum()), int((news - 1).sum())
        q, k, v = (torch.randn(n, h, d, generator=g).bfloat16() for h in (hq, hk, hk))
        cache.append(plan, k.cuda(), v.cuda())
        lse = torch.empty(n, hq, device="cuda")
        out = cache.attend(plan, q.cuda(), k_pre.cuda(), v_pre.cuda(), lse=lse)
        p = _tables(g, n, vocab, torch.float32)
        has = torch.cat([torch.arange(m) < m - 1 for m in news])
        dq = torch.softmax(torch.log(p[has] + 1e-9) + 0.8 * torch.randn(nd, vocab, generator=g), -1)
        draft = torch.multinomial(dq, 1, generator=g)[:, 0].to(torch.int32)
        ua, up = torch.rand(nd, generator=g), torch.rand(events, generator=g)
        acc, tok = cache.verify(plan, p.cuda(), dq.cuda(), draft.cuda(), ua.cuda(), up.cuda())
        B.pad_chunk_status(plan)
        out, lse, at, dat = out.double().cpu().numpy(), lse.double().cpu().numpy(), 0, 0
        lens = cache.commit(plan, acc)
        for e, m in enumerate(int(x) for x in news):
            kk = np.concatenate([k_pre.double().numpy(), held[e][0], stored(k[at:at + m])])
            vv = np.concatenate([v_pre.double().numpy(), held[e][1], stored(v[at:at + m])])
            o, l, mag = oracle.chunk_attention(q[at:at + m].double().numpy(), kk, vv, 20 + len(held[e][0]) + 1, d ** -0.5)
            assert np.all(np.abs(out[at:at + m] - o) <= (2.0 ** -8 + 1e-4) * mag) and np.all(np.abs(lse[at:at + m] - l) <= 1e-4)
            a, t = oracle.draft_verify(p[at:at + m].numpy(), dq[dat:dat + m - 1].numpy(), draft[dat:dat + m - 1].tolist(),
                                       ua[dat:dat + m - 1].numpy(), float(up[e]))
            assert (a, t) == (int(acc[e]), int(tok[e]))
            held[e] = [np.concatenate([held[e][i], stored(x[at:at + a + 1])]) for i, x in enumerate((k, v))]
            assert lens[e] == len(held[e][0])
            at, dat = at + m, dat + m - 1
        in_use = cache.pages.n_pages - cache.pages.free_count
        assert in_use == sum((int(x) + page - 1) // page for x in lens)
    plan = cache.plan([0] * events)
    k, v = cache.read(plan)
    assert np.array_equal(k.double().cpu().numpy(), np.concatenate([h[0] for h in held]))
    assert np.array_equal(v.double().cpu().numpy(), np.concatenate([h[1] for h in held]))


def test_the_example_runs():
    from paper_2607_02963_gb300 import speculative
    kept, cache = speculative.example(events=3, drafts=3, steps=3, prefix=200, vocab=500, h_q=8, h_kv=2)
    assert np.array_equal(cache.event_len, np.sum(kept, axis=0)) and all(1 <= k <= 4 for row in kept for k in row)


@pytest.mark.parametrize("fp8", [False, True])
def test_many_launches_in_a_row_agree(fp8):
    """Calls queued back to back, two batches in turn: every pass gives what the first one gave."""
    cases = [Case(40 + i, [30, 200, 3], [5, 40, 1], [400 + 37 * i], [0, 0, 0], 28, 4, 128, 16, fp8).store().device() for i in range(2)]
    plans = [c.plan(out_dtype=1) for c in cases]
    first = [c.attend(p) for c, p in zip(cases, plans)]
    q = [c.q.cuda() for c in cases]
    pre = [(c.k_pre.cuda(), c.v_pre.cuda()) for c in cases]
    outs = [[torch.full_like(o, 7.0) for o in f] for f in first]
    differ = torch.zeros(2, dtype=torch.int64, device="cuda")
    for i in range(600):
        b = i % 2
        B.pad_chunk_attn(plans[b], q[b], *pre[b], *cases[b].dp, *outs[b], *cases[b].ds)
        if i % 50 >= 48:
            differ[b] += (outs[b][0] != first[b][0]).sum() + (outs[b][1] != first[b][1]).sum()
    assert differ.tolist() == [0, 0]
    for p in plans:
        B.pad_chunk_status(p)


@pytest.mark.parametrize("sms", [1, 0])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,h_q,h_kv,page", [(128, 28, 4, 16), (64, 14, 2, 64), (128, 16, 1, 4), (64, 6, 2, 8)])
@pytest.mark.parametrize("what", [0.0, float("nan"), float("inf")])
def test_both_forms_of_the_tcgen05_kernel(what, d, h_q, h_kv, page, fp8, sms):
    # planned for one SM, where fewer CTAs are better, two slots of tokens share a CTA
    lens, news, prefix, video = [700, 2, 0, 129], [70, 150, 0, 43], [301, 5], [0, 0, 1, 1]
    c = Case(31 + d + page, lens, news, prefix, video, h_q, h_kv, d, page, fp8)
    at = 2 + 120  # a private token of branch 1 that its first 120 new tokens do not see
    if what != 0.0:
        c.v[1][at, 0, 3] = what
    c.store().device()
    prob = B.make_problem(h_q, h_kv, d, page, num_sms=sms, flags=B.FLAG_PREFIX_TC)
    fmt = B.KV_FP8 if fp8 else B.KV_BF16
    c.ws = torch.zeros(B.pad_chunk_workspace_size(prob, prefix, video, lens, news, kv_format=fmt), dtype=torch.uint8, device="cuda")
    plan = B.pad_chunk_plan(prob, None, prefix, video, lens, news, page_table=c.dt, n_pages=c.n_pages, kv_format=fmt, workspace=c.ws)
    if sms == 1:
        per = 2 * (128 // (h_q // h_kv))
        assert plan.info()["tc_items"] == sum(-(-n // per) for n in (70, 150, 43, 70 + 150, 43))
    out, lse = c.attend(plan)
    B.pad_chunk_status(plan)
    if what != 0.0:
        rows, group = slice(70 + 120, 70 + 150), h_q // h_kv
        bad = out[rows, :group].float() if fp8 else out[rows, :group, 3].float()
        assert not torch.isfinite(bad).any()
        keep = torch.ones_like(out, dtype=torch.bool)
        if fp8:
            keep[rows, :group] = False  # (a group that holds it reads back as NaN throughout)
        else:
            keep[rows, :group, 3] = False
        assert torch.isfinite(out[keep]).all()
        c.v[1][at, 0, 3] = 0.0
        if fp8:
            return
        o = out.clone()
        o[~keep] = 0.0
        for e in (0, 1, 3):
            a, want, l, mag = c.want(e)
            n = news[e]
            k = keep[a:a + n].cpu().numpy()
            assert np.all((np.abs(o[a:a + n].double().cpu().numpy() - want) <= (2.0 ** -8 + 1e-4) * mag) | ~k)
            assert np.all(np.abs(lse[a:a + n].double().cpu().numpy() - l) <= 1e-4)
        return
    c.check(out, lse)
