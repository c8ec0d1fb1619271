"""The 4-bit cache on the GPU against its fp64 oracle: written, read back, attended to.

Bounds.  The cache: equal, bit for bit (scale and code are one rounding each, of quotients that no tie is near).
Attention: on the warp-level kernel a weight is rounded to f16 (11 significant bits, half a step of which
is 2^-11 of the value at most, or of the subnormals of 2^15 times the weight 2^-25, 2^-40 of the weight), where
the pages are widened to bf16 (2^-8, as in a bf16 cache); 1e-4 sum p |v| more covers scores, exponentials and sums in
fp32 (scores below 32 in magnitude, each within 2^-20 of that); a bf16 output adds 2^-8 of its magnitude.  The lse: 1e-4.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_02963_gb300 import binding as B
from test_gpu_chunk import _SHAPES, Case

pytestmark = pytest.mark.gpu
FLAGS = [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC]


@pytest.fixture(scope="module", autouse=True)
def _cuda(padlib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()


class Case4(Case):
    """Random branches in 4 bits; slots that hold no token read as NaN."""

    def __init__(self, *a, poison=True, **kw):
        super().__init__(*a, **kw)
        shape = (self.n_pages, self.h_kv, self.page)
        self.pools = [torch.full(shape + (self.d // 2,), 0x77, dtype=torch.uint8) for _ in range(2)]
        self.scales = [torch.full(shape + (self.d // 16,), 0xFF if poison else 0, dtype=torch.uint8) for _ in range(2)]

    def store(self, upto=None):
        for e in range(len(self.lens)):
            n = int((self.lens + self.news)[e] if upto is None else upto[e])
            if n == 0:
                continue
            pos = np.arange(n)
            pg, slot = self.table[e, pos // self.page].astype(np.int64), pos % self.page
            for i, x in enumerate((self.k[e], self.v[e])):
                c, b = oracle.kv4_encode(x[:n].double().numpy())
                self.pools[i][pg, :, slot] = torch.from_numpy(c)
                self.scales[i][pg, :, slot] = torch.from_numpy(b)
        return self

    def cached(self, i, e):
        return oracle.kv4_decode(*oracle.kv4_encode((self.k, self.v)[i][e].double().numpy()))

    def plan(self, out_dtype=0, flags=0, cache=None, stream=None, num_sms=0):
        prob = B.make_problem(self.h_q, self.h_kv, self.d, self.page, out_dtype=out_dtype, flags=flags, num_sms=num_sms)
        n = B.pad_chunk_workspace_size(prob, self.prefix, self.video, self.lens, self.news, kv_format=B.KV_FP4)
        self.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        self.ws[:256] = 0
        return B.pad_chunk_plan(prob, cache, self.prefix, self.video, self.lens, self.news, page_table=self.dt,
                                n_pages=self.n_pages, kv_format=B.KV_FP4, workspace=self.ws, stream=stream)

    def bound(self, e, mag, flags):
        """Of the outputs in 32 bits; events whose pages are widened, and those with a prefix, as in bf16."""
        rows = int(self.news[e]) * (self.h_q // self.h_kv)
        wide = flags == B.FLAG_PREFIX_TC or (self.prefix is not None and self.prefix[self.video[e]] > 0) or (flags == 0 and rows > 32)
        return ((2.0 ** -8 if wide else 2.0 ** -11) + 1e-4) * mag

    def check4(self, out, lse, flags, bf16=False):
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for e in range(len(self.lens)):
            at, o, l, mag = self.want(e)
            n = int(self.news[e])
            tol = self.bound(e, mag, flags) + 2.0 ** -40 * 1e4
            if bf16:
                tol = tol + 2.0 ** -8 * (np.abs(o) + tol)
            assert np.all(np.abs(out[at:at + n] - o) <= tol), f"event {e}: {np.max(np.abs(out[at:at + n] - o) - tol)}"
            assert np.all(np.abs(lse[at:at + n] - l) <= 1e-4)


# ---------------------------------------------------------------------- written and read


def _groups():
    """Groups of every kind: all maxima of eight bits around scales' ties, codes' ties, subnormal scales, saturation, zeros,
    what is not finite."""
    r = np.random.default_rng(3)
    top = torch.arange(0x3000, 0x7F80, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()   # 4e-10 up
    fill = torch.from_numpy(r.uniform(-1, 1, size=(len(top), 15))).float()
    x = torch.cat([top[:, None], fill * top[:, None]], 1)
    ties = torch.tensor([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -0.0])
    scaled = torch.from_numpy(oracle.kv4_scales()[1:]).float()[:, None] * ties
    near = torch.stack([torch.nextafter(torch.zeros(16), ties), ties * (1 + 2 ** -7), ties * (1 - 2 ** -8)])
    near = torch.cat([torch.full((3, 1), 6.0), near[:, 1:]], 1)
    special = torch.zeros(6, 16)
    special[1, 3], special[2, 15], special[3, 0], special[4, 7], special[5] = float("nan"), float("inf"), -float("inf"), -1e-30, 3e38
    return torch.cat([x, scaled, near, special]).bfloat16()


@pytest.mark.parametrize("d,page", [(128, 16), (64, 64), (128, 4), (64, 8)])
def test_written_and_read_back_bit_for_bit(d, page):
    x = _groups()
    h = 2
    per = h * d // 16
    x = torch.cat([x, torch.zeros(-len(x) % per, 16, dtype=torch.bfloat16)]).view(-1, h, d)
    n = len(x)
    c = Case4(1, [3, 0], [n, 5], None, None, 4, h, d, page)
    c.k[0][3:], c.v[0][3:] = x, x.flip(0)
    want = Case4(1, [3, 0], [n, 5], None, None, 4, h, d, page)
    want.k, want.v = c.k, c.v
    want.store()
    c.store(c.lens).device()
    plan = c.plan()
    new = [torch.cat([t[0][3:], t[1]]).cuda() for t in (c.k, c.v)]
    B.pad_chunk_append(plan, *new, *c.dp, *c.ds)
    B.pad_chunk_status(plan)
    for i in range(2):
        got, ref = c.dp[i].cpu(), want.pools[i]
        zero = torch.from_numpy(oracle.kv4_scales()[np.minimum(want.scales[i].numpy(), 226)] == 0).repeat_interleave(8, -1)
        assert torch.equal(c.ds[i].cpu(), want.scales[i])
        assert torch.equal(got[~zero], ref[~zero])
        assert not (got[zero] & 0x77).any()   # (signs of zeros)
    out = [torch.full((plan.n_cached, h, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.pad_chunk_read(plan, *c.dp, *out, *c.ds)
    for i in range(2):
        ref = np.concatenate([c.cached(i, e) for e in range(2)])
        assert np.array_equal(out[i].double().cpu().numpy(), ref, equal_nan=True)


def test_rows_of_a_wider_tensor_and_a_page_outside_the_pool():
    c = Case4(2, [5, 20], [14, 3], None, None, 8, 2, 128, 16)
    c.store(c.lens).device()
    c.dt[0, 1] = c.n_pages
    plan = c.plan()
    wide = torch.full((17, 1024), float("nan"), dtype=torch.bfloat16, device="cuda")
    k, v = wide[:, 8:264].unflatten(1, (2, 128)), wide[:, 512:768].unflatten(1, (2, 128))
    k.copy_(torch.cat([c.k[0][5:], c.k[1][20:]])), v.copy_(torch.cat([c.v[0][5:], c.v[1][20:]]))
    before = [x.clone() for x in c.dp + c.ds]
    B.pad_chunk_append(plan, k, v, *c.dp, *c.ds)
    with pytest.raises(B.PadError, match="DEVICE_BOUNDS"):
        B.pad_chunk_status(plan)
    c.store()
    hit = torch.zeros(c.n_pages, dtype=torch.bool)
    hit[c.table[0, 0]] = hit[c.table[1, 1]] = True
    for got, old, ref in zip(c.dp + c.ds, before, c.pools + c.scales):
        assert torch.equal(got.cpu()[hit], ref[hit]) and torch.equal(got.cpu()[~hit], old.cpu()[~hit])
    out = [torch.full((plan.n_cached, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.pad_chunk_read(plan, *c.dp, *out, *c.ds)
    assert not out[0][16:19].any() and np.array_equal(out[0][:16].double().cpu().numpy(), c.cached(0, 0)[:16])


# ------------------------------------------------------------------------------ attention


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("d,h_q,h_kv,page", [(128, 28, 4, 16), (64, 14, 2, 64), (128, 16, 1, 4), (64, 3, 3, 8),
                                             (128, 4, 2, 32)])
def test_attention(d, h_q, h_kv, page, flags):
    for i, (lens, news, prefix, video) in enumerate(_SHAPES):
        c = Case4(100 * i + d + page, lens, news, prefix, video, h_q, h_kv, d, page).store().device()
        bf16 = (i + page) % 2 == 0
        plan = c.plan(out_dtype=1 if bf16 else 0, flags=flags)
        out, lse = c.attend(plan)
        c.check4(out, lse, flags, bf16)
        B.pad_chunk_status(plan)
        out2, lse2 = c.attend(plan)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("rows", [1, 5, 8, 9, 16, 17, 24, 25, 32, 33, 47, 60])
@pytest.mark.parametrize("d", [64, 128])
def test_every_count_of_rows(d, rows):
    """Group 1: rows are tokens, in one to four groups of eight and in pieces."""
    c = Case4(rows, [50, 131], [rows, max(1, rows // 3)], None, None, 2, 2, d, 16).store().device()
    c.check4(*c.attend(c.plan(flags=B.FLAG_PREFIX_MMA)), B.FLAG_PREFIX_MMA)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("d,lens,news,prefix", [(128, [5000, 3], [1, 1], None), (64, [2500], [17], None),
                                                (128, [64, 10, 0], [5, 2, 8], [3001]), (128, [9000], [40], None)])
def test_attention_over_split_keys(d, lens, news, prefix, flags):
    c = Case4(7, lens, news, prefix, None if prefix is None else [0] * len(lens), 8, 2, d, 16).store().device()
    plan = c.plan(flags=flags)
    i = plan.info()
    assert max(i["page_splits"], i["prefix_splits"]) > 1
    c.check4(*c.attend(plan), flags)
    B.pad_chunk_status(plan)


@pytest.mark.parametrize("flags", FLAGS)
def test_large_scores_and_a_key_that_dominates(flags):
    """Scores that span hundreds, rising along the keys: every block moves the running maximum."""
    c = Case4(8, [700, 30], [3, 40], [300], [0, 0], 8, 2, 128, 16)
    c.q = (4.0 * c.q.float()).bfloat16()
    for e in range(2):
        ramp = torch.linspace(0.1, 2.0, c.k[e].shape[0])[:, None, None]
        c.k[e] = (c.k[e].float() * ramp).bfloat16()
    c.store().device()
    out, lse = (x.double().cpu().numpy() for x in c.attend(c.plan(flags=flags)))
    for e in range(2):
        at, o, l, mag = c.want(e)
        n = int(c.news[e])
        # scores up to 256 in magnitude, each within 2^-20 of that
        assert np.all(np.abs(out[at:at + n] - o) <= (2.0 ** -8 + 1e-3) * mag)
        assert np.all(np.abs(lse[at:at + n] - l) <= 1e-3)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("d", [64, 128])
def test_values_and_queries_at_the_ends_of_their_range(d, flags):
    """V from 2^-16 to 2^15 by token, queries from 2^-100 to 2^90 by row (K the other way round): what a weight of 2^-28
    and more meets is exact to the weight's rounding."""
    c = Case4(14, [200, 15], [2, 3], None, None, 8, 2, d, 16)
    for e in range(2):
        n = c.v[e].shape[0]
        size = torch.tensor([2.0 ** -16, 1.0, 2.0 ** 13])[torch.arange(n) % 3]
        c.v[e] = (c.v[e].float() * size[:, None, None]).bfloat16()
        c.k[e] = (c.k[e].float() * 2.0 ** -8).bfloat16()
    size = torch.tensor([2.0 ** 8, 2.0 ** -100, 2.0 ** 4, 2.0 ** -7])
    c.q = (c.q.float() * size[torch.arange(c.q.shape[0] * 8) % 4].view(-1, 8, 1)).bfloat16()
    c.store().device()
    out, lse = (x.double().cpu().numpy() for x in c.attend(c.plan(flags=flags)))
    for e in range(2):
        at, o, l, mag = c.want(e)
        n = int(c.news[e])
        assert np.all(np.abs(out[at:at + n] - o) <= c.bound(e, mag, flags) + 2.0 ** -40 * 220 * 2.0 ** 16)
        assert np.all(np.abs(lse[at:at + n] - l) <= 1e-4)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("where", ["k", "v"])
def test_what_is_not_finite_stays_with_the_tokens_that_see_it(where, flags):
    """A later chunk token's group holds a NaN: the tokens before it do not notice, it and those after it do."""
    def make():
        return Case4(9, [20, 37], [6, 5], None, None, 8, 2, 128, 16)

    c, clean = make(), make()
    (c.k if where == "k" else c.v)[0][23, 1, 37] = float("inf")   # chunk token 3 of event 0, kv-head 1, group 2
    c.store().device()
    out, lse = c.attend(c.plan(flags=flags))
    out = out.double().cpu().numpy()
    for e in range(2):
        at, o, l, mag = clean.want(e)
        bad = np.zeros(o.shape, bool)
        if e == 0:
            bad[3:, 4:, slice(None) if where == "k" else slice(32, 48)] = True   # query heads 4-7 read kv-head 1
        got = out[at:at + len(o)]
        assert np.isnan(got[bad]).all()
        assert np.all((np.abs(got - o) <= clean.bound(e, mag, flags)) | bad)


@pytest.mark.parametrize("flags", FLAGS)
def test_pages_outside_the_pool_hide_their_tokens(flags):
    c = Case4(11, [40, 3], [2, 1], None, None, 8, 2, 128, 16).store().device()
    c.dt[0, 1], c.dt[1, 0] = c.n_pages + 3, -1
    plan = c.plan(flags=flags)
    out, lse = (x.double().cpu().numpy() for x in c.attend(plan))
    with pytest.raises(B.PadError, match="DEVICE_BOUNDS"):
        B.pad_chunk_status(plan)
    k, v = (np.delete(c.cached(i, 0), np.arange(16, 32), axis=0) for i in range(2))
    o, l, mag = oracle.chunk_attention(c.q[:2].double().numpy(), k, v, 40 + 1 - 16, 1 / 128 ** 0.5)
    assert np.all(np.abs(out[:2] - o) <= c.bound(0, mag, flags) + 1e-8) and np.all(np.abs(lse[:2] - l) <= 1e-4)
    assert not out[2].any() and np.all(lse[2] == -np.inf)


@pytest.mark.parametrize("flags", FLAGS)
def test_calls_in_a_row_and_a_graph_on_another_stream(flags):
    """Append and attention captured once on a stream of their own, replayed with other contents."""
    lens, news = [40, 500, 0], [5, 40, 1]
    cs = [Case4(80 + i, lens, news, [300], [0, 0, 0], 28, 4, 128, 16).store(lens).device() for i in range(3)]
    for o in cs[1:]:
        o.table = cs[0].table
        o.pools, o.scales = [torch.zeros_like(x) for x in o.pools], [torch.full_like(x, 255) for x in o.scales]
        o.store(lens)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        plan = cs[0].plan(flags=flags)
        new = [slice(a, a + b) for a, b in zip(lens, news)]
        sets = [[x.cuda() for x in [o.q, *(torch.cat([x[e][new[e]] for e in range(3)]) for x in (o.k, o.v)), o.k_pre, o.v_pre,
                                    *o.pools, *o.scales]] for o in cs]
        buf = [x.clone() for x in sets[0]]
        out, lse = torch.empty(46, 28, 128, device="cuda"), torch.empty(46, 28, device="cuda")

        def step():
            q, k, v, kp, vp, kc, vc, ks, vs = buf
            B.pad_chunk_append(plan, k, v, kc, vc, ks, vs)
            B.pad_chunk_attn(plan, q, kp, vp, kc, vc, out, lse, ks, vs)

        def load(i):
            for b, x in zip(buf, sets[i]):
                b.copy_(x)
            out.fill_(7), lse.fill_(7)

        want = []
        for i in range(3):
            load(i)
            step()
            want.append((out.clone(), lse.clone()))
            cs[i].check4(out, lse, flags)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for i in (1, 2, 0, 1):
            load(i)
            graph.replay()
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
    B.pad_chunk_status(plan, stream=s)
