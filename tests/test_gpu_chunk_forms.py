"""Chunk attention: both forms of the tcgen05 kernel against the oracle with a value that is not finite in a hidden
place, calls in a row on one workspace, and calls captured in a graph.  Bounds as in test_gpu_chunk.py."""
import numpy as np
import pytest
import torch

from paper_2607_02963_gb300 import binding as B
from test_gpu_chunk import Case, _tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(padlib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()


def _plan(c, **kw):
    prob = B.make_problem(c.h_q, c.h_kv, c.d, c.page, **kw)
    fmt = B.KV_FP8 if c.fp8 else B.KV_BF16
    c.ws = torch.zeros(B.pad_chunk_workspace_size(prob, c.prefix, c.video, c.lens, c.news, kv_format=fmt), dtype=torch.uint8,
                       device="cuda")
    return B.pad_chunk_plan(prob, None, c.prefix, c.video, c.lens, c.news, page_table=c.dt, n_pages=c.n_pages, kv_format=fmt,
                            workspace=c.ws)


@pytest.mark.parametrize("slots", [1, 2])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d,h_q,h_kv,page", [(128, 28, 4, 16), (64, 14, 2, 64), (128, 16, 1, 4), (64, 6, 2, 8)])
@pytest.mark.parametrize("what", [0.0, float("nan"), float("inf")])
def test_each_form_in_every_row_that_does_not_see_it(what, d, h_q, h_kv, page, fp8, slots):
    """Planned for one SM two slots of tokens share a CTA, for as many SMs as slots each has its own."""
    group, length = h_q // h_kv, 640
    per, n = 128 // group, 150 if group > 3 else 170  # (a last slot that is not full)
    c = Case(60 + d + page, [length], [n], None, None, h_q, h_kv, d, page, fp8)
    at = 100  # the chunk token whose value it is
    c.v[0][length + at, 0, 3] = what
    c.store().device()
    c.v[0][length + at, 0, 3] = 0.0
    plan = _plan(c, num_sms=1 if slots == 2 else -(-n // per) * h_kv, flags=B.FLAG_PREFIX_TC)
    assert plan.info()["page_splits"] == 1 and plan.info()["tc_items"] == -(-n // (slots * per))
    out, lse = c.attend(plan)
    B.pad_chunk_status(plan)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    hole = np.zeros(out.shape, bool)
    if fp8:
        hole[at:, :group] = True  # (a group that holds it reads back as NaN throughout)
    else:
        hole[at:, :group, 3] = True
    _, o, l, mag = c.want(0)
    if what == 0.0:
        hole[:] = False
    assert not np.isfinite(out[hole]).any()
    assert np.all((np.abs(out - o) <= (2.0 ** -8 + 1e-4) * mag) | hole)
    assert np.all(np.abs(lse - l) <= 1e-4)


@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC])
@pytest.mark.parametrize("fp8", [False, True])
def test_calls_in_a_row_on_one_workspace(fp8, flags):
    """Two sets of queries in turn on one plan: its partial states are the other set's until they are written anew, so a
    join that came before them would show; outputs are refilled before every pair of calls, and every pass is compared."""
    c = Case(70, [30, 200, 3], [5, 40, 1], [437], [0, 0, 0], 28, 4, 128, 16, fp8).store().device()
    plan = _plan(c, out_dtype=1, flags=flags)
    assert plan.info()["partial_rows"] > 0
    pre = (c.k_pre.cuda(), c.v_pre.cuda())
    q = [c.q.cuda(), (-c.q).cuda()]
    want = [c.attend(plan, x) for x in q]
    c.check(*want[0], bf16=True)
    assert not torch.equal(want[0][0], want[1][0])
    got = [[torch.empty_like(x) for x in w] for w in want]
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        for x in got[0] + got[1]:
            x.fill_(7.0)
        for b in range(2):
            B.pad_chunk_attn(plan, q[b], *pre, *c.dp, *got[b], *c.ds)
        for b in range(2):
            for x, w in zip(got[b], want[b]):
                differ += (x != w).sum()
    assert int(differ) == 0
    B.pad_chunk_status(plan)


@pytest.mark.parametrize("fp8", [False, True])
def test_a_steps_calls_in_a_graph(fp8):
    """Append, attention and verification captured once and replayed with other contents in the same buffers."""
    vocab, lens, news = 300, [40, 500, 0], [5, 40, 1]
    cases = [Case(80 + i, lens, news, [300], [0, 0, 0], 28, 4, 128, 16, fp8).store(lens).device() for i in range(3)]
    c = cases[0]
    for o in cases[1:]:                     # (one placement of the pages for all)
        o.table = c.table
        o.pools = [torch.zeros_like(x) for x in o.pools]
        o.store(lens).device()
    plan = _plan(c)
    n, nd, ne = plan.n_tokens, plan.n_drafts, 3
    g = torch.Generator().manual_seed(4)

    def contents(o):
        new = [slice(a, a + b) for a, b in zip(lens, news)]
        k, v = (torch.cat([x[e][new[e]] for e in range(3)]) for x in (o.k, o.v))
        p = _tables(g, n, vocab, torch.float32)
        dq = torch.softmax(torch.log(p[:nd]) + 0.5 * torch.randn(nd, vocab, generator=g), -1)
        return [o.q, k, v, o.k_pre, o.v_pre, *o.pools, *(x for x in o.scales if x is not None), p, dq,
                torch.randint(0, vocab, (nd,), generator=g).int(), torch.rand(nd, generator=g), torch.rand(ne, generator=g)]

    sets = [[x.cuda() for x in contents(o)] for o in cases]
    buf = [x.clone() for x in sets[0]]
    out, lse = torch.empty(n, 28, 128, device="cuda"), torch.empty(n, 28, device="cuda")
    acc, tok = (torch.empty(ne, dtype=torch.int32, device="cuda") for _ in range(2))

    def step():
        q, k, v, kp, vp, *pools = buf[:9 if fp8 else 7]
        kpool, vpool, ks, vs = pools if fp8 else (*pools, None, None)
        p, dq, draft, ua, up = buf[-5:]
        B.pad_chunk_append(plan, k, v, kpool, vpool, ks, vs)
        B.pad_chunk_attn(plan, q, kp, vp, kpool, vpool, out, lse, ks, vs)
        B.pad_draft_verify(plan, p, dq, draft, ua, up, acc, tok)

    def load(i):
        for b, x in zip(buf, sets[i]):
            b.copy_(x)
        for x in (out, lse, acc, tok):
            x.fill_(7)

    want = []
    for i in range(3):
        load(i)
        step()
        want.append([x.clone() for x in (out, lse, acc, tok)])
        cases[i].check(out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (1, 2, 0, 1):
        load(i)
        graph.replay()
        for x, w in zip((out, lse, acc, tok), want[i]):
            assert torch.equal(x, w)
    B.pad_chunk_status(plan)
