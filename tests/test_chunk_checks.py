"""What the binding of the multi-token step refuses before anything is launched.  No GPU: plans without a workspace,
which the library itself does not launch, and tensors that only claim to be on one."""
import pytest
import torch

from paper_2607_02963_gb300 import binding as B


class OnGpu(torch.Tensor):
    """A host tensor that passes for one in device memory."""
    is_cuda = True


def _zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def _plan(news=(3, 2), lens=(5, 0), **kw):
    prob = B.make_problem(8, 2, 64, 16, num_sms=152)
    table = torch.full((len(news), 4), -1, dtype=torch.int32)
    return B.pad_chunk_plan(prob, None, kw.pop("prefix_len", None), kw.pop("event_video", None), lens, news, page_table=table,
                            n_pages=9, **kw)


def _pools():
    return _zeros(9, 2, 16, 64), _zeros(9, 2, 16, 64)


def _attn(plan, q=None, k_prefix=None, v_prefix=None, pools=None, out=None, **kw):
    n = plan.n_tokens
    B.pad_chunk_attn(plan, _zeros(n, 8, 64) if q is None else q, k_prefix, v_prefix, *(pools or _pools()),
                     _zeros(n, 8, 64, dtype=torch.float32) if out is None else out, stream=0, **kw)


def _verify(plan, p=None, q=None, **kw):
    a = dict(draft=_zeros(plan.n_drafts, dtype=torch.int32), u_accept=_zeros(plan.n_drafts, dtype=torch.float32),
             u_pick=_zeros(plan.n_events, dtype=torch.float32), accepted=_zeros(plan.n_events, dtype=torch.int32),
             token=_zeros(plan.n_events, dtype=torch.int32)) | kw
    B.pad_draft_verify(plan, _zeros(plan.n_tokens, 50, dtype=torch.float32) if p is None else p,
                       _zeros(plan.n_drafts, 50, dtype=torch.float32) if q is None else q, stream=0, **a)


def test_what_passes_reaches_the_library(padlib):
    """The checks' other side: the same calls with nothing wrong end in the library's own refusal of a host-only plan."""
    plan = _plan()
    for call in (lambda: _attn(plan), lambda: _verify(plan)):
        with pytest.raises(B.PadError, match="host-only"):
            call()


@pytest.mark.parametrize("rows", [1, 2])
def test_rows_that_overlap_are_refused(padlib, rows):
    """A broadcast tensor has a row stride of 0, which stands for packed rows in the library: n rows would be read
    from the memory of one."""
    plan = _plan()
    n, nd = plan.n_tokens, plan.n_drafts

    def lap(*shape, dtype=torch.bfloat16):
        """Rows that start 0 elements apart, or one."""
        wide = _zeros(4 * shape[0] * max(shape), *shape[1:], dtype=dtype)
        return wide.as_strided(shape, (rows - 1,) + wide.stride()[1:])

    with pytest.raises(ValueError, match="q: .*overlap"):
        _attn(plan, q=lap(n, 8, 64))
    x = _zeros(n, 2, 64)
    with pytest.raises(ValueError, match="k_new: .*overlap"):
        B.pad_chunk_append(plan, lap(n, 2, 64), x, *_pools(), stream=0)
    with pytest.raises(ValueError, match="v_new: .*overlap"):
        B.pad_chunk_append(plan, x, lap(n, 2, 64), *_pools(), stream=0)
    for dtype in (torch.float32, torch.bfloat16):
        with pytest.raises(ValueError, match="p: .*overlap"):
            _verify(plan, p=lap(n, 50, dtype=dtype), q=_zeros(nd, 50, dtype=dtype))
        with pytest.raises(ValueError, match="q: .*overlap"):
            _verify(plan, p=_zeros(n, 50, dtype=dtype), q=lap(nd, 50, dtype=dtype))


def test_one_row_may_be_broadcast(padlib):
    """A single row has no next one."""
    plan = _plan(news=(1,), lens=(5,))
    q = _zeros(1, 8, 64)
    with pytest.raises(B.PadError, match="host-only"):
        _attn(plan, q=q.expand(1, 8, 64).as_strided((1, 8, 64), (0, 64, 1)))


def test_a_prefix_shorter_than_the_plans_is_refused(padlib):
    """The kernels read k_prefix as far as the plan's last prefix token, whatever the tensor holds."""
    def pre(n):
        return _zeros(n, 2, 64)

    for kw, need in ((dict(prefix_len=[40], event_video=[0, 0]), 40), (dict(prefix_len=[40, 7], event_video=[0, 1]), 47),
                     (dict(prefix_len=[40, 7], event_video=[0, 1], prefix_offset=[100, 3]), 140),
                     # a video whose branches bring no token is not read
                     (dict(prefix_len=[40, 7], event_video=[0, 1], news=(3, 0)), 40),
                     (dict(prefix_len=[0, 0], event_video=[0, 1]), 0)):
        plan = _plan(**kw)
        assert plan.info()["prefix_tokens"] == need
        for n in (need, need + 5):
            with pytest.raises(B.PadError, match="host-only"):
                _attn(plan, k_prefix=pre(n), v_prefix=pre(n))
        for n in {0, need - 1} - {-1, need}:
            with pytest.raises(ValueError, match=f"k_prefix: {n} tokens, the plan reads {need}"):
                _attn(plan, k_prefix=pre(n), v_prefix=pre(n))
            with pytest.raises(ValueError, match="v_prefix"):
                _attn(plan, k_prefix=pre(need), v_prefix=pre(n))


def test_host_tensors_are_refused(padlib):
    """A host tensor's address is not for the kernels: every tensor of every call."""
    plan = _plan(prefix_len=[20], event_video=[0, 0])
    n, nd, ne, f32, i32 = plan.n_tokens, plan.n_drafts, plan.n_events, torch.float32, torch.int32
    t = dict(q=_zeros(n, 8, 64), k_prefix=_zeros(20, 2, 64), v_prefix=_zeros(20, 2, 64), k_pool=_pools()[0], v_pool=_pools()[1],
             out=_zeros(n, 8, 64, dtype=f32), lse=_zeros(n, 8, dtype=f32), k_new=_zeros(n, 2, 64), v_new=_zeros(n, 2, 64),
             k_out=_zeros(plan.n_cached, 2, 64), v_out=_zeros(plan.n_cached, 2, 64), p=_zeros(n, 50, dtype=f32),
             dq=_zeros(nd, 50, dtype=f32), draft=_zeros(nd, dtype=i32), u_accept=_zeros(nd, dtype=f32),
             u_pick=_zeros(ne, dtype=f32), accepted=_zeros(ne, dtype=i32), token=_zeros(ne, dtype=i32))
    calls = {"attn": (B.pad_chunk_attn, ("q", "k_prefix", "v_prefix", "k_pool", "v_pool", "out", "lse")),
             "append": (B.pad_chunk_append, ("k_new", "v_new", "k_pool", "v_pool")),
             "read": (B.pad_chunk_read, ("k_pool", "v_pool", "k_out", "v_out")),
             "verify": (B.pad_draft_verify, ("p", "dq", "draft", "u_accept", "u_pick", "accepted", "token"))}
    for call, names in calls.values():
        with pytest.raises(B.PadError, match="host-only"):
            call(plan, *(t[x] for x in names), stream=0)
        for bad in names:
            host = torch.zeros(t[bad].shape, dtype=t[bad].dtype)
            with pytest.raises(ValueError, match=f"{'q' if bad == 'dq' else bad}: .*device memory"):
                call(plan, *(host if x == bad else t[x] for x in names), stream=0)
    # rows of a wider tensor, and the 8-bit cache's scales
    wide = torch.zeros(n, 1024, dtype=torch.bfloat16)[:, :512].unflatten(1, (8, 64))
    with pytest.raises(ValueError, match="q: .*device memory"):
        _attn(plan, q=wide, k_prefix=t["k_prefix"], v_prefix=t["v_prefix"])
    plan = _plan(kv_format=B.KV_FP8)
    pools, u8 = [_zeros(9, 2, 16, 64, dtype=torch.uint8) for _ in range(2)], torch.uint8
    for bad in range(2):
        scales = [torch.zeros(9, 2, 16, dtype=u8) if i == bad else _zeros(9, 2, 16, dtype=u8) for i in range(2)]
        with pytest.raises(ValueError, match="[kv]_scale: .*device memory"):
            B.pad_chunk_append(plan, t["k_new"], t["v_new"], *pools, *scales, stream=0)


def test_host_workspaces_and_page_tables_are_refused(padlib):
    prob = B.make_problem(8, 2, 64, 16, num_sms=152)
    size = B.pad_chunk_workspace_size(prob, None, None, [5], [3])
    ws, table = torch.zeros(size + 256, dtype=torch.uint8), torch.full((1, 4), -1, dtype=torch.int32)
    with pytest.raises(ValueError, match="workspace: .*device memory"):
        B.pad_chunk_plan(prob, None, None, None, [5], [3], page_table=table.as_subclass(OnGpu), n_pages=4, workspace=ws, stream=0)
    with pytest.raises(ValueError, match="page_table: .*device memory"):
        B.pad_chunk_plan(prob, None, None, None, [5], [3], page_table=table, n_pages=4, workspace=ws.as_subclass(OnGpu), stream=0)


def test_more_cached_tokens_than_a_read_has_ctas_for_are_refused(padlib):
    """pad_chunk_read copies spans of 32 tokens, a CTA each: 2^31 of them and more are no grid."""
    prob = B.make_problem(1, 1, 64, 64, num_sms=152)
    most = [1 << 30] * 63 + [(1 << 30) - 32]           # 2^31 - 1 spans
    assert B.pad_chunk_plan(prob, None, None, None, most, [0] * 64).n_cached == 2 ** 36 - 32
    lens = [1 << 30] * 63 + [(1 << 30) - 64] + [1] * 31  # fewer tokens, more spans
    for call in (lambda: B.pad_chunk_plan(prob, None, None, None, lens, [0] * 95),
                 lambda: B.pad_chunk_workspace_size(prob, None, None, lens, [0] * 95)):
        with pytest.raises(B.PadError, match="too many tokens"):
            call()
