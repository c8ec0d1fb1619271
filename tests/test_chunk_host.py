"""Host side of the multi-token step: page allocation and return, refusals, and the pins of its fp64 oracle.
No GPU: plans without a workspace."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from paper_2607_02963_gb300 import binding as B


def _prob(**kw):
    a = dict(h_q=28, h_kv=4, head_dim=128, page_size=16, num_sms=152)
    a.update(kw)
    return B.make_problem(**a)


def _table(events, pages=64):
    return torch.full((events, pages), -1, dtype=torch.int32)


# ------------------------------------------------------------------------------ oracle pins


def test_e4m3_table_is_torchs():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    want = oracle.e4m3_values()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    assert np.array_equal(got[fine], want[fine])


def test_encode_is_the_nearest_code_and_the_smallest_scale():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((64, 64)) * 2.0 ** rng.integers(-20, 10, size=(64, 1))
    codes, byte = oracle.kv8_encode(x)
    back = oracle.kv8_decode(codes, byte)
    vals = oracle.e4m3_values()
    vals = vals[~np.isnan(vals)]
    for row, got, b in zip(x, back, byte):
        k = int(b) - 127
        assert np.max(np.abs(row)) <= 448 * 2.0 ** k and (k == -120 or np.max(np.abs(row)) > 448 * 2.0 ** (k - 1))
        best = np.min(np.abs(row[:, None] - vals[None, :] * 2.0 ** k), axis=1)
        assert np.array_equal(np.abs(row - got), best)
    # a code is within a sixteenth of its value
    big = np.abs(x) > 448 * 2.0 ** (byte.astype(float)[:, None] - 127) * 2.0 ** -14
    assert np.all(np.abs(back - x)[big] <= np.abs(x)[big] / 16)


def test_encode_of_special_groups():
    z, n, s = np.zeros((1, 64)), np.ones((1, 64)), np.full((1, 64), 1e6)
    n[0, 3] = np.nan
    assert oracle.kv8_encode(z)[1][0] == 0 and not oracle.kv8_decode(*oracle.kv8_encode(z)).any()
    assert oracle.kv8_encode(n)[1][0] == 255 and np.all(np.isnan(oracle.kv8_decode(*oracle.kv8_encode(n))))
    assert np.all(oracle.kv8_decode(*oracle.kv8_encode(s)) == 57344.0)


def test_chunk_attention_is_the_decode_steps_definition_token_by_token():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    out, lse, mag = oracle.chunk_attention(q, k, v, 7, 0.3)
    for t in range(3):
        kk = torch.from_numpy(np.repeat(k[:7 + t], 2, axis=1)).permute(1, 0, 2)
        vv = torch.from_numpy(np.repeat(v[:7 + t], 2, axis=1)).permute(1, 0, 2)
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[t])[:, None], kk, vv, scale=0.3)
        assert np.allclose(out[t], want[:, 0].numpy(), atol=1e-12)
    assert np.all(mag >= np.abs(out) - 1e-12)


def test_verification_returns_tokens_distributed_as_the_target():
    """One drafted token drawn from q, then the rule: over a grid of the uniforms the first token's
    frequencies are p (within the grid's step)."""
    p = np.array([[0.5, 0.25, 0.125, 0.125], [1, 0, 0, 0]], dtype=np.float32)
    q = np.array([[0.25, 0.25, 0.5, 0.0]], dtype=np.float32)
    steps = 64
    freq = np.zeros(4)
    for x in range(4):
        for i in range(steps):
            for j in range(steps):
                a, tok = oracle.draft_verify(p, q, [x], [(i + 0.5) / steps], (j + 0.5) / steps)
                freq[x if a == 1 else tok] += q[0, x] / steps ** 2
    assert np.abs(freq - p[0]).max() <= 2.0 / steps


def test_verification_edges():
    p = np.array([[0.5, 0.5], [0.25, 0.75]], dtype=np.float32)
    assert oracle.draft_verify(p, p[:1], [0], [0.999], 0.0) == (1, 0)
    assert oracle.draft_verify(p, p[:1], [0], [0.999], 0.9) == (1, 1)
    zero = np.zeros((1, 3), dtype=np.float32)
    assert oracle.draft_verify(zero, zero[:0], [], [], 0.5) == (0, -1)
    # nothing left of the difference: p itself
    assert oracle.draft_verify(np.array([[0.0, 0.5], [0, 1]], np.float32), np.array([[0.5, 0.5]], np.float32), [0], [0.0], 0.0) == (0, 1)


# ------------------------------------------------------------------------------ pages


def test_pages_are_the_lowest_free_ones_in_event_order(padlib):
    cache = B.CacheState(32, used_pages=[0, 2, 5])
    lens, news = [15, 16, 0, 33], [2, 1, 40, 0]
    plan = B.pad_chunk_plan(_prob(), cache, [100], [0, 0, 0, 0], lens, news, page_table=_table(4))
    ev, col, pg = plan.new_pages()
    # event 0 starts column 1, event 1 column 1, event 2 columns 0-2, event 3 none
    assert ev.tolist() == [0, 1, 2, 2, 2] and col.tolist() == [1, 1, 0, 1, 2] and pg.tolist() == [1, 3, 4, 6, 7]
    assert cache.free_count == 32 - 3 - 5
    i = plan.info()
    assert i["n_tokens"] == 43 and i["n_cached"] == sum(lens) + 43 and i["n_drafts"] == 1 + 0 + 39


def test_commit_keeps_what_was_accepted_and_returns_the_rest(padlib):
    cache = B.CacheState(16)
    prob = _prob(page_size=4)
    lens, news = [3, 4, 0], [6, 6, 0]
    plan = B.pad_chunk_plan(prob, cache, None, None, lens, news, page_table=_table(3))
    _, _, pg = plan.new_pages()
    assert pg.tolist() == [0, 1, 2, 3] and cache.free_count == 12       # columns 1, 2 and 1, 2
    new = plan.commit(cache, [0, 9, 5])
    # event 0 keeps one token (position 3, its old page), event 1 all six, event 2 had none
    assert new.tolist() == [4, 10, 0]
    assert cache.free_pages()[:2].tolist() == [0, 1] and cache.free_count == 14
    with pytest.raises(B.PadError):
        plan.commit(cache, [0, 0, 0])                                   # once only
    again = B.pad_chunk_plan(prob, cache, None, None, new, [1, 0, 0], page_table=_table(3))
    assert again.new_pages()[2].tolist() == [0]


def test_commit_checks_before_it_changes(padlib):
    cache = B.CacheState(16)
    plan = B.pad_chunk_plan(_prob(page_size=4), cache, None, None, [0], [9], page_table=_table(1))
    with pytest.raises(B.PadError):
        plan.commit(cache, [-1])
    with pytest.raises(B.PadError):
        plan.commit(None, [0])
    assert cache.free_count == 13
    assert plan.commit(cache).tolist() == [9] and cache.free_count == 13


def test_out_of_pages_takes_none(padlib):
    cache = B.CacheState(3)
    with pytest.raises(B.PadError) as e:
        B.pad_chunk_plan(_prob(), cache, None, None, [0, 16], [33, 17], page_table=_table(2))
    assert e.value.status == 3 and cache.free_count == 3


def test_page_allocation_matches_a_simulation(padlib):
    rng = np.random.default_rng(3)
    for _ in range(20):
        ps, n = int(rng.choice([4, 8, 16, 32, 64])), int(rng.integers(1, 9))
        lens, news = rng.integers(0, 70, n), rng.integers(0, 70, n)
        used = rng.choice(400, size=int(rng.integers(0, 200)), replace=False)
        cache = B.CacheState(400, used_pages=used)
        free = sorted(set(range(400)) - set(int(u) for u in used))
        plan = B.pad_chunk_plan(_prob(page_size=ps), cache, None, None, lens, news, page_table=_table(n))
        want = [(e, c) for e in range(n) for c in range((lens[e] + ps - 1) // ps, (lens[e] + news[e] + ps - 1) // ps)]
        ev, col, pg = plan.new_pages()
        assert list(zip(ev.tolist(), col.tolist())) == want and pg.tolist() == free[:len(want)]


# ------------------------------------------------------------------------------ refusals


@pytest.mark.parametrize("change,status", [
    (dict(kv_format=2), 1), (dict(event_len=[-1]), 1), (dict(n_new=[-1]), 1), (dict(n_new=[(1 << 30) + 1]), 1),
    (dict(event_video=[1]), 1), (dict(prefix_len=[-1]), 1), (dict(flags=B.FLAG_PREFIX_SIMT), 2),
    (dict(flags=B.FLAG_FUSED_MERGE), 2), (dict(head_dim=96), 2), (dict(h_q=30), 1), (dict(page_size=24), 2),
    (dict(table=torch.full((1, 2), -1, dtype=torch.int32)), 1), (dict(n_pages=7), 1), (dict(table=None), 1),
    (dict(prefix_offset=[-1]), 1), (dict(h_q=68, h_kv=4), 2)])
def test_plan_refusals(padlib, change, status):
    a = dict(prefix_len=[10], event_video=[0], event_len=[20], n_new=[17], kv_format=0, n_pages=0, table=_table(1),
             prefix_offset=None)
    prob = _prob(**{k: change.pop(k) for k in ("flags", "head_dim", "h_q", "h_kv", "page_size") if k in change})
    a.update(change)
    cache = B.CacheState(8)
    with pytest.raises(B.PadError) as e:
        B.pad_chunk_plan(prob, cache, a["prefix_len"], a["event_video"], a["event_len"], a["n_new"], page_table=a["table"],
                         n_pages=a["n_pages"], kv_format=a["kv_format"], prefix_offset=a["prefix_offset"])
    assert e.value.status == status and cache.free_count == 8


def test_events_out_of_video_order_are_refused(padlib):
    with pytest.raises(B.PadError):
        B.pad_chunk_plan(_prob(), None, [1, 1], [1, 0], [0, 0], [1, 1])


def test_null_arguments_are_refused(padlib):
    L, prob = B.lib(), _prob()
    one = np.ones(1, np.int32).ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    h = ctypes.c_void_p()
    assert L.pad_chunk_plan(None, 0, None, 0, None, None, 1, None, one, one, None, 0, 0, None, 0, None, ctypes.byref(h)) == 1
    assert L.pad_chunk_plan(ctypes.byref(prob), 0, None, 0, None, None, 1, None, None, one, None, 0, 0, None, 0, None,
                            ctypes.byref(h)) == 1
    assert L.pad_chunk_plan(ctypes.byref(prob), 0, None, 0, None, None, 1, None, one, one, None, 0, 0, None, 0, None, None) == 1
    assert L.pad_chunk_workspace_size(None, 0, 0, None, 0, None, None, None) == 0
    assert L.pad_chunk_append(None, None, None, 0, None, None, None, None, None) == 1
    assert L.pad_chunk_get_info(None, None) == 1 and L.pad_chunk_commit(None, None, None, None) == 1
    assert h.value is None


def test_host_only_plans_are_not_launched(padlib):
    plan = B.pad_chunk_plan(_prob(), None, None, None, [5], [3], page_table=_table(1), n_pages=4)
    L = B.lib()
    one = ctypes.c_void_p(256)
    assert L.pad_chunk_append(plan.handle, one, one, 0, one, one, None, None, None) == 1
    assert L.pad_chunk_attn(plan.handle, one, 0, None, None, one, one, None, None, one, None, None) == 1
    assert L.pad_draft_verify(plan.handle, 10, 0, one, 0, one, 0, one, one, one, one, one, None) == 1
    assert b"host-only" in L.pad_last_error()


def test_workspace_size_covers_its_parts(padlib):
    prob = _prob()
    size = B.pad_chunk_workspace_size(prob, [8192], [0] * 13, [64] * 13, [5] * 13)
    plan = B.pad_chunk_plan(prob, None, [8192], [0] * 13, [64] * 13, [5] * 13)
    i = plan.info()
    assert i["workspace_bytes"] == size >= i["partial_rows"] * (128 * 4 + 8)
    # every row has a prefix and a private piece at least
    assert i["partial_rows"] == 13 * 5 * 28 * (i["prefix_splits"] + i["page_splits"])


def test_empty_steps_plan(padlib):
    plan = B.pad_chunk_plan(_prob(), None, None, None, [], [], page_table=torch.zeros((0, 4), dtype=torch.int32))
    assert plan.n_tokens == 0 and plan.commit(None).size == 0
    plan = B.pad_chunk_plan(_prob(), None, [5], [0, 0], [3, 0], [0, 0], page_table=_table(2))
    assert plan.n_tokens == 0 and plan.n_cached == 3 and plan.info()["partial_rows"] == 0
