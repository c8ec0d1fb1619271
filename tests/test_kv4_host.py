"""The 4-bit cache without a GPU: pins of its fp64 oracle, plans, refusals."""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_02963_gb300 import binding as B
from test_chunk_checks import _zeros


def _prob(**kw):
    return B.make_problem(**(dict(h_q=28, h_kv=4, head_dim=128, page_size=16, num_sms=152) | kw))


def test_scales_are_an_f16s_upper_bits():
    got = (torch.arange(227, dtype=torch.int32) << 7).to(torch.int16).view(torch.float16).double().numpy()
    assert np.array_equal(got, oracle.kv4_scales()) and oracle.kv4_scales()[226] == 10240


def test_encode_is_the_nearest_scale_and_code():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64)) * 2.0 ** rng.integers(-22, 16, size=(200, 1))
    codes, byte = oracle.kv4_encode(x)
    assert codes.shape == (200, 32) and byte.shape == (200, 4)
    back = oracle.kv4_decode(codes, byte)
    s, values = oracle.kv4_scales(), np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    values = np.concatenate([values, -values])
    for row, got, bytes_ in zip(x.reshape(-1, 16), back.reshape(-1, 16), byte.reshape(-1)):
        want = np.abs(row).max() / 6
        assert abs(s[bytes_] - want) == np.min(np.abs(s - want))
        best = np.min(np.abs(row[:, None] - values * s[bytes_]), axis=1)
        assert np.array_equal(np.abs(row - got), best)


def test_ties_go_to_the_even_code_and_byte():
    # scale 1 (max 6): every midpoint of the codes
    x = np.array([[6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, 0]])
    codes, byte = oracle.kv4_encode(x)
    assert oracle.kv4_decode(codes, byte)[0].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -1, -2, -2, -4, -4, 0]
    # maxima half way between two scales: 6 (1 + 1/16) and 6 (1 + 3/16)
    for top, want in ((6.375, 120), (7.125, 122)):
        assert oracle.kv4_encode(np.full((1, 16), top))[1][0, 0] == want


def test_encode_of_special_groups():
    z, n, s = np.zeros((1, 32)), np.ones((1, 32)), np.full((1, 16), 1e6)
    n[0, 3] = np.inf
    assert oracle.kv4_encode(z)[1].tolist() == [[0, 0]] and not oracle.kv4_decode(*oracle.kv4_encode(z)).any()
    codes, byte = oracle.kv4_encode(n)
    assert byte[0, 0] == 255 and not codes[0, :8].any()
    back = oracle.kv4_decode(codes, byte)[0]
    assert np.isnan(back[:16]).all() and np.all(back[16:] == 6 * oracle.kv4_scales()[byte[0, 1]])
    assert np.all(oracle.kv4_decode(*oracle.kv4_encode(s)) == 61440.0)


def test_products_of_code_and_scale_are_exact_in_f16_and_bf16():
    v = (oracle.kv4_scales()[:, None] * np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])).ravel()
    t = torch.from_numpy(v)
    assert torch.equal(t.half().double(), t) and torch.equal(t.bfloat16().double(), t)


def test_long_chunks_bring_a_workspace_for_widened_pages(padlib):
    def size(n, fmt, flags=0, lens=5000):
        return B.pad_chunk_workspace_size(_prob(flags=flags), None, None, [lens], [n], kv_format=fmt)

    wide = 2 * 2 * 128 * 4 * 5000
    assert size(4, B.KV_FP4) < wide and size(1000, B.KV_FP4) > size(1000, B.KV_BF16) + wide
    assert size(4, B.KV_FP4, B.FLAG_PREFIX_TC) > wide
    # (a chunk over nothing, a branch without new tokens)
    assert B.pad_chunk_workspace_size(_prob(), None, None, [0, 9], [300, 0], kv_format=B.KV_FP4) > 0


@pytest.mark.parametrize("group,news", [(7, [1, 2, 3, 4, 5, 8, 9]), (16, [1, 2, 3]), (1, [1, 7, 24, 25, 96]), (3, [8, 9, 11])])
def test_items_cover_the_tokens(padlib, group, news):
    """One piece of up to 24 rows, pieces of up to 16 where there are more, about as long as one another."""
    for n in news:
        plan = B.pad_chunk_plan(_prob(h_q=group, h_kv=1), None, None, None, [100], [n], page_table=torch.zeros(1, 64, dtype=torch.int32),
                                n_pages=64, kv_format=B.KV_FP4)
        i = plan.info()
        pieces = 1 if n * group <= 24 else -(-n // (16 // group))
        assert i["tc_items"] == 0 and i["mma_items"] == -(-n // (-(-n // pieces))) * i["page_splits"]


def test_pools_of_more_rows_than_32_bits_count_are_refused(padlib):
    table = torch.zeros(1, 4, dtype=torch.int32)
    def plan(n, fmt):
        return B.pad_chunk_plan(_prob(page_size=64), None, None, None, [5], [1], page_table=table, n_pages=n, kv_format=fmt)
    plan((1 << 24) - 1, B.KV_FP4), plan(1 << 24, B.KV_FP8)
    with pytest.raises(B.PadError, match="2.32 rows"):
        plan(1 << 24, B.KV_FP4)


def test_formats_and_shapes_are_checked(padlib):
    with pytest.raises(B.PadError, match="kv_format=3"):
        B.pad_chunk_workspace_size(_prob(), None, None, [5], [1], kv_format=3)
    prob = B.make_problem(8, 2, 64, 16, num_sms=152)
    plan = B.pad_chunk_plan(prob, None, None, None, [5], [3], page_table=torch.zeros(1, 4, dtype=torch.int32), n_pages=9,
                            kv_format=B.KV_FP4)
    u8 = torch.uint8
    new = [_zeros(3, 2, 64) for _ in range(2)]
    pools, scales = [_zeros(9, 2, 16, 32, dtype=u8) for _ in range(2)], [_zeros(9, 2, 16, 4, dtype=u8) for _ in range(2)]
    with pytest.raises(B.PadError, match="host-only"):
        B.pad_chunk_append(plan, *new, *pools, *scales, stream=0)
    for bad in (_zeros(9, 2, 16, 64, dtype=u8), _zeros(9, 2, 16, 32)):
        with pytest.raises(ValueError, match="k_pool"):
            B.pad_chunk_append(plan, *new, bad, pools[1], *scales, stream=0)
    for bad in (_zeros(9, 2, 16, dtype=u8), _zeros(9, 2, 16, 8, dtype=u8), torch.zeros(9, 2, 16, 4, dtype=u8)):
        with pytest.raises(ValueError, match="v_scale"):
            B.pad_chunk_read(plan, *pools, _zeros(8, 2, 64), _zeros(8, 2, 64), scales[0], bad, stream=0)
