"""Joins of split key ranges: what is not finite in a piece of a row's keys whose weight underflows, and partial states
of another call.  Bounds as in test_gpu_chunk.py."""
import numpy as np
import pytest
import torch

from paper_2607_02963_gb300 import binding as B
from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(padlib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()


def _plan(c, flags, sms):
    prob = B.make_problem(c.h_q, c.h_kv, c.d, c.page, flags=flags, num_sms=sms)
    fmt = B.KV_FP8 if c.fp8 else B.KV_BF16
    c.ws = torch.zeros(B.pad_chunk_workspace_size(prob, c.prefix, c.video, c.lens, c.news, kv_format=fmt), dtype=torch.uint8,
                       device="cuda")
    return B.pad_chunk_plan(prob, None, c.prefix, c.video, c.lens, c.news, page_table=c.dt, n_pages=c.n_pages, kv_format=fmt,
                            workspace=c.ws)


@pytest.mark.parametrize("sms", [1, 2, 4, 0])
@pytest.mark.parametrize("flags", [0, B.FLAG_PREFIX_MMA, B.FLAG_PREFIX_TC])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("where", ["pages", "prefix"])
def test_a_nan_in_a_piece_of_no_weight_is_kept(where, fp8, flags, sms):
    """Each key's value counts p v, and a NaN stays one however small p is: whole pieces of the keys (a range, the
    tiles of one of two halves) lie 240 and more below the others in log2 units, one of their values is a NaN."""
    lens, news, prefix, video = ([3000], [1], None, None) if where == "pages" else ([4], [5], [3000], [0])
    c = Case(50, lens, news, prefix, video, 8, 2, 128, 16, fp8)
    k, v = (c.k[0], c.v[0]) if where == "pages" else (c.k_pre, c.v_pre)
    pos = torch.arange(k.shape[0])
    low = (pos < 2048) | ((pos // 128) % 2 == 0)
    c.q[:, :, 0] = 64.0
    c.k[0][:, :, 0] = 0.0
    k[:, :, 0] = torch.where(low, -30.0, 0.0)[:, None].bfloat16()
    want = c.want(0)[1:]
    v[3, 1, 9] = float("nan")
    c.store().device()
    out, lse = c.attend(_plan(c, flags, sms))
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    hole = np.zeros(out.shape, bool)
    if fp8 and where == "pages":
        hole[:, 4:] = True      # (the group reads back as NaN throughout)
    else:
        hole[:, 4:, 9] = True
    assert np.all(np.isnan(out[hole]))
    o, l, mag = want
    assert np.all((np.abs(out - o) <= (2.0 ** -8 + 1e-4) * mag) | hole)
    assert np.all(np.abs(lse - l) <= 1e-4)
