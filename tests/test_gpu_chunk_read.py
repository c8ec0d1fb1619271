"""Reading the paged cache where a page id lies outside the pool."""
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


def _plan(c, **kw):
    prob = B.make_problem(c.h_q, c.h_kv, c.d, c.page, **kw)
    fmt = B.KV_FP8 if c.fp8 else B.KV_BF16
    c.ws = torch.zeros(B.pad_chunk_workspace_size(prob, c.prefix, c.video, c.lens, c.news, kv_format=fmt), dtype=torch.uint8,
                       device="cuda")
    return B.pad_chunk_plan(prob, None, c.prefix, c.video, c.lens, c.news, page_table=c.dt, n_pages=c.n_pages, kv_format=fmt,
                            workspace=c.ws)


@pytest.mark.parametrize("fp8", [False, True])
def test_a_read_of_a_page_outside_the_pool_gives_zeros(fp8):
    """Its tokens come out as zeros, not as what the output held before, and the page is reported."""
    c = Case(90, [40, 3], [2, 2], None, None, 2, 2, 64, 16, fp8).store().device()
    c.dt[0, 1] = c.n_pages
    c.dt[1, 0] = -1
    plan = _plan(c)
    k, v = (torch.full((plan.n_cached, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.pad_chunk_read(plan, *c.dp, k, v, *c.ds)
    with pytest.raises(B.PadError) as err:
        B.pad_chunk_status(plan)
    assert err.value.status == 7
    for got, i in ((k, 0), (v, 1)):
        want = c.cached(i, 0)
        want[16:32] = 0.0
        got = got.double().cpu().numpy()
        assert np.array_equal(got[:42], want) and np.all(got[42:] == 0.0)
