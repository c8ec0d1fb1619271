"""Attention over a 4-bit cache: branches that are taken in pieces keep the bound of the warp-level kernel up to the last row
count that is planned there.  Bounds as in test_gpu_kv4.py.
"""
import pytest
import torch

from paper_2607_02963_gb300 import binding as B
from test_gpu_kv4 import Case4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(padlib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()


@pytest.mark.parametrize("d,h_q,h_kv,news", [(128, 28, 4, [8, 5, 9]), (64, 14, 2, [13, 1]), (128, 4, 2, [33, 48, 47]), (64, 16, 1, [6, 3]),
                                             (128, 2, 2, [96, 33])])
def test_branches_in_pieces_keep_the_weights_precision(d, h_q, h_kv, news):
    """33 to 96 rows of a branch, as planned by default: on the warp-level kernel, with its bound."""
    c = Case4(31, [150, 2000, 0][:len(news)], news, None, None, h_q, h_kv, d, 16).store().device()
    plan = c.plan()
    assert plan.info()["tc_items"] == 0
    c.check4(*c.attend(plan), B.FLAG_PREFIX_MMA)
    B.pad_chunk_status(plan)


@pytest.mark.parametrize("h_q,h_kv,at", [(2, 2, 96), (4, 2, 48), (12, 4, 32), (16, 1, 6)])
def test_the_edge_between_pieces_and_widened_pages(h_q, h_kv, at):
    """96 rows of a branch are the most that go in pieces; one token more and its pages are widened."""
    for n, wide in ((at, False), (at + 1, True)):
        c = Case4(32, [333], [n], None, None, h_q, h_kv, 128, 16).store().device()
        plan = c.plan()
        assert (plan.info()["tc_items"] > 0) == wide and (plan.info()["mma_items"] > 0) != wide
        c.check4(*c.attend(plan), B.FLAG_PREFIX_TC if wide else B.FLAG_PREFIX_MMA)
        B.pad_chunk_status(plan)
