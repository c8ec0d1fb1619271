"""Probabilities on both sides of every size at which the launch takes another form, in each pair of types.  Bounds as in
test_gpu_rope_probs.py.

A row goes over eight CTAs up to 159232 entries and over 16 beyond; a thread's registers hold the slice in their short form up to
319481 entries where logits or results are in 16 bits (there every one of its vectors is in use) and 327673 in fp32.
"""
import pytest
import torch

from test_gpu_rope_probs import Rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(padlib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()


TYPES = [(False, False), (True, True), (True, False), (False, True)]


@pytest.mark.parametrize("bf16", TYPES)
@pytest.mark.parametrize("vocab", [159232, 159233, 319481, 319482, 327673, 327674, 393152])
def test_both_sides_of_each_edge(vocab, bf16):
    r = Rows(vocab, [1, 2], vocab, 100, 10, 0.5, bf16)
    r.params[0, 0] = 0.0
    r.check(r.run())
    # rows that begin elsewhere, logits and results not alike
    wide = torch.full((3, vocab + 16), float("nan"), dtype=r.logits.dtype, device="cuda")
    out = torch.full((3, vocab + 17), 7.0, dtype=r.kind, device="cuda")
    wide[:, 7:7 + vocab] = r.logits.cuda()
    r.run(wide[:, 7:7 + vocab], out[:, 2:2 + vocab])
    r.check(out[:, 2:2 + vocab])
    assert (out[:, :2] == 7).all() and (out[:, 2 + vocab:] == 7).all()


@pytest.mark.parametrize("bf16", TYPES[:2])
def test_more_long_rows_than_clusters(bf16):
    r = Rows(6, [30, 0, 25], 200001, 300, 20, 0.5, bf16)
    r.check(r.run())
