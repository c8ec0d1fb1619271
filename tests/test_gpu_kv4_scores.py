"""Attention over a 4-bit cache where scores are far from 0.

The keys' first dimension alone is not zero and tokens differ in it by a sixteenth at least, so that beside
the largest score, 2^20 and more in magnitude, every other has a weight of 0 and the output is the mean of V over the tokens
that have it (all equal weights).  Bounds as in test_gpu_kv4.py; the lse, log2(e) times which is the largest score, is a product of
four factors rounded in fp32 and a sum: within 2^-21 of its magnitude.
"""
import numpy as np
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


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("lens,news", [([700, 3], [3, 2]), ([30, 5000], [7, 1]), ([64], [24])])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_of_any_size(d, lens, news, sign):
    r = np.random.default_rng(d + news[0])
    c = Case4(21, lens, news, None, None, 8, 2, d, 16)
    for e in range(len(lens)):
        n = c.k[e].shape[0]
        # values that are their group's largest, six times a scale
        x = 6.0 * (1.0 + r.integers(0, 8, n) / 8) * 2.0 ** r.integers(0, 7, n)
        c.k[e] = torch.zeros_like(c.k[e])
        c.k[e][:, :, 0] = torch.from_numpy(x).bfloat16()[:, None]
    rows = c.q.shape[0] * 8
    size = sign * r.uniform(1.0, 2.0, rows) * 2.0 ** np.resize([23, 0, 26, 29, 100, 32, 40, -3], rows)
    q = torch.zeros(rows, d)
    q[:, 0] = torch.from_numpy(size).float()
    c.q = q.view(-1, 8, d).bfloat16()
    c.store().device()
    out, lse = (x.double().cpu().numpy() for x in c.attend(c.plan(flags=B.FLAG_PREFIX_MMA)))
    for e in range(len(lens)):
        at, o, l, mag = c.want(e)
        n = int(c.news[e])
        tol = c.bound(e, mag, B.FLAG_PREFIX_MMA) + 2.0 ** -40 * 1e4
        # (rows of small scores: as in the other tests, of scores below 4000 in magnitude each within 2^-20 of that)
        tol = tol + 2.0 ** -8 * mag * (np.abs(l) < 4e3)[..., None]
        assert np.all(np.abs(out[at:at + n] - o) <= tol)
        assert np.all(np.abs(lse[at:at + n] - l) <= 2.0 ** -21 * np.abs(l) + 1e-4)
