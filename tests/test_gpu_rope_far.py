"""Rotary positions as far as they go, and frequencies beyond one radian a token, on the GPU against angles in 80 digits.

The value that is rounded to bf16 is within 2^-20 magnitude (|a| + |b|) of the exact one (as in test_gpu_rope_probs.py), so
what comes out is off by that and half a step of bf16 at the exact value or that far from it.
"""
import math
from decimal import Decimal

import numpy as np
import pytest
import torch

from paper_2607_02963_gb300 import binding as B
from test_gpu_rope_probs import Step
from test_rope_turns import exact_turns

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda(padlib):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()


def _half_step(x):
    return 2.0 ** (np.floor(np.log2(np.maximum(x, 1e-30))) - 8)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("spec", [dict(theta=1e6), dict(theta=1e4, scaling="linear", factor=0.01), dict(theta=0.001),
                                  dict(theta=1e6, scaling="turns", factor=4.0, original_len=32768.0)],
                         ids=["plain", "linear", "fast", "turns"])
@pytest.mark.parametrize("d,rotary", [(128, 128), (64, 54)])
def test_far_positions(d, rotary, spec, layout):
    r = np.random.default_rng(5)
    position = np.concatenate([r.integers(-2 ** 31, 2 ** 31, 60), r.integers(2 ** 31 - 9, 2 ** 31, 4), [-2 ** 31, 2 ** 31 - 1, 0, 1]])
    s = Step(12, [9, 50], [30, 38], 8, 2, d)
    q, pos = s.q.cuda(), torch.from_numpy(position.astype(np.int32)).cuda()
    out = torch.empty_like(q)
    B.pad_chunk_append_rope(s.plan, B.Rope(d, rotary, layout=layout, **spec), pos, q, out, s.k.cuda(), s.v.cuda(), *s.pools())
    B.pad_chunk_status(s.plan)
    turns = exact_turns(rotary, **spec)
    angle = np.array([[float(Decimal(int(p)) * t % 1) for t in turns] for p in position]) * 2 * math.pi
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    x, got = s.q.double().numpy(), out.double().cpu().numpy()
    one, two = (slice(0, rotary // 2), slice(rotary // 2, rotary)) if layout == "half" else (slice(0, rotary, 2), slice(1, rotary, 2))
    a, b = x[..., one], x[..., two]
    tol = 2.0 ** -20 * (np.abs(a) + np.abs(b))
    for at, want in ((one, a * cos - b * sin), (two, b * cos + a * sin)):
        assert np.all(np.abs(got[..., at] - want) <= tol + _half_step(np.abs(want) + tol))
    assert np.array_equal(got[..., rotary:], x[..., rotary:])
