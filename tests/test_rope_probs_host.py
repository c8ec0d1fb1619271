"""Rotary positions and probabilities of a multi-token step without a GPU: the pairs' frequencies, pins of the fp64 oracle,
refusals."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2607_02963_gb300 import binding as B
from test_chunk_checks import _plan, _pools, _zeros


def _turns(r):
    return np.array([r.turns.turn[i] for i in range(r.turns.rotary_dim // 2)], dtype=object)


@pytest.mark.parametrize("scaling", B.Rope.SCALINGS)
@pytest.mark.parametrize("rotary,theta", [(128, 1e6), (64, 1e4), (54, 500.0), (4, 10.0)])
def test_frequencies(padlib, scaling, rotary, theta):
    kw = dict(scaling=scaling, factor=4.0, original_len=4096.0, low=1.0, high=32.0)
    got = _turns(B.Rope(128, rotary, theta, **kw)) / 2 ** 64
    want = oracle.rope_frequencies(rotary, theta, **kw) / (2 * math.pi)
    # (two powers and a few products and quotients in 64 bits)
    assert np.all(np.abs(got.astype(float) - want) <= 2.0 ** -48 * want + 2.0 ** -63)


def test_scalings_leave_fast_pairs_and_slow_slow_ones(padlib):
    plain = oracle.rope_frequencies(128, 1e6)
    for scaling in ("turns", "index"):
        f = oracle.rope_frequencies(128, 1e6, scaling, 4.0, 32768.0, 1.0, 4.0)
        assert f[0] == plain[0] and math.isclose(f[-1], plain[-1] / 4, rel_tol=1e-12) and np.all(f <= plain) and np.all(f >= plain / 4.0001)
    assert np.allclose(oracle.rope_frequencies(128, 1e6, "base", 4.0)[-1], plain[-1] / 4)


def test_turning_is_the_decode_steps_rotation():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 2, 64))
    pos = [0, 5, 1000]
    out, _ = oracle.rope_turn(x, pos, oracle.rope_frequencies(64, 1e4))
    z = (x[..., :32] + 1j * x[..., 32:]) * np.exp(1j * np.asarray(pos)[:, None, None] * oracle.rope_frequencies(64, 1e4))
    assert np.allclose(out, np.concatenate([z.real, z.imag], -1), atol=1e-9)
    flip, _ = oracle.rope_turn(x[..., np.arange(64).reshape(2, 32).T.ravel()], pos, oracle.rope_frequencies(64, 1e4), "interleaved")
    assert np.allclose(flip[..., 0::2], out[..., :32]) and np.allclose(flip[..., 1::2], out[..., 32:])


def test_probabilities_of_small_rows():
    p, _ = oracle.logits_to_probs([1.0, 2.0, -1.0, 0.0], 0.5, 2.0, 0.25, 0.125, context=[1, 1, 2, 9, -1], biases=[(3, 1.0), (3, 0.5), (7, 2)],
                                  allowed=[1, 1, 1, 1])
    x = np.array([1.0, 1.0 - 0.625, -2.0 - 0.375, 1.5])
    assert np.allclose(p, np.exp(2 * x) / np.exp(2 * x).sum())
    assert oracle.logits_to_probs([3.0, 3.0], 0.0)[0].tolist() == [1, 0]
    assert not oracle.logits_to_probs([3.0, 3.0], 1.0, allowed=[0, 0])[0].any()
    assert np.isnan(oracle.logits_to_probs([3.0, np.nan], 1.0)[0]).all() and not oracle.logits_to_probs([3.0, np.nan], 0.0)[0].any()


@pytest.mark.parametrize("bad", [dict(head_dim=96), dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=130), dict(theta=0.0),
                                 dict(theta=float("nan")), dict(magnitude=float("inf")), dict(scaling="linear", factor=0.0),
                                 dict(scaling="base", rotary_dim=2), dict(scaling="turns", original_len=0.0),
                                 dict(scaling="turns", original_len=9.0, low=2.0, high=2.0), dict(scaling="index", original_len=9.0, low=0.0),
                                 dict(scaling="index", original_len=9.0, theta=1.0)])
def test_rope_specs_that_are_refused(padlib, bad):
    with pytest.raises(B.PadError):
        B.Rope(**(dict(head_dim=128) | bad))


def test_layouts_and_scalings_by_name(padlib):
    with pytest.raises(ValueError, match="layout"):
        B.Rope(64, layout="whole")
    with pytest.raises(ValueError, match="scaling"):
        B.Rope(64, scaling="more")


def test_what_append_rope_refuses(padlib):
    plan, rope = _plan(), B.Rope(64)
    n = plan.n_tokens
    t = dict(position=_zeros(n, dtype=torch.int32), q=_zeros(n, 8, 64), q_out=_zeros(n, 8, 64), k_new=_zeros(n, 2, 64),
             v_new=_zeros(n, 2, 64), k_pool=_pools()[0], v_pool=_pools()[1])

    def call(r=rope, **kw):
        B.pad_chunk_append_rope(plan, r, *(t | kw).values(), stream=0)

    with pytest.raises(B.PadError, match="host-only"):
        call()
    for name, x in t.items():
        with pytest.raises(ValueError, match=f"{name}: .*device memory"):
            call(**{name: torch.zeros(x.shape, dtype=x.dtype)})
    with pytest.raises(ValueError, match="position"):
        call(position=_zeros(n, dtype=torch.int64))
    with pytest.raises(ValueError, match="q_out"):
        call(q_out=_zeros(n, 8, 64, dtype=torch.float32))
    with pytest.raises(ValueError, match="same token stride"):
        call(k_new=_zeros(n, 256)[:, :128].unflatten(1, (2, 64)))


def test_what_probs_refuses(padlib):
    plan, f32, i32 = _plan(), torch.float32, torch.int32
    n, ne, v = plan.n_tokens, plan.n_events, 70
    t = dict(params=_zeros(ne, 4, dtype=f32), history=_zeros(ne, 9, dtype=i32), history_len=_zeros(ne, dtype=i32),
             tokens=_zeros(n, dtype=i32), bias_token=_zeros(ne, 3, dtype=i32), bias_value=_zeros(ne, 3, dtype=f32),
             bias_len=_zeros(ne, dtype=i32), mask=_zeros(n, 3, dtype=i32))

    def call(logits=None, p=None, **kw):
        B.pad_chunk_probs(plan, _zeros(n, v, dtype=f32) if logits is None else logits, _zeros(n, v, dtype=f32) if p is None else p, stream=0,
                          **kw)

    for kw in ({}, t, dict(params=t["params"])):
        with pytest.raises(B.PadError, match="host-only"):
            call(**kw)
    with pytest.raises(B.PadError, match="host-only"):
        call(logits=_zeros(n, v), p=_zeros(n, v))
    for name, x in t.items():
        with pytest.raises(ValueError, match=f"{name}: .*device memory"):
            call(**(t | {name: torch.zeros(x.shape, dtype=x.dtype)}))
    for bad in (_zeros(n, v, dtype=torch.float16), _zeros(n + 1, v, dtype=f32), torch.zeros(n, v)):
        with pytest.raises(ValueError, match="logits"):
            call(logits=bad)
        with pytest.raises(ValueError, match="p: "):
            call(p=bad)
    with pytest.raises(ValueError, match="mask"):
        call(mask=_zeros(n, 2, dtype=i32))
    for name in ("history", "history_len", "bias_token", "bias_value", "bias_len"):
        with pytest.raises(ValueError, match="come together"):
            call(**{name: t[name]})
    with pytest.raises(B.PadError, match="host-only"):   # (a context and biases of width 0 are none)
        call(history=t["history"][:, :0].contiguous(), history_len=t["history_len"], bias_token=t["bias_token"][:, :0].contiguous(),
             bias_value=t["bias_value"][:, :0].contiguous(), bias_len=t["bias_len"])
