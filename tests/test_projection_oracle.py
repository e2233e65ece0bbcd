"""Pins of the fp64 references of the operators around the attention (oracle/projection_oracle.py): closed forms,
difference quotients, and torch where it has the operation.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import projection_oracle as po


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_norm_without_rotation_is_torch_s(norm):
    rng = np.random.default_rng(0)
    x, w, b = rng.standard_normal((2, 3, 4, 64)) + 0.5, rng.standard_normal(64), rng.standard_normal(64)
    got = po.heads_forward(x, norm, w, b, 1e-3, 0, "halves", 1.0, None)
    t = torch.from_numpy
    want = (torch.nn.functional.layer_norm(t(x), (64,), t(w), t(b), 1e-3) if norm == "layer"
            else torch.nn.functional.rms_norm(t(x), (64,), t(w), 1e-3) + t(b))
    assert np.abs(got - want.numpy()).max() < 1e-13


@pytest.mark.parametrize("axes", [1, 2])
@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
def test_rotation_depends_on_the_distance_alone(axes, pairing):
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((1, 1, 1, 64)), rng.standard_normal((1, 1, 1, 64))
    dot = lambda p, s: float((po._turn(q, axes, 100.0, pairing, np.full((1, axes), p)) * po._turn(k, axes, 100.0, pairing, np.full((1, axes), s))).sum())
    assert abs(dot(7, 3) - dot(104, 100)) < 1e-10 and abs(dot(0, 0) - float((q * k).sum())) < 1e-12
    assert abs(dot(7, 3) - dot(3, 7)) > 1e-3


def test_rotation_by_a_quarter_turn():
    x = np.arange(64.0).reshape(1, 1, 1, 64)
    # base 1: every pair turns by the position itself; positions are real numbers for this reference
    y = po._turn(x, 1, 1.0, "halves", np.array([[np.pi / 2]]))
    assert np.allclose(y[..., :32], -x[..., 32:]) and np.allclose(y[..., 32:], x[..., :32])
    y = po._turn(x, 1, 1.0, "adjacent", np.array([[np.pi / 2]]))
    assert np.allclose(y[..., 0::2], -x[..., 1::2]) and np.allclose(y[..., 1::2], x[..., 0::2])
    y = po._turn(x, 2, 1.0, "halves", np.array([[np.pi / 2, 0.0]]))
    assert np.allclose(y[..., :16], -x[..., 16:32]) and np.allclose(y[..., 32:], x[..., 32:])


@pytest.mark.parametrize("norm", ["layer", "rms", "none"])
@pytest.mark.parametrize("axes,pairing", [(0, "halves"), (1, "adjacent"), (2, "halves")])
def test_gradients_are_the_difference_quotients(norm, axes, pairing):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((1, 3, 2, 64)), rng.standard_normal((1, 3, 2, 64))
    w, b = (rng.standard_normal((2, 64)), rng.standard_normal((2, 64))) if norm != "none" else (None, None)
    pos = rng.integers(0, 50, (3, axes)) if axes else None
    loss = lambda x, w, b: float((po.heads_forward(x, norm, w, b, 1e-5, axes, pairing, 100.0, pos) * dy).sum())
    dx, dw, db = po.heads_backward(x, norm, w, 1e-5, axes, pairing, 100.0, pos, dy, per_head=True)
    h = 1e-5
    for t, grad, call in [(x, dx, lambda t: loss(t, w, b)), (w, dw, lambda t: loss(x, t, b)), (b, db, lambda t: loss(x, w, t))]:
        if t is None:
            continue
        way = rng.standard_normal(t.shape)
        assert abs((call(t + h * way) - call(t - h * way)) / (2 * h) - float((grad * way).sum())) < 1e-6 * max(1.0, abs(float((grad * way).sum())))


def test_mxfp4_of_known_blocks():
    row = np.zeros(32)
    row[:8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0]                    # the ties, at scale 1
    c, s = po.mxfp4_quantise((row.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)[None])
    assert s.tolist() == [[127]] and c[0, :8].tolist() == [0, 2, 2, 4, 4, 6, 6, 6]
    row[:8] = [7.5, -7.5, -0.25, 0.24, -6.0, 5.1, -0.0, 1.0]
    c, s = po.mxfp4_quantise((row.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)[None])
    assert s.tolist() == [[127]] and c[0, :8].tolist() == [7, 15, 8, 0, 15, 7, 8, 2]
    assert po.mxfp4_values(c, s)[0, :8].tolist() == [6.0, -6.0, 0.0, 0.0, -6.0, 6.0, 0.0, 1.0]
    c, s = po.mxfp4_quantise(np.zeros((1, 64), np.uint16))
    assert s.tolist() == [[0, 0]] and not c.any()


def test_mxfp4_scale_is_a_power_of_two_and_the_error_at_most_a_step():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((20, 96)) * np.exp(rng.uniform(-80, 80, (20, 1)))).astype(np.float32)
    bits = (x.view(np.uint32) >> 16).astype(np.uint16)
    c, s = po.mxfp4_quantise(bits)
    x = po.bf16_to_f64(bits)
    top = np.abs(x.reshape(20, 3, 32)).max(-1)
    # the largest element is below 8 scales and comes out as 4 or 6 of them (3.5 upwards rounds to 4)
    assert (top < 8 * np.ldexp(1.0, s - 127)).all() and (top >= 4 * np.ldexp(1.0, s - 127)).all()
    assert (np.abs(po.mxfp4_values(c, s) - x) <= np.repeat(2 * np.ldexp(1.0, s - 127), 32, 1)).all()
