"""The stage operators' oracle against the definitions' own properties: no GPU."""

import numpy as np
import pytest

from oracle import stage_oracle as so


@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
def test_rotation_keeps_pairs_and_composes(pairing):
    rng = np.random.default_rng(1)
    table = so.rope_table(40, 12, 10000.0)
    x = rng.standard_normal((5, 3, 16))
    a, b = so.pair_columns(12, pairing)
    at = np.array([0, 1, 7, 12, 20])
    y = so.rotate(x, table[at], pairing)
    np.testing.assert_allclose(np.hypot(y[..., a], y[..., b]), np.hypot(x[..., a], x[..., b]), rtol=1e-13)
    assert np.array_equal(y[..., 12:], x[..., 12:]) and np.array_equal(y[0], x[0])
    np.testing.assert_allclose(so.rotate(y, table[at + 4], pairing), so.rotate(x, _turn(table, at, 4), pairing),
                               atol=1e-12)
    np.testing.assert_allclose(so.rotate(y, table[at], pairing, -1.0), x, atol=1e-13)


def _turn(table, at, by):
    """Table rows of the positions at + (at + by), by the addition theorems."""
    half = table.shape[1] // 2
    c1, s1, c2, s2 = table[at][:, :half], table[at][:, half:], table[at + by][:, :half], table[at + by][:, half:]
    return np.concatenate((c1 * c2 - s1 * s2, s1 * c2 + c1 * s2), axis=1)


@pytest.mark.parametrize("pairing,rot", [("halves", 8), ("adjacent", 8), ("halves", 4), ("adjacent", 0)])
def test_rope_gradients_against_differences(pairing, rot):
    rng = np.random.default_rng(rot)
    x, dy, w = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8)), 1 + 0.3 * rng.standard_normal(8)
    rows = so.rope_table(20, rot, 100.0)[[3, 0, 11]] if rot else np.zeros((3, 0))
    dx, dw = so.qk_rope_backward(dy, x, w, rows, pairing, 1e-5)
    f = lambda x_, w_: float((dy * so.qk_rope_forward(x_, w_, rows, pairing, 1e-5)).sum())
    step = 1e-6
    for at in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[at] = step
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * step) - dx[at]) < 1e-7
    for i in range(8):
        d = np.zeros(8)
        d[i] = step
        assert abs((f(x, w + d) - f(x, w - d)) / (2 * step) - dw[i]) < 1e-7


def test_distill_gradient_against_differences():
    rng = np.random.default_rng(3)
    logits, top = rng.standard_normal((4, 9)), rng.standard_normal((4, 3))
    ids = np.array([[0, 4, 8], [2, 2, 5], [1, -1, 11], [-1, -1, -1]])     # distinct, one twice, padding, nothing
    weight = np.array([1.0, 0.25, 2.0, 1.0])
    loss, grad = so.distill_loss(logits, ids, top, weight, 1.7)
    assert loss[3] == 0 and not grad[3].any()
    assert np.abs(grad.sum(axis=1)).max() < 1e-12                          # both distributions sum to 1
    for at in np.ndindex(logits.shape):
        d = np.zeros_like(logits)
        d[at] = 1e-6
        up, down = so.distill_loss(logits + d, ids, top, weight, 1.7)[0], so.distill_loss(logits - d, ids, top, weight, 1.7)[0]
        assert abs((up - down).sum() / 2e-6 - grad[at]) < 1e-8


def test_distill_loss_is_a_divergence():
    rng = np.random.default_rng(4)
    logits = rng.standard_normal((6, 12))
    ids = np.tile(np.arange(12), (6, 1))
    same, grad = so.distill_loss(logits, ids, logits, None, 2.0)
    assert np.abs(same).max() < 1e-14 and np.abs(grad).max() < 1e-14
    other, _ = so.distill_loss(logits, ids, rng.standard_normal((6, 12)), None, 2.0)
    assert (other > 0).all()
    masked, grad = so.distill_loss(np.full((1, 12), np.nan), ids[:1], logits[:1], np.zeros(1), 1.0)
    assert masked[0] == 0 and not grad.any()


def test_int8_rows_are_within_half_a_step():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((7, 33)).astype(np.float32).astype(np.float64)
    x[2] = 0.0
    x[3, 5] = np.inf
    q, scale = so.int8_quantize(x)
    assert np.abs(q).max() == 127 and np.array_equal(q, np.rint(q))
    assert scale[2] == 0 and not q[2].any() and np.isnan(scale[3]) and not q[3].any()
    for t in (0, 1, 4, 5, 6):
        assert np.abs(q[t] * scale[t] - x[t]).max() <= scale[t] / 2 * (1 + 1e-6)
    w = rng.integers(-127, 128, (5, 33))
    ws = rng.random(5).astype(np.float32)
    y = so.int8_matmul(q, np.nan_to_num(scale), w, ws)
    np.testing.assert_allclose(y, (q * np.nan_to_num(scale.astype(np.float64))[:, None]) @ (w * ws.astype(np.float64)[:, None]).T, rtol=1e-12)
