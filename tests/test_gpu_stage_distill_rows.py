"""The loss against a teacher's top logits where rows are far from zero, against the oracle in 64 bits with the limits of
test_gpu_stage_distill."""

import numpy as np
import pytest
import torch

from oracle import stage_oracle as so
from paper_2607_13332_b200.stage_ops import distill_loss, distill_loss_grad
from tests.test_gpu_stage_distill import U, f64, limits, make

pytestmark = pytest.mark.gpu


def assert_rows(logits, ids, top, weight, tau, loss, grad=None, far=0.0):
    """far: the largest size of a row's logits.  Their mean, a number of that size, is a quotient of sums in 64 bits whose divisor's
    reciprocal has 2^-45 (one step of Newton's rule from fp32)."""
    host = [f64(logits), ids.cpu().numpy(), f64(top), f64(weight)]
    want, dwant = so.distill_loss(*host, tau)
    lim, dlim = limits(*host, tau, logits.dtype)
    w = 1.0 if weight is None else np.abs(host[3])
    off, lim = np.abs(f64(loss) - want), lim + U * np.abs(want) + w * tau * far * 2.0 ** -44
    assert (off <= lim).all(), f"loss: worst {np.max(off / (lim + 1e-300)):.2f} of the limit"
    if grad is not None:
        off = np.abs(f64(grad) - dwant)
        dlim = dlim * (1 + 2.0 ** -7) + torch.finfo(logits.dtype).eps / 2 * np.abs(dwant) + 1e-37
        assert (off <= dlim).all(), f"gradient: worst {np.max(off / dlim):.2f} of the limit"


@pytest.mark.parametrize("n,vocab,k,dtype,tau", [(40, 5000, 64, "f32", 1.0), (40, 5000, 300, "f32", 2.0), (40, 5000, 1024, "bf16", 0.5),
                                                 (2, 140001, 64, "f32", 1.0), (33, 60001, 70, "bf16", 1.0)])
@pytest.mark.parametrize("shift", [100.0, -1000.0, 30000.0])
def test_a_constant_added_to_the_teacher_or_the_student(n, vocab, k, dtype, tau, shift):
    """Neither distribution changes, and neither do the limits."""
    rng = np.random.default_rng(vocab + k)
    logits, ids, top, weight = make(rng, n, vocab, k, dtype, 0.1)
    top = top + shift
    loss, grad = distill_loss_grad(logits, ids, top, weight, temperature=tau)
    assert_rows(logits, ids, top, weight, tau, loss, grad, far=2 * abs(shift))
    assert torch.equal(distill_loss(logits, ids, top, weight, temperature=tau), loss)
    if dtype == "f32":
        logits = logits + shift / 2
        loss, grad = distill_loss_grad(logits, ids, top, weight, temperature=tau)
        assert_rows(logits, ids, top, weight, tau, loss, grad, far=2 * abs(shift))


@pytest.mark.parametrize("vocab", [4000, 4001])
def test_last_tokens_of_sequences(vocab):
    """A view whose rows are far apart: the gradient made for it holds its rows alone."""
    rng = np.random.default_rng(vocab)
    logits, ids, top, weight = make(rng, 24 * 9, vocab, 16, "bf16")
    last = logits.view(24, 9, vocab)[:, -1]
    loss, grad = distill_loss_grad(last, ids[:24], top[:24], weight[:24])
    assert_rows(last, ids[:24], top[:24], weight[:24], 1.0, loss, grad)
    assert grad.untyped_storage().nbytes() <= 24 * (vocab + 8) * 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_that_start_off_a_boundary(dtype):
    """Logits without their first rows, an odd vocabulary: the gradient made by the call is the one of a caller's buffer."""
    rng = np.random.default_rng(31)
    logits, ids, top, weight = make(rng, 12, 2003, 16, dtype)
    for first in range(8):
        args = logits[first:], ids[first:], top[first:], weight[first:]
        loss, grad = distill_loss_grad(*args)
        assert_rows(*args, 1.0, loss, grad)
        loss2, grad2 = distill_loss_grad(*args, dlogits=torch.empty_like(args[0]))
        assert torch.equal(loss, loss2) and torch.equal(grad, grad2)
