"""The loss against a teacher's top logits, alone and with the gradient, against the oracle in 64 bits.

Tolerances, with u = 2^-24.  L = sum exp((s - m) / tau): the exponent is one rounding of a product (relative 2u of its size),
the exponential 2^-22, a thread adds at most V / 64 terms one after the other and the merges 80 more operations.  The
teacher's p: an exponential of a rounded argument (its size + 40 roundings) and the sum of K terms.  Both enter the loss
and the gradient as written in `limits`; an output is rounded once (half a step of its type)."""

import numpy as np
import pytest
import torch

from oracle import stage_oracle as so
from paper_2607_13332_b200 import binding
from paper_2607_13332_b200.stage_ops import distill_loss, distill_loss_grad

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def limits(logits, ids, top, weight, tau, dt):
    """(limit of the loss, limit of the gradient without its rounding)"""
    n, vocab = logits.shape
    loss, grad = np.zeros(n), np.zeros((n, vocab))
    for t in range(n):
        there = (ids[t] >= 0) & (ids[t] < vocab) & np.isfinite(top[t])
        w = 1.0 if weight is None else abs(weight[t])
        if w == 0 or not there.any() or not np.isfinite(w):
            continue
        x = np.where(np.isfinite(logits[t]), logits[t], -1e300) / tau
        arg = np.minimum(x.max() - x, 200.0)
        q = np.exp(-arg)
        q = q / q.sum()
        sum_l = (vocab / 64 + 80) * U + 2.0 ** -22 + 2 * U * (q * arg).sum()
        a = (top[t][there].max() - top[t][there]) / tau
        p = np.exp(-a)
        p = p / p.sum()
        own = (a + 40 + len(a)) * U                       # relative, of p
        apart = np.abs(np.log(np.maximum(p, 1e-300)) - np.log(np.maximum(q[ids[t][there]], 1e-300)))
        loss[t] = w * tau * tau * (sum_l + (p * own * (apart + 1)).sum())
        grad[t] = w * tau * q * (sum_l + 2 * U * arg + 2.0 ** -21)
        np.add.at(grad[t], ids[t][there], w * tau * p * own)
    return loss, grad


def make(rng, n, vocab, k, dtype, absent=0.0, scale=2.5):
    dt = TORCH[dtype]
    logits = torch.from_numpy((scale * rng.standard_normal((n, vocab))).astype(np.float32)).to(dt).cuda()
    ids = np.stack([rng.choice(vocab, k, replace=k > vocab) for _ in range(n)]).astype(np.int32)
    if absent:
        ids[rng.random((n, k)) < absent] = -1
    top = (6 + 1.5 * rng.standard_normal((n, k))).astype(np.float32)
    weight = rng.uniform(0.1, 2.0, n).astype(np.float32)
    return logits, torch.from_numpy(ids).cuda(), torch.from_numpy(top).cuda(), torch.from_numpy(weight).cuda()


def check(logits, ids, top, weight, tau, loss, grad=None):
    want, dwant = so.distill_loss(f64(logits), ids.cpu().numpy(), f64(top), f64(weight), tau)
    lim, dlim = limits(f64(logits), ids.cpu().numpy(), f64(top), f64(weight), tau, logits.dtype)
    off = np.abs(f64(loss) - want)
    assert (off <= lim + U * np.abs(want)).all(), f"loss: worst {np.max(off / (lim + U * np.abs(want) + 1e-300)):.2f} of the limit"
    if grad is not None:
        off = np.abs(f64(grad) - dwant)
        dlim = dlim * (1 + 2.0 ** -7) + torch.finfo(logits.dtype).eps / 2 * np.abs(dwant) + 1e-37
        assert (off <= dlim).all(), f"gradient: worst {np.max(off / dlim):.2f} of the limit at {np.unravel_index(np.argmax(off / dlim), off.shape)}"


CASES = [
    # n, vocab, K, dtype, tau, share of padding
    (1, 128256, 64, "bf16", 1.0, 0.0),
    (3, 128256, 64, "f32", 2.0, 0.0),
    (3, 140001, 33, "f32", 1.0, 0.1),
    (2, 300007, 20, "bf16", 1.0, 0.0),
    (37, 32003, 20, "bf16", 2.0, 0.3),
    (37, 32000, 32, "f32", 1.0, 0.0),
    (600, 1000, 8, "bf16", 1.5, 0.5),
    (9, 513, 256, "f32", 1.0, 0.2),
    (5, 4097, 1024, "bf16", 4.0, 0.5),
    (7, 66000, 100, "bf16", 1.0, 0.0),
    (4, 1, 1, "f32", 1.0, 0.0),
    (4, 2, 2, "bf16", 1.0, 0.0),
    (6, 7, 5, "bf16", 0.3, 0.0),
    (6, 9, 3, "f32", 1e3, 0.0),
]


@pytest.mark.parametrize("n,vocab,k,dtype,tau,absent", CASES)
def test_loss_and_gradient(n, vocab, k, dtype, tau, absent):
    rng = np.random.default_rng(n + vocab)
    logits, ids, top, weight = make(rng, n, vocab, k, dtype, absent)
    keep = logits.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, grad = distill_loss_grad(logits, ids, top, weight, temperature=tau, dev_status=status)
    check(logits, ids, top, weight, tau, loss, grad)
    assert torch.equal(distill_loss(logits, ids, top, weight, temperature=tau), loss)
    again = distill_loss_grad(logits, ids, top, weight, temperature=tau)
    assert torch.equal(again[0], loss) and torch.equal(again[1], grad) and torch.equal(logits, keep) and int(status) == 0
    # without weights: weights of one
    loss1, grad1 = distill_loss_grad(logits, ids, top, temperature=tau)
    check(logits, ids, top, None, tau, loss1, grad1)
    # in place
    loss2, grad2 = distill_loss_grad(logits, ids, top, weight, temperature=tau, dlogits=logits)
    assert grad2 is logits and torch.equal(loss2, loss) and torch.equal(logits, grad)


@pytest.mark.parametrize("vocab,offset,ld,out_offset,out_ld", [(1001, 3, 1001, 3, 1001), (1001, 1, 1005, 0, 1003), (4096, 0, 4104, 8, 4112),
                                                               (50001, 5, 50003, 5, 50003), (50001, 5, 50003, 2, 50001)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_neighbours(vocab, offset, ld, out_offset, out_ld, dtype):
    """Rows anywhere in a larger buffer; what is between and around the gradient's rows stays as it was."""
    rng = np.random.default_rng(vocab + ld)
    n, k = 6, 12
    logits, ids, top, weight = make(rng, n, vocab, k, dtype)
    want = distill_loss_grad(logits, ids, top, weight)
    src = torch.full((n * ld + offset + 16,), float("nan"), dtype=logits.dtype, device="cuda")
    view = src[offset:offset + n * ld].view(n, ld)[:, :vocab]
    view.copy_(logits)
    out = torch.full((n * out_ld + out_offset + 16,), 33.0, dtype=logits.dtype, device="cuda")
    grad = out[out_offset:out_offset + n * out_ld].view(n, out_ld)[:, :vocab]
    idw, topw = torch.full((n, k + 3), -7, dtype=torch.int32, device="cuda"), torch.full((n, k + 5), float("nan"), device="cuda")
    idw[:, :k], topw[:, :k] = ids, top
    loss, _ = distill_loss_grad(view, idw[:, :k], topw[:, :k], weight, dlogits=grad)
    check(view, ids, top, weight, 1.0, loss, grad)
    grad.fill_(33.0)
    assert bool((out == 33.0).all())


def test_the_same_id_twice():
    rng = np.random.default_rng(8)
    logits, ids, top, weight = make(rng, 5, 700, 40, "f32")
    ids[:, 10:20] = ids[:, 0:10]
    ids[3] = 699
    loss, grad = distill_loss_grad(logits, ids, top, weight, temperature=1.3)
    check(logits, ids, top, weight, 1.3, loss, grad)


@pytest.mark.parametrize("vocab", [997, 70000])
def test_rows_with_nothing_to_learn(vocab):
    rng = np.random.default_rng(9)
    logits, ids, top, weight = make(rng, 8, vocab, 6, "bf16")
    logits[1] = float("nan")
    weight[1] = 0.0                     # a padding token, whatever its logits hold
    logits[2, 5] = float("inf")
    ids[2] = -1                         # no entries
    top[3] = float("-inf")              # entries without mass
    ids[4, 1:] = -1                     # one entry
    top[5, 2:] = float("-inf")          # some without mass
    loss, grad = distill_loss_grad(logits, ids, top, weight)
    for t in (1, 2, 3):
        assert float(loss[t]) == 0.0 and not bool(grad[t].any())
    keep = [0, 4, 5, 6, 7]
    at = torch.tensor(keep, device="cuda")
    check(logits[at], ids[at], top[at], weight[at], 1.0, loss[at], grad[at])
    assert torch.equal(distill_loss(logits, ids, top, weight), loss)


def test_ids_outside_the_vocabulary():
    rng = np.random.default_rng(10)
    logits, ids, top, weight = make(rng, 4, 500, 6, "f32")
    ids[0, 0], ids[1, 3], ids[2, 5] = 500, -2, 2 ** 31 - 1
    ids[3, 2] = -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, grad = distill_loss_grad(logits, ids, top, weight, dev_status=status)
    assert int(status) == binding.SSN_DEV_BAD_ID
    check(logits, ids, top, weight, 1.0, loss, grad)


@pytest.mark.parametrize("dtype,lowest", [("bf16", float("-inf")), ("f32", float("-inf")), ("f32", torch.finfo(torch.float32).min),
                                          ("bf16", torch.finfo(torch.bfloat16).min)])
@pytest.mark.parametrize("vocab", [900, 33000])
def test_masked_logits(dtype, lowest, vocab):
    """Columns of -inf or of the type's lowest value have no probability; whole pieces of a row of them change nothing."""
    rng = np.random.default_rng(11)
    logits, ids, top, weight = make(rng, 5, vocab, 8, dtype)
    ids.copy_((ids.long() % (vocab // 3) + vocab // 3).int())
    logits[:, :vocab // 3] = lowest
    logits[2:, 2 * (vocab // 3):] = lowest
    loss, grad = distill_loss_grad(logits, ids, top, weight)
    check(logits, ids, top, weight, 1.0, loss, grad)
    assert not bool(grad[:, :vocab // 3].any())
    if lowest == float("-inf"):          # the teacher wants what the student cannot give
        ids[1, 0] = 0
        loss, grad = distill_loss_grad(logits, ids, top, weight)
        assert float(loss[1]) == float("inf") and bool(grad.isfinite().all()) and float(grad[1, 0]) < 0
        logits[4] = lowest               # nothing but -inf: no distribution
        loss, grad = distill_loss_grad(logits, ids, top, weight)
        assert bool(loss[4].isnan()) and bool(grad[4].isnan().all()) and bool(loss[[0, 2, 3]].isfinite().all())


def test_nan_stays_in_its_row():
    rng = np.random.default_rng(12)
    logits, ids, top, weight = make(rng, 6, 40000, 8, "bf16")
    clean = distill_loss_grad(logits, ids, top, weight)
    logits[1, 39999] = float("nan")
    logits[2, 17] = float("inf")
    top[3, 4] = float("nan")
    top[4, 4] = float("inf")
    weight[5] = float("nan")
    loss, grad = distill_loss_grad(logits, ids, top, weight)
    assert bool(loss[1:].isnan().all()) and bool(grad[1:3].isnan().any(dim=1).all()) and bool(grad[5].isnan().all())
    assert torch.equal(loss[0], clean[0][0]) and torch.equal(grad[0], clean[1][0])


def test_far_offsets():
    """A leading dimension past 32 bits."""
    rng = np.random.default_rng(13)
    logits, ids, top, weight = make(rng, 2, 1003, 8, "bf16")
    ld = 2 ** 31 + 8
    buf = torch.empty(ld + 1003, dtype=torch.bfloat16, device="cuda")
    view = buf.as_strided((2, 1003), (ld, 1))
    view.copy_(logits)
    want = distill_loss_grad(logits, ids, top, weight)
    loss, _ = distill_loss_grad(view, ids, top, weight, dlogits=view)
    check(logits, ids, top, weight, 1.0, loss, view)
    assert torch.equal(loss[0], want[0][0])     # row 1 starts on another boundary of 16 bytes there: its terms are added in other groups


def test_captured_on_two_streams():
    rng = np.random.default_rng(14)
    logits, ids, top, weight = make(rng, 40, 70001, 16, "bf16")
    want = distill_loss_grad(logits, ids, top, weight)
    graphs, got = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(distill_loss_grad(logits, ids, top, weight))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for outs in got:
            for t in outs:
                t.fill_(-3.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for outs in got for a, b in zip(outs, want))


def test_empty_and_refused():
    rng = np.random.default_rng(15)
    logits, ids, top, weight = make(rng, 3, 100, 4, "bf16")
    loss, grad = distill_loss_grad(logits[:0], ids[:0], top[:0], weight[:0])
    assert loss.shape == (0,) and grad.shape == (0, 100)
    for bad in ((logits.half(), ids, top, weight), (logits, ids.long(), top, weight), (logits, ids, top.double(), weight),
                (logits, ids[:2], top, weight), (logits, ids, top, weight[:2]), (logits.t(), ids, top, weight), (logits.cpu(), ids, top, weight)):
        with pytest.raises(ValueError):
            distill_loss(*bad)
    with pytest.raises(ValueError):
        distill_loss_grad(logits, ids, top, weight, dlogits=logits[:2])
    with pytest.raises(binding.SsnError):
        distill_loss(logits, ids, top, weight, temperature=0.0)
