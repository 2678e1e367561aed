"""Query/key norm with rotary positions against the oracle in 64 bits, forward and backward.

Tolerances: an output is rounded once (half a step, eps / 2 of its type) from fp32 values.  A normed value carries the sum of
squares (at most 16 terms in a row and 5 pairwise steps, halved by the root), the root, two products and the two products and
sum of the rotation: 20 roundings of 2^-24 relative to the pair's values cover them.  The gradient adds a second sum of that
length and two products: 40."""

import numpy as np
import pytest
import torch

from oracle import stage_oracle as so
from paper_2607_13332_b200 import binding
from paper_2607_13332_b200.stage_ops import QKNormRope, rope_table

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def heads(rng, n, h, d, dt, layout, scale=1.0):
    """[n, h, d] values in one of the layouts, inside a buffer with a sentinel around."""
    x = torch.from_numpy((scale * rng.standard_normal((n, h, d))).astype(np.float32)).to(dt)
    if layout == "packed":            # a view of a wider row
        buf = torch.full((n + 2, h * d + 2 * d), 77.0, dtype=dt, device="cuda")
        view = buf[1:n + 1, d:d + h * d].unflatten(1, (h, d))
    elif layout == "heads":           # head-major
        buf = torch.full((h + 2, n, d), 77.0, dtype=dt, device="cuda")
        view = buf[1:h + 1].transpose(0, 1)
    elif layout == "odd":             # nothing on a 16-byte boundary
        buf = torch.full((n * h * (d + 1) + 9,), 77.0, dtype=dt, device="cuda")
        view = buf[1:1 + n * h * (d + 1)].view(n, h, d + 1)[..., :d]
    else:
        buf = torch.full((n, h, d), 77.0, dtype=dt, device="cuda")
        view = buf
    view.copy_(x)
    return view, buf


def untouched(view, buf):
    """Nothing but the view was written."""
    keep = view.clone()
    view.fill_(77.0)
    ok = bool((buf == 77.0).all())
    view.copy_(keep)
    return ok


def pair_bound(x, rot, pairing):
    """|a| + |b| of the pair a value stands in."""
    out = np.abs(x)
    a, b = so.pair_columns(rot, pairing)
    both = out[..., a] + out[..., b]
    out[..., a], out[..., b] = both, both
    return out


def check(got, want, bound, dt, what):
    limit = torch.finfo(dt).eps / 2 * np.abs(want) * (1 + 1e-6) + bound + 1e-37
    bad = ~(np.abs(f64(got) - want) <= limit)      # a NaN is off
    assert not bad.any(), f"{what}: {bad.sum()} values off, worst {np.max(np.abs(f64(got) - want) / limit):.2f} of the limit"


CASES = [
    # n, q heads, k heads, D, rot, dtype, pairing, layout, positions
    (1, 32, 8, 128, 128, "bf16", "halves", "packed", True),
    (5, 3, 1, 128, 128, "bf16", "adjacent", "plain", False),
    (300, 7, 2, 128, 96, "bf16", "halves", "heads", True),
    (2001, 32, 8, 128, 128, "bf16", "halves", "packed", False),
    (65, 4, 4, 64, 64, "f32", "halves", "packed", True),
    (130, 5, 3, 80, 64, "f32", "adjacent", "heads", True),
    (33, 2, 1, 256, 256, "bf16", "halves", "plain", False),
    (33, 2, 2, 256, 100, "f32", "halves", "packed", True),
    (17, 3, 2, 256, 256, "bf16", "adjacent", "odd", True),
    (40, 3, 2, 256, 250, "f32", "halves", "odd", False),
    (40, 3, 1, 96, 0, "bf16", "halves", "plain", False),
    (9, 1, 1, 2, 2, "bf16", "adjacent", "plain", True),
    (9, 2, 1, 6, 2, "f32", "halves", "plain", True),
    (50, 2, 1, 20, 12, "bf16", "adjacent", "heads", True),
    (50, 40, 0, 192, 128, "bf16", "halves", "packed", True),
    (50, 0, 5, 112, 48, "f32", "adjacent", "plain", False),
    # halves at distances that no wide piece divides
    (130, 7, 2, 128, 98, "bf16", "halves", "packed", True),
    (65, 3, 1, 80, 34, "bf16", "halves", "heads", False),
    (21, 5, 2, 256, 2, "bf16", "halves", "plain", True),
    (21, 5, 2, 256, 254, "f32", "halves", "plain", True),
    (33, 2, 1, 96, 30, "f32", "halves", "packed", True),
    (301, 6, 1, 72, 36, "bf16", "halves", "plain", False),
    (11, 3, 2, 24, 22, "bf16", "halves", "plain", True),
    (11, 3, 2, 8, 6, "f32", "halves", "heads", True),
    (77, 9, 3, 128, 98, "bf16", "adjacent", "heads", True),
    (77, 9, 3, 72, 70, "f32", "adjacent", "packed", False),
]


def setup(case, seed=0):
    n, qh, kh, d, rot, dtype, pairing, layout, explicit = case
    rng = np.random.default_rng(n + d + seed)
    dt = TORCH[dtype]
    q, qb = heads(rng, n, qh, d, dt, layout, 3.0) if qh else (None, None)
    k, kb = heads(rng, n, kh, d, dt, layout, 0.2) if kh else (None, None)
    wq = torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).to(dt).cuda()
    wk = None if n == 33 else torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).to(dt).cuda()
    max_pos, seq = 700, 300
    table = rope_table(max_pos, rot, 500.0) if rot else None
    op = QKNormRope(dtype, d, wq, wk, table, eps=EPS, pairing=pairing)
    at = rng.integers(0, max_pos, n) if explicit else np.arange(n) % seq
    pos = torch.from_numpy(at.astype(np.int32)).cuda() if explicit else None
    rows = so.table_rows(f64(table), at)[0] if rot else np.zeros((n, 0))
    return op, q, k, wq, wk, pos, seq, rows, rng, layout, dt


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_forward(case):
    op, q, k, wq, wk, pos, seq, rows, rng, layout, dt = setup(case)
    n, pairing, rot = case[0], case[6], case[4]
    outs = [heads(rng, n, x.shape[1], x.shape[2], dt, layout) if x is not None else (None, None) for x in (q, k)]
    op.forward(q, k, pos=pos, seq_len=seq, q_out=outs[0][0], k_out=outs[1][0])
    fresh = op.forward(q, k, pos=pos, seq_len=seq)
    for x, w, (out, buf), again in zip((q, k), (wq, wk), outs, fresh):
        if x is None:
            assert again is None
            continue
        want = so.qk_rope_forward(f64(x), f64(w), rows, pairing, EPS)
        check(out, want, 20 * U * pair_bound(so.qk_norm(f64(x), f64(w), EPS)[0], rot, pairing), dt, "forward")
        assert untouched(out, buf)
        assert torch.equal(again, out)
    assert op.take_status() == 0


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_backward(case):
    op, q, k, wq, wk, pos, seq, rows, rng, layout, dt = setup(case)
    n, pairing, rot = case[0], case[6], case[4]
    grads = [heads(rng, n, x.shape[1], x.shape[2], dt, "plain")[0] if x is not None else None for x in (q, k)]
    outs = [heads(rng, n, x.shape[1], x.shape[2], dt, layout) if x is not None else (None, None) for x in (q, k)]
    got = op.backward(*grads, q, k, pos=pos, seq_len=seq, dq_in=outs[0][0], dk_in=outs[1][0])
    again = op.backward(*grads, q, k, pos=pos, seq_len=seq)
    for i, (x, w, dy, (out, buf)) in enumerate(zip((q, k), (wq, wk), grads, outs)):
        if x is None:
            assert not bool(got[2 + i].any())      # a side without rows has a gain gradient of zeros
            continue
        dx, dw = so.qk_rope_backward(f64(dy), f64(x), f64(w), rows, pairing, EPS)
        u = np.abs(f64(x)) * so.qk_norm(f64(x), None, EPS)[1]
        g = pair_bound(f64(dy), rot, pairing)
        h = g if w is None else g * np.abs(f64(w))
        r = so.qk_norm(f64(x), None, EPS)[1]
        check(out, dx, 40 * U * r * (h + u * (h * u).mean(axis=-1, keepdims=True)), dt, "backward")
        # at most 100 rows per lane one after the other, 13 steps over lanes and warps, then 64 bits
        check(got[2 + i], dw, 150 * U * (g * u).sum(axis=(0, 1)), torch.float32, "gain")
        assert untouched(out, buf) and torch.equal(again[i], out) and torch.equal(again[2 + i], got[2 + i])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 20)])
def test_gains_without_eps(dtype, d):
    """eps = 0: lanes without a head add nothing, although the root of their zeros is infinite."""
    rng, dt = np.random.default_rng(d), TORCH[dtype]
    q, k, dq, dk = (heads(rng, 7, h, d, dt, "plain")[0] for h in (5, 1, 5, 1))
    got = QKNormRope(dtype, d, eps=0.0).backward(dq, dk, q, k)
    for x, dy, dx, dw in zip((q, k), (dq, dk), got[:2], got[2:]):
        want_x, want_w = so.qk_rope_backward(f64(dy), f64(x), None, np.zeros((7, 0)), "halves", 0.0)
        r = so.qk_norm(f64(x), None, 0.0)[1]
        u, g = np.abs(f64(x)) * r, np.abs(f64(dy))
        check(dx, want_x, 40 * U * r * (g + u * (g * u).mean(axis=-1, keepdims=True)), dt, "backward")
        check(dw, want_w, 150 * U * (g * u).sum(axis=(0, 1)), torch.float32, "gain")


def test_in_place_and_without_gains():
    op, q, k, wq, wk, pos, seq, rows, rng, layout, dt = setup(CASES[3])
    want = op.forward(q, k, pos=pos, seq_len=seq)
    dq, dk = torch.randn_like(want[0]), torch.randn_like(want[1])
    grads = op.backward(dq, dk, q, k, pos=pos, seq_len=seq)
    dq2, dk2 = dq.clone(), dk.clone()
    back = op.backward(dq2, dk2, q, k, pos=pos, seq_len=seq, dq_in=dq2, dk_in=dk2, gains=False)
    assert back[2] is None and torch.equal(dq2, grads[0]) and torch.equal(dk2, grads[1])
    op.forward(q, k, pos=pos, seq_len=seq, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_positions_outside_the_table():
    op, q, k, wq, wk, _, seq, _, rng, layout, dt = setup((6, 4, 2, 64, 48, "bf16", "halves", "plain", True))
    at = np.array([0, 699, 700, -1, 2 ** 31 - 1, 5])
    pos = torch.from_numpy(at.astype(np.int32)).cuda()
    rows, bad = so.table_rows(f64(op.table), at)
    assert bad
    out = op.forward(q, k, pos=pos)
    assert op.take_status() == binding.SSN_DEV_BAD_POS and op.take_status() == 0
    want = so.qk_rope_forward(f64(q), f64(wq), rows, "halves", EPS)
    check(out[0], want, 20 * U * pair_bound(so.qk_norm(f64(q), f64(wq), EPS)[0], 48, "halves"), dt, "forward")
    assert not bool(out[0][2:5, :, :48].any())


def test_rows_keep_to_themselves():
    """A row of zeros, one of infinities and one with a NaN leave the others as they were."""
    op, q, k, wq, wk, pos, seq, rows, rng, layout, dt = setup((40, 4, 2, 128, 128, "bf16", "halves", "plain", True))
    clean = op.forward(q, k, pos=pos)
    q[3, 1] = 0.0
    q[7, 2] = float("inf")
    q[9, 0, 5] = float("nan")
    out = op.forward(q, k, pos=pos)
    assert not bool(out[0][3, 1].any()) and bool(out[0][7, 2].isnan().all()) and bool(out[0][9, 0].isnan().all())
    for t, h in ((3, 1), (7, 2), (9, 0)):
        out[0][t, h] = clean[0][t, h]
    assert torch.equal(out[0], clean[0]) and torch.equal(out[1], clean[1])


def test_broadcast_gradient_and_repeated_rows():
    """Inputs of stride 0: a gradient that every token shares, one row of queries for all heads."""
    op, q, k, wq, wk, pos, seq, rows, rng, layout, dt = setup((70, 8, 2, 64, 64, "f32", "halves", "plain", True))
    dq = torch.randn(1, 8, 64, device="cuda").expand(70, 8, 64)
    q1 = q[:, :1].expand(70, 8, 64)
    got = op.backward(dq, None, q1, None, pos=pos)
    want = op.backward(dq.contiguous(), None, q1.contiguous(), None, pos=pos)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


def test_empty_calls():
    op = QKNormRope("bf16", 64, table=rope_table(8, 64))
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    assert op.forward(q, None, seq_len=4)[0].shape == (0, 4, 64)
    out = op.backward(q, None, q, None, seq_len=4)
    torch.cuda.synchronize()
    assert not bool(out[2].any()) and not bool(out[3].any())


def test_far_offsets():
    """A token stride past 32 bits, in elements and in bytes."""
    stride = 2 ** 31 + 64
    buf = torch.empty(2 * stride, dtype=torch.bfloat16, device="cuda")
    q = buf.as_strided((2, 3, 64), (stride, 64, 1))
    q.copy_(torch.randn(2, 3, 64, device="cuda"))
    op = QKNormRope("bf16", 64, table=rope_table(8, 64))
    want = op.forward(q.contiguous(), None, seq_len=4)[0]
    op.forward(q, None, seq_len=4, q_out=q)
    assert torch.equal(q, want)


@pytest.mark.parametrize("rot,theta", [(128, 10000.0), (64, 500000.0), (2, 10.0)])
def test_table(rot, theta):
    got = rope_table(131072, rot, theta).cpu().numpy().astype(np.float64)
    want = so.rope_table(131072, rot, theta)
    assert np.abs(got - want).max() <= 2.0 ** -25 + 1e-9      # half a step below 1, and the angle's own error in 64 bits


def test_captured_and_on_two_streams():
    """Two captured passes that share no workspace, replayed at once on two streams, against an eager pass."""
    op, q, k, wq, wk, pos, seq, rows, rng, layout, dt = setup(CASES[3])
    dq, dk = torch.randn(q.shape, device="cuda").to(dt), torch.randn(k.shape, device="cuda").to(dt)
    want = op.forward(q, k, seq_len=seq) + op.backward(dq, dk, q, k, seq_len=seq)
    graphs, got = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(op.forward(q, k, seq_len=seq) + op.backward(dq, dk, q, k, seq_len=seq))
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
        for outs in got:
            for a, b in zip(outs, want):
                assert torch.equal(a, b)


def test_python_refusals():
    op = QKNormRope("bf16", 64, table=rope_table(8, 64))
    good = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (good.float(), good[..., :32], good.transpose(1, 2), good.cpu()):
        with pytest.raises(ValueError):
            op.forward(bad, None, seq_len=4)
    with pytest.raises(ValueError):
        op.forward(good, None, pos=torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError):
        op.forward(good, None, pos=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        op.backward(None, None, good, None, seq_len=4)
    with pytest.raises(ValueError):
        op.forward(None, None)
    with pytest.raises(binding.SsnError):
        op.forward(good, None, seq_len=0)
    with pytest.raises(ValueError):
        QKNormRope("bf16", 64, wq=torch.ones(63, dtype=torch.bfloat16, device="cuda"))
