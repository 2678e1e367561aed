"""Every kernel that the stage operators' dispatch can pick (on 148 SMs), with the loops that only large calls reach: several tiles per
CTA, more steps than stages, a ring that wraps between tiles, several rows and tokens per CTA.  Each test asserts which kernel
ran (ssn_last_kernel), so that a dispatch that changes cannot drift away from what is checked."""

import numpy as np
import pytest
import torch

from oracle import stage_oracle as so
from paper_2607_13332_b200 import binding as B
from paper_2607_13332_b200.stage_ops import distill_loss, distill_loss_grad, int8_matmul, int8_quantize
from tests import test_gpu_stage_rope as rope
from tests.test_gpu_stage_distill import TORCH, make
from tests.test_gpu_stage_distill_rows import assert_rows
from tests.test_gpu_stage_int8 import expected, operands, same

pytestmark = pytest.mark.gpu

DOT, UMMA = B.STAGE_KERNEL_INT8_DOT, B.STAGE_KERNEL_INT8_UMMA
PAIR, SWAP, SPLIT, ANYWHERE = B.STAGE_KVAR_PAIR, B.STAGE_KVAR_SWAP, B.STAGE_KVAR_SPLIT, B.STAGE_KVAR_ANYWHERE


# ---- products -----------------------------------------------------------------------------------------------------------------
PRODUCTS = [
    # tokens, inner, outer, family, variant: the tiles per CTA (or pair) behind them
    (2500, 2000, 5003, UMMA, 256 | PAIR),             # 2.7
    (3001, 1800, 12000, UMMA, 256 | PAIR),            # 7.6
    (777, 2000, 5003, UMMA, 256),                     # 0.9
    (4099, 1040, 5003, UMMA, 256),                    # 4.5
    (1003, 700, 8001, UMMA, 256),                     # 1.7
    (1000, 1040, 2000, UMMA, 128),                    # 0.9
    (30001, 1000, 100, UMMA, 128),                    # 1.6
    (60001, 1000, 101, UMMA, 128),                    # 3.2
    (2, 4000, 20003, UMMA, 16 | SWAP),                # 1.1
    (13, 1400, 60003, UMMA, 16 | SWAP),               # 3.2
    (27, 1400, 60003, UMMA, 32 | SWAP),
    (51, 1400, 60003, UMMA, 64 | SWAP),
    (5, 4096, 515, UMMA, 16 | SWAP | SPLIT),
    (20, 4090, 515, UMMA, 32 | SWAP | SPLIT),
    (60, 4096, 515, UMMA, 64 | SWAP | SPLIT),
    (100, 4000, 300, UMMA, 64 | SWAP | SPLIT),
    (1, 4096, 4099, DOT, 1),
    (2, 4000, 4099, DOT, 2),
]


def check_product(rng, n, inner, outer, dtype, family, variant, **at):
    xq, xs, wq, ws = operands(rng, n, inner, outer, **at)
    want = expected(xq, xs, wq, ws, dtype)
    item = TORCH[dtype].itemsize
    # rows of the output close together, on 16-byte boundaries, and off them
    for pitch, off in ((outer, 0), (-(-outer // 8) * 8 + 8, 0), (outer + 3, 1)):
        buf = torch.full((n * pitch + off + 16 // item,), 99.0, dtype=TORCH[dtype], device="cuda")
        out = buf[off:off + n * pitch].view(n, pitch)[:, :outer]
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        int8_matmul(xq, xs, wq, ws, dtype, out=out, dev_status=status)
        assert B.ssn_last_kernel() == (family, variant)
        assert int(status) == 0 and same(out, want)
        out.fill_(99.0)
        assert bool((buf == 99.0).all())


@pytest.mark.parametrize("n,inner,outer,family,variant", PRODUCTS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products(n, inner, outer, family, variant, dtype):
    check_product(np.random.default_rng(n + inner), n, inner, outer, dtype, family, variant)


@pytest.mark.parametrize("n,inner,outer,family,variant", [
    (8, 1401, 60003, UMMA, 16 | SWAP),                # 3.2 tiles per CTA
    (2, 4001, 20003, UMMA, 16 | SWAP),
    (9, 4095, 300, UMMA, 16 | SWAP | SPLIT),
    (40, 1401, 60003, UMMA, 64 | SWAP),
    (40, 4095, 300, UMMA, 64 | SWAP | SPLIT),
    (130, 4095, 300, UMMA, 64 | SWAP | SPLIT),
    (3001, 1401, 1003, UMMA, 128),                    # 1.3
    (5000, 1001, 2003, UMMA, 128),                    # 4.3
    (1, 4001, 4099, DOT, 1),
    (2, 4001, 4099, DOT, 2),
])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products_of_rows_anywhere(n, inner, outer, family, variant, dtype):
    check_product(np.random.default_rng(n + inner), n, inner, outer, dtype, family, variant | ANYWHERE, x_pitch=inner, w_pitch=inner + 2, x_at=3, w_at=5)


@pytest.mark.parametrize("n,inner,outer", [(2500, 2000, 5003), (4099, 1040, 5003), (51, 1400, 60003)])
def test_products_behind_one_another(n, inner, outer):
    """Large calls that start before the one in front has ended, on two streams: each gives what it gave alone."""
    rng = np.random.default_rng(outer)
    sets = [operands(rng, n, inner, outer), operands(rng, n // 2, inner, outer)]
    want = [int8_matmul(*s) for s in sets]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(40):
        with torch.cuda.stream(streams[i & 1]):
            outs.append((int8_matmul(*sets[(i >> 1) & 1]), want[(i >> 1) & 1]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in outs)


# ---- quantisation -------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("pieces,variant", [(1, 2 | 2 << 4), (128, 2 | 2 << 4), (129, 4 | 2 << 4), (512, 4 | 4 << 4), (1000, 4 | 8 << 4), (2048, 4 | 16 << 4),
                                            (2049, 8 | 16 << 4), (4096, 8 | 16 << 4), (4097, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantisation(pieces, variant, dtype):
    rng = np.random.default_rng(pieces)
    item = TORCH[dtype].itemsize
    cols = pieces * (16 // item) - 1                        # the last piece short of an element
    pitch = -(-cols // 16) * 16
    x = torch.zeros(70, pitch, dtype=TORCH[dtype], device="cuda")[:, :cols]
    x.copy_(torch.from_numpy(rng.standard_normal((70, cols)).astype(np.float32)))
    q, scale = int8_quantize(x)
    assert B.ssn_last_kernel() == (B.STAGE_KERNEL_QUANTIZE, variant)
    want, want_scale = so.int8_quantize(x.double().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_scale) and np.array_equal(q.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantisation_of_many_rows_anywhere(dtype):
    """More rows than blocks, none on a 16-byte boundary: 1184 blocks take them in turn."""
    rng = np.random.default_rng(6)
    x = torch.from_numpy(rng.standard_normal((5001, 301)).astype(np.float32)).to(TORCH[dtype]).cuda()
    x[1::7] *= 100.0
    x[2::7] = 0.0
    q, scale = int8_quantize(x)
    assert B.ssn_last_kernel() == (B.STAGE_KERNEL_QUANTIZE, 0)
    want, want_scale = so.int8_quantize(x.double().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), want_scale) and np.array_equal(q.cpu().numpy(), want)


# ---- the loss -----------------------------------------------------------------------------------------------------------------
def distill_variant(many, cluster, grad):
    return B.STAGE_KERNEL_DISTILL, cluster | (B.STAGE_KVAR_MANY if many else 0) | (B.STAGE_KVAR_GRAD if grad else 0)


@pytest.mark.parametrize("n,vocab,k,dtype,many", [
    (5000, 1003, 7, "bf16", False),      # 1184 CTAs with the gradient, 1480 without: four rows each, starting anywhere in 16 bytes
    (5000, 1000, 200, "f32", False),     # more entries than threads
    (3601, 517, 130, "f32", False),
    (1501, 50001, 9, "bf16", True),      # 444 and 592 CTAs
    (1501, 25001, 300, "f32", True),
    (1300, 49152, 64, "bf16", True),
])
def test_several_rows_per_block(n, vocab, k, dtype, many):
    """Rows with nothing to learn, of weight 0 or NaN, and live ones follow one another on a CTA in every order."""
    rng = np.random.default_rng(n + vocab)
    dt = TORCH[dtype]
    logits = torch.randn(n, vocab, device="cuda", generator=torch.Generator("cuda").manual_seed(n)).mul_(2.5).to(dt)
    ids = torch.from_numpy(rng.integers(0, vocab, (n, k)).astype(np.int32)).cuda()
    ids[torch.from_numpy(rng.random((n, k)) < 0.2).cuda()] = -1
    top = torch.from_numpy((6 + 1.5 * rng.standard_normal((n, k))).astype(np.float32)).cuda()
    weight = torch.from_numpy(rng.uniform(0.1, 2.0, n).astype(np.float32)).cuda()
    dead = torch.from_numpy(rng.random(n) < 0.4).cuda()
    kind = torch.from_numpy(rng.integers(0, 3, n)).cuda()
    weight[dead & (kind == 0)] = 0.0
    logits[dead & (kind == 0)] = float("nan")
    ids[dead & (kind == 1)] = -1
    top[dead & (kind == 2)] = float("-inf")
    poisoned = torch.tensor([5, n - 3], device="cuda")
    weight[poisoned], dead[poisoned] = float("nan"), False
    ids[poisoned] = 1
    top[poisoned] = 0.0
    logits[poisoned] = 1.0
    loss, grad = distill_loss_grad(logits, ids, top, weight, temperature=1.3)
    assert B.ssn_last_kernel() == distill_variant(many, 1, True)
    alone = distill_loss(logits, ids, top, weight, temperature=1.3)
    assert B.ssn_last_kernel() == distill_variant(many, 1, False)
    assert not bool(loss[dead].any()) and not bool(grad[dead].any())
    assert bool(loss[poisoned].isnan().all()) and bool(grad[poisoned].isnan().all())
    live = ~dead
    live[poisoned] = False
    assert torch.equal(alone[~live].nan_to_num(7.0), loss[~live].nan_to_num(7.0)) and torch.equal(alone[live], loss[live])
    # rows of every turn, and the last ones
    rows = live.nonzero()[:, 0].cpu().numpy()
    at = torch.from_numpy(np.unique(np.concatenate((rng.choice(rows, 150), rows[-20:], rows[:20])))).cuda()
    assert_rows(logits[at], ids[at], top[at], weight[at], 1.3, loss[at], grad[at])
    if vocab % 8 == 0:      # the same rows taken by other CTAs at other turns, all on one boundary: the same bits
        loss2, grad2 = distill_loss_grad(*(t.roll(-1040, 0) for t in (logits, ids, top, weight)), temperature=1.3)
        assert torch.equal(loss2.roll(1040, 0)[live], loss[live]) and torch.equal(grad2.roll(1040, 0)[live], grad[live])


@pytest.mark.parametrize("n,vocab,dtype,many,cluster", [(1, 128256, "bf16", True, 8), (19, 128256, "bf16", True, 8), (37, 128256, "bf16", True, 8), (74, 128256, "bf16", True, 4),
                                                        (75, 128256, "bf16", True, 2), (148, 70000, "bf16", True, 2), (149, 70000, "bf16", True, 1),
                                                        (18, 50000, "f32", True, 8), (5, 12000, "bf16", False, 4), (5, 4000, "f32", False, 2), (5, 24000, "f32", False, 8), (3, 500, "f32", False, 1)])
def test_rows_shared_by_clusters(n, vocab, dtype, many, cluster):
    rng = np.random.default_rng(n + vocab)
    logits, ids, top, weight = make(rng, n, vocab, 21, dtype, 0.2)
    loss, grad = distill_loss_grad(logits, ids, top, weight)
    assert B.ssn_last_kernel() == distill_variant(many, cluster, True)
    assert torch.equal(distill_loss(logits, ids, top, weight), loss)
    assert B.ssn_last_kernel() == distill_variant(many, cluster, False)
    at = torch.from_numpy(np.unique(np.concatenate(([0, n - 1], rng.integers(0, n, 12))))).cuda()
    assert_rows(logits[at], ids[at], top[at], weight[at], 1.0, loss[at], grad[at])


# ---- query/key norm with rotation ---------------------------------------------------------------------------------------------
ADJ, CROSS, FULL = B.STAGE_KVAR_ADJACENT, B.STAGE_KVAR_CROSSED, B.STAGE_KVAR_FULL
ROPE = [
    # (n, q heads, k heads, D, rot, dtype, pairing, layout, positions), variant forward, and back where it is another
    ((6001, 5, 1, 128, 128, "bf16", "halves", "packed", True), 8 | FULL, None),
    ((6001, 5, 1, 128, 128, "bf16", "adjacent", "heads", False), 8 | ADJ | FULL, None),
    ((6001, 3, 2, 64, 64, "f32", "halves", "packed", True), 4 | FULL, None),
    ((6001, 3, 2, 64, 64, "f32", "adjacent", "plain", True), 4 | ADJ | FULL, None),
    ((3001, 5, 2, 128, 96, "bf16", "halves", "heads", True), 8, None),
    ((3001, 5, 2, 128, 96, "bf16", "adjacent", "heads", True), 8 | ADJ, None),
    ((3001, 4, 1, 96, 96, "f32", "halves", "packed", False), 4, None),
    ((3001, 4, 1, 96, 64, "f32", "adjacent", "packed", False), 4 | ADJ, None),
    ((3001, 4, 1, 72, 72, "bf16", "halves", "plain", False), 4, None),
    ((3001, 4, 1, 72, 72, "bf16", "adjacent", "plain", False), 4 | ADJ, None),
    ((3001, 3, 1, 20, 12, "bf16", "halves", "heads", True), 2, None),
    ((3001, 3, 1, 20, 12, "bf16", "adjacent", "heads", True), 2 | ADJ, None),
    ((3001, 3, 1, 20, 12, "f32", "halves", "heads", True), 2, None),
    ((3001, 3, 1, 20, 12, "f32", "adjacent", "heads", True), 2 | ADJ, None),
    ((1501, 3, 2, 64, 64, "bf16", "halves", "odd", True), 1, None),
    ((1501, 3, 2, 256, 200, "bf16", "adjacent", "odd", True), 1 | ADJ, None),
    ((1501, 3, 2, 256, 200, "f32", "halves", "odd", False), 1, None),
    ((1501, 3, 2, 64, 64, "f32", "adjacent", "odd", False), 1 | ADJ, None),
    ((3001, 7, 2, 128, 98, "bf16", "halves", "packed", True), 8 | CROSS, 4 | CROSS),
    ((3001, 7, 2, 72, 34, "bf16", "halves", "plain", True), 4 | CROSS, None),
    ((3001, 5, 2, 96, 30, "f32", "halves", "packed", True), 4 | CROSS, None),
    ((3001, 4, 1, 96, 0, "bf16", "halves", "plain", False), 8, None),
]


@pytest.mark.parametrize("case,forward,back", ROPE, ids=lambda c: "-".join(map(str, c)) if isinstance(c, tuple) else str(c))
def test_norm_and_rotation(case, forward, back):
    """Several tokens per warp, the last ones of a warp's row short."""
    op, q, k, wq, wk, pos, seq, rows, rng, layout, dt = rope.setup(case)
    n, pairing, rot = case[0], case[6], case[4]
    got = op.forward(q, k, pos=pos, seq_len=seq)
    assert B.ssn_last_kernel() == (B.STAGE_KERNEL_ROPE, forward)
    grads = [rope.heads(rng, n, x.shape[1], x.shape[2], dt, layout)[0] for x in (q, k)]
    outs = [rope.heads(rng, n, x.shape[1], x.shape[2], dt, layout) for x in (q, k)]
    back_got = op.backward(*grads, q, k, pos=pos, seq_len=seq, dq_in=outs[0][0], dk_in=outs[1][0])
    assert B.ssn_last_kernel() == (B.STAGE_KERNEL_ROPE, (forward if back is None else back) | B.STAGE_KVAR_BACK)
    for i, (x, w, dy, (out, buf)) in enumerate(zip((q, k), (wq, wk), grads, outs)):
        x64, w64, dy64 = rope.f64(x), rope.f64(w), rope.f64(dy)
        unit, r = so.qk_norm(x64, None, rope.EPS)
        want = so.qk_rope_forward(x64, w64, rows, pairing, rope.EPS)
        rope.check(got[i], want, 20 * rope.U * rope.pair_bound(unit * w64, rot, pairing), dt, "forward")
        dx, dw = so.qk_rope_backward(dy64, x64, w64, rows, pairing, rope.EPS)
        u, g = np.abs(unit), rope.pair_bound(dy64, rot, pairing)
        h = g * np.abs(w64)
        rope.check(out, dx, 40 * rope.U * r * (h + u * (h * u).mean(axis=-1, keepdims=True)), dt, "backward")
        rope.check(back_got[2 + i], dw, 150 * rope.U * (g * u).sum(axis=(0, 1)), torch.float32, "gain")
        assert rope.untouched(out, buf)
    assert op.take_status() == 0
