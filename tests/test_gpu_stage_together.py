"""The stage operators one after the other, as a distilling stage runs them next to the codec: a frozen teacher whose products
are in 8 bits (expansion of what arrives, norm of the block, projection, query/key norm with rotation, head, top logits), the
student's loss and gradients, and what goes back over the boundary.  Every step is held to the oracle on the values that the
step before it really gave, on a stream of its own, and once more as one captured graph."""

import numpy as np
import pytest
import torch

from oracle import ssn_oracle, stage_oracle as so
from oracle.metrics import max_rel_err
from paper_2607_13332_b200 import binding, stage_ops, synth
from paper_2607_13332_b200.runner import Codec, to_device

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
D, K, SEQ, SEQS, VOCAB, HEADS, KV, HEAD = 512, 40, 96, 3, 2011, 6, 2, 64
TOKENS, TOP = SEQ * SEQS, 24


def f64(t):
    return t.detach().double().cpu().numpy()


def half(t):
    return torch.finfo(t.dtype).eps / 2


@pytest.fixture(scope="module")
def setup():
    wl = synth.Workload("together", D, K, VOCAB, SEQS, SEQ, synth.BF16, "zipf")
    t = synth.codec_inputs(wl, seed=21)
    rng = np.random.default_rng(22)
    dev = lambda a: torch.from_numpy(a.astype(np.float32)).cuda().bfloat16()
    codec = Codec(synth.BF16, to_device(t["U"], synth.BF16), to_device(t["E"], synth.BF16))
    weights = {n: dev(rng.standard_normal((rows, D)) / np.sqrt(D)) for n, rows in (("qkv", (HEADS + 2 * KV) * HEAD), ("head", VOCAB), ("student", VOCAB))}
    rope = stage_ops.QKNormRope("bf16", HEAD, dev(1 + 0.1 * rng.standard_normal(HEAD)), dev(1 + 0.1 * rng.standard_normal(HEAD)),
                                stage_ops.rope_table(256, HEAD), eps=1e-6)
    data = {"Z": to_device(t["Z0"], synth.BF16), "ids": torch.from_numpy(t["ids"]).cuda(), "weight": torch.full((TOKENS,), 1.0 / TOKENS, device="cuda"),
            "dq": dev(rng.standard_normal((TOKENS, HEADS, HEAD))), "dk": dev(rng.standard_normal((TOKENS, KV, HEAD)))}
    data["weight"][::17] = 0.0
    frozen = {n: stage_ops.int8_quantize(weights[n]) for n in ("qkv", "head")}
    return codec, weights, rope, data, frozen


def run(codec, weights, rope, data, frozen):
    r = {}
    r["x"], r["stat"] = codec.decompress_rowsumsq(data["Z"], data["ids"])
    r["normed"] = (r["x"].float() * torch.rsqrt(r["stat"] / D + 1e-6)[:, None]).bfloat16()
    r["xq"], r["xs"] = stage_ops.int8_quantize(r["normed"])
    r["qkv"] = stage_ops.int8_matmul(r["xq"], r["xs"], *frozen["qkv"])
    heads = r["qkv"].view(TOKENS, HEADS + 2 * KV, HEAD)
    q, k = heads[:, :HEADS], heads[:, HEADS:HEADS + KV]
    r["q"], r["k"] = rope.forward(q, k, seq_len=SEQ)
    r["dq"], r["dk"], r["dwq"], r["dwk"] = rope.backward(data["dq"], data["dk"], q, k, seq_len=SEQ)
    r["teacher"] = stage_ops.int8_matmul(r["xq"], r["xs"], *frozen["head"], dtype="f32")
    r["top"], ids = torch.topk(r["teacher"], TOP, dim=1)
    r["ids"] = ids.int()
    r["logits"] = r["normed"] @ weights["student"].t()
    r["loss"], r["dlogits"] = stage_ops.distill_loss_grad(r["logits"], r["ids"], r["top"], data["weight"], temperature=2.0)
    r["back"] = codec.grad_project(r["dlogits"] @ weights["student"])
    return r


def test_every_step_against_the_oracle(setup):
    codec, weights, rope, data, frozen = setup
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = run(*setup)
    side.synchronize()
    assert codec.take_status() == 0 and rope.take_status() == 0
    # the codec's own tolerance at both ends
    x, stat, _ = ssn_oracle.decompress_rowsumsq(f64(data["Z"]), f64(codec.U), f64(codec.E), data["ids"].cpu().numpy(), None, None)
    assert max_rel_err(f64(r["x"]), x) <= 1e-2 and max_rel_err(f64(r["stat"]), stat) <= 1e-5
    xq, xs = so.int8_quantize(f64(r["normed"]))
    assert np.array_equal(r["xq"].cpu().numpy(), xq) and np.array_equal(r["xs"].cpu().numpy(), xs)
    for name, out in (("qkv", r["qkv"]), ("head", r["teacher"])):
        want = so.int8_matmul(xq, xs, f64(frozen[name][0]), f64(frozen[name][1]))
        assert (np.abs(f64(out) - want) <= (half(out) + 3 * U) * np.abs(want) * (1 + 1e-6)).all()   # the sum's conversion and two products
    heads = f64(r["qkv"]).reshape(TOKENS, HEADS + 2 * KV, HEAD)
    rows, _ = so.table_rows(f64(rope.table), np.arange(TOKENS) % SEQ)
    for x, w, y, dy, dx, dw in ((heads[:, :HEADS], rope.wq, r["q"], data["dq"], r["dq"], r["dwq"]),
                                (heads[:, HEADS:HEADS + KV], rope.wk, r["k"], data["dk"], r["dk"], r["dwk"])):
        want = so.qk_rope_forward(x, f64(w), rows, "halves", 1e-6)
        n = np.abs(so.qk_norm(x, f64(w), 1e-6)[0])
        assert (np.abs(f64(y) - want) <= half(y) * np.abs(want) + 20 * U * (n + np.roll(n, HEAD // 2, axis=-1))).all()
        wdx, wdw = so.qk_rope_backward(f64(dy), x, f64(w), rows, "halves", 1e-6)
        u, rr = np.abs(so.qk_norm(x, None, 1e-6)[0]), so.qk_norm(x, None, 1e-6)[1]
        g = np.abs(f64(dy))
        g = g + np.roll(g, HEAD // 2, axis=-1)
        h = g * np.abs(f64(w))
        assert (np.abs(f64(dx) - wdx) <= half(dx) * np.abs(wdx) + 40 * U * rr * (h + u * (h * u).mean(axis=-1, keepdims=True))).all()
        assert (np.abs(f64(dw) - wdw) <= 150 * U * (g * u).sum(axis=(0, 1))).all()
    loss, dlogits = so.distill_loss(f64(r["logits"]), r["ids"].cpu().numpy(), f64(r["top"]), f64(data["weight"]), 2.0)
    assert np.abs(f64(r["loss"]) - loss).max() <= 1e-5 * np.abs(loss).max()
    assert (np.abs(f64(r["dlogits"]) - dlogits) <= half(r["dlogits"]) * np.abs(dlogits) + 1e-5 * np.abs(dlogits).max(axis=1, keepdims=True)).all()
    assert not r["dlogits"][::17].any() and not r["loss"][::17].any()
    back = ssn_oracle.grad_project_coeff(f64(r["dlogits"] @ weights["student"]), f64(codec.U))
    assert max_rel_err(f64(r["back"]), back) <= 1e-2


def test_captured_as_one_graph(setup):
    want = run(*setup)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(*setup)
    for _ in range(3):
        for name in ("q", "dq", "dwq", "loss", "dlogits", "qkv", "back"):
            got[name].fill_(7)
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[name], want[name]) for name in want)


def test_launches_are_counted(setup):
    before = binding.ssn_launch_count()
    codec, weights, rope, data, frozen = setup
    q = torch.zeros(4, HEADS, HEAD, dtype=torch.bfloat16, device="cuda")
    rope.forward(q, None, seq_len=4)
    rope.backward(q, None, q, None, seq_len=4)      # the gradients, and the gains' sums
    stage_ops.int8_matmul(*stage_ops.int8_quantize(q.view(4, -1)), *stage_ops.int8_quantize(q.view(4, -1)))
    assert binding.ssn_launch_count() - before == 6
