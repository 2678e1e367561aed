"""The stage calls by raw addresses (binding) give what the tensor layer gives, and raise what the library refuses."""

import pytest
import torch

from paper_2607_13332_b200 import binding as B
from paper_2607_13332_b200 import stage_ops

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def rows(t):
    """(address, token stride, head stride)"""
    return t.data_ptr(), t.stride(0), t.stride(1)


def test_norm_and_rotation():
    n, d = 37, 64
    heads = torch.randn(n, 8, d, device="cuda").bfloat16()
    q, k, dq, dk = heads[:, :4], heads[:, 4:6], torch.randn(n, 4, d, device="cuda").bfloat16(), torch.randn(n, 2, d, device="cuda").bfloat16()
    w = torch.rand(d, device="cuda").bfloat16()
    table = torch.empty(16, d, device="cuda")
    B.stage_rope_table(table.data_ptr(), d, 16, d, 1e4, stream())
    op = stage_ops.QKNormRope("bf16", d, w, None, table)
    want = op.forward(q, k, seq_len=16) + op.backward(dq, dk, q, k, seq_len=16)
    c = B.make_qk_rope(d, d, B.SSN_BF16, B.STAGE_PAIR_HALVES, 1e-6, w.data_ptr(), 0, table.data_ptr(), d, 16)
    got = [torch.empty_like(t) for t in want]
    B.stage_qk_rope_forward(c, rows(q), 4, rows(k), 2, rows(got[0]), rows(got[1]), 0, n, 16, stream())
    size = B.stage_qk_rope_workspace_bytes(c, n, 4, 2)
    work = torch.empty(size, dtype=torch.uint8, device="cuda")
    B.stage_qk_rope_backward(c, rows(dq), rows(dk), rows(q), 4, rows(k), 2, rows(got[2]), rows(got[3]), got[4].data_ptr(), got[5].data_ptr(), 0, n, 16,
                             work.data_ptr(), size, stream())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(B.SsnError):
        B.stage_qk_rope_forward(c, rows(q), 4, rows(k), 2, rows(got[0]), rows(got[1]), 0, n, 0, stream())
    with pytest.raises(B.SsnError):
        B.stage_qk_rope_backward(c, rows(dq), rows(dk), rows(q), 4, rows(k), 2, rows(got[2]), rows(got[3]), got[4].data_ptr(), 0, 0, n, 16,
                                 work.data_ptr(), size - 1, stream())


def test_loss():
    n, vocab, k = 9, 1003, 5
    logits, top = torch.randn(n, vocab, device="cuda"), torch.randn(n, k, device="cuda")
    ids = torch.randint(0, vocab, (n, k), dtype=torch.int32, device="cuda")
    want = stage_ops.distill_loss_grad(logits, ids, top, temperature=2.0)
    loss, grad, status = torch.empty(n, device="cuda"), torch.empty_like(logits), torch.zeros(1, dtype=torch.int32, device="cuda")
    args = (logits.data_ptr(), vocab, B.SSN_F32, n, vocab, ids.data_ptr(), k, top.data_ptr(), k, k, 0)
    B.stage_distill_loss(*args, 2.0, loss.data_ptr(), grad.data_ptr(), vocab, status.data_ptr(), stream())
    assert torch.equal(loss, want[0]) and torch.equal(grad, want[1]) and int(status) == 0
    with pytest.raises(B.SsnError):
        B.stage_distill_loss(*args, 0.0, loss.data_ptr())


def test_rows_in_8_bits_and_their_product():
    n, inner, outer = 9, 200, 31
    x, w = torch.randn(n, inner, device="cuda"), torch.randn(outer, inner, device="cuda")
    (xq, xs), (wq, ws) = stage_ops.int8_quantize(x), stage_ops.int8_quantize(w)
    want = stage_ops.int8_matmul(xq, xs, wq, ws, "f32")
    q, s, y = torch.empty(n, 208, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, outer, device="cuda")
    B.stage_int8_quantize(x.data_ptr(), inner, B.SSN_F32, n, inner, q.data_ptr(), 208, s.data_ptr(), stream())
    B.stage_int8_matmul(q.data_ptr(), 208, s.data_ptr(), wq.data_ptr(), wq.stride(0), ws.data_ptr(), n, inner, outer, y.data_ptr(), outer, B.SSN_F32,
                        stream=stream())
    assert torch.equal(q[:, :inner], xq) and torch.equal(s, xs) and torch.equal(y, want)
    with pytest.raises(B.SsnError):
        B.stage_int8_quantize(x.data_ptr(), inner - 1, B.SSN_F32, n, inner, q.data_ptr(), 208, s.data_ptr(), stream())
    with pytest.raises(B.SsnError):
        B.stage_int8_matmul(0, 208, s.data_ptr(), wq.data_ptr(), 208, ws.data_ptr(), n, inner, outer, y.data_ptr(), outer, B.SSN_F32)
