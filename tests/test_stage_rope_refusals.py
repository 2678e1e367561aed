"""What the query/key norm refuses on the host: no GPU."""

import ctypes

import pytest
import torch

A = 0x10000      # an aligned address that no call here reaches


def _op(b, **kw):
    args = dict(head_dim=64, rot_dim=64, dtype=b.SSN_BF16, pairing=b.STAGE_PAIR_HALVES, eps=1e-6, table=A, ldt=64, max_pos=16)
    args.update(kw)
    return b.make_qk_rope(**args)


def _forward(b, op, q=(A, 64, 64), qh=4, k=(A, 64, 64), kh=1, qo=(A, 256, 64), ko=(A, 64, 64), pos=None, n=3, seq=8):
    return b.raw("stage_qk_rope_forward")(ctypes.byref(op) if op is not None else None, *q, qh, *k, kh, *qo, *ko, pos, n, seq, None)


@pytest.mark.parametrize("change,status", [
    (dict(head_dim=63), "SHAPE"), (dict(head_dim=0), "SHAPE"), (dict(head_dim=258, rot_dim=0), "SHAPE"), (dict(rot_dim=66), "SHAPE"),
    (dict(rot_dim=-2), "SHAPE"), (dict(rot_dim=7), "SHAPE"), (dict(dtype=3), "DTYPE"), (dict(pairing=2), "DTYPE"),
    (dict(eps=-1.0), "SHAPE"), (dict(eps=float("nan")), "SHAPE"), (dict(eps=float("inf")), "SHAPE"), (dict(table=0), "NULL"),
    (dict(ldt=63), "SHAPE"), (dict(max_pos=0), "SHAPE")])
def test_operator_values(libssn, change, status):
    want = getattr(libssn, "SSN_ERR_" + status)
    assert _forward(libssn, _op(libssn, **change)) == want
    assert libssn.raw("stage_qk_rope_backward")(ctypes.byref(_op(libssn, **change)), *(A, 64, 64) * 2, A, 64, 64, 1, A, 64, 64, 1,
                                                *(A, 64, 64) * 2, None, None, None, 3, 8, None, 0, None) == want
    assert libssn.stage_qk_rope_workspace_bytes(_op(libssn, **change), 3, 4, 1) == 0


@pytest.mark.parametrize("change,status", [
    (dict(q=(None, 64, 64)), "NULL"), (dict(ko=(None, 64, 64)), "NULL"), (dict(q=(A, -1, 64)), "SHAPE"), (dict(k=(A, 64, -64)), "SHAPE"),
    (dict(qo=(A, 255, 64)), "SHAPE"), (dict(qo=(A, 256, 63)), "SHAPE"), (dict(qo=(A, 64, 191)), "SHAPE"), (dict(ko=(A, 63, 0)), "SHAPE"),
    (dict(ko=(A, 0, 64)), "SHAPE"), (dict(n=-1), "SHAPE"), (dict(qh=-1), "SHAPE"), (dict(qh=1 << 20, qo=(A, 1 << 30, 64)), "SHAPE"),
    (dict(seq=0), "SHAPE"), (dict(q=(A, 1 << 62, 64)), "SHAPE"), (dict(q=(A + 1, 64, 64)), "SHAPE")])
def test_call_values(libssn, change, status):
    assert _forward(libssn, _op(libssn), **change) == getattr(libssn, "SSN_ERR_" + status)


def test_empty_calls_and_workspace(libssn):
    b, op = libssn, _op(libssn)
    assert _forward(b, None) == b.SSN_ERR_NULL
    assert _forward(b, op, n=0, q=(None, 0, 0), k=(None, 0, 0), qo=(None, 0, 0), ko=(None, 0, 0)) == b.SSN_OK
    assert _forward(b, op, qh=0, kh=0) == b.SSN_OK
    need = b.stage_qk_rope_workspace_bytes(op, 3, 4, 1)
    assert need >= 2 * 64 * 4
    back = b.raw("stage_qk_rope_backward")
    heads = (A, 64, 64) * 2 + (A, 64, 64, 1) * 2 + (A, 64, 64) * 2
    for ws, size in ((None, need), (A, need - 1), (A + 4, need)):
        assert back(ctypes.byref(op), *heads, A, A, None, 3, 8, ws, size, None) == b.SSN_ERR_WORKSPACE
    table = b.raw("stage_rope_table")
    for args in ((A, 64, 16, 63, 1e4), (A, 62, 16, 64, 1e4), (A, 64, -1, 64, 1e4), (A, 64, 16, 64, 0.0), (A, 64, 16, 64, float("inf")), (A, 64, 16, 0, 1e4)):
        assert table(*args, None) == b.SSN_ERR_SHAPE
    assert table(None, 64, 16, 64, 1e4, None) == b.SSN_ERR_NULL and table(None, 64, 0, 64, 1e4, None) == b.SSN_OK


@pytest.mark.parametrize("change", [dict(table=A + 2), dict(wq=A + 1), dict(wk=A + 1), dict(dev_status=A + 2)])
def test_addresses_off_their_element(libssn, change):
    assert _forward(libssn, _op(libssn, **change)) == libssn.SSN_ERR_SHAPE
    assert _forward(libssn, _op(libssn), pos=A + 2) == libssn.SSN_ERR_SHAPE


def test_an_output_in_place_of_an_input_of_other_strides(libssn):
    b = libssn
    other = dict(q=(2 * A, 256, 64), k=(3 * A, 64, 64), qo=(4 * A, 256, 64), ko=(5 * A, 64, 64))
    assert _forward(b, _op(b), **dict(other, q=(A, 320, 64), qo=(A, 256, 64))) == b.SSN_ERR_SHAPE
    assert _forward(b, _op(b), **dict(other, k=(A, 64, 64), ko=(A, 128, 64))) == b.SSN_ERR_SHAPE
    back = b.raw("stage_qk_rope_backward")
    for out in ((A, 128, 64), (2 * A, 128, 64)):      # dq and q start there
        assert back(ctypes.byref(_op(b)), A, 64, 64, 3 * A, 64, 64, 2 * A, 64, 64, 1, 4 * A, 64, 64, 1, *out, 5 * A, 64, 64, None, None,
                    None, 3, 8, None, 0, None) == b.SSN_ERR_SHAPE


@pytest.fixture
def host_is_current(monkeypatch):
    """Tensors on the host pass for tensors of the current device: no call below reaches the library."""
    stage_ops = pytest.importorskip("paper_2607_13332_b200.stage_ops")
    monkeypatch.setattr(stage_ops, "_current_device", lambda: -1)
    return stage_ops


def test_rows_that_share_elements_have_no_leading_dimension(libssn, host_is_current):
    row = torch.zeros(1, 8)
    assert host_is_current._pitch(row.expand(1, 8), 1, 8) == 8
    assert host_is_current._pitch(torch.zeros(3, 10)[:, :8], 3, 8) == 10
    for shared in (row.expand(4, 8), torch.zeros(64).as_strided((4, 8), (7, 1)), torch.zeros(4, 16)[:, ::2]):
        with pytest.raises(ValueError, match="row-major"):
            host_is_current._pitch(shared, 4, 8)
    with pytest.raises(ValueError, match="row-major"):
        host_is_current.QKNormRope("f32", 8, table=row.expand(4, 8), device="cpu")


def test_an_operator_is_for_one_device(libssn, host_is_current, monkeypatch):
    op = host_is_current.QKNormRope("f32", 8, device="cpu")
    q = torch.zeros(2, 1, 8)
    monkeypatch.setattr(host_is_current, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="device"):
        op.forward(q, None, seq_len=2)
    with pytest.raises(ValueError, match="device"):
        op.backward(q, None, q, None, seq_len=2)
    with pytest.raises(ValueError, match="device"):      # its status word would lie elsewhere
        host_is_current.QKNormRope("f32", 8, device="cpu")
