"""What the 8-bit products refuse on the host: no GPU."""

import pytest

A = 0x10000


def _quantize(b, x=A, ldx=64, dtype=1, rows=3, cols=64, q=A, ldq=64, scale=A):
    return b.raw("stage_int8_quantize")(x, ldx, dtype, rows, cols, q, ldq, scale, None)


def _matmul(b, xq=A, ldx=64, xs=A, wq=A, ldw=64, ws=A, n=3, inner=64, outer=40, y=A, ldy=40, dtype=1):
    return b.raw("stage_int8_matmul")(xq, ldx, xs, wq, ldw, ws, n, inner, outer, y, ldy, dtype, None, None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=5), "DTYPE"), (dict(rows=-1), "SHAPE"), (dict(cols=0), "SHAPE"), (dict(ldx=63), "SHAPE"), (dict(ldq=63), "SHAPE"),
    (dict(ldx=1 << 60), "SHAPE"), (dict(x=None), "NULL"), (dict(q=None), "NULL"), (dict(scale=None), "NULL"), (dict(x=A + 1), "SHAPE")])
def test_quantize_values(libssn, change, status):
    assert _quantize(libssn, **change) == getattr(libssn, "SSN_ERR_" + status)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=5), "DTYPE"), (dict(n=-1), "SHAPE"), (dict(outer=-1), "SHAPE"), (dict(inner=0), "SHAPE"),
    (dict(inner=131072, ldx=131072, ldw=131072), "SHAPE"), (dict(ldx=63), "SHAPE"), (dict(ldw=63), "SHAPE"), (dict(ldy=39), "SHAPE"),
    (dict(ldy=1 << 60), "SHAPE"), (dict(ldw=1 << 60), "SHAPE"), (dict(xq=None), "NULL"), (dict(xs=None), "NULL"), (dict(wq=None), "NULL"),
    (dict(ws=None), "NULL"), (dict(y=None), "NULL"), (dict(y=A + 1), "SHAPE"), (dict(y=A + 2, dtype=0), "SHAPE")])
def test_matmul_values(libssn, change, status):
    assert _matmul(libssn, **change) == getattr(libssn, "SSN_ERR_" + status)


def test_empty_calls(libssn):
    assert _quantize(libssn, rows=0, x=None, q=None, scale=None) == libssn.SSN_OK
    assert _matmul(libssn, n=0, xq=None, xs=None, y=None) == libssn.SSN_OK
    assert _matmul(libssn, outer=0, wq=None, ws=None, y=None) == libssn.SSN_OK


def test_addresses_off_their_element(libssn):
    assert _quantize(libssn, scale=A + 2) == libssn.SSN_ERR_SHAPE
    assert _matmul(libssn, xs=A + 1) == libssn.SSN_ERR_SHAPE and _matmul(libssn, ws=A + 2) == libssn.SSN_ERR_SHAPE
