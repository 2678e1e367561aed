"""What the loss against a teacher's top logits refuses on the host: no GPU."""

import pytest

A = 0x10000


def _call(b, logits=A, ldl=100, dtype=1, n=3, vocab=100, ids=A, ldi=8, top=A, ldt=8, k=8, weight=None, tau=1.0, loss=A, out=2 * A, ldd=100):
    return b.raw("stage_distill_loss")(logits, ldl, dtype, n, vocab, ids, ldi, top, ldt, k, weight, tau, loss, out, ldd, None, None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), "DTYPE"), (dict(n=-1), "SHAPE"), (dict(vocab=0), "SHAPE"), (dict(vocab=1 << 31, ldl=1 << 31, ldd=1 << 31), "SHAPE"),
    (dict(k=0), "SHAPE"), (dict(k=1025, ldi=1025, ldt=1025), "SHAPE"), (dict(ldl=99), "SHAPE"), (dict(ldi=7), "SHAPE"), (dict(ldt=7), "SHAPE"),
    (dict(ldd=99), "SHAPE"), (dict(tau=0.0), "SHAPE"), (dict(tau=-1.0), "SHAPE"), (dict(tau=float("nan")), "SHAPE"),
    (dict(tau=float("inf")), "SHAPE"), (dict(tau=1e-7), "SHAPE"), (dict(logits=None), "NULL"), (dict(ids=None), "NULL"), (dict(top=None), "NULL"),
    (dict(loss=None), "NULL"), (dict(logits=A + 1), "SHAPE"), (dict(out=A + 1), "SHAPE"), (dict(out=A, ldd=108), "SHAPE"),
    (dict(ldl=1 << 60), "SHAPE")])
def test_call_values(libssn, change, status):
    assert _call(libssn, **change) == getattr(libssn, "SSN_ERR_" + status)


def test_no_tokens(libssn):
    assert _call(libssn, n=0, logits=None, ids=None, top=None, loss=None, out=None) == libssn.SSN_OK


@pytest.mark.parametrize("name", ["ids", "top", "weight", "loss"])
def test_addresses_off_their_element(libssn, name):
    assert _call(libssn, **{name: A + 2}) == libssn.SSN_ERR_SHAPE
