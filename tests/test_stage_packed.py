"""The stage calls with their arguments in one struct answer as the calls do: no GPU."""

import ctypes

import pytest

A = 0x10000      # an aligned address that no call here reaches
FAR = 1 << 62

# arguments of a call that would be launched, and for every position a value that is refused there (None: any will do)
CALLS = {
    "stage_qk_rope_forward": [
        ("op", 0), (A, 0), (256, -1), (64, -1), (4, -1), (A, 0), (64, FAR), (64, None), (1, 1 << 20), (2 * A, 0), (256, 255), (64, 63),
        (3 * A, 0), (64, 63), (64, None), (A, A + 2), (3, -1), (8, None), (0, None)],
    "stage_qk_rope_backward": [
        ("op", 0), (A, 0), (256, -1), (64, -1), (A, 0), (64, -1), (64, None), (2 * A, 0), (256, -1), (64, -1), (4, -1), (2 * A, 0), (64, FAR),
        (64, None), (1, 1 << 20), (3 * A, 0), (256, 255), (64, 63), (4 * A, 0), (64, 63), (64, None), (A, A + 1), (A, A + 2), (A, A + 2),
        (3, -1), (8, None), (A, 0), (1 << 24, 16), (0, None)],
    "stage_distill_loss": [
        (A, 0), (128, 127), (1, 7), (3, -1), (128, 0), (A, 0), (4, 3), (A, 0), (4, 3), (4, 0), (A, A + 1), (1.0, 0.0), (A, 0), (2 * A, 2 * A + 1),
        (128, 127), (A, A + 2), (0, None)],
    "stage_int8_quantize": [(A, 0), (64, 63), (1, 7), (3, -1), (64, 0), (A, 0), (64, 63), (A, A + 2), (0, None)],
    "stage_int8_matmul": [
        (A, 0), (64, 63), (A, A + 1), (A, 0), (64, 63), (A, A + 2), (3, -1), (64, 0), (8, -1), (A, 0), (8, 7), (1, 9), (A, A + 1), (0, None)],
}


@pytest.mark.parametrize("name", CALLS)
def test_every_argument_arrives_in_its_place(libssn, name):
    b = libssn
    op = b.make_qk_rope(head_dim=64, rot_dim=0, dtype=b.SSN_F32, pairing=b.STAGE_PAIR_HALVES, eps=1e-6)
    call, pack = b.packed(name)
    direct = b.raw(name)
    assert len(CALLS[name]) == len(direct.argtypes)
    value = lambda v: ctypes.addressof(op) if v == "op" else v
    good = [value(v) for v, _ in CALLS[name]]
    plain = lambda args: direct(*(ctypes.cast(v, t) if t is ctypes.POINTER(type(op)) else v for v, t in zip(args, direct.argtypes)))
    refused = 0
    for at, (_, bad) in enumerate(CALLS[name]):
        if bad is None:
            continue
        args = good[:at] + [bad] + good[at + 1:]
        status = call(pack(*args))
        assert status == plain(args)
        refused += status in (b.SSN_ERR_NULL, b.SSN_ERR_SHAPE, b.SSN_ERR_DTYPE, b.SSN_ERR_WORKSPACE)
    assert refused == sum(bad is not None for _, bad in CALLS[name])
    assert call(None) == b.SSN_ERR_NULL
