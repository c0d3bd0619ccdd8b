"""CPU checks of the rotated rows' C ABI: strides and positions that 64 bits cannot hold are refused before arithmetic on them."""
import ctypes

import pytest

import paper_2510_04008_amd as ra

FREQ = (ctypes.c_double * 128)(*([1.0] * 128))


def _call(name, pos0=0, positions=False, B=3, Hk=2, **strides):
    d = ra.make_rotary_desc(B, 100, 4, Hk, 64, 64, ra.RACE_BF16, pos0=pos0)
    usual = dict(q_strides=(25600, 256, 64), k_strides=(12800, 128, 64), dq_strides=(25600, 256, 64), dk_strides=(12800, 128, 64))
    for n, s in dict(usual, **strides).items():
        setattr(d, n, (ctypes.c_int64 * 3)(*s))
    p = [ctypes.c_void_p(256 * (i + 1)) for i in range(12)]
    place = p[11] if positions else None
    if name == "fwd":
        return ra.lib().race_qk_rotary_fwd(ctypes.byref(d), *p[:4], FREQ, place, p[4], p[5], None)
    if Hk == 0:
        p[9] = None
    # (a null workspace ends a call that is otherwise in order)
    return ra.lib().race_qk_rotary_bwd(ctypes.byref(d), *p[:4], FREQ, place, *p[4:10], None, 0, None)


@pytest.mark.parametrize("big", [(1 << 62, 256, 64), (25600, 1 << 57, 64), (25600, 256, 1 << 62), ((1 << 62) - 1, (1 << 56) - 1, 64), ((1 << 63) - 1, 256, 64)])
def test_rows_beyond_64_bits(big):
    assert _call("fwd", q_strides=big) == ra.RACE_ERR_INVALID_ARG and _call("fwd", k_strides=big) == ra.RACE_ERR_INVALID_ARG
    for n in ("q_strides", "k_strides", "dq_strides", "dk_strides"):
        assert _call("bwd", **{n: big}) == ra.RACE_ERR_INVALID_ARG, n
    # an axis of one element may have any stride, and so may keys that there are not
    one = ((1 << 63) - 1, 256, 64)
    assert _call("bwd", B=1, q_strides=one, k_strides=one, dq_strides=one, dk_strides=one) == ra.RACE_ERR_WORKSPACE
    assert _call("bwd", Hk=0, k_strides=big, dk_strides=big) == ra.RACE_ERR_WORKSPACE


def test_positions_beyond_64_bits():
    for pos0 in ((1 << 63) - 1, (1 << 63) - 100):
        assert _call("fwd", pos0=pos0) == ra.RACE_ERR_INVALID_ARG and _call("bwd", pos0=pos0) == ra.RACE_ERR_INVALID_ARG
        assert _call("bwd", pos0=pos0, positions=True) == ra.RACE_ERR_WORKSPACE         # it is not read
    for pos0 in ((1 << 63) - 101, -(1 << 63)):
        assert _call("bwd", pos0=pos0) == ra.RACE_ERR_WORKSPACE
