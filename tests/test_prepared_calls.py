"""What a prepared call passes to the library: the same as the call that marshals every time, whatever its arguments are."""
import ctypes as C

import pytest

import paper_2511_02647_b200 as fa
from paper_2511_02647_b200 import binding as b

SHAPE = fa.Shape(2, 4, 2, 64, fa.BF16)
FREQ = (C.c_double * 4)(0.5, 1.0, -2.0, 1e-3)
CASES = {
    "fedattn_merge": (None, C.byref(SHAPE), 2 ** 40, 1 << 47, None, 1 << 46, None, 16, None, 7),
    "fedattn_local": (None, C.byref(SHAPE), 16, 32, 48, b._i32_array([0, 5, 9]), 64, None, 1 << 40),
    "fedattn_decode_window": (None, C.byref(SHAPE), 1, 16, 32, 48, -(2 ** 40), 64, 2 ** 31 - 1, -3, 4, 80, None, 0),
    "fedattn_qk_norm_rope": (None, C.byref(SHAPE), 3, 16, 2 ** 33, None, 0, None, None, 1e-6, 32, FREQ, 8, 1, 48, None, 5),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_arguments_arrive_as_they_would(name, monkeypatch):
    """A stand-in of the same C type records them: pointers and 64-bit numbers whole, floats as floats, arrays and structures in place."""
    fn = getattr(b._lib, name)
    got = []

    def record(*args):
        got.append(args)
        return 0

    stand_in = C.CFUNCTYPE(C.c_int, *fn.argtypes)(record)
    fn_like = C.CFUNCTYPE(C.c_int, *fn.argtypes)(C.cast(stand_in, C.c_void_p).value)
    fn_like(*CASES[name])
    untyped = C.CFUNCTYPE(C.c_int)(C.cast(stand_in, C.c_void_p).value)
    call = b.PreparedCall(fn, CASES[name], name, None)
    monkeypatch.setattr(call, "_fn", untyped)
    call()
    call(1 << 41)

    def plain(args):
        return [C.addressof(a.contents) if hasattr(a, "contents") else a for a in args]

    assert plain(got[0]) == plain(got[1]) and plain(got[0])[:-1] == plain(got[2])[:-1] and got[2][-1] == 1 << 41


def test_refusals_raise():
    call = b.PreparedCall(b._lib.fedattn_merge, CASES["fedattn_merge"], "fedattn_merge", None)
    with pytest.raises(fa.FedAttnError) as e:
        call()
    assert e.value.code == 1 and "fedattn_merge" in str(e.value)
