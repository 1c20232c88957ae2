"""What a prepared call takes as a stream: all that the C parameter's type takes.  Needs no GPU: the library's function is a stand-in."""
import ctypes as C

import pytest

import paper_2511_02647_b200 as fa
from paper_2511_02647_b200 import binding as b

SHAPE = fa.Shape(2, 4, 2, 64, fa.BF16)


class Stream:
    """As torch.cuda.Stream and torch.cuda.ExternalStream do it."""

    def __init__(self, raw):
        self.cuda_stream = raw

    @property
    def _as_parameter_(self):
        return C.c_void_p(self.cuda_stream)


@pytest.mark.parametrize("stream,raw", [(1 << 41, 1 << 41), (0, None), (C.c_void_p(1 << 41), 1 << 41), (C.c_void_p(), None),
                                        (Stream(1 << 41), 1 << 41), (None, 48)])
def test_streams(stream, raw, monkeypatch):
    fn, got = b._lib.fedattn_merge, []
    record = C.CFUNCTYPE(C.c_int, *fn.argtypes)(lambda *x: got.append(x) or 0)
    call = b.PreparedCall(fn, (None, C.byref(SHAPE), 3, 1 << 47, None, 16, None, 16, None, 48), "fedattn_merge", None)
    monkeypatch.setattr(call, "_fn", C.CFUNCTYPE(C.c_int)(C.cast(record, C.c_void_p).value))
    call(stream)
    call(stream=stream)
    assert [x[-1] for x in got] == [raw, raw] and got[0][3] == 1 << 47


@pytest.mark.parametrize("stream", [1.5, "stream", object()])
def test_what_is_no_stream(stream):
    call = b.PreparedCall(b._lib.fedattn_merge, (None, C.byref(SHAPE), 3, 16, None, 16, None, 16, None, 48), "fedattn_merge", None)
    with pytest.raises(TypeError):
        call(stream)
