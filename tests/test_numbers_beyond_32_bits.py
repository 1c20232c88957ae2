"""Numbers that the C calls take in 32 bits: what does not fit must not arrive as what its lower half says.  Needs no GPU: tensors are
stand-ins, and the library's functions are stand-ins of the same C type that record what they are given."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

import paper_2511_02647_b200 as fa
from paper_2511_02647_b200 import binding as b

SHAPE = fa.Shape(2, 4, 2, 64, fa.BF16)
CTX = SimpleNamespace(handle=C.c_void_p(64), device=0)
BIG = [2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63, 2 ** 70]


class Tensor:
    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype, self.device = shape, dtype, SimpleNamespace(index=0, type="cuda")

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


def arguments(name, **over):
    """Positional arguments of the binding's function, and where window, n_sink, max_kv_len and mode arrive."""
    a = dict(window=4, n_sink=1, max_kv_len=16, mode=0)
    assert not set(over) - set(a)
    a.update(over)
    q, lens = Tensor(2, 4, 64), Tensor(2, dtype=torch.int32)
    if name == "fedattn_local_window":
        x, kv = Tensor(9, 4, 64), Tensor(9, 2, 64)
        return (CTX, SHAPE, x, kv, kv, [0, 4, 9], a["window"], a["n_sink"], x, None, 0), dict(window=6, n_sink=7)
    if name == "fedattn_decode_window":
        kv = Tensor(2, 32, 2, 64)
        return (CTX, SHAPE, a["mode"], q, kv, kv, 32 * 128, lens, a["max_kv_len"], a["window"], a["n_sink"], q, None, 0), \
            dict(mode=2, max_kv_len=8, window=9, n_sink=10)
    cache = fa.QuantCache(SHAPE, 2, 32, *FOUR)
    return (CTX, SHAPE, a["mode"], q, cache, lens, a["max_kv_len"], q, None, a["window"], a["n_sink"], 0), \
        dict(mode=2, max_kv_len=10, window=11, n_sink=12)


FOUR = [Tensor(2, 2, 32, w, dtype=torch.uint8) for w in (32, 2, 32, 2)]
CALLS = ["fedattn_local_window", "fedattn_decode_window", "fedattn_decode_quant"]


@pytest.fixture
def received(monkeypatch):
    """What the stand-in of a call got, through the plain form and through the prepared one (with the order of the C call)."""
    def run(name, prepared, **over):
        fn, got = getattr(b._lib, name), []
        record = C.CFUNCTYPE(C.c_int, *fn.argtypes)(lambda *x: got.append(x) or 0)
        args, place = arguments(name, **over)
        if prepared:
            call = getattr(fa, name.replace("fedattn_", "prepare_"))(*args)
            monkeypatch.setattr(call, "_fn", C.CFUNCTYPE(C.c_int)(C.cast(record, C.c_void_p).value))
            call()
        else:
            with monkeypatch.context() as m:
                m.setattr(b._lib, name, record)
                getattr(fa, name)(*args)
        return {k: got[0][i] for k, i in place.items()}
    return run


@pytest.mark.parametrize("prepared", [False, True])
@pytest.mark.parametrize("name", CALLS)
def test_windows_and_sinks_beyond_every_length_stay_so(name, prepared, received):
    assert received(name, prepared) | dict(window=4, n_sink=1) == received(name, prepared)
    for big in BIG:
        got = received(name, prepared, window=big, n_sink=big)
        assert (got["window"], got["n_sink"]) == (2 ** 31 - 1, 2 ** 31 - 1), big
    for small in (-1, -2 ** 31, -2 ** 31 - 1, -2 ** 32, -2 ** 32 + 5, -2 ** 63 - 1):      # the C call refuses what is negative
        got = received(name, prepared, window=small, n_sink=small)
        assert got["window"] < 0 and got["n_sink"] < 0, small


@pytest.mark.parametrize("prepared", [False, True])
def test_bounds_and_modes_that_do_not_fit_are_refused(prepared, received):
    for big in BIG[1:]:
        got = received("fedattn_decode_quant", prepared, max_kv_len=big)
        assert got["max_kv_len"] == 2 ** 31 - 1                              # more than any cache has: refused
        got = received("fedattn_decode_quant", prepared, mode=big)
        assert got["mode"] not in (fa.DECODE_LOCAL, fa.DECODE_SYNC)
        assert received("fedattn_decode_window", prepared, mode=big)["mode"] not in (fa.DECODE_LOCAL, fa.DECODE_SYNC)
        with pytest.raises(ValueError):                                      # more rows than the caches hold
            received("fedattn_decode_window", prepared, max_kv_len=big)


@pytest.mark.parametrize("cu", [[0, 2 ** 32 + 4, 9], [0, 4, 2 ** 32 + 9], [-2 ** 32, 4, 9], torch.tensor([0, 2 ** 32 + 4, 9])], ids=str)
def test_segments_that_do_not_fit(cu):
    args, _ = arguments("fedattn_local_window")
    rows = [Tensor(int(cu[-1]), h, 64) for h in (4, 2, 2)]
    with pytest.raises(ValueError):
        b._args_local_window(*args[:2], *rows, cu, 4, 1, rows[0], None, 0)


def test_segments_that_fit():
    args, _ = arguments("fedattn_local_window")
    rows = [Tensor(2 ** 31 - 1, h, 64) for h in (4, 2, 2)]
    for cu in ([0, 5, 2 ** 31 - 1], torch.tensor([0, 5, 2 ** 31 - 1])):
        packed = bytes(b._args_local_window(*args[:2], *rows, cu, 4, 1, rows[0], None, 0)[5])
        assert packed == (5 << 32 | (2 ** 31 - 1) << 64).to_bytes(12, "little")
