"""A prepared call holds the arrays that its pointers belong to, whatever becomes of the cache object it was given.  Needs no GPU: arrays
are stand-ins, and nothing is called."""
import ctypes as C
import gc
import weakref
from types import SimpleNamespace

import pytest
import torch

import paper_2511_02647_b200 as fa

SHAPE = fa.Shape(2, 4, 2, 64, fa.BF16)
CTX = SimpleNamespace(handle=C.c_void_p(64), device=0)


class Tensor:
    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype, self.device = shape, dtype, SimpleNamespace(index=0, type="cuda")

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def stride(self, i):
        return (self.shape[1] * self.shape[2], self.shape[2], 1)[i]


PREPARE = {
    "quantize": lambda c: fa.prepare_quantize_kv(CTX, SHAPE, Tensor(3, 2, 64), Tensor(3, 2, 64), None, c, 0),
    "dequantize": lambda c: fa.prepare_dequantize_kv(CTX, SHAPE, c, None, Tensor(3, 2, 64), Tensor(3, 2, 64), 0),
    "decode": lambda c: fa.prepare_decode_quant(CTX, SHAPE, fa.DECODE_LOCAL, Tensor(2, 4, 64), c, Tensor(2, dtype=torch.int32), 16,
                                                Tensor(2, 4, 64), stream=0),
}


@pytest.mark.parametrize("name", sorted(PREPARE))
def test_arrays_of_a_cache_live_as_long_as_the_call(name):
    cache = fa.QuantCache(SHAPE, 2, 32, *[Tensor(2, 2, 32, w, dtype=torch.uint8) for w in (32, 2, 32, 2)])
    arrays = [weakref.ref(t) for t in cache.arrays()]
    call = PREPARE[name](cache)
    cache.k_codes = cache.k_scales = cache.v_codes = cache.v_scales = None       # (a program that makes its cache larger)
    gc.collect()
    assert all(r() is not None for r in arrays)
    del call
    gc.collect()
    assert all(r() is None for r in arrays)
