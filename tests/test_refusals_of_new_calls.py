"""What the entry points around the path refuse, before anything is launched.  Needs no GPU: a refused call does not look at its
context, so a block of zeros stands for one; a call that was let through would fail at the device (status 4)."""
import ctypes as C

import pytest

import paper_2511_02647_b200 as fa
from paper_2511_02647_b200 import binding

LIB = binding._lib
CTX = C.create_string_buffer(4096)
P = 1 << 20                                       # an aligned address that nothing reads


def call(name, **over):
    shape = fa.Shape(2, 8, 2, 64, fa.BF16)
    freq = (C.c_double * 32)(*([0.5] * 32))
    args = {
        "fedattn_qk_norm_rope": dict(ctx=C.addressof(CTX), shape=C.byref(shape), n=4, q=P, qs=0, k=P, ks=0, wq=P, wk=P, eps=1e-6,
                                     pos=P, freq=freq, rot=64, inter=0, qo=2 * P, ko=2 * P, stream=None),
        "fedattn_quantize_kv": dict(ctx=C.addressof(CTX), shape=C.byref(shape), n=4, k=P, ks=0, v=P, vs=0, at=None, caches=2, cap=32,
                                    kc=P, ksc=P, vc=P, vsc=P, stream=None),
        "fedattn_dequantize_kv": dict(ctx=C.addressof(CTX), shape=C.byref(shape), n=4, at=None, caches=2, cap=32, kc=P, ksc=P, vc=P,
                                      vsc=P, k=P, v=P, stream=None),
        "fedattn_decode_quant": dict(ctx=C.addressof(CTX), shape=C.byref(shape), mode=0, q=P, kc=P, ksc=P, vc=P, vsc=P, cap=32, len=P,
                                     max=32, window=0, sink=0, o=P, lse=None, stream=None),
        "fedattn_local_window": dict(ctx=C.addressof(CTX), shape=C.byref(shape), q=P, k=P, v=P, cu=(C.c_int32 * 3)(0, 4, 9), window=4,
                                     sink=1, o=P, lse=None, stream=None),
        "fedattn_decode_window": dict(ctx=C.addressof(CTX), shape=C.byref(shape), mode=0, q=P, k=P, v=P, stride=2048, len=P, max=16,
                                      window=4, sink=1, o=P, lse=None, stream=None),
    }[name]
    unknown = set(over) - set(args)
    assert not unknown, unknown
    args.update(over)
    return getattr(LIB, name)(*args.values())


def bad_shape(**kw):
    a = dict(n_participants=2, n_q_heads=8, n_kv_heads=2, head_dim=64, dtype=fa.BF16)
    a.update(kw)
    return C.byref(fa.Shape(**a))


INVALID = [
    ("fedattn_qk_norm_rope", o) for o in (
        dict(ctx=None), dict(shape=None), dict(shape=bad_shape(n_kv_heads=3)), dict(n=-1), dict(eps=-1.0), dict(eps=float("nan")),
        dict(eps=float("inf")), dict(rot=12), dict(rot=72), dict(rot=-8), dict(freq=None), dict(inter=2), dict(q=None), dict(qo=None),
        dict(k=None), dict(ko=None), dict(q=P + 8), dict(ko=P + 4), dict(wq=P + 2), dict(qs=256), dict(qs=516), dict(ks=-128),
        dict(qo=P, qs=1024), dict(freq=(C.c_double * 32)(*([0.5] * 31 + [float("nan")]))),
        dict(freq=(C.c_double * 32)(*([float("inf")] * 32))))
] + [
    ("fedattn_quantize_kv", o) for o in (
        dict(ctx=None), dict(shape=None), dict(n=-1), dict(caches=0), dict(cap=24), dict(cap=-16), dict(caches=1 << 27, cap=32),
        dict(kc=None), dict(vsc=None), dict(kc=P + 8), dict(k=None), dict(v=None), dict(k=P + 8), dict(ks=64), dict(vs=132), dict(n=65))
] + [
    ("fedattn_dequantize_kv", o) for o in (
        dict(ctx=None), dict(shape=None), dict(n=-1), dict(caches=0), dict(cap=24), dict(ksc=None), dict(k=None), dict(v=None),
        dict(v=P + 8), dict(n=65))
] + [
    ("fedattn_decode_quant", o) for o in (
        dict(ctx=None), dict(shape=None), dict(mode=2), dict(q=None), dict(o=None), dict(len=None), dict(q=P + 2), dict(o=P + 8),
        dict(cap=24), dict(max=33), dict(max=-1), dict(kc=None), dict(vc=P + 4), dict(window=-1), dict(sink=-1), dict(sink=3))
] + [
    ("fedattn_local_window", o) for o in (
        dict(ctx=None), dict(shape=None), dict(cu=None), dict(window=0), dict(window=-2), dict(sink=-1), dict(q=None), dict(k=None),
        dict(o=None), dict(v=P + 8), dict(cu=(C.c_int32 * 3)(1, 4, 9)), dict(cu=(C.c_int32 * 3)(0, 4, 3)))
] + [
    ("fedattn_decode_window", o) for o in (
        dict(ctx=None), dict(shape=None), dict(mode=2), dict(q=None), dict(k=None), dict(len=None), dict(o=P + 8), dict(max=-1),
        dict(stride=-8), dict(stride=4), dict(window=0), dict(sink=-1))
]


@pytest.mark.parametrize("name,over", INVALID, ids=lambda x: x if isinstance(x, str) else ",".join(x))
def test_invalid_arguments(name, over):
    assert call(name, **over) == 1


@pytest.mark.parametrize("name", ["fedattn_quantize_kv", "fedattn_dequantize_kv", "fedattn_decode_quant"])
@pytest.mark.parametrize("d", [8, 48, 120])
def test_four_bit_caches_need_whole_groups(name, d):
    assert call(name, shape=bad_shape(head_dim=d)) == 2


@pytest.mark.parametrize("name", ["fedattn_qk_norm_rope", "fedattn_quantize_kv", "fedattn_dequantize_kv", "fedattn_decode_quant"])
def test_rows_that_are_not_counted_in_32_bits(name):
    assert call(name, shape=bad_shape(n_q_heads=2 ** 31 - 1, n_kv_heads=2 ** 31 - 1)) == 2


def test_workspace_too_small():
    assert call("fedattn_decode_quant") == 3      # the stand-in's workspace has no bytes


def test_nothing_to_do():
    assert call("fedattn_local_window", cu=(C.c_int32 * 3)(0, 0, 0)) == 0
    assert call("fedattn_qk_norm_rope", n=0) == 0
    assert call("fedattn_qk_norm_rope", q=None, qo=None, k=None, ko=None) == 0
    assert call("fedattn_quantize_kv", n=0) == 0
    assert call("fedattn_dequantize_kv", n=0) == 0
