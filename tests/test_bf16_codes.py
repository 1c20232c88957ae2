"""The two roundings of the 4-bit cache that the kernel decides without an exact quotient, restated step by step in fp32, for
every bf16 value: the codes against every scale that the value can meet, and the scale byte."""
import numpy as np

import reference64 as ref

F = np.float32
VALUES = (np.arange(0, 0x7F80, dtype=np.uint32) << 16).view(F)              # zero and every positive finite bf16


def test_codes_of_every_value_under_every_scale():
    for b in range(256):
        s = F(ref.SCALES[b])
        x = VALUES[VALUES <= 7 * s]
        x = np.concatenate([x, -x])
        want = np.rint(x.astype(np.float64) / ref.SCALES[b]).astype(np.int64)
        inv = F(1) / s
        for near in (inv, np.nextafter(inv, F(0)), np.nextafter(inv, F(1e30)), np.nextafter(np.nextafter(inv, F(0)), F(0)),
                     np.nextafter(np.nextafter(inv, F(1e30)), F(1e30))):     # the reciprocal is an approximation
            t = (x * near).astype(F)
            t = ((t + F(1536)).astype(F) - F(1536)).astype(F)                # to a multiple of 2^-13
            bits = (t + F(12582920)).astype(F).view(np.uint32)
            assert np.array_equal(bits - np.uint32(0x4B400000), (want + 8).astype(np.uint32)), b


def byte_of(amax):
    seventh = np.array([0x3E124924], dtype=np.uint32).view(F)[0]
    bits = (amax * seventh).astype(F).view(np.int32).astype(np.int64)
    return np.clip(((bits + 0xFFFFF) >> 20) - ((127 - 18) << 3), 0, 255)


def test_scale_of_every_value():
    want = np.minimum(np.searchsorted(7 * ref.SCALES, VALUES.astype(np.float64)), 255)
    assert np.array_equal(byte_of(VALUES), want)


def test_scale_of_fp32_values_at_the_borders():
    at = F(7) * ref.SCALES.astype(F)
    amax = np.concatenate([at, np.nextafter(at, F(0)), np.nextafter(at, F(1e30)),
                           np.random.default_rng(1).integers(0, 0x7F800000, 1 << 20).astype(np.uint32).view(F)])
    b = byte_of(amax)
    b = np.where((7 * ref.SCALES[b] < amax) & (b < 255), b + 1, b)           # the comparison that fp32 values add
    assert np.array_equal(b, np.minimum(np.searchsorted(7 * ref.SCALES, amax.astype(np.float64)), 255))
