"""Offsets that pass 32 bits: rows at the far end of caches and row blocks of more than 2^32 bytes or elements.  What is not
looked at is left as the allocator gives it, but for the rows that share a tile with visible ones."""
import numpy as np
import pytest
import torch

import paper_2511_02647_b200 as fa
import reference64 as ref
from helpers import dev, host

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def free_memory():
    yield
    torch.cuda.empty_cache()


def test_rows_at_the_end_of_a_four_bit_cache():
    hq, hkv, d, cap, n = 8, 8, 128, 9_000_000, 70
    assert cap * hkv * d // 2 > 1 << 32 and cap % 16 == 0
    shape = fa.Shape(1, hq, hkv, d, fa.BF16)
    ctx = fa.Context(shape, n, cap)
    arrays = [torch.empty((1, hkv, cap, w), dtype=torch.uint8, device="cuda") for w in (d // 2, d // 32) * 2]
    cache = fa.QuantCache(shape, 1, cap, *arrays)
    rng = np.random.default_rng(1)
    k, v = (ref.rounded(rng.standard_normal((n, hkv, d)), "bf16") for _ in range(2))
    rows = np.concatenate([np.arange(6), np.arange(cap - n + 6, cap)])
    at = torch.tensor(rows, dtype=torch.int32, device="cuda")
    kd, vd = dev(k.astype(np.float32), "bf16"), dev(v.astype(np.float32), "bf16")
    fa.fedattn_quantize_kv(ctx, shape, kd, vd, at, cache)
    kb, vb = torch.empty_like(kd), torch.empty_like(vd)
    fa.fedattn_dequantize_kv(ctx, shape, cache, at, kb, vb)
    kh, vh = (ref.values(*ref.quantise(x)) for x in (k, v))
    assert np.array_equal(host(kb), kh) and np.array_equal(host(vb), vh)
    q = ref.rounded(rng.standard_normal((1, hq, d)), "bf16")
    for mode in (fa.DECODE_LOCAL, fa.DECODE_SYNC):
        o, lse = torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((1, hq), device="cuda")
        fa.fedattn_decode_quant(ctx, shape, mode, dev(q.astype(np.float32), "bf16"), cache,
                                torch.tensor([cap], dtype=torch.int32, device="cuda"), cap, o, lse, window=n - 6, n_sink=6)
        assert ctx.poll() == 0
        ref.check_attention(host(o), host(lse), ref.attend(q, kh, vh, np.ones((1, n), bool), d ** -0.5), "bf16")


def test_window_at_the_end_of_a_bf16_cache():
    hq, hkv, d, cap, window, sink = 8, 8, 128, 4_300_000, 100, 5
    assert cap * hkv * d > 1 << 32
    shape = fa.Shape(1, hq, hkv, d, fa.BF16)
    ctx = fa.Context(shape, 1, cap)
    rng = np.random.default_rng(2)
    keep = np.concatenate([np.arange(sink), np.arange(cap - window, cap)])
    caches, exact = [], []
    for _ in range(2):
        x = torch.empty((cap, hkv, d), dtype=torch.bfloat16, device="cuda")
        x[:256] = 0
        x[cap - 512:] = 0
        y = ref.rounded(rng.standard_normal((sink + window, hkv, d)), "bf16")
        x[torch.from_numpy(keep).cuda()] = dev(y.astype(np.float32), "bf16")
        caches.append(x)
        exact.append(y)
    q = ref.rounded(rng.standard_normal((1, hq, d)), "bf16")
    o, lse = torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((1, hq), device="cuda")
    fa.fedattn_decode_window(ctx, shape, fa.DECODE_SYNC, dev(q.astype(np.float32), "bf16"), *caches, 0,
                             torch.tensor([cap], dtype=torch.int32, device="cuda"), cap, window, sink, o, lse)
    assert ctx.poll() == 0
    ref.check_attention(host(o), host(lse), ref.attend(q, *exact, np.ones((1, sink + window), bool), d ** -0.5), "bf16")


def test_norm_and_rotation_of_many_rows():
    hq, hkv, d, rows = 32, 8, 128, 1_060_000
    assert rows * hq * d > 1 << 32
    shape = fa.Shape(1, hq, hkv, d, fa.BF16)
    ctx = fa.Context(shape, 1, 1)
    qkv = torch.zeros((rows, (hq + 2 * hkv) * d), dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(3)
    x = ref.rounded(rng.standard_normal((3, (hq + 2 * hkv) * d)), "bf16")
    at = [0, rows // 2, rows - 1]
    for i, r in enumerate(at):
        qkv[r] = dev(x[i:i + 1].astype(np.float32), "bf16")[0]
    q, k = qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
    qo, ko = torch.empty((rows, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, hkv, d), dtype=torch.bfloat16, device="cuda")
    freq = [10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
    fa.fedattn_qk_norm_rope(ctx, shape, q, k, None, None, 1e-6, None, freq, False, qo, ko)
    for got, a, h in ((qo, 0, hq), (ko, hq * d, hkv)):
        want, size = ref.norm_rope(x[:, a:a + h * d].reshape(3, h, d), None, float(np.float32(1e-6)), np.array(at), freq, False)
        assert (np.abs(host(got[at]) - want) <= 24 * 2.0 ** -24 * size + 2.0 ** -8 * np.abs(want)).all()
    assert not got[1:rows // 2].any()


@pytest.mark.parametrize("d", [128, 64])
def test_window_over_a_long_segment(d):
    hq, hkv, L, window, sink = 4096 // d, 2, 1_060_000, 70, 3
    assert L * hq * d > 1 << 32
    shape = fa.Shape(2, hq, hkv, d, fa.BF16)
    ctx = fa.Context(shape, 1, 1)
    gen = torch.Generator(device="cuda").manual_seed(4)
    q = torch.empty((L, hq, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    k, v = (torch.empty((L, hkv, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    o, lse = torch.empty_like(q), torch.empty((L, hq), device="cuda")
    first = 1000
    fa.fedattn_local_window(ctx, shape, q, k, v, [0, first, L], window, sink, o, lse)
    assert ctx.poll() == 0
    for row in (first + 5, L // 2, L - 1):
        keys = sorted(set(range(first, first + sink)) | set(range(max(first, row - window + 1), row + 1)))
        want = ref.attend(host(q[row:row + 1]), host(k[keys]), host(v[keys]), np.ones((1, len(keys)), bool), d ** -0.5)
        ref.check_attention(host(o[row:row + 1]), host(lse[row:row + 1]), want, "bf16", "row %d" % row, "bf16" if d == 128 else "f32")
