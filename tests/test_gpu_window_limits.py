"""Windowed calls and 4-bit caches as long as an int counts: the last tile ends where 32-bit sums would wrap.  Most of the memory holds
zeros; the last rows have logits that decide the output."""
import numpy as np
import pytest
import torch

import paper_2511_02647_b200 as fa
import reference64 as ref
from helpers import dev, host

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.fixture(autouse=True)
def free_memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def need(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("needs %d GiB of free device memory" % gib)


def attend_tail(q, k, v, zeros, scale):
    """reference64.attend for rows that see `zeros` keys and values of zero beside k, v [T, 1, d]."""
    s = q[:, 0] @ k[:, 0].T * scale
    m = np.maximum(s.max(1), 0.0)
    p, rest = np.exp(s - m[:, None]), zeros * np.exp(-m)
    z = p.sum(1) + rest
    terms = (np.abs(q[:, 0]) @ np.abs(k[:, 0]).T).max(1) * scale
    return (p @ v[:, 0] / z[:, None])[:, None], (m + np.log(z))[:, None], (p @ np.abs(v[:, 0]) / z[:, None])[:, None], terms[:, None]


def test_decode_window_over_as_many_keys_as_an_int_counts():
    """2^31 - 1 rows of one head of 8 channels, K and V in one buffer (34 GB): all of them by the window, by the sinks, or by both,
    and the last ones alone."""
    need(60)
    T, d, tail = MOST, 8, 1000
    rng = np.random.default_rng(21)
    last = ref.rounded(rng.standard_normal((tail, 1, d)), "bf16")
    q = ref.rounded(16.0 + rng.standard_normal((2, 1, d)), "bf16")
    kv = torch.zeros((T, 1, d), dtype=torch.bfloat16, device="cuda")
    kv[T - tail:] = dev(last.astype(np.float32), "bf16")
    shape = fa.Shape(2, 1, 1, d, fa.BF16)
    ctx = fa.Context(shape, 1, 1)
    qd, length = dev(q.astype(np.float32), "bf16"), torch.tensor([T], dtype=torch.int32, device="cuda")
    for window, sink, seen, zeros in ((MOST, 0, tail, T - tail), (1, MOST, tail, T - tail), (MOST - 70, 7, tail, T - tail - 64),
                                      (500, 3, 500, 3)):
        o = torch.full((2, 1, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((2, 1), float("nan"), device="cuda")
        fa.fedattn_decode_window(ctx, shape, fa.DECODE_SYNC, qd, kv, kv, 0, length, T, window, sink, o, lse)
        assert ctx.poll() == 0
        want = attend_tail(q, last[-seen:], last[-seen:], zeros, d ** -0.5)
        ref.check_attention(host(o), host(lse), want, "bf16", "window %d, %d sinks" % (window, sink), "f32")


@pytest.mark.parametrize("causal", [True, False])
def test_local_window_over_as_many_rows_as_an_int_counts(causal):
    """Two segments that end at row 2^31 - 1, one head of 8 channels, Q, K and V in one buffer (34 GB, and as much output)."""
    need(76)
    T, d, first, window, sink = MOST, 8, 1000, 70, 3
    x = torch.empty((T, 1, d), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(22))
    o = torch.full((T, 1, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    shape = fa.Shape(2, 1, 1, d, fa.BF16, causal=causal)
    ctx = fa.Context(shape, 1, 1)
    fa.fedattn_local_window(ctx, shape, x, x, x, [0, first, T], window, sink, o)
    assert ctx.poll() == 0
    for lo, rows in ((0, [0, first - 1]), (first, [first, first + 200, T // 2, T - 129, T - 71, T - 2, T - 1])):
        hi = first if lo == 0 else T
        for i in rows:
            keys = sorted(set(range(lo, min(lo + sink, hi))) | set(range(max(lo, i - window + 1), min(i + window, hi))))
            keys = [j for j in keys if j <= i or not causal]
            y = host(x[torch.tensor(keys, device="cuda")])
            want = ref.attend(host(x[i:i + 1]), y, y, np.ones((1, len(keys)), bool), d ** -0.5)
            ref.check_attention(host(o[i:i + 1]), None, want, "bf16", "row %d" % i, "f32")


def test_four_bit_cache_of_as_many_rows_as_an_int_counts():
    """2^31 - 16 rows of one head of 32 channels, K and V in the same arrays (37 GB).  The last tile has 16 rows of the cache, and behind
    the length there are some whose logits would decide everything."""
    need(50)
    cap, d, tail, behind = 2 ** 31 - 16, 32, 1000, 5
    length = cap - behind
    shape = fa.Shape(2, 1, 1, d, fa.BF16)
    ctx = fa.Context(shape, tail, 1)
    codes = torch.full((1, 1, cap, d // 2), 0x88, dtype=torch.uint8, device="cuda")      # zeros
    scales = torch.zeros((1, 1, cap, 1), dtype=torch.uint8, device="cuda")
    cache = fa.QuantCache(shape, 1, cap, codes, scales, codes, scales)
    rng = np.random.default_rng(23)
    x = ref.rounded(rng.standard_normal((tail, 1, d)), "bf16")
    at = torch.arange(length - tail, length, dtype=torch.int32, device="cuda")
    xd = dev(x.astype(np.float32), "bf16")
    fa.fedattn_quantize_kv(ctx, shape, xd, xd, at, cache)
    held = ref.values(*ref.quantise(x))
    back = torch.empty_like(xd), torch.empty_like(xd)
    fa.fedattn_dequantize_kv(ctx, shape, cache, at, *back)
    assert ctx.poll() == 0 and all(np.array_equal(host(t), held) for t in back)
    codes[:, :, length:], scales[:, :, length:] = 0xff, 200
    q = ref.rounded(8.0 + rng.standard_normal((2, 1, d)), "bf16")
    for window, sink, seen, zeros in ((0, 0, tail, length - tail), (MOST, 3, tail, length - tail), (1, MOST, tail, length - tail),
                                      (500, 40, 500, 40)):
        o, lse = torch.full((2, 1, d), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((2, 1), float("nan"), device="cuda")
        fa.fedattn_decode_quant(ctx, shape, fa.DECODE_SYNC, dev(q.astype(np.float32), "bf16"), cache,
                                torch.tensor([length], dtype=torch.int32, device="cuda"), cap, o, lse, window, sink)
        assert ctx.poll() == 0
        ref.check_attention(host(o), host(lse), attend_tail(q, held[-seen:], held[-seen:], zeros, d ** -0.5), "bf16",
                            "window %d, %d sinks" % (window, sink))
