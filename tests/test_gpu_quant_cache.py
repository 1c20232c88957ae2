"""The 4-bit cache: rows in and out bit for bit, decode against the softmax in 64 bits over the values the cache holds."""
import numpy as np
import pytest
import torch

import paper_2511_02647_b200 as fa
import reference64 as ref
from helpers import dev, host

pytestmark = pytest.mark.gpu


def code_of(dtype):
    return fa.BF16 if dtype == "bf16" else fa.F32


def rows_of(rng, n, hkv, d, dtype):
    """Rows over the whole range of scales, with zero groups, ties and group maxima at the border of two scales among them."""
    x = rng.standard_normal((n, hkv, d)) * np.exp2(rng.integers(-24, 20, (n, hkv, 1)))
    x[rng.random((n, hkv)) < 0.05] = 0
    s = ref.SCALES[rng.integers(0, 256, (n, hkv, 1))]
    ties = (rng.integers(-7, 7, (n, hkv, d)) + 0.5) * s
    ties[..., 0::32] = 7 * s                                      # the scale is s exactly
    pick = rng.random((n, hkv)) < 0.3
    x[pick] = ties[pick]
    return ref.rounded(x, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("n,hkv", [(1, 1), (75, 3), (512, 8)])
def test_rows_in_and_out_are_exact(dtype, d, n, hkv):
    rng = np.random.default_rng([d, n, hkv])
    k, v = rows_of(rng, n, hkv, d, dtype), rows_of(rng, n, hkv, d, dtype)
    caches, cap = 3, 16 * (-(-n // 32) + 1)
    shape = fa.Shape(caches, hkv, hkv, d, code_of(dtype))
    ctx = fa.Context(shape, n, n)
    cache = fa.QuantCache(shape, caches, cap)
    for t in cache.arrays():
        t.fill_(0xA5)
    at = rng.permutation(caches * cap)[:n].astype(np.int32)
    if n > 1:
        at[n // 2] = -1                                           # skipped
    atd = torch.from_numpy(at).cuda()
    wide = torch.cat([dev(k.astype(np.float32), dtype), dev(v.astype(np.float32), dtype)], 1)          # strided rows
    fa.fedattn_quantize_kv(ctx, shape, wide[:, :hkv], wide[:, hkv:], atd, cache)
    ko = torch.full((n, hkv, d), 9.0, dtype=wide.dtype, device="cuda")
    vo = ko.clone()
    fa.fedattn_dequantize_kv(ctx, shape, cache, atd, ko, vo)
    assert ctx.poll() == 0
    for x, codes, scales, out in ((k, cache.k_codes, cache.k_scales, ko), (v, cache.v_codes, cache.v_scales, vo)):
        code, byte = ref.quantise(x)
        want_c = np.full((caches, cap, hkv, d // 2), 0xA5, np.uint8)
        want_s = np.full((caches, cap, hkv, d // 32), 0xA5, np.uint8)
        for i in range(n):
            if at[i] >= 0:
                want_c[at[i] // cap, at[i] % cap], want_s[at[i] // cap, at[i] % cap] = ref.pack(code[i]), byte[i]
        assert np.array_equal(scales.cpu().numpy(), want_s.transpose(0, 2, 1, 3))
        assert np.array_equal(codes.cpu().numpy(), want_c.transpose(0, 2, 1, 3))
        want = np.where((at >= 0)[:, None, None], ref.values(code, byte), 9.0)
        assert np.array_equal(host(out), want)


def test_an_index_beyond_the_caches_is_reported_and_skipped():
    shape = fa.Shape(2, 2, 2, 64, fa.BF16)
    ctx = fa.Context(shape, 4, 4)
    cache = fa.QuantCache(shape, 2, 16)
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([31, 32, 0], dtype=torch.int32, device="cuda")
    fa.fedattn_quantize_kv(ctx, shape, x, x, at, cache)
    assert ctx.poll() == 6
    out = torch.full_like(x, 5.0)
    fa.fedattn_dequantize_kv(ctx, shape, cache, at, out, out.clone())
    assert ctx.poll() == 6
    assert (out[1] == 5.0).all() and (out[0] - 1).abs().max() < 0.08 and torch.equal(out[0], out[2])
    fa.fedattn_quantize_kv(ctx, shape, x[:1], x[:1], at[:1], cache)
    assert ctx.poll() == 0


def filled(rng, shape, caches, cap, lens):
    """Caches of quantised rows with channels of different size; behind every length, garbage."""
    hkv, d = shape.n_kv_heads, shape.head_dim
    held = {}
    arrays = {}
    for x in "kv":
        rows = rng.standard_normal((caches, hkv, cap, d)) * np.exp(0.7 * rng.standard_normal((caches, hkv, 1, d)))
        code, byte = ref.quantise(ref.rounded(rows, "bf16"))
        codes, scales = ref.pack(code), byte.astype(np.uint8)
        for c in range(caches):
            codes[c, :, lens[c]:] = rng.integers(0, 256, codes[c, :, lens[c]:].shape)
            scales[c, :, lens[c]:] = 255
        held[x] = ref.values(code, byte).transpose(0, 2, 1, 3)
        arrays[x + "_codes"], arrays[x + "_scales"] = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    return fa.QuantCache(shape, caches, cap, **arrays), held["k"], held["v"]


def decode(mode, dtype, n, hq, hkv, d, lens, cap, window=0, sink=0, spread=1.0, most=None, stale=0):
    rng = np.random.default_rng([n, hq, d, cap, window])
    shape = fa.Shape(n, hq, hkv, d, code_of(dtype))
    ctx = fa.Context(shape, n, cap)
    caches = 1 if mode == fa.DECODE_SYNC else n
    cache, k, v = filled(rng, shape, caches, cap, lens)
    q = ref.rounded(rng.standard_normal((n, hq, d)) * spread, dtype)
    o = torch.full((n, hq, d), float("nan"), dtype=shape.torch_dtype, device="cuda")
    lse = torch.full((n, hq), float("nan"), device="cuda")
    qd = dev(q.astype(np.float32), dtype)
    lend = torch.tensor(lens, dtype=torch.int32, device="cuda")
    args = (ctx, shape, mode, qd, cache, lend, max(lens) if most is None else most, o, lse, window, sink)
    fa.fedattn_decode_quant(*args)
    assert ctx.poll() == 0
    j = np.arange(cap)
    for i in range(n):
        c = 0 if mode == fa.DECODE_SYNC else i
        seen = j < lens[c]
        if window:
            seen &= (j >= lens[c] - window) | (j < sink)
        want = ref.attend(q[i:i + 1], k[c], v[c], seen[None], d ** -0.5)
        ref.check_attention(host(o)[i:i + 1], host(lse)[i:i + 1], want, dtype, "participant %d" % i)
    return args


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (14, 2), (20, 1)])
def test_local_decode_of_ragged_caches(dtype, d, hq, hkv):
    decode(fa.DECODE_LOCAL, dtype, 7, hq, hkv, d, [0, 1, 15, 16, 33, 200, 130], 208)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,hq,hkv,d,length", [(1, 4, 4, 128, 700), (3, 8, 2, 64, 1), (8, 32, 8, 128, 333), (5, 12, 2, 96, 1000),
                                               (16, 8, 2, 128, 517), (2, 2, 1, 32, 0)])
def test_shared_decode(dtype, n, hq, hkv, d, length):
    decode(fa.DECODE_SYNC, dtype, n, hq, hkv, d, [length], 1008)


@pytest.mark.parametrize("mode", ["local", "sync"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (16, 4), (31, 40), (100, 5), (600, 4), (2 ** 31 - 1, 2 ** 31 - 1), (50, 1000)])
def test_window_and_sinks(mode, d, window, sink):
    m = fa.DECODE_SYNC if mode == "sync" else fa.DECODE_LOCAL
    decode(m, "bf16", 4, 8, 2, d, [601] if m else [601, 3, 0, 97], 608, window, sink)


@pytest.mark.parametrize("dtype,n,hq,hkv,d,length", [("bf16", 2, 8, 2, 128, 9000), ("bf16", 8, 8, 2, 64, 9001), ("f32", 3, 2, 1, 96, 8200),
                                                     ("bf16", 12, 4, 2, 32, 20000)])
def test_long_shared_caches_take_the_two_launch_form(dtype, n, hq, hkv, d, length):
    args = decode(fa.DECODE_SYNC, dtype, n, hq, hkv, d, [length], -(-length // 16) * 16)
    ctx = args[0]
    before = ctx.launch_count()
    fa.fedattn_decode_quant(*args)
    assert ctx.launch_count() - before == 2


@pytest.mark.parametrize("mode,n,hq,hkv,lens,window,sink,spread", [
    ("sync", 8, 8, 2, [9001], 0, 0, 1.0), ("sync", 8, 8, 2, [2049], 0, 0, 40.0), ("sync", 5, 8, 2, [2300], 0, 0, 0.0),
    ("sync", 17, 8, 2, [3333], 0, 0, 1.0), ("sync", 8, 16, 4, [20000], 5000, 4, 1.0), ("sync", 8, 8, 2, [2500], 2200, 300, 8.0),
    ("sync", 8, 8, 2, [2560], 1, 2040, 1.0), ("local", 3, 24, 1, [0, 2100, 129], 0, 0, 1.0), ("local", 2, 64, 2, [5000, 127], 0, 0, 3.0),
    ("sync", 8, 8, 2, [1], 0, 0, 1.0), ("sync", 8, 8, 2, [0], 0, 0, 1.0)])
def test_many_rows_to_a_key(mode, n, hq, hkv, lens, window, sink, spread):
    """More than 16 query rows share the keys of long caches: four column tiles to a warp, several chunks of rows."""
    cap = max(-(-max(lens) // 16) * 16, 4096)
    decode(fa.DECODE_SYNC if mode == "sync" else fa.DECODE_LOCAL, "bf16", n, hq, hkv, 128, lens, cap, window, sink, spread, most=max(max(lens), 4096))


def test_references_that_grow_along_the_walk():
    """Keys whose logits rise from tile to tile by far more than 2^8 a time, and fall again."""
    d, n, hq, length = 128, 8, 4, 4096
    shape = fa.Shape(n, hq, 1, d, fa.BF16)
    ctx = fa.Context(shape, n, length)
    rng = np.random.default_rng(8)
    level = np.concatenate([np.linspace(-60, 60, length // 2), np.linspace(60, -60, length // 2)])
    k = rng.standard_normal((1, 1, length, d)) * 0.1 + (level / d ** 0.5)[None, None, :, None]
    v = rng.standard_normal((1, 1, length, d))
    (kc, kb), (vc, vb) = ref.quantise(ref.rounded(k, "bf16")), ref.quantise(ref.rounded(v, "bf16"))
    cache = fa.QuantCache(shape, 1, length, *(torch.from_numpy(x).cuda() for x in
                          (ref.pack(kc), kb.astype(np.uint8), ref.pack(vc), vb.astype(np.uint8))))
    q = ref.rounded(np.abs(rng.standard_normal((n, hq, d))) + 0.5, "bf16")
    o, lse = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((n, hq), device="cuda")
    fa.fedattn_decode_quant(ctx, shape, fa.DECODE_SYNC, dev(q.astype(np.float32), "bf16"), cache,
                            torch.tensor([length], dtype=torch.int32, device="cuda"), length, o, lse)
    assert ctx.poll() == 0
    want = ref.attend(q, ref.values(kc, kb)[0].transpose(1, 0, 2), ref.values(vc, vb)[0].transpose(1, 0, 2), np.ones((n, length), bool), d ** -0.5)
    ref.check_attention(host(o), host(lse), want, "bf16")


@pytest.mark.parametrize("spread", [0.0, 30.0, 3000.0])
def test_flat_and_steep_rows(spread):
    decode(fa.DECODE_LOCAL, "bf16", 3, 8, 2, 128, [300, 47, 160], 304, spread=spread)


def test_lengths_beyond_the_bound_count_as_the_bound():
    shape = fa.Shape(2, 4, 2, 128, fa.BF16)
    ctx = fa.Context(shape, 2, 64)
    rng = np.random.default_rng(3)
    cache, _, _ = filled(rng, shape, 2, 64, [64, 64])
    q = torch.randn((2, 4, 128), device="cuda").bfloat16()
    a, b = torch.empty_like(q), torch.empty_like(q)
    fa.fedattn_decode_quant(ctx, shape, fa.DECODE_LOCAL, q, cache, torch.tensor([48, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), 48, a)
    fa.fedattn_decode_quant(ctx, shape, fa.DECODE_LOCAL, q, cache, torch.tensor([48, 48], dtype=torch.int32, device="cuda"), 48, b)
    assert torch.equal(a, b)
    fa.fedattn_decode_quant(ctx, shape, fa.DECODE_LOCAL, q, cache, torch.tensor([-5, 48], dtype=torch.int32, device="cuda"), 48, b)
    assert (b[0] == 0).all() and torch.equal(a[1], b[1])


def test_results_repeat_and_survive_a_graph():
    rng = np.random.default_rng(11)
    shape = fa.Shape(4, 8, 2, 128, fa.BF16)
    ctx = fa.Context(shape, 4, 20000)
    cache, _, _ = filled(rng, shape, 1, 20000, [20000])
    length = torch.tensor([20000], dtype=torch.int32, device="cuda")
    q, o = torch.randn((4, 8, 128), device="cuda").bfloat16(), torch.empty((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    call = fa.prepare_decode_quant(ctx, shape, fa.DECODE_SYNC, q, cache, length, 20000, o)
    call()
    first = o.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            fa.fedattn_decode_quant(ctx, shape, fa.DECODE_SYNC, q, cache, length, 20000, o)
    for _ in range(3):
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, first)


def test_what_the_binding_refuses():
    shape = fa.Shape(2, 4, 2, 64, fa.BF16)
    ctx = fa.Context(shape, 4, 4)
    cache = fa.QuantCache(shape, 2, 32)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    length = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        fa.QuantCache(shape, 2, 30)
    with pytest.raises(ValueError):
        fa.QuantCache(fa.Shape(2, 4, 2, 72, fa.BF16), 2, 32)
    with pytest.raises(ValueError):
        fa.fedattn_quantize_kv(ctx, shape, x, x[:3], None, cache)
    with pytest.raises(ValueError):
        fa.fedattn_quantize_kv(ctx, shape, x, x, torch.zeros(4, dtype=torch.int64, device="cuda"), cache)
    with pytest.raises(ValueError):
        fa.fedattn_decode_quant(ctx, shape, fa.DECODE_SYNC, q, cache, length[:1], 32, q)
    with pytest.raises(ValueError):
        fa.fedattn_decode_quant(ctx, shape, fa.DECODE_LOCAL, q, cache, length[:1], 32, q)
    with pytest.raises(fa.FedAttnError):
        fa.fedattn_decode_quant(ctx, shape, fa.DECODE_LOCAL, q, cache, length, 48, q)
