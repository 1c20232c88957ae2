"""The norm with rotation, the windows and the 4-bit caches as a program runs them: prefill, then tokens; and random sequences of
them and of the older calls over shared buffers, whose results must not depend on what overlaps."""
import numpy as np
import pytest
import torch

import paper_2511_02647_b200 as fa
import reference64 as ref
from helpers import dev, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 8, 2), ("bf16", 64, 6, 2), ("f32", 96, 4, 4)])
def test_prefill_and_tokens_of_a_windowed_model(dtype, d, hq, hkv):
    """Three participants' prompts through one block (norm and rotation at global positions, windowed local attention, rows into
    4-bit caches), then four tokens each (norm and rotation, append, decode), then a chunk over the rows read back.  Every
    step is judged on what the one before left."""
    lens, window, sink, steps, cap, eps = [70, 1, 133], 48, 4, 4, 144, float(np.float32(1e-6))
    n, L = len(lens), sum(lens)
    cu = [0] + [int(x) for x in np.cumsum(lens)]
    rng = np.random.default_rng(d)
    shape = fa.Shape(n, hq, hkv, d, fa.BF16 if dtype == "bf16" else fa.F32)
    ctx, dt = fa.Context(shape, L, n * cap), shape.torch_dtype
    freq = [10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
    wq, wk = (ref.rounded(1 + 0.2 * rng.standard_normal(d), dtype) for _ in range(2))
    wqd, wkd = dev(wq.astype(np.float32), dtype), dev(wk.astype(np.float32), dtype)
    cache = fa.QuantCache(shape, n, cap)
    held = [np.zeros((n, cap, hkv, d)) for _ in range(2)]

    def projected(rows):
        x = ref.rounded(rng.standard_normal((rows, (hq + 2 * hkv) * d)), dtype)
        xd = dev(x.astype(np.float32), dtype)
        views = [xd[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]
        return x, views

    def rope_and_cache(rows, pos, at):
        x, (q, k, v) = projected(rows)
        qo, ko = torch.empty((rows, hq, d), dtype=dt, device="cuda"), torch.empty((rows, hkv, d), dtype=dt, device="cuda")
        posd, atd = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (pos, at))
        fa.fedattn_qk_norm_rope(ctx, shape, q, k, wqd, wkd, eps, posd, freq, False, qo, ko)
        for got, a, h, w in ((qo, 0, hq, wq), (ko, hq * d, hkv, wk)):
            want, size = ref.norm_rope(x[:, a:a + h * d].reshape(rows, h, d), w, eps, np.asarray(pos), freq, False)
            tol = 24 * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
            assert (np.abs(host(got) - want) <= tol).all()
        fa.fedattn_quantize_kv(ctx, shape, ko, v, atd, cache)
        for store, y in zip(held, (host(ko), x[:, (hq + hkv) * d:].reshape(rows, hkv, d))):
            store.reshape(n * cap, hkv, d)[at] = ref.values(*ref.quantise(y))
        return qo, ko, v.contiguous()

    at = [i * cap + j for i in range(n) for j in range(lens[i])]
    q, k, v = rope_and_cache(L, list(range(L)), at)
    o, lse = torch.empty_like(q), torch.empty((L, hq), device="cuda")
    fa.fedattn_local_window(ctx, shape, q, k, v, cu, window, sink, o, lse)
    weights = "bf16" if dtype == "bf16" and d == 128 else "f32"
    for a, b in zip(cu[:-1], cu[1:]):
        want = ref.attend(host(q)[a:b], host(k)[a:b], host(v)[a:b], ref.window_mask(b - a, window, sink, True), d ** -0.5)
        ref.check_attention(host(o)[a:b], host(lse)[a:b], want, dtype, "prefill", weights)

    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    od, lsed = torch.empty((n, hq, d), dtype=dt, device="cuda"), torch.empty((n, hq), device="cuda")
    for t in range(steps):
        now = [m + t for m in lens]
        q, _, _ = rope_and_cache(n, [L + t] * n, [i * cap + now[i] for i in range(n)])
        length += 1
        fa.fedattn_decode_quant(ctx, shape, fa.DECODE_LOCAL, q, cache, length, max(now) + 1, od, lsed, window, sink)
        for i in range(n):
            j = np.arange(cap)
            seen = (j < now[i] + 1) & ((j >= now[i] + 1 - window) | (j < sink))
            want = ref.attend(host(q)[i:i + 1], held[0][i], held[1][i], seen[None], d ** -0.5)
            ref.check_attention(host(od)[i:i + 1], host(lsed)[i:i + 1], want, dtype, "token %d of %d" % (t, i))

    rows = [2 * cap + j for j in range(lens[2] + steps)]
    kb, vb = (torch.empty((len(rows), hkv, d), dtype=dt, device="cuda") for _ in range(2))
    fa.fedattn_dequantize_kv(ctx, shape, cache, torch.tensor(rows, dtype=torch.int32, device="cuda"), kb, vb)
    assert np.array_equal(host(kb), held[0][2, :len(rows)]) and np.array_equal(host(vb), held[1][2, :len(rows)])
    chunk = dev(ref.rounded(rng.standard_normal((9, hq, d)), dtype).astype(np.float32), dtype)
    oc, lsec = torch.empty_like(chunk), torch.empty((9, hq), device="cuda")
    pos = torch.arange(len(rows) - 9, len(rows), dtype=torch.int32, device="cuda")
    fa.fedattn_sync(ctx, shape, chunk, pos, kb, vb, None, len(rows), False, oc, lsec)
    assert ctx.poll() == 0
    want = ref.attend(host(chunk), held[0][2, :len(rows)], held[1][2, :len(rows)], np.arange(len(rows)) <= host(pos)[:, None], d ** -0.5)
    # (fedattn_sync of bf16 at 128 channels takes a quarter of its exponentials from a polynomial of relative error 7.5e-5: not its lse)
    ref.check_attention(host(oc), None if weights == "bf16" else host(lsec), want, dtype, "chunk", weights)


def sequence(dtype, d, hq, hkv, seed, mode, n_ops=36):
    N, L, cap, T = 3, 80, 96, 1408
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    shape = fa.Shape(N, hq, hkv, d, fa.BF16 if dtype == "bf16" else fa.F32)
    ctx = fa.Context(shape, N * L, T)
    g = torch.Generator(device="cuda").manual_seed(5)

    def new(*s):
        return torch.randn(s, generator=g, device="cuda").to(dt)

    def ints(xs):
        return torch.tensor(xs, dtype=torch.int32, device="cuda")

    rows, cu = N * L, [0, L, 2 * L, N * L]
    q, k, v, q2, k2 = new(rows, hq, d), new(rows, hkv, d), new(rows, hkv, d), new(rows, hq, d), new(rows, hkv, d)
    o, lse = [torch.zeros_like(q) for _ in range(2)], [torch.zeros(rows, hq, device="cuda") for _ in range(2)]
    od, lsed = [torch.zeros(N, hq, d, dtype=dt, device="cuda") for _ in range(3)], torch.zeros(N, hq, device="cuda")
    local, shared = fa.QuantCache(shape, N, cap), fa.QuantCache(shape, 1, T)
    kt, vt = torch.zeros(hkv, N * 16, d, dtype=dt, device="cuda"), torch.zeros(hkv, N * 16, d, dtype=dt, device="cuda")
    post, sel = torch.zeros(hkv, N * 16, dtype=torch.int32, device="cuda"), torch.zeros(hkv, N * 16, dtype=torch.int32, device="cuda")
    at, back = ints([(i // L) * cap + i % L for i in range(rows)]), ints([(i * 7) % rows for i in range(rows)])
    spread = ints([(i * 5) % T for i in range(rows)])
    pos, lens, total, plain = ints(range(rows)), ints([L, 17, cap]), ints([T]), ints([L] * N)
    freq = [100.0 ** (-2.0 * i / d) for i in range(d // 2)]
    snaps = torch.zeros(n_ops // 6, 3, N, hq, d, dtype=dt, device="cuda")

    def split(x):
        return [x[cu[i]:cu[i + 1]] for i in range(N)]

    calls = [
        lambda: fa.fedattn_qk_norm_rope(ctx, shape, q, k, None, None, 1e-5, pos, freq, False, q2, k2),
        lambda: fa.fedattn_qk_norm_rope(ctx, shape, o[0], None, None, None, 1e-5, pos, freq, True, q2, None),
        lambda: fa.fedattn_local_window(ctx, shape, q2, k2, v, cu, 20, 3, o[0], lse[0]),
        lambda: fa.fedattn_local(ctx, shape, q2, k2, v, cu, o[1], lse[1]),
        lambda: fa.fedattn_quantize_kv(ctx, shape, k2, v, at, local),
        lambda: fa.fedattn_quantize_kv(ctx, shape, k2, v, spread, shared),
        lambda: fa.fedattn_dequantize_kv(ctx, shape, shared, back, k2, v),
        # a decode's output is the next one's query
        lambda: fa.fedattn_decode_quant(ctx, shape, fa.DECODE_LOCAL, od[2], local, lens, cap, od[0], lsed, 30, 2),
        lambda: fa.fedattn_decode_quant(ctx, shape, fa.DECODE_SYNC, od[0], shared, total, T, od[1]),
        lambda: fa.fedattn_decode_window(ctx, shape, fa.DECODE_LOCAL, od[1], k2, v, L * hkv * d, plain, L, 33, 4, od[2]),
        lambda: fa.fedattn_decode(ctx, shape, fa.DECODE_SYNC, o[0][:N], k2, v, 0, plain[:1], L, od[2]),
        lambda: fa.fedattn_aggregate_kv(ctx, shape, fa.AGG_TOPK_KNORM, split(k2), split(v), [L] * N, [16] * N, None, kt, vt, post, None, sel),
        lambda: fa.fedattn_merge(ctx, shape, N, od[0], lsed, od[1], lsed, od[2]),
        lambda: od[2].add_(od[1]).mul_(0.5),
    ]
    for i in (0, 4, 5, 2):
        calls[i]()
    od[2].copy_(q[:N])
    order = np.random.default_rng(seed).integers(0, len(calls), n_ops)
    torch.cuda.synchronize()

    def walk():
        for i, c in enumerate(order):
            calls[c]()
            if mode == "synchronised":
                torch.cuda.synchronize()
            if i % 6 == 5:
                for j in range(3):
                    snaps[i // 6, j].copy_(od[j])

    if mode == "graph":
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            walk()
        graph.replay()
    elif mode == "stream":
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            walk()
    else:
        walk()
    torch.cuda.synchronize()
    assert ctx.poll() == 0
    return [snaps, q2, k2, v, kt, vt, post, lsed, *o, *lse, *od, *local.arrays(), *shared.arrays()]


@pytest.mark.parametrize("dtype,d,hq,hkv", [("bf16", 128, 8, 2), ("bf16", 64, 4, 2), ("f32", 96, 4, 4), ("bf16", 128, 24, 2)])
@pytest.mark.parametrize("seed", range(4))
def test_sequences_without_synchronisation(dtype, d, hq, hkv, seed):
    want = sequence(dtype, d, hq, hkv, seed, "synchronised")
    for mode in ("free", "stream", "graph"):
        for i, (a, b) in enumerate(zip(sequence(dtype, d, hq, hkv, seed, mode), want)):
            assert torch.equal(a, b), (mode, i)


def test_two_contexts_at_once_on_two_streams():
    """Calls that overlap on the GPU share nothing but their inputs when each stream has a context of its own."""
    n, hq, hkv, d, cap = 8, 32, 2, 128, 4096
    shape = fa.Shape(n, hq, hkv, d, fa.BF16)
    gen = torch.Generator(device="cuda").manual_seed(7)
    cache = fa.QuantCache(shape, 1, cap, *[torch.randint(0, 256, (1, hkv, cap, w), dtype=torch.uint8, device="cuda", generator=gen) for w in (64, 4) * 2])
    cache.k_scales.fill_(18 * 8)
    cache.v_scales.fill_(18 * 8)
    length = torch.tensor([cap], dtype=torch.int32, device="cuda")
    qs = [torch.randn((n, hq, d), device="cuda", generator=gen).bfloat16() for _ in range(2)]
    ctxs, streams = [fa.Context(shape, n, cap) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    want = []
    for c, q in zip(ctxs, qs):
        want.append(torch.empty_like(q))
        fa.fedattn_decode_quant(c, shape, fa.DECODE_SYNC, q, cache, length, cap, want[-1])
        torch.cuda.synchronize()
    outs = [[torch.empty_like(qs[0]) for _ in range(20)] for _ in range(2)]
    for i in range(20):
        for c, q, s, o in zip(ctxs, qs, streams, outs):
            fa.fedattn_decode_quant(c, shape, fa.DECODE_SYNC, q, cache, length, cap, o[i], stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w, x) for x in o)


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("cap,window", [(300, 100), (20000, 15000)])
def test_windowed_decodes_that_feed_one_another(d, cap, window):
    """Every output is the next call's queries, in one launch and in two: as with a synchronisation behind each call, and replayed."""
    n, hq, hkv = 3, 8, 2
    g = torch.Generator(device="cuda").manual_seed(d)
    shape = fa.Shape(n, hq, hkv, d, fa.BF16)
    ctx = fa.Context(shape, n, cap)
    k, v = (torch.randn((cap, hkv, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    start = torch.randn((n, hq, d), generator=g, device="cuda").bfloat16()
    length = torch.tensor([cap], dtype=torch.int32, device="cuda")
    x = [start.clone() for _ in range(3)]

    def chain(wait):
        for i in range(12):
            fa.fedattn_decode_window(ctx, shape, fa.DECODE_SYNC, x[i % 3], k, v, 0, length, cap, window, 4, x[(i + 1) % 3])
            if wait:
                torch.cuda.synchronize()
        return x[0].clone()

    def again(run):
        x[0].copy_(start)
        out = run()
        torch.cuda.synchronize()
        return out

    want = again(lambda: chain(True))
    assert torch.equal(again(lambda: chain(False)), want)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        chain(False)

    def replay():
        graph.replay()
        return x[0].clone()

    for _ in range(2):
        assert torch.equal(again(replay), want)
