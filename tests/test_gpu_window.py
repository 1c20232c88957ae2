"""Attention through a sliding window with sinks, local and decode, against the softmax in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2511_02647_b200 as fa
import reference64 as ref
from helpers import dev, host

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


def shape_of(n, hq, hkv, d, dtype, causal=True, scale=0.0):
    return fa.Shape(n, hq, hkv, d, fa.BF16 if dtype == "bf16" else fa.F32, int(causal), scale)


def weights_of(dtype, d):
    """bf16 at head_dim 128 keeps its softmax weights in bf16, below in two bf16 parts (or better), fp32 in fp32."""
    return "f32" if dtype == "f32" else ("bf16" if d == 128 else "2 x bf16")


def local(dtype, hq, hkv, d, lens, window, sink, causal=True, spread=1.0, check=None):
    rng = np.random.default_rng([hq, d, sum(lens), window % 1000, sink % 1000])
    L, n = sum(lens), len(lens)
    cu = [0] + [int(x) for x in np.cumsum(lens)]
    q, k, v = (ref.rounded(rng.standard_normal((L, h, d)) * s, dtype) for h, s in ((hq, spread), (hkv, 1.0), (hkv, 1.0)))
    shape = shape_of(n, hq, hkv, d, dtype, causal)
    ctx = fa.Context(shape, L, L)
    qd, kd, vd = (dev(x.astype(np.float32), dtype) for x in (q, k, v))
    o = torch.full_like(qd, float("nan"))
    lse = torch.full((L, hq), float("nan"), device="cuda")
    fa.fedattn_local_window(ctx, shape, qd, kd, vd, cu, window, sink, o, lse)
    assert ctx.poll() == 0
    go, gl = host(o), host(lse)
    assert np.isfinite(go).all()
    for a, b in zip(cu[:-1], cu[1:]):
        rows = np.arange(b - a) if check is None else np.unique(rng.integers(0, max(1, b - a), check)) if b > a else np.arange(0)
        mask = ref.window_mask(b - a, window, sink, causal, rows)
        want = ref.attend(q[a:b][rows], k[a:b], v[a:b], mask, d ** -0.5)
        ref.check_attention(go[a:b][rows], gl[a:b][rows], want, dtype, "segment at %d" % a, weights_of(dtype, d))
    return ctx


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 64, 96, 8, 120])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,sink", [(1, 0), (2, 1), (64, 4), (100, 0), (129, 300)])
def test_ragged_segments(dtype, d, causal, window, sink):
    local(dtype, 4, 2, d, [1, 130, 0, 257, 64], window, sink, causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sink", [(MOST, 0), (MOST, MOST), (1, MOST), (700, 0), (701, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_windows_and_sinks_beyond_the_lengths(dtype, window, sink, causal):
    local(dtype, 2, 1, 128, [700, 33], window, sink, causal, check=60)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hq,hkv", [(3, 3), (6, 2), (7, 1), (8, 8), (10, 2)])
@pytest.mark.parametrize("window,sink,causal", [(150, 5, True), (40, 129, False), (256, 0, True)])
def test_groups_of_every_form(d, hq, hkv, window, sink, causal):
    """Pairs of heads, lone heads, heads that straddle two query tiles, and halves."""
    local("bf16", hq, hkv, d, [600, 470, 129], window, sink, causal, check=40)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("bf16", 96), ("f32", 128)])
@pytest.mark.parametrize("lens", [[2048, 1500], [9001]])
def test_long_segments_skip_what_no_row_sees(dtype, d, lens):
    local(dtype, 8, 2, d, lens, 300, 4, True, check=40)


@pytest.mark.parametrize("hq,hkv", [(12, 4), (10, 2), (9, 3)])
def test_many_items(hq, hkv):
    local("bf16", hq, hkv, 128, [3000, 2500, 1, 4000, 777], 513, 7, True, check=25)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("spread", [0.0, 40.0])
def test_flat_and_steep_rows(dtype, d, spread):
    local(dtype, 4, 2, d, [300, 140], 70, 3, True, spread)


@pytest.mark.parametrize("causal", [True, False])
def test_first_seen_keys_may_lie_far_below_the_reference(causal):
    """Rows of a tile whose first tile shows them nothing, and rows whose sinks are far above or below the window's logits."""
    d, L = 128, 500
    rng = np.random.default_rng(9)
    q, k, v = (ref.rounded(rng.standard_normal((L, 2, d)), "bf16") for _ in range(3))
    for level in (-20.0, 20.0):
        kk = k.copy()
        kk[:4] = ref.rounded(level * np.ones((4, 2, d)) / d ** 0.5, "bf16")
        qq = ref.rounded(np.abs(q), "bf16")
        shape = shape_of(1, 2, 2, d, "bf16", causal)
        ctx = fa.Context(shape, L, L)
        qd, kd, vd = (dev(x.astype(np.float32), "bf16") for x in (qq, kk, v))
        o, lse = torch.full_like(qd, float("nan")), torch.full((L, 2), float("nan"), device="cuda")
        fa.fedattn_local_window(ctx, shape, qd, kd, vd, [0, L], 33, 4, o, lse)
        assert ctx.poll() == 0
        want = ref.attend(qq, kk, v, ref.window_mask(L, 33, 4, causal), d ** -0.5)
        ref.check_attention(host(o), host(lse), want, "bf16")


def test_bf16_runs_on_the_tensor_cores_without_lse():
    shape = shape_of(2, 4, 2, 128, "bf16")
    ctx = fa.Context(shape, 600, 600)
    x = torch.randn((600, 4, 128), device="cuda").bfloat16()
    kv = torch.randn((600, 2, 128), device="cuda").bfloat16()
    a, b, lse = torch.empty_like(x), torch.empty_like(x), torch.empty((600, 4), device="cuda")
    fa.fedattn_local_window(ctx, shape, x, kv, kv, [0, 333, 600], 99, 2, a)
    fa.fedattn_local_window(ctx, shape, x, kv, kv, [0, 333, 600], 99, 2, b, lse)
    assert ctx.tensor_core_launch_count() == 2 and torch.equal(a, b)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 96), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_non_finite_values_outside_the_windows_stay_there(dtype, d, causal):
    """Rows that do not see the bad key are as without it (head dims below 128 and fp32: non-finite rows are redone without it)."""
    L, bad, window, sink = 400, 200, 50, 3
    rng = np.random.default_rng(4)
    q, k, v = (ref.rounded(rng.standard_normal((L, 2, d)), dtype) for _ in range(3))
    shape = shape_of(1, 2, 2, d, dtype, causal)
    ctx = fa.Context(shape, L, L)
    qd, kd, vd = (dev(x.astype(np.float32), dtype) for x in (q, k, v))
    vd[bad] = float("inf")
    kd[bad + 1] = float("nan")
    o = torch.empty_like(qd)
    fa.fedattn_local_window(ctx, shape, qd, kd, vd, [0, L], window, sink, o)
    mask = ref.window_mask(L, window, sink, causal)
    clean = np.flatnonzero(~mask[:, bad] & ~mask[:, bad + 1])
    want = ref.attend(q[clean], k, v, mask[clean], d ** -0.5)
    ref.check_attention(host(o)[clean], None, want, dtype, weights=weights_of(dtype, d))


def decode(mode, dtype, n, hq, hkv, d, lens, cap, window, sink, spread=1.0, behind=float("nan")):
    rng = np.random.default_rng([n, hq, d, cap, window % 1000])
    shape = shape_of(n, hq, hkv, d, dtype)
    ctx = fa.Context(shape, n, cap)
    caches = 1 if mode == fa.DECODE_SYNC else n
    q = ref.rounded(rng.standard_normal((n, hq, d)) * spread, dtype)
    k, v = (ref.rounded(rng.standard_normal((caches, cap, hkv, d)), dtype) for _ in range(2))
    qd, kd, vd = (dev(x.astype(np.float32), dtype) for x in (q, k, v))
    for c in range(caches):
        kd[c, lens[c]:] = behind
        vd[c, lens[c]:] = behind
    o, lse = torch.full_like(qd, float("nan")), torch.full((n, hq), float("nan"), device="cuda")
    fa.fedattn_decode_window(ctx, shape, mode, qd, kd, vd, cap * hkv * d, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                             max(lens), window, sink, o, lse)
    assert ctx.poll() == 0
    for i in range(n):
        c = 0 if mode == fa.DECODE_SYNC else i
        j = np.arange(cap)
        seen = (j < lens[c]) & ((j >= lens[c] - window) | (j < sink))
        want = ref.attend(q[i:i + 1], k[c], v[c], seen[None], d ** -0.5)
        ref.check_attention(host(o)[i:i + 1], host(lse)[i:i + 1], want, dtype, "participant %d" % i, weights_of(dtype, d))
    return ctx


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 40)])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (64, 4), (63, 65), (200, 0), (5, 1000), (MOST, MOST)])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (20, 1)])
def test_decode_of_ragged_caches(dtype, d, window, sink, hq, hkv):
    decode(fa.DECODE_LOCAL, dtype, 6, hq, hkv, d, [0, 1, 64, 300, 65, 257], 300, window, sink)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 96), ("f32", 64)])
@pytest.mark.parametrize("window,sink", [(3, 0), (100, 70), (1000, 4), (2500, 4)])
def test_decode_of_a_shared_cache(dtype, d, window, sink):
    decode(fa.DECODE_SYNC, dtype, 5, 8, 2, d, [2801], 2816, window, sink)


@pytest.mark.parametrize("window,launches", [(600, 1), (30000, 2)])
def test_decode_in_one_and_in_two_launches(window, launches):
    ctx = decode(fa.DECODE_SYNC, "bf16", 3, 8, 2, 128, [40001], 40001, window, 130)
    assert ctx.launch_count() == launches


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("hq,hkv,n,window,launches", [(4, 4, 3, 777, 1), (7, 1, 3, 30000, 2), (12, 1, 3, 65, 1)])
def test_decode_at_every_head_dim_of_the_tensor_cores(d, hq, hkv, n, window, launches):
    ctx = decode(fa.DECODE_SYNC, "bf16", n, hq, hkv, d, [40001], 40001, window, 130)
    assert ctx.launch_count() == launches


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("mode", [fa.DECODE_LOCAL, fa.DECODE_SYNC])
def test_decode_never_multiplies_rows_behind_the_window(d, mode):
    """Between the sinks and the window lie Inf and NaN, in the tiles that both reach into."""
    n, hq, hkv, L, window, sink = 2, 4, 2, 331, 100, 5
    rng = np.random.default_rng(d)
    shape = shape_of(n, hq, hkv, d, "bf16")
    ctx = fa.Context(shape, n, L)
    q = ref.rounded(rng.standard_normal((n, hq, d)), "bf16")
    k, v = (ref.rounded(rng.standard_normal((n, L, hkv, d)), "bf16") for _ in range(2))
    qd, kd, vd = (dev(x.astype(np.float32), "bf16") for x in (q, k, v))
    kd[:, sink:L - window] = float("nan")
    vd[:, sink:L - window] = float("inf")
    o = torch.empty_like(qd)
    lens = torch.tensor([L] * (1 if mode == fa.DECODE_SYNC else n), dtype=torch.int32, device="cuda")
    fa.fedattn_decode_window(ctx, shape, mode, qd, kd, vd, L * hkv * d, lens, L, window, sink, o)
    j = np.arange(L)
    seen = (j >= L - window) | (j < sink)
    for i in range(n):
        c = 0 if mode == fa.DECODE_SYNC else i
        want = ref.attend(q[i:i + 1], k[c], v[c], seen[None], d ** -0.5)
        ref.check_attention(host(o)[i:i + 1], None, want, "bf16", weights=weights_of("bf16", d))


def test_decode_sees_what_the_last_row_of_a_local_call_sees():
    d, L, hq, hkv = 128, 391, 4, 2
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn((L, h, d), generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    shape = shape_of(1, hq, hkv, d, "bf16")
    ctx = fa.Context(shape, L, L)
    o, od = torch.empty_like(q), torch.empty((1, hq, d), dtype=q.dtype, device="cuda")
    lse, lsed = torch.empty((L, hq), device="cuda"), torch.empty((1, hq), device="cuda")
    fa.fedattn_local_window(ctx, shape, q, k, v, [0, L], 100, 4, o, lse)
    fa.fedattn_decode_window(ctx, shape, fa.DECODE_LOCAL, q[-1:].contiguous(), k[None], v[None], 0,
                             torch.tensor([L], dtype=torch.int32, device="cuda"), L, 100, 4, od, lsed)
    # the same key set, weights in bf16 (2^-8 each) and a rounding of the output each: magnitudes below 4
    assert (o[-1].float() - od[0].float()).abs().max() < 4 * 2.0 ** -8 * 4
    assert (lse[-1] - lsed[0]).abs().max() < 1e-4


def test_what_is_refused():
    shape = shape_of(1, 2, 2, 64, "bf16")
    ctx = fa.Context(shape, 8, 8)
    x = torch.zeros((8, 2, 64), dtype=torch.bfloat16, device="cuda")
    one = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    length = torch.zeros(1, dtype=torch.int32, device="cuda")
    for window, sink in ((0, 0), (-1, 4), (4, -1)):
        with pytest.raises(fa.FedAttnError):
            fa.fedattn_local_window(ctx, shape, x, x, x, [0, 8], window, sink, x.clone())
        with pytest.raises(fa.FedAttnError):
            fa.fedattn_decode_window(ctx, shape, fa.DECODE_LOCAL, one, x, x, 0, length, 8, window, sink, one.clone())
    with pytest.raises(ValueError):
        fa.fedattn_decode_window(ctx, shape, fa.DECODE_LOCAL, one, x, x[:7], 0, length, 8, 4, 0, one.clone())
    with pytest.raises(ValueError):
        fa.fedattn_local_window(ctx, shape, x, x, x, [0, 7], 4, 0, x.clone())
    with pytest.raises(ValueError):
        fa.fedattn_local_window(ctx, shape, x.float(), x, x, [0, 8], 4, 0, x.clone())
    assert ctx.launch_count() == 0
