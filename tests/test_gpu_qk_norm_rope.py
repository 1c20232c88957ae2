"""fedattn_qk_norm_rope against the formula in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2511_02647_b200 as fa
import reference64 as ref
from helpers import dev, host

pytestmark = pytest.mark.gpu


def freqs(rot, base=10000.0):
    return [base ** (-2.0 * i / rot) for i in range(rot // 2)]


def close(got, want, size, dtype, what=""):
    """fp32: sum of squares, root, quotient, weight, sine and cosine (1 ulp each, off by half an ulp of an eighth of a turn), two
    products and their sum: at most 24 half-ulps of |a| + |b|.  bf16: one rounding of the result."""
    tol = 24 * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d values, worst %.3e" % (what, bad.sum(), np.abs(got - want)[bad].max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (128, 128, True), (128, 64, False), (64, 64, False), (64, 16, True),
                                         (96, 96, False), (72, 72, False), (40, 24, True), (8, 8, False), (24, 0, False),
                                         (120, 8, False)])
@pytest.mark.parametrize("rows,hq,hkv", [(1, 8, 2), (37, 7, 1), (700, 6, 3)])
def test_against_the_formula(dtype, d, rot, inter, rows, hq, hkv):
    rng = np.random.default_rng([d, rot, rows, hq])
    q, k = rng.standard_normal((rows, hq, d)) * 3, rng.standard_normal((rows, hkv, d)) * 0.02
    wq, wk = 1 + 0.3 * rng.standard_normal(d), 1 + 0.3 * rng.standard_normal(d)
    pos = rng.integers(-2 ** 31, 2 ** 31, rows)
    pos[0] = 2 ** 31 - 1
    q, k, wq, wk = (ref.rounded(x, dtype) for x in (q, k, wq, wk))
    shape = fa.Shape(1, hq, hkv, d, fa.BF16 if dtype == "bf16" else fa.F32)
    ctx = fa.Context(shape, rows, rows)
    qd, kd = dev(q.astype(np.float32), dtype), dev(k.astype(np.float32), dtype)
    qo, ko = torch.full_like(qd, float("nan")), torch.full_like(kd, float("nan"))
    fa.fedattn_qk_norm_rope(ctx, shape, qd, kd, dev(wq.astype(np.float32), dtype), dev(wk.astype(np.float32), dtype), 1e-6,
                            torch.tensor(pos, dtype=torch.int32, device="cuda"), freqs(rot), inter, qo, ko)
    for got, x, w in ((qo, q, wq), (ko, k, wk)):
        want, size = ref.norm_rope(x, w, float(np.float32(1e-6)), pos, freqs(rot), inter)
        close(host(got), want, size, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_joint_projection_without_weights_and_positions(dtype):
    rows, hq, hkv, d = 300, 8, 2, 128
    rng = np.random.default_rng(5)
    x = ref.rounded(rng.standard_normal((rows, (hq + 2 * hkv) * d)), dtype)
    xd = dev(x.astype(np.float32), dtype)
    before = xd.clone()
    shape = fa.Shape(1, hq, hkv, d, fa.BF16 if dtype == "bf16" else fa.F32)
    ctx = fa.Context(shape, rows, rows)
    q, k = xd[:, :hq * d].unflatten(1, (hq, d)), xd[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
    qo, ko = torch.empty_like(q.contiguous()), torch.empty_like(k.contiguous())
    fa.fedattn_qk_norm_rope(ctx, shape, q, k, None, None, 1e-5, None, freqs(d), False, qo, ko)
    for got, a, h in ((qo, 0, hq), (ko, hq * d, hkv)):
        want, size = ref.norm_rope(x[:, a:a + h * d].reshape(rows, h, d), None, float(np.float32(1e-5)), np.arange(rows), freqs(d), False)
        close(host(got), want, size, dtype)
    assert torch.equal(xd, before)


@pytest.mark.parametrize("dtype,d,rot,inter,hq,hkv,rows", [("bf16", 128, 128, False, 4, 1, 5003), ("bf16", 64, 64, True, 3, 1, 9001),
                                                           ("bf16", 72, 40, False, 2, 2, 5001), ("f32", 96, 48, False, 4, 2, 4999),
                                                           ("f32", 64, 0, False, 2, 1, 9003), ("bf16", 128, 16, True, 32, 8, 3203),
                                                           ("bf16", 128, 128, False, 96, 16, 1300)])
def test_many_rows(dtype, d, rot, inter, hq, hkv, rows):
    """Enough rows for every warp to walk several of them; one head of zeros, rows of a joint projection, then in place."""
    rng = np.random.default_rng([d, rows])
    x = ref.rounded(rng.standard_normal((rows, (hq + hkv) * d + 8)), dtype)
    x[:, :d] = 0
    wq, wk = (ref.rounded(1 + 0.3 * rng.standard_normal(d), dtype) for _ in range(2))
    pos = rng.integers(0, 1 << 20, rows)
    xd = dev(x.astype(np.float32), dtype)
    shape = fa.Shape(1, hq, hkv, d, fa.BF16 if dtype == "bf16" else fa.F32)
    ctx = fa.Context(shape, rows, rows)
    q, k = xd[:, :hq * d].unflatten(1, (hq, d)), xd[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
    qo, ko = torch.full((rows, hq, d), float("nan"), dtype=xd.dtype, device="cuda"), torch.full((rows, hkv, d), float("nan"), dtype=xd.dtype, device="cuda")
    rest = (dev(wq.astype(np.float32), dtype), dev(wk.astype(np.float32), dtype), 1e-6, torch.tensor(pos, dtype=torch.int32, device="cuda"), freqs(rot), inter)
    fa.fedattn_qk_norm_rope(ctx, shape, q, k, *rest, qo, ko)
    for got, a, h, w in ((qo, 0, hq, wq), (ko, hq * d, hkv, wk)):
        want, size = ref.norm_rope(x[:, a:a + h * d].reshape(rows, h, d), w, float(np.float32(1e-6)), pos, freqs(rot), inter)
        close(host(got), want, size, dtype)
    q, k = q.contiguous(), k.contiguous()
    fa.fedattn_qk_norm_rope(ctx, shape, q, k, *rest, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    k.copy_(xd[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)))
    fa.fedattn_qk_norm_rope(ctx, shape, None, k, *rest, None, k)
    assert torch.equal(k, ko)


def test_in_place_alone_and_on_another_stream():
    rows, hq, hkv, d = 257, 4, 4, 64
    rng = np.random.default_rng(6)
    q = ref.rounded(rng.standard_normal((rows, hq, d)), "bf16")
    shape = fa.Shape(1, hq, hkv, d, fa.BF16)
    ctx = fa.Context(shape, rows, rows)
    want, size = ref.norm_rope(q, None, float(np.float32(1e-6)), np.arange(rows), freqs(32), True)
    side = torch.cuda.Stream()
    qd = dev(q.astype(np.float32), "bf16")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fa.fedattn_qk_norm_rope(ctx, shape, qd, None, None, None, 1e-6, None, freqs(32), True, qd, None)
    side.synchronize()
    close(host(qd), want, size, "bf16")
    kd, ko = dev(q.astype(np.float32), "bf16"), torch.empty((rows, hkv, d), dtype=torch.bfloat16, device="cuda")
    fa.fedattn_qk_norm_rope(ctx, shape, None, kd, None, None, 1e-6, None, freqs(32), True, None, ko)
    assert torch.equal(ko, qd)


def test_zero_rows_and_zero_epsilon():
    shape = fa.Shape(1, 2, 2, 128, fa.F32)
    ctx = fa.Context(shape, 4, 4)
    x = torch.zeros((4, 2, 128), device="cuda")
    out = torch.full_like(x, float("nan"))
    fa.fedattn_qk_norm_rope(ctx, shape, x, None, None, None, 1e-6, None, freqs(128), False, out, None)
    assert torch.equal(out, torch.zeros_like(out))
    x[:, :, 5] = 1e-3
    fa.fedattn_qk_norm_rope(ctx, shape, x, None, None, None, 0.0, None, [], False, out, None)
    want = torch.zeros_like(out)
    want[:, :, 5] = 128 ** 0.5
    assert torch.allclose(out, want, rtol=1e-6, atol=0)


def test_what_the_binding_refuses():
    shape = fa.Shape(1, 2, 2, 64, fa.BF16)
    ctx = fa.Context(shape, 4, 4)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    ok = (None, None, 1e-6, None, freqs(64), False)
    for q, out, rest in ((x.float(), x, ok), (x[:, :1], x, ok), (x, x[:3], ok), (x.transpose(0, 1), x, ok),
                         (x, x, (None, None, 1e-6, torch.zeros(4, dtype=torch.int64, device="cuda"), freqs(64), False)),
                         (x.cpu(), x, ok)):
        with pytest.raises(ValueError):
            fa.fedattn_qk_norm_rope(ctx, shape, q, None, *rest, out, None)
    with pytest.raises(fa.FedAttnError):
        fa.fedattn_qk_norm_rope(ctx, shape, x, None, None, None, 1e-6, None, freqs(72), False, x, None)
