"""Calls whose first run in a process is inside a stream capture: kernels are loaded and their attributes set then and there."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = r"""
import sys
import torch
import paper_2511_02647_b200 as fa
dtype, d = getattr(fa, sys.argv[1]), int(sys.argv[2])
dt = torch.bfloat16 if dtype == fa.BF16 else torch.float32
n, hq, hkv, cap, rows = 4, 8, 2, 512, 6000
shape = fa.Shape(n, hq, hkv, d, dtype)
ctx = fa.Context(shape, n * cap, n * cap)
g = torch.Generator(device="cuda").manual_seed(5)
rand = lambda *s: torch.empty(s, device="cuda").normal_(generator=g).to(dt)
q, kc, vc = rand(n, hq, d), rand(n, cap, hkv, d), rand(n, cap, hkv, d)
x, k, v = rand(rows, hq, d), rand(rows, hkv, d), rand(rows, hkv, d)
length = torch.tensor([cap, 7, 0, 300], dtype=torch.int32, device="cuda")
cache = fa.QuantCache(shape, n, cap)
freq = [10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
od, lse, ox, lx, ok = torch.empty_like(q), torch.empty((n, hq), device="cuda"), torch.empty_like(x), torch.empty((rows, hq), device="cuda"), torch.empty_like(k)
kb, vb = torch.empty_like(k[:n * cap]), torch.empty_like(k[:n * cap])
L = fa.DECODE_LOCAL
# (what has been there longer runs before: the windows have kernels of their own)
fa.fedattn_decode(ctx, shape, L, q, kc, vc, cap * hkv * d, length, cap, od, lse)
fa.fedattn_local(ctx, shape, x, k, v, [0, 100, 100, 2500, rows], ox, lx)
for out, call in [
    ((od, lse), lambda: fa.fedattn_decode_window(ctx, shape, L, q, kc, vc, cap * hkv * d, length, cap, 100, 3, od, lse)),
    ((ox, lx), lambda: fa.fedattn_local_window(ctx, shape, x, k, v, [0, 100, 100, 2500, rows], 100, 3, ox, lx)),
    ((ox, ok), lambda: fa.fedattn_qk_norm_rope(ctx, shape, x, k, None, None, 1e-6, None, freq, False, ox, ok)),
    (cache.arrays(), lambda: fa.fedattn_quantize_kv(ctx, shape, k[:n * cap], v[:n * cap], None, cache)),
    ((kb, vb), lambda: fa.fedattn_dequantize_kv(ctx, shape, cache, None, kb, vb)),
    ((od, lse), lambda: fa.fedattn_decode_quant(ctx, shape, L, q, cache, length, cap, od, lse)),
]:
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t in out:
        t.fill_(99)
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in out]
    for t in out:
        t.fill_(77)
    call()
    assert ctx.poll() == 0
    assert all(torch.equal(a, b) for a, b in zip(got, out)) and all((a != 99).any() for a in got)
print("same")
"""


@pytest.mark.parametrize("dtype,d", [("BF16", 64), ("BF16", 128), ("F32", 96)])
def test_first_calls_are_captured(dtype, d):
    r = subprocess.run([sys.executable, "-c", CODE, dtype, str(d)], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr
