"""Operators around federated attention that a served model needs beside it, as measured cases: the norm of queries and
keys with their rotation, attention through a sliding window with first tokens that stay visible (local and decode), and
the cache held in 4 bits (writing and reading rows, decode over it).

``own`` chooses what ``run`` does: the operators' plain form in elementary torch operations, or the calls that a user makes
of the package.  Sizes are those of the repository's workloads and tests, or generic.
"""
import math

import torch

own = False

LENS_8 = "1467,650,1400,1484,2698,4093,845,996"         # eight lengths uniform on [256, 4096], 13 633 tokens
LENS_6 = "300,517,64,700,129,450"                       # ragged prompts, 2 160 tokens
GROUP = 32                                              # channels that share a scale of the 4-bit cache


def listed():
    return [
        # one new token of eight participants on its way into a decode step: all latency
        dict(name="rope_8_tokens", kind="rope", rows=8, first=4096, hq=32, hkv=8, d=128, rot=128, inter=False, packed=True,
             dtype="bf16"),
        # the prompts of a whole round, read out of the projections' packed rows: bound by memory
        dict(name="rope_8xragged", kind="rope", rows=13633, first=0, hq=32, hkv=8, d=128, rot=128, inter=False, packed=True,
             dtype="bf16"),
        # a windowed block of four equal participants
        dict(name="window_4x2048", kind="local", lens="2048,2048,2048,2048", window=512, sink=4, hq=32, hkv=8, d=128,
             dtype="bf16", causal=True),
        # the same of prompts of very different length under a long window: the largest
        dict(name="window_8xragged", kind="local", lens=LENS_8, window=1024, sink=4, hq=32, hkv=8, d=128, dtype="bf16",
             causal=True),
        # 64 channels, short ragged prompts, a window that ends inside a tile, no sinks
        dict(name="window_d64_ragged", kind="local", lens=LENS_6, window=200, sink=0, hq=16, hkv=4, d=64, dtype="bf16",
             causal=True),
        # an encoder's two-sided window in fp32
        dict(name="window_f32_bidir", kind="local", lens="512,333", window=100, sink=1, hq=8, hkv=2, d=64, dtype="f32",
             causal=False),
        # one windowed block of a decode step: the caches are full, the window is what is read
        dict(name="decode_window_8x4096", kind="decode", n=8, cap=4096, low=1.0, window=1024, sink=4, hq=32, hkv=8, d=128,
             dtype="bf16"),
        # a prefill's keys and values on their way into the 4-bit caches of four participants, and read back
        dict(name="cache_4x2048", kind="cache", n=4, rows=2048, cap=4096, hkv=8, d=128, dtype="bf16"),
        # one new token of eight participants appended, and read back
        dict(name="cache_8_tokens", kind="cache", n=8, rows=1, cap=4096, hkv=8, d=128, dtype="bf16"),
        # one block of a decode step over full 4-bit caches: bound by memory
        dict(name="quant_local_8x4096", kind="quant", mode="local", n=8, cap=4096, low=1.0, window=0, sink=0, hq=32, hkv=8,
             d=128, dtype="bf16"),
        # a synchronised block: every participant's query over one shared 4-bit cache
        dict(name="quant_sync_8x4096", kind="quant", mode="sync", n=8, cap=32768, low=1.0, window=0, sink=0, hq=32, hkv=8,
             d=128, dtype="bf16"),
        # 64 channels, uneven short caches through a window: latency
        dict(name="quant_window_4x700", kind="quant", mode="local", n=4, cap=704, low=0.1, window=256, sink=4, hq=16, hkv=4,
             d=64, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "local", "local", "decode", "cache", "quant", "quant"])
    hkv, g = rng.choice([(8, 4), (8, 4), (8, 3), (8, 2), (4, 4), (2, 7), (8, 1)])
    c = dict(kind=kind, hq=hkv * g, hkv=hkv, d=rng.choice([128, 128, 128, 64, 96]), dtype="f32" if rng.random() < 0.2 else "bf16")
    small = c["dtype"] == "f32"
    if kind == "rope":
        c["rows"] = _log_int(rng, 1, 4096 if small else 12000)
        c["first"] = rng.choice([0, _log_int(rng, 1, 1 << 20)])
        c["rot"] = rng.choice([c["d"], c["d"], c["d"] // 2, 16])
        c["inter"], c["packed"] = rng.random() < 0.3, rng.random() < 0.6
        return c
    if kind == "local":
        total = _log_int(rng, 64, 1024 if small else 8192)
        n = max(rng.randint(1, 8), -(-total // 4096) * 2)
        w = [rng.uniform(0.2, 1.8) for _ in range(n)]
        even = rng.random() < 0.3
        c["lens"] = ",".join(str(max(1, total // n if even else min(4096, int(total * x / sum(w))))) for x in w)
        c["window"] = _log_int(rng, 1, 1024)
        c["sink"] = rng.choice([0, 1, 4, _log_int(rng, 1, 200)])
        c["causal"] = rng.random() < 0.75
        return c
    c["n"] = rng.randint(1, 16)
    if kind == "cache":
        c["rows"] = _log_int(rng, 1, max(1, (2048 if small else 8192) // c["n"]))
        c["cap"] = -(-(c["rows"] + rng.randint(0, 300)) // 16) * 16
        return c
    c["low"] = rng.choice([1.0, 0.7, 0.1])                          # shortest cache over the longest
    if kind == "decode":
        c["cap"] = _log_int(rng, 16, max(16, (4096 if small else 32768) // c["n"]))
        c["window"] = _log_int(rng, 1, 4096)
        c["sink"] = rng.choice([0, 1, 4, _log_int(rng, 1, 200)])
        return c
    c["mode"] = rng.choice(["local", "local", "sync"])
    most = 4096 if small else 32768
    c["cap"] = -(-_log_int(rng, 16, most if c["mode"] == "sync" else max(16, most // c["n"])) // 16) * 16
    c["window"], c["sink"] = rng.choice([(0, 0), (0, 0), (_log_int(rng, 1, 4096), rng.choice([0, 4, 37]))])
    return c


# ---- what a program has in hand ------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lens_of(case):
    return [int(x) for x in case["lens"].split(",")]


def _scale_values(device):
    """The values of the 256 scale bytes of the 4-bit cache: eight steps of every power of two, 2^-18 to 1.875 * 2^13."""
    b = torch.arange(256, device=device)
    return (1 + (b & 7).double() / 8) * torch.exp2((b >> 3).double() - 18)


def _quantised(x):
    """Plain form of the 4-bit rows: x [..., d] -> signed codes -7..7 (int64) and scale bytes [..., d / 32].  A group's scale
    is the least of the 256 whose sevenfold reaches its largest magnitude; ties of the code go to the even one."""
    xg = x.double().unflatten(-1, (x.shape[-1] // GROUP, GROUP))
    table = _scale_values(x.device)
    byte = torch.searchsorted(7 * table, xg.abs().amax(-1)).clamp(max=255)
    return torch.round(xg / table[byte].unsqueeze(-1)).clamp(-7, 7).long().flatten(-2), byte


def _values(code, byte):
    return (code.unflatten(-1, (byte.shape[-1], GROUP)) * _scale_values(code.device)[byte].unsqueeze(-1)).flatten(-2).float()


def _pack(code):
    """Codes as the cache holds them: two a byte, offset by 8, the even channel in the low half."""
    n = (code + 8).to(torch.uint8)
    return (n[..., 0::2] | (n[..., 1::2] << 4)).contiguous()


def _unpack(codes):
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long() - 8


def prepare(case, seed):
    gen, dt = torch.Generator(device="cuda").manual_seed(seed), _dtype(case)
    hq, hkv, d, kind = case["hq"] if "hq" in case else case["hkv"], case["hkv"], case["d"], case["kind"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    def channels():                                                  # some channels of keys and values are larger than others
        return torch.exp(0.5 * normal(hkv, d))

    def empty(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = dict(case=case)
    n = 1
    if kind == "rope":
        rows, rot = case["rows"], case["rot"]
        if case["packed"]:                                           # rows of the projections: queries, keys, values
            qkv = normal(rows, (hq + 2 * hkv) * d).to(dt)
            s["q"], s["k"] = qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
        else:
            s["q"], s["k"] = normal(rows, hq, d).to(dt), normal(rows, hkv, d).to(dt)
        s["wq"], s["wk"] = (1 + 0.1 * normal(d)).to(dt), (1 + 0.1 * normal(d)).to(dt)
        s["pos"] = (case["first"] + torch.arange(rows, device="cuda")).to(torch.int32)
        s["freq"] = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
        s["freq_dev"] = torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
    elif kind == "local":
        lens = _lens_of(case)
        n, L = len(lens), sum(lens)
        cu = [0]
        for x in lens:
            cu.append(cu[-1] + x)
        s["cu"] = cu
        s["q"], s["k"], s["v"] = normal(L, hq, d).to(dt), normal(L, hkv, d).to(dt), normal(L, hkv, d).to(dt)
    elif kind == "cache":
        n, rows, cap = case["n"], case["rows"], case["cap"]
        s["k"], s["v"] = (normal(n * rows, hkv, d) * channels()).to(dt), (normal(n * rows, hkv, d) * channels()).to(dt)
        # a participant's rows go behind what its cache holds already
        held = (torch.rand(n, generator=gen, device="cuda") * (cap - rows + 1)).long().clamp(max=cap - rows)
        s["at"] = (torch.arange(n, device="cuda")[:, None] * cap + held[:, None] + torch.arange(rows, device="cuda")).flatten()
        s["at"] = s["at"].to(torch.int32)
    else:
        n, cap = case["n"], case["cap"]
        caches = 1 if case.get("mode") == "sync" else n
        lens = cap * (case["low"] + (1 - case["low"]) * torch.rand(caches, generator=gen, device="cuda"))
        s["len"] = lens.round().clamp(1, cap).to(torch.int32)
        s["q"] = normal(n, hq, d).to(dt)
        if kind == "decode":
            s["k"], s["v"] = normal(n, cap, hkv, d).to(dt), normal(n, cap, hkv, d).to(dt)
        else:
            for x in ("k", "v"):
                code, byte = _quantised((normal(caches, cap, hkv, d) * channels()).to(dt).transpose(1, 2))
                s[x + "_codes"], s[x + "_scales"] = _pack(code), byte.to(torch.uint8)       # [caches, hkv, cap, ...]
    if own:
        import paper_2511_02647_b200 as fa
        shape = fa.Shape(n, hq, hkv, d, fa.BF16 if dt == torch.bfloat16 else fa.F32, causal=int(case.get("causal", True)))
        ctx = fa.Context(shape, case.get("rows", 1) if kind != "local" else s["cu"][-1], case.get("cap", 1))
        if kind == "rope":
            s["out"] = [empty(rows, hq, d), empty(rows, hkv, d)]
            s["calls"] = [fa.prepare_qk_norm_rope(ctx, shape, s["q"], s["k"], s["wq"], s["wk"], 1e-6, s["pos"], s["freq"],
                                                  case["inter"], *s["out"])]
        elif kind == "local":
            s["out"] = [empty(L, hq, d), empty(L, hq, dtype=torch.float32)]
            s["calls"] = [fa.prepare_local_window(ctx, shape, s["q"], s["k"], s["v"], s["cu"], case["window"], case["sink"],
                                                  *s["out"])]
        elif kind == "cache":
            cache = fa.QuantCache(shape, n, cap)
            s["out"] = [torch.empty_like(s["k"]), torch.empty_like(s["v"])]
            s["calls"] = [fa.prepare_quantize_kv(ctx, shape, s["k"], s["v"], s["at"], cache),
                          fa.prepare_dequantize_kv(ctx, shape, cache, s["at"], *s["out"])]
        else:
            s["out"] = [empty(n, hq, d), empty(n, hq, dtype=torch.float32)]
            if kind == "decode":
                s["calls"] = [fa.prepare_decode_window(ctx, shape, fa.DECODE_LOCAL, s["q"], s["k"], s["v"], cap * hkv * d,
                                                       s["len"], cap, case["window"], case["sink"], *s["out"])]
            else:
                cache = fa.QuantCache(shape, caches, cap, k_codes=s["k_codes"], k_scales=s["k_scales"], v_codes=s["v_codes"],
                                      v_scales=s["v_scales"])
                s["calls"] = [fa.prepare_decode_quant(ctx, shape, fa.DECODE_SYNC if case["mode"] == "sync" else fa.DECODE_LOCAL,
                                                      s["q"], cache, s["len"], cap, *s["out"], window=case["window"],
                                                      n_sink=case["sink"])]
    return s


# ---- one pass ---------------------------------------------------------------------------------------------

def _rope_plain(s, x, w):
    case, dt = s["case"], x.dtype
    rot, half = case["rot"], case["rot"] // 2
    y = x.float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w.float()
    angle = s["pos"].double()[:, None] * s["freq_dev"]
    c, n = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if case["inter"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:rot]
        turned = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(dt)


def _attend_plain(q, k, v, seen):
    """q [R, hq, d], k, v [T, hkv, d] in 32 bits, seen [R, T]: softmax over the seen keys, and its log-sum."""
    R, hq, d = q.shape
    hkv = k.shape[1]
    x = q.unflatten(1, (hkv, hq // hkv)).permute(1, 2, 0, 3).flatten(1, 2)              # [hkv, g R, d]
    t = torch.matmul(x, k.permute(1, 2, 0)).unflatten(1, (hq // hkv, R)) * d ** -0.5    # [hkv, g, R, T]
    t = t.masked_fill(~seen, -math.inf)
    m = t.amax(-1, keepdim=True)
    p = torch.exp(t - m)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(1, 2), v.transpose(0, 1)).unflatten(1, (hq // hkv, R)) / z
    return o.permute(2, 0, 1, 3).flatten(1, 2), (m + torch.log(z)).squeeze(-1).permute(2, 0, 1).flatten(1, 2)


def _local_plain(s):
    case, cu = s["case"], s["cu"]
    w, sink, dev = case["window"], case["sink"], s["q"].device
    out, lse = [], []
    for a, b in zip(cu[:-1], cu[1:]):
        k, v = s["k"][a:b].float(), s["v"][a:b].float()
        for r0 in range(0, b - a, 512):                              # the keys that some of 512 rows see
            r1 = min(r0 + 512, b - a)
            lo, hi = max(0, r0 - w + 1), r1 if case["causal"] else min(b - a, r1 + w - 1)
            j = torch.cat([torch.arange(min(sink, lo), device=dev), torch.arange(lo, hi, device=dev)])
            i = torch.arange(r0, r1, device=dev)[:, None]
            seen = (i - j < w) | (j < sink)
            seen &= (j <= i) if case["causal"] else (j - i < w) | (j < sink)
            o, x = _attend_plain(s["q"][a + r0:a + r1].float(), k[j], v[j], seen)
            out.append(o)
            lse.append(x)
    return [torch.cat(out).to(s["q"].dtype), torch.cat(lse)]


def _decode_plain(s):
    case, n = s["case"], s["q"].shape[0]
    sync = case.get("mode") == "sync"
    lens = s["len"].long()[:, None]
    j = torch.arange(case["cap"], device=s["q"].device)
    seen = j < lens
    if case["window"] > 0:
        seen = seen & ((j >= lens - case["window"]) | (j < case["sink"]))
    kv = {}
    for x in ("k", "v"):
        if case["kind"] == "quant":
            kv[x] = _values(_unpack(s[x + "_codes"]), s[x + "_scales"].long()).transpose(1, 2)
        else:
            kv[x] = s[x].float()
    if sync:
        o, lse = _attend_plain(s["q"].float(), kv["k"][0], kv["v"][0], seen)
    else:
        rows = [_attend_plain(s["q"][i:i + 1].float(), kv["k"][i], kv["v"][i], seen[i:i + 1]) for i in range(n)]
        o, lse = torch.cat([r[0] for r in rows]), torch.cat([r[1] for r in rows])
    return [o.to(s["q"].dtype), lse]


def run(s):
    if own:
        for call in s["calls"]:
            call()
        return s["out"]
    kind = s["case"]["kind"]
    if kind == "rope":
        return [_rope_plain(s, s["q"], s["wq"]), _rope_plain(s, s["k"], s["wk"])]
    if kind == "local":
        return _local_plain(s)
    if kind == "cache":
        return [_values(*_quantised(x)).to(x.dtype) for x in (s["k"], s["v"])]
    return _decode_plain(s)


# ---- what a pass cannot do without ---------------------------------------------------------------------

def _pairs(n, w, sink, causal):
    """(query, key) pairs of a segment of n rows."""
    full = sum(min(i + 1, w) for i in range(n)) if n < w else w * (w + 1) // 2 + (n - w) * w
    if not causal:
        full = 2 * full - n                                          # the window ahead, self counted once
    # sinks that the window does not reach: rows i with i - w + 1 > j for a sink j (and, two-sided, j - i >= w)
    far = sum(max(0, n - w - j) for j in range(min(sink, n)))
    if not causal:
        far += sum(max(0, j - w + 1) for j in range(min(sink, n)))
    return full + far


def work(case):
    hkv, d, kind = case["hkv"], case["d"], case["kind"]
    e = 2 if case["dtype"] == "bf16" else 4
    if kind == "rope":
        x = case["rows"] * (case["hq"] + hkv) * d
        return {"bytes": 2 * x * e + 4 * case["rows"] + 2 * d * e, "flops": 8.0 * x}
    if kind == "local":
        lens, hq = _lens_of(case), case["hq"]
        L = sum(lens)
        pairs = sum(_pairs(n, case["window"], case["sink"], case["causal"]) for n in lens)
        return {"bytes": 2 * L * hq * d * e + 2 * L * hkv * d * e + 4 * L * hq, "flops": 4.0 * d * hq * pairs}
    held = d // 2 + d // GROUP                                       # bytes of a row of one head in 4 bits
    if kind == "cache":
        rows = case["n"] * case["rows"] * hkv * 2
        return {"bytes": rows * (2 * d * e + 2 * held) + 8 * case["n"] * case["rows"], "flops": 8.0 * rows * d}
    n, hq, cap = case["n"], case["hq"], case["cap"]
    keys = cap * (1 + case["low"]) / 2
    if case["window"] > 0:
        keys = min(keys, case["window"] + case["sink"])
    caches = 1 if case.get("mode") == "sync" else n
    row = held if kind == "quant" else d * e
    return {"bytes": caches * keys * hkv * 2 * row + 2 * n * hq * d * e + 4 * n * hq, "flops": 4.0 * d * hq * n * keys}


# ---- the operators' definitions in 64 bits -----------------------------------------------------------------

def _held_exact(x):
    """The value that a 4-bit cache holds for every element: scales have four significant bits, rounded up."""
    y = x.double()
    g = y.reshape(*y.shape[:-1], -1, GROUP)
    mant, exp = torch.frexp(g.abs().amax(-1, keepdim=True) / 7)
    unit = torch.exp2(exp.double() - 4)
    scale = (torch.ceil(mant * 16) * unit).clamp(2.0 ** -18, 15 * 2.0 ** 10)
    return (scale * torch.clamp(torch.round(g / scale), -7, 7)).reshape(y.shape)


def _softmax_rows_exact(q, k, v, allowed):
    """One KV head: q [R, g, d], k, v [T, d], allowed [R, T]."""
    t = torch.einsum("rgd,td->rgt", q, k) / math.sqrt(q.shape[-1])
    t = torch.where(allowed[:, None], t, torch.full_like(t, -math.inf))
    lse = torch.logsumexp(t, -1)
    return torch.einsum("rgt,td->rgd", torch.exp(t - lse[..., None]), v), lse


def exact(case, seed):
    s = prepare(case, seed)
    kind, dev = case["kind"], "cuda"
    if kind == "rope":
        res = []
        rot = case["rot"]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=dev), s["pos"].double()[:, None] * s["freq_dev"])[:, None]
        for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
            y = x.double()
            y = w.double() * y / torch.sqrt(y.square().sum(-1, keepdim=True) / case["d"] + 1e-6)
            z = y.clone()
            i = torch.arange(rot // 2, device=dev)
            first, second = (2 * i, 2 * i + 1) if case["inter"] else (i, i + rot // 2)
            pair = torch.complex(y[..., first], y[..., second]) * turn
            z[..., first], z[..., second] = pair.real, pair.imag
            res.append(z)
        return res
    if kind == "cache":
        return [_held_exact(s["k"]), _held_exact(s["v"])]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g, w, sink = hq // hkv, case["window"], case["sink"]
    q = s["q"].double().reshape(-1, hkv, g, d)
    o = torch.empty_like(q)
    lse = torch.empty(q.shape[:3], dtype=torch.float64, device=dev)
    if kind == "local":
        for a, b in zip(s["cu"][:-1], s["cu"][1:]):
            place = torch.arange(b - a, device=dev)
            for r in range(a, b, 256):
                e = min(r + 256, b)
                dist = place[r - a:e - a, None] - place
                allowed = (dist.abs() < w) | (place < sink)
                if case["causal"]:
                    allowed &= dist >= 0
                for h in range(hkv):
                    o[r:e, h], lse[r:e, h] = _softmax_rows_exact(q[r:e, h], s["k"][a:b, h].double(), s["v"][a:b, h].double(), allowed)
    else:
        for i in range(case["n"]):
            c = 0 if case.get("mode") == "sync" else i
            m = int(s["len"][c])
            j = torch.arange(m, device=dev)
            allowed = ((j >= m - w) | (j < sink) if w > 0 else j >= 0)[None]
            for h in range(hkv):
                if kind == "decode":
                    k, v = s["k"][c, :m, h].double(), s["v"][c, :m, h].double()
                else:
                    k, v = ((_nibbles(s[x + "_codes"][c, h, :m]) - 8).double().reshape(m, -1, GROUP)
                            * _scale_exact(s[x + "_scales"][c, h, :m])[..., None] for x in ("k", "v"))
                    k, v = k.reshape(m, d), v.reshape(m, d)
                o[i:i + 1, h], lse[i:i + 1, h] = _softmax_rows_exact(q[i:i + 1, h], k, v, allowed)
    return [o.reshape(-1, hq, d), lse.reshape(-1, hq)]


def _nibbles(codes):
    wide = codes.to(torch.int16)
    return torch.cat([(wide % 16)[..., None], (wide // 16)[..., None]], -1).reshape(*codes.shape[:-1], -1)


def _scale_exact(byte):
    b = byte.to(torch.int64)
    return torch.ldexp((8 + b % 8).double(), b // 8 - 21)
