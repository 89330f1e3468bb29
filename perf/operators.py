"""Timed cases of the operators that stand around the attention in a decoder layer, and their plain forms.

A case is one call.  Its field `op` says which:
    norm     residual sum and root-mean-square norm of `rows` rows of `n`, to 8 bits with a scale per 128 columns
             (out8) or to the rows' own type
    gate     silu(gate) * up of `rows` rows of `n` to 8 bits with scales; gated = False: the rows themselves
    matmul   C[rows, n] = A[rows, k] B[n, k]^T, both in 8-bit floats with scales of blocks of 128, C in `dtype`
    rotary   the q, k and v heads of a product [batch, length, (heads + 2 kv_heads) * d] go to the layouts that the
             attention takes, q and k rotated by their positions; inverse = True: rotated back
    sample   a token of each row of logits [rows, n]; filters: which of temperature, top-k, top-p, min-p are in use

Scales are powers of two, held as their exponent plus 127 in a byte.  8-bit rows start at multiples of 16 bytes
and their scales at multiples of 4, as in a user's buffers.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BLOCK = 128
_EPS = 1e-5
_BASE = 10000.0
_SCRATCH = 32 << 20  # bytes of scratch memory that a program keeps for all its products


def _norm(rows, n, dtype="bf16", residual=True, out8=True, name=None):
    return _named(dict(op="norm", rows=rows, n=n, dtype=dtype, residual=residual, out8=out8), name)


def _gate(rows, n, dtype="bf16", gated=True, name=None):
    return _named(dict(op="gate", rows=rows, n=n, dtype=dtype, gated=gated), name)


def _matmul(rows, n, k, dtype="bf16", name=None):
    return _named(dict(op="matmul", rows=rows, n=n, k=k, dtype=dtype), name)


def _rotary(batch, length, heads, kv_heads, d, rot, interleaved=False, inverse=False, dtype="bf16", name=None):
    return _named(dict(op="rotary", batch=batch, length=length, heads=heads, kv_heads=kv_heads, d=d, rot=rot,
                       interleaved=interleaved, inverse=inverse, dtype=dtype), name)


def _sample(rows, n, dtype="f32", filters="tkpm", name=None):
    return _named(dict(op="sample", rows=rows, n=n, dtype=dtype, filters=filters), name)


def _named(case, name):
    return dict(case, name=name) if name else case


def listed():
    return [
        # a token of one sequence in a 7B layer (32 heads x 128): the smallest call, where latency counts
        _norm(1, 4096, name="norm_token"),
        # eight prompts of 2048 tokens in a 13B layer (40 heads x 128)
        _norm(16384, 5120, name="norm_prompt"),
        # a step of 24 sequences: the middle of the MLP
        _gate(24, 11008, name="gate_batch"),
        # prompts of no round length together, the same
        _gate(7001, 11008, name="gate_prompt"),
        # a token through the QKV product of a 7B layer: its weights have to be read
        _matmul(1, 12288, 4096, name="matmul_token"),
        # a step of 48 sequences through the MLP's last product
        _matmul(48, 4096, 11008, name="matmul_batch"),
        # a chunk of 333 tokens to the logits of an odd vocabulary
        _matmul(333, 32003, 4096, dtype="f32", name="matmul_logits"),
        # four prompts of 2048 tokens through the MLP's first two products
        _matmul(8192, 22016, 4096, name="matmul_prompt"),
        # a step of 16 sequences with grouped heads
        _rotary(16, 1, 32, 8, 128, 128, name="rotary_step"),
        # eight prompts, 32 heads, pairs of neighbours
        _rotary(8, 2048, 32, 32, 128, 128, interleaved=True, name="rotary_prompt"),
        # a chat loop's token: every filter in use
        _sample(1, 32000, name="sample_token"),
        # many sequences' tokens from the larger vocabulary of a 13B shape, top-p and min-p
        _sample(256, 50272, dtype="bf16", filters="tpm", name="sample_batch"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """A width between the two: a multiple of 64 more often than not."""
    n = _log_int(rng, lo, hi)
    n = max(lo, n // 64 * 64) if rng.random() < 0.7 else n
    return n if n != 48 * 64 else n + 64


def draw(rng):
    """One more case: rows 1 to 16384 of widths 64 to 16384, products of 1 to 8192 rows up to 7.4e11 multiplications, 1 to
    96 heads of 64 or 128 (whole or in part rotated) over 1 to 8192 tokens, vocabularies of 100 to 150000."""
    op = rng.choice(["norm", "gate", "matmul", "matmul", "rotary", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("norm", "gate"):
        n = _width(rng, 64, 16384)
        rows = _log_int(rng, 1, min(16384, (40_000_000 if dtype == "f32" else 70_000_000) // n))
        if op == "gate":
            return _gate(rows, n, dtype, gated=rng.random() < 0.6)
        return _norm(rows, n, dtype, residual=rng.random() < 0.7, out8=rng.random() < 0.7)
    if op == "matmul":
        k, n = _width(rng, 64, 16384), _width(rng, 64, 32768)
        return _matmul(_log_int(rng, 1, min(8192, int(7.3e11 / n / k), 180_000_000 // n)), n, k, dtype)
    if op == "rotary":
        d = rng.choice([64, 128])
        kv = rng.choice([1, 4, 8, rng.randint(1, 32)])
        heads = min(96, kv * rng.choice([1, 1, 4, rng.randint(1, 8)]))
        heads -= heads % kv
        if (heads + 2 * kv) * d == 48 * 64 or heads * d == 48 * 64:
            heads += kv
        tokens = _log_int(rng, 1, min(8192, 150_000_000 // (d * (heads + 2 * kv)) // (2 if dtype == "f32" else 1)))
        batch = rng.choice([1, min(4, tokens), tokens])
        rot = d if rng.random() < 0.6 else 2 * rng.randint(1, d // 2)
        return _rotary(batch, max(1, tokens // batch), heads, kv, d, rot, rng.random() < 0.5, rng.random() < 0.3, dtype)
    n = _log_int(rng, 100, 150000)
    filters = "".join(c for c in "tkpm" if rng.random() < 0.6)
    return _sample(_log_int(rng, 1, min(512, 12_000_000 // n)), n, dtype, filters)


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _up(x, m):
    return -(-x // m) * m


def _normal(shape, gen, dtype=torch.float32):
    return torch.randn(shape, dtype=dtype, generator=gen, device="cuda")


def _activations(rows, n, gen, dtype):
    """Rows as a trained model's: a few channels stand out by a factor of ten to thirty, rows differ in size."""
    x = _normal((rows, n), gen, dtype)
    loud = torch.rand(n, generator=gen, device="cuda") < 0.004
    x *= torch.where(loud, 20.0, 1.0).to(dtype) * (0.3 + torch.rand(n, generator=gen, device="cuda")).to(dtype)
    x *= torch.exp(0.3 * _normal((rows, 1), gen)).to(dtype)
    return x


def _eight_bit_buffers(rows, n):
    """What a user keeps for 8-bit rows: the values, and a byte of scale per 128 columns."""
    return (torch.zeros(rows, _up(n, 16), dtype=torch.float8_e4m3fn, device="cuda")[:, :n],
            torch.zeros(rows, _up(-(-n // _BLOCK), 4), dtype=torch.uint8, device="cuda")[:, : -(-n // _BLOCK)])


def _scale_bytes(top):
    """The smallest b >= 0 with top <= 448 * 2^(b - 127), from the bits of the blocks' largest values."""
    bits = top.view(torch.int32)
    return ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(0, 254)


def _blocks(y):
    rows, n = y.shape
    return torch.nn.functional.pad(y, (0, _up(n, _BLOCK) - n)).view(rows, -1, _BLOCK)


def _to_eight_bits(y):
    """fp32 rows to 8-bit floats and the bytes of their scales."""
    rows, n = y.shape
    blocks = _blocks(y)
    byte = _scale_bytes(blocks.abs().amax(2))
    q = blocks * torch.exp2(127.0 - byte.float())[:, :, None]
    return q.view(rows, -1)[:, :n].to(torch.float8_e4m3fn), byte.to(torch.uint8)


def _weights(n, k, gen):
    """Weights in 8 bits with a scale for each 128 x 128."""
    w = _normal((n, k), gen, torch.bfloat16).float() * 0.02
    tiles = torch.nn.functional.pad(w, (0, _up(k, _BLOCK) - k, 0, _up(n, _BLOCK) - n))
    tiles = tiles.view(-(-n // _BLOCK), _BLOCK, -(-k // _BLOCK), _BLOCK)
    byte = _scale_bytes(tiles.abs().amax(3).amax(1))
    q = (tiles * torch.exp2(127.0 - byte.float())[:, None, :, None]).view(_up(n, _BLOCK), -1)[:n, :k]
    b, scales = _eight_bit_buffers(n, k)
    scales = scales[: -(-n // _BLOCK)]
    b.copy_(q.to(torch.float8_e4m3fn))
    scales.copy_(byte.to(torch.uint8))
    return b, scales


def _cos_sin(rows, rot):
    """[rows, rot]: the cosines of a position's rot / 2 angles, then their sines."""
    f = _BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "norm":
        rows, n = case["rows"], case["n"]
        s.update(x=_activations(rows, n, gen, dt), weight=(1.0 + 0.1 * _normal((n,), gen)).to(dt))
        if case["residual"]:
            s.update(residual=_activations(rows, n, gen, dt), total=torch.empty(rows, n, dtype=dt, device="cuda"))
        if case["out8"]:
            s["q"], s["scales"] = _eight_bit_buffers(rows, n)
        else:
            s["out"] = torch.empty(rows, n, dtype=dt, device="cuda")
    elif case["op"] == "gate":
        rows, n = case["rows"], case["n"]
        x = _activations(rows, 2 * n if case["gated"] else n, gen, dt)  # gate and up: one product's two halves
        s.update(x=x[:, -n:], gate=x[:, :n] if case["gated"] else None)
        s["q"], s["scales"] = _eight_bit_buffers(rows, n)
    elif case["op"] == "matmul":
        rows, n, k = case["rows"], case["n"], case["k"]
        a, a_scales = _eight_bit_buffers(rows, k)
        q, byte = _to_eight_bits(_activations(rows, k, gen, torch.bfloat16).float())
        a.copy_(q)
        a_scales.copy_(byte)
        b, b_scales = _weights(n, k, gen)
        s.update(a=a, a_scales=a_scales, b=b, b_scales=b_scales, c=torch.empty(rows, n, dtype=dt, device="cuda"))
        s["workspace"] = torch.empty(_SCRATCH, dtype=torch.uint8, device="cuda")
    elif case["op"] == "rotary":
        batch, length, heads, kv, d = case["batch"], case["length"], case["heads"], case["kv_heads"], case["d"]
        x = _normal((batch, length, (heads + 2 * kv) * d), gen, dt)
        first = torch.randint(0, 30000, (batch, 1), generator=gen, device="cuda")
        pos = (first + torch.arange(length, device="cuda")).int()
        s.update(x=x, pos=pos, table=_cos_sin(30000 + length, case["rot"]))
        s["o"] = [torch.empty(batch, h, length, d, dtype=dt, device="cuda") for h in (heads, kv, kv)]
    else:
        rows, n = case["rows"], case["n"]
        x = 2.0 * _normal((rows, n), gen)
        few = torch.rand(rows, n, generator=gen, device="cuda") < 30.0 / n  # a row's likely tokens
        x += few * (6.0 + 3.0 * torch.rand(rows, n, generator=gen, device="cuda"))
        s["logits"] = x.to(dt)
        s["noise"] = torch.empty(rows, n, device="cuda").exponential_(generator=gen)
        row = lambda lo, hi: lo + (hi - lo) * torch.rand(rows, generator=gen, device="cuda")  # noqa: E731
        s["temperature"] = row(0.5, 1.2) if "t" in case["filters"] else None
        s["top_k"] = row(20, 200).int() if "k" in case["filters"] else None
        s["top_p"] = row(0.7, 0.99) if "p" in case["filters"] else None
        s["min_p"] = row(0.001, 0.1) if "m" in case["filters"] else None
        s["token"] = torch.empty(rows, dtype=torch.int32, device="cuda")
        s["prob"] = torch.empty(rows, device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------

def _values(scales):
    """The bytes of scales as the numbers they stand for."""
    return scales.view(torch.float8_e8m0fnu)


def _heads_of(s):
    """The q, k and v heads of the product as [batch, length, heads, d]."""
    c, x = s["case"], s["x"]
    x = x.view(c["batch"], c["length"], -1, c["d"])
    return x.split([c["heads"], c["kv_heads"], c["kv_heads"]], 2)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2407_20485_amd import binding as B
    c = s["case"]
    if c["op"] == "norm":
        total, out, q, scales = s.get("total"), s.get("out"), s.get("q"), s.get("scales")
        B.a2sf_rms_norm(s["x"], s["weight"], _EPS, residual=s.get("residual"), total=total, out=out, q=q, scales=scales)
        return {"total": total, "out": out, "q": q, "scales": _values(scales) if q is not None else None}
    if c["op"] == "gate":
        B.a2sf_quantize(s["x"], s["q"], s["scales"], gate=s["gate"])
        return {"q": s["q"], "scales": _values(s["scales"])}
    if c["op"] == "matmul":
        B.a2sf_matmul_scaled(s["a"], s["a_scales"], s["b"], s["b_scales"], s["c"], workspace=s["workspace"])
        return s["c"]
    if c["op"] == "rotary":
        q, k, v = _heads_of(s)
        oq, ok, ov = (o.transpose(1, 2) for o in s["o"])
        B.a2sf_rotary([(q, oq), (k, ok), (v, ov, False)], s["pos"], s["table"], interleaved=c["interleaved"],
                      inverse=c["inverse"])
        return s["o"]
    B.a2sf_sample(s["logits"], s["noise"], s["token"], temperature=s["temperature"], top_k=s["top_k"],
                  top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"])
    return {"token": s["token"], "prob": s["prob"]}


def _turn(x, cos, sin, rot, interleaved):
    """The first `rot` elements of the heads [batch, length, heads, d] rotated, pair by pair."""
    y = x.float().clone()
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    else:
        a, b = y[..., : rot // 2], y[..., rot // 2: rot]
    a1, b1 = a * cos - b * sin, b * cos + a * sin
    a.copy_(a1)
    b.copy_(b1)
    return y


def _run_plain(s):
    c = s["case"]
    dt = _DTYPES[c["dtype"]]
    if c["op"] == "norm":
        h = s["x"].float()
        if c["residual"]:
            h = h + s["residual"].float()
        y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + _EPS) * s["weight"].float()
        got = {"total": h.to(dt) if c["residual"] else None, "out": None, "q": None, "scales": None}
        if c["out8"]:
            got["q"], byte = _to_eight_bits(y)
            got["scales"] = _values(byte)
        else:
            got["out"] = y.to(dt)
        return got
    if c["op"] == "gate":
        y = s["x"].float()
        if c["gated"]:
            g = s["gate"].float()
            y = g / (1.0 + torch.exp(-g)) * y
        q, byte = _to_eight_bits(y)
        return {"q": q, "scales": _values(byte)}
    if c["op"] == "matmul":
        rows, n, k = c["rows"], c["n"], c["k"]
        a = s["a"].float() * _values(s["a_scales"]).float().repeat_interleave(_BLOCK, 1)[:, :k]
        w = _values(s["b_scales"]).float().repeat_interleave(_BLOCK, 0)[:n].repeat_interleave(_BLOCK, 1)[:, :k]
        return torch.matmul(a, (s["b"].float() * w).t()).to(dt)
    if c["op"] == "rotary":
        q, k, v = _heads_of(s)
        cs = s["table"][s["pos"].long()][:, :, None]
        cos, sin = cs[..., : c["rot"] // 2], cs[..., c["rot"] // 2:]
        if c["inverse"]:
            sin = -sin
        q, k = (_turn(x, cos, sin, c["rot"], c["interleaved"]) for x in (q, k))
        return [x.transpose(1, 2).to(dt).contiguous() for x in (q, k, v)]
    logits = s["logits"].float()
    sorted_, order = torch.sort(logits, dim=1, descending=True, stable=True)
    t = s["temperature"][:, None] if s["temperature"] is not None else 1.0
    y = (sorted_ - sorted_[:, :1]) / t
    w = torch.exp(y)
    kept = torch.ones_like(w, dtype=torch.bool)
    if s["top_k"] is not None:
        kept &= torch.arange(c["n"], device="cuda") < s["top_k"][:, None]
    if s["top_p"] is not None:
        inside = torch.where(kept, w, 0.0)
        kept &= torch.cumsum(inside, 1) - inside < s["top_p"][:, None] * inside.sum(1, keepdim=True)
    if s["min_p"] is not None:
        kept &= w >= s["min_p"][:, None]
    key = torch.where(kept, y - torch.log(s["noise"].gather(1, order)), -math.inf)
    at = key.argmax(1, keepdim=True)
    z = torch.where(kept, w, 0.0).sum(1, keepdim=True)
    return {"token": order.gather(1, at)[:, 0].int(), "prob": (w.gather(1, at) / z)[:, 0]}


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] in ("norm", "gate"):
        size, scales = c["rows"] * c["n"], c["rows"] * -(-c["n"] // _BLOCK)
        if c["op"] == "gate":  # x (and the gate) in, 8 bits and scales out
            return {"bytes": size * (e * (2 if c["gated"] else 1) + 1) + scales, "flops": size * (6 if c["gated"] else 2)}
        # x and the residual in, their sum and the normed rows out, the weight once
        out = size + scales if c["out8"] else size * e
        return {"bytes": size * e * (3 if c["residual"] else 1) + out + c["n"] * e, "flops": 6 * size}
    if c["op"] == "matmul":
        m, n, k = c["rows"], c["n"], c["k"]
        kb = -(-k // _BLOCK)
        return {"bytes": m * k + n * k + m * kb + -(-n // _BLOCK) * kb + m * n * e, "flops": 2.0 * m * n * k}
    if c["op"] == "rotary":
        tokens = c["batch"] * c["length"]
        size = tokens * (c["heads"] + 2 * c["kv_heads"]) * c["d"]
        return {"bytes": 2 * size * e + tokens * 4 + c["length"] * c["rot"] * 4,
                "flops": tokens * (c["heads"] + c["kv_heads"]) * c["rot"] * 3}
    # the logits; without a filter that ends the tail every token takes part with its random number
    every = not set(c["filters"]) & set("kpm")
    return {"bytes": c["rows"] * c["n"] * (e + (4 if every else 0)) + c["rows"] * 24, "flops": 3.0 * c["rows"] * c["n"]}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------

def _eight_bits_exact(y):
    """Values of the 8-bit rows and of their scales: 448 * scale reaches the block's largest value."""
    rows, n = y.shape
    blocks = _blocks(y)
    top = blocks.abs().amax(2)
    e = torch.where(top > 0, torch.ceil(torch.log2(top / 448.0) - 1e-13), -127.0).clamp(min=-127.0)
    scale = torch.pow(2.0, e)
    v = blocks / scale[:, :, None]
    # three bits behind the leading one; below 2^-6 steps of 2^-9
    step = torch.pow(2.0, torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(v / step) * step).view(rows, -1)[:, :n], scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm":
        h = s["x"].double() + (s["residual"].double() if c["residual"] else 0.0)
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / c["n"] + _EPS) * s["weight"].double()
        q, scales = _eight_bits_exact(y) if c["out8"] else (None, None)
        return {"total": h if c["residual"] else None, "out": None if c["out8"] else y, "q": q, "scales": scales}
    if c["op"] == "gate":
        y = s["x"].double()
        if c["gated"]:
            y = y * s["gate"].double() * torch.sigmoid(s["gate"].double())
        q, scales = _eight_bits_exact(y)
        return {"q": q, "scales": scales}
    if c["op"] == "matmul":
        m, n, k = c["rows"], c["n"], c["k"]
        sa, sb = (torch.pow(2.0, s[x].double() - 127.0) for x in ("a_scales", "b_scales"))
        at = torch.arange(k, device="cuda") // _BLOCK
        a = s["a"].double() * sa[:, at]
        got = torch.empty(m, n, dtype=torch.float64, device="cuda")
        for n0 in range(0, n, 8192):  # weights in parts: 64 bits of all would be eight times their size
            rows = torch.arange(n0, min(n, n0 + 8192), device="cuda")
            got[:, n0: n0 + len(rows)] = a @ (s["b"][n0: n0 + len(rows)].double() * sb[rows // _BLOCK][:, at]).t()
        return got
    if c["op"] == "rotary":
        got = []
        half = torch.arange(c["rot"] // 2, device="cuda")
        first, second = (2 * half, 2 * half + 1) if c["interleaved"] else (half, half + c["rot"] // 2)
        table = s["table"].double()[s["pos"].long()]
        angle = torch.complex(table[..., : c["rot"] // 2], table[..., c["rot"] // 2:])[:, :, None]
        for x, turned in zip(_heads_of(s), (True, True, False)):
            y = x.double().clone()
            if turned:
                z = torch.complex(y[..., first], y[..., second]) * (angle.conj() if c["inverse"] else angle)
                y[..., first], y[..., second] = z.real, z.imag
            got.append(y.transpose(1, 2))
        return got
    l = s["logits"].double()
    if s["temperature"] is not None:
        l = l / s["temperature"].double()[:, None]
    # a token's rank is how many stand before it: larger ones, and equal ones of a lower index
    order = torch.argsort(l, dim=1, descending=True, stable=True)
    p = torch.softmax(l, 1).gather(1, order)
    rank = torch.arange(c["n"], device="cuda")[None, :]
    last = torch.full((c["rows"], 1), c["n"], device="cuda")
    if s["top_k"] is not None:
        last = torch.minimum(last, s["top_k"].long()[:, None])
    p = torch.where(rank < last, p, 0.0)
    if s["top_p"] is not None:
        before = torch.cumsum(p, 1) - p
        last = torch.minimum(last, (before < s["top_p"].double()[:, None] * p.sum(1, keepdim=True)).sum(1, keepdim=True))
    if s["min_p"] is not None:
        last = torch.minimum(last, (p >= s["min_p"].double()[:, None] * p[:, :1]).sum(1, keepdim=True))
    p = torch.where(rank < last, p, 0.0)
    p = p / p.sum(1, keepdim=True)
    at = (p / s["noise"].double().gather(1, order)).argmax(1, keepdim=True)
    return {"token": order.gather(1, at)[:, 0].int(), "prob": p.gather(1, at)[:, 0]}
