"""Timed cases of keys and values in pages (new ones go in, attention reads them) and of log probabilities, and their plain forms.

A case is one call.  Its field `op` says which:
    append    the q, k and v heads of a product's rows [tokens, (heads + 2 kv_heads) * d]: q and k rotated by their positions, q to
              rows of its own, k and v to their sequences' pages, in the rows' type or in 8 bits with a scale per token and head
    attend    attention of each sequence's new tokens over its pages: a token sees those up to itself, with a window only the newest
              `window` of them and the first `sinks`
    logprobs  of each row of logits [rows, n] the log probabilities of `given` tokens, the entropy and the `top` likeliest tokens

`sequences` sequences have up to `past` cached tokens and up to `new` new ones (mixed: the first has so many, the others one each).
Pages hold `page` tokens of all K/V heads.  They lie in no order; those that no new token sees are handed back (-1).
Scales are powers of two, held as their exponent plus 127 in a byte.
"""
import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BASE = 10000.0
_SCRATCH = 64 << 20  # bytes of scratch memory that a program keeps for its attention calls


def _append(sequences, past, new, heads, kv_heads, d, page, rot, interleaved=False, dtype="bf16", eight=False, salt=0, name=None):
    return _named(dict(op="append", sequences=sequences, past=past, new=new, mixed=False, heads=heads, kv_heads=kv_heads, d=d, page=page,
                       rot=rot, interleaved=interleaved, dtype=dtype, eight=eight, window=0, sinks=0, salt=salt), name)


def _attend(sequences, past, new, heads, kv_heads, d, page, window=0, sinks=0, mixed=False, dtype="bf16", eight=False, salt=0, name=None):
    return _named(dict(op="attend", sequences=sequences, past=past, new=new, mixed=mixed, heads=heads, kv_heads=kv_heads, d=d, page=page,
                       window=window, sinks=sinks, dtype=dtype, eight=eight, salt=salt), name)


def _logprobs(rows, n, dtype="f32", given=1, top=5, name=None):
    return _named(dict(op="logprobs", rows=rows, n=n, dtype=dtype, given=given, top=top), name)


def _named(case, name):
    return dict(case, name=name) if name else case


def listed():
    return [
        # a step of 16 sequences with grouped heads: the smallest call, where latency counts
        _append(16, 500, 1, 32, 8, 128, 16, 128, name="append_step"),
        # four prompts of up to 2048 tokens, pairs of neighbours
        _append(4, 0, 2048, 32, 32, 128, 64, 128, interleaved=True, name="append_prompts"),
        # prompts behind a common system prompt go into pages of 8 bits
        _append(24, 200, 400, 32, 8, 128, 32, 128, eight=True, name="append_8bit"),
        # a chat loop's token: one sequence of 4096
        _attend(1, 4095, 1, 32, 8, 128, 16, name="attend_token"),
        # a batch in the middle of its answers, pages of 8 bits
        _attend(48, 8191, 1, 32, 8, 128, 64, eight=True, name="attend_batch"),
        # long documents
        _attend(4, 65535, 1, 32, 8, 128, 256, name="attend_long"),
        # a large batch of streams under a window with a few first tokens
        _attend(200, 15000, 1, 40, 40, 128, 16, window=1000, sinks=4, name="attend_streams"),
        # a step of a serving loop: a chunk of a long prompt together with the tokens of others
        _attend(16, 4096, 512, 32, 8, 128, 32, mixed=True, name="attend_mixed"),
        # prompts of up to 2048 tokens together
        _attend(4, 0, 2048, 32, 32, 128, 64, name="attend_prompts"),
        # one long prompt under a window with a few first tokens
        _attend(1, 0, 16384, 32, 8, 128, 64, window=2048, sinks=4, name="attend_window"),
        # a token's likelihood and its alternatives, as a chat interface shows them
        _logprobs(1, 32000, name="logprobs_token"),
        # an evaluation: the tokens of a text of 2000, from a larger vocabulary
        _logprobs(2000, 50272, dtype="bf16", top=20, name="logprobs_text"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case: 1 to 256 sequences of up to 16 K/V heads' 65000 tokens (2.6e8 elements of K at most), 1 to 40 heads of 64 or 128
    in groups of 1 to 16, pages of 1 to 256 tokens, windows from one token on, prompts of up to 2.5e11 multiplications, vocabularies of
    50 to 150000."""
    op = rng.choice(["append", "step", "step", "ragged", "ragged", "logprobs"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "logprobs":
        n = _log_int(rng, 50, 150000)
        return _logprobs(_log_int(rng, 1, min(2000, (50_000_000 if dtype == "f32" else 100_000_000) // n)), n, dtype,
                         given=rng.choice([1, 1, rng.randint(2, 5)]), top=rng.choice([0, 1, rng.randint(2, 32)]))
    d = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 8, rng.randint(1, 16)])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 7, 8, 12, 16) if g * kv <= 40])
    page = 2 ** rng.choice([0, 3, 4, 4, 5, 6, 7, 8])
    salt, eight = rng.randint(1, 10 ** 6), rng.random() < 0.35
    if op == "append":
        sequences = _log_int(rng, 1, 256)
        rot = d if rng.random() < 0.6 else 2 * rng.randint(1, d // 2)
        tokens = min(8192, 90_000_000 // (d * (heads + 2 * kv)) // (2 if dtype == "f32" else 1))
        new = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, tokens // sequences))
        return _append(sequences, _log_int(rng, 1, 512), new, heads, kv, d, page, rot, rng.random() < 0.5, dtype, eight, salt)
    window, sinks = (0, 0) if rng.random() < 0.5 else (_log_int(rng, 1, 4096), rng.choice([0, 1, 4, rng.randint(0, 100)]))
    if op == "step":
        sequences = _log_int(rng, 1, 256)
        tokens = min(65000, 260_000_000 // (kv * d) // sequences // (2 if dtype == "f32" else 1))
        return _attend(sequences, _log_int(rng, 1, tokens), 1, heads, kv, d, page, window, sinks, False, dtype, eight, salt)
    sequences, past = _log_int(rng, 1, 32), rng.choice([0, _log_int(rng, 1, 8192)])
    past = min(past, 200_000_000 // (kv * d) // sequences)
    # all new tokens of all sequences against half of themselves and all of what is cached; fp32 at a tenth
    products = (2.5e11 if dtype == "bf16" else 2.5e10) / (2 * d * heads * sequences)
    new = max(1, int(math.sqrt(past * past + 2 * products)) - past)
    return _attend(sequences, past, _log_int(rng, 1, min(16384, new)), heads, kv, d, page, window, sinks, rng.random() < 0.3, dtype, eight,
                   salt)


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _lengths(c):
    """(cached tokens, new tokens) of each sequence: the first has the most."""
    rng = random.Random(c["salt"])
    got = []
    for i in range(c["sequences"]):
        past = c["past"] if i == 0 else rng.randint(c["past"] // 4, c["past"])
        new = c["new"] if i == 0 else 1 if c["mixed"] else rng.randint(max(1, c["new"] // 4), c["new"])
        got.append((past, new))
    return got


def _normal(shape, gen, dtype=torch.float32):
    return torch.randn(shape, dtype=dtype, generator=gen, device="cuda")


def _scale_bytes(top):
    """The smallest b >= 0 with top <= 448 * 2^(b - 127), from the bits of the rows' largest values."""
    bits = top.view(torch.int32)
    return ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(0, 254)


def _to_eight_bits(y):
    """fp32 rows to 8-bit floats and the bytes of their scales, one a row."""
    byte = _scale_bytes(y.abs().amax(-1))
    return (y * torch.exp2(127.0 - byte.float())[..., None]).to(torch.float8_e4m3fn), byte.to(torch.uint8)


def _cos_sin(rows, rot):
    """[rows, rot]: the cosines of a position's rot / 2 angles, then their sines."""
    f = _BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _unseen(c, past, page):
    """A page of a sequence that none of its new tokens sees."""
    if not c["window"]:
        return False
    first, last = page * c["page"], (page + 1) * c["page"] - 1
    return first >= c["sinks"] and last <= past - c["window"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    c, dt = case, _DTYPES[case["dtype"]]
    s = {"case": c}
    if c["op"] == "logprobs":
        rows, n = c["rows"], c["n"]
        x = 2.0 * _normal((rows, n), gen, dt)
        few = torch.rand(rows, n, generator=gen, device="cuda") < 30.0 / n  # a row's likely tokens
        x += (few * (6.0 + 3.0 * torch.rand(rows, n, generator=gen, device="cuda"))).to(dt)
        s["logits"] = x
        s["tokens"] = torch.randint(0, n, (rows, c["given"]), generator=gen, device="cuda").int()
        s["tokens"][:, 0] = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.7, x.argmax(1).int(), s["tokens"][:, 0])
        s["logp"] = torch.empty(rows, c["given"], device="cuda")
        s["entropy"] = torch.empty(rows, device="cuda")
        k = min(c["top"], n)
        s["top"] = torch.empty(rows, k, device="cuda") if k else None
        s["top_tokens"] = torch.empty(rows, k, dtype=torch.int32, device="cuda") if k else None
        return s
    heads, kv, d, page = c["heads"], c["kv_heads"], c["d"], c["page"]
    lengths = _lengths(c)
    width = max(-(-(past + new) // page) for past, new in lengths)
    seen = [[p < -(-(past + new) // page) and not _unseen(c, past, p) for p in range(width)] for past, new in lengths]
    used = sum(map(sum, seen))
    pages = used + used // 16 + 1
    # the order of pages: a permutation, the same for all seeds of a case
    order = list(range(pages))
    random.Random(c["salt"] + 1).shuffle(order)
    order = iter(order)
    table = torch.tensor([[next(order) if x else -1 for x in row] for row in seen], dtype=torch.int32)
    starts = [0]
    for _, new in lengths:
        starts.append(starts[-1] + new)
    s["tokens"] = starts[-1]
    s["table"] = table.cuda()
    s["len"] = torch.tensor([past + new for past, new in lengths], dtype=torch.int32).cuda()
    s["starts"] = torch.tensor(starts, dtype=torch.int32).cuda() if c["new"] > 1 else None
    s["lengths"] = lengths
    shape = (pages, kv, page, d)
    if c["op"] == "append":
        s["x"] = _normal((s["tokens"], (heads + 2 * kv) * d), gen, dt)
        s["rotary"] = _cos_sin(c["past"] + c["new"], c["rot"])
        for x in "kv":
            s[x] = torch.zeros(shape, dtype=torch.float8_e4m3fn if c["eight"] else dt, device="cuda")
            s[x + "_scales"] = torch.zeros(shape[:3], dtype=torch.uint8, device="cuda") if c["eight"] else None
        s["q_out"] = torch.empty(s["tokens"], heads, d, dtype=dt, device="cuda")
        return s
    # queries lean towards the keys' common direction; some channels of the keys stand out, as a trained model's do
    lean = _normal((kv, 1, d), gen)
    loud = 1.0 + 2.0 * (torch.rand(d, generator=gen, device="cuda") < 0.03)
    for x in "kv":
        y = _normal(shape, gen, torch.bfloat16 if c["eight"] else dt)
        if x == "k":
            y += (0.5 * lean).to(y.dtype)
            y *= loud.to(y.dtype)
        s[x], s[x + "_scales"] = y, None
        if c["eight"]:
            q = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
            byte = torch.empty(shape[:3], dtype=torch.uint8, device="cuda")
            for i in range(0, pages, max(1, 2 ** 26 // (kv * page * d))):
                at = slice(i, i + max(1, 2 ** 26 // (kv * page * d)))
                q[at], byte[at] = _to_eight_bits(y[at].float())
            s[x], s[x + "_scales"] = q, byte
    s["q"] = (_normal((s["tokens"], heads, d), gen) + 0.3 * lean[:, 0].repeat_interleave(heads // kv, 0)).to(dt)
    s["o"] = torch.empty_like(s["q"])
    s["workspace"] = torch.empty(_SCRATCH, dtype=torch.uint8, device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------

def _values(scales):
    """The bytes of scales as the numbers they stand for."""
    return scales.view(torch.float8_e8m0fnu) if scales is not None else None


def _heads_of(s):
    """The q, k and v heads of the product as [tokens, heads, d]."""
    c = s["case"]
    return s["x"].view(s["tokens"], -1, c["d"]).split([c["heads"], c["kv_heads"], c["kv_heads"]], 1)


def _appended(s, q):
    return {"q": q, "k": s["k"], "v": s["v"], "k_scales": _values(s["k_scales"]), "v_scales": _values(s["v_scales"])}


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2407_20485_amd import binding as B
    c = s["case"]
    if c["op"] == "logprobs":
        B.a2sf_log_probs(s["logits"], s["tokens"], s["logp"], entropy=s["entropy"], top=s["top"], top_tokens=s["top_tokens"])
        return {"logp": s["logp"], "entropy": s["entropy"], "top": s["top"], "top_tokens": s["top_tokens"]}
    if "pages" not in s:  # the handle that a program keeps with its cache
        s["pages"] = B.Pages.of(s["k"], s["v"], s["k_scales"], s["v_scales"])
    if c["op"] == "append":
        q, k, v = _heads_of(s)
        B.a2sf_paged_append(q, k, v, s["pages"], s["table"], s["len"], starts=s["starts"], q_out=s["q_out"], rotary=s["rotary"],
                            interleaved=c["interleaved"])
        return _appended(s, s["q_out"])
    B.a2sf_paged_attention(s["q"], s["pages"], s["table"], s["len"], s["o"], starts=s["starts"], window=c["window"] or None,
                           sinks=c["sinks"], workspace=s["workspace"])
    return s["o"]


def _turn(x, cos, sin, rot, interleaved):
    """The first `rot` elements of the heads [tokens, heads, d] rotated, pair by pair."""
    y = x.float().clone()
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    else:
        a, b = y[..., : rot // 2], y[..., rot // 2: rot]
    a1, b1 = a * cos - b * sin, b * cos + a * sin
    a.copy_(a1)
    b.copy_(b1)
    return y


def _places(s):
    """Of each new token: its position, its page and its place there."""
    c = s["case"]
    starts = s["starts"] if s["starts"] is not None else torch.arange(c["sequences"] + 1, device="cuda")
    new = (starts[1:] - starts[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(c["sequences"], device="cuda"), new, output_size=s["tokens"])
    pos = torch.arange(s["tokens"], device="cuda") - starts.long()[seq] + (s["len"].long() - new)[seq]
    return pos, s["table"][seq, pos // c["page"]].long(), pos % c["page"]


def _run_plain(s):
    c = s["case"]
    dt = _DTYPES[c["dtype"]]
    if c["op"] == "logprobs":
        x = s["logits"].float()
        top = x.amax(1, keepdim=True)
        y = x - top
        w = torch.exp(y)
        z = w.sum(1, keepdim=True)
        lse = torch.log(z)
        got = {"logp": y.gather(1, s["tokens"].long()) - lse, "entropy": (lse - (w * y).sum(1, keepdim=True) / z)[:, 0],
               "top": None, "top_tokens": None}
        if s["top"] is not None:
            value, order = torch.sort(y, dim=1, descending=True, stable=True)
            k = s["top"].shape[1]
            got.update(top=value[:, :k] - lse, top_tokens=order[:, :k].int())
        return got
    if c["op"] == "append":
        q, k, v = _heads_of(s)
        pos, page, place = _places(s)
        cs = s["rotary"][pos][:, None]
        cos, sin = cs[..., : c["rot"] // 2], cs[..., c["rot"] // 2:]
        q, k = (_turn(x, cos, sin, c["rot"], c["interleaved"]) for x in (q, k))
        for name, x in (("k", k), ("v", v.float())):
            if c["eight"]:
                x, byte = _to_eight_bits(x)
                s[name].view(torch.uint8)[page, :, place] = x.view(torch.uint8)
                s[name + "_scales"][page, :, place] = byte
            else:
                s[name][page, :, place] = x.to(dt)
        return _appended(s, q.to(dt))
    group, o, at = c["heads"] // c["kv_heads"], s["o"], 0
    for i, (past, new) in enumerate(s["lengths"]):
        # the tokens that some new one sees
        first = max(0, past - c["window"] + 1) if c["window"] else 0
        j = torch.cat([torch.arange(0, min(first, c["sinks"]), device="cuda"), torch.arange(first, past + new, device="cuda")])
        page, place = s["table"][i, j // c["page"]].long(), j % c["page"]
        k, v = (_plain_rows(s, x, page, place) for x in "kv")  # [kv_heads, tokens, d]
        for r0 in range(0, new, 512):
            rows = min(512, new - r0)
            q = s["q"][at + r0: at + r0 + rows].float().view(rows, c["kv_heads"], group, c["d"])
            q = q.permute(1, 2, 0, 3).reshape(c["kv_heads"], group * rows, c["d"])
            upto = len(j) - new + r0 + rows
            x = torch.matmul(q, k[:, :upto].transpose(1, 2).contiguous()) / math.sqrt(c["d"])
            pos = past + torch.arange(r0, r0 + rows, device="cuda").repeat(group)[:, None]
            away = pos - j[:upto]
            hidden = away < 0
            if c["window"]:
                hidden |= (away >= c["window"]) & (j[:upto] >= c["sinks"])
            x = torch.where(hidden, -math.inf, x)
            w = torch.exp(x - x.amax(2, keepdim=True))
            y = torch.matmul(w, v[:, :upto]) / w.sum(2, keepdim=True)
            y = y.view(c["kv_heads"], group, rows, c["d"]).permute(2, 0, 1, 3).reshape(rows, c["heads"], c["d"])
            o[at + r0: at + r0 + rows] = y.to(dt)
        at += new
    return o


def _plain_rows(s, x, page, place):
    y = s[x][page, :, place].float()
    if s[x + "_scales"] is not None:
        y = y * _values(s[x + "_scales"][page, :, place]).float()[..., None]
    return y.transpose(0, 1).contiguous()


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "logprobs":
        out = 8 * c["given"] + 4 + 8 * min(c["top"], c["n"])  # given tokens in, their values, the entropy and alternatives out
        return {"bytes": c["rows"] * (c["n"] * e + out), "flops": 5.0 * c["rows"] * c["n"]}
    lengths, d, kv, heads = _lengths(c), c["d"], c["kv_heads"], c["heads"]
    tokens = sum(new for _, new in lengths)
    row = d + 1 if c["eight"] else d * e  # of a page: 8 bits and a scale
    if c["op"] == "append":
        return {"bytes": tokens * ((2 * heads + 2 * kv) * d * e + 2 * kv * row + 4) + min(tokens, c["past"] + c["new"]) * c["rot"] * 4,
                "flops": 3.0 * tokens * (heads + kv) * c["rot"]}
    seen = pairs = 0
    for past, new in lengths:
        if not c["window"]:
            seen += past + new
            pairs += new * past + new * (new + 1) // 2
            continue
        first = max(0, past - c["window"] + 1)
        seen += past + new - first + min(first, c["sinks"])
        for p in range(past, past + new):
            oldest = max(0, p - c["window"] + 1)
            pairs += p - oldest + 1 + min(oldest, c["sinks"])
    return {"bytes": 2 * seen * kv * row + 2 * tokens * heads * d * e, "flops": 4.0 * d * heads * pairs}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------

def _eight_bits_exact(y):
    """Values of the 8-bit rows and of their scales: 448 * scale reaches the row's largest value."""
    top = y.abs().amax(-1)
    e = torch.where(top > 0, torch.ceil(torch.log2(top / 448.0) - 1e-13), -127.0).clamp(min=-127.0)
    scale = torch.pow(2.0, e)
    v = y / scale[..., None]
    # three bits behind the leading one; below 2^-6 steps of 2^-9
    step = torch.pow(2.0, torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(v / step) * step, scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "logprobs":
        got = {"logp": [], "entropy": [], "top": [], "top_tokens": []}
        k = min(c["top"], c["n"])
        for r0 in range(0, c["rows"], 256):
            x = s["logits"][r0: r0 + 256].double()
            logp = torch.log_softmax(x, 1)
            p = torch.exp(logp)
            got["logp"].append(logp.gather(1, s["tokens"][r0: r0 + 256].long()))
            got["entropy"].append(-(p * logp).sum(1))
            order = torch.argsort(x, dim=1, descending=True, stable=True)[:, :k]
            got["top"].append(logp.gather(1, order))
            got["top_tokens"].append(order.int())
        return {x: torch.cat(y) if k or not x.startswith("top") else None for x, y in got.items()}
    if c["op"] == "append":
        half = torch.arange(c["rot"] // 2, device="cuda")
        first, second = (2 * half, 2 * half + 1) if c["interleaved"] else (half, half + c["rot"] // 2)
        got = {x: torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in "kv"}
        scales = {x + "_scales": torch.full(s[x].shape[:3], 2.0 ** -127, dtype=torch.float64, device="cuda") if c["eight"] else None
                  for x in "kv"}
        pos, page, place = [], [], []
        table = s["table"].tolist()
        for i, (past, new) in enumerate(s["lengths"]):
            for p in range(past, past + new):
                pos.append(p)
                page.append(table[i][p // c["page"]])
                place.append(p % c["page"])
        pos, page, place = (torch.tensor(x, device="cuda") for x in (pos, page, place))
        turn = s["rotary"].double()[pos]
        angle = torch.complex(turn[:, : c["rot"] // 2], turn[:, c["rot"] // 2:])[:, None]
        for name, x in zip("qkv", _heads_of(s)):
            y = x.double().clone()
            if name != "v":
                z = torch.complex(y[..., first], y[..., second]) * angle
                y[..., first], y[..., second] = z.real, z.imag
            if name == "q":
                got["q"] = y
                continue
            if c["eight"]:
                y, scale = _eight_bits_exact(y)
                scales[name + "_scales"][page, :, place] = scale
            got[name][page, :, place] = y
        return {"q": got["q"], "k": got["k"], "v": got["v"], **scales}
    group, o, at = c["heads"] // c["kv_heads"], [], 0
    for i, (past, new) in enumerate(s["lengths"]):
        n = past + new
        page = s["table"][i, : -(-n // c["page"])].long().clamp(min=0)
        out = torch.empty(new, c["heads"], c["d"], dtype=torch.float64, device="cuda")
        for h in range(c["kv_heads"]):
            k, v = (_exact_rows(s, x, page, h)[:n] for x in "kv")
            for r0 in range(0, new, 1024):
                r1 = min(new, r0 + 1024)
                upto = past + r1
                p = torch.arange(past + r0, past + r1, device="cuda")[:, None]
                j = torch.arange(upto, device="cuda")[None, :]
                seen = j <= p
                if c["window"]:
                    seen &= (j > p - c["window"]) | (j < c["sinks"])
                for g in range(h * group, (h + 1) * group):
                    x = s["q"][at + r0: at + r1, g].double() @ k[:upto].t() / math.sqrt(c["d"])
                    out[r0:r1, g] = torch.softmax(x.masked_fill(~seen, -math.inf), 1) @ v[:upto]
        o.append(out)
        at += new
    return torch.cat(o)


def _exact_rows(s, x, page, h):
    y = s[x][page, h].double()
    if s[x + "_scales"] is not None:
        y = y * torch.pow(2.0, s[x + "_scales"][page, h].double() - 127.0)[..., None]
    return y.reshape(-1, y.shape[-1])
