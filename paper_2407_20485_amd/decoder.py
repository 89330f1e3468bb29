"""A small decoder whose layers run on the library alone: norm, 8-bit products, rotary positions, the A2SF attention with its
evicting cache, or attention over pages that keep every token or a window of them, the gated MLP, and sampling, on random weights.

    python -m paper_2407_20485_amd.decoder [--layers 4] [--heads 32] [--kv-heads 8] [--batch 4] [--prompt 512] [--steps 64]
                                           [--paged [--page 64] [--window N] [--sinks 4] [--cache8]]

A layer's step is ten calls: norm -> QKV product -> rotary -> attention -> 8 bits -> product -> norm -> gate and up product -> gate ->
product (over pages: append, which rotates, in the place of rotary).  torch holds the memory, looks up the embedding's rows and draws the
random numbers; this file only sequences the calls.
"""
from __future__ import annotations

import argparse
import dataclasses
import time

import torch

from . import binding as B


@dataclasses.dataclass
class Config:
    layers: int = 4
    heads: int = 32
    kv_heads: int = 8
    d: int = 128
    inner: int = 11008       # columns of the gate and of the up projection
    vocabulary: int = 32000
    rotary_dims: int = 128
    base: float = 10000.0
    eps: float = 1e-5

    @property
    def width(self):
        return self.heads * self.d


def eight_bit(rows, n, scale_rows=None, device="cuda"):
    """Memory for 8-bit rows and their scales.  Rows start at multiples of 16 bytes and are no longer than that asks for (64 bytes more
    where they are whole kilobytes, weights from memory: 1 row x 12288 x 4096 11.2 us, with them 11.5; 48 x 4096 x 11008 17.8, 22.5)."""
    nb = -(-n // 128)
    return (torch.zeros(rows, -(-n // 16) * 16, dtype=torch.float8_e4m3fn, device=device)[:, :n],
            torch.zeros(scale_rows or rows, -(-nb // 4) * 4, dtype=torch.uint8, device=device)[:, :nb])


class Linear:
    """Weights [n, k] in 8 bits."""

    def __init__(self, w):
        self.q, self.scales = eight_bit(*w.shape, scale_rows=-(-w.shape[0] // 128))
        B.a2sf_quantize_weight(w, self.q, self.scales)

    def __call__(self, rows8, c, workspace):
        B.a2sf_matmul_scaled(*rows8, self.q, self.scales, c, workspace=workspace)
        return c


class Decoder:
    """Weights and, per batch of sequences of one length, the caches and the memory of a pass."""

    def __init__(self, config: Config, seed=0, positions=32768):
        c, self.config = config, config
        gen = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *shape, s: (s * torch.randn(*shape, generator=gen, device="cuda")).bfloat16()  # noqa: E731
        self.embedding = draw(c.vocabulary, c.width, s=1.0)
        self.layers = []
        for _ in range(c.layers):
            self.layers.append({
                "norm1": 1 + draw(c.width, s=0.1), "norm2": 1 + draw(c.width, s=0.1),
                "qkv": Linear(draw((c.heads + 2 * c.kv_heads) * c.d, c.width, s=c.width ** -0.5)),
                "out": Linear(draw(c.width, c.width, s=c.width ** -0.5)),
                "gate_up": Linear(draw(2 * c.inner, c.width, s=c.width ** -0.5)),
                "down": Linear(draw(c.width, c.inner, s=c.inner ** -0.5))})
        self.norm = 1 + draw(c.width, s=0.1)
        self.pages = None
        self.head = Linear(draw(c.vocabulary, c.width, s=c.width ** -0.5))
        self.table = torch.empty(positions, c.rotary_dims, device="cuda")
        B.a2sf_rotary_table(self.table, base=c.base)

    def start(self, batch, alpha, select, recent, spare=0):
        """Empty caches for `batch` sequences under a budget of select + recent tokens a head."""
        c = self.config
        self.batch, self.alpha, self.budget = batch, alpha, (select, recent)
        self.caches = [B.Cache(batch * c.kv_heads, select + recent + 1 + spare, c.d, torch.bfloat16) for _ in self.layers]
        self.position = 0
        self._rows = self.pages = None

    def start_paged(self, sequences, capacity, page_size=64, window=None, sinks=0, eight=False):
        """Empty pages for `sequences` sequences of up to `capacity` tokens each, which nothing is evicted from; a window: a token sees the
        newest `window` ones and the first `sinks`.  eight: keys and values in 8 bits."""
        if capacity > self.table.shape[0]:
            raise ValueError(f"sequences of {capacity} tokens: the decoder was made for {self.table.shape[0]} positions")
        c, per = self.config, -(-capacity // page_size)
        kind = torch.float8_e4m3fn if eight else torch.bfloat16
        self.pages = [B.Pages(sequences * per, page_size, c.kv_heads, c.d, kind) for _ in self.layers]
        # a page of each sequence in turn, as a server would hand them out
        self.page_table = torch.arange(sequences * per, dtype=torch.int32, device="cuda").view(per, sequences).t().contiguous()
        self.window, self.sinks, self.capacity = window, sinks, capacity
        self.lengths = [0] * sequences
        self._rows = None

    def _memory(self, rows, n):
        """The buffers of a pass over `rows` rows (n per sequence), kept until a pass of another size."""
        if self._rows == (rows, n):
            return self._m
        c, new = self.config, lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        b = rows // n
        heads = c.heads + 2 * c.kv_heads
        products = ((heads * c.d, c.width), (c.width, c.width), (2 * c.inner, c.width), (c.width, c.inner))
        scratch = [B.a2sf_matmul_workspace_bytes(rows, *p) for p in products]
        scratch.append(B.a2sf_matmul_workspace_bytes(b, c.vocabulary, c.width))
        cache = self.caches[0]
        scratch.append(B.a2sf_workspace_bytes(b * c.heads, n, cache.capacity, c.d, B.A2SF_BF16, *self.budget))
        m = dict(stream=new(rows, c.width), delta=new(rows, c.width), x8=eight_bit(rows, c.width), inner8=eight_bit(rows, c.inner),
                 qkv=new(rows, heads * c.d), gate_up=new(rows, 2 * c.inner), q=new(b, c.heads, n, c.d), k=new(b, c.kv_heads, n, c.d),
                 v=new(b, c.kv_heads, n, c.d), o=new(b, c.heads, n, c.d), rows=new(rows, c.width), last8=eight_bit(b, c.width),
                 logits=new(b, c.vocabulary, t=torch.float32), workspace=new(max(scratch) + 16, t=torch.uint8),
                 pos=new(b, n, t=torch.int32))
        self._rows, self._m = (rows, n), m
        return m

    def forward(self, tokens):
        """tokens [batch, n] behind what the caches hold (n > 1 only as the prompt): logits [batch, vocabulary] of the last one."""
        c = self.config
        if self.pages is not None:
            return self.feed(list(tokens))
        b, n = tokens.shape
        if n > 1 and self.position > 0:
            raise ValueError(f"{n} tokens behind {self.position} that are cached: a prompt goes into empty caches (start), then one token a call")
        m = self._memory(b * n, n)
        group = c.heads // c.kv_heads
        m["pos"].copy_(torch.arange(self.position, self.position + n, dtype=torch.int32, device="cuda").expand(b, n))
        ws = m["workspace"]
        torch.index_select(self.embedding, 0, tokens.reshape(-1), out=m["stream"])

        def attend(i):
            parts = m["qkv"].view(b, n, -1, c.d).split([c.heads, c.kv_heads, c.kv_heads], 2)
            B.a2sf_rotary([(parts[0], m["q"].transpose(1, 2)), (parts[1], m["k"].transpose(1, 2)),
                           (parts[2], m["v"].transpose(1, 2), False)], m["pos"], self.table)
            self._attend(m, self.caches[i], n, group, ws)
            if n > 1:  # back to a token's heads side by side: a part that is not rotated is copied through its strides
                B.a2sf_rotary([(m["o"].transpose(1, 2), m["rows"].view(b, n, c.heads, c.d), False)], m["pos"], self.table)
            return m["rows"] if n > 1 else m["o"].view(b, c.width)

        self._layers(m, attend)
        # the last token of each sequence: every n-th row
        last = slice(n - 1, None, n)
        B.a2sf_rms_norm(m["delta"][last], self.norm, c.eps, residual=m["stream"][last], q=m["last8"][0], scales=m["last8"][1])
        self.position += n
        return self.head(m["last8"], m["logits"], ws)

    def _layers(self, m, attend):
        """All layers on the rows of m["stream"]; attend(layer): the rows of its attention.  The last layer's product is left in m["delta"]."""
        c, delta, ws = self.config, m["delta"], m["workspace"]
        for i, layer in enumerate(self.layers):
            self._norm(layer["norm1"], delta if i else None, m)
            layer["qkv"](m["x8"], m["qkv"], ws)
            B.a2sf_quantize(attend(i), *m["x8"])
            layer["out"](m["x8"], delta, ws)
            self._norm(layer["norm2"], delta, m)
            layer["gate_up"](m["x8"], m["gate_up"], ws)
            B.a2sf_quantize(m["gate_up"][:, c.inner:], *m["inner8"], gate=m["gate_up"][:, :c.inner])
            layer["down"](m["inner8"], delta, ws)

    def feed(self, texts, every=False):
        """Over pages: each sequence's next tokens, a 1-D tensor each (any number of them, an empty one for a sequence that waits), behind what
        it has; logits [sequences, vocabulary] of their last ones (of a sequence that waits: of no meaning), or with every = True [tokens,
        vocabulary] of all."""
        c, counts = self.config, [len(t) for t in texts]
        if len(texts) != len(self.lengths):
            raise ValueError(f"{len(texts)} texts for {len(self.lengths)} sequences")
        if any(have + n > self.capacity for have, n in zip(self.lengths, counts)):
            raise ValueError(f"sequences of {self.lengths} tokens have no room for {counts} more: pages for {self.capacity} each")
        rows, b = sum(counts), len(texts)
        if rows == 0:
            raise ValueError("no tokens")
        single = all(n == 1 for n in counts)
        m = self._memory_paged(rows, rows if every else b)
        starts = [0]
        for n in counts:
            starts.append(starts[-1] + n)
        lengths = [have + n for have, n in zip(self.lengths, counts)]
        lens = torch.tensor(lengths, dtype=torch.int32).cuda()
        at = None if single else torch.tensor(starts, dtype=torch.int32).cuda()
        torch.index_select(self.embedding, 0, torch.cat(texts), out=m["stream"])

        def attend(i):
            q, k, v = m["qkv"].view(rows, -1, c.d).split([c.heads, c.kv_heads, c.kv_heads], 1)
            B.a2sf_paged_append(q, k, v, self.pages[i], self.page_table, lens, starts=at, q_out=m["q"], rotary=self.table)
            B.a2sf_paged_attention(m["q"], self.pages[i], self.page_table, lens, m["rows"], starts=at, window=self.window, sinks=self.sinks,
                                   workspace=m["workspace"])
            return m["rows"].view(rows, c.width)

        self._layers(m, attend)
        self.lengths = lengths  # (a call that fails before this has added no token: the next one writes the same rows)
        delta, stream = m["delta"], m["stream"]
        if not every and not single:
            last = torch.tensor([max(s - 1, 0) for s in starts[1:]]).cuda()
            delta, stream = delta[last], stream[last]
        B.a2sf_rms_norm(delta, self.norm, c.eps, residual=stream, q=m["last8"][0], scales=m["last8"][1])
        return self.head(m["last8"], m["logits"], m["workspace"])

    def _memory_paged(self, rows, outputs):
        if self._rows == (rows, outputs, "paged"):
            return self._m
        c, new = self.config, lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        heads = c.heads + 2 * c.kv_heads
        products = ((heads * c.d, c.width), (c.width, c.width), (2 * c.inner, c.width), (c.width, c.inner))
        scratch = [B.a2sf_matmul_workspace_bytes(rows, *p) for p in products]
        scratch.append(B.a2sf_matmul_workspace_bytes(outputs, c.vocabulary, c.width))
        scratch.append(B.a2sf_paged_workspace_bytes(rows, c.heads, c.kv_heads, c.d, len(self.lengths),
                                                    self.page_table.shape[1] * self.pages[0].page_size))
        self._m = dict(stream=new(rows, c.width), delta=new(rows, c.width), x8=eight_bit(rows, c.width), inner8=eight_bit(rows, c.inner),
                       qkv=new(rows, heads * c.d), gate_up=new(rows, 2 * c.inner), q=new(rows, c.heads, c.d), rows=new(rows, c.heads, c.d),
                       last8=eight_bit(outputs, c.width), logits=new(outputs, c.vocabulary, t=torch.float32),
                       workspace=new(max(scratch) + 16, t=torch.uint8))
        self._rows = (rows, outputs, "paged")
        return self._m

    def score(self, texts, alternatives=0):
        """Over empty pages: of each text (a 1-D tensor of two tokens or more) the log probabilities of its tokens behind the first, the entropy
        of the model at each, and the likeliest tokens there [n - 1, alternatives] with theirs (None without): a list of (logp, entropy, top,
        top_tokens)."""
        if any(self.lengths):
            raise ValueError("texts are scored from their beginning: start_paged first")
        counts = [len(t) for t in texts]
        logits = self.feed(texts, every=True)
        rows, f = logits.shape[0], torch.float32
        after = torch.cat([torch.cat([t[1:], t[:1]]) for t in texts]).to(torch.int32).view(rows, 1)  # (the last one's is not looked at)
        logp, entropy = (torch.empty(s, dtype=f, device="cuda") for s in ((rows, 1), (rows,)))
        top = torch.empty(rows, alternatives, dtype=f, device="cuda") if alternatives else None
        ids = torch.empty(rows, alternatives, dtype=torch.int32, device="cuda") if alternatives else None
        B.a2sf_log_probs(logits, after, logp, entropy, top, ids)
        got = zip(logp[:, 0].split(counts), entropy.split(counts), *(x.split(counts) if x is not None else [None] * len(counts) for x in (top, ids)))
        return [tuple(x[:-1] if x is not None else None for x in one) for one in got]

    def _norm(self, weight, delta, m):
        stream = m["stream"]
        q, scales = m["x8"]
        if delta is None:
            B.a2sf_rms_norm(stream, weight, self.config.eps, q=q, scales=scales)
        else:
            B.a2sf_rms_norm(delta, weight, self.config.eps, residual=stream, total=stream, q=q, scales=scales)

    def _attend(self, m, cache, n, group, ws):
        kept = self.budget
        if n > 1 or self.position == 0:
            if group > 1:
                B.a2sf_prefill_gqa(m["q"], m["k"], m["v"], n, group, self.alpha, *kept, cache, o=m["o"], workspace=ws)
            else:
                B.a2sf_prefill(m["q"], m["k"], m["v"], n, self.alpha, *kept, cache, o=m["o"], workspace=ws)
        elif group > 1:
            B.a2sf_decode_step_gqa(m["q"], m["k"], m["v"], self.position, cache, group, self.alpha, *kept, m["o"], workspace=ws)
        else:
            B.a2sf_decode_step(m["q"], m["k"], m["v"], self.position, cache, self.alpha, *kept, m["o"], workspace=ws)

    def generate(self, prompt, steps, temperature=0.8, top_k=50, top_p=0.95, min_p=0.0, seed=0):
        """`steps` tokens behind the prompts [batch, n]: [batch, steps] int32.  A sequence with an infinity or a NaN in its activations has
        no token to take: -1 from there on."""
        b = prompt.shape[0]
        gen = torch.Generator(device="cuda").manual_seed(seed)
        row = lambda v, t: torch.full((b,), v, dtype=t, device="cuda")  # noqa: E731
        filters = dict(temperature=row(temperature, torch.float32), top_k=row(top_k, torch.int32), top_p=row(top_p, torch.float32),
                       min_p=row(min_p, torch.float32))
        noise = torch.empty(b, self.config.vocabulary, device="cuda")
        out = torch.empty(steps, b, dtype=torch.int32, device="cuda")
        tokens = prompt
        for i in range(steps):
            logits = self.forward(tokens)
            B.a2sf_sample(logits, noise.exponential_(generator=gen), out[i], **filters)
            tokens = out[i].view(b, 1).clamp_min(0)
        return out.t()


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("layers", 4), ("heads", 32), ("kv-heads", 8), ("batch", 4), ("prompt", 512), ("steps", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--ratio", type=float, default=0.2, help="cache ratio: the budget's share of the prompt, half of it recent tokens")
    ap.add_argument("--alpha", type=float, default=0.5)
    ap.add_argument("--paged", action="store_true", help="keep every token, in pages, in the place of a budget")
    for name, value in (("page", 64), ("window", None), ("sinks", 0)):
        ap.add_argument("--" + name, type=int, default=value, help="with --paged")
    ap.add_argument("--cache8", action="store_true", help="with --paged: keys and values in 8 bits")
    a = ap.parse_args()
    model = Decoder(Config(layers=a.layers, heads=a.heads, kv_heads=a.kv_heads), positions=a.prompt + a.steps + 1)
    budget = max(2, int(a.ratio * a.prompt))
    prompt = torch.randint(0, model.config.vocabulary, (a.batch, a.prompt), device="cuda")
    for _ in range(2):  # the second time is the one that counts
        if a.paged:
            model.start_paged(a.batch, a.prompt + a.steps + 1, a.page, a.window, a.sinks, a.cache8)
        else:
            model.start(a.batch, a.alpha, budget // 2, budget - budget // 2)
        torch.cuda.synchronize()
        t0 = time.time()
        first = model.generate(prompt, 1, seed=1)
        torch.cuda.synchronize()
        t1 = time.time()
        rest = model.generate(first.long(), a.steps, seed=2)
        torch.cuda.synchronize()
        t2 = time.time()
    print(f"{a.layers} layers, {a.heads} heads on {a.kv_heads} K/V heads, {a.batch} sequences: prompt of {a.prompt} tokens {1e3 * (t1 - t0):.2f} ms, "
          f"then {a.steps} steps of {1e3 * (t2 - t1) / a.steps:.3f} ms with "
          + (f"every token in pages of {a.page}" if a.paged else f"{budget} cached tokens a head"))
    print("first sequence:", torch.cat([first, rest], 1)[0].tolist())


if __name__ == "__main__":
    main()
