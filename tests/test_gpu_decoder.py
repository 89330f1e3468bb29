"""The small decoder: the library's calls together, against a plain float64 model on the weights that the 8 bits stand for."""
import math

import pytest
import torch

from paper_2407_20485_amd import decoder as D

pytestmark = pytest.mark.gpu


def values(linear):
    s = torch.pow(2.0, linear.scales.double() - 127.0)
    s = s.repeat_interleave(128, 0)[: linear.q.shape[0]].repeat_interleave(128, 1)[:, : linear.q.shape[1]]
    return linear.q.double() * s


def plain(model, tokens):
    """Logits of every position: full causal attention, activations never in 8 bits."""
    c = model.config
    b, n = tokens.shape
    h = model.embedding[tokens].double()
    norm = lambda x, w: x / torch.sqrt(x.square().mean(-1, keepdim=True) + c.eps) * w.double()  # noqa: E731
    table = model.table[:n].double()
    cos, sin = table[:, None, : c.rotary_dims // 2], table[:, None, c.rotary_dims // 2:]

    def turn(x):
        r = c.rotary_dims // 2
        a, e = x[..., :r], x[..., r: 2 * r]
        return torch.cat([a * cos - e * sin, e * cos + a * sin, x[..., 2 * r:]], -1)

    hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
    for layer in model.layers:
        x = norm(h, layer["norm1"]) @ values(layer["qkv"]).t()
        q, k, v = x.view(b, n, -1, c.d).split([c.heads, c.kv_heads, c.kv_heads], 2)
        q, k = turn(q), turn(k)
        k, v = (y.repeat_interleave(c.heads // c.kv_heads, 2) for y in (k, v))
        p = torch.matmul(q.transpose(1, 2).contiguous(), k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(c.d)
        p = torch.softmax(p.masked_fill(hidden, -math.inf), -1)
        o = torch.matmul(p, v.transpose(1, 2).contiguous()).transpose(1, 2).reshape(b, n, c.width)
        h = h + o @ values(layer["out"]).t()
        g, u = (norm(h, layer["norm2"]) @ values(layer["gate_up"]).t()).split(c.inner, -1)
        h = h + (g * torch.sigmoid(g) * u) @ values(layer["down"]).t()
    return norm(h, model.norm) @ values(model.head).t()


SMALL = [D.Config(layers=2, heads=8, kv_heads=2, d=64, inner=700, vocabulary=1003, rotary_dims=64),
         D.Config(layers=1, heads=4, kv_heads=4, d=128, inner=512, vocabulary=777, rotary_dims=32)]


@pytest.mark.parametrize("config", SMALL)
def test_logits_of_prompt_and_steps(config):
    """A budget that nothing is evicted from: the same function.  An activation in 8 bits is off by 2^-5 at most half the time, 3 %
    in the mean square; four such products per layer, each diluted by the residual stream: under 10 % together."""
    model = D.Decoder(config, positions=64)
    tokens = torch.randint(0, config.vocabulary, (3, 40), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    want = plain(model, tokens)
    model.start(3, 0.5, 40, 40)
    got = [model.forward(tokens[:, :33]).clone()] + [model.forward(tokens[:, i: i + 1]).clone() for i in range(33, 40)]
    for i, g in enumerate(got):
        w = want[:, 32 + i]
        assert float((g.double() - w).norm() / w.norm()) < 0.1, i
        assert bool((torch.nn.functional.cosine_similarity(g.double(), w, dim=1) > 0.99).all())


def test_generation_under_a_budget_repeats():
    model = D.Decoder(SMALL[0], positions=256)
    prompt = torch.randint(0, 1003, (4, 100), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    runs = []
    for _ in range(2):
        model.start(4, 0.5, 10, 10)
        runs.append(model.generate(prompt, 30, seed=5))
        assert all(int(c.len.max()) == 20 for c in model.caches)
    assert torch.equal(*runs) and int(runs[0].min()) >= 0 and int(runs[0].max()) < 1003
    model.start(4, 0.5, 10, 10)
    greedy = model.generate(prompt, 4, temperature=0.0)
    model.start(4, 0.5, 10, 10)
    assert torch.equal(greedy[:, 0], model.forward(prompt).argmax(1).int())


def test_a_sequence_that_is_not_finite_gives_no_tokens_and_leaves_the_others():
    model = D.Decoder(SMALL[0], positions=128)
    prompt = torch.randint(10, 1003, (3, 50), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    model.start(3, 0.5, 10, 10)
    want = model.generate(prompt, 6, seed=4)
    model.embedding[5] = math.inf
    prompt[1, -1] = 5
    model.start(3, 0.5, 10, 10)
    got = model.generate(prompt, 6, seed=4)
    assert bool((got[1] == -1).all()) and torch.equal(got[::2], want[::2])


def test_a_prompt_goes_into_empty_caches_only():
    model = D.Decoder(SMALL[1], positions=64)
    tokens = torch.randint(0, 777, (2, 9), device="cuda")
    model.start(2, 0.5, 10, 10)
    first = model.forward(tokens).clone()
    with pytest.raises(ValueError):
        model.forward(tokens)
    assert model.position == 9
    model.start(2, 0.5, 10, 10)
    assert torch.equal(model.forward(tokens), first)
