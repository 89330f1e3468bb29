"""The small decoder over pages: append, attention and log probabilities together, against the plain float64 model."""
import math

import pytest
import torch

from paper_2407_20485_amd import decoder as D
from test_gpu_decoder import SMALL, plain

pytestmark = pytest.mark.gpu


def texts(config, lengths, seed=1):
    gen = torch.Generator("cuda").manual_seed(seed)
    return [torch.randint(0, config.vocabulary, (n,), device="cuda", generator=gen) for n in lengths]


@pytest.mark.parametrize("config", SMALL)
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("page", [8, 16, 64])
def test_logits_of_prompts_chunks_and_steps(config, eight, page):
    """Prompts of different lengths, a chunk behind one while others go on or wait, single tokens: the plain model's logits.  The same bound as
    over the dense caches: activations in 8 bits; keys and values in 8 bits are off by as much as one such activation more."""
    model = D.Decoder(config, positions=64)
    t = texts(config, (40, 33, 51))
    model.start_paged(3, 60, page, eight=eight)
    at = [20, 33 - 7, 30]
    got = [(model.feed([x[:n] for x, n in zip(t, at)]).clone(), list(at))]
    for counts in ((9, 1, 0), (1, 1, 1), (1, 1, 1), (9, 0, 16), (0, 4, 1)):
        got.append((model.feed([x[a: a + n] for x, a, n in zip(t, at, counts)]).clone(), [a + n if n else 0 for a, n in zip(at, counts)]))
        at = [a + n for a, n in zip(at, counts)]
    for i, x in enumerate(t):
        want = plain(model, x[None])[0]
        for logits, last in got:
            if last[i] == 0:
                continue
            w = want[last[i] - 1]
            assert float((logits[i].double() - w).norm() / w.norm()) < 0.1
            assert float(torch.nn.functional.cosine_similarity(logits[i].double(), w, dim=0)) > 0.99


def test_generation_over_pages_repeats_and_forward_takes_a_batch():
    config = SMALL[0]
    model = D.Decoder(config, positions=256)
    prompt = torch.stack(texts(config, (100,) * 4, 2))
    runs = []
    for _ in range(2):
        model.start_paged(4, 140, 16, window=64, sinks=4)
        runs.append(model.generate(prompt, 30, seed=5))
        assert model.lengths == [129] * 4
    assert torch.equal(*runs) and int(runs[0].min()) >= 0 and int(runs[0].max()) < 1003
    model.start(4, 0.5, 10, 10)                      # and back to a budget
    assert model.generate(prompt, 4, seed=5).shape == (4, 4)


def test_scores_are_the_log_probabilities_of_the_logits():
    config = SMALL[1]
    model = D.Decoder(config, positions=64)
    t = texts(config, (17, 2, 40), 3)
    model.start_paged(3, 40, 16)
    logits = model.feed(t, every=True).double().clone()
    model.start_paged(3, 40, 16)
    scores = model.score(t, alternatives=5)
    at = 0
    for x, (logp, entropy, top, ids) in zip(t, scores):
        n = len(x) - 1
        want = torch.log_softmax(logits[at: at + n], 1)
        # within 2 roundings of a logit of at most 64, and those of a sum of 777 terms
        slack = 4e-5
        assert logp.shape == (n,) and bool(((logp.double() - want.gather(1, x[1:, None])[:, 0]).abs() <= slack).all())
        assert bool(((entropy.double() + (want.exp() * want).sum(1)).abs() <= slack * 10).all())
        order = torch.argsort(logits[at: at + n], dim=1, descending=True, stable=True)[:, :5]
        assert torch.equal(ids.long(), order) and bool(((top.double() - want.gather(1, order)).abs() <= slack).all())
        at += n + 1
    assert all(math.isfinite(float(s[0].sum())) for s in scores)


def test_what_does_not_fit_is_refused():
    model = D.Decoder(SMALL[1], positions=64)
    t = texts(SMALL[1], (10, 10))
    model.start_paged(2, 16, 8)
    with pytest.raises(ValueError):
        model.feed(t[:1])
    with pytest.raises(ValueError):
        model.feed([x[:0] for x in t])
    first = model.feed(t).clone()
    with pytest.raises(ValueError):
        model.feed([t[0][:7], t[1][:1]])
    with pytest.raises(ValueError):
        model.score(t)
    assert model.lengths == [10, 10]
    model.start_paged(2, 16, 8)
    assert torch.equal(model.feed(t), first)
