"""The small decoder over pages: what it refuses and what it keeps when a call fails."""
import pytest
import torch

from paper_2407_20485_amd import decoder as D
from test_gpu_decoder import SMALL
from test_gpu_decoder_pages import texts

pytestmark = pytest.mark.gpu


def test_more_tokens_than_positions_are_refused():
    """Behind the rotary table there is no rotation for a token: the pages would hold NaN."""
    model = D.Decoder(SMALL[1], positions=64)
    with pytest.raises(ValueError):
        model.start_paged(2, 65, 16)
    t = texts(SMALL[1], (64, 3))
    model.start_paged(2, 64, 16)
    assert bool(torch.isfinite(model.feed(t, every=True)).all())
    with pytest.raises(ValueError):
        model.feed([t[0][:1], t[1][:1]])


def test_a_call_that_fails_adds_no_tokens():
    """Tokens in memory of the host: the same call with them on the GPU gives what it would have given at first."""
    model = D.Decoder(SMALL[1], positions=64)
    t = texts(SMALL[1], (10, 7))
    model.start_paged(2, 40, 8)
    want = model.feed(t).clone()
    again = model.feed([x[:3] for x in t]).clone()
    model.start_paged(2, 40, 8)
    with pytest.raises(Exception):
        model.feed([x.cpu() for x in t])
    assert model.lengths == [0, 0]
    assert torch.equal(model.feed(t), want)
    with pytest.raises(Exception):
        model.feed([x[:3].float() for x in t])
    assert model.lengths == [10, 7]
    assert torch.equal(model.feed([x[:3] for x in t]), again)
