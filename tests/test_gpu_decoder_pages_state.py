"""The small decoder over pages: what it refuses, what it keeps when a call fails, and logits under a window."""
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
