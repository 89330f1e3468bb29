"""Forms of attention over pages that are chosen by the caller or by a call's sizes: probabilities as two numbers, shares of single tokens
where there are many pieces, a workspace that is too small.  Tolerances as in test_gpu_pages.py."""
import numpy as np
import pytest
import torch

from paper_2407_20485_amd import binding as B
from test_gpu_pages import RAGGED, Batch, check_attention, strided

pytestmark = pytest.mark.gpu


def run(b, q, window=None, sinks=0, workspace=None, wide_sums=False):
    o = torch.full_like(q, 5.0)
    B.a2sf_paged_attention(q, b.cache, b.table, b.len, o, starts=b.starts, window=window, sinks=sinks, workspace=workspace,
                           wide_sums=wide_sums)
    return o


def space(b, heads, fill=0xFF):
    n = B.a2sf_paged_workspace_bytes(b.tokens, heads, b.kv, b.d, len(b.lengths), b.table.shape[1] * b.page)
    return torch.full((n,), fill, dtype=torch.uint8, device="cuda")


# ---- probabilities as two bf16 numbers ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("lengths", RAGGED)
@pytest.mark.parametrize("kv,group,d,page,window,sinks", [(2, 4, 128, 16, None, 0), (1, 1, 64, 32, None, 0), (2, 3, 64, 1, 50, 3), (1, 20, 128, 64, 7, 0)])
def test_wide_sums(eight, lengths, kv, group, d, page, window, sinks):
    """The tolerance of single tokens: 2^-17 of each probability instead of 2^-8."""
    b = Batch(50, lengths, kv, d, page, "bf16", eight).fill()
    q, _ = strided(b.tokens, kv * group, d, b.dt, np.random.default_rng([50, 1]), 2.0)
    for ws in (space(b, kv * group), None):
        check_attention(b, q, run(b, q, window, sinks, ws, wide_sums=True), window or 1 << 30, sinks)


@pytest.mark.parametrize("dtype,one_each", [("f32", False), ("f32", True), ("bf16", True)])
def test_wide_sums_where_there_is_nothing_to_choose(dtype, one_each):
    b = Batch(52, [(40, 1), (3, 1)] if one_each else [(40, 9), (0, 30)], 2, 64, 16, dtype, one_each=one_each).fill()
    q, _ = strided(b.tokens, 4, 64, b.dt, np.random.default_rng([52, 1]), 2.0)
    assert torch.equal(run(b, q), run(b, q, wide_sums=True))


def test_wide_sums_through_ctypes(monkeypatch):
    b = Batch(53, [(0, 30), (60, 50)], 2, 128, 16, "bf16").fill()
    q, _ = strided(b.tokens, 4, 128, b.dt, np.random.default_rng([53, 1]), 2.0)
    got = [run(b, q, wide_sums=True)]
    assert not torch.equal(got[0], run(b, q))
    monkeypatch.setattr(B, "_call", B._NoExtension)
    got.append(run(b, q, wide_sums=True))
    assert torch.equal(*got)
