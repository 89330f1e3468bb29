"""Forms of attention over pages that are chosen by the caller or by a call's sizes: probabilities as two numbers, shares of single tokens
where there are many pieces, a workspace that is too small; and calls as a serving loop makes them.  Tolerances as in test_gpu_pages.py."""
import numpy as np
import pytest
import torch

from paper_2407_20485_amd import binding as B
from test_gpu_pages import DT, RAGGED, Batch, check_attention, check_log_probs, strided

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


# ---- single tokens of many sequences ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("sequences,kv,group,d,dtype,eight,longest",
                         [(130, 8, 1, 128, "bf16", False, 4200), (200, 8, 1, 64, "bf16", False, 6500), (129, 8, 2, 128, "bf16", True, 4200),
                          (130, 8, 1, 128, "f32", False, 4200), (512, 2, 3, 128, "bf16", False, 4100), (140, 16, 1, 64, "f32", True, 9000)])
def test_many_pieces_of_unequal_lengths(sequences, kv, group, d, dtype, eight, longest):
    """More than 1024 and 2048 pieces (d = 64: 1536), one of them a hundred times as long as the others: dealt out evenly, through the
    workspace that was asked for; the same bits again, and without a workspace the same values."""
    g = np.random.default_rng(sequences)
    past = g.integers(10, 2 * longest // 100, sequences)
    lengths = [(int(p), 1) if i % 17 else (0, 0) for i, p in enumerate(past)]
    lengths[sequences // 3] = (longest - 1, 1)
    b = Batch(54, lengths, kv, d, 64, dtype, eight, one_each=True).fill()
    q, _ = strided(b.tokens, kv * group, d, b.dt, g, 2.0)
    ws = space(b, kv * group)
    assert ws.numel() > 0
    o = run(b, q, workspace=ws)
    assert not bool((ws == 0xFF).all())
    check_attention(b, q, o, 1 << 30, 0)
    assert torch.equal(o, run(b, q, workspace=ws))
    plain = run(b, q)
    check_attention(b, q, plain, 1 << 30, 0)
    assert bool((o[[i for i in range(sequences) if i % 17 == 0 and i != sequences // 3]] == 0).all())


def test_many_pieces_with_too_little_room():
    """Room for fewer workgroups than half of those that would share: a piece to each, the workspace is left alone."""
    lengths = [(20 + i % 50, 1) for i in range(130)]
    lengths[7] = (4300, 1)
    b = Batch(55, lengths, 8, 128, 64, "bf16", one_each=True).fill()
    q, _ = strided(b.tokens, 8, 128, b.dt, np.random.default_rng([55, 1]), 2.0)
    ws = space(b, 8)
    of_one = 2 * (128 + 2) * 4                                   # of a workgroup: two places for a row
    few, most = ws[: 200 * of_one], ws[: 400 * of_one]          # 512 share where there is room
    check_attention(b, q, run(b, q, workspace=few), 1 << 30, 0)
    assert bool((ws == 0xFF).all())
    check_attention(b, q, run(b, q, workspace=most), 1 << 30, 0)
    assert not bool((most == 0xFF).all()) and bool((ws[most.numel():] == 0xFF).all())


# ---- shares of prompts and chunks ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("past,new", [(448, 64), (0, 64), (200, 100), (900, 17)])
def test_shares_in_a_table_with_room_for_more(past, new, eight):
    """A share has at least two tiles of 64 tokens also where the table has room for a thousand: no row has more parts than that gives."""
    b = Batch(56, [(past, new)], 1, 128, 64, "bf16", eight).fill()
    wide = torch.full((1, 1024), -1, dtype=torch.int32, device="cuda")
    wide[:, : b.table.shape[1]] = b.table
    b.table = wide
    q, _ = strided(b.tokens, 4, 128, b.dt, np.random.default_rng([56, 1]), 2.0)
    ws = space(b, 4)
    check_attention(b, q, run(b, q, workspace=ws), 1 << 30, 0, one_product=True)
    written = int((ws.view(torch.int32) != -1).sum())
    tiles = -(-(past + new) // 64)
    assert written <= b.tokens * 4 * -(-tiles // 2) * (128 + 2)


@pytest.mark.parametrize("dtype,eight,wide", [("bf16", False, False), ("bf16", True, True), ("f32", False, False)])
@pytest.mark.parametrize("share", [0.02, 0.1, 0.4, 0.7])
def test_chunks_with_less_workspace(dtype, eight, wide, share):
    """Less room than the shares of a chunk would take: fewer of them, and nothing behind the room is written."""
    b = Batch(57, [(1900, 40), (700, 1), (0, 90)], 2, 64, 32, dtype, eight).fill()
    q, _ = strided(b.tokens, 6, 64, b.dt, np.random.default_rng([57, 1]), 2.0)
    ws = space(b, 6)
    some = ws[: int(ws.numel() * share) // 16 * 16]
    for window, sinks in ((None, 0), (300, 5)):
        check_attention(b, q, run(b, q, window, sinks, some, wide), window or 1 << 30, sinks, one_product=not wide and dtype == "bf16")
    assert bool((ws[some.numel():] == 0xFF).all())
    if share > 0.5:
        assert not bool((some == 0xFF).all())


# ---- calls of a serving loop ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,eight", [("bf16", False), ("bf16", True), ("f32", False)])
def test_two_graphs_share_a_workspace(dtype, eight):
    """A step and a chunk captured apart on the same workspace and replayed in turn, eager calls between them: the eager results each time."""
    step = Batch(58, [(900, 1), (0, 0), (3000, 1)], 2, 128, 16, dtype, eight, one_each=True).fill()
    chunk = Batch(59, [(1500, 30), (0, 70)], 2, 128, 16, dtype, eight).fill()
    gen = torch.Generator("cuda").manual_seed(58)
    calls = []
    ws = torch.empty(max(space(step, 8).numel(), space(chunk, 8).numel()), dtype=torch.uint8, device="cuda")
    for b in (step, chunk):
        q = torch.randn(b.tokens, 8, 128, device="cuda", generator=gen).to(b.dt)
        o = torch.empty_like(q)
        go = lambda b=b, q=q, o=o: B.a2sf_paged_attention(q, b.cache, b.table, b.len, o, starts=b.starts, window=2000, sinks=3,  # noqa: E731
                                                          workspace=ws)
        go()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go()
        calls.append((b, q, o, graph))
    for turn in range(4):
        for b, q, o, _ in calls:
            q.copy_(torch.randn(q.shape, device="cuda", generator=gen))
            o.zero_()
        for i in ((0, 1), (1, 0), (0, 0, 1), (1,))[turn]:
            calls[i][3].replay()
        torch.cuda.synchronize()
        for i, (b, q, o, _) in enumerate(calls):
            if (turn, i) != (3, 0):
                assert torch.equal(o, run(b, q, 2000, 3, ws)), (turn, i)


@pytest.mark.parametrize("dtype,eight", [("bf16", False), ("f32", True)])
def test_append_leaves_tokens_behind_the_last_sequence(dtype, eight):
    """A padded batch: rows that no sequence has write nothing, before the first start and behind the last."""
    b = Batch(60, [(5, 9), (0, 4), (30, 0), (17, 12)], 2, 64, 8, dtype, eight)
    heads, total = 3, 40
    x = torch.randn(total, (heads + 4) * 64, device="cuda", generator=torch.Generator("cuda").manual_seed(60)).to(b.dt)
    q, k, v = x.unflatten(1, (-1, 64)).split([heads, 2, 2], 1)
    table = torch.empty(64, 64, device="cuda")
    B.a2sf_rotary_table(table)
    first = 6
    want = torch.empty(25, heads, 64, dtype=b.dt, device="cuda")
    B.a2sf_paged_append(q[first: first + 25], k[first: first + 25], v[first: first + 25], b.cache, b.table, b.len, starts=b.starts, q_out=want,
                        rotary=table)
    bits = lambda t: t.clone().view(torch.uint8)  # noqa: E731
    kept = [bits(t) for t in b.cache.tensors()]
    b.rubbish()
    out = torch.full((total, heads, 64), 5.0, dtype=b.dt, device="cuda")
    B.a2sf_paged_append(q, k, v, b.cache, b.table, b.len, starts=b.starts + first, q_out=out, rotary=table)
    assert torch.equal(out[first: first + 25], want) and bool((out[:first] == 5).all()) and bool((out[first + 25:] == 5).all())
    assert all(torch.equal(bits(t), w) for t, w in zip(b.cache.tensors(), kept))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,given", [(70, 257), (9000, 1030), (9000, 1024), (300, 2000)])
def test_log_probs_of_more_tokens_than_lanes(dtype, n, given):
    """The same tokens again and again, some that are none, more of them than a row has lanes."""
    x = torch.randn(3, n, device="cuda", generator=torch.Generator("cuda").manual_seed(n)).to(DT[dtype])
    tokens = torch.randint(-1, n + 1, (3, given), dtype=torch.int32, device="cuda", generator=torch.Generator("cuda").manual_seed(given))
    logp = torch.full((3, given), 7.0, device="cuda")
    B.a2sf_log_probs(x, tokens, logp)
    check_log_probs(x, tokens, logp, None, None, None)
