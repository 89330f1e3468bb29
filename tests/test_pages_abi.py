"""Refusals of keys and values in pages and of log probabilities: found on the host, before any launch."""
import contextlib
import ctypes

import pytest
import torch

from paper_2407_20485_amd import binding as B

FAKE = 0x10000  # never dereferenced on these paths
ref = ctypes.byref
three, two = ctypes.c_int64 * 3, ctypes.c_int64 * 2


def heads(data=FAKE, stride=(1024, 128)):
    return ref(B.Heads(data, two(*stride)))


def pages(k=FAKE, v=FAKE, ks=None, vs=None, stride=(16384, 2048, 128), scale_stride=(128, 16, 1), pages=9, page_size=16, kv_heads=8, d=128,
          dtype=B.A2SF_BF16):
    return ref(B.PagesStruct(k, v, ks, vs, three(*stride), three(*scale_stride), pages, page_size, kv_heads, d, dtype))


def sequences(table=FAKE, lens=FAKE, starts=None, stride=4, n=5, table_pages=4):
    return ref(B.Sequences(table, lens, starts, stride, n, table_pages))


def append(q=None, k=None, v=None, tokens=5, h=8, dtype=B.A2SF_BF16, seqs=None, cache=None, table=FAKE, rows=32, rot=128, pairs=0, q_out=None):
    return B.lib().a2sf_paged_append(q, k or heads(), v or heads(), tokens, h, dtype, seqs or sequences(), cache or pages(), table, rows, rot,
                                     pairs, q_out, None)


def attend(q=None, tokens=5, h=8, dtype=B.A2SF_BF16, seqs=None, cache=None, window=B.A2SF_NO_WINDOW, sinks=0, o=None, ws=None, nbytes=0):
    return B.lib().a2sf_paged_attention(q or heads(), tokens, h, dtype, seqs or sequences(), cache or pages(), window, sinks,
                                        o or heads(2 * FAKE), ws, nbytes, None)


@pytest.mark.parametrize("call", [append, attend])
def test_pages_and_sequences_that_are_refused(call):
    eight = dict(dtype=B.A2SF_E4M3, ks=FAKE, vs=FAKE)
    assert call(cache=pages(k=None)) == B.A2SF_EINVAL
    assert call(cache=pages(v=FAKE + 8)) == B.A2SF_EINVAL                         # rows start at multiples of 16 bytes
    assert call(cache=pages(stride=(16384, 2048, 132))) == B.A2SF_ESHAPE
    assert call(cache=pages(stride=(16384, 2048, 64))) == B.A2SF_ESHAPE            # rows overlap
    assert call(cache=pages(stride=(-16384, 2048, 128))) == B.A2SF_ESHAPE
    assert call(cache=pages(stride=(1 << 45, 2048, 128))) == B.A2SF_ESHAPE
    assert call(cache=pages(d=96)) == B.A2SF_ESHAPE
    for size in (0, 24, -16, 131072):
        assert call(cache=pages(page_size=size)) == B.A2SF_ESHAPE
    assert call(cache=pages(pages=0)) == B.A2SF_ESHAPE
    assert call(cache=pages(kv_heads=0)) == B.A2SF_ESHAPE
    assert call(cache=pages(dtype=B.A2SF_F32)) == B.A2SF_EDTYPE                     # not the call's type
    assert call(cache=pages(dtype=3)) == B.A2SF_EDTYPE
    assert call(dtype=B.A2SF_E4M3, cache=pages(**eight)) == B.A2SF_EDTYPE           # the call's tensors are never of 8 bits
    assert call(cache=pages(dtype=B.A2SF_E4M3)) == B.A2SF_EINVAL                    # without scales
    assert call(cache=pages(ks=FAKE, vs=FAKE)) == B.A2SF_EINVAL                     # scales of no use
    assert call(cache=pages(scale_stride=(128, 0, 1), **eight)) == B.A2SF_ESHAPE
    assert call(cache=None, seqs=sequences(table=None)) == B.A2SF_EINVAL
    assert call(seqs=sequences(lens=None)) == B.A2SF_EINVAL
    assert call(seqs=sequences(starts=FAKE + 2)) == B.A2SF_EINVAL
    assert call(seqs=sequences(n=0)) == B.A2SF_ESHAPE
    assert call(seqs=sequences(n=4)) == B.A2SF_ESHAPE                               # a token each, but five tokens
    assert call(seqs=sequences(stride=3)) == B.A2SF_ESHAPE
    assert call(seqs=sequences(table_pages=0)) == B.A2SF_ESHAPE
    assert call(seqs=sequences(table_pages=1 << 27, stride=1 << 27)) == B.A2SF_ESHAPE  # positions of more than 31 bits
    assert call(tokens=0, seqs=sequences(starts=FAKE)) == B.A2SF_ESHAPE
    assert call(dtype=7) == B.A2SF_EDTYPE


def test_append_refusals():
    assert append(k=heads(None)) == B.A2SF_EINVAL
    assert append(k=heads(FAKE + 1)) == B.A2SF_EINVAL                               # not even an element's alignment
    assert append(v=heads(stride=(1024, 100))) == B.A2SF_ESHAPE
    assert append(v=heads(stride=(64, 128))) == B.A2SF_ESHAPE
    assert append(q=heads()) == B.A2SF_EINVAL                                       # nowhere to put it
    assert append(q_out=heads()) == B.A2SF_EINVAL
    assert append(q=heads(), q_out=heads(), h=0) == B.A2SF_ESHAPE
    assert append(q=heads(), q_out=heads(stride=(2048, 256))) == B.A2SF_EINVAL      # in place with another layout
    assert append(rot=126 + 4) == B.A2SF_ESHAPE
    assert append(rot=63) == B.A2SF_ESHAPE
    assert append(rows=0) == B.A2SF_ESHAPE
    assert append(pairs=2) == B.A2SF_EINVAL
    assert append(table=FAKE + 2) == B.A2SF_EINVAL


def test_attention_refusals():
    assert attend(q=heads(None)) == B.A2SF_EINVAL
    assert attend(o=heads(2 * FAKE + 1)) == B.A2SF_EINVAL
    assert attend(o=heads()) == B.A2SF_EINVAL                                       # in the place of q
    assert attend(o=heads(2 * FAKE, stride=(1024, 64))) == B.A2SF_ESHAPE
    assert attend(h=9) == B.A2SF_ESHAPE                                             # no multiple of the K/V heads
    assert attend(h=0) == B.A2SF_ESHAPE
    assert attend(window=0) == B.A2SF_EINVAL
    assert attend(window=-5) == B.A2SF_EINVAL
    assert attend(sinks=-1) == B.A2SF_EINVAL
    assert attend(ws=FAKE + 4, nbytes=1 << 20) == B.A2SF_EWORKSPACE
    assert attend(tokens=0x7FFFFFF, h=32 * 8, seqs=sequences(starts=FAKE)) == B.A2SF_ESHAPE


def test_choice_of_probabilities_is_checked_with_the_type():
    wide = B.A2SF_WIDE_SUMS
    assert attend(dtype=7 | wide) == B.A2SF_EDTYPE and attend(dtype=B.A2SF_E4M3 | wide) == B.A2SF_EDTYPE
    assert attend(dtype=B.A2SF_BF16 | 0x200) == B.A2SF_EDTYPE
    assert append(dtype=B.A2SF_BF16 | wide) == B.A2SF_EDTYPE                        # nothing to choose
    for dtype in (B.A2SF_BF16, B.A2SF_F32):
        assert attend(dtype=dtype | wide, cache=pages(dtype=dtype), window=0) == B.A2SF_EINVAL


def test_workspace_of_attention():
    f = B.a2sf_paged_workspace_bytes
    assert f(0, 32, 8, 128, 4, 4096) == 0 and f(4, 33, 8, 128, 4, 4096) == 0 and f(4, 32, 8, 96, 4, 4096) == 0
    assert f(4, 32, 8, 128, 4, 0) == 0 and f(1 << 40, 32, 8, 128, 4, 4096) == 0
    assert f(1, 32, 8, 128, 1, 16) == 0                                             # nothing to split
    one = f(1, 32, 8, 128, 1, 4096)
    assert 0 < one <= 512 * 2 * 4 * 130 * 4 and one % 4 == 0                        # two places of a group's heads per workgroup
    assert f(4096, 32, 8, 128, 4096, 4096) == 0                                     # workgroups enough


def test_workspace_of_many_pieces():
    """Two pieces and more for each workgroup: of use only where the table has room for long ones, and then whatever the window."""
    f = B.a2sf_paged_workspace_bytes
    shares = lambda d, g: (768 if d == 64 else 512) * 2 * g * (d + 2) * 4  # noqa: E731
    for sequences, kv, d, longest in ((255, 8, 128, 8160), (400, 8, 128, 12800), (300, 8, 64, 9600), (512, 16, 128, 32768)):
        assert f(sequences, 2 * kv, kv, d, sequences, longest) == shares(d, 2)
        assert f(sequences, 2 * kv, kv, d, sequences, longest - 1) == 0
    assert f(127, 16, 8, 128, 127, 300) >= shares(128, 2)                           # fewer: each is cut
    assert f(513, 16, 8, 128, 513, 1 << 20) == 0                                    # too many lengths to look at
    assert f(512, 4, 4, 128, 512, (1 << 31) - 512) == shares(128, 1)                # a window may leave few enough of them


def test_log_probs_refusals():
    r = lambda data=FAKE, stride=256: ref(B.Rows(data, stride))  # noqa: E731

    def f(x=None, rows=4, n=200, dtype=B.A2SF_F32, tokens=None, given=0, logp=None, entropy=FAKE, top=None, ids=None, k=0):
        return B.lib().a2sf_log_probs(x or r(), rows, n, dtype, tokens, given, logp, entropy, top, ids, k, None)

    assert f(entropy=None) == B.A2SF_EINVAL                                         # nothing is asked for
    assert f(entropy=FAKE + 2) == B.A2SF_EINVAL
    assert f(x=r(None)) == B.A2SF_EINVAL
    assert f(x=r(FAKE + 2)) == B.A2SF_EINVAL
    assert f(x=r(stride=199)) == B.A2SF_ESHAPE
    assert f(dtype=B.A2SF_E4M3) == B.A2SF_EDTYPE
    assert f(rows=0) == B.A2SF_ESHAPE and f(n=0) == B.A2SF_ESHAPE
    assert f(n=B.A2SF_MAX_VOCABULARY + 1, rows=1) == B.A2SF_ESHAPE
    assert f(tokens=r()) == B.A2SF_EINVAL                                           # given = 0
    assert f(given=2) == B.A2SF_EINVAL
    assert f(given=2, tokens=r()) == B.A2SF_EINVAL
    assert f(given=-1) == B.A2SF_ESHAPE
    assert f(given=300, tokens=r(), logp=r()) == B.A2SF_ESHAPE                      # rows overlap
    assert f(given=2, tokens=r(FAKE + 2), logp=r()) == B.A2SF_EINVAL
    assert f(k=5) == B.A2SF_EINVAL
    assert f(top=r()) == B.A2SF_EINVAL
    assert f(k=-1, top=r()) == B.A2SF_ESHAPE
    assert f(k=65, top=r()) == B.A2SF_ESHAPE
    assert f(k=9, n=8, top=r()) == B.A2SF_ESHAPE
    assert f(k=5, top=r(stride=4)) == B.A2SF_ESHAPE
    assert f(k=5, ids=r(None)) == B.A2SF_EINVAL


@contextlib.contextmanager
def refused():
    """An error, and not the one of a launch that was tried."""
    with pytest.raises(B.A2SFError) as e:
        yield
    assert e.value.status in (B.A2SF_EINVAL, B.A2SF_ESHAPE, B.A2SF_EDTYPE)


@pytest.fixture
def no_gpu():
    if torch.cuda.is_available():
        pytest.skip("looks at what the binding refuses in memory of the host")


def test_binding_takes_sizes_and_types_from_the_tensors(no_gpu):
    bf = torch.bfloat16
    with refused():
        B.Pages(4, 16, 2, 128, torch.float16, device="cpu")
    k = torch.zeros(4, 2, 16, 128, dtype=bf)
    with refused():
        B.Pages.of(k, k.transpose(1, 2).contiguous().transpose(1, 2))               # laid out differently
    with refused():
        B.Pages.of(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn))            # without scales
    both = torch.zeros(4, 2, 2, 16, 128, dtype=bf)
    cache = B.Pages.of(both[:, 0], both[:, 1])
    assert (cache.pages, cache.kv_heads, cache.page_size, cache.d) == (4, 2, 16, 128) and cache.struct.stride[0] == 2 * 2 * 16 * 128
    q, o = torch.zeros(3, 4, 128, dtype=bf), torch.empty(3, 4, 128, dtype=bf)
    table, lens = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    bad = [dict(q=q.float()), dict(q=q[..., :64]), dict(o=o[:2]), dict(o=o.float()), dict(table=table.long()), dict(lens=lens[:2]),
           dict(starts=torch.zeros(3, dtype=torch.int32)), dict(q=q[:, :3]), dict(window=0), dict(window=1 << 31), dict(sinks=-1)]
    for change in bad:
        a = dict(q=q, cache=cache, table=table, lens=lens, o=o, starts=None, window=None, sinks=0, stream=0)
        a.update(change)
        with refused():
            B.a2sf_paged_attention(**a)
    kn = torch.zeros(3, 2, 128, dtype=bf)
    for change in (dict(k=kn[:, :1]), dict(v=kn[:2]), dict(v=kn.float()), dict(q=q), dict(rotary=torch.zeros(5, 130)),
                   dict(rotary=torch.zeros(5, 64, dtype=torch.float64))):
        a = dict(q=None, k=kn, v=kn, cache=cache, table=table, lens=lens, stream=0)
        a.update(change)
        with refused():
            B.a2sf_paged_append(**a)
    x = torch.zeros(3, 50)
    for a in (dict(), dict(tokens=torch.zeros(3, 1, dtype=torch.int32)), dict(tokens=torch.zeros(3, 1), logp=torch.zeros(3, 1)),
              dict(entropy=torch.zeros(2)), dict(top=torch.zeros(3, 51)), dict(top=torch.zeros(3, 5), top_tokens=torch.zeros(3, 4, dtype=torch.int32)),
              dict(tokens=torch.zeros(3, 2, dtype=torch.int32), logp=torch.zeros(3, 1))):
        with refused():
            B.a2sf_log_probs(x, stream=0, **a)


def test_extension_leaves_unusual_arguments_to_ctypes():
    bf = torch.bfloat16
    k = torch.zeros(4, 2, 16, 128, dtype=bf)
    cache = B.Pages.of(k, k.clone())
    q = torch.zeros(3, 4, 128, dtype=bf)
    table, lens = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    at = B._entry("a2sf_paged_attention")
    good = dict(q=q, cache=cache, table=table, lens=lens, o=q.clone(), starts=None, window=None, sinks=0, workspace=None, nbytes=None,
                stream=None)
    assert B._call.paged_attention(at, *good.values()) == -1                                    # not on a GPU
    for change in (dict(q=5), dict(cache=cache.struct), dict(window=2.0), dict(sinks=None), dict(stream=0), dict(table=None), dict(lens=None)):
        assert B._call.paged_attention(at, *{**good, **change}.values()) == -1
    with pytest.raises(TypeError):
        B._call.paged_attention(at, q)
    assert B._call.paged_append(B._entry("a2sf_paged_append"), q, k, k, cache, table, lens, None, None, None, False, None) == -1
    assert B._call.log_probs(B._entry("a2sf_log_probs"), torch.zeros(3, 9), None, None, torch.zeros(3), None, None, None) == -1
