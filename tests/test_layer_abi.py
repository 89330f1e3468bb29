"""Refusals of the operators around the attention: found on the host, before any launch."""
import ctypes
import os
import re

import pytest
import torch

from paper_2407_20485_amd import binding as B

FAKE = 0x10000  # never dereferenced on these paths
ref = ctypes.byref


def rows(data=FAKE, stride=256):
    return ref(B.Rows(data, stride))


def rows8(data=FAKE, scales=FAKE, stride=256, scale_stride=4):
    return ref(B.Rows8(data, scales, stride, scale_stride))


def norm(x=None, residual=None, weight=FAKE, eps=1e-5, m=4, n=200, dtype=B.A2SF_BF16, total=None, out=None, out8=None):
    return B.lib().a2sf_rms_norm(x or rows(), residual, weight, eps, m, n, dtype, total, out, out8, None)


def test_rms_norm_refusals():
    assert norm() == B.A2SF_EINVAL                                        # no output
    assert norm(out=rows(None)) == B.A2SF_EINVAL
    assert norm(out=rows(FAKE + 1)) == B.A2SF_EINVAL                      # not even an element's alignment
    assert norm(x=rows(FAKE + 2), out=rows(), dtype=B.A2SF_F32) == B.A2SF_EINVAL
    assert norm(out=rows(), dtype=7) == B.A2SF_EDTYPE
    assert norm(out=rows(), n=0) == B.A2SF_ESHAPE
    assert norm(out=rows(), m=0) == B.A2SF_ESHAPE
    assert norm(out=rows(), n=B.A2SF_MAX_ROW + 1, m=1) == B.A2SF_ESHAPE
    assert norm(out=rows(stride=199)) == B.A2SF_ESHAPE                    # rows overlap
    assert norm(out=rows(), weight=None) == B.A2SF_EINVAL
    assert norm(out=rows(), residual=rows(None)) == B.A2SF_EINVAL
    for eps in (-1e-5, float("nan"), float("inf")):
        assert norm(out=rows(), eps=eps) == B.A2SF_EINVAL
    assert norm(out8=rows8(scales=None)) == B.A2SF_EINVAL
    assert norm(out8=rows8(FAKE + 8)) == B.A2SF_EINVAL
    assert norm(out8=rows8(stride=200)) == B.A2SF_ESHAPE                  # 8-bit rows start at multiples of 16
    assert norm(out8=rows8(scale_stride=2)) == B.A2SF_ESHAPE
    assert norm(out8=rows8(scale_stride=1)) == B.A2SF_ESHAPE


def test_quantize_refusals():
    f = B.lib().a2sf_quantize
    assert f(rows(), None, 4, 200, B.A2SF_BF16, None, None, None) == B.A2SF_EINVAL
    assert f(None, None, 4, 200, B.A2SF_BF16, None, rows8(), None) == B.A2SF_EINVAL
    assert f(rows(), rows(stride=10), 4, 200, B.A2SF_BF16, None, rows8(), None) == B.A2SF_ESHAPE
    assert f(rows(), None, 4, 200, 2, None, rows8(), None) == B.A2SF_EDTYPE
    assert f(rows(), None, 2 ** 31 - 1, 200, B.A2SF_BF16, None, rows8(), None) == B.A2SF_ESHAPE
    w = B.lib().a2sf_quantize_weight
    assert w(rows(), 4, 200, B.A2SF_BF16, None, None) == B.A2SF_EINVAL
    assert w(rows(), 0, 200, B.A2SF_BF16, rows8(), None) == B.A2SF_ESHAPE
    assert w(rows(), 200, 200, B.A2SF_BF16, rows8(scale_stride=3), None) == B.A2SF_ESHAPE


def test_matmul_refusals():
    def f(a=None, b=None, c=None, m=4, n=200, k=200, dtype=B.A2SF_BF16, ws=None, nbytes=0):
        return B.lib().a2sf_matmul_scaled(a or rows8(), b or rows8(), m, n, k, c or rows(), dtype, ws, nbytes, None)

    assert f(a=rows8(None)) == B.A2SF_EINVAL
    assert f(b=rows8(FAKE + 4)) == B.A2SF_EINVAL
    assert f(a=rows8(scales=FAKE + 1)) == B.A2SF_EINVAL
    assert f(a=rows8(stride=200)) == B.A2SF_ESHAPE
    assert f(b=rows8(stride=208), k=209) == B.A2SF_ESHAPE
    assert f(c=rows(stride=199)) == B.A2SF_ESHAPE
    assert f(c=rows(FAKE + 1)) == B.A2SF_EINVAL
    assert f(k=0) == B.A2SF_ESHAPE
    assert f(m=0) == B.A2SF_ESHAPE
    assert f(dtype=9) == B.A2SF_EDTYPE
    assert f(k=(1 << 20) + 1, a=rows8(stride=1 << 21), b=rows8(stride=1 << 21)) == B.A2SF_ESHAPE
    assert f(a=rows8(stride=1 << 24)) == B.A2SF_ESHAPE
    assert f(ws=FAKE + 8, nbytes=1 << 20) == B.A2SF_EWORKSPACE
    assert B.a2sf_matmul_workspace_bytes(0, 5, 5) == 0
    assert B.a2sf_matmul_workspace_bytes(8192, 8192, 4096) == 0          # tiles enough
    assert B.a2sf_matmul_workspace_bytes(64, 4096, 16384) <= 32 << 20


def test_matmul_refuses_scales_too_far_apart():
    far = rows8(scale_stride=(1 << 23) + 4)
    assert B.lib().a2sf_matmul_scaled(far, rows8(), 4, 200, 200, rows(), B.A2SF_BF16, None, 0, None) == B.A2SF_ESHAPE
    assert B.lib().a2sf_matmul_scaled(rows8(), far, 4, 200, 200, rows(), B.A2SF_BF16, None, 0, None) == B.A2SF_ESHAPE


def part(x=FAKE, y=FAKE + 4096, xs=(4096, 512, 64), ys=(4096, 512, 64), heads=8, rotate=1):
    return B.RotaryPart(x, y, (ctypes.c_int64 * 3)(*xs), (ctypes.c_int64 * 3)(*ys), heads, rotate)


def test_rotary_refusals():
    def f(*parts, n=None, batch=2, length=8, d=64, dtype=B.A2SF_BF16, pos=FAKE, pos_stride=8, table=FAKE, table_rows=32, rot=64, pairs=0):
        made = (B.RotaryPart * max(1, len(parts)))(*parts)
        return B.lib().a2sf_rotary(made, len(parts) if n is None else n, batch, length, d, dtype, pos, pos_stride, table,
                                   table_rows, rot, pairs, 0, None)

    assert f() == B.A2SF_EINVAL
    assert f(part(), n=5) == B.A2SF_EINVAL
    assert f(part(), dtype=3) == B.A2SF_EDTYPE
    assert f(part(), pairs=2) == B.A2SF_EINVAL
    assert f(part(), rot=63) == B.A2SF_ESHAPE
    assert f(part(), rot=66) == B.A2SF_ESHAPE
    assert f(part(), d=513) == B.A2SF_ESHAPE
    assert f(part(), pos=None) == B.A2SF_EINVAL
    assert f(part(), pos_stride=7) == B.A2SF_ESHAPE
    assert f(part(), table_rows=0) == B.A2SF_ESHAPE
    assert f(part(heads=0)) == B.A2SF_ESHAPE
    assert f(part(x=FAKE + 1)) == B.A2SF_EINVAL
    assert f(part(xs=(4096, -512, 64))) == B.A2SF_ESHAPE
    assert f(part(y=FAKE, ys=(4096, 64, 512))) == B.A2SF_EINVAL           # in place with another layout
    t = B.lib().a2sf_rotary_table
    assert t(None, 8, 64, 1e4, 1.0, 0, 0.0, 0.0, 1.0, None) == B.A2SF_EINVAL
    assert t(FAKE, 8, 63, 1e4, 1.0, 0, 0.0, 0.0, 1.0, None) == B.A2SF_ESHAPE
    assert t(FAKE, 8, 64, 0.0, 1.0, 0, 0.0, 0.0, 1.0, None) == B.A2SF_EINVAL
    assert t(FAKE, 8, 64, 1e4, 0.0, 0, 0.0, 0.0, 1.0, None) == B.A2SF_EINVAL
    assert t(FAKE, 8, 64, 1e4, 2.0, 100, 4.0, 1.0, 1.0, None) == B.A2SF_EINVAL
    assert t(FAKE, 8, 64, 1e4, 2.0, -1, 1.0, 4.0, 1.0, None) == B.A2SF_EINVAL


def test_sample_refusals():
    def f(logits=None, noise=None, m=4, n=200, dtype=B.A2SF_F32, token=FAKE, temperature=None, prob=None):
        return B.lib().a2sf_sample(logits or rows(), noise, m, n, dtype, temperature, None, None, None, token, prob, None)

    assert f(token=None) == B.A2SF_EINVAL
    assert f(token=FAKE + 2) == B.A2SF_EINVAL
    assert f(prob=FAKE + 2) == B.A2SF_EINVAL
    assert f(temperature=FAKE + 1) == B.A2SF_EINVAL
    assert f(noise=rows(FAKE + 2)) == B.A2SF_EINVAL
    assert f(noise=rows(stride=100)) == B.A2SF_ESHAPE
    assert f(logits=rows(FAKE + 2)) == B.A2SF_EINVAL
    assert f(n=0) == B.A2SF_ESHAPE
    assert f(m=1, n=B.A2SF_MAX_VOCABULARY + 1) == B.A2SF_ESHAPE
    assert f(dtype=4) == B.A2SF_EDTYPE


def test_python_calls_refuse_what_does_not_fit_together():
    """Tensors on the host: the extension leaves them to the ctypes form, which names the error before anything is called."""
    x = torch.zeros(4, 200, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 208, dtype=torch.float8_e4m3fn)[:, :200], torch.zeros(4, 4, dtype=torch.uint8)[:, :2]

    def status(call):
        with pytest.raises(B.A2SFError) as e:
            call()
        return e.value.status

    w = torch.ones(200, dtype=torch.bfloat16)
    assert status(lambda: B.a2sf_rms_norm(x, w[:100], 1e-5, q=q, scales=s)) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_rms_norm(x, w.float(), 1e-5, q=q, scales=s)) == B.A2SF_EDTYPE
    assert status(lambda: B.a2sf_rms_norm(x, w, 1e-5, residual=x[:3], q=q, scales=s)) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_rms_norm(x, w, 1e-5, q=q)) == B.A2SF_EINVAL
    assert status(lambda: B.a2sf_rms_norm(x, w, 1e-5)) == B.A2SF_EINVAL
    assert status(lambda: B.a2sf_rms_norm(x.t(), w[:4], 1e-5, out=x.t())) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_rms_norm(x.half(), w.half(), 1e-5, out=x.half())) == B.A2SF_EDTYPE
    assert status(lambda: B.a2sf_quantize(x, q, s[:, :1])) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_quantize(x, q.view(torch.float8_e5m2), s)) == B.A2SF_EDTYPE
    assert status(lambda: B.a2sf_quantize(x, q, s, gate=x.float())) == B.A2SF_EDTYPE
    b, bs = torch.zeros(9, 208, dtype=torch.uint8)[:, :200], torch.zeros(1, 4, dtype=torch.uint8)[:, :2]
    assert status(lambda: B.a2sf_matmul_scaled(q, s, b, bs, torch.zeros(4, 8))) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_matmul_scaled(q, s, b[:, :150], bs, torch.zeros(4, 9))) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_matmul_scaled(q, s, b, bs, torch.zeros(4, 9).half())) == B.A2SF_EDTYPE
    h, pos, table = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(9, 64)
    assert status(lambda: B.a2sf_rotary([], pos, table)) == B.A2SF_EINVAL
    assert status(lambda: B.a2sf_rotary([(h, h[:1])], pos, table)) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_rotary([(h, h)], pos[:1], table)) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_rotary([(h, h)], pos.long(), table)) == B.A2SF_EDTYPE
    assert status(lambda: B.a2sf_rotary([(h, h.bfloat16())], pos, table)) == B.A2SF_EDTYPE
    assert status(lambda: B.a2sf_rotary([(h, h)], pos, torch.zeros(9, 66))) == B.A2SF_ESHAPE
    logits, token = torch.zeros(4, 50), torch.zeros(4, dtype=torch.int32)
    assert status(lambda: B.a2sf_sample(logits, logits[:, :49], token)) == B.A2SF_ESHAPE
    assert status(lambda: B.a2sf_sample(logits, logits.bfloat16(), token)) == B.A2SF_EDTYPE
    assert status(lambda: B.a2sf_sample(logits, logits, token.long())) == B.A2SF_EDTYPE
    assert status(lambda: B.a2sf_sample(logits, logits, token, top_k=torch.ones(4))) == B.A2SF_EDTYPE
    assert status(lambda: B.a2sf_sample(logits, logits, token[:3])) == B.A2SF_ESHAPE


def test_extension_leaves_unusual_arguments_to_ctypes():
    B.lib()
    x = torch.zeros(4, 200)
    t = torch.zeros(4, dtype=torch.int32)
    assert B._call.rms_norm(B._entry("a2sf_rms_norm"), x, x[0], 1e-5, None, None, x, None, None, None) == -1  # not on a GPU
    assert B._call.rms_norm(B._entry("a2sf_rms_norm"), x, x[0], 1, None, None, x, None, None, None) == -1     # eps no float
    assert B._call.sample(B._entry("a2sf_sample"), x, None, t, None, None, None, None, None, 5) == -1
    assert B._call.rotary(B._entry("a2sf_rotary"), ((x, x),), t, x, False, False, None) == -1                 # no list
    assert B._call.rotary(B._entry("a2sf_rotary"), [(x, x)], t, x, False, False, None) == -1
    assert B._call.quantize(B._entry("a2sf_quantize"), 5, None, None, None, None, None) == -1
    assert B._call.matmul_scaled(B._entry("a2sf_matmul_scaled"), x, x, x, x, x, None, None, None) == -1
    with pytest.raises(TypeError):
        B._call.sample(x)


def test_matmul_choice_of_sums_is_checked_with_the_type():
    f = lambda dtype, k=200: B.lib().a2sf_matmul_scaled(rows8(), rows8(), 4, 200, k, rows(), dtype, None, 0, None)
    assert f(9 | B.A2SF_WIDE_SUMS) == B.A2SF_EDTYPE
    assert f(B.A2SF_BF16 | 0x200) == B.A2SF_EDTYPE
    assert f(B.A2SF_BF16 | B.A2SF_WIDE_SUMS, k=0) == B.A2SF_ESHAPE
    header = open(os.path.join(os.path.dirname(B.__file__), "..", "include", "a2sf.h")).read()
    assert int(re.search(r"#define A2SF_WIDE_SUMS (0x[0-9a-f]+)", header)[1], 16) == B.A2SF_WIDE_SUMS


def test_calls_of_more_lanes_than_a_launch_takes_are_refused():
    """Found on the host: no launch is tried."""
    L, far = B.lib(), 1 << 17
    for n, m in ((1025, 2 ** 24), (5000, 2 ** 24), (10000, 2 ** 23), (40000, 2 ** 22), (128, 2 ** 26 + 4)):
        assert L.a2sf_rms_norm(rows(stride=far), None, FAKE, 1e-5, m, n, B.A2SF_F32, None, rows(stride=far), None, None) == B.A2SF_ESHAPE, n
    for gate in (None, rows(stride=far)):
        assert L.a2sf_quantize(rows(stride=far), gate, 2 ** 28, 100, B.A2SF_BF16, rows(stride=far), None, None) == B.A2SF_ESHAPE
        assert L.a2sf_quantize(rows(stride=far), gate, 2 ** 27, 200, B.A2SF_F32, rows(stride=far), None, None) == B.A2SF_ESHAPE
    out8 = rows8(stride=far, scale_stride=1024)
    assert L.a2sf_quantize_weight(rows(stride=far), 2 ** 24, 2 ** 14, B.A2SF_BF16, out8, None) == B.A2SF_ESHAPE
    assert L.a2sf_sample(rows(stride=far), None, 2 ** 22, 100, B.A2SF_F32, None, None, None, None, FAKE, None, None) == B.A2SF_ESHAPE
    made = (B.RotaryPart * 1)(part(xs=(far, far, 512), ys=(far, far, 512), heads=64))
    assert L.a2sf_rotary(made, 1, 2 ** 24, 4, 512, B.A2SF_F32, FAKE, 4, FAKE, 32, 64, 0, 0, None) == B.A2SF_ESHAPE


def test_tensors_of_another_device_are_refused():
    """Not handed on as addresses; here "meta" stands for the other device."""
    x = torch.zeros(4, 200, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 208, dtype=torch.uint8)[:, :200], torch.zeros(4, 4, dtype=torch.uint8)[:, :2]
    w, b, bs = torch.ones(200, dtype=torch.bfloat16), torch.zeros(9, 208, dtype=torch.uint8)[:, :200], torch.zeros(1, 4, dtype=torch.uint8)[:, :2]
    c, ws = torch.zeros(4, 9), torch.zeros(64, dtype=torch.uint8)
    h, pos, table = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(9, 64)
    logits, token, k, f = torch.zeros(4, 50), torch.zeros(4, dtype=torch.int32), torch.ones(4, dtype=torch.int32), torch.ones(4)

    def away(t):  # the same sizes and strides elsewhere
        return torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="meta")

    calls = [(B.a2sf_rms_norm, (x, w, 1e-5), dict(residual=x, total=x, out=x, q=q, scales=s)), (B.a2sf_quantize, (x, q, s), dict(gate=x, out=x)),
             (B.a2sf_quantize_weight, (x, q, torch.zeros(1, 4, dtype=torch.uint8)[:, :2]), {}), (B.a2sf_matmul_scaled, (q, s, b, bs, c), dict(workspace=ws)),
             (lambda y, pos, table, v: B.a2sf_rotary([(h, y), (v, v, False)], pos, table), (h, pos, table, h), {}),
             (B.a2sf_sample, (logits, logits, token), dict(temperature=f, top_k=k, top_p=f, min_p=f, prob=f))]
    for call, args, named in calls:
        for i, t in enumerate(args):
            if isinstance(t, torch.Tensor):
                with pytest.raises(B.A2SFError) as e:
                    call(*args[:i], away(t), *args[i + 1:], **named)
                assert e.value.status == B.A2SF_EINVAL, (call, i)
        for name, t in named.items():
            with pytest.raises(B.A2SFError) as e:
                call(*args, **{**named, name: away(t)})
            assert e.value.status == B.A2SF_EINVAL, (call, name)


def test_sizes_above_32_bits_are_refused():
    """Rows repeated in place (no memory behind them): 2^32 + 1 of them are not 1."""
    many = lambda n, dtype: torch.zeros(1, n, dtype=dtype).expand(2 ** 32 + 1, n)  # noqa: E731
    x, q, s = many(128, torch.bfloat16), many(128, torch.uint8), many(1, torch.uint8)
    h, pos = torch.zeros(1, 1, 1, 64).expand(2 ** 32 + 1, 1, 1, 64), torch.zeros(1, 1, dtype=torch.int32).expand(2 ** 32 + 1, 1)
    for call in (lambda: B.a2sf_quantize(x, q, s), lambda: B.a2sf_rms_norm(x, x[0], 1e-5, out=x),
                 lambda: B.a2sf_quantize_weight(x, q, torch.zeros(1, 1, dtype=torch.uint8).expand(2 ** 25 + 1, 1)),
                 lambda: B.a2sf_matmul_scaled(q, s, q[:1], s[:1], torch.zeros(1, 1).expand(2 ** 32 + 1, 1)),
                 lambda: B.a2sf_rotary([(h, h)], pos, torch.zeros(4, 64)),
                 lambda: B.a2sf_rotary_table(torch.zeros(1, 0).expand(2 ** 32 + 1, 0)),
                 lambda: B.a2sf_sample(x, None, torch.zeros(1, dtype=torch.int32).expand(2 ** 32 + 1))):
        with pytest.raises(B.A2SFError) as e:
            call()
        assert e.value.status == B.A2SF_ESHAPE
    assert B.a2sf_matmul_workspace_bytes(2 ** 32 + 100, 4096, 11008) == 0
