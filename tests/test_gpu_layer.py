"""The operators around the attention on the GPU against the float64 oracle.

Tolerances, from the arithmetic (u = 2^-24 is fp32's unit of rounding):
  * a sum of n squares by fused multiply-adds, at most 64 + 16 of them one after the other, is off by at most 80 u, its root by 40 u;
    with the additions, divisions and products around it a norm is within 48 u = 3e-6 of its value, plus 2^-8 where it is
    rounded to bf16;
  * silu: two instructions of about one u each, the exponent's argument off by |g| u with |g| <= 88: 100 u = 6e-6;
  * 8-bit values: half a step of three bits, 2^-4 of the value, or half a step of the smallest, 2^-10 of the scale;
    without arithmetic before it (plain rows) the conversion is exact to the bit;
  * a product of k terms in fp32: k u times the sum of the magnitudes; for a bf16 result the matrix instruction cuts each of eight
    products under 2^-13 of the largest of them: 8 * 2^-13 of that sum; of small whole numbers it is exact.
"""
import math

import numpy as np
import pytest
import torch

from oracle import layer_oracle as L
from paper_2407_20485_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BF16 = 2.0 ** -8  # half of the distance 2^-7 between neighbours of seven bits behind the point, of the smallest value that has it


def up(x, m):
    return -(-x // m) * m


def rng(*key):
    return np.random.default_rng([7, *key])


def on_gpu(a, dtype, stride=None, offset=0):
    """A tensor of a's values whose rows lie `stride` elements apart and start `offset` elements into an allocation."""
    a = torch.from_numpy(np.ascontiguousarray(a)).float()
    rows, n = a.shape
    stride = stride or n
    store = torch.full((offset + rows * stride + 16,), 7.0, dtype=dtype, device="cuda")
    t = torch.as_strided(store, (rows, n), (stride, 1), offset)
    t.copy_(a)
    return t


def host(t):
    return t.detach().double().cpu().numpy()


def eight(rows, n, scale_rows=None, extra=0):
    """8-bit buffers filled with marks, so that what is written past a row's end shows."""
    q = torch.full((rows, up(n, 16) + extra), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((scale_rows or rows, up(-(-n // 128), 4)), 0x55, dtype=torch.uint8, device="cuda")
    return q[:, :n], s[:, : -(-n // 128)]


def check_marks(q, s):
    n, nb = q.shape[1], s.shape[1]
    assert bool((q._base[:, n:] == 0x55).all()) and bool((s._base[:, nb:] == 0x55).all())


def check_eight(q, s, y, rel, rows_per_scale=1):
    """q, s stand for y (float64) as the format says, y being known to `rel`."""
    q, s = q.cpu().numpy(), s.cpu().numpy()
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            at = slice(i * rows_per_scale, (i + 1) * rows_per_scale), slice(j * 128, (j + 1) * 128)
            block = y[at]
            if not np.isfinite(block).all():
                assert s[i, j] == 255 and (q[at] == 0x7F).all()
                continue
            top, unit = np.abs(block).max(), 2.0 ** (float(s[i, j]) - 127)
            assert top <= 448 * unit * (1 + rel)
            assert s[i, j] == 0 or top > 224 * unit * (1 - rel)
            off = np.abs(L.E4M3[q[at]] * unit - block)
            assert (off <= np.maximum(2.0 ** -4 * np.abs(block), 2.0 ** -10 * unit) + rel * np.abs(block)).all()


# ---- norm -----------------------------------------------------------------------------------------------------------------

NORM = [(1, 1), (3, 7), (2, 64), (5, 127), (4, 128), (3, 129), (9, 512), (6, 1000), (5, 1024), (2, 1025), (7, 2048), (3, 2500), (1, 4096),
        (600, 4096), (2, 5120), (520, 5125), (2, 8192), (515, 9000), (3, 12000), (514, 16384), (2, 20001), (1, 40000), (2, 65536)]


@pytest.mark.parametrize("rows,n", NORM)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rms_norm(rows, n, dtype):
    g = rng(rows, n)
    dt = DT[dtype]
    x = on_gpu(g.normal(size=(rows, n)) * g.choice([0.01, 1.0, 30.0], size=(rows, 1)), dt)
    r = on_gpu(g.normal(size=(rows, n)), dt, stride=n + 3, offset=5)
    w = on_gpu(1 + 0.1 * g.normal(size=(1, n)), dt)[0]
    total, out = (on_gpu(np.zeros((rows, n)), dt, stride=n + s) for s in (0, 8))
    q, s = eight(rows, n)
    B.a2sf_rms_norm(x, w, 1e-5, residual=r, total=total, out=out, q=q, scales=s)
    few = slice(0, rows, max(1, rows // 8))
    h, y = L.rms_norm(host(x[few]), host(r[few]), host(w), 1e-5)
    half = BF16 if dtype == "bf16" else 0.0
    assert (np.abs(host(total[few]) - h) <= (half + 2.0 ** -24) * np.abs(h)).all()
    # a sum that nearly cancels keeps the error of its rounding, relative to the terms
    slack = 3e-6 * np.abs(y) + 2.0 ** -24 * np.abs(y / np.where(h == 0, 1, h)) * (np.abs(host(x[few])) + np.abs(host(r[few])))
    assert (np.abs(host(out[few]) - y) <= half * np.abs(y) + slack).all()
    check_eight(q[few], s[few], y, 5e-6 if dtype == "f32" else 5e-6)
    check_marks(q, s)
    # the same without the residual, 8 bits alone, and again: the same bits
    q2, s2 = eight(rows, n)
    B.a2sf_rms_norm(x, w, 1e-5, q=q2, scales=s2)
    check_eight(q2[few], s2[few], L.rms_norm(host(x[few]), None, host(w), 1e-5)[1], 5e-6)
    q3, s3 = eight(rows, n)
    B.a2sf_rms_norm(x, w, 1e-5, q=q3, scales=s3)
    assert torch.equal(q2, q3) and torch.equal(s2, s3)


@pytest.mark.parametrize("rows,n", [(4100, 1100), (4097, 1999), (513, 2600), (513, 6143), (514, 6145), (512, 12290)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rms_norm_many_rows(rows, n, dtype):
    test_rms_norm(rows, n, dtype)


def test_rms_norm_rounds_to_8_bits_once():
    """Next to no 8-bit value is another than that of the result in 64 bits: of those the result lies within 2^-22 of half-way (the
    units' sums of eight squares in 32 bits are off by 8 * 2^-24 at most, their root's by half of that, and the products by less)."""
    g = rng(19)
    x, w = on_gpu(g.normal(size=(400, 2048)), torch.bfloat16), on_gpu(1 + 0.1 * g.normal(size=(1, 2048)), torch.bfloat16)[0]
    q, s = eight(400, 2048)
    B.a2sf_rms_norm(x, w, 1e-6, q=q, scales=s)
    h = host(x)
    y = h / np.sqrt((h ** 2).mean(1, keepdims=True) + float(np.float32(1e-6))) * host(w)
    at = lambda f: L.quantize(y * (1 + f * 2.0 ** -22))
    (lo, slo), (hi, shi) = at(-1), at(1)
    got, gots = q.cpu().numpy(), s.cpu().numpy()
    same = np.repeat(slo == shi, 128, 1)
    assert ((got == lo) | (got == hi))[same].all() and ((gots == slo) | (gots == shi)).all()
    want, _ = L.quantize(y)
    assert (got != want).sum() <= 5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rms_norm_in_place(dtype):
    g = rng(1)
    x, r = (g.normal(size=(70, 777)) for _ in range(2))
    w = on_gpu(g.normal(size=(1, 777)), DT[dtype])[0]
    tx, tr = on_gpu(x, DT[dtype]), on_gpu(r, DT[dtype])
    total, out = torch.empty_like(tx), torch.empty_like(tx)
    B.a2sf_rms_norm(tx, w, 1e-6, residual=tr, total=total, out=out)
    B.a2sf_rms_norm(tx, w, 1e-6, residual=tr, total=tr, out=tx)
    assert torch.equal(tr, total) and torch.equal(tx, out)


@pytest.mark.parametrize("rows,n", [(3, 200), (5, 1000), (520, 2500), (2, 4096), (515, 9000), (2, 12000), (3, 40000)])
@pytest.mark.parametrize("size", [3e38, 1e30, 4e19, 1e19, 1e17, 1e-15, 1e-18, 1e-25, 1e-36])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rms_norm_at_the_ends_of_the_range(rows, n, size, dtype):
    """Finite rows whose squares are no finite or no normal numbers of 32 bits, without eps where it would be all of the mean.  The same
    tolerance as in the middle of the range."""
    g = rng(26, rows, n)
    dt = DT[dtype]
    x, r = (g.uniform(-0.49, 0.49, size=(rows, n)) * size for _ in range(2))
    x[:, n // 3] = 0.5 * size                      # all of a row, or one element of it, is that large
    x[1, : n // 2], r[1] = x[1, : n // 2] * 1e-3, 0.0
    x, r = on_gpu(x, dt, stride=n + 1), on_gpu(r, dt)
    w = on_gpu(1 + 0.1 * g.normal(size=(1, n)), dt)[0]
    total, out = (on_gpu(np.zeros((rows, n)), dt, stride=n + s) for s in (2, 8))
    q, s = eight(rows, n)
    eps = 0.0 if size < 1 else 1e-5
    B.a2sf_rms_norm(x, w, eps, residual=r, total=total, out=out, q=q, scales=s)
    few = slice(0, rows, max(1, rows // 4))
    h, y = L.rms_norm(host(x[few]), host(r[few]), host(w), eps)
    half = BF16 if dtype == "bf16" else 0.0
    # (bf16's subnormal numbers are 2^-133 apart)
    assert (np.abs(host(total[few]) - h) <= (half + 2.0 ** -24) * np.abs(h) + (2.0 ** -134 if half else 0.0)).all()
    slack = 3e-6 * np.abs(y) + 2.0 ** -24 * np.abs(y / np.where(h == 0, 1, h)) * (np.abs(host(x[few])) + np.abs(host(r[few])))
    assert (np.abs(host(out[few]) - y) <= half * np.abs(y) + slack).all()
    check_eight(q[few], s[few], y, 5e-6)
    check_marks(q, s)


def test_rms_norm_of_subnormal_numbers_without_eps():
    x = torch.zeros(3, 300, device="cuda")
    x[0, 7], x[1] = 1e-45, 3e-42
    out = torch.empty_like(x)
    B.a2sf_rms_norm(x, torch.ones(300, device="cuda"), 0.0, out=out)
    assert abs(float(out[0, 7]) - math.sqrt(300)) < 1e-4 and float(out[0].abs().sum()) == float(out[0, 7])
    assert bool(((out[1] - 1).abs() < 1e-6).all()) and bool(torch.isnan(out[2]).all())   # a row of zeros: 0 / 0


def test_rms_norm_rows_that_are_not_numbers():
    x = torch.randn(6, 300, device="cuda")
    x[1, 5], x[2, 299] = math.nan, math.inf
    x[3] = 0.0
    x[4] = 1e-30  # squares vanish beside eps
    w = torch.ones(300, device="cuda")
    out = torch.empty_like(x)
    q, s = eight(6, 300)
    B.a2sf_rms_norm(x, w, 1e-5, out=out, q=q, scales=s)
    assert bool(torch.isnan(out[1]).all()) and bool((s[1] == 255).all()) and bool((q[1] == 0x7F).all())
    assert bool(torch.isnan(out[2, 299])) and bool((out[2, :299] == 0).all())     # divided by infinity
    assert s[2].tolist() == [0, 0, 255]
    assert bool((out[3] == 0).all()) and s[3].tolist() == [0, 0, 0] and bool((q[3] == 0).all())
    _, y = L.rms_norm(host(x[4:]), None, np.ones(300), 1e-5)
    check_eight(q[4:], s[4:], y, 5e-6)
    check_marks(q, s)


# ---- rows to 8 bits ---------------------------------------------------------------------------------------------------------

QUANT = [(1, 1), (1, 15), (3, 128), (2, 130), (17, 257), (5, 1001), (64, 4096), (3, 11008), (2, 70001)]


@pytest.mark.parametrize("rows,n", QUANT)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_is_exact(rows, n, dtype):
    g = rng(2, rows, n)
    v = g.normal(size=(rows, n)) * 2.0 ** g.integers(-12, 12, size=(rows, n))
    v[:, :: 37] = 0.0
    x = on_gpu(v, DT[dtype], stride=n + 1, offset=3)
    q, s = eight(rows, n, extra=16)
    B.a2sf_quantize(x, q, s)
    wq, ws = L.quantize(host(x))
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(q.cpu().numpy(), wq)
    check_marks(q, s)


def test_quantize_at_the_edges_of_the_scale():
    """Blocks whose largest value is 448 times a power of two, or a little more; ties; values too small to be seen; ends of the range."""
    v = np.zeros((7, 128))
    v[0, :4] = 448.0, -1.0, 18.0, 19.0          # 18, 19: steps of 2; 19 and 17 are ties
    v[1, :4] = 448.1, 17.0, 1.0, 2.0 ** -9
    v[2, :4] = 1e-45, 3e-45, -1e-45, 0.0        # subnormal numbers
    v[3, :4] = 3.3e38, 1.0, -3.3e38, 1e30
    v[4, :4] = 448.0, 2.0 ** -10, 1.5 * 2.0 ** -9, 2.0 ** -9
    v[5, 0], v[5, 1] = math.inf, 1.0
    v[6, 100] = math.nan
    x = torch.from_numpy(v).float().cuda()
    q, s = eight(7, 128)
    B.a2sf_quantize(x, q, s)
    wq, ws = L.quantize(host(x))
    assert s[:, 0].tolist() == ws[:, 0].tolist() and np.array_equal(q.cpu().numpy(), wq)


@pytest.mark.parametrize("rows,n", QUANT)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gated_rows(rows, n, dtype):
    g = rng(3, rows, n)
    both = on_gpu(g.normal(size=(rows, 2 * n)) * 4, DT[dtype])   # gate and up: two halves of one product
    gate, x = both[:, :n], both[:, n:]
    out = on_gpu(np.zeros((rows, n)), DT[dtype], stride=n + 5)
    q, s = eight(rows, n)
    B.a2sf_quantize(x, q, s, gate=gate, out=out)
    y = L.gated(host(x), host(gate))
    half = BF16 if dtype == "bf16" else 0.0
    assert (np.abs(host(out) - y) <= (half + 6e-6) * np.abs(y)).all()
    check_eight(q, s, y, 6e-6)
    check_marks(q, s)
    only = torch.empty(rows, n, dtype=DT[dtype], device="cuda")
    B.a2sf_quantize(x, None, None, gate=gate, out=only)
    assert torch.equal(only, out)


def test_gate_far_from_zero():
    g = torch.tensor([[-1e4, -200.0, -88.0, 88.0, 200.0, 1e4, 0.0, -0.0]], device="cuda")
    out = torch.empty_like(g)
    B.a2sf_quantize(torch.ones_like(g), None, None, gate=g, out=out)
    assert np.allclose(host(out), L.gated(np.ones((1, 8)), host(g)), rtol=1e-5, atol=1e-30)


def test_gate_is_good_to_a_few_units_wherever_it_is():
    """fp32: exp 2 u and its correction u, that twice (above and below the line), the sum u, the reciprocal 2 u, three products: 12 u."""
    g = rng(25)
    gate = on_gpu(np.concatenate([np.linspace(-86, 88, 30000), g.normal(size=30000) * 8])[None].clip(-86, 88), torch.float32)
    x, out = on_gpu(g.normal(size=gate.shape), torch.float32), torch.empty_like(gate)
    B.a2sf_quantize(x, None, None, gate=gate, out=out)
    y = L.gated(host(x), host(gate))
    assert (np.abs(host(out) - y) / np.abs(y).clip(1e-300)).max() <= 12 * 2.0 ** -24


def test_gate_of_what_is_not_finite():
    inf, nan = math.inf, math.nan
    gate = torch.tensor([[inf, -inf, nan, inf, 3e38, -3e38, 1.0, 1.0, 0.0]], device="cuda")
    x = torch.tensor([[1.0, 1.0, 1.0, -2.0, 0.5, 1.0, inf, nan, inf]], device="cuda")
    out = torch.empty_like(x)
    B.a2sf_quantize(x, None, None, gate=gate, out=out)
    want = torch.tensor([[inf, nan, nan, -inf, 1.5e38, -0.0, inf, nan, nan]], device="cuda")
    assert torch.allclose(out, want, rtol=1e-6, equal_nan=True)


@pytest.mark.parametrize("n,k", [(1, 1), (128, 128), (129, 127), (300, 513), (77, 4100)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_weight_is_exact(n, k, dtype):
    g = rng(4, n, k)
    w = on_gpu(g.normal(size=(n, k)) * 2.0 ** g.integers(-8, 3, size=(n, 1)), DT[dtype], stride=k + 2)
    q, s = eight(n, k, scale_rows=-(-n // 128))
    B.a2sf_quantize_weight(w, q, s)
    wq, ws = L.quantize(host(w), 128)
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(q.cpu().numpy(), wq)
    check_marks(q, s)


# ---- products ---------------------------------------------------------------------------------------------------------------

def filled(rows, cols, codes, scales, pad):
    """8-bit rows of these bytes; the bytes behind them are NaN."""
    q = torch.full((rows, up(cols, 16) + pad), 0x7F, dtype=torch.uint8, device="cuda")
    q[:, :cols] = torch.from_numpy(codes).cuda()
    s = torch.full((scales.shape[0], up(scales.shape[1], 4)), 0xFF, dtype=torch.uint8, device="cuda")
    s[:, : scales.shape[1]] = torch.from_numpy(scales).cuda()
    return q[:, :cols], s[:, : scales.shape[1]]


def operands(g, m, n, k, whole):
    """Bytes and scales of A and B.  whole: small whole numbers and scales that leave every sum exact in 32 bits."""
    nb = -(-k // 128)
    if whole:
        codes = np.array([L.to_e4m3(np.array([float(v)]))[0] for v in range(-4, 5)], np.uint8)
        draw = lambda r: codes[g.integers(0, 9, size=(r, k))]
        scale = lambda r: g.integers(126, 129, size=(r, nb)).astype(np.uint8)
    else:
        def draw(r):
            c = g.integers(0, 256, size=(r, k)).astype(np.uint8)
            c[(c & 0x7F) == 0x7F] = 0
            return c
        scale = lambda r: g.integers(112, 132, size=(r, nb)).astype(np.uint8)
    return (draw(m), scale(m)), (draw(n), scale(-(-n // 128)))


MATMUL = [(1, 1, 1), (1, 16, 128), (1, 257, 384), (1, 4096, 1024), (2, 100, 15), (3, 65, 200), (5, 1000, 1000), (16, 129, 129), (17, 31, 4096),
          (31, 500, 640), (33, 64, 16), (48, 4100, 512), (64, 256, 2048), (65, 640, 130), (96, 33, 5000), (100, 2000, 300), (127, 127, 127),
          (128, 128, 128), (129, 257, 256), (200, 1030, 900), (256, 512, 2304), (257, 300, 384), (300, 3001, 129), (512, 768, 1024),
          (700, 513, 77), (1000, 1111, 640), (2049, 130, 260), (4100, 300, 96), (2100, 5000, 384)]


@pytest.mark.parametrize("m,n,k", MATMUL)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("workspace", [True, False])
def test_matmul_of_whole_numbers_is_exact(m, n, k, dtype, workspace):
    g = rng(5, m, n, k)
    (a, sa), (b, sb) = operands(g, m, n, k, True)
    ta, tsa = filled(m, k, a, sa, 0)
    tb, tsb = filled(n, k, b, sb, 32)
    c = on_gpu(np.zeros((m, n)), DT[dtype], stride=n + 3, offset=1)
    c._base.fill_(99.0)
    ws = torch.full((B.a2sf_matmul_workspace_bytes(m, n, k),), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
    B.a2sf_matmul_scaled(ta, tsa, tb, tsb, c, workspace=ws)
    # sums of quarters below 2^22: exact in 64 bits as in 32
    want = torch.from_numpy(L.values(a, sa)).cuda() @ torch.from_numpy(L.values(b, sb, 128)).cuda().t()
    assert float(want.abs().max()) < 2 ** 21
    assert torch.equal(c, want.to(DT[dtype])), (c.double() - want).abs().max()
    assert bool((torch.as_strided(c._base, (m, 3), (n + 3, 1), 1 + n) == 99).all()) and float(c._base[0]) == 99


@pytest.mark.parametrize("m", [1, 15, 16, 17, 33, 48, 49, 64])
@pytest.mark.parametrize("n,k", [(4096, 127), (4097, 128), (5003, 700), (8200, 1152), (13000, 513), (21000, 2048)])
def test_matmul_of_few_rows_and_many_columns_is_exact(m, n, k):
    """Several strips of columns to a workgroup, parts of k of no, one and several steps."""
    g = rng(16, m, n, k)
    (a, sa), (b, sb) = operands(g, m, n, k, True)
    ta, tsa = filled(m, k, a, sa, 16)
    tb, tsb = filled(n, k, b, sb, 0)
    want = torch.from_numpy(L.values(a, sa)).cuda() @ torch.from_numpy(L.values(b, sb, 128)).cuda().t()
    for dtype in (torch.bfloat16, torch.float32):
        c = on_gpu(np.zeros((m, n)), dtype, stride=n + 5, offset=3)
        c._base.fill_(99.0)
        B.a2sf_matmul_scaled(ta, tsa, tb, tsb, c)
        assert torch.equal(c, want.to(dtype)), (c.double() - want).abs().max()
        assert bool((torch.as_strided(c._base, (m, 5), (n + 5, 1), 3 + n) == 99).all()) and bool((c._base[:3] == 99).all())


@pytest.mark.parametrize("m,n,k", [(65, 300, 1100), (66, 2000, 130), (97, 515, 2049), (129, 40, 4000), (200, 4100, 640), (333, 100, 3000),
                                   (513, 513, 2047), (1000, 33, 5000), (1024, 64, 1024)])
def test_matmul_of_several_parts_of_rows_is_exact(m, n, k):
    test_matmul_of_whole_numbers_is_exact(m, n, k, "bf16", False)
    test_matmul_of_whole_numbers_is_exact(m, n, k, "f32", True)


# (m, n) whose tiles are of 64 x 64, 64 x 128, 128 x 128 and 256 x 256 (fp32: 128 x 128) where k is that short
@pytest.mark.parametrize("m,n", [(1100, 128), (1100, 1000), (64, 32000), (2000, 2000), (4096, 4096)])
@pytest.mark.parametrize("k", [1, 15, 16, 32, 48, 63, 65, 127])
def test_matmul_of_less_than_a_block_of_k_is_exact(m, n, k):
    """The first half block is the last one, and its end is filled with zeros (several tiles to a workgroup too)."""
    g = rng(21, m, n, k)
    (a, sa), (b, sb) = operands(g, m, n, k, True)
    ta, tsa = filled(m, k, a, sa, 0)
    tb, tsb = filled(n, k, b, sb, 16)
    want = torch.from_numpy(L.values(a, sa)).cuda() @ torch.from_numpy(L.values(b, sb, 128)).cuda().t()
    for dtype in (torch.bfloat16, torch.float32):
        c = torch.full((m, n), 99.0, dtype=dtype, device="cuda")
        B.a2sf_matmul_scaled(ta, tsa, tb, tsb, c)
        assert torch.equal(c, want.to(dtype)), (c.double() - want).abs().max()


@pytest.mark.parametrize("m,n,k", [(1, 300, 1000), (7, 777, 4096), (40, 200, 333), (150, 700, 2000), (300, 300, 8000), (1030, 600, 500)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matmul(m, n, k, dtype):
    g = rng(6, m, n, k)
    (a, sa), (b, sb) = operands(g, m, n, k, False)
    ta, tsa = filled(m, k, a, sa, 16)
    tb, tsb = filled(n, k, b, sb, 0)
    c = torch.empty(m, n, dtype=DT[dtype], device="cuda")
    ws = torch.empty(B.a2sf_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device="cuda")
    B.a2sf_matmul_scaled(ta, tsa, tb, tsb, c, workspace=ws)
    va, vb = torch.from_numpy(L.values(a, sa)).cuda(), torch.from_numpy(L.values(b, sb, 128)).cuda().t()
    want = va @ vb
    bound = (max(k, 16) * 2.0 ** -24 + (8 * 2.0 ** -13 if dtype == "bf16" else 0)) * (va.abs() @ vb.abs())
    bound += BF16 * want.abs() if dtype == "bf16" else 0
    assert bool(((c.double() - want).abs() <= bound).all())
    again = torch.empty_like(c)
    B.a2sf_matmul_scaled(ta, tsa, tb, tsb, again, workspace=ws)
    assert torch.equal(c, again)


@pytest.mark.parametrize("m,n,k", [(1, 300, 1000), (7, 777, 4096), (20, 5003, 640), (40, 200, 333), (60, 4200, 513), (150, 700, 2000), (300, 300, 8000),
                                   (700, 1500, 640), (1030, 600, 500), (2100, 2000, 384)])
@pytest.mark.parametrize("workspace", [True, False])
def test_matmul_with_wide_sums(m, n, k, workspace):
    """A bf16 C whose sums are fp32's: the fp32 C, rounded once."""
    g = rng(24, m, n, k)
    (a, sa), (b, sb) = operands(g, m, n, k, False)
    ta, tsa = filled(m, k, a, sa, 16)
    tb, tsb = filled(n, k, b, sb, 0)
    c = on_gpu(np.zeros((m, n)), torch.bfloat16, stride=n + 3, offset=1)
    f = torch.empty(m, n, device="cuda")
    ws = torch.empty(B.a2sf_matmul_workspace_bytes(m, n, k), dtype=torch.uint8, device="cuda") if workspace else None
    B.a2sf_matmul_scaled(ta, tsa, tb, tsb, c, workspace=ws, wide_sums=True)
    B.a2sf_matmul_scaled(ta, tsa, tb, tsb, f, workspace=ws)
    assert torch.equal(c, f.bfloat16())
    va, vb = torch.from_numpy(L.values(a, sa)).cuda(), torch.from_numpy(L.values(b, sb, 128)).cuda().t()
    want = va @ vb
    assert bool(((c.double() - want).abs() <= max(k, 16) * 2.0 ** -24 * (va.abs() @ vb.abs()) + BF16 * want.abs()).all())


@pytest.mark.parametrize("m", [1, 17, 40, 64, 130, 700, 2100])
def test_matmul_wide_sums_keep_what_cancels(m):
    """Products of 2^8 and -2^8 with seven of 2^-6 beside each: 7 * 2^-5 is left, exactly."""
    n, k = 1100, 512
    a, b = np.zeros((m, k)), np.ones((n, k))
    a[:, :8], a[:, 64:72] = 2.0 ** -6, 2.0 ** -6
    a[:, 3], a[:, 68] = 256.0, -256.0
    ones = lambda r: np.full((r, 4), 127, np.uint8)
    c = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    B.a2sf_matmul_scaled(*filled(m, k, L.to_e4m3(a), ones(m), 0), *filled(n, k, L.to_e4m3(b), ones(9), 0), c, wide_sums=True)
    assert bool((c == 14 * 2.0 ** -6).all())


@pytest.mark.parametrize("m,n,k", [(3, 100, 256), (40, 4200, 384), (200, 300, 1000), (2100, 600, 640)])
@pytest.mark.parametrize("of_a,of_b", [((10, 13), (220, 240)), ((241, 247), (10, 14)), ((10, 14), (241, 247)), ((60, 80), (120, 180))])
def test_matmul_in_32_bits_at_the_ends_of_the_scales(m, n, k, of_a, of_b):
    """All 8-bit values under scale bytes from 10 to 246."""
    g = rng(28, m, of_a[0])
    (a, sa), (b, sb) = operands(g, m, n, k, False)
    sa, sb = (g.integers(*r, size=s.shape).astype(np.uint8) for r, s in ((of_a, sa), (of_b, sb)))
    c = torch.empty(m, n, device="cuda")
    B.a2sf_matmul_scaled(*filled(m, k, a, sa, 0), *filled(n, k, b, sb, 0), c)
    va, vb = torch.from_numpy(L.values(a, sa)).cuda(), torch.from_numpy(L.values(b, sb, 128)).cuda().t()
    assert bool(((c.double() - va @ vb).abs() <= max(k, 16) * 2.0 ** -24 * (va.abs() @ vb.abs())).all())


@pytest.mark.parametrize("m,n,k,parts", [(300, 1000, 11008, 4), (500, 2048, 8192, 2)])
def test_matmul_takes_a_workspace_that_its_own_parts_fit(m, n, k, parts):
    """32-bit sums would be split in more parts than the 8-bit instruction's: a workspace for the fewer is enough for those."""
    g = rng(27, m, n, k)
    (a, sa), (b, sb) = operands(g, m, n, k, False)
    args = (*filled(m, k, a, sa, 16), *filled(n, k, b, sb, 0))

    def product(size):
        c = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
        B.a2sf_matmul_scaled(*args, c, workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if size else None)
        return c

    own = parts * m * n * 4
    whole = B.a2sf_matmul_workspace_bytes(m, n, k)
    assert own < whole
    with_parts, without = product(whole), product(0)
    assert not torch.equal(with_parts, without)
    assert torch.equal(product(own), with_parts) and torch.equal(product(own - 16), without)


@pytest.mark.parametrize("m", [1, 20, 200, 600])
def test_matmul_scales_that_are_no_numbers_reach_their_rows_only(m):
    g = rng(7, m)
    n, k = 300, 640
    (a, sa), (b, sb) = operands(g, m, n, k, True)
    sa[m // 2, 2] = 255
    a[m // 3, 100] = 0x7F
    sb[1, 4] = 255
    c = torch.empty(m, n, device="cuda")
    B.a2sf_matmul_scaled(*filled(m, k, a, sa, 0), *filled(n, k, b, sb, 0), c)
    want = np.zeros((m, n), bool)
    want[[m // 2, m // 3]] = True
    want[:, 128:256] = True
    assert np.array_equal(torch.isnan(c).cpu().numpy(), want)


def test_matmul_of_what_the_norm_and_the_weights_give():
    g = rng(8)
    m, n, k = 50, 384, 1000
    x, w = on_gpu(g.normal(size=(m, k)), torch.bfloat16), on_gpu(g.normal(size=(n, k)) * 0.05, torch.bfloat16)
    a, b = eight(m, k), eight(n, k, scale_rows=3)
    B.a2sf_rms_norm(x, torch.ones(k, dtype=torch.bfloat16, device="cuda"), 1e-5, q=a[0], scales=a[1])
    B.a2sf_quantize_weight(w, *b)
    c = torch.empty(m, n, device="cuda")
    B.a2sf_matmul_scaled(*a, *b, c)
    y = L.rms_norm(host(x), None, np.ones(k), 1e-5)[1]
    # a value keeps 2^-4 at worst, 2^-5.2 on the average of squares; a thousand independent errors
    want = y @ host(w).T
    assert np.linalg.norm(host(c) - want) < 0.05 * np.linalg.norm(want)


# ---- rotary -------------------------------------------------------------------------------------------------------------------

ROTARY = [(1, 1, 1, 1, 64, 64), (2, 1, 32, 8, 128, 128), (1, 7, 3, 1, 128, 32), (3, 5, 4, 2, 64, 24), (2, 9, 2, 1, 96, 96), (1, 300, 5, 5, 128, 128),
          (4, 3, 40, 40, 128, 64), (2, 4, 2, 2, 10, 6), (1, 5, 1, 1, 7, 2), (1, 2, 2, 1, 512, 512), (2, 3, 3, 1, 511, 510), (70, 1, 2, 2, 64, 64)]


@pytest.mark.parametrize("batch,length,heads,kv,d,rot", ROTARY)
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_splits_a_product(batch, length, heads, kv, d, rot, neighbours, dtype):
    g = rng(9, batch, length, heads, d, rot)
    dt = DT[dtype]
    all_heads = heads + 2 * kv
    x = on_gpu(g.normal(size=(batch * length, all_heads * d)), dt, stride=all_heads * d + 6)
    x = x.unflatten(0, (batch, length)).unflatten(2, (all_heads, d))
    pos = torch.from_numpy(g.integers(0, 500, size=(batch, length)).astype(np.int32)).cuda()
    table = torch.empty(500, rot, device="cuda")
    B.a2sf_rotary_table(table)
    parts = x.split([heads, kv, kv], 2)
    outs = [torch.full((batch, h, length, d), 3.0, dtype=dt, device="cuda") for h in (heads, kv, kv)]
    call = [(p, o.transpose(1, 2), i < 2) for i, (p, o) in enumerate(zip(parts, outs))]
    t = host(table)[pos.cpu().numpy()][:, :, None]
    for inverse in (False, True):
        B.a2sf_rotary(call, pos, table, interleaved=neighbours, inverse=inverse)
        for i, (p, o) in enumerate(zip(parts, outs)):
            v = host(p)
            want = L.rotate(v, t[..., : rot // 2], t[..., rot // 2:], rot, neighbours, inverse) if i < 2 else v
            # a pair's sum of two products: 3 u of the pair's size
            a, b = (slice(0, rot, 2), slice(1, rot, 2)) if neighbours else (slice(0, rot // 2), slice(rot // 2, rot))
            size = np.zeros(v.shape)
            if i < 2:
                size[..., a] = size[..., b] = np.abs(v[..., a]) + np.abs(v[..., b])
            bound = 3 * 2.0 ** -24 * size + (BF16 * np.abs(want) if dtype == "bf16" else 0)
            assert (np.abs(host(o.transpose(1, 2)) - want) <= bound).all()
    # in place: the same bits
    before = [o.clone() for o in outs]
    y = x.clone()
    ys = y.split([heads, kv, kv], 2)
    B.a2sf_rotary([(p, p, i < 2) for i, p in enumerate(ys)], pos, table, interleaved=neighbours, inverse=True)
    for p, o in zip(ys, before):
        assert torch.equal(p, o.transpose(1, 2))


@pytest.mark.parametrize("rot", [2, 6, 14, 16, 18, 26, 38, 60, 100, 112, 118, 122, 126])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_parts_of_any_size(rot, neighbours, dtype):
    """Against the oracle; and in place, where items keep to their own elements, the same bits."""
    test_rotary_splits_a_product(2, 5, 6, 3, 128, rot, neighbours, dtype)
    g = rng(20, rot)
    x = on_gpu(g.normal(size=(60, 128)), DT[dtype]).view(3, 4, 5, 128)
    y, table = torch.empty_like(x), torch.empty(90, rot, device="cuda")
    B.a2sf_rotary_table(table)
    pos = torch.from_numpy(g.integers(0, 90, size=(3, 4)).astype(np.int32)).cuda()
    B.a2sf_rotary([(x, y)], pos, table, interleaved=neighbours)
    B.a2sf_rotary([(x, x)], pos, table, interleaved=neighbours)
    assert torch.equal(x, y)


def test_rotary_there_and_back():
    x = torch.randn(2, 50, 3, 128, device="cuda")
    pos = torch.arange(100, dtype=torch.int32, device="cuda").view(2, 50) * 1000
    table = torch.empty(100000, 128, device="cuda")
    B.a2sf_rotary_table(table)
    y, z = torch.empty_like(x), torch.empty_like(x)
    B.a2sf_rotary([(x, y)], pos, table)
    B.a2sf_rotary([(y, z)], pos, table, inverse=True)
    # the table's cosine and sine are rounded: their squares add up to 1 within 2 u; the two turns add 6 u of a pair's size
    assert float((z - x).abs().max()) <= 10 * 2.0 ** -24 * 2 * float(x.abs().max())


def test_rotary_is_its_gradient_by_differences():
    """d (g . turn(x)) / dx = turn back (g): the turn is linear, so the difference quotient is exact up to rounding."""
    g = rng(10)
    x, d = (torch.from_numpy(g.normal(size=(1, 6, 2, 64))).float().cuda() for _ in range(2))
    up_ = torch.from_numpy(g.normal(size=(1, 6, 2, 64))).float().cuda()
    pos = torch.arange(6, dtype=torch.int32, device="cuda")[None]
    table = torch.empty(6, 64, device="cuda")
    B.a2sf_rotary_table(table)
    turn = lambda v, inverse=False: (lambda y: (B.a2sf_rotary([(v, y)], pos, table, inverse=inverse), y)[1])(torch.empty_like(v))
    quotient = (up_.double() * (turn(x + d).double() - turn(x).double())).sum()
    gradient = (turn(up_, True).double() * d.double()).sum()
    scale = float((up_.abs().double() * (x.abs() + d.abs()).double()).sum())
    assert abs(float(quotient - gradient)) <= 12 * 2.0 ** -24 * scale


def test_rotary_positions_outside_the_table_are_not_numbers():
    x = torch.randn(1, 4, 2, 64, device="cuda")
    pos = torch.tensor([[0, 9, -1, 10]], dtype=torch.int32, device="cuda")
    table = torch.empty(10, 32, device="cuda")
    B.a2sf_rotary_table(table)
    y, v = torch.empty_like(x), torch.empty_like(x)
    B.a2sf_rotary([(x, y), (x, v, False)], pos, table)
    bad = torch.isnan(y)
    assert bool(bad[0, 2:, :, :32].all()) and not bool(bad[0, :2].any()) and torch.equal(y[..., 32:], x[..., 32:])
    assert torch.equal(v, x)


@pytest.mark.parametrize("args", [dict(), dict(base=500000.0, factor=8.0, original_length=8192, low=1.0, high=4.0),
                                  dict(factor=4.0, magnitude=1.1386), dict(factor=2.0, original_length=2048, low=1.0, high=32.0)])
def test_rotary_table(args):
    table = torch.empty(200000, 96, device="cuda")
    B.a2sf_rotary_table(table, **args)
    at = np.array([0, 1, 2, 77, 4096, 65535, 131071, 199999])
    m = args.get("magnitude", 1.0)
    f = L.frequencies(96, args.get("base", 10000.0), args.get("factor", 1.0), args.get("original_length", 0), args.get("low", 0.0),
                      args.get("high", 0.0))
    angle = at[:, None] * f
    got = host(table)[at]
    # one rounding of values up to m; the angle in 64 bits is off by 2e5 * 2^-52 at most
    assert np.abs(got - m * np.concatenate([np.cos(angle), np.sin(angle)], 1)).max() <= m * 2.0 ** -24 * 1.01


# ---- sampling ------------------------------------------------------------------------------------------------------------------

def draw_tokens(logits, noise, **filters):
    rows, n = logits.shape
    token = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((rows,), -7.0, device="cuda")
    on = {k: (None if v is None else torch.from_numpy(np.asarray(v)).cuda().to(torch.int32 if k == "top_k" else torch.float32))
          for k, v in filters.items()}
    B.a2sf_sample(logits, noise, token, prob=prob, **on)
    return token.cpu().numpy(), prob.double().cpu().numpy()


def check_tokens(logits, noise, **filters):
    got = draw_tokens(logits, noise, **filters)
    l, e = host(logits), host(noise) if noise is not None else None
    for r in range(l.shape[0]):
        one = {k: float(np.float32(v[r])) if k != "top_k" else int(v[r]) for k, v in filters.items() if v is not None}
        token, prob = L.sample(l[r], e[r] if e is not None else None, **one)
        assert got[0][r] == token, (r, one)
        # the weights' exponents are off by 2 u of their size (under 150 octaves), the sum by its chains of additions
        assert abs(got[1][r] - prob) <= 3e-5 * prob, (r, one)


VOCABULARY = [1, 2, 63, 200, 1024, 5000, 8192, 8193, 20001, 32000, 50272, 65536, 70001, 128256]


@pytest.mark.parametrize("n", VOCABULARY)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("filters", ["", "t", "k", "p", "m", "tkpm", "kp"])
def test_sample(n, dtype, filters):
    rows = 5
    g = rng(11, n, len(filters))
    l = 2 * g.normal(size=(rows, n)) + (g.random((rows, n)) < 30 / n) * (5 + 3 * g.random((rows, n)))
    logits = on_gpu(l, DT[dtype], stride=n + 3, offset=1)
    noise = on_gpu(g.exponential(size=(rows, n)) + 1e-9, torch.float32, stride=n + 1)
    f = {}
    if "t" in filters:
        f["temperature"] = [0.3, 0.0, 1.0, 1.7, 0.01]
    if "k" in filters:
        f["top_k"] = [1, 40, 0, 100000, 700]
    if "p" in filters:
        f["top_p"] = [0.9, 0.5, 1.0, 0.0, 0.999]
    if "m" in filters:
        f["min_p"] = [0.05, 0.0, 2.0, 0.3, 1e-4]
    check_tokens(logits, noise, **f)


@pytest.mark.parametrize("n", [300, 5000, 70001])
def test_sample_equal_logits_go_by_index(n):
    """All tokens in one bin, more of them than are ranked at once, or a few values with many ties."""
    g = rng(12, n)
    flat = torch.zeros(4, n, device="cuda")
    noise = on_gpu(g.exponential(size=(4, n)) + 1e-9, torch.float32)
    check_tokens(flat, noise, top_k=[1, 7, n // 2, n - 1])
    check_tokens(flat, noise, top_p=[0.1, 0.5, 0.9, 0.01])
    steps = on_gpu(np.round(2 * g.normal(size=(4, n))) / 2, torch.bfloat16)
    check_tokens(steps, noise, top_k=[3, 100, 150, n // 3], top_p=[0.5, 0.9, 1.0, 0.7], temperature=[1.0, 0.5, 2.0, 1.0])


def test_sample_values_close_together():
    """Thousands of different logits in one bin of the first histogram: it is split by their bits."""
    g = rng(13)
    logits = on_gpu(1.0 + g.random((3, 9000)) * 1e-3, torch.float32)
    noise = on_gpu(g.exponential(size=(3, 9000)) + 1e-9, torch.float32)
    check_tokens(logits, noise, top_k=[4000, 8999, 1500])
    check_tokens(logits, noise, top_p=[0.3, 0.77, 0.5], top_k=[0, 5000, 2])


@pytest.mark.parametrize("filters", [dict(top_k=[512] * 48), dict(top_p=[0.9] * 48), dict(min_p=[0.5] * 48),
                                     dict(top_k=[3000] * 48, top_p=[0.9] * 48)])
def test_sample_equal_weights_go_to_the_lowest_index(filters):
    """Without random numbers the first of the largest logits, wherever the others stand."""
    g = rng(17)
    l = np.where(g.random((48, 8192)) < 0.5, 1.5, g.normal(size=(48, 8192)) - 5)
    l[g.random(l.shape) < 0.05] = 2.0
    check_tokens(on_gpu(l, torch.bfloat16), None, **filters)


@pytest.mark.parametrize("p", [0.5, 0.9, 0.99, 0.9999, 0.9999999])
def test_sample_long_and_short_cuts(p):
    """A few tokens with nearly all of the mass, a few thousand, nearly all of the row."""
    g = rng(18)
    n = 40000
    l = g.normal(size=(6, n)) * np.array([0.01, 0.5, 1.0, 2.0, 4.0, 12.0])[:, None]
    noise = on_gpu(g.exponential(size=(6, n)) + 1e-9, torch.float32)
    for dtype in (torch.float32, torch.bfloat16):
        check_tokens(on_gpu(l, dtype), noise, top_p=[p] * 6)
        check_tokens(on_gpu(l, dtype), noise, top_p=[p] * 6, min_p=[0.01] * 6)
        check_tokens(on_gpu(l, dtype), noise, top_p=[p] * 6, top_k=[600, 5000, 8000, 9000, 20000, 39999])


def test_sample_infinities_and_nan():
    inf, nan = math.inf, math.nan
    rows = [[-inf, nan, -inf, nan], [inf, 1.0, inf, 2.0], [nan, -inf, 3.0, -inf], [-inf, 0.0, 1.0, nan], [nan, inf, nan, -1.0],
            [-3e38, 3e38, 3e38, -3e38]]
    logits = torch.tensor(rows, device="cuda")
    noise = torch.tensor([[1.0, 2.0, 0.5, 3.0]] * 6, device="cuda")
    for f in ({}, {"top_k": [3] * 6}, {"top_p": [0.99] * 6}, {"top_k": [3] * 6, "top_p": [0.5] * 6, "min_p": [0.2] * 6},
              {"temperature": [0.0] * 6}, {"temperature": [1e-38] * 6}):
        check_tokens(logits, noise, **f)
    check_tokens(logits, None, top_k=[2] * 6)


@pytest.mark.parametrize("octaves", [20.0, 30.0, 31.9, 32.1, 33.0, 36.0])
def test_sample_long_tails_have_their_mass(octaves):
    """One token and 150 000 that many octaves below it: a share p of the whole is reached so far along the tail.  Without random numbers the
    first token is drawn, and its probability says how much was left (a sum in 32 bits)."""
    n = 150000
    l = np.full((1, n), -octaves * math.log(2.0), np.float32)
    l[0, 70000] = 0.0
    w = float(np.exp(float(l[0, 0])))
    logits, total = torch.from_numpy(l).cuda(), 1 + (n - 1) * w
    for share in (0.0, 0.25, 0.5, 0.9, 1.0):    # of the tail
        p = float(np.float32((1 + share * (n - 1) * w) / total))
        if p >= 1:
            continue
        token, prob = draw_tokens(logits, None, top_p=[p])
        kept = min(max(p * total, 1.0), total)
        # what is left is p of the whole and not more than one token of the tail beyond it.  Roundings: a mass 2^-42 and the exponent of its weight
        # 2^-18 of it; of the sum the 150 tokens beside the first in its lane and ten additions across the lanes, the quotient, its inverse
        assert token[0] == 70000
        assert abs(1 / prob[0] - kept) <= 151 * w + 14 * 2.0 ** -24 + (n - 1) * (w * 2.0 ** -18 + 2.0 ** -42)


def test_sample_deep_tails_are_in_reach_of_top_p():
    """Half of the mass of a tail 32.5 octaves down: its tokens can be drawn, and the last ones cannot."""
    n, octaves = 150000, 32.5
    l = np.full((1, n), -octaves * math.log(2.0), np.float32)
    l[0, 0] = 0.0
    w = math.exp(float(l[0, 1]))
    whole = 1 + (n - 1) * w
    p = np.float32(1 - 0.5 * (n - 1) * w / whole)
    assert p < 1
    last = int(math.ceil((float(p) * whole - 1) / w))   # tokens 0 .. last are left, give or take the rounding of a mass: 2^-42 of 2^-32.5
    for at, drawn in ((1, True), (last // 2, True), (last - last // 500, True), (last + last // 500, False), (n - 1, False)):
        noise = torch.ones(1, n, device="cuda")
        noise[0, at] = 1e-30
        token, _ = draw_tokens(torch.from_numpy(l).cuda(), noise, top_p=[float(p)])
        assert (token[0] == at) == drawn, (at, last, token)


@pytest.mark.parametrize("n", [1, 5, 100, 511, 1000, 5003])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_min_p_that_keeps_every_token(n, dtype):
    """Shares and temperatures that put the last logit kept at -infinity: what is kept ends with the row all the same, also where the
    next row's logits are larger."""
    g = rng(22, n)
    l = g.normal(size=(6, n)) + 3 * np.arange(6)[:, None]
    l[:, n // 2:][g.random((6, n - n // 2)) < 0.2] = -math.inf
    l[:, 0] = 0.0
    logits, noise = on_gpu(l, DT[dtype]), on_gpu(g.exponential(size=(6, n)) + 1e-9, torch.float32)
    check_tokens(logits, noise, min_p=[1e-40, 1e-38, 1e-30, 1e-45, 1e-20, 1e-40])
    check_tokens(logits, noise, min_p=[1e-40, 0.5, 1e-30, 0.1, 1e-6, 1.0], temperature=[1e38, math.inf, 1e38, 3e38, math.inf, math.inf])


@pytest.mark.parametrize("live,nans", [(1000, 1000), (600, 1400), (599, 50), (800, 3000), (2000, 2000), (30, 5000)])
@pytest.mark.parametrize("values", ["different", "few", "one and ties", "close"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_long_rows_with_nan(live, nans, values, dtype):
    """NaN and -infinity among the logits count for nothing, whatever way the cut is found: k below and above the number of finite
    ones, and below and above that of all but the -infinities."""
    g = rng(23, live, nans, len(values))
    n = live + nans + 500
    l = np.full((7, n), -math.inf)
    for r in range(7):
        at = g.permutation(n)
        l[r, at[:live]] = {"different": g.normal(size=live) * 3, "few": np.round(g.normal(size=live)), "close": 1 + 1e-3 * g.random(live),
                           "one and ties": np.where(np.arange(live) < 10, 5 + 0.1 * np.arange(live), 1.0)}[values]
        l[r, at[live: live + nans]] = math.nan
    logits = on_gpu(l, DT[dtype])
    noise = on_gpu(g.exponential(size=(7, n)) + 1e-9, torch.float32)
    k = [513, min(live + 1, n - 1), live + nans // 2, live + nans, n - 1, 100, max(1, live - 1)]
    check_tokens(logits, noise, top_k=k)
    check_tokens(logits, None, top_k=k)
    check_tokens(logits, noise, top_k=k, top_p=[0.5, 0.9, 0.99, 0.999, 0.3, 0.9, 0.7])
    check_tokens(logits, noise, top_p=[0.5, 0.9, 0.99, 0.999, 0.3, 0.9, 0.7], min_p=[0.0, 0.1, 0.0, 0.5, 0.0, 0.0, 0.01])
    check_tokens(logits, noise, top_k=k, temperature=[math.inf, 1e30, 100.0, 0.01, 1e-30, math.inf, 1.0])
    check_tokens(logits, noise, min_p=[0.5, 1e-40, 0.01, 0.1, 1.0, 1e-9, 0.3], temperature=[math.inf, 1.0, 100.0, 0.01, 1e-30, math.inf, 1.0])


@pytest.mark.parametrize("n", [1, 2, 700, 9000])
def test_sample_min_p_above_one_leaves_the_first_alone(n):
    """Equal logits too stand behind it."""
    g = rng(29, n)
    l = np.where(g.random((5, n)) < 0.3, 2.0, g.normal(size=(5, n)) - 3)
    l[:, n // 2] = 2.0
    noise = on_gpu(g.exponential(size=(5, n)) + 1e-9, torch.float32)
    check_tokens(on_gpu(l, torch.bfloat16), noise, min_p=[1.5, 2.0, 1.0, 3e38, math.inf])
    check_tokens(on_gpu(l, torch.float32), noise, min_p=[1.5, 2.0, 1.0, 1e10, math.inf], top_p=[0.9] * 5, top_k=[0, 5, 3, 600, 1])


def test_sample_without_prob_and_with_numbers_that_are_zero():
    logits = torch.zeros(1, 10, device="cuda")
    noise = torch.ones(1, 10, device="cuda")
    noise[0, 6] = 0.0
    token = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.a2sf_sample(logits, noise, token)
    assert token.tolist() == [6]


def test_sample_frequencies():
    """20 000 draws of one distribution: each token about as often as it is likely (five standard deviations)."""
    g = rng(14)
    n, draws = 37, 20000
    l = g.normal(size=n)
    logits = torch.from_numpy(np.repeat(l[None], draws, 0)).float().cuda()
    noise = torch.empty(draws, n, device="cuda").exponential_(generator=torch.Generator("cuda").manual_seed(3))
    token = torch.empty(draws, dtype=torch.int32, device="cuda")
    B.a2sf_sample(logits, noise, token)
    p = np.exp(l) / np.exp(l).sum()
    share = np.bincount(token.cpu().numpy(), minlength=n) / draws
    assert (np.abs(share - p) <= 5 * np.sqrt(p * (1 - p) / draws)).all()


# ---- streams, graphs, host paths ---------------------------------------------------------------------------------------------

def layer_calls(m=6, k=640, n=384):
    """One of each call on small data; returns (function that makes them, the tensors they write)."""
    g = rng(15)
    x, w = on_gpu(g.normal(size=(m, k)), torch.bfloat16), on_gpu(1 + 0.1 * g.normal(size=(1, k)), torch.bfloat16)[0]
    weight = on_gpu(g.normal(size=(n, k)) * 0.1, torch.bfloat16)
    a, b, h = eight(m, k), eight(n, k, scale_rows=3), eight(m, n)
    c = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    table, pos = torch.empty(64, 64, device="cuda"), torch.arange(m, dtype=torch.int32, device="cuda")[None]
    y = torch.zeros(1, 6, m, 64, dtype=torch.bfloat16, device="cuda")
    logits = on_gpu(3 * g.normal(size=(m, 2000)), torch.float32)
    noise = on_gpu(g.exponential(size=(m, 2000)) + 1e-9, torch.float32)
    token, prob = torch.zeros(m, dtype=torch.int32, device="cuda"), torch.zeros(m, device="cuda")
    p = torch.full((m,), 0.9, device="cuda")
    B.a2sf_rotary_table(table)
    B.a2sf_quantize_weight(weight, *b)
    ws = torch.empty(max(1, B.a2sf_matmul_workspace_bytes(m, n, k)), dtype=torch.uint8, device="cuda")

    def calls(stream=None):
        B.a2sf_rms_norm(x, w, 1e-5, q=a[0], scales=a[1], stream=stream)
        B.a2sf_matmul_scaled(*a, *b, c, workspace=ws, stream=stream)
        B.a2sf_rotary([(c.view(1, m, 6, 64), y.transpose(1, 2))], pos, table, stream=stream)
        B.a2sf_quantize(c, *h, gate=c, stream=stream)
        B.a2sf_sample(logits, noise, token, top_p=p, prob=prob, stream=stream)

    return calls, [*a, c, y, *h, token, prob]


def test_calls_replay_from_a_hip_graph():
    calls, outs = layer_calls()
    calls()
    torch.cuda.synchronize()
    eager = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(4):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, e) for t, e in zip(outs, eager))


def test_calls_on_another_stream_and_through_ctypes(monkeypatch):
    calls, outs = layer_calls()
    calls()
    torch.cuda.synchronize()
    eager = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    for way in ("current", "named", "ctypes"):
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        if way == "current":
            with torch.cuda.stream(side):
                calls()
        elif way == "named":
            calls(side.cuda_stream)
        else:
            monkeypatch.setattr(B, "_call", B._NoExtension)
            calls()
        torch.cuda.synchronize()
        assert all(torch.equal(t, e) for t, e in zip(outs, eager)), way


def test_tensors_of_the_host_are_refused_and_pinned_ones_taken():
    logits = torch.randn(4, 50, device="cuda")
    token, k = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.tensor([1, 2, 3, 4], dtype=torch.int32)
    for at in (dict(top_k=k), dict(top_p=torch.ones(4)), dict(prob=torch.ones(4))):
        with pytest.raises(B.A2SFError) as e:
            B.a2sf_sample(logits, None, token, **at)
        assert e.value.status == B.A2SF_EINVAL
    for args in ((logits.cpu(), None, token), (logits.cpu(), None, token.cpu()), (logits, None, token.cpu()), (logits, logits.cpu(), token)):
        with pytest.raises(B.A2SFError) as e:
            B.a2sf_sample(*args)
        assert e.value.status == B.A2SF_EINVAL
    x, w = torch.randn(3, 256, device="cuda"), torch.ones(256)
    with pytest.raises(B.A2SFError):
        B.a2sf_rms_norm(x, w, 1e-5, out=torch.empty_like(x))
    with pytest.raises(B.A2SFError):
        B.a2sf_rotary_table(torch.empty(8, 64))
    out = torch.empty(4, dtype=torch.int32, pin_memory=True)
    B.a2sf_sample(logits, None, out, top_k=k.pin_memory())
    torch.cuda.synchronize()
    assert torch.equal(out, logits.argmax(1).int().cpu())
