"""The product of block-scaled matrices at the ends of its scales' range: the least and
the largest scale on either side, sums that leave fp32 at both ends, blocks far apart
within a row, NaN scales and NaN codes, and E4M3 rows with uneven columns."""
import numpy as np
import pytest

import paper_2608_11249_amd as dl
from gpu_common import log, shape

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
MAX = float(torch.finfo(torch.float32).max)
E2M1 = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
E4M3 = torch.tensor([(-1 if c & 128 else 1) * ((c & 7) * 2.0 ** -9 if c & 0x78 == 0 else
                                               (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10)) for c in range(256)],
                    dtype=torch.float64)
E4M3[[0x7F, 0xFF]] = float("nan")


@pytest.fixture(scope="module")
def m():
    with dl.Model(shape(vocab=256, n_layers=0), max_chunk=1) as model:
        yield model


def codes_of(fmt, rows, cols, seed, positive=False):
    g = torch.Generator().manual_seed(seed)
    if fmt == "fp4":
        return torch.randint(0, 8 if positive else 16, (rows, cols), generator=g)
    c = torch.randint(0, 0x7F, (rows, cols), generator=g)
    return c if positive else c | torch.randint(0, 2, (rows, cols), generator=g) << 7


def matrix(fmt, codes, scales):
    """codes [rows, cols] with scale bytes [rows, blocks]: (MXMatrix, values in 64 bits
    without the scales)."""
    rows, cols = codes.shape
    q = dl.MXMatrix.empty(fmt, rows, cols, "cuda")
    q.codes.zero_()
    q.scales.fill_(127)
    if fmt == "fp4":
        c = torch.nn.functional.pad(codes, (0, cols % 2))
        q.codes[:, : c.shape[1] // 2] = (c[:, 0::2] | c[:, 1::2] << 4).to(torch.uint8).cuda()
    else:
        q.codes[:, :cols] = codes.to(torch.uint8).cuda()
    for b in range(scales.shape[1]):
        q.scales[b // 8, :rows, b % 8] = scales[:, b].to(torch.uint8).cuda()
    return q, (E2M1 if fmt == "fp4" else E4M3)[codes].cuda()


def per_instruction(a, b):
    """Sum over 64-column steps of the largest |a| times the sum of |b|."""
    pad = lambda t: torch.nn.functional.pad(t.abs(), (0, -t.shape[1] % 64)).view(len(t), -1, 64)  # noqa: E731
    return pad(a).amax(2) @ pad(b).sum(2).t()


def tolerance(fmt, a, b):
    """Of fp32 results: each 64-column step adds to the accumulator, at most one step
    (2 U) of what the magnitudes add up to; with E4M3 it drops up to 2^-13 of its
    largest product for each product."""
    t = 2 * U * -(-a.shape[1] // 64) * (a.abs() @ b.abs().t())
    return t + 2.0 ** -13 * per_instruction(a, b) if fmt == "fp8" else t


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("M,N,K", [(5, 40, 300), (1, 64, 32), (33, 1001, 1000)])
def test_scales_from_the_least_to_the_largest(m, fmt, M, N, K):
    """Every pair of scales: results are those of scales of 1 times a power of two, with
    fp32's own range: subnormal steps below, infinities (or NaN, where partial sums
    were infinite) above."""
    ca, cb = codes_of(fmt, M, K, 1), codes_of("fp4", N, K, 2)
    blocks = -(-K // 32)
    qa, a = matrix(fmt, ca, torch.full((M, blocks), 127))
    qb, b = matrix("fp4", cb, torch.full((N, blocks), 127))
    want, size, tol = a @ b.t(), a.abs() @ b.abs().t(), tolerance(fmt, a, b)
    ends = (0, 1, 64, 120, 127, 134, 190, 253, 254)
    for sa in ends:
        for sb in ends:
            qa.scales.fill_(sa)
            qb.scales.fill_(sb)
            out = m.mx_matmul(qa, qb).double()
            p = 2.0 ** (sa + sb - 254)
            # a step of fp32's subnormal numbers for each addition
            off = tol * p + 2.0 ** -149 * -(-K // 64)
            inside = (size + tol) * p < MAX
            assert bool(((out - want * p).abs() <= off)[inside].all()), (sa, sb)
            assert not bool(torch.isfinite(out[(want.abs() - tol) * p > MAX * (1 + U)]).any()), (sa, sb)
            if sa + sb == 254:
                assert bool(inside.all()) and bool((out != 0).any())


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_sums_past_the_range_of_fp32(m, fmt):
    """Of positive products: +inf, in bf16 too; and negative ones -inf."""
    M, N, K = 9, 70, 200
    ca, cb = codes_of(fmt, M, K, 3, True), codes_of("fp4", N, K, 4, True)
    blocks = -(-K // 32)
    for sign, inf in ((0, float("inf")), (8, float("-inf"))):
        qa, a = matrix(fmt, ca, torch.full((M, blocks), 254))
        qb, b = matrix("fp4", cb | sign, torch.full((N, blocks), 254))
        assert bool(((a @ b.t()).abs() > 1).all())
        for dt in (torch.float32, torch.bfloat16):
            assert bool((m.mx_matmul(qa, qb, dt) == inf).all())


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("M,N,K", [(3, 50, 64), (40, 300, 1000), (515, 17001, 2300)])
def test_blocks_far_apart(m, fmt, M, N, K):
    """Scales of neighbouring blocks that differ by up to 2^40 on either side: a block's
    products lose nothing to another's."""
    log("far apart", fmt, M, N, K, dl.mx_tiles(fmt, M, N, K))
    g = torch.Generator().manual_seed(5)
    blocks = -(-K // 32)
    sa, sb = (torch.randint(107, 148, (n, blocks), generator=g) for n in (M, N))
    qa, a = matrix(fmt, codes_of(fmt, M, K, 6), sa)
    qb, b = matrix("fp4", codes_of("fp4", N, K, 7), sb)
    spread = lambda s, n: torch.exp2(s.double() - 127).repeat_interleave(32, 1)[:, :n].cuda()  # noqa: E731
    a, b = a * spread(sa, K), b * spread(sb, K)
    out = m.mx_matmul(qa, qb).double()
    t = 2 * U * -(-K // 64) * (a.abs() @ b.abs().t())
    if fmt == "fp8":  # 2^-13 of the largest product of the same block, not of the 64 columns
        pad = lambda x: torch.nn.functional.pad(x.abs(), (0, -K % 32)).view(len(x), -1, 32)  # noqa: E731
        t += 2.0 ** -13 * (pad(a).amax(2) @ pad(b).sum(2).t())
    assert bool(((out - a @ b.t()).abs() <= t).all())


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("M,N,K", [(4, 40, 200), (300, 33001, 700)])
def test_nan_scales_and_codes(m, fmt, M, N, K):
    blocks = -(-K // 32)
    ca, cb = codes_of(fmt, M, K, 8), codes_of("fp4", N, K, 9)
    ca[1, 32:64] = 0  # zeros under a NaN scale
    sa, sb = torch.full((M, blocks), 127), torch.full((N, blocks), 127)
    sa[1, 1] = 255
    sb[N - 2, blocks - 1] = 255
    bad = torch.zeros(M, N, dtype=torch.bool)
    bad[1], bad[:, N - 2] = True, True
    if fmt == "fp8":
        ca[2, 70], ca[3, 5] = 0x7F, 0xFF
        bad[2:4] = True
    out = m.mx_matmul(matrix(fmt, ca, sa)[0], matrix("fp4", cb, sb)[0])
    assert torch.equal(torch.isnan(out).cpu(), bad)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_from_the_least_values_that_are_quantised(m, fmt):
    """Subnormal and least normal fp32 values times values of 2^100 and more."""
    M, N, K = 6, 20, 100
    r = np.random.default_rng(4)
    x = torch.from_numpy((r.standard_normal((M, K)) * np.exp2(r.integers(-149, -120, (M, 1)))).astype(np.float32)).cuda()
    w = torch.from_numpy((r.standard_normal((N, K)) * 2.0 ** 110).astype(np.float32)).cuda()
    qa, qb = m.mx_quantize(x, fmt), m.mx_quantize(w, "fp4")
    a, b = (m.mx_dequantize(q, torch.float32).double() for q in (qa, qb))
    assert bool((a != 0).any())
    out = m.mx_matmul(qa, qb).double()
    assert bool(((out - a @ b.t()).abs() <= tolerance(fmt, a, b)).all())


@pytest.mark.parametrize("M,N,K", [(64, 500, 4096), (300, 17001, 2300)])
def test_e4m3_rows_with_uneven_columns(m, M, N, K):
    """Columns a hundred times the others', and sums that cancel.  What is dropped of a
    product lies below 2^-13 of its step's largest: 2^-13 / sqrt(3) as a root mean
    square, for 64 products 8 / sqrt(3) 2^-13 = 4.62 2^-13 of the largest, whose own
    squares add up to less than all products' do."""
    log("uneven", M, N, K)
    g = torch.Generator().manual_seed(11)
    x = torch.randn(M, K, generator=g) * torch.where(torch.rand(K, generator=g) < .01, 100.0, 1.0)
    x[:, K // 2: K // 2 * 2] = -x[:, : K // 2]
    w = torch.randn(N, K, generator=g)
    w[:, K // 2: K // 2 * 2] = w[:, : K // 2] + (torch.rand(N, K // 2, generator=g) < .05) * 0.5
    qa, qb = m.mx_quantize(x.cuda(), "fp8"), m.mx_quantize(w.cuda(), "fp4")
    a, b = (m.mx_dequantize(q, torch.float32).double() for q in (qa, qb))
    out = m.mx_matmul(qa, qb).double()
    err = (out - a @ b.t()).abs()
    assert bool((err <= tolerance("fp8", a, b)).all())
    size = (a ** 2 @ (b ** 2).t()).sqrt()  # of the products, as independent terms
    print("error of the products' root sum of squares:", float(err.norm() / size.norm()))
    assert float(err.norm()) <= 4.7 * 2.0 ** -13 * float(size.norm())
