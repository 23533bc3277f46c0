"""Block-scaled values through the public binding: quantisation and its inverse,
the norm that writes them, and the product, each against the definition in 64
bits; masks of infinities and NaN, odd sizes, strides, streams, graphs, refusals."""
import numpy as np
import pytest

import paper_2608_11249_amd as dl
from gpu_common import log, shape
from mx_common import TOP, blocks, held, scale_exp, step

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32, relative


@pytest.fixture(scope="module")
def m():
    with dl.Model(shape(vocab=256, n_layers=0), max_chunk=1) as model:
        yield model


def rng(*key):
    return np.random.default_rng(list(key))


def scales_of(q):
    """Bytes [rows, blocks] of q's scales."""
    return q.scales[:, : q.rows].permute(1, 0, 2).reshape(q.rows, -1).cpu().numpy()


def awkward(rows, cols, key):
    """Rows of many magnitudes, with blocks of zeros, ties and range borders."""
    r = rng(rows, cols, key)
    x = r.standard_normal((rows, cols)) * np.exp2(r.integers(-20, 20, (rows, 1)))
    x[:, ::7] *= 2.0 ** -6
    b = x[: rows // 2 + 1]
    b[:, : cols // 3] = r.choice([0, .25, .5, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 448, 464, -3.5, 2 ** -10],
                                 b[:, : cols // 3].shape)
    if rows > 1:
        x[1] = 0
    if rows > 2:
        x[2] *= 2.0 ** -100  # down to scales near the least
    if rows > 3:
        x[3] = x[3] * 0 + 1e-41 * r.integers(-9, 9, cols)  # subnormal
    return x.astype(np.float32)


# ---------------------------------------------------------------- quantisation
@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (5, 33), (9, 255), (8, 256), (33, 257), (70, 1000),
                                       (4, 4096), (1, 8200)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_is_the_definition(m, fmt, rows, cols, dtype):
    log("quantize", fmt, rows, cols, dtype)
    x = torch.from_numpy(awkward(rows, cols, 1)).to(getattr(torch, dtype)).cuda()
    q = m.mx_quantize(x, fmt)
    x64 = x.float().cpu().double().numpy()
    assert np.array_equal(scales_of(q)[:, : -(-cols // 32)], scale_exp(x64, fmt) + 127)
    assert np.array_equal(m.mx_dequantize(q, torch.float32).cpu().double().numpy(), held(x64, fmt))
    # columns past cols are zero in the codes
    per = 2 if fmt == "fp4" else 1
    tail = q.codes[:, -(-cols // per):].cpu().numpy() & 0x7F
    assert not tail.any()


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
def test_quantize_extremes(m, fmt):
    x = np.ones((6, 96), np.float32)
    x[0, 5], x[1, 40], x[2, 95] = np.inf, np.nan, -np.inf
    x[3] = np.finfo(np.float32).max
    x[4] = np.finfo(np.float32).tiny
    x[5, :32], x[5, 32:] = -0.0, np.finfo(np.float32).min
    q = m.mx_quantize(torch.from_numpy(x).cuda(), fmt)
    got = m.mx_dequantize(q, torch.float32).cpu().double().numpy()
    want = held(x.astype(np.float64), fmt)
    # the largest finite value rounds up past the range of fp32
    want = np.where(np.abs(want) > np.finfo(np.float32).max, np.copysign(np.inf, want), want)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[0, :32]).all() and np.isfinite(got[0, 32:]).all()
    b = m.mx_dequantize(q)
    assert torch.equal(torch.isnan(b).cpu(), torch.from_numpy(np.isnan(want)))


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantize_strided_and_unaligned_rows(m, fmt, dtype):
    base = torch.randn(20, 700, generator=torch.Generator().manual_seed(3)).to(getattr(torch, dtype)).cuda()
    for view in (base[:, 1:301], base[::3, 8:264], base[2:, 3:4], base[5:6, 7:]):
        log("strided", tuple(view.shape), view.stride())
        q = m.mx_quantize(view, fmt)
        p = m.mx_quantize(view.contiguous(), fmt)
        assert torch.equal(q.codes, p.codes)
        assert np.array_equal(scales_of(q), scales_of(p))
        assert torch.equal(m.mx_dequantize(q, view.dtype), m.mx_dequantize(p, view.dtype))


def test_dequantize_leaves_the_rest_of_a_wider_buffer(m):
    q = m.mx_quantize(torch.randn(5, 40, device="cuda"), "fp8")
    out = torch.full((7, 64), 9.0, device="cuda")
    m._on_current_stream(out.device, dl.lib().dlmc_mx_dequantize, q.codes, q.scales, 1, 5, 40, out, 0, 64)
    assert torch.equal(out[:5, :40], m.mx_dequantize(q, torch.float32))
    assert bool((out[5:] == 9).all()) and bool((out[:, 40:] == 9).all())


def test_empty(m):
    x = torch.empty(0, 48, device="cuda")
    q = m.mx_quantize(x, "fp4")
    assert q.codes.shape == (0, 128) and m.mx_dequantize(q).shape == (0, 48)
    r, q = m.add_norm_mx(x, x, fmt="fp8")
    assert r.shape == (0, 48)
    w = m.mx_quantize(torch.randn(7, 48, device="cuda"), "fp4")
    assert m.mx_matmul(q, w).shape == (0, 7)
    a = m.mx_quantize(torch.randn(7, 48, device="cuda"), "fp8")
    none = m.mx_quantize(x, "fp4")
    assert m.mx_matmul(a, none).shape == (7, 0)


# ---------------------------------------------------------------- norm
def check_norm(r, q, got, gain, kind, eps, fmt):
    """q holds norm(r) gain: scales that fit, values within half a step.

    fp32 error of y = (r - mean) gain / sqrt(...), counted in half steps U: a sum over
    a row takes at most 32 additions in a lane, 6 + 2 across lanes; squares, the
    division, the root, two products: fewer than 64 in all.  The mean's own error is
    of the size of the row's largest value."""
    r = r.astype(np.float64)
    c = r - r.mean(1, keepdims=True) if kind == "layernorm" else r
    y = c / np.sqrt((c ** 2).mean(1, keepdims=True) + eps)
    inv = 1 / np.sqrt((c ** 2).mean(1, keepdims=True) + eps)
    off = 64 * U * np.abs(y)
    if kind == "layernorm":
        off = off + 64 * U * np.abs(r).max(1, keepdims=True) * inv
    if gain is not None:
        y, off = y * gain, off * np.abs(gain) + U * np.abs(y * gain)
    s = np.exp2(scales_of(q)[:, : -(-r.shape[1] // 32)].astype(np.float64) - 127)
    big, slack = np.abs(blocks(y)).max(2), blocks(off).max(2)
    assert (big <= TOP[fmt] * s + slack).all()
    assert ((big + slack > TOP[fmt] * s / 2) | (s == 2.0 ** -127)).all()
    cols = r.shape[1]
    wide = np.repeat(s, 32, 1)[:, :cols]
    # a value next to a binade's border may be rounded with the step above it
    half = 0.5 * step((np.abs(y) + off) / wide, fmt) * wide
    assert (np.abs(got.astype(np.float64) - y) <= half + off).all()


@pytest.mark.parametrize("kind", ["rmsnorm", "layernorm"])
@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 32), (5, 77), (2, 512), (6, 513), (4, 768), (3, 1024), (3, 1025),
                                       (2, 2048), (2, 2056), (5, 4096), (2, 4099), (2, 8192)])
def test_norm(m, kind, fmt, rows, cols):
    r = rng(rows, cols)
    for dt, dd, gained in (("float32", "bfloat16", True), ("bfloat16", "float32", False), ("float32", None, True),
                           ("bfloat16", "bfloat16", True), ("float32", "float32", False)):
        log("norm", kind, fmt, rows, cols, dt, dd)
        x = torch.from_numpy((r.standard_normal((rows, cols)) * 3 + 1).astype(np.float32)).to(getattr(torch, dt)).cuda()
        d = None
        if dd:
            d = torch.from_numpy(r.standard_normal((rows, cols)).astype(np.float32)).to(getattr(torch, dd)).cuda()
        g = torch.from_numpy((1 + 0.3 * r.standard_normal(cols)).astype(np.float32)).cuda() if gained else None
        keep = x.clone()
        out, q = m.add_norm_mx(x, d, gain=g, fmt=fmt, norm=kind, eps=1e-5)
        want = x if d is None else (x.float() + d.float()).to(x.dtype)
        assert torch.equal(out, want) and out.dtype == x.dtype
        assert torch.equal(x, keep)
        check_norm(want.float().cpu().numpy(), q, m.mx_dequantize(q, torch.float32).cpu().numpy(),
                   g.double().cpu().numpy() if gained else None, kind, 1e-5, fmt)


def test_norm_in_place_strides_and_rows_apart(m):
    base = torch.randn(12, 900, generator=torch.Generator().manual_seed(5)).cuda()
    d = torch.randn(12, 901, generator=torch.Generator().manual_seed(6)).bfloat16().cuda()
    for lo, n in ((0, 768), (1, 768), (4, 333)):
        x, dv = base[:, lo:lo + n], d[:, lo:lo + n]
        want, q = m.add_norm_mx(x.contiguous(), dv.contiguous())
        into = base.clone()
        xi = into[:, lo:lo + n]
        got, p = m.add_norm_mx(xi, dv, out=xi)
        assert got.data_ptr() == xi.data_ptr()
        assert torch.equal(got, want) and torch.equal(p.codes, q.codes)
        assert np.array_equal(scales_of(p), scales_of(q))
        mask = torch.ones_like(into, dtype=torch.bool)
        mask[:, lo:lo + n] = False
        assert torch.equal(into[mask], base[mask])
        # a row's codes do not depend on the others
        _, one = m.add_norm_mx(x[7:8].contiguous(), dv[7:8].contiguous())
        assert torch.equal(one.codes[0], q.codes[7])


def test_norm_of_extreme_rows(m):
    x = torch.zeros(4, 64, device="cuda")
    x[1] = 5.0                      # layer norm: no spread
    x[2, 3] = float("nan")
    x[3, 3] = float("inf")
    for kind in ("rmsnorm", "layernorm"):
        _, q = m.add_norm_mx(x, norm=kind, eps=1e-5)
        v = m.mx_dequantize(q, torch.float32)
        assert bool((v[0] == 0).all())
        assert bool(torch.isnan(v[2]).all())
        # inf / inf in the block that holds it; finite values over an infinite root are 0
        assert bool(torch.isnan(v[3, :32]).all())
        if kind == "layernorm":
            assert bool((v[1] == 0).all())


# ---------------------------------------------------------------- product
def operands(m, M, N, K, fmt, seed=0):
    g = torch.Generator().manual_seed(seed + M + 7 * N + 11 * K)
    a = torch.randn(M, K, generator=g) * torch.exp2(torch.randint(-6, 7, (M, 1), generator=g).float())
    b = torch.randn(N, K, generator=g)
    b *= torch.exp2(torch.randint(-9, 9, (N, K), generator=g).float() * (torch.rand(N, 1, generator=g) < .3))
    return m.mx_quantize(a.cuda(), fmt), m.mx_quantize(b.cuda(), "fp4")


def check_product(m, qa, qb, out, fmt):
    """Against 64 bits.  fp32: each of the 4 groups instructions adds its sum to the
    accumulator, at most one step (2 U) each of what the terms' magnitudes add up to.
    E4M3: an instruction also drops up to 2^-13 of the largest of its 64 products for
    each of them.  bf16 output: half a step more."""
    a = m.mx_dequantize(qa, torch.float32).double()
    b = m.mx_dequantize(qb, torch.float32).double()
    want = a @ b.t()
    tol = 2 * U * 4 * -(-qa.cols // 256) * (a.abs() @ b.abs().t())
    if fmt == "fp8":
        pa = torch.nn.functional.pad(a.abs(), (0, -qa.cols % 64)).view(qa.rows, -1, 64)
        pb = torch.nn.functional.pad(b.abs(), (0, -qa.cols % 64)).view(qb.rows, -1, 64)
        tol += 2.0 ** -13 * pa.amax(2) @ pb.sum(2).t()
    if out.dtype == torch.bfloat16:
        tol += 2.0 ** -8 * (want.abs() + tol)
    bad = (out.double() - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), float((out.double() - want).abs().max()))
    # and as a whole: an operand element is held with a half step of 2^-4 or 2^-2, a
    # mistake in one term of a hundred would show at 1e-2
    if out.dtype == torch.float32:
        assert float((out.double() - want).norm() / want.norm().clamp_min(1e-30)) < 2e-5


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 32), (2, 33, 64), (31, 129, 256), (32, 128, 257), (33, 100, 300),
                                   (65, 4099, 512), (128, 128, 1024), (129, 257, 1000), (257, 300, 33),
                                   (1, 4096, 4096), (16, 5000, 2304), (300, 777, 768)])
def test_product(m, fmt, M, N, K):
    qa, qb = operands(m, M, N, K, fmt)
    for dt in (torch.float32, torch.bfloat16):
        log("product", fmt, M, N, K, dt)
        check_product(m, qa, qb, m.mx_matmul(qa, qb, dt), fmt)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("M,N,K", [(1000, 12288, 768), (2048, 9000, 512), (4100, 4099, 256), (700, 32768, 1024)])
def test_product_of_many_tiles(m, fmt, M, N, K):
    log("product", fmt, M, N, K)
    qa, qb = operands(m, M, N, K, fmt)
    check_product(m, qa, qb, m.mx_matmul(qa, qb), fmt)


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("M,N,K", [(2048, 4096, 1000), (1900, 4090, 1281), (300, 17001, 2000), (129, 32768, 1537)])
def test_product_of_about_a_tile_a_cu(m, fmt, M, N, K):
    """And the same bits for its last rows in a launch of their own."""
    log("product", fmt, M, N, K)
    qa, qb = operands(m, M, N, K, fmt)
    out = m.mx_matmul(qa, qb)
    check_product(m, qa, qb, out, fmt)
    assert torch.equal(m.mx_matmul(rows_of(qa, M - 33, M), qb), out[M - 33:])
    assert torch.equal(m.mx_matmul(qa, qb, torch.bfloat16), out.bfloat16())


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_product_over_many_columns(m, fmt):
    """Groups past those that the wide tiles' 32-bit offsets take (2^21 columns)."""
    M, N, K = 40, 70, 2200001
    log("columns", fmt, K)
    g = torch.Generator(device="cuda").manual_seed(3)
    # integers that E2M1 holds: their products and sums up to 2^24 are exact in fp32
    a = torch.randint(0, 3, (M, K), generator=g, device="cuda", dtype=torch.int32).float()
    b = torch.randint(-1, 2, (N, K), generator=g, device="cuda", dtype=torch.int32).float()
    a[:, ::32], b[:, ::32] = 6, -6  # a block's scale is 1, or 2^-6 with E4M3's 448 above 6 2^6
    qa, qb = m.mx_quantize(a, fmt), m.mx_quantize(b, "fp4")
    a, b = a.double(), b.double()
    assert torch.equal(m.mx_dequantize(qa, torch.float32).double(), a)
    assert torch.equal(m.mx_dequantize(qb, torch.float32).double(), b)
    assert torch.equal(m.mx_matmul(qa, qb).double(), a @ b.t())


def rows_of(q, lo, hi):
    """Rows lo .. hi - 1 of q, their codes and scales as they are.  (Quantising the
    values again may hold them with another scale: the same values in other codes,
    of whose products the unit drops other bits.)"""
    p = dl.MXMatrix.empty(q.fmt, hi - lo, q.cols, q.codes.device)
    p.codes.copy_(q.codes[lo:hi])
    p.scales.fill_(255)
    p.scales[:, : hi - lo].copy_(q.scales[:, lo:hi])
    return p


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
def test_product_row_does_not_depend_on_the_launch(m, fmt):
    """Every tile shape gives a row the same bits: the decoder's launches have other
    rows than the encoder's."""
    qa, qb = operands(m, 2048, 9001, 900, fmt)
    whole = m.mx_matmul(qa, qb)
    for rows in (1, 2, 16, 31, 32, 33, 64, 100, 128, 200, 256, 400, 777, 1024, 2047):
        log("rows", fmt, rows)
        got = m.mx_matmul(rows_of(qa, 2048 - rows, 2048), qb)
        assert torch.equal(got, whole[2048 - rows:]), rows
    for cols in (1, 64, 300, 3000):
        assert torch.equal(m.mx_matmul(qa, rows_of(qb, 0, cols)), whole[:, :cols]), cols


@pytest.mark.parametrize("fmt", ["fp8", "fp4"])
@pytest.mark.parametrize("M,N", [(5, 70), (100, 300), (1024, 17000)])
def test_product_passes_nan_on(m, fmt, M, N):
    a, b = torch.ones(M, 100), torch.ones(N, 100)
    a[M // 2, 40] = float("nan")
    b[N // 3, 99] = float("inf")
    out = m.mx_matmul(m.mx_quantize(a.cuda(), fmt), m.mx_quantize(b.cuda(), "fp4"))
    bad = torch.isnan(out)
    assert bool(bad[M // 2].all()) and bool(bad[:, N // 3].all())
    assert int(bad.sum()) == M + N - 1
    assert bool((out[~bad] == 100).all())


def test_product_writes_its_rows_alone(m):
    qa, qb = operands(m, 45, 131, 200, "fp8")
    want = m.mx_matmul(qa, qb)
    for dt in (torch.float32, torch.bfloat16):
        for lo in (0, 1, 3):
            buf = torch.full((50, 160), 7.0, dtype=dt, device="cuda")
            out = m.mx_matmul(qa, qb, out=buf[:45, lo:lo + 131])
            assert torch.equal(out, want.to(dt))
            buf[:45, lo:lo + 131] = 7.0
            assert bool((buf == 7).all())


def test_product_past_32_bit_offsets(m):
    """Codes and outputs beyond 2^31 elements: the last rows equal a product of their own."""
    N, K = 600000, 8192
    log("large product", N, K)
    qb = dl.MXMatrix.empty("fp4", N, K, "cuda")
    qb.codes.random_(0, 256, generator=torch.Generator(device="cuda").manual_seed(2))
    qb.scales.fill_(124)
    M = 3600
    a = torch.randn(M, K, generator=torch.Generator().manual_seed(1)).cuda()
    qa = m.mx_quantize(a, "fp8")
    out = m.mx_matmul(qa, qb, torch.bfloat16)  # 2.16e9 outputs of 2.46e9 bytes of codes
    last = dl.MXMatrix.empty("fp4", 500, K, "cuda")
    last.codes.copy_(qb.codes[-500:])
    last.scales.fill_(124)
    assert torch.equal(out[-40:, -500:], m.mx_matmul(m.mx_quantize(a[-40:], "fp8"), last, torch.bfloat16))
    first = dl.MXMatrix.empty("fp4", 500, K, "cuda")
    first.codes.copy_(qb.codes[:500])
    first.scales.fill_(124)
    assert torch.equal(out[-40:, :500], m.mx_matmul(m.mx_quantize(a[-40:], "fp8"), first, torch.bfloat16))


def test_more_rows_than_one_launch_takes(m):
    """Rows past 2^24: a grid of one block each has more threads than 32 bits count."""
    n = (1 << 24) + 5
    log("rows past 2^24", n)
    x = torch.randn(n, 2, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    last = torch.cat((x[:3], x[(1 << 23) - 2: (1 << 23) + 2], x[-6:]))
    pick = lambda t: torch.cat((t[:3], t[(1 << 23) - 2: (1 << 23) + 2], t[-6:]))  # noqa: E731
    for fmt in ("fp8", "fp4"):
        q = m.mx_quantize(x, fmt)
        got = m.mx_dequantize(q, torch.float32)
        assert torch.equal(pick(got), m.mx_dequantize(m.mx_quantize(last, fmt), torch.float32))
        # off by less than a half step of 2^-4 or 2^-2, whose values all blocks have
        assert bool(((got - x).abs() <= x.abs().amax(1, keepdim=True) * 0.25).all())
        del q, got
    wide = torch.zeros(n, 1100, dtype=torch.bfloat16, device="cuda")  # a block a row
    wide[:, :2] = x
    r, q = m.add_norm_mx(wide, wide, fmt="fp4", norm="rmsnorm", eps=1e-5)
    small = pick(wide)
    want, p = m.add_norm_mx(small, small, fmt="fp4", norm="rmsnorm", eps=1e-5)
    assert torch.equal(pick(r), want) and torch.equal(pick(q.codes), p.codes)
    assert torch.equal(pick(q.scales[:, :n].transpose(0, 1)), p.scales[:, : len(small)].transpose(0, 1))
    for t in range(0, n, 1 << 22):  # no row was left out
        assert torch.equal(r[t: t + (1 << 22)], wide[t: t + (1 << 22)] * 2)


# ---------------------------------------------------------------- together
def chain(m, x, d, w, tokens):
    r, q = m.add_norm_mx(x, d, fmt="fp8", norm="rmsnorm", eps=1e-5)
    lg = m.mx_matmul(q, w)
    return (r, lg) + tuple(m.token_scores(lg, tokens, top=4))


def test_norm_product_scores_together():
    """One position's row up to a chunk's: the head as a program runs it, against 64
    bits from the values that the norm gave."""
    V, K = 3001, 640
    g = torch.Generator().manual_seed(8)
    with dl.Model(shape(vocab=V, n_layers=0), max_chunk=1) as m:
        w = m.mx_quantize((torch.randn(V, K, generator=g) / 8).cuda(), "fp4")
        wv = m.mx_dequantize(w, torch.float32).double()
        for n in (1, 7, 300):
            log("chain", n)
            x, d = torch.randn(n, K, generator=g).cuda(), torch.randn(n, K, generator=g).bfloat16().cuda()
            tok = torch.randint(0, V, (n,), generator=g, dtype=torch.int32).cuda()
            r, lg, lp, h, ids, tlp = chain(m, x, d, w, tok)
            assert torch.equal(r, x + d.float())
            _, q = m.add_norm_mx(x, d, norm="rmsnorm", eps=1e-5)
            p = torch.log_softmax(m.mx_dequantize(q, torch.float32).double() @ wv.t(), 1) / np.log(2)
            # logits: up to 6e-4 of their 5 or so from the E4M3 products (2^-13 of the
            # largest product for each); entropies weigh 12 bits of such errors
            assert float((lp.double() - p.gather(1, tok.long()[:, None])[:, 0]).abs().max()) < 1e-2
            assert float((h.double() + (p.exp2() * p).sum(1)).abs().max()) < 1e-1
            assert torch.equal(ids, torch.sort(lg, dim=1, descending=True, stable=True)[1][:, :4].int())
            assert float((tlp.double() - p.gather(1, ids.long())).abs().max()) < 1e-2


def test_streams_and_a_captured_graph():
    """The calls follow their stream, and a captured run replays with new inputs, with
    eager calls of the same model between the replays."""
    V, K, n = 5003, 512, 40
    g = torch.Generator().manual_seed(4)
    with dl.Model(shape(vocab=V, n_layers=0), max_chunk=1) as m:
        w = m.mx_quantize(torch.randn(V, K, generator=g).cuda(), "fp4")
        x, d = torch.zeros(n, K).cuda(), torch.zeros(n, K).bfloat16().cuda()
        tok = torch.randint(0, V, (n,), generator=g, dtype=torch.int32).cuda()
        fresh = [(torch.randn(n, K, generator=g).cuda(), torch.randn(n, K, generator=g).bfloat16().cuda())
                 for _ in range(3)]
        want = [[t.clone() for t in chain(m, a, b, w, tok)] for a, b in fresh]
        side = torch.cuda.Stream()
        busy = torch.eye(4096, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                busy = busy @ busy
            x.copy_(fresh[0][0])
            d.copy_(fresh[0][1])
            late = chain(m, x, d, w, tok)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(late, want[0]))
        graph = torch.cuda.CUDAGraph()
        log("capture")
        with torch.cuda.graph(graph, stream=side):
            out = chain(m, x, d, w, tok)
        for k in (1, 2, 0, 1):
            with torch.cuda.stream(side):
                x.copy_(fresh[k][0])
                d.copy_(fresh[k][1])
                graph.replay()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want[k])), k
            eager = chain(m, *fresh[(k + 1) % 3], w, tok)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, want[(k + 1) % 3]))


def test_a_capture_on_streams_the_model_has_not_seen():
    """Eager calls on the default stream first; then a capture on one stream, with a
    branch on another."""
    V, K, n = 3001, 512, 9
    g = torch.Generator().manual_seed(14)
    with dl.Model(shape(vocab=V, n_layers=0), max_chunk=1) as m:
        w = m.mx_quantize(torch.randn(V, K, generator=g).cuda(), "fp4")
        x, y = torch.randn(n, K, generator=g).cuda(), torch.randn(n, K, generator=g).cuda()
        tok = torch.zeros(n, dtype=torch.int32).cuda()
        want = [t.clone() for t in chain(m, x, y.bfloat16(), w, tok)]
        other = m.mx_matmul(m.mx_quantize(y, "fp8"), w)
        torch.cuda.synchronize()
        a, b = torch.cuda.Stream(), torch.cuda.Stream()
        d = y.bfloat16()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        log("capture on new streams")
        with torch.cuda.graph(graph, stream=a):
            q = m.mx_quantize(y, "fp8")
            b.wait_stream(a)
            with torch.cuda.stream(b):
                branch = m.mx_matmul(q, w)
            out = chain(m, x, d, w, tok)
            a.wait_stream(b)
        for _ in range(3):
            branch.zero_()
            for t in out:
                t.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(a):
                graph.replay()
            a.synchronize()
            assert all(torch.equal(s, t) for s, t in zip(out, want)) and torch.equal(branch, other)
            eager = chain(m, x, d, w, tok)
            assert all(torch.equal(s, t) for s, t in zip(eager, want))


# ---------------------------------------------------------------- refusals
def test_refusals(m):
    x = torch.randn(4, 64, device="cuda")
    q8, q4 = m.mx_quantize(x, "fp8"), m.mx_quantize(x, "fp4")
    bad = [
        lambda: m.mx_quantize(x, "fp6"),
        lambda: m.mx_quantize(x.half(), "fp4"),
        lambda: m.mx_quantize(x.cpu(), "fp4"),
        lambda: m.mx_quantize(x[0], "fp4"),
        lambda: m.mx_quantize(x.t(), "fp4"),
        lambda: m.mx_quantize(x.expand(4, 64)[:1].expand(3, 64), "fp4"),
        lambda: m.mx_quantize(torch.empty(3, 0, device="cuda"), "fp4"),
        lambda: m.mx_dequantize(q8, torch.float16),
        lambda: m.mx_dequantize(x),
        lambda: m.mx_dequantize(dl.MXMatrix(q4.codes, q4.scales, "fp8", 4, 64)),
        lambda: m.mx_dequantize(dl.MXMatrix(q8.codes, q8.scales, "fp8", 4, 300)),
        lambda: m.mx_dequantize(dl.MXMatrix(q8.codes.cpu(), q8.scales, "fp8", 4, 64)),
        lambda: m.mx_matmul(q4, q8),
        lambda: m.mx_matmul(q8, m.mx_quantize(torch.randn(4, 65, device="cuda"), "fp4")),
        lambda: m.mx_matmul(q8, q4, torch.float16),
        lambda: m.mx_matmul(q8, q4, out=torch.empty(4, 5, device="cuda")),
        lambda: m.mx_matmul(q8, q4, torch.bfloat16, out=torch.empty(4, 4, device="cuda")),
        lambda: m.mx_matmul(q8, q4, out=torch.empty(4, 4, device="cuda").t()[:, ::2]),
        lambda: m.add_norm_mx(x, x[:2]),
        lambda: m.add_norm_mx(x, x[:, :32]),
        lambda: m.add_norm_mx(x, x.double()),
        lambda: m.add_norm_mx(x, norm="groupnorm"),
        lambda: m.add_norm_mx(x, eps=-1.0),
        lambda: m.add_norm_mx(x, eps=float("nan")),
        lambda: m.add_norm_mx(x, gain=torch.ones(63, device="cuda")),
        lambda: m.add_norm_mx(x, gain=torch.ones(64, device="cuda").bfloat16()),
        lambda: m.add_norm_mx(x, x, out=torch.empty(4, 64, device="cuda").bfloat16()),
        lambda: m.add_norm_mx(torch.zeros(1, 8193, device="cuda")),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(dl.DlmcError) as e:
            call()
        assert e.value.code == -1, i
    # the C entry's own checks: types, rows that overlap, alignment of the codes
    L, h = dl.lib(), m.handle
    assert L.dlmc_mx_quantize(h, x.data_ptr(), 2, 64, 4, 64, 0, q4.codes.data_ptr(), q4.scales.data_ptr()) == -1
    assert L.dlmc_mx_quantize(h, x.data_ptr(), 0, 63, 4, 64, 0, q4.codes.data_ptr(), q4.scales.data_ptr()) == -1
    assert L.dlmc_mx_quantize(h, x.data_ptr(), 0, 64, 4, 64, 0, q4.codes.data_ptr() + 4, q4.scales.data_ptr()) == -1
    assert L.dlmc_mx_quantize(h, x.data_ptr() + 2, 0, 64, 4, 64, 0, q4.codes.data_ptr(), q4.scales.data_ptr()) == -1
    assert L.dlmc_mx_quantize(h, None, 0, 64, 4, 64, 0, q4.codes.data_ptr(), q4.scales.data_ptr()) == -1
    assert L.dlmc_mx_matmul(h, q8.codes.data_ptr(), q8.scales.data_ptr(), 1, q4.codes.data_ptr(),
                            q4.scales.data_ptr(), 4, -1, 64, x.data_ptr(), 0, 64) == -1
