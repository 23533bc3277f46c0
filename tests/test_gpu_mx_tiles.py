"""The product of block-scaled matrices on every kind of tile, in both formats: sizes
that are no multiple of a tile, odd and even numbers of column groups, outputs in
fp32 (past the caches too) and bf16, and row counts that only the device knows."""
import numpy as np
import pytest

import paper_2608_11249_amd as dl
import workloads as wl
from gpu_common import log, shape

torch = pytest.importorskip("torch")

# (format, M, N, K): products of 572 MiB, 625 MiB and less, on 7 to 21 groups of columns
WHOLE = [("fp4", 2501, 60001, 4096), ("fp4", 3670, 24571, 2892), ("fp4", 130, 60001, 2300), ("fp4", 777, 33001, 5307),
         ("fp4", 1300, 33001, 700), ("fp8", 1301, 126001, 2892), ("fp8", 2047, 24571, 4096), ("fp8", 130, 60001, 1700),
         ("fp8", 515, 33001, 5307), ("fp8", 1300, 60001, 700)]
ROWS = (1, 17, 33, 65, 95, 129, 200, 257, 400, 515, 777, 1301, 2047)
COLS = (33, 129, 300, 1001, 4099, 8193, 12289, 17001, 24571, 33001, 60001)


def kinds_of(fmt):
    return {k for k in dl.MX_TILES if fmt == "fp8" or k != "128x256deep"}


def parts(fmt, M, N, K):
    """Smaller products of the same columns, three of each kind of tile that any takes."""
    by = {}
    for m in ROWS:
        for n in COLS:
            if m <= M and n <= N:
                by.setdefault(dl.mx_tiles(fmt, m, n, K), []).append((m, n))
    return {k: sorted({v[0], v[len(v) // 2], v[-1]}) for k, v in by.items()}


def test_the_cases_reach_every_kind_of_tile():
    """Without a GPU: each kind, in both formats, is taken by a part of a case, the
    largest also by a whole one, in fp32 past the caches; and no other is taken at any
    size."""
    for fmt in ("fp4", "fp8"):
        cases = [c[1:] for c in WHOLE if c[0] == fmt]
        assert set().union(*(parts(fmt, *c) for c in cases)) == kinds_of(fmt)
        big = [(M, N, K) for M, N, K in cases if dl.mx_tiles(fmt, M, N, K) == "256x256"]
        assert any(M * N * 4 >= 512 << 20 for M, N, K in big)
        assert {-(-K // 256) % 2 for _, _, K in big} == {0, 1}
        taken = {dl.mx_tiles(fmt, M, N, K) for M in (1, 16, 32, 33, 64, 100, 128, 256, 777, 1024, 2048, 65536)
                 for N in (1, 64, 500, 4096, 12288, 32768, 126464) for K in (1, 256, 768, 1024, 4096, 12288, 1 << 21)}
        assert taken <= kinds_of(fmt)
    for bad in (("fp4", 0, 5, 5), ("fp8", 5, 0, 5), ("fp4", 5, 5, 0), ("fp8", 5, 5, (1 << 24) + 1)):
        with pytest.raises(dl.DlmcError) as e:
            dl.mx_tiles(*bad)
        assert e.value.code == -1


@pytest.fixture(scope="module")
def m():
    with dl.Model(shape(vocab=256, n_layers=0), max_chunk=1) as model:
        yield model


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,M,N,K", WHOLE)
def test_every_kind_of_tile_gives_the_same_bits(m, fmt, M, N, K):
    """The whole product against 64 bits; the others, of some of its rows and columns,
    have its bits, whatever tiles they take."""
    from test_gpu_mx import check_product, operands, rows_of
    log("tiles", fmt, M, N, K, dl.mx_tiles(fmt, M, N, K))
    qa, qb = operands(m, M, N, K, fmt)
    out = m.mx_matmul(qa, qb)
    check_product(m, qa, qb, out, fmt)
    assert torch.equal(m.mx_matmul(qa, qb, torch.bfloat16), out.bfloat16())
    for kind, sizes in parts(fmt, M, N, K).items():
        for rows, cols in sizes:
            log("part", kind, rows, cols)
            a, b = rows_of(qa, M - rows, M), rows_of(qb, N - cols, N)
            want = out[M - rows:, N - cols:]
            assert torch.equal(m.mx_matmul(a, b), want), (kind, rows, cols)
            assert torch.equal(m.mx_matmul(a, b, torch.bfloat16), want.bfloat16()), (kind, rows, cols)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,M,N,K,kind", [("fp8", 2047, 24571, 4096, "256x256"), ("fp4", 3670, 24571, 2892, "256x256"),
                                            ("fp8", 700, 60001, 700, "128x256"), ("fp4", 515, 33001, 1000, "128x256")])
def test_large_tiles_write_their_rows_alone(m, fmt, M, N, K, kind):
    from test_gpu_mx import operands
    assert dl.mx_tiles(fmt, M, N, K) == kind
    log("rows alone", fmt, M, N, K)
    qa, qb = operands(m, M, N, K, fmt)
    want = m.mx_matmul(qa, qb)
    for dt in (torch.float32, torch.bfloat16):
        for lo in (0, 1, 8):
            buf = torch.full((M + 2, N + 16), 7.0, dtype=dt, device="cuda")
            out = m.mx_matmul(qa, qb, out=buf[1:M + 1, lo:lo + N])
            assert torch.equal(out, want.to(dt))
            buf[1:M + 1, lo:lo + N] = 7.0
            assert bool((buf == 7).all())


@pytest.mark.gpu
def test_a_head_whose_row_count_only_the_device_knows():
    """Chunks alone and in a batch: launches of 40 and of 2000 rows, about half of them
    live, on other tiles, give a masked position the same logits."""
    T, B = 40, 50
    sh = shape(dtype="bf16-mx4head", d_model=2048, n_heads=16, d_ffn=2112, vocab=126464, n_layers=1, ffn="swiglu",
               norm="rmsnorm")
    assert dl.mx_tiles("fp8", T * B, sh.vocab, 2048) == "256x256" != dl.mx_tiles("fp8", T, sh.vocab, 2048)
    log("device row count", T, B)
    st = wl.random_state(7, B, T, sh.vocab, 0.5).astype(np.int32)
    st[:, 0] = sh.mask_id
    st[1, 1:] = 0  # a chunk with a single masked position
    dev = torch.from_numpy(st).cuda()
    with dl.Model(sh, max_chunk=T, max_batch=B) as model:
        together, rows = model.forward_logits(dev)
        rows = rows.cpu().numpy()
        assert bool(torch.isfinite(together).all()) and 0.3 * T * B < len(rows) < 0.7 * T * B
        for b in (0, 1, 30, B - 1):
            alone, r1 = model.forward_logits(dev[b:b + 1])
            mine = np.nonzero(rows // T == b)[0]
            assert np.array_equal(r1.cpu().numpy(), rows[mine] - b * T)
            assert torch.equal(alone, together[int(mine[0]):int(mine[-1]) + 1])
