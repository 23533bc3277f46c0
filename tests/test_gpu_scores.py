"""Model.token_scores against 64 bits: log2 probabilities of given tokens, entropies,
the most probable symbols with ties, masked symbols, rows without a distribution,
and every way a row can be laid out."""
import numpy as np
import pytest

import paper_2608_11249_amd as dl
import workloads as wl
from gpu_common import log, shape

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def model(V):
    return dl.Model(shape(vocab=V, n_layers=0), max_chunk=1)


def reference(lg, tokens, top):
    lg = lg.astype(np.float64)
    with np.errstate(all="ignore"):
        mx = lg.max(1, keepdims=True)
        t = (lg - mx) / np.log(2)
        z = np.exp2(t).sum(1, keepdims=True)
        lp = t - np.log2(z)
        h = -(np.exp2(lp) * np.where(np.isneginf(lp), 0, lp)).sum(1)
    order = np.stack([np.lexsort((np.arange(lg.shape[1]), -r)) for r in lg])[:, :top]
    tok = lp[np.arange(len(lg)), tokens] if tokens is not None else None
    return tok, h, order, np.take_along_axis(lp, order, 1)


def check(got, want, V):
    """Tolerances: a lane adds at most V / 256 + 8 terms in fp32 where one block takes
    the row, then joins with 256 others in 8 steps; a term's own error is a few half
    steps of its exponent's argument.  The logarithm keeps the sum's relative error
    as an absolute one; arguments t are two roundings of their own size.  An entropy
    is the mean of up to log2 V + |t| bits with the same relative errors."""
    rel = 2.0 ** -24 * (V / 256 + 64)
    lp, h, ids, tlp = [None if t is None else t.cpu().numpy() for t in got]
    for a, b in ((lp, want[0]), (tlp, want[3])):
        if a is None:
            continue
        # below -3.4028e38, the type's lowest logit against a usual one's log2 e = 1.44
        # times, fp32 rounds to -inf
        inf = b < -float(np.finfo(np.float32).max)
        assert np.array_equal(np.isneginf(a), inf)
        assert (np.abs(a - b)[~inf] <= 1.5 * rel + 2.0 ** -22 * np.abs(b[~inf])).all()
    assert (np.abs(h - want[1]) <= rel * 2 * (np.log2(V) + 2)).all()
    assert (h >= 0).all()
    assert np.array_equal(ids, want[2])


@pytest.mark.parametrize("V", [2, 3, 63, 64, 65, 256, 500, 511, 512, 513, 1025, 4099, 32768, 50257, 126464])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_scores(V, dtype):
    with model(V) as m:
        for n, top, scale in ((1, min(20, V), 9.0), (5, 0, 1.0), (3, min(64, V), 2.0), (40, 1, 30.0), (7, min(8, V), 0.0)):
            log("scores", V, dtype, n, top, scale)
            lg = torch.from_numpy(wl.random_logits(V + n, n, V, scale).astype(np.float32)).to(getattr(torch, dtype))
            tok = np.random.default_rng(V + n).integers(0, V, n).astype(np.int32)
            got = m.token_scores(lg.cuda(), torch.from_numpy(tok).cuda(), top=top)
            check(got, reference(lg.float().numpy(), tok, top), V)


@pytest.mark.parametrize("n,V", [(2500, 1200), (2048, 4099), (300, 40000), (65537, 60)])
def test_many_rows(n, V):
    with model(V) as m:
        log("rows", n, V)
        lg = wl.random_logits(n, n, V, 3.0).astype(np.float32)
        tok = np.random.default_rng(n).integers(0, V, n).astype(np.int32)
        got = m.token_scores(torch.from_numpy(lg).cuda(), torch.from_numpy(tok).cuda(), top=5)
        check(got, reference(lg, tok, 5), V)


@pytest.mark.parametrize("n,V", [(3, 1023), (3, 1024), (3, 1025), (511, 5120), (682, 9000), (683, 9000), (2048, 5120),
                                 (2049, 5120), (2049, 5121), (2051, 10240), (2051, 10241), (4095, 11000), (4097, 11000)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_either_side_of_the_launchs_choices(n, V, dtype):
    """A row to a wave, to a block, or to several blocks; rows that do not fill a block."""
    g = torch.Generator(device="cuda").manual_seed(n + V)
    lg = (torch.randn(n, V, generator=g, device="cuda") * 4).to(getattr(torch, dtype))
    lg[n // 2, : V - 30] = float("-inf")
    tok = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    some = torch.arange(0, n, max(1, n // 40), device="cuda")
    some = torch.cat((some, torch.tensor([n // 2, n - 1], device="cuda")))
    with model(V) as m:
        for top in (0, 3, 30):
            log("choices", n, V, dtype, top)
            got = m.token_scores(lg, tok, top=top)
            check([t[some] for t in got], reference(lg[some].float().cpu().numpy(), tok[some].cpu().numpy(), top), V)
            order = torch.sort(lg, dim=1, descending=True, stable=True)[1][:, :top]
            assert torch.equal(got[2], order.int())


@pytest.mark.parametrize("V", [700, 5000, 40001])
def test_ties_and_orders(V):
    """Equal logits go by id, in rows that rise, fall, hold few values or one; -0 is 0."""
    r = np.random.default_rng(V)
    lg = np.stack([np.zeros(V), np.arange(V) / 64, -np.arange(V) / 64, r.integers(0, 3, V), np.arange(V) // 100 % 7,
                   np.where(np.arange(V) % 2, 0.0, -0.0), np.full(V, -1e30), np.r_[np.zeros(V - 1), 1],
                   np.r_[1, np.zeros(V - 1)]]).astype(np.float32)
    tok = np.full(len(lg), V - 1, np.int32)
    with model(V) as m:
        for top in (1, 2, 33, 64):
            log("ties", V, top)
            got = m.token_scores(torch.from_numpy(lg).cuda(), torch.from_numpy(tok).cuda(), top=top)
            check(got, reference(lg, tok, top), V)
            # in one block a row too
            many = np.tile(lg, (250, 1))
            got = m.token_scores(torch.from_numpy(many).cuda(), top=top)
            want = reference(lg, None, top)
            assert got[0] is None
            assert np.array_equal(got[2].cpu().numpy(), np.tile(want[2], (250, 1)))


@pytest.mark.parametrize("V", [600, 1500, 5000, 40001])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_ties_where_lists_fill_up(V, dtype):
    """Rows that rise, so that every tile lies above what came before, in steps of equal
    logits, of a lane's eight in either order, and of -inf: the lists are cut in the
    middle of a tile, whose later columns hold equal logits of lower and higher ids."""
    r = np.random.default_rng(V)
    at = np.arange(V)
    lg = np.stack([at // 37, at // 8 % 64, at % 8, 7 - at % 8, at // 4 % 2 + at // 512, r.integers(0, 2, V),
                   at // 300, np.where(at % 5, -np.inf, at // 100), np.where(at < V - 20, -np.inf, 1.0),
                   np.where(at // 256 % 2, at // 512, -at // 512), -(at // 90), np.zeros(V)])
    lg = torch.from_numpy(lg.astype(np.float32)).to(getattr(torch, dtype)).cuda()
    for many in (1, 260):
        x = lg.repeat(many, 1)
        if many > 1 and V == 40001:
            x = x[:2500]
        want = torch.sort(x, dim=1, descending=True, stable=True)[1]
        with model(V) as m:
            for top in (3, 16, 17, 40, 64):
                log("lists", V, dtype, many, top)
                assert torch.equal(m.token_scores(x, top=top)[2], want[:, :top].int()), top


@pytest.mark.parametrize("V", [100, 3000, 126464])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_masked_symbols(V, dtype):
    """-inf rules symbols out, down to a single one left; the type's lowest value
    does not, and a row of it throughout is uniform."""
    dt = getattr(torch, dtype)
    r = np.random.default_rng(V)
    lg = torch.from_numpy(r.standard_normal((8, V)).astype(np.float32)).to(dt)
    low = torch.finfo(dt).min
    lg[0, 1:] = float("-inf")
    lg[1, : V - 1] = float("-inf")
    lg[2, r.random(V) < 0.97] = float("-inf")
    lg[2, V // 2] = 1.0
    lg[3, :] = low
    lg[4, : V // 2] = low
    lg[5, : V - 3] = low
    lg[6, V // 3:] = float("-inf")
    lg[7, :] = low
    lg[7, 5] = torch.finfo(dt).max
    tok = np.array([0, V - 1, V // 2, V - 1, V - 1, V - 1, V - 1, 5], np.int32)
    top = min(V, 64)
    with model(V) as m:
        log("masked", V, dtype)
        got = m.token_scores(lg.cuda(), torch.from_numpy(tok).cuda(), top=top)
        check(got, reference(lg.float().numpy(), tok, top), V)
        assert float(got[1][0]) == 0 and float(got[0][0]) == 0
        assert abs(float(got[1][3]) - np.log2(V)) < 1e-4


@pytest.mark.parametrize("V", [70, 2000, 33000])
def test_rows_without_a_distribution(V):
    lg = torch.randn(6, V, generator=torch.Generator().manual_seed(V))
    lg[0] = float("-inf")
    lg[1, V - 1] = float("nan")
    lg[2, 0] = float("inf")
    lg[3] = float("nan")
    lg[4, : V - 1], lg[4, V - 1] = float("-inf"), float("nan")
    tok = torch.zeros(6, dtype=torch.int32)
    with model(V) as m:
        for top in (0, 3):
            lp, h, ids, tlp = [t.cpu() for t in m.token_scores(lg.cuda(), tok.cuda(), top=top)]
            assert bool(torch.isnan(lp[:5]).all()) and bool(torch.isnan(h[:5]).all())
            assert bool((ids[:5] == -1).all()) and bool(torch.isnan(tlp[:5]).all())
            assert bool(torch.isfinite(lp[5])) and bool(torch.isfinite(h[5])) and bool((ids[5] >= 0).all())


def test_tokens_that_are_none_or_outside():
    V = 900
    lg = torch.randn(5, V, generator=torch.Generator().manual_seed(1)).cuda()
    tok = torch.tensor([-1, V, 2 ** 31 - 1, -2 ** 31, 7], dtype=torch.int32).cuda()
    with model(V) as m:
        lp = m.token_scores(lg, tok)[0].cpu()
        assert float(lp[0]) == 0 and bool(torch.isnan(lp[1:4]).all())
        assert float(lp[4]) == pytest.approx(float(torch.log_softmax(lg[4].double(), 0)[7]) / np.log(2), abs=1e-5)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strided_and_unaligned_rows(dtype):
    """Row starts at every offset from a 16-byte border give the same as aligned rows."""
    V = 2999
    base = torch.randn(9, 3100, generator=torch.Generator().manual_seed(2)).to(getattr(torch, dtype)).cuda()
    tok = torch.arange(9, dtype=torch.int32).cuda() * 300
    with model(V) as m:
        for lo in range(9):
            view = base[:, lo:lo + V]
            log("offset", lo, dtype)
            got = m.token_scores(view, tok, top=9)
            check(got, reference(view.float().cpu().numpy(), tok.cpu().numpy(), 9), V)
        got = m.token_scores(base[::4, 1:1 + V], tok[::4], top=9)  # and tokens with a stride
        check(got, reference(base[::4, 1:1 + V].float().cpu().numpy(), tok[::4].cpu().numpy(), 9), V)


def test_agrees_with_the_entropies_and_ranks_of_the_coder():
    V = 4099
    lg = torch.from_numpy(wl.random_logits(5, 60, V, 4.0)).cuda()
    with model(V) as m:
        H = m.entropy_cdf(lg, 24, want_cdf=False)[0]
        lp, h, ids, tlp = m.token_scores(lg, torch.zeros(60, dtype=torch.int32, device="cuda"), top=16)
        assert float((h - H).abs().max()) < 1e-4
        for j in range(16):
            assert bool((m.rank_rows(lg, ids[:, j].contiguous()) == j).all())


def test_offsets_past_32_bits():
    V, n = 126464, 17500  # 2.2e9 logits
    log("large", n, V)
    lg = torch.empty(n, V, dtype=torch.bfloat16, device="cuda")
    lg.normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    tok = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(4), dtype=torch.int32).cuda()
    with model(V) as m:
        got = m.token_scores(lg, tok, top=3)
        tail = [t[-3:] for t in got]
        check(tail, reference(lg[-3:].float().cpu().numpy(), tok[-3:].cpu().numpy(), 3), V)


def test_more_rows_than_one_launch_takes():
    """Rows past 2^24: a grid of one block each has more threads than 32 bits count."""
    V, n = 5, (1 << 24) + 3
    log("rows past 2^24", n)
    g = torch.Generator(device="cuda").manual_seed(7)
    lg = torch.randn(n, V, generator=g, device="cuda")
    tok = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    with model(V) as m:
        lp, h, ids, tlp = m.token_scores(lg, tok, top=2)
        p = torch.log_softmax(lg.double(), 1) / np.log(2)
        # five terms: a few half steps of fp32 relative to the sum, and of |log2 p| < 32
        assert float((lp - p.gather(1, tok.long()[:, None])[:, 0]).abs().max()) < 64 * 2.0 ** -24 * 32
        assert float((h + (p.exp2() * p).sum(1)).abs().max()) < 64 * 2.0 ** -24 * 32
        want = torch.sort(lg, dim=1, descending=True, stable=True)[1][:, :2]
        assert torch.equal(ids, want.int())
        assert float((tlp - p.gather(1, want)).abs().max()) < 64 * 2.0 ** -24 * 32


def test_no_rows_and_refusals():
    V = 300
    lg = torch.randn(4, V, device="cuda")
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    with model(V) as m:
        lp, h, ids, tlp = m.token_scores(lg[:0], tok[:0], top=2)
        assert lp.shape == (0,) and h.shape == (0,) and ids.shape == (0, 2) and tlp.shape == (0, 2)
        bad = [lambda: m.token_scores(lg[:, :299], tok), lambda: m.token_scores(lg, tok[:3]),
               lambda: m.token_scores(lg, tok.long()), lambda: m.token_scores(lg, tok, top=65),
               lambda: m.token_scores(lg, tok, top=-1), lambda: m.token_scores(lg.half(), tok),
               lambda: m.token_scores(lg.cpu(), tok), lambda: m.token_scores(lg, tok.cpu()),
               lambda: m.token_scores(lg.t().contiguous().t(), tok), lambda: m.token_scores(lg[0], tok)]
        for i, call in enumerate(bad):
            with pytest.raises(dl.DlmcError) as e:
                call()
            assert e.value.code == -1, i
        # the C entry: a workspace that is needed and missing, too small or not
        # aligned, tokens without a place for their result, no place for alternatives
        L, h_, p = dl.lib(), m.handle, lg.data_ptr()
        out = torch.empty(4, device="cuda")
        o = out.data_ptr()
        assert L.dlmc_token_scores(h_, p, 0, V, 4, tok.data_ptr(), 0, None, o, None, None, None, 0) == -1
        assert L.dlmc_token_scores(h_, p, 0, V, 4, None, 1, None, o, None, None, None, 0) == -1
        assert L.dlmc_token_scores(h_, p, 0, V - 1, 4, None, 0, None, o, None, None, None, 0) == -1
        assert L.dlmc_token_scores(h_, p, 0, V, -1, None, 0, None, o, None, None, None, 0) == -1
    with model(50000) as m:
        import ctypes
        need = ctypes.c_uint64()
        assert dl.lib().dlmc_token_scores_ws(m.handle, 1, 4, ctypes.byref(need)) == 0 and need.value > 0
        big = torch.zeros(1, 50000, device="cuda")
        o = torch.empty(8, device="cuda")
        ids = torch.empty(8, dtype=torch.int32, device="cuda")
        ws = torch.empty(need.value + 16, dtype=torch.uint8, device="cuda")
        for at, size in ((None, need.value), (ws.data_ptr(), need.value - 1), (ws.data_ptr() + 8, need.value)):
            assert dl.lib().dlmc_token_scores(m.handle, big.data_ptr(), 0, 50000, 1, None, 4, None, o.data_ptr(),
                                              ids.data_ptr(), o.data_ptr() + 16, at, size) == -1
