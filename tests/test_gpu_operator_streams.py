"""Streams of the operators that return without waiting: work on one does not hold up
calls on another, and the model's own passes keep their stream meanwhile."""
import numpy as np
import pytest

import paper_2608_11249_amd as dl
import workloads as wl
from gpu_common import codec, log, shape

torch = pytest.importorskip("torch")


@pytest.mark.skipif(not dl.os.path.exists(dl.LIB_PATH), reason="libdlmc.so not built")
def test_no_model():
    assert dl.lib().dlmc_set_operator_stream(None, None) == -1


def inputs(V, K, n, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, K, generator=g).cuda(), torch.randn(n, K, generator=g).bfloat16().cuda(),
            torch.randint(0, V, (n,), generator=g, dtype=torch.int32).cuda())


def chain(m, w, x, d, tok):
    r, q = m.add_norm_mx(x, d, norm="rmsnorm", eps=1e-5)
    lg = m.mx_matmul(q, w)
    return (r, m.mx_dequantize(q), lg) + tuple(m.token_scores(lg, tok, top=4))


@pytest.mark.gpu
def test_a_busy_stream_does_not_hold_up_calls_on_another():
    V, K, n = 3001, 512, 20
    with dl.Model(shape(vocab=V, n_layers=0), max_chunk=1) as m:
        w = m.mx_quantize(torch.randn(V, K, generator=torch.Generator().manual_seed(1)).cuda(), "fp4")
        one, two = inputs(V, K, n, 2), inputs(V, K, n, 3)
        want = [[t.clone() for t in chain(m, w, *i)] for i in (one, two)]
        busy = torch.eye(8192, device="cuda", dtype=torch.bfloat16)
        a, b = torch.cuda.Stream(), torch.cuda.Stream()
        for s in (a, b):  # everything loaded and allocated once
            with torch.cuda.stream(s):
                chain(m, w, *one)
        torch.cuda.synchronize()
        done = torch.cuda.Event()
        log("busy stream")
        with torch.cuda.stream(a):
            for _ in range(200):  # a tenth of a second and more
                busy = busy @ busy
            on_a = chain(m, w, *one)
            done.record()
        with torch.cuda.stream(b):
            on_b = chain(m, w, *two)
        # the host came this far while a is busy (whether b's work runs meanwhile goes by
        # the hardware queues that the two streams were given)
        assert not done.query()
        with torch.cuda.stream(a):  # back on the busy stream, behind its work
            again = m.mx_matmul(m.mx_quantize(two[0], "fp8"), w)
        assert not done.query()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(on_b, want[1]))
        assert all(torch.equal(s, t) for s, t in zip(on_a, want[0]))
        assert torch.equal(again, m.mx_matmul(m.mx_quantize(two[0], "fp8"), w))


@pytest.mark.gpu
def test_passes_keep_their_stream():
    """Encoding step by step, with operators and stage hooks on other streams between."""
    sh = shape(vocab=700, d_model=256, n_heads=4)
    cp = codec(48, k=4, P=16, W=64)
    toks = wl.markov1_tokens(48 * 5 + 17, sh.vocab, 3).astype(np.int32)
    x = torch.randn(30, 700, generator=torch.Generator().manual_seed(5)).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    log("steps between")
    with dl.Model(sh, max_chunk=48, max_batch=4) as m:
        want = m.encode(toks, cp, batch=4)
        scores = [t.clone() for t in m.token_scores(x, top=3)[1:]]
        H = m.entropy_cdf(x, 16, want_cdf=False)[0]
        torch.cuda.synchronize()
        enc = m.encoder(cp, toks, batch=4)
        k = 0
        while not enc.step():
            k += 1
            with torch.cuda.stream(side if k % 2 else torch.cuda.default_stream()):
                got = m.token_scores(x, top=3)[1:]
                if k % 3 == 0:
                    assert torch.equal(m.entropy_cdf(x, 16, want_cdf=False)[0], H)
                torch.cuda.current_stream().synchronize()
                assert all(torch.equal(s, t) for s, t in zip(got, scores))
        assert enc.finish() == want
        with torch.cuda.stream(side):
            m.mx_quantize(x, "fp8")
        assert np.array_equal(m.decode(want), toks)


@pytest.mark.gpu
def test_set_stream_gives_the_operators_their_stream_too():
    """The C entries by themselves: dlmc_set_stream for all calls, then another stream
    for the operators alone."""
    V = 900
    lg = torch.randn(5, V, generator=torch.Generator().manual_seed(1)).cuda()
    H = torch.zeros(5, device="cuda")
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    L = dl.lib()
    busy = torch.eye(8192, device="cuda", dtype=torch.bfloat16)
    with dl.Model(shape(vocab=V, n_layers=0), max_chunk=1) as m:
        want = m.token_scores(lg)[1].clone()
        torch.cuda.synchronize()
        call = lambda: L.dlmc_token_scores(m.handle, lg.data_ptr(), 0, V, 5, None, 0, None, H.data_ptr(), None, None,  # noqa: E731
                                           None, 0)
        m.set_stream(a.cuda_stream)
        done, late = torch.cuda.Event(), torch.cuda.Event()
        with torch.cuda.stream(a):
            for _ in range(100):
                busy = busy @ busy
            done.record()
        assert call() == 0  # behind the work on a
        late.record(a)
        assert L.dlmc_set_operator_stream(m.handle, b.cuda_stream) == 0
        other = torch.zeros(5, device="cuda")
        b.wait_stream(torch.cuda.current_stream())
        assert L.dlmc_token_scores(m.handle, lg.data_ptr(), 0, V, 5, None, 0, None, other.data_ptr(), None, None, None,
                                   0) == 0
        assert not done.query()
        b.synchronize()
        assert torch.equal(other, want)
        late.synchronize()
        assert torch.equal(H, want)
        m.set_stream(None)
        H.zero_()
        torch.cuda.synchronize()
        assert call() == 0
        torch.cuda.synchronize()
        assert torch.equal(H, want)
