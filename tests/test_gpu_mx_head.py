"""Models whose LM head is held in block-scaled values (dtype "bf16-mx4head"): the
weights, the logits against the oracle and against the operators one by one, and
lossless round trips under every schedule and coder."""
import dataclasses

import numpy as np
import pytest

import paper_2608_11249_amd as dl
import workloads as wl
from gpu_common import codec, log, payloads, shape
from mx_common import held, scale_exp, step
from oracle import model as OM
from oracle import weights as OW

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MX = "bf16-mx4head"


def bf16_of(sh):
    return dataclasses.replace(sh, dtype="bf16")


def head_of(sh):
    """The head's values in 64 bits: E2M1 of the bf16 weights."""
    return held(OW.gen_tensor(sh.seed, 2, (sh.vocab, sh.d_model), sh.head_exp, "bf16"), "fp4")


@pytest.mark.parametrize("d,V", [(128, 500), (640, 333), (768, 1000)])
def test_head_weights_are_the_definition(d, V):
    sh = shape(dtype=MX, d_model=d, n_heads=d // 64, n_layers=0, vocab=V)
    log("mx head weights", d, V)
    with dl.Model(sh, max_chunk=8) as m:
        assert np.array_equal(m.weight(2, V, d), OW.bf16_bits(head_of(sh)))
        # the other tensors are the bf16 model's
        assert np.array_equal(m.weight(1, V + 1, d), OW.bf16_bits(
            OW.gen_tensor(sh.seed, 1, (V + 1, d), sh.embed_exp, "bf16")))


def state_of(sh, B, T, frac, seed=0):
    st = wl.random_state(seed, B, T, sh.vocab, frac).astype(np.int32)
    st[0, 0] = sh.mask_id
    return st


@pytest.mark.parametrize("kw,B,T", [
    (dict(n_layers=0), 1, 40), (dict(n_layers=2), 2, 100), (dict(n_layers=1, vocab=4099, d_model=256, n_heads=2), 1, 300),
    (dict(n_layers=2, ffn="swiglu", norm="rmsnorm", d_model=384, n_heads=3, vocab=1000), 3, 64)])
def test_logits_against_oracle(kw, B, T):
    """Each weight's bf16 is E2M1-held (exactly known), each row element off by at
    most half a step of its block's E4M3: their sum bounds the head's error.  The
    layers below add the bf16 model's own 2e-2 of the row's largest logit."""
    sh = shape(dtype=MX, **kw)
    st = state_of(sh, B, T, 0.6)
    W, head = OW.Weights(bf16_of(sh)), head_of(sh)
    log("mx head logits", kw, B, T)
    with dl.Model(sh, max_chunk=T, max_batch=B) as m:
        lg, rows = m.forward_logits(torch.from_numpy(st).cuda())
        lg, rows = lg.cpu().numpy(), rows.cpu().numpy()
    r = 0
    for b in range(B):
        h, pos = OM.hidden(bf16_of(sh), W, st[b]), OM.masked_positions(sh, st[b])
        h = h[pos]
        assert np.array_equal(rows[r: r + len(pos)], b * T + pos)
        s = np.repeat(np.exp2(scale_exp(h, "fp8").astype(np.float64)), 32, 1)[:, : sh.d_model]
        half = step(h / s, "fp8") * s
        want = h @ head.T
        tol = half @ np.abs(head).T + 2e-2 * np.abs(want).max(1, keepdims=True)
        assert (np.abs(lg[r: r + len(pos)] - want) <= tol).all()
        # as a whole: the roundings are independent, a 2^-4 half step at most each
        assert np.linalg.norm(lg[r: r + len(pos)] - want) <= 2.0 ** -4 * np.linalg.norm(want)
        r += len(pos)
    assert r == len(rows)


@pytest.mark.parametrize("norm", ["layernorm", "rmsnorm"])
@pytest.mark.parametrize("T,V", [(1, 700), (20, 4099), (700, 999)])
def test_head_is_the_operators_one_by_one(norm, T, V):
    """Without layers a row of the residual stream is [MASK]'s embedding: its norm,
    the product and the scores by the hooks give the model's bits."""
    sh = shape(dtype=MX, n_layers=0, vocab=V, d_model=640, n_heads=10, norm=norm)
    st = np.full((1, T), sh.mask_id, np.int32)
    log("mx head by hooks", norm, T, V)
    with dl.Model(sh, max_chunk=T) as m, dl.Model(bf16_of(sh), max_chunk=T) as plain:
        lg, _ = m.forward_logits(torch.from_numpy(st).cuda())
        as_f32 = lambda bits: torch.from_numpy(bits.astype(np.uint32) << 16).view(torch.float32)  # noqa: E731
        x = as_f32(m.weight(1, V + 1, 640)[V:].astype(np.uint32)).expand(T, 640).contiguous().cuda()
        w = as_f32(plain.weight(2, V, 640).astype(np.uint32)).cuda()
        _, q = m.add_norm_mx(x)
        by_hand = m.mx_matmul(q, m.mx_quantize(w.bfloat16(), "fp4"))
        assert torch.equal(by_hand, lg)
        tok = torch.arange(T, dtype=torch.int32).cuda() % V
        lp, h, ids, _ = m.token_scores(lg, tok, top=5)
        p = torch.log_softmax(lg.double(), 1) / np.log(2)
        assert float((lp.double() - p.gather(1, tok.long()[:, None])[:, 0]).abs().max()) < 1e-4
        assert float((h - m.entropy_cdf(lg, 16, want_cdf=False)[0]).abs().max()) < 1e-4
        assert torch.equal(ids, torch.sort(lg, dim=1, descending=True, stable=True)[1][:, :5].int())


CODECS = [
    codec(48, k=4, P=16, W=64), codec(48, tau=6.0, mmin=1, mmax=16, P=16, W=64, coder="rans"),
    codec(48, k=8, P=16, W=64, coder="rank", rank_compressor="zlib", rank_level=6),
    codec(48, mmin=1, mmax=24, P=16, W=64, schedule="uniform", blocks=5),
    codec(48, mmin=1, mmax=48, P=16, W=64, schedule="progressive", u1=2, growth=1.5, context=6, context_kind="random"),
    codec(48, k=6, P=16, W=64, context=8, context_kind="attention"),
]


@pytest.mark.parametrize("i", range(len(CODECS)))
def test_round_trips_and_batches(i):
    cp = CODECS[i]
    sh = shape(dtype=MX, vocab=700, d_model=256, n_heads=4)
    toks = wl.markov1_tokens(48 * 5 + 17, sh.vocab, 3).astype(np.int32)
    log("mx head round trip", cp)
    with dl.Model(sh, max_chunk=48, max_batch=4) as m:
        one = m.encode(toks, cp, batch=1, crc=True)
        many = m.encode(toks, cp, batch=4, crc=True)
        assert payloads(one) == payloads(many) or cp.coder == "rank"
        assert np.array_equal(m.decode(one, batch=3), toks)
        assert np.array_equal(m.decode(many, batch=1), toks)
        for mode in (1, 2):
            m.head_logits_mode(mode)
            assert m.encode(toks, cp, batch=4, crc=True) == many
        m.head_logits_mode(0)
        with dl.Model(bf16_of(sh), max_chunk=48) as other:
            with pytest.raises(dl.DlmcError) as e:
                other.decode(one)
            assert e.value.code == -4
            with pytest.raises(dl.DlmcError) as e:
                m.decode(other.encode(toks, cp, batch=1))
            assert e.value.code == -4


def test_round_trip_at_the_small_models_width():
    """Tiles of every kind: many masked rows at first, few at the end."""
    sh = dataclasses.replace(wl.with_layers(wl.SMALL, 1), dtype=MX, vocab=9001)
    cp = codec(512, tau=9.0, mmin=32, mmax=256, P=24, W=64)
    toks = wl.markov1_tokens(512 * 3 + 100, sh.vocab, 5).astype(np.int32)
    log("mx head small")
    with dl.Model(sh, max_chunk=512, max_batch=3) as m:
        data = m.encode(toks, cp, batch=3)
        assert np.array_equal(m.decode(data, batch=2), toks)
        m.inject_nonfinite(True)
        with pytest.raises(dl.DlmcError) as e:
            m.encode(toks, cp, batch=3)
        assert e.value.code == -7
        m.inject_nonfinite(False)
        assert m.encode(toks, cp, batch=3) == data
