"""Outputs that an eager graph knows: writing into a tensor whose values a graph has saved
is seen by it, a tensor that requires a gradient is no output, and what the
operators return requires none."""
import pytest

import paper_2608_11249_amd as dl
from gpu_common import shape

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    with dl.Model(shape(vocab=256, n_layers=0), max_chunk=1) as model:
        yield model


def writers(m):
    x = torch.randn(5, 64, device="cuda")
    w = m.mx_quantize(torch.randn(64, 64, device="cuda"), "fp4")
    q = m.mx_quantize(x, "fp8")
    return x, [lambda out: m.mx_matmul(q, w, out=out), lambda out: m.add_norm_mx(x, x, out=out)]


def test_a_graph_that_saved_the_output_sees_the_write(m):
    _, calls = writers(m)
    for call in calls:
        out = torch.randn(5, 64, device="cuda")
        p = torch.randn(5, 64, device="cuda", requires_grad=True)
        before = out._version
        y = (p * out).sum()  # keeps out for p's gradient
        call(out)
        assert out._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
        call(out[:, :])  # a view of it counts too
        z = (p * out).sum()
        z.backward()
        assert torch.equal(p.grad, out)
        part = torch.zeros(9, 80, device="cuda")
        y = (torch.randn(9, 80, device="cuda", requires_grad=True) * part).sum()
        call(part[2:7, 3:67])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def test_outputs_that_require_a_gradient(m):
    _, calls = writers(m)
    for call in calls:
        out = torch.zeros(5, 64, device="cuda", requires_grad=True)
        with pytest.raises(dl.DlmcError) as e:
            call(out)
        assert e.value.code == -1 and not bool(out.detach().any())
        with torch.no_grad():
            call(out)
        assert bool(out.detach().any())
        with torch.inference_mode():
            call(torch.zeros(5, 64, device="cuda"))


def test_results_require_none(m):
    x = torch.randn(5, 256, device="cuda", requires_grad=True)
    r, q = m.add_norm_mx(x, x)
    lp, h, ids, top = m.token_scores(x, torch.zeros(5, dtype=torch.int32, device="cuda"), top=2)
    for t in (r, m.mx_dequantize(m.mx_quantize(x, "fp4")), m.mx_matmul(q, m.mx_quantize(x, "fp4")), lp, h, top):
        assert not t.requires_grad
    assert m.add_norm_mx(x)[0] is x  # without an addition the residual is the input itself
