"""Where add_norm_mx stores its sum: in x, in delta, in other columns of the same
buffer; any other overlap, whose rows would be read after they are written, is
refused."""
import pytest

import paper_2608_11249_amd as dl
from gpu_common import shape

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    with dl.Model(shape(vocab=256, n_layers=0), max_chunk=1) as model:
        yield model


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols", [(1, 64), (7, 100), (5, 1500), (3, 4096)])
def test_sum_in_x_in_delta_or_beside_them(m, dtype, rows, cols):
    g = torch.Generator().manual_seed(rows + cols)
    x, d = (torch.randn(rows, cols, generator=g).to(getattr(torch, dtype)).cuda() for _ in range(2))
    want, q = m.add_norm_mx(x, d)
    for place in ("x", "delta", "beside", "after"):
        buf = torch.zeros(2 * rows, 3 * cols, dtype=x.dtype, device="cuda")
        xv, dv = buf[:rows, :cols], buf[:rows, cols:2 * cols]
        xv.copy_(x)
        dv.copy_(d)
        out = {"x": xv, "delta": dv, "beside": buf[:rows, 2 * cols:], "after": buf[rows:, 1:cols + 1]}[place]
        r, p = m.add_norm_mx(xv, dv, out=out)
        assert r is out and torch.equal(out, want), place
        assert torch.equal(p.codes, q.codes), place
        assert place == "x" or torch.equal(xv, x)
        assert place == "delta" or torch.equal(dv, d)


def test_other_overlaps_are_refused(m):
    buf = torch.randn(12, 400, device="cuda")
    x, d = buf[:4, :64], buf[6:10, 200:264]
    bad = [buf[1:5, :64], buf[:4, 1:65], buf[:4, 63:127], buf[5:9, 200:264], buf[6:10, 180:244], buf[7:11, 263:327],
           buf.view(-1)[: 4 * 128].view(4, 128)[:, :64], buf.view(-1)[8:8 + 256].view(4, 64)]
    keep = buf.clone()
    for i, out in enumerate(bad):
        with pytest.raises(dl.DlmcError) as e:
            m.add_norm_mx(x, d, out=out)
        assert e.value.code == -1, i
    # fp32 sums in the place of bf16 values, row by row
    pairs = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(dl.DlmcError):
        m.add_norm_mx(x, pairs[:, :64], out=pairs.view(torch.float32))
    assert torch.equal(buf, keep) and not bool(pairs.any())
    want, _ = m.add_norm_mx(x, d)
    for out in (buf[4:8, :64], buf[:4, 64:128], buf[2:6, 264:328], buf[2:6, 136:200]):
        assert torch.equal(m.add_norm_mx(x, d, out=out)[0], want)
