"""Token scores of more rows than a launch takes, long enough that the few rows of the
last launch would be split if they were all."""
import pytest

import paper_2608_11249_amd as dl
from gpu_common import log, shape

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [0, 3])
def test_the_last_part_is_scored_as_the_others(top):
    V, n = 8186, (1 << 23) + 1
    assert dl.score_launches(1, V, top)[0][1] > 2 and dl.score_launches(n, V, top)[1] == (1, 1, 0)
    torch.cuda.empty_cache()
    need = n * V * 2
    if torch.cuda.mem_get_info()[0] < need + (4 << 30):
        pytest.skip(f"{need >> 30} GiB of logits do not fit beside what is held")
    log("last part", n, V, top)
    lg = torch.zeros(n, V, dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 1, (1 << 23) - 1, 1 << 23], device="cuda")
    lg[some] = torch.randn(4, V, generator=torch.Generator().manual_seed(top)).bfloat16().cuda()
    tok = torch.arange(n, dtype=torch.int32, device="cuda") % V
    with dl.Model(shape(vocab=V, n_layers=0), max_chunk=1) as m:
        got = m.token_scores(lg, tok, top=top)
        few = lg[some].contiguous()
        torch.cuda.synchronize()
        want = m.token_scores(few.repeat(700, 1), tok[some].repeat(700), top=top)  # in one launch, not split
        p = torch.log_softmax(few.double(), 1) / torch.log(torch.tensor(2.0, dtype=torch.double))
        # fp32 sums of 8186 / 256 + 64 terms at most one after another, each with a
        # half step of 2^-24, and two roundings of an exponent of less than 32 bits
        tol = 2.0 ** -24 * (V / 256 + 64 + 64) * 2
        assert float((got[0][some] - p.gather(1, tok[some].long()[:, None])[:, 0]).abs().max()) <= tol
        assert float((got[1][some] + (p.exp2() * p).sum(1)).abs().max()) <= tol * 15
        assert torch.equal(got[2][some], want[2][:4])
        assert torch.equal(got[2][some], torch.sort(few, dim=1, descending=True, stable=True)[1][:, :top].int())
        # the other rows are uniform
        rest = torch.ones(n, dtype=torch.bool, device="cuda")
        rest[some] = False
        assert float((got[1][rest] - 12.998943).abs().max()) < 1e-3
    del lg, got, few
    torch.cuda.empty_cache()
