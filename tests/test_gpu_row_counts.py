"""Rows that the library's 32-bit counts do not hold are refused, not cut to what is left of
them."""
import pytest

import paper_2608_11249_amd as dl
from gpu_common import log, shape

torch = pytest.importorskip("torch")


@pytest.mark.skipif(not dl.os.path.exists(dl.LIB_PATH), reason="libdlmc.so not built")
@pytest.mark.parametrize("rows", [2 ** 31, 2 ** 32, 2 ** 32 + 3, 2 ** 40])
def test_matrices_of_too_many_rows(rows):
    for fmt in ("fp4", "fp8"):
        with pytest.raises(dl.DlmcError) as e:
            dl.MXMatrix(torch.empty(0, dtype=torch.uint8), torch.empty(0, dtype=torch.uint8), fmt, rows, 8)
        assert e.value.code == -1 and str(rows) in str(e.value)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [2 ** 31, 2 ** 32 + 3])
def test_tensors_of_too_many_rows(rows):
    log("rows", rows)
    with dl.Model(shape(vocab=2, n_layers=0), max_chunk=1) as m:
        x = torch.empty(rows, 2, dtype=torch.bfloat16, device="cuda")
        for call in (lambda: m.token_scores(x), lambda: m.mx_quantize(x), lambda: m.add_norm_mx(x)):
            with pytest.raises(dl.DlmcError) as e:
                call()
            assert e.value.code == -1 and "rows" in str(e.value)
    del x
    torch.cuda.empty_cache()
