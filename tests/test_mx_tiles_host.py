"""The choice of tiles for very many rows or columns, without a GPU: a launch's tiles
have to be fewer than 2^24, as a grid's threads are counted in 32 bits."""
import os

import pytest

import paper_2608_11249_amd as dl

pytestmark = pytest.mark.skipif(not os.path.exists(dl.LIB_PATH), reason="libdlmc.so not built")


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("M,N,K,live", [
    (1 << 30, 64, 256, -1), ((1 << 30) + 1, 1, 100, -1), (2_000_000_000, 1, 256, -1), (1, 2_000_000_000, 256, -1),
    (33, (1 << 30) + 5, 200, -1), (1 << 20, 65536, 768, -1), (1 << 20, 32768, 768, 1), (1 << 20, 32768, 4096, 16),
    (1 << 19, 126464, 1024, 40), (1 << 20, 32768, 768, 0)])
def test_a_launch_has_fewer_tiles_than_its_grid_counts(fmt, M, N, K, live):
    bm, bn = map(int, dl.mx_tiles(fmt, M, N, K, live).removesuffix("deep").split("x"))
    tiles = -(-M // bm) * -(-N // bn)
    assert tiles < (1 << 24) - 8


def test_live_rows_choose_among_the_tiles_that_fit():
    assert dl.mx_tiles("fp8", 2048, 126464, 4096, 16) == dl.mx_tiles("fp8", 16, 126464, 4096)
    assert dl.mx_tiles("fp8", 2048, 126464, 4096, 5000) == dl.mx_tiles("fp8", 2048, 126464, 4096)
    assert dl.mx_tiles("fp8", 2048, 126464, 4096, -1) == "256x256"


def test_products_past_every_kind_of_tile_are_refused():
    with pytest.raises(dl.DlmcError) as e:
        dl.mx_tiles("fp8", 1 << 30, 1 << 30, 256)
    assert e.value.code == -1 and "tiles" in str(e.value)


@pytest.mark.parametrize("fmt", ["fp4", "fp8"])
@pytest.mark.parametrize("M,N", [(2 ** 31 - 1, 1), (2 ** 31 - 200, 30), (1, 2 ** 31 - 1), (2 ** 31 - 1, 64)])
def test_sizes_next_to_the_last_int(fmt, M, N):
    """Rounding up to whole tiles passes 2^31."""
    bm, bn = map(int, dl.mx_tiles(fmt, M, N, 256).removesuffix("deep").split("x"))
    assert -(-M // bm) * -(-N // bn) < (1 << 24) - 8
    small = 2 ** 31 - 300
    assert dl.mx_tiles(fmt, M, N, 256) == dl.mx_tiles(fmt, min(M, small), min(N, small), 256)
