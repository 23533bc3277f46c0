"""The launches that token scores are made in, without a GPU: every row once, and no
launch with more workspace than the call was given."""
import os

import pytest

import paper_2608_11249_amd as dl

pytestmark = pytest.mark.skipif(not os.path.exists(dl.LIB_PATH), reason="libdlmc.so not built")

PART = 1 << 23
VOCABS = [2, 60, 1024, 1025, 5000, 8185, 8186, 8192, 10241, 32768, 126464, 1 << 20]


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("top", [0, 1, 16, 20, 64])
def test_parts_take_every_row_and_no_more_workspace_than_the_call(V, top):
    top = min(top, V)
    for n in (1, 2, 64, 341, 682, 683, 2048, 2049, 4097, PART - 1, PART, PART + 1, PART + 2, PART + 100, PART + 682,
              PART + 683, 2 * PART, 2 * PART + 1, 3 * PART + 600, 2 ** 31 - 1):
        launches = dl.score_launches(n, V, top)
        assert sum(r for r, _, _ in launches) == n
        assert all(0 < r <= PART for r, _, _ in launches)
        # the workspace asked for is the first launch's; a row is split alike in all
        assert all(ws <= launches[0][2] for _, _, ws in launches), (n, launches)
        assert {s for _, s, _ in launches} == {launches[0][1]}, (n, launches)
        if n > 2048:
            assert launches[0][1:] == (1, 0)


def test_few_long_rows_are_split():
    (rows, splits, ws), = dl.score_launches(3, 126464, 20)
    assert rows == 3 and splits > 2 and ws == 3 * splits * (16 + 16 * 10)


def test_no_rows_and_refusals():
    assert dl.score_launches(0, 100, 0) == []
    for bad in ((-1, 100, 0), (1, 1, 0), (1, 100, 65), (1, 5, 6), (1, 100, -1)):
        with pytest.raises(dl.DlmcError) as e:
            dl.score_launches(*bad)
        assert e.value.code == -1
