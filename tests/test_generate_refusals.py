"""What appending, attending, reordering and selecting refuse before any launch (CPU)."""
import pytest

import paper_2403_09636_gb300 as P
from paper_2403_09636_gb300 import build as B


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()


def test_null_handles():
    assert P.dmc_cache_append(None, 0, 0, 1, 16, 16, 16, None, 1, 1, None, None, 0, None, 0) == P.DMC_ERR_INVALID_ARG
    assert P.dmc_cache_attend(None, 0, 16, 32, 0) == P.DMC_ERR_INVALID_ARG
    assert P.dmc_cache_reorder(None, 0, 1, 16, 0) == P.DMC_ERR_INVALID_ARG
    assert P.dmc_beam_select(None, 16, 8, 16, None, -1, 16, 16, 16, 16, 0) == P.DMC_ERR_INVALID_ARG
    assert P.dmc_beam_destroy(None) == P.DMC_OK


@pytest.mark.parametrize("bad", [(0, 1, 1, 10, 0), (1, 0, 1, 10, 0), (1, 33, 1, 10, 0), (1, 1, 0, 10, 0), (1, 1, 33, 100, 0),
                                 (1, 2, 7, 3, 0), (1, 1, 1, 0, 0), (1, 1, 1, (1 << 28) + 1, 0), (1, 1, 1, 10, 2),
                                 ((1 << 20) + 1, 1, 1, 10, 0)])
def test_selections_that_need_zero_bytes(bad):
    assert P.dmc_beam_required_bytes(P.dmc_beam_config(*bad)) == 0


def test_selection_sizes():
    """Scratch: lists of `keep` 8-byte keys and one 8-byte pair for each piece of a row; a counter for each group."""
    need = lambda *c: P.dmc_beam_required_bytes(P.dmc_beam_config(*c))  # noqa: E731
    assert need(1, 1, 1, 1, 0) == 3 * 256
    assert need(1, 2, 6, 3, 1) > 0  # beams x vocab continuations may all be kept
    rows, keep = 4096, 32
    assert need(rows // 32, 32, keep, 32000, 1) == pytest.approx(rows * (keep + 1) * 8, rel=0.01)  # rows of one piece
    assert need(1 << 20, 32, 32, 50, 0) > 8 << 30  # passes 32 bits


def test_create_refuses_bad_arenas():
    cfg = P.dmc_beam_config(1, 4, 4, 1000, 1)
    n = P.dmc_beam_required_bytes(cfg)
    assert P.dmc_beam_create(cfg, 0, n, 0)[0] == P.DMC_ERR_INVALID_ARG
    assert P.dmc_beam_create(cfg, 4096 + 16, n, 0)[0] == P.DMC_ERR_INVALID_ARG
    assert P.dmc_beam_create(cfg, 4096, n - 1, 0)[0] == P.DMC_ERR_ARENA_TOO_SMALL
    assert P.dmc_beam_create(P.dmc_beam_config(1, 40, 4, 1000, 1), 4096, n, 0)[0] == P.DMC_ERR_INVALID_ARG
