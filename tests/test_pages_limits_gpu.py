"""Forking and compaction of pages on both sides of what the one launch takes: rows, pages, table entries."""
import numpy as np
import pytest

from tests.test_kv4_gpu import PAGE, check_compact, check_fork, page_case, thi  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,out,MP,P", [(1024, 1024, 3, 4000), (1025, 1024, 3, 4000), (1024, 1025, 3, 4000), (60, 90, 6, 8192), (60, 90, 6, 8193),
                                           (256, 256, 128, 3000), (257, 256, 128, 3000), (255, 258, 128, 3000)])
def test_fork_limits(thi, rows, out, MP, P):  # noqa: F811
    c = page_case(rows + P, rows, MP, P, min(MP, 6) * PAGE, words=4, layers=1)
    rng = c["rng"]
    check_fork(thi, c, rng.integers(-1, rows + 1, out), rng.integers(-3, 200, out), "limits")
    check_fork(thi, c, np.arange(out) % rows, None, "limits, no headroom")


@pytest.mark.parametrize("rows,MP,P", [(60, 6, 16384), (60, 6, 16385), (1024, 4096, 3000), (1025, 4096, 3000)])
def test_compact_limits(thi, rows, MP, P):  # noqa: F811
    c = page_case(rows + P, rows, MP, P, 3 * PAGE, words=4, layers=2)
    assert check_compact(thi, c, "limits")
