"""Attention over the 4-bit cache where a request has more rows than max_q says: the first max_q are what they are in a call with all rows, the others are not written."""
import numpy as np
import pytest

from tests import kv4_reference as ref
from tests.gpu_common import say
from tests.test_kv4_gpu import PAGE, attention_case, run_attention, thi  # noqa: F401

pytestmark = pytest.mark.gpu


def check(thi, c, max_q, what):
    scale = c["q"].shape[2] ** -0.5
    say(f"[case] {what} max_q={max_q} rows={np.diff(c['offsets']).tolist()} lens={c['lens'].tolist()}")
    y, S, E = ref.attention(c["q"], c["pages"], c["table"], c["lens"], c["offsets"], scale)
    tol = ref.attention_tolerance(y, S, E, c["q"].shape[2], c["table"].shape[1] * PAGE)
    got = run_attention(thi, c, scale, max_q=max_q)
    for b, (first, end) in enumerate(zip(c["offsets"][:-1], c["offsets"][1:])):
        last = min(first + max_q, end)
        assert np.array_equal(np.isnan(got[first:last]), np.isnan(y[first:last])), b
        fine = ~np.isnan(y[first:last])
        assert (np.abs(got[first:last] - y[first:last]) <= tol[first:last])[fine].all(), b
        assert (got[last:end] == 777).all(), b


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("max_q,lens,new", [
    (1, [3, 70, 1, 64, 2], [3, 2, 3, 1, 5]),             # one row of each, some of which see nothing
    (3, [80, 5, 2, 130], [5, 5, 4, 2]),                  # a few
    (90, [200, 120, 95, 64, 20], [120, 120, 100, 90, 120]),      # prompts
])
def test_more_rows_than_max_q(thi, max_q, lens, new, D):  # noqa: F811
    check(thi, attention_case(max_q + D, 4, 2, D, lens, new), max_q, "rows past max_q")


@pytest.mark.parametrize("max_q,new", [(1, 3), (3, 5), (90, 97)])
def test_what_only_unwritten_rows_see_does_not_matter(thi, max_q, new):  # noqa: F811
    """Not a number at the positions of the rows that are not written."""
    c = attention_case(7, 4, 2, 128, [190, 100], [new, new])
    nan = np.full((2, 128), np.nan)
    for pos in range(190 - new + max_q, 190):
        ref.store(c["pages"], int(c["table"][0, pos // PAGE]) * PAGE + pos % PAGE, nan, nan)
    check(thi, c, max_q, "NaN behind")
