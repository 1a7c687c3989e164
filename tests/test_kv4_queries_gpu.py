"""Attention over the 4-bit cache: queries reach the products as four summands, weights of up to 64 rows of a cache head as two, all of them."""
import numpy as np
import pytest

from tests import kv4_bounds as bounds
from tests.gpu_common import say
from tests.test_kv4_gpu import attention_case, run_attention, thi  # noqa: F401

pytestmark = pytest.mark.gpu


def check(thi, c, scale, decode, what, **how):
    y, tol = bounds.attention(c, scale, **how)
    say(f"[case] {what} rows={np.diff(c['offsets']).tolist()[:6]} q={c['q'].shape}")
    got = run_attention(thi, c, scale, decode)
    err = np.abs(got - y)
    worst = np.unravel_index((err / tol).argmax(), err.shape)
    assert (err <= tol).all(), f"{(err / tol).max():.3g} of the tolerance at {worst}: {got[worst]}, exact {y[worst]}"


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,lens,new", [
    (4, 2, [2] * 40, [1] * 40),                          # one token a request
    (16, 1, [3] * 12, [1] * 12),
    (4, 2, [4] * 12, [3] * 12),                          # a few
    (8, 1, [8] * 3, [8] * 3),
    (8, 1, [12] * 3, [12] * 3),                          # a prompt
    (34, 2, [9] * 3, [9] * 3),
])
def test_small_columns_beside_a_large_one(thi, Hq, Hkv, lens, new, D):  # noqa: F811
    """What three summands leave of such a query moves a score by half."""
    c = bounds.far_queries(Hq + D + new[0], Hq, Hkv, D, lens, new)
    rows = max(new) * Hq // Hkv
    check(thi, c, 0.125, max(new) == 1, "a large column", weight=bounds.TWO_SUMMANDS if rows <= 64 else bounds.ONE_SUMMAND)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,lens,new", [(4, 2, [2, 3, 4, 5, 7, 9, 12, 16] * 3, [1] * 24), (8, 1, [3, 4, 5, 6, 9], [3] * 5), (8, 2, [8, 11, 16], [8] * 3)])
def test_weights_of_few_rows(thi, Hq, Hkv, lens, new, D):  # noqa: F811
    """Queries and scale that lose nothing on the way: what is left is the weights' rounding, which shows where values nearly cancel."""
    c, scale = bounds.whole_queries(attention_case(D + new[0], Hq, Hkv, D, lens, new))
    check(thi, c, scale, max(new) == 1, "weights", weight=bounds.TWO_SUMMANDS, query=0.0)
