"""Attention over the 4-bit cache where requests are cut into chunks of pages: several new tokens, prompts, rows that see nothing of a chunk, chunks without a
page, NaN in one of them."""
import numpy as np
import pytest

from tests import kv4_reference as ref
from tests.gpu_common import say
from tests.test_kv4_gpu import PAGE, attention_case, dev, host, thi  # noqa: F401

pytestmark = pytest.mark.gpu


def check(thi, c, what, rows=None):
    """Against the definition, and that chunks met in the workspace; `rows`: those that are compared."""
    import torch
    T, Hq, D = c["q"].shape
    B, MP = c["table"].shape
    Hkv, max_q, scale = c["pages"].shape[1], int(np.diff(c["offsets"]).max()), D ** -0.5
    say(f"[case] chunks {what} Hq={Hq} Hkv={Hkv} D={D} lens={c['lens'].tolist()} rows={np.diff(c['offsets']).tolist()}")
    y, S, E = ref.attention(c["q"], c["pages"], c["table"], c["lens"], c["offsets"], scale)
    tol = ref.attention_tolerance(y, S, E, D, MP * PAGE)
    ws = thi.Workspace(thi.thi_kv4_attention_workspace_bytes(B, T, Hq, Hkv, D, max_q, MP), init=False)
    ws.buffer.fill_(255)
    args = [dev(c[k]) for k in ("q", "pages", "table", "lens", "offsets")]
    outs = []
    for _ in range(2):
        outs.append(torch.full((T + 1, Hq, D), 777.0, dtype=torch.float16, device="cuda"))
        thi.thi_kv4_attention(*args, scale, outs[-1][:T], max_q, ws)
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16)), "two runs differ"
    assert bool((ws.buffer != 255).any()), "no chunks"
    got = host(outs[0].double())
    assert (got[T] == 777).all()
    got = got[:T]
    assert np.array_equal(np.isnan(got), np.isnan(y))
    fine = ~np.isnan(y)
    assert (np.abs(got - y) <= tol)[fine].all(), f"worst {(np.abs(got - y) / tol)[fine].max():.3g} of the tolerance"
    return y


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,lens,new", [
    (4, 2, [1300, 200, 0, 515], [3, 3, 3, 1]),            # a few new tokens next to one, of long and short requests
    (16, 2, [2100], [8]),                                 # four tiles of rows
    (6, 2, [1029, 1150], [5, 0]),
    (2, 2, [2200, 300, 1090], [90, 33, 70]),              # chunks of prompts
    (16, 1, [1500, 2], [12, 1]),
    (1, 1, [1100], [1100]),                               # a prompt, whose first rows see nothing of the later chunks
])
def test_chunks(thi, Hq, Hkv, lens, new, D):  # noqa: F811
    check(thi, attention_case(Hq + D + lens[0], Hq, Hkv, D, lens, new), "plain")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,new", [(4, 2, 1), (4, 2, 3), (4, 2, 70)])
def test_chunks_without_pages_and_with_nan(thi, Hq, Hkv, new, D):  # noqa: F811
    lens = [2200, 1900, 1500]
    c = attention_case(new + D, Hq, Hkv, D, lens, [new] * 3)
    c["table"][0, 3:31] = -1                              # whole chunks of every plan
    c["table"][1, :] = [-1, len(c["pages"])][new > 1]
    check(thi, c, "missing pages")
    nan = np.full((Hkv, D), np.nan)
    k, v = ref.load(c["pages"], int(c["table"][2, 20]) * PAGE + 9)
    v[:, 40] = np.nan
    ref.store(c["pages"], int(c["table"][2, 20]) * PAGE + 9, k, v)      # one block of a value in a later chunk
    y = check(thi, c, "a value that is not a number")
    assert np.isnan(y).any() and not np.isnan(y[:, :, 0]).any()
    if new > 1:                                           # seen by the last row alone
        pos = lens[2] - 1
        ref.store(c["pages"], int(c["table"][2, pos // PAGE]) * PAGE + pos % PAGE, nan, nan)
        y = check(thi, c, "NaN for the last row")
        assert np.isnan(y[-1]).all() and not np.isnan(y[-2, :, 0]).any()
