"""The head's calls in several chunks of tokens: by a chunk's statistics, by its 16-bit numbers, by its most rows."""

import pytest
import torch

from tests import test_gpu_linear_xent as T
from tests.gpu_util import flush
from tests.test_head_workspace import LOOSE, _ws

pytestmark = pytest.mark.gpu
BF, F4 = torch.bfloat16, torch.float32


def test_scores_in_chunks():
    """More rows than the statistics of the widest vocabulary allow in one chunk."""
    N, V, d = 9000, 1 << 20, 64
    flush("scores in chunks", N, V, d)
    shared = lambda n: _ws(N=n, V=V, d=d) - (2 * d + 16) * n  # noqa: E731
    assert abs(shared(N) - shared(4608)) < LOOSE  # two chunks: half the rows, in whole tiles
    i = T._inputs(N, V, d, 0.1, "plain")
    o = T._outputs(i, grads="")
    T._call(i, o)
    torch.cuda.synchronize()
    live = (i["labels"] >= 0) & (i["labels"] < V)
    assert o["inv_n"].item() == pytest.approx(1 / int(live.sum()), rel=2.0 ** -23)
    for at in torch.arange(N, device="cuda").split(1000):
        rows = {k: i[k][at] for k in ("x", "labels")}
        want = T._want({**i, **rows}, False)
        T._check({k: o[k][at] for k in ("row_loss", "lse")}, want)
