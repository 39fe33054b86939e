"""The bounds that the GPU tests of scored attention hold the table's gradient to are far below the gradient itself, in the
buckets of the table's ends too: zeros or a wrong sign there do not pass."""
import numpy as np
import pytest
import torch

import oracle
from tests import _score
from tests._gpu import to64
from tests._score import Inputs

WHOLE = lambda: _score.whole([200, 1, 0, 77, 333])  # noqa: E731


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("d,kw", [
    (WHOLE, dict(buckets=32)),
    (WHOLE, dict(buckets=16, two_sided=False, reach=40, bias_type=torch.float32)),
    (WHOLE, dict(buckets=32, cap=10.0, sharp=2.0)),
    (lambda: _score.shard(1, (0, 130, 300, 300, 470)), dict(buckets=32)),
    (lambda: _score.shard(1, (0, 400, 598, 994)), dict(buckets=16, reach=64)),
], ids=["whole", "one-sided", "cap", "shard", "long shard"])
def test_gradients_of_the_tables_ends_stand_above_their_bounds(d, kw, hd):
    x = Inputs(d(), 4, 2, hd, 11, "cpu", **kw)
    ref = oracle.score_forward(x.d, x.ref, *x.f64(), x.scale)
    out, lse = to64(torch.from_numpy(ref["out"]).to(torch.bfloat16)), ref["lse"].astype(np.float32).astype(np.float64)
    got = oracle.score_backward(x.d, x.ref, *x.f64(), to64(x.do), x.scale, out, lse)
    nb = x.ref["bias"].shape[0]
    ends = [nb // 2 - 1, nb - 1] if x.ref["two_sided"] else [nb - 1]
    times = np.abs(got["dbias"][ends]) / got["tol_dbias"][ends]
    assert np.median(times) > 4 and (times > 1).mean() >= 0.75, times
