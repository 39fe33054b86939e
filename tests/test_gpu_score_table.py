"""The gradient of the table of scored attention, where pairs lie beyond the table's reach: by calls that hold every key of
a row, and by calls that hold some of them."""
import numpy as np
import pytest
import torch

import oracle
from tests import _score
from tests._gpu import HAVE_GPU, api, to64
from tests._score import Inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="needs a GPU")]
DEV = "cuda:0"


def final(x):
    """The exact out and lse, as a forward stores them."""
    ref = oracle.score_forward(x.d, x.ref, *x.f64(), x.scale)
    return torch.from_numpy(ref["out"]).to(torch.bfloat16), torch.from_numpy(ref["lse"]).float()


@pytest.mark.parametrize("score", [dict(buckets=32), dict(buckets=16, two_sided=False, reach=40, bias_type=torch.float32),
                                   dict(buckets=32, cap=10.0, sharp=2.0, causal=True)], ids=["two-sided", "one-sided", "cap causal"])
@pytest.mark.parametrize("hd", [64, 128])
def test_one_block_at_a_time(hd, score):
    """A backward of one block of a shard a call, from the final out and lse: each block's share by the formulas, for rows
    that have most, some and next to none of their weight there."""
    ends, rank = (0, 400, 800, 1200, 1230), 1
    x = Inputs(_score.shard(rank, ends), 2, 1, hd, 41, DEV, **score)
    out, lse = final(x)
    n = ends[rank + 1] - ends[rank]
    for a, b in zip(ends, ends[1:]):
        d = _score._descs.desc((0, n), [1], [0], [1], (0, b - a), [0], 1, q_offset=[ends[rank]], k_offset=[a])
        k, v = (t[a:b].contiguous() for t in x.dev[1:])
        got = api.score_bwd(api.SegDesc.of(d), x.score, x.dev[0], k, v, out.to(DEV), lse.to(DEV), x.do_dev, x.scale)
        want = oracle.score_backward(d, x.ref, to64(x.q), to64(k), to64(v), to64(x.do), x.scale, to64(out), lse.double().numpy())
        for name, t in zip(("dq", "dk", "dv", "dbias"), got):
            _score.check(f"{name} of [{a}, {b})", t, want[name], want["tol_" + name])
