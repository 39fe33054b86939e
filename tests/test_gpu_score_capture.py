"""What a captured call of scored attention needs of the eager call in front of it."""
import numpy as np
import pytest
import torch

from tests import _score
from tests._gpu import HAVE_GPU, api
from tests._score import Inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="needs a GPU")]
DEV = "cuda:0"


def step(x, s, grad=True):
    out, lse, _, _ = api.score_fwd(x.desc, s, *x.dev, x.scale)
    return [t for t in (out, lse, *api.score_bwd(x.desc, s, *x.dev, out, lse, x.do_dev, x.scale, bias_grad=grad and s.bias is not None))
            if t is not None]


@pytest.mark.parametrize("d", [_score.whole([211, 40]), _score.shard(1, (0, 603, 901, 1400))], ids=["whole", "shard"])
def test_captured_with_another_score_than_the_eager_call(d):
    """The schedule and the buckets are those of the eager calls, cap, slope, table and key intervals others."""
    x = Inputs(d, 4, 2, 64, 71, DEV, buckets=32)
    n = d["cu_seqlens_q"][-1]
    bias = x.score.bias
    lo = torch.as_tensor(np.arange(n) % 7, dtype=torch.int32, device=DEV)
    hi = torch.as_tensor(np.arange(n) % 90 + d["q_offset"][0], dtype=torch.int32, device=DEV)
    slope = torch.tensor([0.5, 0.25, 0.125, 0.0], device=DEV)
    step(x, api.Score(bias=bias))
    step(x, api.Score(bias=bias), grad=False)
    for make in (lambda: api.Score(bias=(-bias).float(), cap=15.0, key_hi=hi), lambda: api.Score(slope=slope, key_lo=lo, key_hi=hi),
                 lambda: api.Score(cap=30.0)):
        s = make()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = step(x, s)
        want = None
        for _ in range(3):
            g.replay()
            want = step(x, s)
            torch.cuda.synchronize()
            assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
