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


def test_buckets_beyond_the_reach_do_not_take_the_rounding_of_out():
    """198 rows of 994 keys, one head: D from an out in bf16 puts the table's gradient off by 0.76% (the oracle's 0.0109 of
    1.434), nearly all of it in the two buckets beyond the reach.  There a row's D is what makes its dA add up to zero, which
    leaves the error of pairs nearer than that (0.06%, by the oracle) and the roundings of P (the absolute dA come to 890 times
    the gradient: 2^-20 of each, all of one sign, to 0.09%)."""
    ends, rank = (0, 400, 598, 994), 1
    x = Inputs(_score.shard(rank, ends), 1, 1, 64, 42, DEV, buckets=32, bias_type=torch.float32)
    out, lse = final(x)
    given = to64(out), lse.double().numpy()
    q, k, v = x.f64()
    exact = oracle.score_backward(x.d, x.ref, q, k, v, to64(x.do), x.scale)["dbias"]
    parts = 0.0  # dA by the given out throughout: the shares of calls of one block
    for a, b in zip(ends, ends[1:]):
        d = _score._descs.desc((0, 198), [1], [0], [1], (0, b - a), [0], 1, q_offset=[ends[rank]], k_offset=[a])
        parts = parts + oracle.score_backward(d, x.ref, q, k[a:b], v[a:b], to64(x.do), x.scale, *given)["dbias"]
    off = np.linalg.norm(parts - exact)
    assert off > 0.007 * np.linalg.norm(exact)
    got = api.score_bwd(x.desc, x.score, *x.dev, out.to(DEV), lse.to(DEV), x.do_dev, x.scale)[3]
    assert np.linalg.norm(to64(got) - exact) < off / 4


@pytest.mark.parametrize("cap", [0.0, 10.0])
@pytest.mark.parametrize("hd", [64, 128])
def test_gradients_with_the_tables_do_not_depend_on_the_launch(hd, cap):
    """Four segments of 512 rows and 12 heads, 384 items of dQ and dK/dV (two launches with d = 128, one with 64), against each
    on its own, 96 items in one launch: the same bits, and a table's gradient that is the sum of theirs."""
    x = Inputs(_score.whole([512] * 4), 12, 12, hd, 43, DEV, buckets=32, cap=cap, causal=True, bias_type=torch.float32)
    out, lse, _, _ = api.score_fwd(x.desc, x.score, *x.dev, x.scale)
    got = api.score_bwd(x.desc, x.score, *x.dev, out, lse, x.do_dev, x.scale)
    total = 0.0
    for i in range(4):
        part = [t[512 * i:512 * (i + 1)].contiguous() for t in (*x.dev, out, lse, x.do_dev)]
        one = api.score_bwd(api.SegDesc.of(_score.whole([512])), x.score, *part, x.scale)
        for n, s, t in zip(("dq", "dk", "dv"), got, one):
            assert torch.equal(s[512 * i:512 * (i + 1)], t), (n, i)
        total = total + one[3].double()
    # fp32 sums of the same items, of 16 a head here and of 4 there, with a rounding each
    assert ((got[3].double() - total).abs() <= 20 * 2.0 ** -24 * 4 * total.abs().max()).all()
