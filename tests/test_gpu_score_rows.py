"""Rows of scored attention that see nothing, and rows whose gradients are no numbers: what they reach, and what they do not."""
import numpy as np
import pytest
import torch

import oracle
from tests import _score
from tests._gpu import HAVE_GPU, api, to64
from tests._score import Inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="needs a GPU")]
DEV = "cuda:0"
NAN, INF = float("nan"), float("inf")


def by_table(make, what):
    """An input whose table masks: bucket 0 of head 1, which holds a row's own key and those behind it (the first row of a
    segment sees nothing), or all of head 1."""
    x = make(buckets=16, two_sided=False, reach=40, bias_type=torch.float32)
    for t in (x.ref["bias"], x.score.bias):
        t[0 if what == "bucket" else slice(None), 1] = -INF
    return x


@pytest.mark.parametrize("cap", [0.0, 10.0])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("what,d,H", [("bucket", _score.whole([150, 40, 1, 1]), 4), ("head", _score.whole([150, 40, 1]), 4),
                                      ("head", _score.whole([300]), 24), ("head", _score.shard(1, (0, 700, 1100, 1800)), 4)],
                         ids=["bucket", "head", "many", "shard"])
def test_rows_that_a_table_leaves_without_a_key(what, d, H, causal, hd, cap):
    """Such rows have an output of zero, whatever V holds, and no part in a gradient, whatever q, out and dout hold there."""
    x = by_table(lambda **kw: Inputs(d, H, 2, hd, 51, DEV, causal=causal, cap=cap, **kw), what)
    out, lse, ref = _score.forward(x)
    none = torch.isinf(lse)
    assert none[:, 1].any() and not none[:, [0, 2]].any()
    at = np.flatnonzero(ref["lse"][:, 1] == -np.inf)
    want = oracle.score_backward(x.d, x.ref, *x.f64(), to64(x.do), x.scale, to64(out), lse.cpu().double().numpy())
    q, k, v = x.dev
    for t, val in ((q, NAN), (out, INF), (x.do_dev, NAN)):
        t[none] = val
    for grad in (True, False):  # without the table's gradient a shard's keys are shared by two groups of waves
        got = api.score_bwd(x.desc, x.score, q, k, v, out, lse, x.do_dev, x.scale, bias_grad=grad)
        for n, t in zip(("dq", "dk", "dv", "dbias"), got):
            if t is not None:
                _score.check(n, t, want[n], want["tol_" + n])
        assert not got[0][torch.as_tensor(at, device=DEV), 1].any()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("few", [False, True])
def test_outputs_of_rows_that_a_table_leaves_without_a_key(few, hd):
    """Infinities in V do not reach them, of a block that no mask runs through."""
    d = _score.tokens([3], [500]) if few else _score.whole([200])
    x = by_table(lambda **kw: Inputs(d, 4, 2, hd, 52, DEV, **kw), "head")
    x.dev[2][7], x.dev[2][77, 0, 3] = INF, NAN
    out, lse, _, _ = api.score_fwd(x.desc, x.score, *x.dev, x.scale)
    assert not out[:, 1].any() and (lse[:, 1] == -INF).all() and torch.isinf(out[:, 0]).any()
    if few:
        _, _, op, lp = api.score_fwd(x.desc, x.score, *x.dev, x.scale, partials=True)
        assert not op[:, :, 1].any() and (lp[:, :, 1] == -INF).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window", [False, True])
@pytest.mark.parametrize("score", [{}, dict(cap=10.0), dict(slope=True), dict(buckets=32, bias_type=torch.float32),
                                   dict(buckets=32, bias_type=torch.float32, cap=10.0)],
                         ids=["plain", "cap", "slope", "bucket", "cap bucket"])
def test_rows_without_a_gradient_reach_only_what_they_see(score, window, hd):
    """An infinity or a NaN in dout of a row: its own dq and the dk of the keys that it sees are no numbers, all others' are
    as if the row had no gradient, and so are the table's buckets that hold none of its pairs."""
    n, bad = 300, {70: INF, 131: NAN, 200: -INF}
    p = np.arange(n)
    masks = dict(lo=p - 33, hi=p + 1) if window else {}
    x = Inputs(_score.whole([n]), 2, 2, hd, 53, DEV, causal=True, **masks, **score)
    out, lse, _ = _score.forward(x)
    do = x.do_dev.clone()
    for i, val in bad.items():
        do[i, 0, i % hd] = val
    got = api.score_bwd(x.desc, x.score, *x.dev, out, lse, do, x.scale)
    x.do[list(bad), 0] = 0
    want = oracle.score_backward(x.d, x.ref, *x.f64(), to64(x.do), x.scale, to64(out), lse.cpu().double().numpy())
    rows = np.ones((n, 2), bool)
    rows[list(bad), 0] = False
    keys = np.ones((n, 2), bool)
    for i in bad:
        keys[max(0, i - 33 if window else 0):i + 1, 0] = False
    for name, t, at in (("dq", got[0], rows), ("dk", got[1], keys), ("dv", got[2], keys)):
        _score.check(name, t[torch.as_tensor(at, device=DEV)], want[name][at], want["tol_" + name][at])
        hit = t[torch.as_tensor(~at, device=DEV)]
        assert not torch.isfinite(hit).all(-1).any() if name != "dv" else not torch.isfinite(hit).all()
    if got[3] is not None:
        assert not got[3][17:].any()  # keys behind their rows: none is seen
        _score.check("dbias", got[3][:, 1], want["dbias"][:, 1], want["tol_dbias"][:, 1])
        if window:
            assert not got[3][13:16, 0].any()  # keys 46 positions and more in front of their rows
