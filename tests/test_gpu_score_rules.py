"""Scored attention on both sides of the sizes at which its kernels change, against the fp64 oracle."""
import numpy as np
import pytest
import torch

from tests import _score
from tests._gpu import HAVE_GPU, api
from tests._score import Inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="needs a GPU")]
DEV = "cuda:0"


@pytest.mark.parametrize("score", [dict(causal=True), dict(slope=True), dict(buckets=32, cap=10.0)], ids=["causal", "slope", "cap bucket"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("keys", [511, 512, 513, 639, 640, 641])
def test_shards_around_the_keys_that_two_groups_of_waves_share(keys, hd, score):
    """From 512 keys on two groups of waves share the keys of an item (without the table's gradient, in the backward); of
    partials, from 512 a block."""
    ends = (0, 300, keys)
    x = Inputs(_score.shard(1, ends), 2, 1, hd, 81, DEV, **score)
    _, _, ref = _score.forward(x)
    got, want = _score.backward(x)
    out, lse = torch.from_numpy(ref["out"]).to(DEV, torch.bfloat16), torch.from_numpy(ref["lse"]).to(DEV, torch.float32)
    dq, dk, dv, _ = api.score_bwd(x.desc, x.score, *x.dev, out, lse, x.do_dev, x.scale, bias_grad=False)
    _score.check("dq", dq, want["dq"], want["tol_dq"])
    assert torch.equal(dk, got[1]) and torch.equal(dv, got[2])
    y = Inputs(_score.shard(0, (0, keys, 2 * keys - 1)), 2, 1, hd, 82, DEV, **score)  # a key less than two blocks of that many
    _, _, op, lp = api.score_fwd(y.desc, y.score, *y.dev, y.scale, partials=True)
    _, _, ref = _score.forward(y)
    _score.check("o_part", op, ref["o_part"], ref["tol_o_part"])
    _score.check("lse_part", lp, ref["lse_part"], ref["tol_lse_part"])


@pytest.mark.parametrize("H", [128, 129])
def test_shards_around_the_items_that_two_groups_of_waves_share(H):
    """130 rows, two tiles: 256 items of 128 heads are shared, 258 of 129 are not."""
    x = Inputs(_score.shard(1, (0, 400, 530)), H, H, 64, 83, DEV, causal=True, slope=False)
    _score.forward(x)
    _score.backward(x)


@pytest.mark.parametrize("score", [dict(slope=True), dict(buckets=32, cap=10.0)], ids=["slope", "cap bucket"])
@pytest.mark.parametrize("rows,keys,G", [(32, 300, 1), (33, 300, 1), (16, 300, 2), (17, 300, 2), (33, 2047, 1), (33, 2048, 1),
                                         (256, 2048, 1), (257, 2048, 1), (64, 2048, 4), (65, 2048, 4), (1, 639, 1), (1, 640, 1),
                                         (1, 641, 1), (2, 4096, 2), (2, 4097, 2), (1, 32768, 1), (1, 32769, 1)])
def test_tokens_around_the_sizes_of_the_kernel_for_few_rows(rows, keys, G, score):
    """Up to 32 rows of a K/V head, or 256 against 2048 keys and more; one chunk up to 640 keys, chunks of 256 doubled while
    16 of them are less than the keys."""
    pos = np.arange(rows) + keys - rows - keys // 9
    x = Inputs(_score.tokens([rows], [keys]), G, 1, 64, 84, DEV, causal=True, q_pos=pos, **score)
    _score.forward(x)


@pytest.mark.parametrize("rows,keys,G", [(255, 600, 2), (256, 600, 2), (479, 480, 2), (481, 480, 2), (720, 100, 3)])
def test_gradients_around_the_rows_that_divide_a_group_s_heads(rows, keys, G):
    """dK and dV in parts of some of a group's heads, from 256 rows and 480 that the parts save."""
    d = _score.shard(0, (0, rows)) if rows == keys else dict(_score.shard(0, (0, keys)), cu_seqlens_q=(0, rows), q_offset=(keys // 2,))
    x = Inputs(d, G, 1, 64, 85, DEV, causal=True, cap=20.0)
    _score.forward(x)
    _score.backward(x)
