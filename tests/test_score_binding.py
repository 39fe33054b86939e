"""What a call of scored attention takes of a ``Score``: the tensors that it holds then."""
import numpy as np
import pytest
import torch

from paper_2608_01150_amd import api
from tests import _score
from tests._score import Inputs

FIELDS = dict(slope=torch.float32, bias=torch.bfloat16, key_lo=torch.int32, key_hi=torch.int32, q_pos=torch.int32)


@pytest.mark.parametrize("name", FIELDS)
def test_a_tensor_whose_storage_is_swapped(name):
    make = lambda: torch.ones((8, 4) if name == "bias" else 8, dtype=FIELDS[name])  # noqa: E731
    t = make()
    s = api.Score(**{name: t})
    for change in (lambda: setattr(t, "data", make()), lambda: t.set_(make()), lambda: setattr(s, name, make())):
        change()
        s.ptr()
        assert getattr(s.c, name) == getattr(s, name).data_ptr()
    setattr(s, name, None)
    s.ptr()
    assert getattr(s.c, name) is None


def test_what_takes_a_tensor_s_place_is_checked():
    d = api.SegDesc.of(_score.whole([8]))
    q, s = torch.zeros((8, 4, 64), dtype=torch.bfloat16), api.Score(bias=torch.zeros((32, 4)), key_lo=torch.zeros(8, dtype=torch.int32))
    for name, t, needle in (("bias", torch.zeros((4, 32)).t(), "contiguous"), ("bias", torch.zeros(4), "bias must be"),
                            ("bias", torch.zeros((16, 2)), "bias has shape"), ("key_lo", torch.zeros(7, dtype=torch.int32), "key_lo has shape"),
                            ("key_lo", torch.zeros(8), "key_lo has dtype"), ("slope", torch.zeros(3), "slope has shape")):
        old = getattr(s, name)
        setattr(s, name, t)
        with pytest.raises(api.ZlError) as e:
            api.score_fwd(d, s, q, q, q, 1.0)
        assert e.value.status == api.ZL_ERR_INVALID_ARG and needle in str(e.value)
        setattr(s, name, old)
    s.bias = torch.zeros((16, 4), dtype=torch.bfloat16)
    s.ptr()
    assert s.c.num_buckets == 16 and s.c.bias_dtype == api.ZL_BF16


@pytest.mark.parametrize("by", [dict(causal=True), dict(window=4), dict(documents=[[0, 25]])])
def test_intervals_of_a_shard_need_its_position(by):
    d = dict(_score.shard(1, (0, 20, 40)))
    lo, hi = api.key_intervals(api.SegDesc.of(d), **by)
    assert hi[7] == (28 if "causal" in by else 1 << 30) and lo[7] == (24 if "window" in by else 25 if "documents" in by else 0)
    d["q_offset"] = None
    with pytest.raises(api.ZlError) as e:
        api.key_intervals(api.SegDesc.of(d), **by)
    assert e.value.status == api.ZL_ERR_INVALID_ARG and "q_offset" in str(e.value)
    lo, hi = api.key_intervals(api.SegDesc.of(d), prefix=[7])  # the same for every row
    assert set(lo.tolist()) == {0} and set(hi.tolist()) == {1 << 30}


def test_intervals_of_a_shard_in_front_of_the_last_positions():
    """A shard's rows are placed by q_offset; its first block may end at position 2^30 with fewer keys than it has rows."""
    top = 1 << 30
    d = dict(_score.shard(0, (0, 20, 40)), cu_seqlens_q=(0, 30), q_offset=(100,), k_offset=(top - 20, 0))
    lo, hi = api.key_intervals(api.SegDesc.of(d), causal=True)
    assert lo[0] == 0 and hi[0] == 101 and hi[29] == 130
    for over in (dict(q_offset=(top - 29,)),):
        with pytest.raises(api.ZlError) as e:
            api.key_intervals(api.SegDesc.of(dict(d, **over)), causal=True)
        assert e.value.status == api.ZL_ERR_UNSUPPORTED
    w = dict(_score.whole([20]), q_offset=None, k_offset=(top - 19,))
    with pytest.raises(api.ZlError):
        api.key_intervals(api.SegDesc.of(w), causal=True)


def test_a_shard_s_chain_works_on_its_tensors_device(monkeypatch):
    """Partials, merge and backward of tensors on another GPU than the current one: each call makes theirs current.  The
    library and the devices are stand-ins."""
    here, calls = [0], []

    class Device:
        def __init__(self, device):
            self.index = device.index

        def __enter__(self):
            here.append(self.index)

        def __exit__(self, *_):
            here.pop()

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: here[-1], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(api, "_stream", lambda device: 0)
    for name in ("_score_ws", "_score_fwd", "_score_bwd", "_merge", "_merge_ex"):
        monkeypatch.setattr(api, name, lambda *_, name=name: calls.append((name, here[-1])) or api.ZL_OK)
    d = api.SegDesc.of(_score.shard(1, (0, 20, 40)))
    q, lse = torch.zeros((20, 2, 64), dtype=torch.bfloat16), torch.zeros((20, 2))
    k, op, lp = torch.zeros((40, 2, 64), dtype=torch.bfloat16), torch.zeros((2, 20, 2, 64)), torch.zeros((2, 20, 2))
    ws, s = torch.zeros(256, dtype=torch.uint8), api.Score()
    for gpu in (1, 0):
        monkeypatch.setattr(api, "_same_gpu", lambda *_, gpu=gpu: torch.device("cuda", gpu))
        calls.clear()
        api.score_fwd(d, s, q, k, k, 1.0, out=q, lse=lse, o_part=op, lse_part=lp, workspace=ws)
        api.lse_merge(d, op, lp, q, lse)
        api.lse_merge(d, op.bfloat16(), lp, q, lse)
        api.score_bwd(d, s, q, k, k, q, lse, q, 1.0, dq=q, dk=k, dv=k, workspace=ws)
        assert calls == [(n, gpu) for n in ("_score_fwd", "_merge", "_merge_ex", "_score_bwd")]


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
def test_a_call_reads_the_swapped_storage():
    x = Inputs(_score.whole([90]), 2, 2, 64, 61, "cuda:0", buckets=32, hi=np.arange(90) + 1)
    call = lambda s: api.score_fwd(x.desc, s, *x.dev, x.scale)[0]  # noqa: E731
    first = call(x.score)
    x.score.bias.data = -x.score.bias
    x.score.key_hi = x.score.key_hi - 1
    want = call(api.Score(bias=x.score.bias.clone(), key_hi=x.score.key_hi.clone(), key_lo=x.score.key_lo))
    assert torch.equal(call(x.score), want) and not torch.equal(first, want)
