"""Scored attention of more work items than one launch of 2^32 threads takes."""
import time

import numpy as np
import pytest
import torch

from tests._gpu import HAVE_GPU, api

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not HAVE_GPU, reason="needs a GPU")]
DEV = "cuda:0"


def test_one_token_segments_past_a_grid_of_2_32_threads():
    """262,144 segments of one token and 64 heads: 2^24 items of 256 threads in the forward and dQ, of 512 in dK/dV.  A row
    sees itself alone: out = v and dv = dout to the bit, the LSE is its score, and dA = dO.v - dO.O is fp32's error,
    2 E |dO||v| with E = 64 2^-24, times scale |k| below 6 in dq and dk: 0.125 * 6 * 2 * 2^-18 * 64 * 36 < 0.02."""
    n, H, hd = 1 << 18, 64, 64
    t0 = time.monotonic()
    cu, ids = np.arange(n + 1), np.arange(n)
    desc = api.SegDesc(cu, np.zeros(n), ids, np.ones(n), cu, np.zeros(n), 0)
    g = torch.Generator(device=DEV).manual_seed(5)
    q, k, v, do = (torch.randn((n, H, hd), generator=g, device=DEV, dtype=torch.bfloat16).clamp_(-6, 6) for _ in range(4))
    score = api.Score(causal=True)
    try:
        out, lse, _, _ = api.score_fwd(desc, score, q, k, v, 0.125)
        torch.cuda.synchronize()
        print(f"forward {time.monotonic() - t0:.1f} s", flush=True)
        assert torch.equal(out, v)
        for a in (0, n // 2, n - 1000):
            s = 0.125 * (q[a:a + 1000].float() * k[a:a + 1000].float()).sum(-1)
            assert ((lse[a:a + 1000] - s).abs() <= 2.0 ** -18 * 0.125 * 64 * 36 + 2.0 ** -20 * s.abs()).all()
        dq, dk, dv, _ = api.score_bwd(desc, score, q, k, v, out, lse, do, 0.125)
        torch.cuda.synchronize()
        print(f"backward {time.monotonic() - t0:.1f} s", flush=True)
        assert torch.equal(dv, do)
        assert float(dq.abs().max()) < 0.02 and float(dk.abs().max()) < 0.02
    finally:
        api.shutdown()  # the schedules take 1.6 GB


def test_single_tokens_past_a_grid_of_2_32_threads():
    """The kernel for few rows: 262,144 tokens against a cache of one key each, 64 heads."""
    n, H, hd = 1 << 18, 64, 64
    cu, ids = np.arange(n + 1), np.arange(n)
    desc = api.SegDesc(cu, np.ones(n), ids, np.ones(n), cu, np.zeros(n), 1, q_offset=np.zeros(n), k_offset=np.zeros(n))
    g = torch.Generator(device=DEV).manual_seed(6)
    q, k, v = (torch.randn((n, H, hd), generator=g, device=DEV, dtype=torch.bfloat16) for _ in range(3))
    try:
        out, lse, _, _ = api.score_fwd(desc, api.Score(causal=True), q, k, v, 0.125)
        assert torch.equal(out, v) and torch.isfinite(lse).all()
    finally:
        api.shutdown()
