"""Drafts over a 4-bit run, written to the caller's own tensors."""
import numpy as np
import pytest
import torch

from paper_2605_16928_amd import rtp, workloads as wl
from paper_2605_16928_amd.pipeline import Kv4DecodeRun
from test_gpu_kv4_run import _more

pytestmark = pytest.mark.gpu


def test_outputs_of_the_callers():
    """[B, T, n_q_heads, 128] and [B, T, n_q_heads], as they are returned, or packed; others are refused before anything is written."""
    w = wl.small_decode("cuda:0", seed=9, ctx=(300, 16, 1))
    run, T = Kv4DecodeRun(w, 16, room=8), 3
    run.grow(*_more(np.random.default_rng(9), w, T))
    H = w.layer.n_q_heads
    q = torch.randn((3, T, H, 128), device="cuda:0").to(torch.bfloat16)
    want, want_lse = run.draft_attn(q)
    for shape in ((3, T), (3 * T,)):
        out, lse = torch.full((*shape, H, 128), 7.0, dtype=q.dtype, device="cuda:0"), torch.full((*shape, H), 7.0, device="cuda:0")
        got, got_lse = run.draft_attn(q, out, lse)
        assert got.data_ptr() == out.data_ptr() and got_lse.data_ptr() == lse.data_ptr()
        assert torch.equal(out.view(want.shape), want) and torch.equal(lse.view(want_lse.shape), want_lse) and got.shape == want.shape
    out, lse = torch.full_like(q, 7.0), torch.full((3, T, H), 7.0, device="cuda:0")
    for bad in ((out[:, :2], lse), (out, lse[:2]), (out.transpose(1, 2).contiguous().transpose(1, 2), lse), (out.half(), lse), (out, lse.half()),
                (out[..., :64], lse), (out, lse.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises(rtp.RtpError) as e:
            run.draft_attn(q, *bad)
        assert e.value.code == rtp.RTP_ERR_INVALID_ARG
    assert (out == 7.0).all() and (lse == 7.0).all()
