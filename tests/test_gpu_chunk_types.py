"""Tensors of another type than the layer's, on the GPU: refused before anything is launched."""
import numpy as np
import pytest
import torch

from chunk_util import Batch
from paper_2605_16928_amd import rtp, workloads as wl
from paper_2605_16928_amd.pipeline import Kv4DecodeRun
from test_gpu_chunk import run
from test_gpu_kv4_run import _more

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv_dtype", ["bf16", "fp16"])
def test_drafts(kv_dtype):
    w = wl.small_decode("cuda:0", seed=9, ctx=(70, 16), kv_dtype=kv_dtype)
    four = Kv4DecodeRun(w, 16, room=8)
    four.grow(*_more(np.random.default_rng(9), w, 2))
    mine, other = (torch.bfloat16, torch.float16) if kv_dtype == "bf16" else (torch.float16, torch.bfloat16)
    q = torch.zeros((2, 2, w.layer.n_q_heads, 128), dtype=mine, device="cuda:0")
    four.draft_attn(q)
    for bad in (q.to(other), q.view(torch.int16), q[:, :, :1].contiguous()):
        with pytest.raises(rtp.RtpError) as e:
            four.draft_attn(bad)
        assert e.value.code == rtp.RTP_ERR_INVALID_ARG


def test_caches():
    b = Batch(new=[5, 1], past=[40, 100], seed=2)
    q, cache, chunk = b.device()
    run(b, prepared=(q, cache, chunk))
    K, V, table = cache._keepalive
    for kind in (torch.float16, torch.int16):
        with pytest.raises(rtp.RtpError, match="a cache of"):
            run(b, prepared=(q, rtp.kv_cache(K.view(kind), V.view(kind), table), chunk))
