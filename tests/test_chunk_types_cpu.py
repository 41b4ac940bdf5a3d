"""Tensors of another type than the layer's are refused by the calls over new tokens, on the host."""
import pytest
import torch

from paper_2605_16928_amd import rtp
from test_chunk_cpu import QKV, Rows, _calls, _layer

BF16, FP16 = torch.bfloat16, torch.float16


class Typed(Rows):
    def __init__(self, t):
        super().__init__(t)
        self.dtype = t.dtype


def _refused(name, match, layer=None, cache=None, **kw):
    call, args = _calls(layer=layer, cache=cache)[name]
    with pytest.raises(rtp.RtpError, match=match) as e:
        call(**dict(args, **kw))
    assert e.value.code == rtp.RTP_ERR_INVALID_ARG, str(e.value)


@pytest.mark.parametrize("name", ["dense", "local", "dense4", "local4"])
@pytest.mark.parametrize("layer_type,others", [(rtp.RTP_DTYPE_BF16, (FP16, torch.int16)), (rtp.RTP_DTYPE_FP16, (BF16, torch.int16))])
def test_attention(name, layer_type, others):
    for other in others:
        layer, q, out = _layer(kv_dtype=layer_type), torch.zeros((50, 12, 128), dtype=other)[:, :8], torch.zeros((50, 8, 128), dtype=other)
        _refused(name, "q of torch.*expected", layer, q=Typed(q))
        _refused(name, "out of torch.*expected", layer, out=Typed(out))
    for other in (torch.int32, torch.uint8):
        lse = torch.zeros((50, 8) if other is torch.int32 else (200, 8), dtype=other)
        _refused(name, "lse.*expected", lse=Typed(lse))


@pytest.mark.parametrize("layer_type,others", [(rtp.RTP_DTYPE_BF16, (FP16, torch.int16)), (rtp.RTP_DTYPE_FP16, (BF16, torch.int16))])
def test_append(layer_type, others):
    for other in others:
        layer, fused = _layer(kv_dtype=layer_type), torch.zeros((50, 12, 128), dtype=other)
        for key, x in (("q", fused[:, :8]), ("k", fused[:, 8:10]), ("v", fused[:, 10:]), ("q_out", fused.flatten(1)[:, :1024].unflatten(1, (8, 128)).contiguous())):
            _refused("append", f"{key} of torch.*expected", layer, **{key: Typed(x)})


@pytest.mark.parametrize("name", ["append", "dense", "local"])
@pytest.mark.parametrize("layer_type,others", [(rtp.RTP_DTYPE_BF16, (FP16, torch.int16)), (rtp.RTP_DTYPE_FP16, (BF16, torch.int16))])
def test_caches(name, layer_type, others):
    for other in others:
        rows = [torch.zeros((2, 5, 64, 128), dtype=other) for _ in range(2)]
        _refused(name, "a cache of torch.*expected", _layer(kv_dtype=layer_type), rtp.kv_cache(*rows, torch.zeros((3, 32), dtype=torch.int32)))
