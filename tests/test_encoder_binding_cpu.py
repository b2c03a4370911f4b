"""Workspaces that a caller gives the calls of an encoder's layers: one on the host, or of another type, is refused before anything is launched. The other
tensors are stand-ins with what the checks ask for, so that the refusal can be seen without a GPU."""
import pytest
import torch

from paper_2604_04451_amd import binding as B

BF = torch.bfloat16


class OnDevice:
    is_cuda, device = True, "cpu"

    def __init__(self, *shape, dtype=BF):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s) if i is None else s[i]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 16

    def numel(self):
        return 1 << 30


def attention():
    q, k = OnDevice(2, 40, 4, 64), OnDevice(2, 2000, 2, 64)
    return q, k, OnDevice(32, 4, dtype=torch.float32), OnDevice(257, dtype=torch.int32), OnDevice(2, 4, 40, dtype=torch.float32)


def forward(ws):
    q, k, table, bucket, _ = attention()
    B.chorus_attention_bias(q, k, k, q, table, bucket, ws=ws)


def backward(ws):
    q, k, table, bucket, lse = attention()
    B.chorus_attention_bias_backward(q, k, k, q, q, lse, q, table, bucket, q, k, k, table, ws=ws)


def gated_backward(ws):
    x, w, pre, dh = OnDevice(4, 64), OnDevice(256, 64), OnDevice(4, 256), OnDevice(4, 128)
    B.chorus_gated_ffn_backward(x, w, pre, dh, B.ACT_GELU, x, w, ws=ws)


@pytest.mark.parametrize("ws", [torch.empty(1 << 22, dtype=torch.uint8), OnDevice(1 << 22, dtype=torch.float32)])
@pytest.mark.parametrize("call", [forward, backward, gated_backward])
def test_workspaces(call, ws, monkeypatch):
    monkeypatch.setattr(B, "_stream", lambda: None)
    with pytest.raises(TypeError, match="ws"):
        call(ws)
