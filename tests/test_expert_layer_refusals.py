"""What an expert layer refuses without a device."""
import pytest
import torch

from paper_2510_02676_amd import ecf8
from paper_2510_02676_amd.experts import CompressedExperts


def test_a_refused_step_decodes_nothing(monkeypatch):
    """The tensors are looked at before the first launch: the decode writes where the layer's device is, whichever is the current one."""
    queued = []
    monkeypatch.setattr(ecf8, "ecf8_decode_batched", lambda *a: queued.append(a))
    layer = CompressedExperts.__new__(CompressedExperts)
    layer.decode, layer.x8, layer.x_scale, layer.h8 = None, torch.zeros((5, 256), dtype=torch.uint8), torch.zeros((5, 2)), torch.zeros((10, 128), dtype=torch.uint8)
    for x in (torch.zeros((5, 256)), torch.zeros((4, 256)), torch.zeros((5, 256), dtype=torch.float16)):      # on the host, of other sizes, of another type
        with pytest.raises(ecf8.Ecf8Error) as e:
            layer(x, torch.zeros((5, 3)))
        assert e.value.code == ecf8.E_ARG and not queued


def test_no_experts():
    with pytest.raises(ecf8.Ecf8Error) as e:
        CompressedExperts([], 5, 2)
    assert e.value.code == ecf8.E_ARG
