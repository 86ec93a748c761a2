"""What an expert layer refuses when it is built: blobs that its decode would read beyond, sizes and options that a step's calls would refuse."""
import pytest
import torch

from paper_2510_02676_amd import ecf8
from paper_2510_02676_amd.experts import CompressedExperts
from test_gpu_expert_layer import DEV, layer_weights

pytestmark = pytest.mark.gpu


def refused(*args, **more):
    with pytest.raises(ecf8.Ecf8Error) as e:
        CompressedExperts(*args, **more)
    return e.value.code == ecf8.E_ARG


@pytest.mark.parametrize("name", ["gate", "up", "down"])
def test_blobs_that_are_not_what_their_headers_say(name):
    packed, _ = layer_weights(2, 128, 256, 5)
    hdr, blob, scale = packed[1][name]
    apart = torch.zeros((blob.numel(), 2), dtype=torch.uint8, device=DEV)[:, 0]
    for other in (blob[:hdr.total_size - 1], blob[:0], apart, blob.to(torch.int32), blob[:blob.numel() // 4 * 4].view(torch.int32)):
        assert refused([packed[0], dict(packed[1], **{name: (hdr, other, scale)})], 5, 2)
    longer = torch.cat((blob, blob[:7]))                                   # more than there is to read does no harm
    assert CompressedExperts([packed[0], dict(packed[1], **{name: (hdr, longer, scale)})], 5, 2).top == 2


@pytest.mark.parametrize("inner,hidden", [(128, (1 << 20) + 128), ((1 << 20) + 128, 128)])
def test_more_columns_than_a_steps_calls_take(inner, hidden):
    """Rows to E4M3, the gate and the sum take up to 2^20.  The headers say no more than their sizes: what looks further at them refuses them for that."""
    blob = torch.zeros(64, dtype=torch.uint8, device=DEV)
    part = lambda rows, cols: (ecf8.Header(rows=rows, cols=cols), blob, torch.ones((rows // 128, cols // 128), device=DEV))  # noqa: E731
    assert refused([{"gate": part(inner, hidden), "up": part(inner, hidden), "down": part(hidden, inner)}], 5, 1)


@pytest.mark.parametrize("name", ["routes", "stream"])
def test_options_that_a_step_gives_itself(name):
    packed, _ = layer_weights(2, 128, 128, 6)
    with pytest.raises(TypeError):
        CompressedExperts(packed, 5, 2, **{name: None})
