"""ecfm_gate where exp(-|gate|) is below what fp32 holds, and the product with a large `up` is not."""
import math

import pytest
import torch

from test_gpu_expert_rows import BF, DEV, check_gate
from attention_reference import E4M3
from paper_2510_02676_amd import ecfm

pytestmark = pytest.mark.gpu
FAR = [(-86.9, 1e30), (-87.1, 1e9), (-87.4, 1e30), (-88.0, 3e38), (-88.5, 1e12), (-89.0, 1e36), (-95.0, -3e38), (-103.9, 1e38), (-104.1, 3e38), (-120.0, 3e38), (-160.0, 3e38), (-176.2, 3.3e38),
       (-180.0, 3.3e38), (-181.3, 3.3e38), (-190.0, 3.3e38), (-1000.0, 3e38), (-3e38, 3e38), (-88.0, 1.0), (-88.0, 1e-30), (-95.0, 0.0)]


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("cols", [256, 9000 * 16])
def test_products_that_fp32_holds(dtype, cols):
    gen = torch.Generator().manual_seed(cols)
    noise = torch.rand((2, len(FAR), cols), generator=gen) * 0.002 + 0.999
    g, u = (torch.tensor([f[i] for f in FAR])[:, None].mul(noise[i]).to(dtype) for i in range(2))
    check_gate(g, u, 0)
    check_gate(g[:, :256], u[:, :256], 128)


def test_beside_ordinary_numbers():
    """One far number in each eight, in places of all kinds, among others."""
    gen = torch.Generator().manual_seed(1)
    g, u = torch.randn((len(FAR), 512), generator=gen), torch.randn((len(FAR), 512), generator=gen)
    for i, (a, b) in enumerate(FAR):
        g[i, i % 8::8], u[i, i % 8::8] = a, b
    for group in (0, 128):
        check_gate(g, u, group)


def test_infinities_beside_far_numbers():
    g, u = torch.full((3, 128), -88.0), torch.full((3, 128), 1e30)
    g[0, 5], g[1, 6], u[2, 7] = -math.inf, math.nan, math.inf
    q, s = ecfm.ecfm_gate(g.to(DEV), u.to(DEV))
    want = 88 * math.exp(-88) * 1e30 / 448
    assert abs(s[0].item() / want - 1) < 2.0 ** -18 and s[1].isnan() and s[2].item() == math.inf
    v = E4M3[q[0].cpu().view(torch.uint8).numpy()]
    assert v[5] == 0 and (v[:5] == -448).all() and (v[6:] == -448).all()
