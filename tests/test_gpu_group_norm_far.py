"""Group norm at the largest number of channels and groups that it takes."""
import pytest
import torch

import paper_2002_11082_b200 as ogq

pytestmark = pytest.mark.gpu
U24 = 2.0 ** -24


def test_as_many_channels_and_groups_as_are_taken():
    """2^31 - 1 channels of one pixel, each its own group: the last tile of channels ends past 2^31, and a CTA per group and one per eight channels are more than a
    grid holds.  The mean is x, y = 0; dz = dy: dbeta = dy, dgamma = 0, dx = rstd (dz - dz), off by the rounding of rstd dz."""
    torch.cuda.empty_cache()
    C = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("100 GB of device memory")
    BF = ogq.OGQ_BF16
    x = torch.empty(C, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(5))
    out = torch.full((C,), 7.0, dtype=torch.bfloat16, device="cuda")
    mean, rstd, dg, db = (torch.full((C,), 7.0, device="cuda") for _ in range(4))
    ws = torch.empty(ogq.ogq_group_norm_workspace_bytes(1, 1, C, C), dtype=torch.uint8, device="cuda")
    ogq.ogq_group_norm_forward(x, 1, 1, C, C, BF, None, None, 1e-5, ogq.OGQ_ACT_NONE, 0, 0, 0, out, mean, rstd, None, None, ws, ws.numel())
    assert not out.any()
    step = 1 << 28
    for i in range(0, C, step):
        assert torch.equal(mean[i:i + step], x[i:i + step].float())
    assert float((rstd - 1e-5 ** -0.5).abs().max()) < 1e-4
    out.fill_(7.0)
    ogq.ogq_group_norm_backward(x, x, None, None, 1, 1, C, C, BF, None, None, ogq.OGQ_ACT_NONE, mean, rstd, out, dg, db, ws, ws.numel())
    assert not dg.any()
    for i in range(0, C, step):
        part = x[i:i + step].float()
        assert torch.equal(db[i:i + step], part)
        assert bool((out[i:i + step].float().abs() <= 2 * U24 * 317 * part.abs()).all())
