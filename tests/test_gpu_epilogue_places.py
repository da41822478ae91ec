"""Outputs of the calls with an epilogue that take the place of an operand, where that is allowed."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dy_dtype", [BF16, F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(5, 64), (700, 264)], ids=str)
def test_backward_in_the_place_of_its_operands(gpu_api, shape, dy_dtype):
    g = torch.Generator().manual_seed(5)
    host = [torch.randn(shape, generator=g).to(t) for t in (dy_dtype, BF16, BF16)]
    dz, dmul, db = gpu_api.epilogue_backward(*(t.cuda() for t in host[:2]), "gelu", mul=host[2].cuda(), want_dbias=True)
    for a, b in ((0, 1), (1, 0), (2, 1), (1, 2), (0, 2), (2, 0)):   # dz and dmul at dy (0), z (1) or mul (2)
        if dy_dtype == F32 and 0 in (a, b):
            continue
        at = [t.cuda() for t in host]
        got = gpu_api.epilogue_backward(at[0], at[1], "gelu", mul=at[2], dz=at[a], dmul=at[b], want_dbias=True)
        assert got[0] is at[a] and got[1] is at[b]
        assert torch.equal(got[0], dz) and torch.equal(got[1], dmul) and torch.equal(got[2], db)
    if dy_dtype == F32:
        dy = host[0].cuda()
        over = dy.view(BF16).view(-1)[: dz.numel()].view(shape)
        with pytest.raises(gpu_api.QaloraError) as e:
            gpu_api.epilogue_backward(dy, host[1].cuda(), "gelu", dz=over)
        assert e.value.status == gpu_api.EINVAL and torch.equal(dy.cpu(), host[0])
