"""The operators around the attention at the ends of the sizes that they take."""
import pytest
import torch

from paper_2506_03065_amd import binding as svd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.mark.parametrize("L", [2 ** 31 - 1, 2 ** 31 - 8])
def test_norms_of_the_most_rows(L):
    """As many rows as a call takes, of 8 channels (34 GB a tensor): the last rows against the same rows alone, and a sum over the
    rows whose exact value is known."""
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    n = 1000
    g = torch.Generator(device=DEV).manual_seed(L % 1000)
    x = torch.full((1, L, 8), 2.0, device=DEV, dtype=BF)
    x[:, -n:] = torch.randn(1, n, 8, device=DEV, generator=g).to(BF)
    h, last = torch.full((1, L, 8), 7.0, device=DEV, dtype=BF), torch.empty(1, n, 8, device=DEV, dtype=BF)
    svd.svd_residual_norm_forward(x, h=h)
    svd.svd_residual_norm_forward(x[:, -n:], h=last)
    assert torch.equal(h[:, -n:], last)
    for i in range(0, L - n, 1 << 28):
        assert not h[:, i:min(i + (1 << 28), L - n)].any()   # constant rows
    dh = h
    dh.zero_()
    dh[:, -n:] = 3.0
    dx, dshift = torch.full((1, L, 8), 7.0, device=DEV, dtype=BF), torch.empty(1, 1, 8, device=DEV)
    ws = torch.empty(svd.svd_residual_norm_backward_workspace_bytes(1, L, 8), dtype=torch.uint8, device=DEV)
    svd.svd_residual_norm_backward(x, None, dh, None, dx=dx, dshift=dshift, norm="rms", workspace=ws)
    svd.svd_residual_norm_backward(x[:, -n:], None, dh[:, -n:], None, dx=last, norm="rms")
    assert torch.equal(dx[:, -n:], last) and (dshift == 3.0 * n).all()
    for i in range(0, L - n, 1 << 28):
        assert not dx[:, i:min(i + (1 << 28), L - n)].any()
