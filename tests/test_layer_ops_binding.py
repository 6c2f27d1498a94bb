"""The binding of the operators around an attention: what it refuses by itself."""
import pytest
import torch

from paper_2506_03065_amd import binding as svd


@pytest.mark.parametrize("B,L,D", [(2 ** 32 + 1, 5, 64), (1, 2 ** 32 + 5, 64), (1, 5, 2 ** 32 + 64), (-1, 5, 64)])
def test_workspace_of_sizes_past_32_bits(B, L, D, monkeypatch):
    monkeypatch.setattr(svd, "lib", lambda: pytest.fail("reached the library"))
    with pytest.raises(ValueError, match="2\\^31"):
        svd.svd_rope_backward_workspace_bytes(B, L, D)


class Recorded:
    """The library's entry points, none of which runs: their arguments."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def recorded(monkeypatch):
    r = Recorded()
    monkeypatch.setattr(svd._Kinds.get(), "device", staticmethod(lambda: -1))   # the CPU's
    monkeypatch.setattr(svd._Kinds, "stream", classmethod(lambda cls, stream, device: None))
    monkeypatch.setattr(svd, "lib", lambda: r)
    return r


@pytest.mark.parametrize("columns", [100, 128, 300])
def test_scales_of_some_rows(columns, recorded):
    """The first rows of a matrix with their scales, cut to these rows: the stride of a single block of scales says nothing."""
    v, s = svd.blockscale_empty(40, columns, "cpu")
    out = torch.empty(5, 5, dtype=torch.bfloat16)
    svd.svd_blockscale_matmul(v[:5], s[:, :5], v[16:21], s[:, 16:21], out)
    svd.svd_blockscale_quantise(torch.zeros(5, columns), v[:5], s[:, :5])
    d = recorded.calls[0][1][0]._obj
    assert (d.M, d.N, d.K) == (5, 5, columns)
    for stride in (d.a_scale_stride, d.b_scale_stride, recorded.calls[1][1][9]):
        assert stride % 16 == 0 and stride >= 5 and (columns <= 128 or stride == s.stride(0))


def test_scales_of_the_norm_of_some_rows(recorded):
    x = torch.zeros(1, 5, 64, dtype=torch.bfloat16)
    v, s = svd.blockscale_empty(16, 64, "cpu")
    svd.svd_residual_norm_forward(x, h=v[:5].view(1, 5, 64), h_scales=s[:, :5])
    stride = recorded.calls[0][1][7]
    assert stride % 16 == 0 and stride >= 5
