"""The operators around the attention at the ends of the sizes that they take."""
import pytest
import torch

from paper_2506_03065_amd import binding as svd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def memory_given_back():
    yield
    torch.cuda.empty_cache()


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


@pytest.mark.parametrize("H,L", [(40, 139_900), (3, (1 << 24) + 5)])
def test_rotary_positions_inside_a_joint_projection_past_4_gib(H, L):
    """q and k among the rows of q, k, v: more memory than a head of the attention may span, more rows.  The last rows against the
    same rows alone, the ones before against a part of the sequence at the same place."""
    D = 128 if H > 3 else 64
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    desc = svd.rope_desc(27, 720, 864, (8, 12, 12), first=77)   # over 2^24 tokens
    table = torch.empty(svd.svd_rope_table_bytes(desc) // 8, 2, device=DEV)
    svd.svd_rope_table(desc, table)
    qkv = torch.empty(1, L, 3, H, D, device=DEV, dtype=BF)
    for i in range(0, L, 1 << 20):
        qkv[:, i:i + (1 << 20)].normal_()
    assert qkv.numel() * 2 > 1 << 32
    q, k, v = (t.transpose(1, 2) for t in qkv.unbind(2))
    w = torch.linspace(0.5, 1.5, D, device=DEV)
    spots = [slice(0, 300), slice(L // 2, L // 2 + 300), slice(L - 300, L)]
    alone, grads, kept = [], [], v[:, :, -300:].clone()
    for s in spots:
        part = svd.rope_desc(27, 720, 864, (8, 12, 12), first=77, row_offset=s.start)
        a, g = [t[:, :, s].clone() for t in (q, k)], [t[:, :, s].clone() for t in (q, k)]
        svd.svd_rope_backward(part, table, [(k[:, :, s].clone(), g[0], g[0], w), (q[:, :, s].clone(), g[1], g[1], w)], norm="rms")
        svd.svd_rope_forward(part, table, [(a[0], a[0], w), (a[1], a[1], w)], norm="rms")
        alone.append(a)
        grads.append(g)
    dq, dk = (torch.empty(1, H, L, D, device=DEV, dtype=BF) for _ in range(2))
    svd.svd_rope_backward(desc, table, [(k, q, dq, w), (q, k, dk, w)], norm="rms")
    svd.svd_rope_forward(desc, table, [(q, q, w), (k, k, w)], norm="rms")
    for s, a, g in zip(spots, alone, grads):
        assert torch.equal(q[:, :, s], a[0]) and torch.equal(k[:, :, s], a[1])
        assert torch.equal(dq[:, :, s], g[0]) and torch.equal(dk[:, :, s], g[1])
    assert torch.equal(v[:, :, -300:], kept)
