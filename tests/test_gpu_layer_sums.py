"""Sums over many rows in the operators around the attention, on data for which they are whole numbers below 2^24: whatever their order
and wherever they are held, they have no rounding and must be equal.  Every row adds something, so a row that is missing or counted
twice shows.  (Rows of +-1 have mean 0, where they come in pairs of either sign, and mean square 1; 1 + 1e-30 is 1 in 32 bits, and so
the norm leaves them as they are.)"""
import pytest
import torch

from oracle import layer_ops as O
from paper_2506_03065_amd import binding as svd
from test_gpu_blockscale import bytes_of, check_product, quantised

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
EPS = 1e-30


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def whole(g, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, device=DEV, generator=g)


def signs(g, *shape):
    """+-1, the second channel of a pair of the other sign."""
    s = whole(g, 0, 1, *shape[:-1], shape[-1] // 2) * 2 - 1
    return torch.stack([s, -s], -1).flatten(-2)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("B,heads,L,D", [(2, (3, 3), 9001, 64), (2, (3, 3), 9001, 128), (1, (48, 8), 333, 128), (5, (1,), 40, 64), (1, (2, 1), 1, 64),
                                         (3, (7, 5), 1037, 64), (1, (1, 2), 70001, 128)])
def test_gradients_of_the_rotary_norm_weights(B, heads, L, D, pairing, kind):
    """A third of the tokens turn, by a quarter: (a, b) -> (b, -a) on the way back."""
    g = gen(L + D)
    n = max(1, L // 3)
    desc = svd.rope_desc(n, 1, 1, (D // 2, 0, 0), first=L // 4, pairing=pairing)
    table = torch.tensor([0.0, 1.0], device=DEV).repeat(n * D // 2, 1)
    tensors, want = [], []
    for H in heads:
        x, d = signs(g, B, H, L, D), whole(g, 1, 3, B, H, L, D)
        r = [x.to(BF), d.to(BF), torch.empty(B, H, L, D, device=DEV, dtype=BF), None, torch.empty(D, device=DEV), torch.empty(D, device=DEV)]
        tensors.append(r)
        a, b = (slice(0, D // 2), slice(D // 2, None)) if pairing == "halves" else (slice(0, None, 2), slice(1, None, 2))
        back, video = d.clone(), slice(L // 4, L // 4 + n)
        back[:, :, video, a], back[:, :, video, b] = d[:, :, video, b], -d[:, :, video, a]
        want.append(((back * x).sum((0, 1, 2)), back.sum((0, 1, 2))))
    ws = torch.full((svd.svd_rope_backward_workspace_bytes(B, L, D),), 255, dtype=torch.uint8, device=DEV)   # NaN
    svd.svd_rope_backward(desc, table, tensors, norm=kind, eps=EPS, workspace=ws)
    for r, (dw, db) in zip(tensors, want):
        assert torch.equal(r[4].double(), dw.double()) and torch.equal(r[5].double(), db.double())


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("stream", [BF, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,L,C,first,group", [
    (1, 33000, 8, 0, 1), (2, 9107, 96, 77, 0), (1, 20000, 512, 0, 1000), (2, 5000, 784, 3, 7), (1, 70001, 128, 226, 5000), (3, 1, 64, 0, 0), (2, 33, 1032, 0, 2),
    (1, 4001, 1920, 26, 100), (1, 3000, 5120, 0, 0), (2, 701, 9216, 1, 300), (1, 2000, 16384, 0, 0)])
def test_gradients_of_the_norm_vectors(B, L, C, first, group, stream, norm):
    g = gen(L + C)
    groups = torch.from_numpy(O.row_groups(L, first, group)).to(DEV)
    G = int(groups.max()) + 1
    x, y, dh, up = signs(g, B, L, C), signs(g, B, L, C), whole(g, 1, 3, B, L, C), whole(g, 1, 3, B, L, C)
    scale, gate = whole(g, 0, 2, B, G, C), whole(g, 1, 3, B, G, C)
    w, b, pw = whole(g, 1, 2, C), whole(g, 0, 2, C), whole(g, 1, 2, C)

    def of_groups(v):
        return torch.zeros(B, G, C, device=DEV, dtype=torch.int64).index_add_(1, groups, v)

    s1, s2, t2 = of_groups(dh), of_groups(dh * x), of_groups(up * y)
    want = dict(dshift=s1, dscale=w * s2 + b * s1, dweight=((1 + scale) * s2).sum((0, 1)), dbias=((1 + scale) * s1).sum((0, 1)),
                dgate=pw * t2, dpost_weight=(gate * t2).sum((0, 1)))
    assert all(int(v.abs().max()) < 1 << 24 for v in want.values())
    ws = torch.full((svd.svd_residual_norm_backward_workspace_bytes(B, L, C, first, group),), 255, dtype=torch.uint8, device=DEV)   # NaN
    kw = dict(norm=norm, eps=EPS, first_rows=first, group_rows=group, workspace=ws)
    got = {k: torch.full(v.shape, float("nan"), device=DEV) for k, v in want.items()}
    dx, dy = torch.empty(B, L, C, device=DEV, dtype=stream), torch.empty(B, L, C, device=DEV, dtype=BF)
    of = lambda *names: {k: got[k] for k in names}  # noqa: E731
    svd.svd_residual_norm_backward(x.to(stream), None, dh.to(BF), None, dx=dx, weight=w.float(), bias=b.float(), scale=scale.float(), **kw,
                                   **of("dshift", "dscale", "dweight", "dbias"))
    ws.fill_(255)
    svd.svd_residual_norm_backward(x.to(stream), y.to(BF), None, up.to(stream), dx=dx, dy=dy, post_norm=norm, gate=gate.float(), post_weight=pw.float(),
                                   **kw, **of("dgate", "dpost_weight"))
    for k, v in want.items():
        assert torch.equal(got[k].double(), v.double()), k


# A weight's gradient sums over the rows of the activations: parts of K to a wave, 128 x 128 tiles, 256 x 256 and quarters.
@pytest.mark.parametrize("M,N,K", [(200, 150, 30011), (17, 300, 115456), (1500, 1480, 32777), (4300, 4100, 30001)])
def test_product_over_many_rows(M, N, K):
    """Whole numbers, whose sums the matrix instruction and 32 bits hold: rounded once."""
    g = gen(K)
    a, b = whole(g, -3, 3, M, (K + 7) // 8 * 8).float()[:, :K], whole(g, -3, 3, N, (K + 7) // 8 * 8).float()[:, :K]
    a8, b8 = quantised(a), quantised(b)
    out = torch.full((M, N), float("nan"), device=DEV, dtype=BF)
    svd.svd_blockscale_matmul(*a8, *b8, out)
    want = a.double() @ b.double().T.contiguous()
    assert torch.equal(out, want.to(BF)) and int(want.abs().max()) < 1 << 24
    bytes_of(b8[0])[:, K - 1] = 0    # the last row is counted: without it, what it brought is missing
    svd.svd_blockscale_matmul(*a8, *b8, out)
    assert torch.equal(out, (want - a[:, K - 1:].double() * b[:, K - 1:].double().T).to(BF))


@pytest.mark.parametrize("M,N,K", [(200, 150, 30011), (33, 64, 75600)])
def test_product_over_many_rows_of_normal_data(M, N, K):
    g = gen(K)
    a, b = (torch.randn(n, (K + 7) // 8 * 8, device=DEV, generator=g)[:, :K] for n in (M, N))
    a8, b8 = quantised(a), quantised(b)
    out = torch.empty(M, N, device=DEV, dtype=BF)
    svd.svd_blockscale_matmul(*a8, *b8, out)
    check_product(out, a8, b8, None)
