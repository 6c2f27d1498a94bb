"""Infinities and NaN in the operators around the attention: what is formed from them is NaN, and everything else keeps its bits."""
import pytest
import torch

from paper_2506_03065_amd import binding as svd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
NAN, INF = float("nan"), float("inf")


def eight_bits(x, **kw):
    B, L, C = x.shape
    h, s = svd.blockscale_empty(B * L, C, DEV)
    h.untyped_storage().fill_(0x55)
    s.fill_(0x55)
    svd.svd_residual_norm_forward(x, h=h.view(B, L, C), h_scales=s, **kw)
    return h, s


# a row to 16, 32 and 64 lanes, to one wave and more, a last block that ends early
WIDTHS = [96, 256, 512, 784, 1040, 2064, 5120]


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("stream", [BF, torch.float32], ids=["bf16", "f32"])
def test_rows_of_the_eight_bit_norm(C, norm, stream):
    g = torch.Generator(device=DEV).manual_seed(C)
    x = torch.randn(1, 37, C, device=DEV, generator=g).to(stream)
    clean, clean_s = eight_bits(x, norm=norm)
    at = C - 3
    bad = {2: NAN, 17: INF, 31: -INF}
    for r, v in bad.items():
        x[0, r, at] = v
    h, s = eight_bits(x, norm=norm)
    blocks = s.shape[0]
    want = clean_s[:, :37].clone()
    for r, v in bad.items():
        want[:, r] = 255
        if norm == "rms" and r != 2:   # x / inf: zeros, but inf / inf
            want[:, r] = 0
            want[at // 128, r] = 255
    assert torch.equal(s[:, :37], want)
    keep = [r for r in range(37) if r not in bad]
    assert torch.equal(h.view(torch.uint8)[keep], clean.view(torch.uint8)[keep])
    w, ws = svd.blockscale_empty(40, C, DEV)
    svd.svd_blockscale_quantise(torch.randn(40, C, device=DEV, generator=g), w, ws)
    out = torch.empty(37, 40, device=DEV, dtype=BF)
    svd.svd_blockscale_matmul(h, s, w, ws, out)
    nan = torch.zeros(37, 40, dtype=torch.bool, device=DEV)
    nan[list(bad)] = True
    assert torch.equal(torch.isnan(out), nan) and torch.isfinite(out[keep].float()).all()
    assert blocks == -(-C // 128)


@pytest.mark.parametrize("C", WIDTHS)
def test_a_channel_of_the_modulation(C):
    """Only the block that meets it; the largest finite number still has a scale."""
    x = torch.randn(2, 9, C, device=DEV)
    shift = torch.zeros(2, 1, C, device=DEV)
    clean, clean_s = eight_bits(x, shift=shift)
    shift[1, 0, 5] = NAN
    shift[0, 0, C - 1] = 3.0e38
    h, s = eight_bits(x, shift=shift)
    last = (C - 1) // 128
    assert (s[0, 9:18] == 255).all()
    if last:
        assert torch.equal(s[1:, 9:18], clean_s[1:, 9:18]) and torch.equal(s[:last, :9], clean_s[:last, :9])
        assert torch.equal(h.view(torch.uint8)[9:, 128:], clean.view(torch.uint8)[9:, 128:])
    # 3e38 = 1.76 * 2^127: over 1.75 * 2^127 = 448 * 2^119, so 2^120, and 3e38 / 2^120 = 225.7 rounds to 224
    assert (s[last, :9] == 127 + 120).all() and (h[:9, C - 1].float() == 224.0).all()


@pytest.mark.parametrize("C", [8, 96, 512, 1000, 1032, 5120, 16384])
@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("where", ["x_out", "y", "dh", "dx_out"])
def test_rows_of_the_norms_gradients(C, norm, where):
    """dx and dy of the rows that are finite, and the sums of groups that are."""
    B, L = 1, 23
    g = torch.Generator(device=DEV).manual_seed(C)
    t = {k: torch.randn(B, L, C, device=DEV, generator=g) for k in ("x_out", "y", "dh", "dx_out")}
    t["y"], t["dh"] = t["y"].to(BF), t["dh"].to(BF)
    ws = torch.empty(svd.svd_residual_norm_backward_workspace_bytes(B, L, C, 0, 5), dtype=torch.uint8, device=DEV)

    def grads():
        out = dict(dx=torch.empty(B, L, C, device=DEV), dy=torch.empty(B, L, C, device=DEV, dtype=BF))
        out.update({k: torch.empty(B, 5, C, device=DEV) for k in ("dgate", "dscale", "dshift")})
        svd.svd_residual_norm_backward(*(t[k] for k in ("x_out", "y", "dh", "dx_out")), norm=norm, post_norm="rms", group_rows=5, workspace=ws, **out)
        return out

    clean = grads()
    t[where][0, 12, C // 2] = NAN   # in group 2
    got = grads()
    rows = [r for r in range(L) if r != 12]
    groups = [0, 1, 3, 4]
    assert torch.isfinite(clean["dx"]).all() and torch.isfinite(clean["dgate"]).all()
    for k in ("dx", "dy"):
        assert torch.equal(got[k][:, rows], clean[k][:, rows]), k
    for k in ("dgate", "dscale", "dshift"):
        assert torch.equal(got[k][:, groups], clean[k][:, groups]), k
    assert torch.isnan(got["dy"][0, 12]).all()
    assert torch.equal(got["dx"], clean["dx"]) if where == "y" else torch.isnan(got["dx"][0, 12, C // 2])


@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
def test_rows_of_the_rotary_gradients(pairing):
    desc = svd.rope_desc(2, 3, 4, (8, 12, 12), first=3, pairing=pairing)
    table = torch.empty(svd.svd_rope_table_bytes(desc) // 8, 2, device=DEV)
    svd.svd_rope_table(desc, table)
    x, d = (torch.randn(2, 3, 30, 64, device=DEV).to(BF) for _ in range(2))
    clean, got = torch.empty_like(x), torch.empty_like(x)
    svd.svd_rope_backward(desc, table, [(x, d, clean)], norm="layer")
    d[1, 2, 7, 40] = NAN
    x[0, 1, 20, 3] = INF
    svd.svd_rope_backward(desc, table, [(x, d, got)], norm="layer")
    for b, h, l in ((1, 2, 7), (0, 1, 20)):
        assert torch.isnan(got[b, h, l]).all()
        got[b, h, l] = clean[b, h, l]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("D", [64, 128])
def test_what_does_not_turn_keeps_its_bits(pairing, D):
    """Tokens outside the video, pairs without an axis and position 0: infinities, zeros of either sign and NaN beside them."""
    desc = svd.rope_desc(3, 2, 2, (8, 4, 4), first=5, pairing=pairing)
    table = torch.empty(svd.svd_rope_table_bytes(desc) // 8, 2, device=DEV)
    svd.svd_rope_table(desc, table)
    values = torch.tensor([1.5, INF, -0.0, 0.0, -INF, 3.0, NAN, -2.0], device=DEV)
    pick = torch.randint(0, 8, (2, 2, 40, D), device=DEV, generator=torch.Generator(device=DEV).manual_seed(D))
    x = values[pick].to(BF)
    pair = torch.arange(D, device=DEV) % (D // 2) if pairing == "halves" else torch.arange(D, device=DEV) // 2
    still = torch.ones(40, D, dtype=torch.bool, device=DEV)
    still[6:17] = pair >= 16                # the video but its first token; pairs from the 16th on have no axis
    out, back = torch.empty_like(x), torch.empty_like(x)
    svd.svd_rope_forward(desc, table, [(x, out)])
    svd.svd_rope_backward(desc, table, [(None, x, back)])
    number = still & ~torch.isnan(x)
    for o in (out, back):
        assert torch.equal(o.view(torch.int16)[number], x.view(torch.int16)[number])
        assert torch.isnan(o[still & torch.isnan(x)]).all()
