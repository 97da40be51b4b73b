"""Token operators on more rows, runs or states than one dimension of a launch holds."""
import pytest
import torch

from paper_2305_16513_amd import binding as B

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("b,t", [(70, 131072), (66000, 9)])
def test_short_convolution_of_more_runs_than_a_launch_has_in_y(b, t):
    """Sequences do not meet: each is what it is by itself."""
    torch.manual_seed(1)
    c, k = 8, 4
    x, gy = (torch.randn(b, t, c, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w, bias = torch.randn(c, k, device="cuda"), torch.randn(c, device="cuda")
    how = dict(bias=bias, act=1, unit=4, unit_channels=8)
    y = B.sws_short_conv(x, w, **how)
    gx, gw, gb = B.sws_short_conv_grad(x, w, gy, **how)
    for i in (0, 1, b // 2, b - 4, b - 1):
        assert torch.equal(y[i:i + 1], B.sws_short_conv(x[i:i + 1], w, **how))
        assert torch.equal(gx[i:i + 1], B.sws_short_conv_grad(x[i:i + 1], w, gy[i:i + 1], **how)[0])
    # the sums over all tokens against those of halves of the batch: sums of n terms of size one, in fp32 and in another order
    half = [B.sws_short_conv_grad(x[s], w, gy[s], **how) for s in (slice(0, b // 2), slice(b // 2, b))]
    for got, parts in ((gw, [h[1] for h in half]), (gb, [h[2] for h in half])):
        assert (got - (parts[0] + parts[1])).abs().max().item() <= 1e-5 * (b * t) ** 0.5 * 4


# A launch has fewer than 2^32 threads in x: 2^24 workgroups of 256
@gpu
def test_norms_of_more_rows_than_a_launch_has_in_x():
    """Rows of one column: 32 of them a workgroup."""
    rows = 2 ** 29 + 37
    gen = torch.Generator(device="cuda").manual_seed(2)
    r = torch.empty(rows, 1, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    w = torch.full((1,), 1.5, device="cuda")
    n = B.sws_norm_add(r, w)[1]
    y = B.sws_norm_gate(r[:, None], r[:, None], w)
    for s in range(0, rows, 2 ** 27):                  # two roundings of numbers of 2 at most, and of r sigmoid(r) below 6
        x = r[s:s + 2 ** 27].float()
        ref = x * torch.rsqrt(x * x + 1e-6) * 1.5
        assert (n[s:s + 2 ** 27].float() - ref).abs().max().item() <= 2 ** -7
        assert (y[s:s + 2 ** 27, 0].float() - ref * x * torch.sigmoid(x)).abs().max().item() <= 2 ** -4


@gpu
def test_wide_rows_more_than_a_launch_has_in_x():
    """One token again and again, in one place: rows of 2048 columns take a workgroup each."""
    x, w = torch.randn(1, 1, 2048, device="cuda"), torch.randn(2048, device="cuda")
    many = 2 ** 24 + 3
    y = torch.zeros(1, 1, 2048, device="cuda")
    B.sws_norm_gate(x.expand(many, 1, 2048), x.expand(many, 1, 2048), w, y=y.expand(many, 1, 2048))
    assert torch.equal(y, B.sws_norm_gate(x, x, w))


@gpu
def test_single_tokens_of_more_states_than_a_launch_has_in_x():
    b = 2 ** 24 + 3
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v, g, beta = (torch.rand(b, 1, 1, 1, device="cuda", generator=gen) for _ in range(5))
    o = B.sws_delta_rule(q, k, v, -g[..., 0], beta[..., 0], 1.0)
    assert (o - q * k * beta * v).abs().max().item() <= 2 ** -21


@gpu
def test_sums_of_more_columns_than_a_launch_has_in_x():
    """The gradients of a convolution of 30 million channels: 150 million sums, 32 to a workgroup of 1024."""
    c, k = 30_000_000, 4
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, gy = (torch.randn(1, 1, c, device="cuda", generator=gen) for _ in range(2))
    w = torch.randn(c, k, device="cuda", generator=gen)
    gx, gw, gb = B.sws_short_conv_grad(x, w, gy, bias=torch.zeros(c, device="cuda"))
    assert torch.equal(gb, gy[0, 0]) and not gw[:, :k - 1].any()
    assert torch.equal(gw[:, k - 1], (x * gy)[0, 0]) and torch.equal(gx[0, 0], w[:, k - 1] * gy[0, 0])
