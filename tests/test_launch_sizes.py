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
