"""cmsd_layernorm without a weight: the bias's gradient in the bias's type, whatever x's is."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype,wdtype", [(BF16, F32), (F32, BF16), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("R,d", [(30, 72), (700, 1001)])
def test_gradient_in_the_biass_type(R, d, dtype, wdtype):
    from paper_2508_15371_gb300 import cmsd
    g = torch.Generator(device="cuda")
    g.manual_seed(R + d)
    x, d_y = (torch.randn(R, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    b = torch.randn(d, generator=g, device="cuda").to(wdtype)
    o = cmsd.layernorm(x, bias=b)
    got = cmsd.layernorm_backward(x, None, o["mean"], o["rstd"], d_y, dtype=wdtype)
    assert got["d_bias"].dtype is wdtype and got["d_weight"].dtype is wdtype and got["d_x"].dtype is dtype
    # the same as with a weight of ones, which says the type
    ones = torch.ones(d, device="cuda", dtype=wdtype)
    for given in (None, wdtype):
        want = cmsd.layernorm_backward(x, ones, o["mean"], o["rstd"], d_y, dtype=given)
        assert all(torch.equal(got[k], want[k]) for k in want)
    # a sum of R in fp32 (R 2^-24 of the magnitudes), rounded once
    s, m = d_y.double().sum(0), d_y.double().abs().sum(0)
    tol = R * 2.0 ** -24 * m
    assert ((got["d_bias"].double() - s).abs() <= tol + torch.finfo(wdtype).eps / 2 * (s.abs() + tol)).all()
    # without either, x's
    assert cmsd.layernorm_backward(x, None, o["mean"], o["rstd"], d_y)["d_bias"].dtype is dtype
