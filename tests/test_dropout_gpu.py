"""cmsd_dropout and cmsd_dropout_backward: the mask against the generator's
words, entry by entry; the values against the definition in 64 bits.

Tolerance: the scale is rounded to fp32 (u = 2^-24), the product and the sum of
the residual once more each, then half a step of the dtype.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


def _keep(cmsd, n, p, seed, iteration, site, first=0):
    """The definition's mask of entries first .. first + n (first a multiple of 8), by the generator's words."""
    groups = (n + 7) // 8
    g0 = first // 8
    w = cmsd.philox_fill(seed, g0 & 0xFFFFFFFF, g0 >> 32, site, (iteration << 2 | 3) & 0xFFFFFFFF, 4 * groups)
    halves = w.cpu().numpy().astype("<i4").view("<u2")[:n]
    return torch.from_numpy((halves.astype(np.int64) >= round(p * 65536))).cuda()


def _check(got, x, keep, p, residual=None):
    t = round(p * 65536)
    s = 65536 / (65536 - t) if t < 65536 else 0.0
    want = torch.where(keep.reshape(x.shape), x.double() * s, 0.0)
    tol = 3 * U * want.abs()
    if residual is not None:
        want = want + residual.double()
        tol = tol + 2 * U * want.abs()
    tol = tol + torch.finfo(x.dtype).eps / 2 * (want.abs() + tol) + 2.0 ** -140
    assert ((got.double() - want).abs() <= tol).all()
    if residual is None:
        assert (got.reshape(-1)[~keep] == 0).all()
    else:
        assert torch.equal(got.reshape(-1)[~keep], residual.reshape(-1)[~keep])


SIZES = [(1,), (2,), (7,), (8,), (9,), (15, 1), (33, 31), (64, 1024), (37, 1040), (333, 1001), (3, 5, 7), (2048, 129)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SIZES)
@pytest.mark.parametrize("p", [0.0, 0.1, 0.37, 0.999, 1.0])
def test_values_and_gradient(cmsd, shape, p, dtype):
    x, r = torch.randn(shape, device="cuda").to(dtype), torch.randn(shape, device="cuda").to(dtype)
    seed, it, site = (11 << 40) + 5, 77, 3
    keep = _keep(cmsd, x.numel(), p, seed, it, site)
    _check(cmsd.dropout(x, p, seed, it, site)["y"], x, keep, p)
    _check(cmsd.dropout(x, p, seed, it, site, residual=r)["y"], x, keep, p, r)
    _check(cmsd.dropout_backward(r, p, seed, it, site)["d_x"], r, keep, p)


def test_words_against_the_oracle(cmsd):
    """The generator itself in plain integers, on the CPU, for a few entries of one call."""
    from oracle import philox
    n, p, seed, it, site = 80, 0.4, (3 << 33) + 123456789, 9, 17
    x = torch.ones(n, device="cuda")
    y = cmsd.dropout(x, p, seed, it, site)["y"].cpu()
    for e in range(n):
        words = philox.philox4x32_10((e >> 3, 0, site, it << 2 | 3), (seed & 0xFFFFFFFF, seed >> 32))
        half = int(words[(e >> 1) & 3]) >> (16 * (e & 1)) & 0xFFFF
        assert (float(y[e]) != 0) == (half >= round(p * 65536)), e


@pytest.mark.parametrize("p,t", [(2.0 ** -18, 0), (2.0 ** -17, 0), (3 * 2.0 ** -17, 2), (0.1, 6554), (1 - 2.0 ** -16, 65535)])
def test_rates_are_multiples_of_2_to_minus_16(cmsd, p, t):
    n = 1 << 20
    x = torch.ones(n, device="cuda")
    y = cmsd.dropout(x, p, 5)["y"]
    keep = _keep(cmsd, n, t / 65536, 5, 0, 0)
    assert torch.equal(y != 0, keep)
    assert torch.equal(y[keep], torch.full_like(y[keep], 65536 / (65536 - t)))


def test_rate(cmsd):
    """The share of dropped entries lies within six standard deviations."""
    n = 1 << 24
    x = torch.ones(n, device="cuda")
    for p in (0.1, 0.5):
        for it in (0, 1):
            dropped = int((cmsd.dropout(x, p, 99, it)["y"] == 0).sum())
            assert abs(dropped - n * p) < 6 * (n * p * (1 - p)) ** 0.5 + n * 2.0 ** -17


def test_masks_differ(cmsd):
    x = torch.ones(1 << 16, device="cuda")
    base = dict(seed=1, iteration=2, site=3)
    first = cmsd.dropout(x, 0.5, **base)["y"]
    for more in (dict(seed=2), dict(seed=1 + (1 << 32)), dict(iteration=3), dict(site=4)):
        other = cmsd.dropout(x, 0.5, **{**base, **more})["y"]
        same = int(((other == 0) == (first == 0)).sum())
        assert abs(same - (1 << 15)) < 6 * 128, more
    assert torch.equal(first, cmsd.dropout(x, 0.5, **base)["y"])


def test_dropped_entries_reach_nothing(cmsd):
    n = 5000
    x = torch.full((n,), float("nan"), device="cuda")
    r = torch.randn(n, device="cuda")
    keep = _keep(cmsd, n, 0.3, 8, 0, 0)
    y = cmsd.dropout(x, 0.3, 8, residual=r)["y"]
    assert torch.equal(y[~keep], r[~keep]) and y[keep].isnan().all()
    assert (cmsd.dropout(x, 1.0, 8)["y"] == 0).all()
    assert torch.equal(cmsd.dropout(x, 1.0, 8, residual=r)["y"], r)


def test_linear_and_the_gradient_its_adjoint(cmsd):
    """<c, dropout(x)> = <dropout_backward(c), x>, and differences of the first are the gradient: whole numbers and a
    scale of 2, exactly."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randint(-9, 10, (700,), generator=g, device="cuda").float()
    c = torch.randint(-9, 10, (700,), generator=g, device="cuda").float()
    f = lambda v: float((cmsd.dropout(v, 0.5, 6, 1, 2)["y"] * c).sum())  # noqa: E731
    d_x = cmsd.dropout_backward(c, 0.5, 6, 1, 2)["d_x"]
    assert f(x) == float((d_x * x).sum())
    for e in range(0, 700, 37):
        up, down = x.clone(), x.clone()
        up[e] += 1
        down[e] -= 1
        assert (f(up) - f(down)) / 2 == float(d_x[e])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 9, 1000, 4096 + 3, 100000 + 5])
def test_guard_bands(cmsd, n, dtype):
    x, r = torch.randn(n, device="cuda").to(dtype), torch.randn(n, device="cuda").to(dtype)
    band = torch.full((n + 256,), 77, dtype=dtype, device="cuda")
    y = band[128:128 + n]
    cmsd.dropout(x, 0.2, 3, residual=r, out={"y": y})
    assert (band[:128] == 77).all() and (band[-128:] == 77).all()
    _check(y, x, _keep(cmsd, n, 0.2, 3, 0, 0), 0.2, r)


def test_step_on_the_device_and_replays(cmsd):
    """A captured call draws another mask at each replay, its backward pass the same one; on another stream too."""
    n, p, seed = 10001, 0.25, 12
    x, c = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = {"y": torch.empty_like(x), "d_x": torch.empty_like(x)}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cmsd.dropout(x, p, seed, 5, 1, step=step, out=out)
        cmsd.dropout_backward(c, p, seed, 5, 1, step=step, out=out)
        step.add_(1)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        keep = _keep(cmsd, n, p, seed, 5 + k, 1)
        _check(out["y"], x, keep, p)
        _check(out["d_x"], c, keep, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = cmsd.dropout(x, p, seed, 7, 1)["y"]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, out["y"])


def test_iterations_wrap_as_documented(cmsd):
    x = torch.randn(3000, device="cuda")
    a = cmsd.dropout(x, 0.5, 2, iteration=3)["y"]
    assert torch.equal(a, cmsd.dropout(x, 0.5, 2, iteration=3 + (1 << 30))["y"])
    step = torch.tensor([-2], dtype=torch.int32, device="cuda")
    assert torch.equal(a, cmsd.dropout(x, 0.5, 2, iteration=5, step=step)["y"])


def test_over_2_32_entries(cmsd):
    """Places past 31 and 32 bits."""
    n = (1 << 32) + (1 << 20) + 3
    x = torch.ones(n, dtype=BF16, device="cuda")
    y = cmsd.dropout(x, 0.5, 21, 4, 2)["y"]
    for first in (0, (1 << 31) - 4096, (1 << 32) - 4096, n - 4099):
        first = first // 8 * 8
        m = min(8192, n - first)
        keep = _keep(cmsd, m, 0.5, 21, 4, 2, first)
        assert torch.equal(y[first:first + m] != 0, keep), first


def test_empty(cmsd):
    x = torch.empty(0, 8, device="cuda")
    assert cmsd.dropout(x, 0.1, 1)["y"].shape == (0, 8)
    assert cmsd.dropout_backward(x, 0.1, 1)["d_x"].shape == (0, 8)
