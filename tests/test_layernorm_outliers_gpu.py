"""cmsd_layernorm of rows with entries far above the others, wherever they stand: the other entries and the mean keep
what a mean taken twice in fp32 gives them.

Tolerances, derived and not tuned (u = 2^-24, half a step of fp32).  A row's sums have at most D = 24 + d / 256
additions in a row.  m: the mean, s: the mean of |x - m|, p: the row's first entry.
  c      a first mean, either of the differences from p, each rounded (u), summed (D u), divided (3 u), and p added
         (u of the result): off by (D + 4) u (|p - m| + s) + 2 u |m|; or that of a set of n columns with 2 n >= d,
         off by s (what those are above the mean, the others are below it: the sum over the set is at most d s / 2)
         and by their sum's rounding, (D + 4) u of the mean of their |x| <= |m| + 2 s.  Together:
         dc = s + (D + 4) u (|p - m| + |m| + 3 s) + 2 u |m|
  e      the mean of h = x - c, each rounded, summed, divided: off by de = (D + 4) u (s + dc)
  mean   c + e, rounded: de + 2 u |m|
  h - e  two roundings of the entry's own size, e's error, and e's product with rstd: da = 2 u |x - m| + de + 4 u dc
  var    mean of h^2 less e^2: dv = (D + 8) u (var + dc^2) + 2 dc de; rstd, relative: dr = dv / (var + eps) + 4 u
         (dv / 2 in first order; the other half is above all that follows)
  y      |w| (rstd da + |h| dr) + 3 u (|h w| + |b|), then half a step of y's type
All times 1 + 2^-10 for the products of these with one another.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


def _check(o, x, w, b):
    d = x.shape[1]
    X, W, B = x.double(), w.double(), b.double()
    D = 24 + d / 256
    m = X.mean(1, keepdim=True)
    var = (X - m).square().mean(1, keepdim=True)
    s = (X - m).abs().mean(1, keepdim=True)
    rstd = (var + EPS).rsqrt()
    more = 1 + 2.0 ** -10
    dc = s + (D + 4) * U * ((X[:, :1] - m).abs() + m.abs() + 3 * s) + 2 * U * m.abs()
    de = (D + 4) * U * (s + dc)
    da = 2 * U * (X - m).abs() + de + 4 * U * dc
    dv = (D + 8) * U * (var + dc.square()) + 2 * dc * de
    dr = dv / (var + EPS) + 4 * U
    h = (X - m) * rstd
    want = h * W + B
    tol = more * (W.abs() * (rstd * da + h.abs() * dr) + 3 * U * ((h * W).abs() + B.abs()))
    tol = tol + torch.finfo(x.dtype).eps / 2 * (want.abs() + tol) + 2.0 ** -130
    err = (o["y"].double() - want).abs()
    assert (err <= tol).all(), (err / tol).max()
    err = (o["mean"].double() - m[:, 0]).abs() / (more * (de + 2 * U * m.abs()) + 2.0 ** -140)[:, 0]
    assert (err <= 1).all(), err.max()
    err = (o["rstd"].double() / rstd[:, 0] - 1).abs() / (more * (dr + U))[:, 0]
    assert (err <= 1).all(), err.max()


# a CTA a row (up to 608 rows of 257 to 2048 entries, and over 4096), the grid that stays, rows off 16 bytes, rows that
# do not fit into registers
SIZES = [(4, 2048), (1000, 2048), (608, 1001), (700, 1001), (4, 64), (1000, 200), (9, 4096), (9, 4095), (3, 8192), (3, 16001),
         (3, 32768), (3, 40001)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e2, 1e4, 3e7])
@pytest.mark.parametrize("columns", [(0,), (-1,), (0, 0.3, 0.6, -1), (0.5,)])
@pytest.mark.parametrize("R,d", SIZES)
def test_an_outlier_costs_the_others_nothing(cmsd, R, d, columns, size, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(R + 7 * d)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = 0.3 + n(R, d)
    for k, c in enumerate(columns):
        sign = 1 if k % 2 == 0 else -1
        x[:, d - 1 if c == -1 else int(c * d)] = sign * size * (1 + torch.rand(R, generator=g, device="cuda"))
    x, w, b = x.to(dtype), 1 + 0.2 * n(d), 0.3 * n(d)
    _check(cmsd.layernorm(x, w, b, eps=EPS), x, w, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mean", [1e3, 1e6])
@pytest.mark.parametrize("R,d", SIZES)
def test_outliers_of_rows_far_from_zero(cmsd, R, d, mean, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(R + 7 * d + 1)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = mean * (1 + torch.rand(R, 1, generator=g, device="cuda")) + n(R, d)
    x[::2, 0] = -3e4
    x[1::3, 0] = 0.0
    x, w, b = x.to(dtype), 1 + 0.2 * n(d), 0.3 * n(d)
    _check(cmsd.layernorm(x, w, b, eps=EPS), x, w, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,d", SIZES)
def test_rows_of_one_number_give_the_bias(cmsd, R, d, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(R + 7 * d + 2)
    v = (torch.randn(R, 1, generator=g, device="cuda") * torch.tensor(10.0) ** torch.randint(-9, 14, (R, 1), generator=g, device="cuda")).to(dtype)
    b = torch.randn(d, generator=g, device="cuda")
    o = cmsd.layernorm(v.expand(R, d).contiguous(), torch.full_like(b, 3.0), b, eps=EPS)
    assert torch.equal(o["y"], b.to(dtype).expand(R, d)) and torch.equal(o["mean"], v[:, 0].float())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,d", [(12, 1000), (700, 300), (700, 1000), (700, 1001), (12, 4096), (12, 9000)])
def test_not_finite_stays_in_its_row(cmsd, R, d, dtype):
    """Infinities and NaN among the entries that a first mean is made from, and among the others."""
    g = torch.Generator(device="cuda")
    g.manual_seed(R + 7 * d + 3)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, w, b = n(R, d).to(dtype), n(d), n(d)
    good, bad, inf = cmsd.layernorm(x, w, b), x.clone(), float("inf")
    bad[1, 0], bad[2, -1], bad[4, d // 2], bad[5, 3], bad[7, -1] = inf, inf, -inf, float("nan"), float("nan")
    bad[8, 0], bad[8, -1] = inf, -inf
    o = cmsd.layernorm(bad, w, b)
    rows = [1, 2, 4, 5, 7, 8]
    assert o["y"][rows].isnan().all() and o["rstd"][rows].isnan().all() and not o["mean"][rows].isfinite().any()
    rest = [r for r in range(R) if r not in rows]
    assert all(torch.equal(o[k][rest], good[k][rest]) for k in o)
