"""cmsd_layernorm and cmsd_layernorm_backward against the definitions in 64
bits.

Tolerances, derived and not tuned (u = 2^-24, half a step of fp32; half: that of
the output's dtype).  A row's sums have at most D = 128 + d / 128 additions in a
row, those over rows at most 512 + R / 64; k = D u.
  mean   sums are of differences from a number among the row's, at most 2 s from
         any entry, s the largest |x - mean|; each is rounded (u), so their mean is
         off by (k + u) 2 s: dm = (2 k + 4 u) s; mean itself is rounded, u |mean|.
  var    squares about a mean that is off by dm, summed: relative (k + 4 u) of
         each term, and dm^2; rstd: half of the relative error of var, and 4 u of
         its own: dr = (k + 8 u) / 2 + dm^2 / (2 var) + 4 u (relative; var + eps
         is never below var).
  h      |h| (dr + 4 u) + dm rstd
  y      |w| dh + 2 u (|h w| + |b|), then half of y.
Gradients, with mean and rstd as given: h is off by 3 u |h| + u |mean| rstd (the
difference from the mean is one rounding of a number of its own size), g by u |g|.
  d_x    rstd (2 u |g| + (k + 4 u) a1 + |h| ((k + 8 u) a2) + dh |m2| + 4 u (|g| + |m1| + |h m2|)),
         a1, a2 the means of |g| and |g| (|h| + dh), then half of it.
  d_w    the sum of |d_y| (dh + u |h|), and (512 + R / 64) u of the sum of
         magnitudes; d_b the latter alone; then half of it.
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


def _half(t):
    return torch.finfo(t.dtype).eps / 2


def _inputs(R, d, dtype, wdtype, seed=0, mean=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(R + 7 * d + 1000003 * seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = ((n(R, d) + mean * n(R, 1)) * (0.5 + 2 * torch.rand(R, 1, generator=g, device="cuda"))).to(dtype)
    return x, (1 + 0.2 * n(d)).to(wdtype), (0.3 * n(d)).to(wdtype), n(R, d).to(dtype)


def _check(o, x, w, b, eps=EPS):
    R, d = x.shape
    X = x.double()
    W = w.double() if w is not None else torch.ones(d, dtype=torch.float64, device="cuda")
    B = b.double() if b is not None else torch.zeros(d, dtype=torch.float64, device="cuda")
    k = (128 + d / 128) * U
    m = X.mean(1, keepdim=True)
    var = (X - m).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    s = (X - m).abs().amax(1, keepdim=True)
    dm = (2 * k + 4 * U) * s
    dr = (k + 8 * U) / 2 + dm.square() / (2 * (var + eps)) + 4 * U
    h = (X - m) * rstd
    dh = h.abs() * (dr + 4 * U) + dm * rstd
    want = h * W + B
    tol = W.abs() * dh + 2 * U * ((h * W).abs() + B.abs())
    tol = tol + _half(o["y"]) * (want.abs() + tol) + 2.0 ** -130
    err = (o["y"].double() - want).abs()
    assert (err <= tol).all(), (err - tol).max()
    if "mean" in o:
        assert ((o["mean"].double() - m[:, 0]).abs() <= (dm + U * m.abs() + 2.0 ** -140)[:, 0]).all()
        assert ((o["rstd"].double() / rstd[:, 0] - 1).abs() <= (dr + U)[:, 0]).all()


def _check_grads(o, x, w, mean, rstd, d_y):
    R, d = x.shape
    k = (128 + d / 128) * U
    W = w.double() if w is not None else torch.ones(d, dtype=torch.float64, device="cuda")
    M, S = mean.double()[:, None], rstd.double()[:, None]
    G = d_y.double()
    h = (x.double() - M) * S
    dh = 3 * U * h.abs() + U * M.abs() * S
    g = G * W
    if "d_x" in o:
        m1, m2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
        a1, a2 = g.abs().mean(1, keepdim=True), (g.abs() * (h.abs() + dh)).mean(1, keepdim=True)
        want = S * (g - m1 - h * m2)
        tol = S * (2 * U * g.abs() + (k + 4 * U) * a1 + h.abs() * ((k + 8 * U) * a2 + (g.abs() * dh).mean(1, keepdim=True))
                   + dh * m2.abs() + 4 * U * (g.abs() + m1.abs() + (h * m2).abs()))
        tol = tol + _half(o["d_x"]) * (want.abs() + tol) + 2.0 ** -130
        err = (o["d_x"].double() - want).abs()
        assert (err <= tol).all(), (err - tol).max()
    along = (512 + R / 64) * U
    for name, terms, off in (("d_weight", G * h, G.abs() * (dh + U * h.abs())), ("d_bias", G, 0 * G)):
        if name in o:
            want = terms.sum(0)
            tol = off.sum(0) + along * terms.abs().sum(0)
            tol = tol + _half(o[name]) * (want.abs() + tol) + 2.0 ** -130
            err = (o[name].double() - want).abs()
            assert (err <= tol).all(), (name, (err - tol).max())


# widths about 16-byte boundaries, a warp's and a CTA's share, the widest; rows about a warp and more than a grid
SIZES = [(1, 1), (1, 2), (3, 7), (5, 8), (2, 31), (33, 32), (9, 33), (64, 64), (65, 100), (17, 255), (300, 256),
         (31, 257), (16, 512), (7, 513), (130, 1000), (333, 1001), (64, 1024), (1000, 1026), (40, 2040), (77, 2048),
         (12, 2049), (5, 4096), (6, 4100), (3, 8191), (9, 8192), (2, 8200), (4, 16384), (3, 16390), (2, 32768),
         (2, 65535), (3, 65536), (5000, 40), (20011, 64), (4099, 520)]


@pytest.mark.parametrize("dtype,wdtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("R,d", SIZES)
def test_norm_and_gradients(cmsd, R, d, dtype, wdtype):
    x, w, b, d_y = _inputs(R, d, dtype, wdtype)
    o = cmsd.layernorm(x, w, b, eps=EPS)
    _check(o, x, w, b)
    y = cmsd.layernorm(x, w, b, eps=EPS, stats=False)
    assert list(y) == ["y"] and torch.equal(y["y"], o["y"])
    gr = cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], d_y)
    assert gr["d_weight"].dtype is wdtype and gr["d_x"].dtype is dtype
    _check_grads(gr, x, w, o["mean"], o["rstd"], d_y)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,d", [(255, 2048), (256, 2047), (257, 2046), (608, 2048), (608, 65), (609, 2048), (609, 65), (608, 2050),
                                 (304, 4097), (305, 4097), (608, 2056), (100, 8192), (30, 8191), (30, 8194)])
def test_gradients_about_the_rows_of_one_launch(cmsd, R, d, dtype):
    """Rows about those that a thread requests at once, and about the most that are summed without a join."""
    x, w, b, d_y = _inputs(R, d, dtype, F32, seed=3)
    o = cmsd.layernorm(x, w, b, eps=EPS)
    _check_grads(cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], d_y), x, w, o["mean"], o["rstd"], d_y)


@pytest.mark.parametrize("R", [3, 700])
def test_captured_behind_another_stream(cmsd, R):
    """In a graph, calls that wait for the launch before and for another stream's work at once."""
    d = 264
    x, w, b, d_y = _inputs(R, d, BF16, F32, seed=4)
    ref = cmsd.layernorm(x, w, b)
    want = cmsd.layernorm_backward(x, w, ref["mean"], ref["rstd"], d_y)
    src, src_y = x.clone(), d_y.clone()
    x.zero_()
    d_y.zero_()
    out = {k: torch.empty_like(v) for k, v in {**ref, **want}.items()}
    ws = cmsd.layernorm_backward_workspace(R, d)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            d_y.copy_(src_y)
        x.copy_(src)
        cmsd.layernorm(x, w, b, out=out)
        main.wait_stream(side)
        cmsd.layernorm_backward(x, w, out["mean"], out["rstd"], d_y, out=out, ws=ws)
        cmsd.dropout(out["d_x"], 0.0, 1, out={"y": x})
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], {**ref, **want}[k]), k
        assert torch.equal(x, want["d_x"])


@pytest.mark.parametrize("R,d", [(1, 16), (70, 1000), (300, 2048), (40, 1001), (9, 20000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_without_parameters(cmsd, R, d, dtype):
    x, w, b, d_y = _inputs(R, d, dtype, dtype, seed=1)
    _check(cmsd.layernorm(x), x, None, None)
    _check(cmsd.layernorm(x, w), x, w, None)
    o = cmsd.layernorm(x, bias=b)
    _check(o, x, None, b)
    gr = cmsd.layernorm_backward(x, None, o["mean"], o["rstd"], d_y)
    assert gr["d_weight"].dtype is dtype
    _check_grads(gr, x, None, o["mean"], o["rstd"], d_y)


@pytest.mark.parametrize("R,d", [(70, 1000), (500, 2048), (40, 1001), (9, 20000), (3000, 64)])
def test_each_gradient_alone_is_the_same(cmsd, R, d):
    x, w, b, d_y = _inputs(R, d, BF16, F32, seed=2)
    o = cmsd.layernorm(x, w, b)
    both = cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], d_y)
    for keep in range(1, 8):
        want = [bool(keep & 1), bool(keep & 2), bool(keep & 4)]
        some = cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], d_y, *want)
        assert list(some) == [n for n, t in zip(("d_x", "d_weight", "d_bias"), want) if t]
        for n in some:
            assert torch.equal(some[n], both[n]), n
    with pytest.raises(cmsd.CmsdError):
        cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], d_y, False, False, False)


def test_no_rows(cmsd):
    x, w, b, d_y = _inputs(1, 40, F32, F32)
    assert cmsd.layernorm(x[:0], w, b)["y"].shape == (0, 40)
    e = torch.empty(0, device="cuda")
    gr = cmsd.layernorm_backward(x[:0], w, e, e, d_y[:0], out={"d_weight": torch.full_like(w, 3), "d_bias": torch.full_like(w, 3)})
    assert gr["d_x"].shape == (0, 40) and (gr["d_weight"] == 0).all() and (gr["d_bias"] == 0).all()


@pytest.mark.parametrize("d", [64, 1000, 1001, 2048, 16390])
@pytest.mark.parametrize("mean", [300.0, 30000.0])
def test_means_far_from_zero(cmsd, d, mean):
    """Rows whose mean is far above their spread: the differences from it are what counts."""
    x, w, b, _ = _inputs(50, d, F32, F32, seed=3, mean=mean)
    _check(cmsd.layernorm(x, w, b), x, w, b)


@pytest.mark.parametrize("d", [8, 1000, 2047, 4096, 30000])
def test_outliers_and_constant_rows(cmsd, d):
    """One entry far above the others at either end or within, rows of one number, of zeros, of the smallest ones."""
    x, w, b, _ = _inputs(9, d, F32, F32, seed=4)
    x[0, 0], x[1, -1], x[2, d // 2] = 1e4, -1e4, 1e6
    x[3], x[4], x[5], x[6] = 0.0, 7.0, 1e-30, -12345.678
    x[7, :] = 1e15
    x[8] = x[8] * 1e15
    _check(cmsd.layernorm(x, w, b), x, w, b)


@pytest.mark.parametrize("eps", [1e-12, 1e-3, 10.0])
def test_eps(cmsd, eps):
    x, w, b, _ = _inputs(20, 136, F32, F32, seed=5)
    x[0] *= 1e-4
    _check(cmsd.layernorm(x, w, b, eps=eps), x, w, b, eps=eps)


@pytest.mark.parametrize("d", [40, 1000, 1001, 20000])
def test_not_finite_stays_in_its_row(cmsd, d):
    x, w, b, d_y = _inputs(40, d, BF16, F32, seed=6)
    good = cmsd.layernorm(x, w, b)
    bad = x.clone()
    bad[3, d - 1], bad[17, 0] = float("nan"), float("inf")
    o = cmsd.layernorm(bad, w, b)
    assert o["y"][3].isnan().all() and o["y"][17].isnan().all()
    gr = cmsd.layernorm_backward(bad, w, o["mean"], o["rstd"], d_y)
    ref = cmsd.layernorm_backward(x, w, good["mean"], good["rstd"], d_y)
    rest = [r for r in range(40) if r not in (3, 17)]
    for k in o:
        assert torch.equal(o[k][rest], good[k][rest])
    assert torch.equal(gr["d_x"][rest], ref["d_x"][rest]) and gr["d_x"][3].isnan().all()
    assert torch.equal(gr["d_bias"], ref["d_bias"])


@pytest.mark.parametrize("d", [5, 24])
def test_gradients_are_the_differences(cmsd, d):
    """Against central differences of L = sum c y in 64 bits (step 1e-4: the third derivative's part is below 1e-6)."""
    R = 4
    x, w, b, c = _inputs(R, d, F32, F32, seed=7)
    o = cmsd.layernorm(x, w, b)
    gr = cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], c)

    def loss(X, W, B):
        m = X.mean(1, keepdim=True)
        return float((((X - m) / ((X - m).square().mean(1, keepdim=True) + EPS).sqrt() * W + B) * c.double()).sum())

    args = [x.double(), w.double(), b.double()]
    for name, which in (("d_x", 0), ("d_weight", 1), ("d_bias", 2)):
        flat = args[which].reshape(-1)
        got = gr[name].double().reshape(-1)
        for e in range(flat.numel()):
            keep = float(flat[e])
            flat[e] = keep + 1e-4
            up = loss(*args)
            flat[e] = keep - 1e-4
            down = loss(*args)
            flat[e] = keep
            assert abs((up - down) / 2e-4 - float(got[e])) <= 2e-5 * (1 + abs(float(got[e]))), (name, e)


@pytest.mark.parametrize("dtype,wdtype", [(F32, F32), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("R,d", [(41, 136), (41, 137), (600, 2048), (7, 20001)])
def test_guard_bands(cmsd, R, d, dtype, wdtype):
    x, w, b, d_y = _inputs(R, d, dtype, wdtype, seed=8)

    def banded(shape, dtype):
        count = 1
        for s in shape:
            count *= s
        t = torch.full((count + 256,), 77, dtype=dtype, device="cuda")
        return t, t[128:128 + count].view(shape)

    bands, out = [], {}
    for name, shape, t in (("y", (R, d), dtype), ("mean", (R,), F32), ("rstd", (R,), F32), ("d_x", (R, d), dtype),
                           ("d_weight", (d,), wdtype), ("d_bias", (d,), wdtype),
                           ("ws", (cmsd.lib().cmsd_layernorm_backward_workspace_bytes(R, d),), torch.uint8)):
        band, out[name] = banded(shape, t)
        bands.append(band)
    cmsd.layernorm(x, w, b, out=out)
    cmsd.layernorm_backward(x, w, out["mean"], out["rstd"], d_y, out=out, ws=out["ws"])
    for t in bands:
        assert (t[:128] == 77).all() and (t[-128:] == 77).all()
    _check({k: out[k] for k in ("y", "mean", "rstd")}, x, w, b)
    _check_grads({k: out[k] for k in ("d_x", "d_weight", "d_bias")}, x, w, out["mean"], out["rstd"], d_y)


@pytest.mark.parametrize("R,d", [(60, 1000), (2000, 512), (900, 2048), (50, 16390)])
def test_equal_calls_on_streams_and_in_a_graph(cmsd, R, d):
    one, two = _inputs(R, d, BF16, F32, seed=9), _inputs(R, d, BF16, F32, seed=10)
    ws = cmsd.layernorm_backward_workspace(R, d)

    def step(x, w, b, d_y, out=None, ws=None):
        o = dict(out or {})
        o.update(cmsd.layernorm(x, w, b, out=o))
        o.update(cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], d_y, out=o, ws=ws))
        return o

    a, b = step(*one, ws=ws), step(*one)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = step(*one)
    want = step(*two)
    torch.cuda.current_stream().wait_stream(side)
    for k in a:
        assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]), k
    bufs = [t.clone() for t in one]
    out = {k: torch.empty_like(v) for k, v in a.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*bufs, out=out, ws=ws)
    for src, ref in ((one, a), (two, want), (one, a)):
        for dst, s in zip(bufs, src):
            dst.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        for k in a:
            assert torch.equal(out[k], ref[k]), k


def test_more_than_2_31_entries(cmsd):
    R, d = 1100000, 2048
    x = torch.zeros(R, d, dtype=BF16, device="cuda")
    rows = [0, 1048575, 1048576, 1048577, R - 1]
    some, w, b, d_y = _inputs(len(rows), d, BF16, F32, seed=11)
    x[rows] = some
    o = cmsd.layernorm(x, w, b)
    _check({k: v[rows] for k, v in o.items()}, some, w, b)
    g = torch.zeros(R, d, dtype=BF16, device="cuda")
    g[rows] = d_y
    gr = cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], g, out={"d_x": o["y"]})
    _check_grads({"d_x": gr["d_x"][rows], "d_weight": gr["d_weight"], "d_bias": gr["d_bias"]}, some, w, o["mean"][rows],
                 o["rstd"][rows], d_y)
