"""cmsd_embedding and cmsd_embedding_backward against the definitions in 64
bits.

Tolerances, derived and not tuned (u = 2^-24, half a step of fp32; half: that of
the dtype, 2^-8 for bf16, u for fp32):
  x        one product in fp32, rounded to the dtype: u and half of it.
  d_table  a sum of n entries in fp32 in some order: n u of the sum of their
           magnitudes; the product with scale and the sum with what was there:
           u of each; then half of the result.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

IGNORE = -100
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


@pytest.fixture(autouse=True)
def no_errors_before(cmsd):
    cmsd.embedding_errors()


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _gen(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(hash(key) % (1 << 40))
    return g


def _tokens(R, V, g, ignored=0.0, hot=False):
    """Frequencies that fall as one over the rank; hot: one token has half of the rows."""
    rank = torch.exp(torch.rand(R, generator=g, device="cuda", dtype=torch.float64) * math.log(V + 1)).long() - 1
    t = torch.randperm(V, generator=g, device="cuda")[rank.clamp(0, V - 1)]
    if hot:
        t[torch.rand(R, generator=g, device="cuda") < 0.5] = V - 1
    t[torch.rand(R, generator=g, device="cuda") < ignored] = IGNORE
    return t.int()


def _check_rows(x, tokens, table, scale, ignore=IGNORE):
    keep = (tokens != ignore) & (tokens >= 0) & (tokens < table.shape[0])
    want = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    want[keep] = table[tokens[keep].long()].double() * scale
    tol = want.abs() * (U + _half(table.dtype) * (1 + U)) + 2.0 ** -140
    assert ((x.double() - want).abs() <= tol).all()
    assert (x[~keep] == 0).all()


def _check_table(got, tokens, d_x, V, scale, ignore=IGNORE, base=None):
    keep = (tokens != ignore) & (tokens >= 0) & (tokens < V)
    t = tokens[keep].long()
    rows = d_x[keep].double()
    d = d_x.shape[1]
    n = torch.bincount(t, minlength=V)
    want = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, t, rows) * scale
    mags = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, t, rows.abs()) * abs(scale)
    tol = (n[:, None] + 2) * U * mags + 2.0 ** -120
    if base is not None:
        want += base.double()
        tol += U * (want.abs() + tol)
    tol += _half(d_x.dtype) * (want.abs() + tol)
    some = n > 0
    err = (got.double() - want).abs()
    assert (err <= tol)[some].all(), (err - tol)[some].max()
    if base is None:
        assert (got[~some] == 0).all()
    else:
        assert torch.equal(got[~some], base[~some])


# widths about 16-byte boundaries, rows about a warp, a CTA and the ways of ordering them, hot tokens
SIZES = [(1, 1, 1), (1, 8, 2), (2, 3, 2), (7, 1000, 50), (31, 64, 33), (33, 1001, 70), (64, 1024, 3001), (65, 40, 1),
         (255, 72, 129), (256, 12, 31000), (257, 24, 257), (1000, 130, 4), (1025, 264, 1024), (2049, 66, 70001),
         (4099, 16, 9), (4099, 48, 32001), (9001, 20, 500), (20001, 8, 40000), (33000, 10, 3), (70001, 16, 128256)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,d,V", SIZES)
def test_rows_and_gradient(cmsd, R, d, V, dtype):
    g = _gen(R, d, V)
    tokens = _tokens(R, V, g, ignored=0.2 if R % 2 else 0.0, hot=R % 3 == 0)
    table = torch.randn(V, d, generator=g, device="cuda").to(dtype)
    d_x = torch.randn(R, d, generator=g, device="cuda").to(dtype)
    scale = float(torch.tensor(math.sqrt(d)))
    _check_rows(cmsd.embedding(tokens, table, scale=scale)["x"], tokens, table, scale)
    ws = cmsd.embedding_backward_workspace(R, d, V)
    got = cmsd.embedding_backward(tokens, d_x, V, scale=scale, ws=ws)["d_table"]
    _check_table(got, tokens, d_x, V, scale)
    base = torch.randn(V, d, generator=g, device="cuda").to(dtype)
    added = cmsd.embedding_backward(tokens, d_x, V, scale=scale, add=True, out={"d_table": base.clone()}, ws=ws)
    _check_table(added["d_table"], tokens, d_x, V, scale, base=base)
    assert cmsd.workspace_errors(ws) == 0 and cmsd.embedding_errors() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,d,V", [(3, 65536, 5), (40, 65535, 7), (600, 2048, 128256), (5000, 2046, 1000)])
def test_wide_rows(cmsd, R, d, V, dtype):
    g = _gen(R, d, V, 1)
    tokens = _tokens(R, V, g, ignored=0.1)
    table = torch.randn(V, d, generator=g, device="cuda").to(dtype)
    d_x = torch.randn(R, d, generator=g, device="cuda").to(dtype)
    _check_rows(cmsd.embedding(tokens, table)["x"], tokens, table, 1.0)
    _check_table(cmsd.embedding_backward(tokens, d_x, V)["d_table"], tokens, d_x, V, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,d,V", [(8191, 64, 900), (8192, 64, 900), (8193, 512, 40), (9001, 504, 3000), (40000, 8, 70000), (8200, 520, 50),
                                   (12001, 256, 2000), (7168, 64, 900), (7169, 64, 900), (16384, 24, 40),
                                   (16385, 24, 40), (32767, 24, 3000), (32768, 24, 3000), (9728, 64, 30),
                                   (9729, 64, 30), (19457, 512, 300), (50000, 128, 12), (38913, 256, 7)])
def test_narrow_rows(cmsd, R, d, V, dtype):
    """Many rows of up to 64 vectors, which are looked up whatever row a vector is of, and one that is wider."""
    tokens = _tokens(R, V, _gen(R, 9), ignored=0.2)
    tokens[5], tokens[R - 1], tokens[0] = V, -1, 0
    table, d_x = (torch.randn(n, d, generator=_gen(d, 9), device="cuda").to(dtype) for n in (V, R))
    _check_rows(cmsd.embedding(tokens, table, scale=1.5)["x"], tokens, table, 1.5)
    assert cmsd.embedding_errors() == 1
    _check_table(cmsd.embedding_backward(tokens, d_x, V, scale=1.5)["d_table"], tokens, d_x, V, 1.5)
    assert cmsd.embedding_errors() == 1


@pytest.mark.parametrize("R,V", [(8192, 300), (600011, 40), (8193, 1 << 20), (9000, (1 << 21) + 5), (530000, 3000), (10000, 1)])
def test_many_rows_and_tokens(cmsd, R, V):
    """Ordering with over 2048 rows a CTA, with two and three passes, and of one token alone."""
    d = 8
    g = _gen(R, V, 8)
    tokens = _tokens(R, V, g, ignored=0.1)
    d_x = torch.randn(R, d, generator=g, device="cuda")
    _check_table(cmsd.embedding_backward(tokens, d_x, V)["d_table"], tokens, d_x, V, 1.0)


def test_the_largest_vocabulary(cmsd):
    """2^30 - 1 tokens, one column: four passes; the table's last bytes are not a whole vector."""
    V, R = (1 << 30) - 1, 9001
    g = _gen(5)
    tokens = torch.randint(0, V, (R,), generator=g, device="cuda").int()
    tokens[:3000] = tokens[3000:6000]
    tokens[0], tokens[1], tokens[2] = V - 1, V - 1, 0
    d_x = torch.randint(1, 5, (R, 1), generator=g, device="cuda").bfloat16()
    out = torch.full((V + 128, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    got = cmsd.embedding_backward(tokens, d_x, V, out={"d_table": out[:V]})["d_table"]
    rows, at = torch.unique(tokens.long(), return_inverse=True)
    want = torch.zeros(rows.numel(), dtype=torch.float64, device="cuda").index_add_(0, at, d_x[:, 0].double())
    assert torch.equal(got[rows, 0].double(), want)                  # small whole numbers: exact
    assert int(torch.count_nonzero(got)) == rows.numel() and (out[V:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,d,V", [(400, 129, 20011), (100, 1001, 3001), (512, 3, 100003), (70, 2046, 700), (9, 1, 5000), (300, 130, 301), (5, 65533, 7)])
def test_zeros_of_rows_off_16_bytes(cmsd, R, d, V, dtype):
    """Few tokens: what was there goes everywhere, and no sum is written over."""
    tokens = _tokens(R, V, _gen(R, 8), ignored=0.1)
    tokens[0] = V - 1
    d_x = torch.randn(R, d, generator=_gen(d, 8), device="cuda").to(dtype)
    for _ in range(3):
        t = torch.full((V, d), 77, dtype=dtype, device="cuda")
        cmsd.embedding_backward(tokens, d_x, V, out={"d_table": t})
        _check_table(t, tokens, d_x, V, 1.0)


@pytest.mark.parametrize("R", [1, 33, 5000])
def test_every_row_padding(cmsd, R):
    d, V = 24, 100
    tokens = torch.full((R,), IGNORE, dtype=torch.int32, device="cuda")
    d_x = torch.full((R, d), float("nan"), device="cuda")
    table = torch.randn(V, d, device="cuda")
    assert (cmsd.embedding(tokens, table)["x"] == 0).all()
    assert (cmsd.embedding_backward(tokens, d_x, V, out={"d_table": torch.full_like(table, 3.0)})["d_table"] == 0).all()
    base = table.clone()
    assert torch.equal(cmsd.embedding_backward(tokens, d_x, V, add=True, out={"d_table": base})["d_table"], table)
    assert cmsd.embedding_errors() == 0


def test_no_rows(cmsd):
    tokens = torch.empty(0, dtype=torch.int32, device="cuda")
    table = torch.randn(9, 16, device="cuda")
    assert cmsd.embedding(tokens, table)["x"].shape == (0, 16)
    out = torch.full_like(table, 3.0)
    assert (cmsd.embedding_backward(tokens, table[:0], 9, out={"d_table": out})["d_table"] == 0).all()
    base = table.clone()
    cmsd.embedding_backward(tokens, table[:0], 9, add=True, out={"d_table": base})
    assert torch.equal(base, table)


@pytest.mark.parametrize("R", [50, 3000, 40000])
def test_tokens_out_of_range(cmsd, R):
    """Rows of zeros, no gradient, an error bit in the workspace and the device's; the other rows as without them."""
    d, V = 24, 300
    g = _gen(R)
    tokens = _tokens(R, V, g)
    bad = torch.rand(R, generator=g, device="cuda") < 0.1
    bad[R // 2] = True
    wrong = tokens.clone()
    wrong[bad] = torch.tensor([V, -1, 2**31 - 1, -2**31, 5 * V], dtype=torch.int32,
                              device="cuda")[torch.arange(int(bad.sum()), device="cuda") % 5]
    gone = tokens.clone()
    gone[bad] = IGNORE
    table = torch.randn(V, d, generator=g, device="cuda")
    d_x = torch.randn(R, d, generator=g, device="cuda")
    assert torch.equal(cmsd.embedding(wrong, table)["x"], cmsd.embedding(gone, table)["x"])
    assert cmsd.embedding_errors() == 1 and cmsd.embedding_errors() == 0
    ws = cmsd.embedding_backward_workspace(R, d, V)
    a = cmsd.embedding_backward(wrong, d_x, V, ws=ws)["d_table"]
    assert cmsd.workspace_errors(ws) == 1 and cmsd.workspace_errors(ws) == 0 and cmsd.embedding_errors() == 1
    _check_table(a, wrong, d_x, V, 1.0)
    assert torch.equal(a, cmsd.embedding_backward(gone, d_x, V, ws=ws)["d_table"])
    assert cmsd.workspace_errors(ws) == 0 and cmsd.embedding_errors() == 0


def test_ignore_index_inside_the_vocabulary(cmsd):
    R, d, V = 900, 40, 50
    g = _gen(7)
    tokens = _tokens(R, V, g)
    tokens[::3] = 1
    table, d_x = torch.randn(V, d, generator=g, device="cuda"), torch.randn(R, d, generator=g, device="cuda")
    _check_rows(cmsd.embedding(tokens, table, ignore_index=1)["x"], tokens, table, 1.0, ignore=1)
    got = cmsd.embedding_backward(tokens, d_x, V, ignore_index=1)["d_table"]
    _check_table(got, tokens, d_x, V, 1.0, ignore=1)
    assert (got[1] == 0).all() and cmsd.embedding_errors() == 0


@pytest.mark.parametrize("R", [40, 20000])
def test_values_that_are_not_finite(cmsd, R):
    """They stay in their own token's row."""
    d, V = 24, 60
    tokens = _tokens(R, V, _gen(R, 2))
    tokens[3] = 7
    d_x = torch.randn(R, d, device="cuda")
    d_x[3, 5], d_x[3, 6] = float("nan"), float("inf")
    got = cmsd.embedding_backward(tokens, d_x, V)["d_table"]
    assert got[7, 5].isnan() and not got[7, 6].isfinite()
    rest = torch.ones(V, d, dtype=torch.bool, device="cuda")
    rest[7, 5:7] = False
    assert got[rest].isfinite().all()


def test_gradient_is_the_differences(cmsd):
    """dL/dtable of L = sum c x against L's differences, which are exact for a linear function but for rounding."""
    R, d, V, scale = 60, 5, 11, 3.0
    g = _gen(3)
    tokens = _tokens(R, V, g, ignored=0.2)
    table = torch.randint(-8, 9, (V, d), generator=g, device="cuda").float()
    c = torch.randint(-8, 9, (R, d), generator=g, device="cuda").float()
    got = cmsd.embedding_backward(tokens, c, V, scale=scale)["d_table"]
    for v in range(V):
        for j in range(d):
            up, down = table.clone(), table.clone()
            up[v, j] += 1.0
            down[v, j] -= 1.0
            diff = (cmsd.embedding(tokens, up, scale=scale)["x"] * c).sum() - (cmsd.embedding(tokens, down, scale=scale)["x"] * c).sum()
            assert float(diff) / 2 == float(got[v, j])          # whole numbers: no rounding


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,d,V", [(100, 33, 60), (5000, 64, 900), (20000, 40, 32001)])
def test_guard_bands(cmsd, R, d, V, dtype):
    """Nothing is written before or behind the outputs and the workspace."""
    tokens = _tokens(R, V, _gen(R, 3), ignored=0.1)
    table, d_x = torch.randn(V, d, device="cuda").to(dtype), torch.randn(R, d, device="cuda").to(dtype)

    def banded(count, dtype):
        t = torch.full((count + 256,), 77, dtype=dtype, device="cuda")
        return t, t[128:128 + count]

    xb, x = banded(R * d, dtype)
    tb, t = banded(V * d, dtype)
    wb, ws = banded(cmsd.lib().cmsd_embedding_backward_workspace_bytes(R, d, V), torch.uint8)
    cmsd.embedding(tokens, table, out={"x": x.view(R, d)})
    cmsd.embedding_backward(tokens, d_x, V, out={"d_table": t.view(V, d)}, ws=ws)
    for b in (xb, tb, wb):
        assert (b[:128] == 77).all() and (b[-128:] == 77).all()
    _check_rows(x.view(R, d), tokens, table, 1.0)
    _check_table(t.view(V, d), tokens, d_x, V, 1.0)


@pytest.mark.parametrize("R,d,V", [(90, 64, 500), (6000, 72, 3000), (30000, 64, 32000)])
def test_equal_calls_on_streams_and_in_a_graph(cmsd, R, d, V):
    """Twice the same to the bit, on another stream at the same time, and captured with new inputs in the same buffers."""
    def made(seed):
        g = _gen(R, seed, 4)
        return _tokens(R, V, g, ignored=0.2), torch.randn(R, d, generator=g, device="cuda").bfloat16()

    table = torch.randn(V, d, device="cuda").bfloat16()

    def step(t, d_x, out=None, ws=None):
        o = dict(out or {})
        o.update(cmsd.embedding(t, table, scale=2.0, out=o))
        o.update(cmsd.embedding_backward(t, d_x, V, scale=2.0, out=o, ws=ws))
        return o

    one, two = made(0), made(1)
    ws = cmsd.embedding_backward_workspace(R, d, V)
    a, b = step(*one, ws=ws), step(*one)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = step(*one)
    want = step(*two)                                    # at the same time as the other stream's
    torch.cuda.current_stream().wait_stream(side)
    for k in a:
        assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]), k
    tb, xb = one[0].clone(), one[1].clone()
    out = {k: torch.empty_like(v) for k, v in a.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(tb, xb, out=out, ws=ws)
    for src, ref in ((one, a), (two, want), (one, a)):
        tb.copy_(src[0])
        xb.copy_(src[1])
        graph.replay()
        torch.cuda.synchronize()
        for k in a:
            assert torch.equal(out[k], ref[k]), k


def test_a_table_of_over_2_31_entries(cmsd):
    """Offsets past 32 bits, in the table and in its gradient."""
    V, d, R = 1100000, 2048, 70
    table = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    tokens = torch.randint(V - 1000, V, (R,), device="cuda").int()
    tokens[:5] = torch.tensor([0, 1048575, 1048576, 1048577, V - 1], device="cuda")
    table[tokens.long()] = torch.randn(R, d, device="cuda").bfloat16()
    x = cmsd.embedding(tokens, table)["x"]
    assert torch.equal(x, table[tokens.long()])
    d_table = cmsd.embedding_backward(tokens, x, V, out={"d_table": table})["d_table"]
    rows = torch.unique(tokens.long())
    sums = torch.zeros(rows.numel(), d, dtype=torch.float64, device="cuda")
    at = torch.searchsorted(rows, tokens.long())
    sums.index_add_(0, at, x.double())
    mags = torch.zeros_like(sums).index_add_(0, at, x.double().abs())
    tol = (R + 2) * U * mags
    tol += 2.0 ** -8 * (sums.abs() + tol)
    assert ((d_table[rows].double() - sums).abs() <= tol).all()
    assert int((d_table != 0).any(1).sum()) == rows.numel()
