"""cmsd_lmhead_loss and cmsd_lmhead_loss_backward against the definitions in
64 bits.

Tolerances, derived and not tuned (u = 2^-24, b = 2^-8: half a step of fp32 and
bf16):
  logits   a dot product of d exact products, summed in fp32 in some order:
           |dz| <= d 2^-23 sum_j |h_j w_vj| =: e (each addition off by at most
           one unit in the last place of a partial sum).
  lse      the largest e of the row; the exponentials (2^-22 of each, and the
           rounding of an exponent of at most 2^8: 2^-16 of a term that small
           changes the sum by under 2^-16 2^-22) and their sum (at most 512
           additions in a row: 2^-15); the logarithm and its scale: 4 u |lse|.
  loss     lse's and the label's logit.
  P        the exponential's 2^-22, e and lse's rounding: (e + 2^-20) p, and
           its rounding to bf16: b |P|.
  sums     K 2^-23 of the sum of magnitudes, and b of the result.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

IGNORE = -100


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


def _inputs(R, d, V, seed=0, ignored=0.0, scale=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 * seed + R + 7 * d + 13 * V)
    w = (torch.randn(V, d, generator=g, device="cuda") * (scale / math.sqrt(d))).bfloat16()
    y = torch.randint(0, V, (R,), generator=g, device="cuda")
    up = 6.0 * torch.rand(R, 1, generator=g, device="cuda")
    wy = w[y].float()
    h = (torch.randn(R, d, generator=g, device="cuda") + up * wy / wy.square().sum(1, keepdim=True)).bfloat16()
    gone = torch.rand(R, generator=g, device="cuda") < ignored
    y[gone] = IGNORE
    grad = torch.randn(R, generator=g, device="cuda") / R
    return h, w, y.int(), grad


def _logits(h, w):
    h, w = h.double(), w.double()
    return h @ w.T, h.shape[1] * 2.0 ** -23 * (h.abs() @ w.abs().T)


def _check_loss(o, h, w, y, V):
    keep = (y >= 0) & (y < V)
    z, e = _logits(h[keep], w)
    lse = torch.logsumexp(z, 1)
    el = e.amax(1)
    tol = el + 2.0 ** -15 + 4 * 2.0 ** -24 * lse.abs()
    got = o["lse"][keep].double()
    assert (got - lse).abs().le(tol).all(), (got - lse).abs().max()
    zy = z.gather(1, y[keep].long()[:, None])[:, 0]
    tol = tol + el + 2.0 ** -23 * (lse - zy).abs()
    got = o["loss"][keep].double()
    assert (got - (lse - zy)).abs().le(tol).all(), (got - (lse - zy)).abs().max()
    assert (o["lse"][~keep] == 0).all() and (o["loss"][~keep] == 0).all()


def _check_grads(o, h, w, y, lse, grad, V):
    """Against the definition, with lse as it was given."""
    keep = (y >= 0) & (y < V)
    R, d = h.shape
    hk, yk = h[keep], y[keep].long()
    z, e = _logits(hk, w)
    p = torch.exp(z - lse[keep].double()[:, None])
    off = p * (e + 2.0 ** -20)
    p[torch.arange(hk.shape[0], device="cuda"), yk] -= 1.0
    g = grad[keep].double()[:, None]
    p, off = p * g, off * g.abs()
    b = 2.0 ** -8
    off = off + b * (p.abs() + off) + 2.0 ** -120
    if "d_hidden" in o:
        want = torch.zeros(R, d, dtype=torch.float64, device="cuda")
        tol = want.clone()
        want[keep] = p @ w.double()
        tol[keep] = (off + V * 2.0 ** -23 * p.abs()) @ w.double().abs()
        tol = tol + b * (want.abs() + tol)
        err = (o["d_hidden"].double() - want).abs()
        assert err.le(tol).all(), (err - tol).max()
    if "d_weight" in o:
        want = p.T @ hk.double()
        tol = (off + hk.shape[0] * 2.0 ** -23 * p.abs()).T @ hk.double().abs()
        tol = tol + b * (want.abs() + tol)
        err = (o["d_weight"].double() - want).abs()
        assert err.le(tol).all(), (err - tol).max()


# rows about a tile of 128 and 256, vocabularies about one of 128 and 256, widths about a box of 64
SIZES = [(1, 8, 2), (1, 64, 128), (2, 72, 257), (33, 136, 1000), (64, 64, 129), (127, 128, 255), (128, 200, 256),
         (129, 8, 300), (255, 512, 511), (256, 264, 513), (257, 320, 4099), (600, 1040, 770), (5, 2048, 32001),
         (32, 1000, 20000), (96, 96, 5000), (97, 2056, 39001), (16, 704, 1 << 18)]


@pytest.mark.parametrize("R,d,V", SIZES)
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_loss_and_gradients(cmsd, R, d, V, ignored):
    h, w, y, g = _inputs(R, d, V, ignored=ignored)
    ws = cmsd.lmhead_loss_workspace(R, d, V)
    o = cmsd.lmhead_loss(h, w, y, ws=ws)
    _check_loss(o, h, w, y, V)
    wb = cmsd.lmhead_loss_backward_workspace(R, d, V)
    gr = cmsd.lmhead_loss_backward(h, w, y, o["lse"], g, ws=wb)
    _check_grads(gr, h, w, y, o["lse"], g, V)
    assert cmsd.workspace_errors(ws) == 0 and cmsd.workspace_errors(wb) == 0


@pytest.mark.parametrize("hidden,weight", [(True, False), (False, True)])
@pytest.mark.parametrize("R,d,V", [(40, 136, 700), (300, 256, 1025)])
def test_one_gradient_alone_is_the_same(cmsd, R, d, V, hidden, weight):
    h, w, y, g = _inputs(R, d, V, ignored=0.2)
    lse = cmsd.lmhead_loss(h, w, y)["lse"]
    both = cmsd.lmhead_loss_backward(h, w, y, lse, g)
    one = cmsd.lmhead_loss_backward(h, w, y, lse, g, hidden_grad=hidden, weight_grad=weight)
    assert sorted(one) == [n for n, k in (("d_hidden", hidden), ("d_weight", weight)) if k]
    for k in one:
        assert torch.equal(one[k], both[k]), k
    with pytest.raises(cmsd.CmsdError):
        cmsd.lmhead_loss_backward(h, w, y, lse, g, hidden_grad=False, weight_grad=False)


@pytest.mark.parametrize("R,d,V", [(2048, 64, 40000), (1000, 128, 150000), (100, 72, 300001)])
def test_vocabulary_in_pieces(cmsd, R, d, V):
    """P over the whole vocabulary is over 128 MB: several pieces, the last one short."""
    h, w, y, g = _inputs(R, d, V, ignored=0.1)
    o = cmsd.lmhead_loss(h, w, y)
    rows = torch.arange(0, R, 41, device="cuda")
    _check_loss({k: v[rows] for k, v in o.items()}, h[rows], w, y[rows], V)
    _check_grads(cmsd.lmhead_loss_backward(h, w, y, o["lse"], g), h, w, y, o["lse"], g, V)


def test_gradient_against_differences(cmsd):
    """Central differences of the loss in 64 bits, along single entries of h and of W.  A step t leaves an
    error of t^2 / 6 of the third derivative, at most 4 |w|_max^3 sum |g| (of |h|_max^3 for W)."""
    R, d, V = 37, 72, 300
    h, w, y, g = _inputs(R, d, V, ignored=0.2)
    lse = cmsd.lmhead_loss(h, w, y)["lse"]
    o = cmsd.lmhead_loss_backward(h, w, y, lse, g)
    keep = y >= 0

    def loss(hd, wd):
        z = hd[keep] @ wd.T
        return ((torch.logsumexp(z, 1) - z.gather(1, y[keep].long()[:, None])[:, 0]) * g[keep].double()).sum()

    hd, wd = h.double(), w.double()
    t = 2.0 ** -10
    cut = 4 * t * t / 6 * g.double().abs().sum()
    p = torch.softmax(hd @ wd.T, 1)
    p[torch.arange(R, device="cuda")[keep], y[keep].long()] -= 1
    p = (p * (g.double() * keep)[:, None]).abs()
    b = 2.0 ** -7                                   # P's rounding and the result's, with the fp32 sums' below both
    th, tw = b * (p @ wd.abs()), b * (p.T @ hd.abs())
    gen = torch.Generator().manual_seed(3)
    for _ in range(24):
        i, j, v = (int(torch.randint(0, k, (1,), generator=gen)) for k in (R, d, V))
        step = torch.zeros_like(hd)
        step[i, j] = t
        num = (loss(hd + step, wd) - loss(hd - step, wd)) / (2 * t)
        assert (o["d_hidden"][i, j].double() - num).abs() <= th[i, j] + cut * wd.abs().max() ** 3
        step = torch.zeros_like(wd)
        step[v, j] = t
        num = (loss(hd, wd + step) - loss(hd, wd - step)) / (2 * t)
        assert (o["d_weight"][v, j].double() - num).abs() <= tw[v, j] + cut * hd.abs().max() ** 3


def test_ignored_rows_reach_nothing(cmsd):
    """NaN and infinities in ignored rows' hidden states, lse and gradients; labels out of range."""
    R, d, V = 70, 128, 500
    h, w, y, g = _inputs(R, d, V, ignored=0.3)
    clean = cmsd.lmhead_loss(h, w, y)
    cb = cmsd.lmhead_loss_backward(h, w, y, clean["lse"], g)
    gone = y < 0
    h2, lse2, g2 = h.clone(), clean["lse"].clone(), g.clone()
    h2[gone] = float("nan")
    h2[gone, ::3] = float("inf")
    lse2[gone] = float("-inf")
    g2[gone] = float("nan")
    y2 = y.clone()
    at = torch.nonzero(gone)[:, 0]
    y2[at[0]], y2[at[1]], y2[at[2]] = V, -1, 2 ** 31 - 1
    ws = cmsd.lmhead_loss_workspace(R, d, V)
    wb = cmsd.lmhead_loss_backward_workspace(R, d, V)
    ws[4:] = 255                                     # whatever the workspace holds
    wb[4:] = 255
    o = cmsd.lmhead_loss(h2, w, y2, ws=ws)
    ob = cmsd.lmhead_loss_backward(h2, w, y2, lse2, g2, ws=wb)
    for k in clean:
        assert torch.equal(o[k], clean[k]), k
    for k in cb:
        assert torch.equal(ob[k], cb[k]), k
    assert (ob["d_hidden"][gone] == 0).all()
    assert cmsd.workspace_errors(ws) == 1 and cmsd.workspace_errors(wb) == 1
    assert cmsd.workspace_errors(ws) == 0            # read once


@pytest.mark.parametrize("R", [1, 5, 257])
def test_every_row_ignored(cmsd, R):
    d, V = 64, 300
    h, w, y, g = _inputs(R, d, V)
    y[:] = IGNORE
    ws = cmsd.lmhead_loss_workspace(R, d, V)
    o = cmsd.lmhead_loss(h, w, y, ws=ws)
    ob = cmsd.lmhead_loss_backward(h, w, y, o["lse"], g)
    assert (o["loss"] == 0).all() and (o["lse"] == 0).all()
    assert (ob["d_hidden"] == 0).all() and (ob["d_weight"] == 0).all()
    assert cmsd.workspace_errors(ws) == 0


def test_no_rows(cmsd):
    h, w, y, g = _inputs(1, 64, 300)
    ob = cmsd.lmhead_loss_backward(h[:0], w, y[:0], g[:0], g[:0], out={"d_weight": torch.full_like(w, 3.0)})
    assert ob["d_hidden"].shape == (0, 64) and (ob["d_weight"] == 0).all()
    assert cmsd.lmhead_loss(h[:0], w, y[:0])["loss"].shape == (0,)


def test_ignore_index_inside_the_vocabulary(cmsd):
    R, d, V = 50, 64, 200
    h, w, y, g = _inputs(R, d, V)
    y[::4] = 7
    ws = cmsd.lmhead_loss_workspace(R, d, V)
    o = cmsd.lmhead_loss(h, w, y, ignore_index=7, ws=ws)
    y2 = torch.where(y == 7, torch.full_like(y, IGNORE), y)
    want = cmsd.lmhead_loss(h, w, y2)
    for k in want:
        assert torch.equal(o[k], want[k])
    assert cmsd.workspace_errors(ws) == 0


def test_rows_do_not_depend_on_their_neighbours(cmsd):
    """A row's loss and hidden gradient, alone and among others, to the bit within a block of rows."""
    R, d, V = 200, 192, 900
    h, w, y, g = _inputs(R, d, V)
    o = cmsd.lmhead_loss(h, w, y)
    perm = torch.randperm(R, device="cuda")
    o2 = cmsd.lmhead_loss(h[perm], w, y[perm])
    assert torch.equal(o["lse"][perm], o2["lse"]) and torch.equal(o["loss"][perm], o2["loss"])
    b = cmsd.lmhead_loss_backward(h, w, y, o["lse"], g, weight_grad=False)["d_hidden"]
    b2 = cmsd.lmhead_loss_backward(h[perm], w, y[perm], o2["lse"], g[perm].contiguous(), weight_grad=False)["d_hidden"]
    assert torch.equal(b[perm], b2)


def test_extreme_logits(cmsd):
    """Logits of +-1000 and equal ones: no overflow, a loss of 0 or of thousands, P of 0 and 1."""
    d, V, R = 64, 600, 6
    w = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    w[:, 0] = 1.0
    w[5, 0] = -1.0
    w[9, 1] = 1.0
    h = torch.zeros(R, d, dtype=torch.bfloat16, device="cuda")
    h[0, 0], h[1, 0], h[2, 1], h[3, 1], h[4, 1] = 1000.0, -1000.0, 1000.0, 1000.0, -30000.0
    y = torch.tensor([5, 5, 9, 3, 9, 0], dtype=torch.int32, device="cuda")
    g = torch.ones(R, device="cuda")
    o = cmsd.lmhead_loss(h, w, y)
    _check_loss(o, h, w, y, V)
    _check_grads(cmsd.lmhead_loss_backward(h, w, y, o["lse"], g), h, w, y, o["lse"], g, V)


def test_guard_bands(cmsd):
    """Nothing is written before or behind the outputs."""
    R, d, V = 41, 136, 333
    h, w, y, g = _inputs(R, d, V, ignored=0.2)
    n = cmsd.lib().cmsd_lmhead_loss_backward_workspace_bytes(R, d, V)
    nf = cmsd.lib().cmsd_lmhead_loss_workspace_bytes(R, d, V)

    def banded(count, dtype):
        t = torch.full((count + 256,), 77, dtype=dtype, device="cuda")
        return t, t[128:128 + count]

    lse_b, lse = banded(R, torch.float32)
    loss_b, loss = banded(R, torch.float32)
    dh_b, dh = banded(R * d, torch.bfloat16)
    dw_b, dw = banded(V * d, torch.bfloat16)
    wf_b, wf = banded(nf, torch.uint8)
    wb_b, wb = banded(n, torch.uint8)
    cmsd.lmhead_loss(h, w, y, out={"lse": lse, "loss": loss}, ws=wf)
    cmsd.lmhead_loss_backward(h, w, y, lse, g, out={"d_hidden": dh.view(R, d), "d_weight": dw.view(V, d)}, ws=wb)
    torch.cuda.synchronize()
    for t in (lse_b, loss_b, dh_b, dw_b, wf_b, wb_b):
        assert (t[:128] == 77).all() and (t[-128:] == 77).all()


def test_equal_calls_on_streams_and_in_a_graph(cmsd):
    """Twice the same, on another stream, and captured with new inputs in the same buffers."""
    R, d, V = 150, 256, 1500
    h, w, y, g = _inputs(R, d, V, ignored=0.2)
    h2, _, y2, g2 = _inputs(R, d, V, seed=1, ignored=0.5)
    wf, wb = cmsd.lmhead_loss_workspace(R, d, V), cmsd.lmhead_loss_backward_workspace(R, d, V)

    def step(h, y, g, out=None, wf=None, wb=None):
        o = dict(out or {})
        o.update(cmsd.lmhead_loss(h, w, y, out=o, ws=wf))
        o.update(cmsd.lmhead_loss_backward(h, w, y, o["lse"], g, out=o, ws=wb))
        return o

    a, b = step(h, y, g, wf=wf, wb=wb), step(h, y, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = step(h, y, g)
    torch.cuda.current_stream().wait_stream(side)
    for k in a:
        assert torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]), k
    want = step(h2, y2, g2)
    hb, yb, gb = h.clone(), y.clone(), g.clone()
    out = {k: torch.empty_like(v) for k, v in a.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(hb, yb, gb, out=out, wf=wf, wb=wb)
    for src, ref in (((h, y, g), a), ((h2, y2, g2), want), ((h, y, g), a)):
        for dst, s in zip((hb, yb, gb), src):
            dst.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        for k in a:
            assert torch.equal(out[k], ref[k]), k


@pytest.mark.parametrize("R", [40, 300])
def test_nan_is_not_lost(cmsd, R):
    """A kept row that holds a NaN has a NaN loss, alone; a NaN in one row of the weight reaches every loss."""
    d, V = 136, 3000
    h, w, y, _ = _inputs(R, d, V, ignored=0.2)
    keep = torch.nonzero(y >= 0)[:, 0]
    clean = cmsd.lmhead_loss(h, w, y)
    h2 = h.clone()
    h2[keep[3], 7] = float("nan")
    o = cmsd.lmhead_loss(h2, w, y)
    others = torch.ones(R, dtype=torch.bool, device="cuda")
    others[keep[3]] = False
    for k in clean:
        assert torch.isnan(o[k][keep[3]]) and torch.equal(o[k][others], clean[k][others])
    for v in (0, 1500, V - 1):
        w2 = w.clone()
        w2[v, 5] = float("nan")
        o = cmsd.lmhead_loss(h, w2, y)
        assert torch.isnan(o["loss"][keep]).all() and torch.isnan(o["lse"][keep]).all()
        assert (o["loss"][y < 0] == 0).all()


def test_calls_at_once_on_two_streams(cmsd):
    """Each with its own workspace; both kinds of kernels, many times over."""
    sizes = [(70, 256, 3000), (700, 136, 2500)]
    data = [_inputs(R, d, V, ignored=0.3) for R, d, V in sizes]
    streams = [torch.cuda.Stream() for _ in sizes]

    def step(i, wf, wb):
        h, w, y, g = data[i]
        o = cmsd.lmhead_loss(h, w, y, ws=wf)
        o.update(cmsd.lmhead_loss_backward(h, w, y, o["lse"], g, ws=wb))
        return o

    spaces = [(cmsd.lmhead_loss_workspace(*z), cmsd.lmhead_loss_backward_workspace(*z)) for z in sizes]
    want = [step(i, *spaces[i]) for i in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(step(i, *spaces[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for o in got[i]:
            assert all(torch.equal(o[k], want[i][k]) for k in want[i])
        assert cmsd.workspace_errors(spaces[i][0]) == 0 and cmsd.workspace_errors(spaces[i][1]) == 0


@pytest.mark.parametrize("R", [6, 200])
def test_without_the_loss(cmsd, R):
    """lse alone, as a gradient needs it."""
    h, w, y, _ = _inputs(R, 64, 500, ignored=0.3)
    want = cmsd.lmhead_loss(h, w, y)["lse"]
    ws = cmsd.lmhead_loss_workspace(R, 64, 500)
    lse = torch.full((R,), 9.0, device="cuda")
    rc = cmsd.lib().cmsd_lmhead_loss(h.data_ptr(), w.data_ptr(), y.data_ptr(), R, 64, 500, IGNORE, None, lse.data_ptr(),
                                     ws.data_ptr(), ws.numel(), cmsd._stream())
    assert rc == cmsd.OK and torch.equal(lse, want)


def test_binding_refuses_on_the_device(cmsd):
    h, w, y, g = _inputs(8, 64, 300)
    lse = cmsd.lmhead_loss(h, w, y)["lse"]
    small = cmsd.lmhead_loss_workspace(8, 64, 300)[:64]
    wide = torch.zeros(8, 128, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: cmsd.lmhead_loss(wide[:, :64], w, y), lambda: cmsd.lmhead_loss(h, w, y.cpu()),
                 lambda: cmsd.lmhead_loss(h, w, y, ws=small), lambda: cmsd.lmhead_loss(h, w, y, ws=small.cpu()),
                 lambda: cmsd.lmhead_loss_backward(h, w, y, lse, g, out={"d_hidden": h}),
                 lambda: cmsd.lmhead_loss_backward(h, w, y, lse, g, out={"d_weight": w}),
                 lambda: cmsd.lmhead_loss(h.reshape(-1)[4:4 + 7 * 64].view(7, 64), w, y[:7])):
        with pytest.raises(cmsd.CmsdError):
            call()


def test_offsets_past_32_bits(cmsd):
    """A weight of 2.4 G entries (4.9 GB): rows from its far end."""
    R, d, V = 3, 8192, 300000
    g = torch.Generator(device="cuda").manual_seed(5)
    w = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    w[-1000:] = (torch.randn(1000, d, generator=g, device="cuda") * 0.03).bfloat16()
    h = torch.randn(R, d, generator=g, device="cuda").bfloat16()
    y = torch.tensor([V - 1, V - 700, 0], dtype=torch.int32, device="cuda")
    o = cmsd.lmhead_loss(h, w, y)
    _check_loss(o, h, w, y, V)
    gr = torch.ones(R, device="cuda")
    ob = cmsd.lmhead_loss_backward(h, w, y, o["lse"], gr)
    z = h.double() @ w[-1000:].double().T
    p = torch.exp(z - o["lse"].double()[:, None])
    p[0, 999] -= 1
    p[1, 300] -= 1
    b = 2.0 ** -8
    e = d * 2.0 ** -23 * (h.double().abs() @ w[-1000:].double().abs().T)
    tol = ((b * p.abs() * 1.01 + (e + 2.0 ** -20) * torch.exp(z - o["lse"].double()[:, None])).T @ h.double().abs()) * 1.01
    want = p.T @ h.double()
    assert (ob["d_weight"][-1000:].double() - want).abs().le(tol + b * want.abs()).all()
    wanth = p @ w[-1000:].double()
    told = (b * p.abs() * 1.01 + (e + V * 2.0 ** -23) * p.abs() + 2.0 ** -20) @ w[-1000:].double().abs()
    assert (ob["d_hidden"].double() - wanth).abs().le(told + b * wanth.abs()).all()
