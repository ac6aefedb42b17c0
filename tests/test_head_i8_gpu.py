"""cmsd_quantize_rows and cmsd_lmhead_i8 against their definitions, to the bit:
the integers are exactly defined, the sums are whole numbers, and the scales'
products are single roundings."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


def _quantized(x):
    """127 x / a rounded half to even, in 64 bits: 127 x is exact there, and a quotient that is no tie is
    further from one (2^-33 of it at least) than it rounds (2^-53)."""
    x = x.double().cpu().numpy()
    a = np.abs(x).max(1)
    q = np.rint(127.0 * x / np.where(a > 0, a, 1.0)[:, None])
    with np.errstate(under="ignore"):
        return q.astype(np.int8), a.astype(np.float32) / np.float32(127)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,d", [(1, 16), (3, 32), (7, 208), (33, 1024), (5, 2048), (2, 2064), (300, 4096), (3, 8176),
                                 (2, 65536), (70000, 16), (8192, 512), (8193, 528), (9001, 256), (32770, 1024)])
def test_quantize_rows(cmsd, R, d, dtype):
    g = torch.Generator(device="cuda").manual_seed(R + d)
    x = torch.randn(R, d, generator=g, device="cuda") * torch.exp(4 * torch.randn(R, 1, generator=g, device="cuda"))
    x = x.to(dtype)
    o = cmsd.quantize_rows(x)
    q, s = _quantized(x)
    assert np.array_equal(o["scale"].cpu().numpy(), s)
    assert np.array_equal(o["q"].cpu().numpy(), q)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_ties_and_their_neighbours(cmsd, dtype):
    """x = (k + 1/2) a / 127 and the numbers beside it, for many a: every tie goes to the even integer."""
    g = torch.Generator().manual_seed(4)
    a = (1.0 + torch.rand(256, 1, generator=g)).to(dtype).float()
    a[:64] = (127.0 * 2.0 ** torch.arange(-32, 32, dtype=torch.float32))[:, None]     # ties are exact here
    k = torch.arange(0, 127, dtype=torch.float32)[None] + 0.5
    t = (a.double() * k.double() / 127).to(dtype)
    up = torch.nextafter(t, torch.full_like(t, float("inf")))
    down = torch.nextafter(t, torch.zeros_like(t))
    x = torch.cat([a.to(dtype), t, -t, up, -up, down, -down, -a.to(dtype), a.to(dtype) / 2], 1)
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % 16)).contiguous()
    o = cmsd.quantize_rows(x.cuda())
    q, s = _quantized(x)
    assert np.array_equal(o["scale"].cpu().numpy(), s)
    assert np.array_equal(o["q"].cpu().numpy(), q)


def test_quantize_extreme_rows(cmsd):
    """Zeros, the largest and the smallest numbers, infinities and NaN."""
    x = torch.zeros(8, 32)
    x[1] = torch.linspace(-1, 1, 32) * 3.3e38
    x[2] = torch.linspace(-1, 1, 32) * 1e-38
    x[3] = torch.linspace(-1, 1, 32) * 1e-42
    x[3, 5] = 2.0 ** -149
    x[4, 3] = -2.0 ** -149
    x[5] = 1.0
    x[5, 7] = float("inf")
    x[6] = 1.0
    x[6, 30] = float("nan")
    x[6, 2] = float("-inf")
    x[7] = 1e30
    x[7, 1:] = 1e-30
    for dtype in (torch.float32, torch.bfloat16):
        xd = x.to(dtype)
        o = cmsd.quantize_rows(xd.cuda())
        q, s = o["q"].cpu().numpy(), o["scale"].cpu().numpy()
        fine = [0, 1, 2, 3, 4, 7]
        qr, sr = _quantized(xd[fine])
        assert np.array_equal(q[fine], qr) and np.array_equal(s[fine], sr)
        assert (q[5] == 0).all() and s[5] == np.inf
        assert (q[6] == 0).all() and np.isnan(s[6])


def _ints(R, d, seed, full=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if full:
        return torch.randint(-128, 128, (R, d), generator=g, device="cuda", dtype=torch.int8)
    return (torch.randn(R, d, generator=g, device="cuda") * 36).round().clamp(-127, 127).to(torch.int8)


def _logits(hq, hs, wq, ws, dtype):
    # fp64 products and sums of these integers are exact (below 2^53)
    s = hq.double() @ wq.double().T
    z = s.float() * hs[:, None] * ws[None]
    return z.to(dtype)


def _same(got, want):
    assert got.dtype == want.dtype
    i = torch.int32 if got.dtype == torch.float32 else torch.int16
    bad = (got.view(i) != want.view(i)) & ~((got == 0) & (want == 0))
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:4].tolist())


# rows about 16, 32, 64, 128, 192; vocabularies about 128 and 256; widths about 128 and about 1024, whose sums are
# kept apart
SIZES = [(1, 16, 2), (1, 128, 256), (2, 144, 257), (16, 1024, 1000), (17, 1040, 4099), (33, 2064, 513),
         (64, 2048, 2000), (65, 112, 255), (127, 1008, 300), (128, 3104, 129), (130, 4096, 1025), (300, 272, 70001), (192, 256, 1000), (193, 256, 999), (385, 144, 500),
         (513, 512, 640), (20, 4096, 900), (20, 4112, 901), (128, 1024, 33001), (97, 1360, 2500), (3, 65536, 600)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,d,V", SIZES)
def test_product(cmsd, R, d, V, dtype):
    hq, wq = _ints(R, d, 1, full=R % 2 == 1), _ints(V, d, 2, full=V % 2 == 1)
    hs = torch.rand(R, device="cuda") * 0.1
    wsc = torch.rand(V, device="cuda") * 0.01
    ws = cmsd.lmhead_i8_workspace(R, d, V)
    ws[4:] = 255
    _same(cmsd.lmhead_i8(hq, hs, wq, wsc, dtype=dtype, ws=ws)["logits"], _logits(hq, hs, wq, wsc, dtype))
    assert cmsd.workspace_errors(ws) == 0


@pytest.mark.parametrize("d", [1024, 2048, 2080, 16384, 65536])
def test_largest_sums(cmsd, d):
    """Every product 16384 or 16129, of one sign or of both: sums up to 2^30, odd ones among them."""
    R, V = 3, 300
    hq = torch.full((R, d), -128, dtype=torch.int8, device="cuda")
    hq[1] = 127
    hq[2, ::2] = 127
    wq = torch.full((V, d), -128, dtype=torch.int8, device="cuda")
    wq[1::3] = 127
    wq[2::3, 1::2] = 127
    wq[2::3, 0] = 1
    one = torch.ones(R, device="cuda")
    onev = torch.ones(V, device="cuda")
    _same(cmsd.lmhead_i8(hq, one, wq, onev, dtype=torch.float32)["logits"], _logits(hq, one, wq, onev, torch.float32))


@pytest.mark.parametrize("R,d,V", [(300, 2576, 1500), (40, 1536, 40000), (129, 8192, 700), (191, 1200, 900),
                                   (600, 1296, 3000), (90, 2064, 45000)])
def test_large_tokens_among_small_ones(cmsd, R, d, V):
    """Tokens whose magnitudes add up to more than 2^17, just to it, and to less, in one tile and in others."""
    hq, wq = _ints(R, d, 9), _ints(V, d, 10, full=True)
    hq.clamp_(-30, 30)
    hq[R // 2] = 127
    hq[R - 1] = 0
    hq[R - 1, :1024] = -128                          # 2^17 exactly
    hq[R // 3] = hq[R - 1]
    hq[R // 3, 1024] = 1
    hs, wsc = torch.rand(R, device="cuda"), torch.rand(V, device="cuda")
    wq[3], wq[V - 1] = -128, 127
    _same(cmsd.lmhead_i8(hq, hs, wq, wsc, dtype=torch.float32)["logits"], _logits(hq, hs, wq, wsc, torch.float32))


def test_scales_of_any_kind(cmsd):
    """Zeros, infinities and NaN in the scales show in their rows and columns alone."""
    R, d, V = 20, 64, 300
    hq, wq = _ints(R, d, 3), _ints(V, d, 4)
    hs, wsc = torch.rand(R, device="cuda"), torch.rand(V, device="cuda")
    hs[1], hs[2], wsc[5], wsc[6] = 0.0, float("inf"), float("nan"), 0.0
    got = cmsd.lmhead_i8(hq, hs, wq, wsc, dtype=torch.float32)["logits"]
    want = _logits(hq, hs, wq, wsc, torch.float32)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))


def test_guard_bands_streams_and_graph(cmsd):
    R, d, V = 37, 272, 1001
    hq, wq = _ints(R, d, 5), _ints(V, d, 6)
    hs, wsc = torch.rand(R, device="cuda"), torch.rand(V, device="cuda")
    want = _logits(hq, hs, wq, wsc, torch.float32)
    n = cmsd.lib().cmsd_lmhead_i8_workspace_bytes(R, d, V)
    wb = torch.full((n + 512,), 77, dtype=torch.uint8, device="cuda")
    ob = torch.full((R * V + 512,), 77.0, device="cuda")
    out, ws = ob[256:256 + R * V].view(R, V), wb[256:256 + n]
    cmsd.lmhead_i8(hq, hs, wq, wsc, out={"logits": out}, dtype=torch.float32, ws=ws)
    torch.cuda.synchronize()
    _same(out, want)
    for t in (wb, ob):
        assert (t[:256] == 77).all() and (t[-256:] == 77).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cmsd.lmhead_i8(hq, hs, wq, wsc, dtype=torch.float32)["logits"]
    torch.cuda.current_stream().wait_stream(side)
    _same(got, want)
    # a row buffer quantised and multiplied inside a graph
    x = torch.randn(R, d, device="cuda").bfloat16()
    q = {"q": torch.empty(R, d, dtype=torch.int8, device="cuda"), "scale": torch.empty(R, device="cuda")}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cmsd.quantize_rows(x, out=q)
        cmsd.lmhead_i8(q["q"], q["scale"], wq, wsc, out={"logits": out}, dtype=torch.float32, ws=ws)
    for seed in (1, 2):
        x.copy_(torch.randn(R, d, generator=torch.Generator().manual_seed(seed)).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        r = cmsd.quantize_rows(x)
        _same(out, _logits(r["q"], r["scale"], wq, wsc, torch.float32))


@pytest.mark.parametrize("R,d,V", [(40, 2576, 1500), (300, 2576, 1500)])
def test_a_graph_replayed_with_larger_and_smaller_tokens(cmsd, R, d, V):
    """What the tokens hold decides how sums are formed: not what they held at the capture."""
    wq = _ints(V, d, 12, full=True)
    small, large = _ints(R, d, 13).clamp_(-20, 20), _ints(R, d, 14, full=True)
    large[::2] = 127
    hq = small.clone()
    hs, wsc = torch.rand(R, device="cuda"), torch.rand(V, device="cuda")
    out = {"logits": torch.empty(R, V, device="cuda")}
    ws = cmsd.lmhead_i8_workspace(R, d, V)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cmsd.lmhead_i8(hq, hs, wq, wsc, dtype=torch.float32, out=out, ws=ws)
    for src in (small, large, small, large):
        hq.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        _same(out["logits"], _logits(src, hs, wq, wsc, torch.float32))
    assert cmsd.workspace_errors(ws) == 0


def test_calls_at_once_on_two_streams(cmsd):
    sizes = [(20, 512, 4000), (260, 272, 3000)]
    data = [(_ints(R, d, 1), torch.rand(R, device="cuda"), _ints(V, d, 2), torch.rand(V, device="cuda"))
            for R, d, V in sizes]
    spaces = [cmsd.lmhead_i8_workspace(*z) for z in sizes]
    want = [_logits(*x, torch.bfloat16) for x in data]
    streams = [torch.cuda.Stream() for _ in sizes]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got.append((i, cmsd.lmhead_i8(*data[i], ws=spaces[i])["logits"]))
    torch.cuda.synchronize()
    for i, z in got:
        _same(z, want[i])


def test_offsets_past_32_bits(cmsd):
    """2.6 G logits, and 2.2 G numbers quantised."""
    R, d, V = 20000, 16, 128256
    hq, wq = _ints(R, d, 7), _ints(V, d, 8)
    hs, wsc = torch.rand(R, device="cuda"), torch.rand(V, device="cuda")
    got = cmsd.lmhead_i8(hq, hs, wq, wsc)["logits"]
    rows = torch.tensor([0, 1, 9999, 16745, 16746, R - 1], device="cuda")
    _same(got[rows], _logits(hq[rows], hs[rows], wq, wsc, torch.bfloat16))
    del got
    x = torch.ones(135000, 16384, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.linspace(-3, 3, 16384).bfloat16()
    o = cmsd.quantize_rows(x)
    q, s = _quantized(x[-2:])
    assert np.array_equal(o["q"][-2:].cpu().numpy(), q) and np.array_equal(o["scale"][-2:].cpu().numpy(), s)


def test_train_quantise_and_decode(cmsd):
    """The operators as they are used: a head is trained for a few steps, then served in 8 bits, its logits
    read by the confidence pass."""
    R, d, V = 96, 256, 2000
    g = torch.Generator(device="cuda").manual_seed(11)
    w = (torch.randn(V, d, generator=g, device="cuda") * 0.05).bfloat16()
    h = torch.randn(R, d, generator=g, device="cuda").bfloat16()
    y = torch.randint(0, V, (R,), generator=g, device="cuda").int()
    y[::5] = -100
    keep = y >= 0
    grad = keep.float() / keep.sum()
    master = w.float()
    for _ in range(3):
        w = master.bfloat16()
        o = cmsd.lmhead_loss(h, w, y)
        dw = cmsd.lmhead_loss_backward(h, w, y, o["lse"], grad, hidden_grad=False)["d_weight"]
        master -= 4.0 * dw.float()
    # the last step's gradient, against the definition through another path: the head's own logits
    z = cmsd.lmhead_confidence(h, w, logits=True)["logits"].double()
    assert ((torch.logsumexp(z, 1) - o["lse"].double()).abs()[keep] < 1e-4).all()
    wq = cmsd.quantize_rows(master.bfloat16())
    hq = cmsd.quantize_rows(h)
    z8 = cmsd.lmhead_i8(hq["q"], hq["scale"], wq["q"], wq["scale"], dtype=torch.float32)["logits"]
    _same(z8, _logits(hq["q"], hq["scale"], wq["q"], wq["scale"], torch.float32))
    # each factor is off by at most half a step of its row
    hd, wd = h.double(), master.bfloat16().double()
    eh, ew = hq["scale"].double()[:, None] / 2, wq["scale"].double()[:, None] / 2
    bound = hd.abs() @ ew.expand_as(wd).T + eh.expand_as(hd) @ wd.abs().T + d * eh * ew.T
    assert ((z8.double() - hd @ wd.T).abs() <= bound * 1.001 + 1e-5).all()
    c = cmsd.confidence(z8.view(8, 12, V))
    assert torch.equal(c["argmax"].view(R).long(), z8.argmax(1))
    lse = torch.logsumexp(z8.double(), 1)
    assert ((c["lse"].view(R).double() - lse).abs() < 1e-5).all()
