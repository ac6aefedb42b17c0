"""The head operators with more rows than one round of a kernel's CTAs takes, and
rows wider than what is requested ahead: the packing of over 8192 rows (16 and
more of them a CTA) and of rows over 2048 wide, the gradient's rounding over
65535 rows, and the 8-bit product's tokens over 65536."""
import pytest

torch = pytest.importorskip("torch")

from test_head_loss_gpu import _check_grads, _check_loss, _inputs  # noqa: E402  (its bounds stand there)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


@pytest.mark.parametrize("R,d,V", [(8200, 64, 300), (20001, 72, 257), (70000, 40, 2000), (300, 2056, 700),
                                   (300, 4104, 500), (8193, 2056, 130)])
@pytest.mark.parametrize("ignored", [0.3, 0.98])
def test_rows_find_their_places(cmsd, R, d, V, ignored):
    h, w, y, g = _inputs(R, d, V, ignored=ignored)
    y[R // 2:R // 2 + 40] = -100                     # (whole groups of a CTA ignored)
    y[-9:] = -100
    h[y < 0] = float("nan")
    ws, wb = cmsd.lmhead_loss_workspace(R, d, V), cmsd.lmhead_loss_backward_workspace(R, d, V)
    ws[4:], wb[4:] = 255, 255
    o = cmsd.lmhead_loss(h, w, y, ws=ws)
    _check_loss(o, h, w, y, V)
    _check_grads(cmsd.lmhead_loss_backward(h, w, y, o["lse"], g, ws=wb), h, w, y, o["lse"], g, V)
    assert cmsd.workspace_errors(ws) == 0 and cmsd.workspace_errors(wb) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_past_one_round(cmsd, dtype):
    """Tokens on both sides of row 65536 whose magnitudes add up to more than 2^17, among smaller ones."""
    R, d, V = 70000, 1040, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    hq = (torch.randn(R, d, generator=g, device="cuda") * 36).round().clamp(-127, 127).to(torch.int8)
    wq = torch.randint(-128, 128, (V, d), generator=g, device="cuda", dtype=torch.int8)
    wq[3], wq[V - 1] = -128, 127
    for r in (0, 191, 65535, 65536, 65727, 65729, 69999):
        hq[r] = 127 if r % 2 else -128
        hq[r, ::7] += 1 if r % 2 == 0 else -1
    hs, wsc = torch.rand(R, generator=g, device="cuda"), torch.rand(V, generator=g, device="cuda")
    got = cmsd.lmhead_i8(hq, hs, wq, wsc, dtype=dtype)["logits"]
    want = ((hq.double() @ wq.double().T).float() * hs[:, None] * wsc).to(dtype)     # (the sums are exact)
    assert got.dtype == want.dtype and torch.equal(got, want)
