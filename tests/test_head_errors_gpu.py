"""What the head operators' kernels find wrong is read after a call whose
workspace nobody kept."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


def _inputs(R, d=64, V=500):
    g = torch.Generator(device="cuda").manual_seed(R)
    h = torch.randn(R, d, generator=g, device="cuda").bfloat16()
    w = torch.randn(V, d, generator=g, device="cuda").bfloat16()
    y = torch.randint(0, V, (R,), generator=g, device="cuda").int()
    y[::3] = -100
    return h, w, y


@pytest.mark.parametrize("R", [6, 200])
@pytest.mark.parametrize("bad", [-1, 500, 2 ** 31 - 1])
def test_a_bad_label_shows_without_a_workspace(cmsd, R, bad):
    h, w, y = _inputs(R)
    cmsd.lmhead_errors()
    lse = cmsd.lmhead_loss(h, w, y)["lse"]
    cmsd.lmhead_loss_backward(h, w, y, lse, lse)
    assert cmsd.lmhead_errors() == 0
    y[R - 1] = bad
    o = cmsd.lmhead_loss(h, w, y)
    assert cmsd.lmhead_errors() == 1 and o["loss"][R - 1] == 0
    assert cmsd.lmhead_errors() == 0                 # read once
    cmsd.lmhead_loss_backward(h, w, y, lse, lse)
    assert cmsd.lmhead_errors() == 1


def test_a_bad_label_shows_in_both_words(cmsd):
    h, w, y = _inputs(40)
    y[1] = 500
    ws = cmsd.lmhead_loss_workspace(40, 64, 500)
    cmsd.lmhead_errors()
    cmsd.lmhead_loss(h, w, y, ws=ws)
    assert cmsd.lmhead_errors() == 1 and cmsd.workspace_errors(ws) == 1


def test_a_bad_label_shows_on_replay(cmsd):
    """A captured call whose workspace lives in the graph alone; the word is read outside it, on another stream."""
    h, w, y = _inputs(40)
    good, bad = y.clone(), y.clone()
    bad[1] = 500
    cmsd.lmhead_loss(h, w, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cmsd.lmhead_loss(h, w, y)
    cmsd.lmhead_errors()
    for src, want in ((good, 0), (bad, 1), (good, 0)):
        y.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            assert cmsd.lmhead_errors() == want


def test_the_8_bit_product_reports_nothing(cmsd):
    q = torch.ones(3, 32, dtype=torch.int8, device="cuda")
    s = torch.ones(3, device="cuda")
    cmsd.lmhead_errors()
    cmsd.lmhead_i8(q, s, q, s)
    assert cmsd.lmhead_errors() == 0


def test_a_wait_that_gives_up_is_reported(cmsd):
    """A barrier that nobody arrives at: the kernel ends by itself, both words have bit 2, the next call is right."""
    h, w, y = _inputs(40)
    want = cmsd.lmhead_loss(h, w, y)
    ws = cmsd.lmhead_loss_workspace(40, 64, 500)
    cmsd.lmhead_errors()
    for arrive, bits in ((1, 0), (0, 4)):
        assert cmsd.lib().cmsd_test_head_wait(arrive, ws.data_ptr(), ws.numel(), cmsd._stream()) == cmsd.OK
        assert cmsd.workspace_errors(ws) == bits and cmsd.lmhead_errors() == bits
    got = cmsd.lmhead_loss(h, w, y, ws=ws)
    assert torch.equal(got["loss"], want["loss"]) and cmsd.workspace_errors(ws) == 0
