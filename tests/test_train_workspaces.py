"""A workspace that is large enough for some rows is so for fewer of them, as a program's last batch has: the sizes of
the embedding's and layer norm's workspaces do not fall as rows are added."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2508_15371_gb300")
# every number of rows up to 40000, and about powers of two above
ROWS = list(range(1, 40001)) + sorted(r for k in range(16, 28) for r in ((1 << k) - 1, 1 << k, (1 << k) + 1, (1 << k) * 5 // 4))


@pytest.fixture(scope="module")
def cmsd():
    if not os.path.exists(os.path.join(PKG, "libcmsd.so")):
        from paper_2508_15371_gb300 import build
        build.build()
    from paper_2508_15371_gb300 import cmsd as c
    c.lib()
    return c


@pytest.mark.parametrize("d", [1, 64, 300, 1000, 2048, 65536])
@pytest.mark.parametrize("V", [1, 1000, 1024, 128256, 1 << 30])
def test_embedding(cmsd, d, V):
    if V * d >= 1 << 46:
        pytest.skip("beyond the table's sizes")
    size = cmsd.lib().cmsd_embedding_backward_workspace_bytes
    last = 0
    for R in ROWS:
        n = size(R, d, V)
        assert n >= last, R
        last = n


@pytest.mark.parametrize("d", [1, 256, 257, 1001, 2048, 8192, 8193, 65536])
def test_norm(cmsd, d):
    size = cmsd.lib().cmsd_layernorm_backward_workspace_bytes
    last = 0
    for R in ROWS:
        n = size(R, d)
        assert n >= last, R
        last = n


@pytest.mark.gpu
@pytest.mark.parametrize("d", [72, 513])
def test_one_workspace_for_all_batches(cmsd, d):
    """The largest batch's workspace, used for shorter ones: nothing behind a shorter one's size is written."""
    torch = pytest.importorskip("torch")
    V, most = 3000, 20000
    ws, norm_ws = cmsd.embedding_backward_workspace(most, d, V), cmsd.layernorm_backward_workspace(most, d)
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    for R in (20000, 19457, 16385, 16384, 9729, 7169, 7168, 4865, 4864, 700, 513, 512, 7):
        t = torch.randint(0, V, (R,), generator=g, device="cuda").int()
        x, d_y = (torch.randn(R, d, generator=g, device="cuda") for _ in range(2))
        own = cmsd.embedding_backward_workspace(R, d, V)
        assert own.numel() <= ws.numel()
        ws[own.numel():] = 77
        got = cmsd.embedding_backward(t, d_y, V, ws=ws)["d_table"]
        assert torch.equal(got, cmsd.embedding_backward(t, d_y, V, ws=own)["d_table"]), R
        assert (ws[own.numel():] == 77).all(), R
        o = cmsd.layernorm(x)
        own = cmsd.layernorm_backward_workspace(R, d)
        got = cmsd.layernorm_backward(x, None, o["mean"], o["rstd"], d_y, ws=norm_ws)
        want = cmsd.layernorm_backward(x, None, o["mean"], o["rstd"], d_y, ws=own)
        assert all(torch.equal(got[k], want[k]) for k in want), R
    assert cmsd.workspace_errors(ws) == 0
