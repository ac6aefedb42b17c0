"""The type of layer norm's parameters' gradients, where it is asked for: what is refused."""
import os

import pytest

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2508_15371_gb300")


@pytest.fixture(scope="module")
def cmsd():
    if not os.path.exists(os.path.join(PKG, "libcmsd.so")):
        from paper_2508_15371_gb300 import build
        build.build()
    from paper_2508_15371_gb300 import cmsd as c
    c.lib()
    return c


def test_types(cmsd):
    x, p, f, ws = torch.zeros(4, 24), torch.zeros(24), torch.zeros(4), torch.zeros(64, dtype=torch.uint8)
    call = lambda w, **kw: cmsd.layernorm_backward(x, w, f, f, x, ws=ws, **kw)  # noqa: E731
    for w, dtype in ((None, torch.float16), (None, torch.float64), (p, torch.float16), (p, torch.bfloat16),
                     (p.bfloat16(), torch.float32)):
        with pytest.raises(cmsd.CmsdError, match="dtype"):
            call(w, dtype=dtype)
    for w, dtype in ((None, torch.bfloat16), (None, torch.float32), (None, None), (p, torch.float32), (p, None)):
        with pytest.raises(cmsd.CmsdError, match="CUDA"):
            call(w, dtype=dtype)
