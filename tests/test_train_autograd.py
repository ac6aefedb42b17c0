"""What autograd would follow and the embedding's, layer norm's and dropout's calls could not is refused, in both
directions; else the next check (CUDA tensors) is reached."""
import os

import pytest

torch = pytest.importorskip("torch")
fwAD = torch.autograd.forward_ad

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


TOKENS, F = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
WS = torch.zeros(64, dtype=torch.uint8)
TABLE, X, P = torch.zeros(100, 24), torch.zeros(4, 24), torch.zeros(24)

# the calls of one tensor that a derivative may be wanted by, the others being constants
BACKWARD = {
    "embedding_backward(d_x)": (X, lambda c, t: c.embedding_backward(TOKENS, t, 100, ws=WS)),
    "embedding_backward(d_table)": (TABLE, lambda c, t: c.embedding_backward(TOKENS, X, 100, add=True, out={"d_table": t}, ws=WS)),
    "layernorm_backward(x)": (X, lambda c, t: c.layernorm_backward(t, P, F, F, X, ws=WS)),
    "layernorm_backward(weight)": (P, lambda c, t: c.layernorm_backward(X, t, F, F, X, ws=WS)),
    "layernorm_backward(mean)": (F, lambda c, t: c.layernorm_backward(X, P, t, F, X, ws=WS)),
    "layernorm_backward(rstd)": (F, lambda c, t: c.layernorm_backward(X, P, F, t, X, ws=WS)),
    "layernorm_backward(d_y)": (X, lambda c, t: c.layernorm_backward(X, None, F, F, t, ws=WS)),
    "dropout_backward(d_y)": (X, lambda c, t: c.dropout_backward(t, 0.1, 1)),
}


@pytest.mark.parametrize("name", BACKWARD)
def test_second_derivatives(cmsd, name):
    t, call = BACKWARD[name]
    t = t.clone().requires_grad_()
    with pytest.raises(cmsd.CmsdError, match="autograd"):
        call(cmsd, t)
    with torch.no_grad(), pytest.raises(cmsd.CmsdError, match="CUDA"):
        call(cmsd, t)
    with pytest.raises(cmsd.CmsdError, match="CUDA"):
        call(cmsd, t.detach())


@pytest.mark.gpu
def test_from_a_function(cmsd):
    """In an autograd.Function the first derivatives pass, and a graph of them is refused."""
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            o = cmsd.layernorm(x, weight)
            ctx.save_for_backward(x, weight, o["mean"], o["rstd"])
            return o["y"]

        @staticmethod
        def backward(ctx, d_y):
            x, weight, mean, rstd = ctx.saved_tensors
            g = cmsd.layernorm_backward(x, weight, mean, rstd, d_y.contiguous(), bias_grad=False)
            return g["d_x"], g["d_weight"]

    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x, w, c = (torch.randn(*s, generator=g, device="cuda") for s in ((7, 24), (24,), (7, 24)))
    x.requires_grad_()
    w.requires_grad_()
    (Norm.apply(x, w) * c).sum().backward()
    with torch.no_grad():
        o = cmsd.layernorm(x, w)
        want = cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], c)
    assert torch.equal(x.grad, want["d_x"]) and torch.equal(w.grad, want["d_weight"])
    with pytest.raises(cmsd.CmsdError, match="autograd"):
        torch.autograd.grad((Norm.apply(x, w) * c).sum(), x, create_graph=True)


# the tensors that a forward derivative may come with
FORWARD = {
    "embedding(table)": (TABLE, lambda c, t: c.embedding(TOKENS, t)),
    "layernorm(x)": (X, lambda c, t: c.layernorm(t, P, P)),
    "layernorm(weight)": (P, lambda c, t: c.layernorm(X, t, P)),
    "layernorm(bias)": (P, lambda c, t: c.layernorm(X, P, t)),
    "dropout(x)": (X, lambda c, t: c.dropout(t, 0.1, 1)),
    "dropout(residual)": (X, lambda c, t: c.dropout(X, 0.1, 1, residual=t)),
}


@pytest.mark.parametrize("name", [*FORWARD, *BACKWARD])
def test_tangents(cmsd, name):
    t, call = {**FORWARD, **BACKWARD}[name]
    with fwAD.dual_level():
        dual = fwAD.make_dual(t, torch.ones_like(t))
        with pytest.raises(cmsd.CmsdError, match="autograd"):
            call(cmsd, dual)
        with torch.no_grad(), pytest.raises(cmsd.CmsdError, match="autograd"):      # (stops no tangent)
            call(cmsd, dual)
        with pytest.raises(cmsd.CmsdError, match="CUDA"):
            call(cmsd, t)
        with pytest.raises(cmsd.CmsdError, match="CUDA"):
            call(cmsd, fwAD.unpack_dual(dual).primal)


def test_tangents_of_a_function_are_its_own(cmsd):
    """In an autograd.Function's forward nothing follows the tangents: its jvp makes them."""
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            with pytest.raises(cmsd.CmsdError, match="CUDA"):
                cmsd.layernorm(x, P, P)
            return x * 2

        @staticmethod
        def jvp(ctx, t):
            return t * 2

    with fwAD.dual_level():
        y = Norm.apply(fwAD.make_dual(X.clone(), torch.ones_like(X)))
        assert (fwAD.unpack_dual(y).tangent == 2).all()
