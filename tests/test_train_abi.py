"""The embedding's, layer norm's and dropout's calls without a GPU: argument
errors are found on the host before anything is enqueued, and workspace sizes
depend on the sizes of the call alone."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2508_15371_gb300")
A = 4096            # addresses that nothing reads: every call here is refused
I1, I2, I3, I4, I5, O1, O2, O3, WS = (A + (k << 46) for k in range(9))      # far enough apart


@pytest.fixture(scope="module")
def cmsd():
    if not os.path.exists(os.path.join(PKG, "libcmsd.so")):
        from paper_2508_15371_gb300 import build
        build.build()
    from paper_2508_15371_gb300 import cmsd as c
    c.lib()
    return c


def _embed(c, tokens=I1, table=I2, dtype=1, R=4, d=24, V=100, scale=1.0, x=O1):
    return c.lib().cmsd_embedding(tokens, table, dtype, R, d, V, -100, scale, x, None)


def _embed_back(c, tokens=I1, d_x=I2, dtype=1, R=4, d=24, V=100, scale=1.0, add=0, d_table=O1, ws=WS, ws_bytes=None):
    n = c.lib().cmsd_embedding_backward_workspace_bytes(R, d, V) if ws_bytes is None else ws_bytes
    return c.lib().cmsd_embedding_backward(tokens, d_x, dtype, R, d, V, -100, scale, add, d_table, ws, n, None)


def _norm(c, x=I1, w=I2, b=I3, dtype=1, wdtype=0, R=4, d=24, eps=1e-5, y=O1, mean=O2, rstd=O3):
    return c.lib().cmsd_layernorm(x, w, b, dtype, wdtype, R, d, eps, y, mean, rstd, None)


def _norm_back(c, x=I1, w=I2, mean=I3, rstd=I4, dy=I5, dtype=1, wdtype=0, R=4, d=24, dx=O1, dw=O2, db=O3, ws=WS,
               ws_bytes=None):
    n = c.lib().cmsd_layernorm_backward_workspace_bytes(R, d) if ws_bytes is None else ws_bytes
    return c.lib().cmsd_layernorm_backward(x, w, mean, rstd, dy, dtype, wdtype, R, d, dx, dw, db, ws, n, None)


def _drop(c, x=I1, r=I2, dtype=1, n=100, p=0.1, step=None, y=O1):
    return c.lib().cmsd_dropout(x, r, dtype, n, p, 1, 2, 3, step, y, None)


def _drop_back(c, dy=I1, dtype=1, n=100, p=0.1, step=None, dx=O1):
    return c.lib().cmsd_dropout_backward(dy, dtype, n, p, 1, 2, 3, step, dx, None)


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kw", [dict(R=-1), dict(d=0), dict(d=-8), dict(d=65537), dict(V=0), dict(V=-1),
                                dict(R=(1 << 28) + 1), dict(V=(1 << 30) + 1),
                                dict(V=1 << 30, d=65536)])
def test_embedding_sizes_refused(cmsd, kw):
    assert _embed(cmsd, **kw) == cmsd.EINVAL
    assert _embed_back(cmsd, ws_bytes=1 << 40, **kw) == cmsd.EINVAL
    a = {**dict(R=4, d=24, V=100), **kw}
    assert cmsd.lib().cmsd_embedding_backward_workspace_bytes(a["R"], a["d"], a["V"]) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), "EDTYPE"), (dict(scale=INF), "EINVAL"), (dict(scale=NAN), "EINVAL"), (dict(tokens=None), "EINVAL"),
    (dict(table=None), "EINVAL"), (dict(x=None), "EINVAL"), (dict(tokens=A + 2), "EALIGN"), (dict(table=A + 8), "EALIGN"),
    (dict(x=A + 4), "EALIGN"), (dict(x=I1), "EINVAL"), (dict(x=I2 + 100 * 48 - 16), "EINVAL"),
    (dict(x=I2 - 4 * 48 + 16), "EINVAL"), (dict(R=0, tokens=None, table=None, x=None), "OK")])
def test_embedding_refused(cmsd, kw, code):
    assert _embed(cmsd, **kw) == getattr(cmsd, code)


@pytest.mark.parametrize("add", [0, 1])
@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), "EDTYPE"), (dict(scale=INF), "EINVAL"), (dict(tokens=None), "EINVAL"), (dict(d_x=None), "EINVAL"),
    (dict(d_table=None), "EINVAL"), (dict(tokens=A + 1), "EALIGN"), (dict(d_x=A + 8), "EALIGN"),
    (dict(d_table=A + 8), "EALIGN"), (dict(ws=None), "ENOWS"), (dict(ws_bytes=255), "ENOWS"), (dict(ws=A + 8), "EALIGN"),
    (dict(d_table=I2), "EINVAL"), (dict(d_table=I1), "EINVAL"), (dict(ws=O1 + 16), "EINVAL"), (dict(ws=I2 + 16), "EINVAL"),
    (dict(d_table=WS), "EINVAL"), (dict(R=0, d_table=None), "EINVAL"), (dict(R=0, d_table=A + 8), "EALIGN")])
def test_embedding_backward_refused(cmsd, kw, code, add):
    assert _embed_back(cmsd, add=add, **kw) == getattr(cmsd, code)


def test_nothing_to_add(cmsd):
    assert _embed_back(cmsd, R=0, add=1, tokens=None, d_x=None, ws=None) == cmsd.OK


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), "EDTYPE"), (dict(wdtype=2), "EDTYPE"), (dict(R=-1), "EINVAL"), (dict(d=0), "EINVAL"),
    (dict(d=65537), "EINVAL"), (dict(R=(1 << 28) + 1), "EINVAL"),
    (dict(eps=0.0), "EINVAL"), (dict(eps=-1.0), "EINVAL"), (dict(eps=INF), "EINVAL"), (dict(eps=NAN), "EINVAL"),
    (dict(x=None), "EINVAL"), (dict(y=None), "EINVAL"), (dict(x=A + 8), "EALIGN"), (dict(w=A + 8), "EALIGN"),
    (dict(b=A + 4), "EALIGN"), (dict(y=A + 8), "EALIGN"), (dict(mean=A + 2), "EALIGN"), (dict(rstd=A + 1), "EALIGN"),
    (dict(y=I1), "EINVAL"), (dict(y=I2 + 80), "EINVAL"), (dict(mean=I3), "EINVAL"), (dict(rstd=O2 + 12), "EINVAL"),
    (dict(mean=O1 + 4 * 48 - 4), "EINVAL"), (dict(R=0, x=None, y=None, mean=None, rstd=None), "OK")])
def test_norm_refused(cmsd, kw, code):
    assert _norm(cmsd, **kw) == getattr(cmsd, code)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), "EDTYPE"), (dict(wdtype=-1), "EDTYPE"), (dict(R=-1), "EINVAL"), (dict(d=0), "EINVAL"),
    (dict(d=65537), "EINVAL"), (dict(x=None), "EINVAL"), (dict(mean=None), "EINVAL"), (dict(rstd=None), "EINVAL"),
    (dict(dy=None), "EINVAL"), (dict(dx=None, dw=None, db=None), "EINVAL"), (dict(x=A + 8), "EALIGN"),
    (dict(w=A + 8), "EALIGN"), (dict(dy=A + 8), "EALIGN"), (dict(dx=A + 8), "EALIGN"), (dict(dw=A + 8), "EALIGN"),
    (dict(db=A + 8), "EALIGN"), (dict(mean=A + 2), "EALIGN"), (dict(rstd=A + 2), "EALIGN"), (dict(ws=None), "ENOWS"),
    (dict(ws_bytes=16), "ENOWS"), (dict(ws=A + 8), "EALIGN"), (dict(dx=I1), "EINVAL"), (dict(dx=I5), "EINVAL"),
    (dict(dw=I2), "EINVAL"), (dict(db=O2), "EINVAL"), (dict(db=O2 + 80), "EINVAL"), (dict(dw=I3), "EINVAL"),
    (dict(ws=O1), "EINVAL"), (dict(dx=WS), "EINVAL"), (dict(ws=I4 - 16), "EINVAL"),
    (dict(R=0, dx=None, dw=None, db=None), "EINVAL"), (dict(R=0, dw=A + 8), "EALIGN"), (dict(R=0, dw=O3), "EINVAL"),
    (dict(R=0, x=None, mean=None, rstd=None, dy=None, dw=None, db=None, ws=None), "OK")])
def test_norm_backward_refused(cmsd, kw, code):
    assert _norm_back(cmsd, **kw) == getattr(cmsd, code)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), "EDTYPE"), (dict(n=-1), "EINVAL"), (dict(n=1 << 42), "EINVAL"), (dict(p=-0.1), "EINVAL"),
    (dict(p=1.0001), "EINVAL"), (dict(p=NAN), "EINVAL"), (dict(x=None), "EINVAL"), (dict(y=None), "EINVAL"),
    (dict(x=A + 8), "EALIGN"), (dict(y=A + 2), "EALIGN"), (dict(r=A + 4), "EALIGN"), (dict(step=A + 2), "EALIGN"),
    (dict(y=I1), "EINVAL"), (dict(y=I2 + 192), "EINVAL"), (dict(step=O1 + 4), "EINVAL"),
    (dict(n=0, x=None, r=None, y=None), "OK")])
def test_dropout_refused(cmsd, kw, code):
    assert _drop(cmsd, **kw) == getattr(cmsd, code)
    if "r" not in kw and kw.get("y") != I2 + 192:
        back = {{"x": "dy", "y": "dx"}.get(k, k): v for k, v in kw.items()}
        assert _drop_back(cmsd, **back) == getattr(cmsd, code)


def test_errors_need_a_place(cmsd):
    assert cmsd.lib().cmsd_embedding_errors(None, None) == cmsd.EINVAL


def test_workspaces_are_small(cmsd):
    """They grow with the rows times the width, or with the width; not with the vocabulary times the width."""
    for R, d, V in ((1, 1, 1), (4096, 2048, 128256), (1 << 20, 2048, 1 << 20)):
        n = cmsd.lib().cmsd_embedding_backward_workspace_bytes(R, d, V)
        assert 0 < n <= (1 << 20) + 64 * R + 16 * V + 8 * R * d
        n = cmsd.lib().cmsd_layernorm_backward_workspace_bytes(R, d)
        assert 0 < n <= 4096 + 1024 * 8 * d


# ---- the binding ------------------------------------------------------------------

def test_binding_refuses_before_the_library(cmsd):
    torch = pytest.importorskip("torch")
    t, w = torch.zeros(4, dtype=torch.int32), torch.zeros(100, 24)
    x, f, p = torch.zeros(4, 24), torch.zeros(4), torch.zeros(24)
    ws = torch.zeros(64, dtype=torch.uint8)
    bad = [lambda: cmsd.embedding(t.long(), w), lambda: cmsd.embedding(t, w.half()), lambda: cmsd.embedding(t, w[0]),
           lambda: cmsd.embedding(t, w, out={"x": x[:2]}), lambda: cmsd.embedding(t.view(2, 2), w),
           lambda: cmsd.embedding(t, w, out={"x": x.bfloat16()}),
           lambda: cmsd.embedding_backward(t, x, 100, add=True), lambda: cmsd.embedding_backward(t, x, 0),
           lambda: cmsd.embedding_backward(t, x, 100, add=True, out={"x": x}),
           lambda: cmsd.embedding_backward(t, x, 100, out={"d_table": w.bfloat16()}, ws=ws),
           lambda: cmsd.embedding_backward(t[:3], x, 100, ws=ws), lambda: cmsd.embedding_backward(t, x[0], 100, ws=ws),
           lambda: cmsd.layernorm(x, p.half()), lambda: cmsd.layernorm(x, p, p.bfloat16()), lambda: cmsd.layernorm(x, p[:3]),
           lambda: cmsd.layernorm(x[0]), lambda: cmsd.layernorm(x.double()), lambda: cmsd.layernorm(x, out={"y": x.t()}),
           lambda: cmsd.layernorm(x, out={"y": x, "mean": f.double(), "rstd": f}),
           lambda: cmsd.layernorm_backward(x, p, f, f, x.bfloat16(), ws=ws),
           lambda: cmsd.layernorm_backward(x, p, f, f[:2], x, ws=ws),
           lambda: cmsd.layernorm_backward(x, p.half(), f, f, x, ws=ws),
           lambda: cmsd.layernorm_backward(x, p, f, f, x, out={"d_weight": p.bfloat16()}, ws=ws),
           lambda: cmsd.dropout(x.half(), 0.1, 1), lambda: cmsd.dropout(x, 0.1, 1, iteration=-1),
           lambda: cmsd.dropout(x, 0.1, 1, site=1 << 32), lambda: cmsd.dropout(x, 0.1, 1, residual=x[:2]),
           lambda: cmsd.dropout(x, 0.1, 1, residual=x.bfloat16()), lambda: cmsd.dropout(x, 0.1, 1, step=t[:1].long()),
           lambda: cmsd.dropout(x, 0.1, 1, step=t), lambda: cmsd.dropout_backward(x, 0.1, 1, out={"d_x": f}),
           # CPU tensors: there is no CPU path
           lambda: cmsd.embedding(t, w), lambda: cmsd.embedding_backward(t, x, 100, ws=ws), lambda: cmsd.layernorm(x, p, p),
           lambda: cmsd.layernorm_backward(x, p, f, f, x, ws=ws), lambda: cmsd.dropout(x, 0.1, 1),
           lambda: cmsd.dropout_backward(x, 0.1, 1)]
    for n, call in enumerate(bad):
        with pytest.raises(cmsd.CmsdError):
            call()
            pytest.fail(str(n))


def test_sizes_past_32_bits(cmsd):
    torch = pytest.importorskip("torch")
    meta = {"device": "meta"}
    big = torch.empty(2**32 + 5, 8, **meta)
    few = torch.empty(5, 8, **meta)
    t, f = torch.empty(5, dtype=torch.int32, **meta), torch.empty(2**32 + 5, **meta)
    ws = torch.zeros(64, dtype=torch.uint8)
    for call in (lambda: cmsd.embedding(t, big), lambda: cmsd.embedding(f.int(), few),
                 lambda: cmsd.embedding_backward(f.int(), big, 9, ws=ws),
                 lambda: cmsd.embedding_backward(t, few, 2**32 + 9, ws=ws), lambda: cmsd.layernorm(big),
                 lambda: cmsd.layernorm_backward(big, None, f, f, big, ws=ws),
                 lambda: cmsd.embedding_backward_workspace(2**32 + 4, 8, 9),
                 lambda: cmsd.embedding_backward_workspace(4, 8, 2**32 + 9),
                 lambda: cmsd.layernorm_backward_workspace(2**32 + 4, 8)):
        with pytest.raises(cmsd.CmsdError, match="out of range"):
            call()
    with pytest.raises(cmsd.CmsdError, match="ignore_index"):
        cmsd.embedding(t, few, ignore_index=2**31)


def test_nothing_is_detached_in_silence(cmsd):
    """Where autograd records, a result that it could not follow is refused; else the next check is reached."""
    torch = pytest.importorskip("torch")
    t, p = torch.zeros(4, dtype=torch.int32), torch.zeros(24)
    w, x = torch.zeros(100, 24, requires_grad=True), torch.zeros(4, 24, requires_grad=True)
    q = torch.zeros(24, requires_grad=True)
    calls = (lambda: cmsd.embedding(t, w), lambda: cmsd.layernorm(x, p, p), lambda: cmsd.layernorm(x.detach(), q, p),
             lambda: cmsd.layernorm(x.detach(), p, q), lambda: cmsd.dropout(x, 0.1, 1),
             lambda: cmsd.dropout(x.detach(), 0.1, 1, residual=x))
    for call in calls:
        with pytest.raises(cmsd.CmsdError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(cmsd.CmsdError, match="CUDA"):
            call()
