"""The head's loss, its gradients, the 8-bit rows and the 8-bit product without
a GPU: argument errors are found on the host before anything is enqueued, and
workspace sizes depend on the sizes of the call alone."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2508_15371_gb300")
A = 4096            # addresses that nothing reads: every call here is refused
H, W, Y, X1, X2, O1, O2, WS = (A + (k << 32) for k in range(8))      # far enough apart


@pytest.fixture(scope="module")
def cmsd():
    if not os.path.exists(os.path.join(PKG, "libcmsd.so")):
        from paper_2508_15371_gb300 import build
        build.build()
    from paper_2508_15371_gb300 import cmsd as c
    c.lib()
    return c


def _loss(c, R=4, d=64, V=100, hidden=H, weight=W, labels=Y, loss=O1, lse=O2, ws=WS, ws_bytes=None):
    n = c.lib().cmsd_lmhead_loss_workspace_bytes(R, d, V) if ws_bytes is None else ws_bytes
    return c.lib().cmsd_lmhead_loss(hidden, weight, labels, R, d, V, -100, loss, lse, ws, n, None)


def _back(c, R=4, d=64, V=100, hidden=H, weight=W, labels=Y, lse=X1, grad=X2, dh=O1, dw=O2, ws=WS, ws_bytes=None):
    n = c.lib().cmsd_lmhead_loss_backward_workspace_bytes(R, d, V) if ws_bytes is None else ws_bytes
    return c.lib().cmsd_lmhead_loss_backward(hidden, weight, labels, lse, grad, R, d, V, -100, dh, dw, ws, n, None)


def _i8(c, R=4, d=64, V=100, h=H, hs=X1, w=W, wsc=X2, out=O1, dtype=1, ws=WS, ws_bytes=None):
    n = c.lib().cmsd_lmhead_i8_workspace_bytes(R, d, V) if ws_bytes is None else ws_bytes
    return c.lib().cmsd_lmhead_i8(h, hs, w, wsc, R, d, V, out, dtype, ws, n, None)


def _quant(c, R=4, d=64, x=H, q=O1, scale=O2, dtype=1):
    return c.lib().cmsd_quantize_rows(x, dtype, R, d, q, scale, None)


@pytest.mark.parametrize("kw", [dict(R=-1), dict(d=0), dict(d=4), dict(d=12), dict(d=(1 << 20) + 8), dict(V=1),
                                dict(R=1 << 23, V=1 << 23), dict(R=(1 << 28) + 1), dict(V=(1 << 30) + 1),
                                dict(R=1 << 27, d=1 << 20), dict(V=1 << 27, d=1 << 20)])
def test_loss_sizes_refused(cmsd, kw):
    assert _loss(cmsd, **kw) == cmsd.EINVAL
    assert _back(cmsd, **kw) == cmsd.EINVAL
    a = dict(R=4, d=64, V=100)
    a.update(kw)
    assert cmsd.lib().cmsd_lmhead_loss_workspace_bytes(a["R"], a["d"], a["V"]) == 0
    assert cmsd.lib().cmsd_lmhead_loss_backward_workspace_bytes(a["R"], a["d"], a["V"]) == 0


def test_loss_pointers_refused(cmsd):
    for name in ("hidden", "weight", "labels", "lse"):
        assert _loss(cmsd, **{name: None}) == cmsd.EINVAL, name
    for name in ("hidden", "weight", "ws"):
        assert _loss(cmsd, **{name: A + 8}) == cmsd.EALIGN, name
    for name in ("labels", "loss", "lse"):
        assert _loss(cmsd, **{name: A + 2}) == cmsd.EALIGN, name
    assert _loss(cmsd, ws=None) == cmsd.ENOWS
    n = cmsd.lib().cmsd_lmhead_loss_workspace_bytes(4, 64, 100)
    assert _loss(cmsd, ws_bytes=n - 1) == cmsd.ENOWS
    assert _loss(cmsd, R=0, hidden=None, weight=None, labels=None, lse=None, ws=None) == cmsd.OK


def test_backward_pointers_refused(cmsd):
    for name in ("hidden", "weight", "labels", "lse", "grad"):
        assert _back(cmsd, **{name: None}) == cmsd.EINVAL, name
    for name in ("hidden", "weight", "dh", "dw", "ws"):
        assert _back(cmsd, **{name: A + 8}) == cmsd.EALIGN, name
    for name in ("labels", "lse", "grad"):
        assert _back(cmsd, **{name: A + 2}) == cmsd.EALIGN, name
    assert _back(cmsd, dh=None, dw=None) == cmsd.EINVAL
    assert _back(cmsd, R=0, dh=None, dw=None) == cmsd.EINVAL
    assert _back(cmsd, R=0, dw=None) == cmsd.OK
    assert _back(cmsd, R=0, dw=A + 8) == cmsd.EALIGN
    assert _back(cmsd, ws=None) == cmsd.ENOWS
    n = cmsd.lib().cmsd_lmhead_loss_backward_workspace_bytes(4, 64, 100)
    assert _back(cmsd, ws_bytes=n - 1) == cmsd.ENOWS


@pytest.mark.parametrize("kw,code", [
    (dict(R=-1), "EINVAL"), (dict(d=8), "EINVAL"), (dict(d=24), "EINVAL"), (dict(d=(1 << 16) + 16), "EINVAL"),
    (dict(V=1), "EINVAL"), (dict(R=1 << 23, V=1 << 23), "EINVAL"), (dict(dtype=2), "EDTYPE"),
    (dict(R=(1 << 28) + 1), "EINVAL"), (dict(V=(1 << 30) + 1), "EINVAL"), (dict(hs=A + 2), "EALIGN"),
    (dict(wsc=A + 1), "EALIGN"),
    (dict(h=None), "EINVAL"), (dict(hs=None), "EINVAL"), (dict(w=None), "EINVAL"), (dict(wsc=None), "EINVAL"),
    (dict(out=None), "EINVAL"), (dict(h=A + 8), "EALIGN"), (dict(w=A + 4), "EALIGN"), (dict(out=A + 2), "EALIGN"),
    (dict(ws=None), "ENOWS"), (dict(ws_bytes=16), "ENOWS"), (dict(ws=A + 8), "EALIGN"),
    (dict(R=0, h=None, hs=None, w=None, wsc=None, out=None, ws=None), "OK")])
def test_i8_refused(cmsd, kw, code):
    assert _i8(cmsd, **kw) == getattr(cmsd, code)


@pytest.mark.parametrize("kw,code", [
    (dict(R=-1), "EINVAL"), (dict(d=8), "EINVAL"), (dict(d=40), "EINVAL"), (dict(d=(1 << 16) + 16), "EINVAL"),
    (dict(dtype=-1), "EDTYPE"), (dict(x=None), "EINVAL"), (dict(q=None), "EINVAL"), (dict(scale=None), "EINVAL"),
    (dict(R=1 << 30, d=1 << 16), "EINVAL"), (dict(scale=A + 2), "EALIGN"),
    (dict(x=A + 8), "EALIGN"), (dict(q=A + 4), "EALIGN"), (dict(R=0, x=None, q=None, scale=None), "OK")])
def test_quantize_refused(cmsd, kw, code):
    assert _quant(cmsd, **kw) == getattr(cmsd, code)


def test_outputs_share_no_bytes(cmsd):
    """An output in an input's, the workspace's or another output's place, or on its last or first bytes."""
    R, d, V = 4, 64, 100
    hb, wb, ib = R * d * 2, V * d * 2, R * d
    for kw in (dict(lse=Y), dict(loss=O2), dict(lse=O1 + R * 4 - 4), dict(loss=H + hb - 4), dict(lse=WS), dict(ws=W)):
        assert _loss(cmsd, **kw) == cmsd.EINVAL, kw
    for kw in (dict(dh=H), dict(dw=W), dict(dw=H - 16), dict(dh=W + wb - 16), dict(dh=O2 + 16), dict(ws=O1), dict(dh=X1),
               dict(dw=WS + 256)):
        assert _back(cmsd, **kw) == cmsd.EINVAL, kw
    assert _back(cmsd, dw=None, dh=H) == cmsd.EINVAL
    for kw in (dict(out=H), dict(out=W), dict(out=X1 - 16), dict(out=WS), dict(ws=X2)):
        assert _i8(cmsd, **kw) == cmsd.EINVAL, kw
    for kw in (dict(q=H), dict(q=H + hb - 16), dict(scale=H), dict(scale=O1 + ib - 4)):
        assert _quant(cmsd, **kw) == cmsd.EINVAL, kw


def test_workspaces_do_not_hold_the_logits(cmsd):
    """At most a sixteenth of the bf16 logits forward; backward a piece of 128 MB, the sums of d_hidden and
    the packed rows, whatever the vocabulary."""
    R, d = 4096, 2048
    for V in (128256, 1 << 20):
        logits = 2 * R * V
        assert cmsd.lib().cmsd_lmhead_loss_workspace_bytes(R, d, V) <= logits // 16 + 4 * R * d
        assert cmsd.lib().cmsd_lmhead_loss_backward_workspace_bytes(R, d, V) <= (128 << 20) + 40 * R * d


def test_binding_refuses_before_the_library(cmsd):
    torch = pytest.importorskip("torch")
    h, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(100, 64, dtype=torch.bfloat16)
    y = torch.zeros(4, dtype=torch.int32)
    f = torch.zeros(4)
    bad = [lambda: cmsd.lmhead_loss(h.float(), w, y), lambda: cmsd.lmhead_loss(h, w[:, :32], y),
           lambda: cmsd.lmhead_loss(h, w, y.long()), lambda: cmsd.lmhead_loss(h, w, y[:3]),
           lambda: cmsd.lmhead_loss(h, w, y, out={"lse": f[:2], "loss": f}),
           lambda: cmsd.lmhead_loss(h, w, y, out={"lse": None, "loss": f}),
           lambda: cmsd.lmhead_loss_backward(h, w, y, f.double(), f),
           lambda: cmsd.lmhead_loss_backward(h, w, y, f, f[:1]),
           lambda: cmsd.lmhead_loss_backward(h, w, y, f, f, out={"d_weight": w.float()}),
           lambda: cmsd.quantize_rows(h[0]), lambda: cmsd.quantize_rows(h.half()),
           lambda: cmsd.lmhead_i8(h, f, w, f), lambda: cmsd.lmhead_i8(h.char(), f, w.char(), f),
           lambda: cmsd.lmhead_i8(h.char(), f, w.char(), torch.zeros(100), dtype=torch.float16),
           lambda: cmsd.lmhead_loss(h, w, y, out={"lse": f, "loss": f})]      # CPU tensors: there is no CPU path
    for call in bad:
        with pytest.raises(cmsd.CmsdError):
            call()


# ---- sizes that a C int does not hold (they would be taken modulo 2^32) ----------------

@pytest.mark.parametrize("call", ["lmhead_loss_workspace", "lmhead_loss_backward_workspace", "lmhead_i8_workspace"])
@pytest.mark.parametrize("sizes", [(2**32 + 5, 64, 100), (5, 2**32 + 64, 100), (5, 64, 2**32 + 100), (2**31, 64, 100)])
def test_workspace_sizes_past_32_bits(cmsd, call, sizes):
    with pytest.raises(cmsd.CmsdError, match="out of range"):
        getattr(cmsd, call)(*sizes)


def test_rows_past_32_bits(cmsd):
    torch = pytest.importorskip("torch")
    big, few = (2**32 + 5, 64), (5, 64)
    meta = {"device": "meta"}
    bf16, i8 = torch.bfloat16, torch.int8
    for h, w in ((big, few), (few, big)):
        hidden, weight = torch.empty(h, dtype=bf16, **meta), torch.empty(w, dtype=bf16, **meta)
        rows = torch.empty(h[0], **meta)
        labels = torch.empty(h[0], dtype=torch.int32, **meta)
        with pytest.raises(cmsd.CmsdError, match="out of range"):
            cmsd.lmhead_loss(hidden, weight, labels)
        with pytest.raises(cmsd.CmsdError, match="out of range"):
            cmsd.lmhead_loss_backward(hidden, weight, labels, rows, rows)
        with pytest.raises(cmsd.CmsdError, match="out of range"):
            cmsd.lmhead_i8(hidden.to(i8), rows, weight.to(i8), torch.empty(w[0], **meta))
    with pytest.raises(cmsd.CmsdError, match="out of range"):
        cmsd.quantize_rows(torch.empty(big, **meta))


@pytest.mark.parametrize("ignore", [2**32 - 100, 2**31, -2**31 - 1])
def test_ignore_index_past_32_bits(cmsd, ignore):
    torch = pytest.importorskip("torch")
    h, w = torch.empty(5, 64, dtype=torch.bfloat16), torch.empty(9, 64, dtype=torch.bfloat16)
    y, f = torch.zeros(5, dtype=torch.int32), torch.zeros(5)
    with pytest.raises(cmsd.CmsdError, match="ignore_index"):
        cmsd.lmhead_loss(h, w, y, ignore_index=ignore)
    with pytest.raises(cmsd.CmsdError, match="ignore_index"):
        cmsd.lmhead_loss_backward(h, w, y, f, f, ignore_index=ignore)


def test_errors_need_a_place(cmsd):
    assert cmsd.lib().cmsd_lmhead_errors(None, None) == cmsd.EINVAL


@pytest.mark.parametrize("who", ["hidden", "weight"])
def test_loss_is_not_detached_in_silence(cmsd, who):
    """Where autograd records, a loss that it could not follow is refused; else the next check is reached."""
    torch = pytest.importorskip("torch")
    t = {"hidden": torch.zeros(4, 64, dtype=torch.bfloat16), "weight": torch.zeros(100, 64, dtype=torch.bfloat16)}
    t[who].requires_grad_()
    y = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(cmsd.CmsdError, match="autograd"):
        cmsd.lmhead_loss(t["hidden"], t["weight"], y)
    with torch.no_grad(), pytest.raises(cmsd.CmsdError, match="CUDA"):
        cmsd.lmhead_loss(t["hidden"], t["weight"], y)


def test_loss_and_gradients_make_an_autograd_function(cmsd, monkeypatch):
    """Both calls from inside an autograd.Function, on leaves that require gradients; the library is stood in for."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(cmsd, "_need", lambda cur, specs: None)
    monkeypatch.setattr(cmsd, "_stream_of", lambda cur: 0)
    seen = []

    class Lib:
        def cmsd_lmhead_loss(self, *a):
            seen.append("loss")
            return cmsd.OK

        def cmsd_lmhead_loss_backward(self, *a):
            seen.append("backward")
            return cmsd.OK
    monkeypatch.setattr(cmsd, "lib", lambda: Lib())
    ws = torch.zeros(64, dtype=torch.uint8)

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, h, w, y):
            o = cmsd.lmhead_loss(h, w, y, ws=ws)
            ctx.save_for_backward(h, w, y, o["lse"])
            return o["loss"]

        @staticmethod
        def backward(ctx, grad):
            o = cmsd.lmhead_loss_backward(*ctx.saved_tensors, grad.contiguous(), ws=ws)
            return o["d_hidden"].zero_(), o["d_weight"].zero_(), None
    h = torch.zeros(4, 64, dtype=torch.bfloat16, requires_grad=True)
    w = torch.zeros(100, 64, dtype=torch.bfloat16, requires_grad=True)
    Loss.apply(h, w, torch.zeros(4, dtype=torch.int32)).sum().backward()
    assert seen == ["loss", "backward"] and h.grad.shape == h.shape and w.grad.shape == w.shape


def test_wait_test_needs_a_workspace(cmsd):
    assert cmsd.lib().cmsd_test_head_wait(1, None, 256, None) == cmsd.ENOWS
    assert cmsd.lib().cmsd_test_head_wait(1, A, 3, None) == cmsd.ENOWS
    assert cmsd.lib().cmsd_test_head_wait(1, A + 2, 256, None) == cmsd.EALIGN
