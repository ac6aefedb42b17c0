"""A drafter's training step through the library's calls, as a program makes it:
tokens, embedding, dropout with a residual, layer norm, the head's loss, and all
the way back to the table that the head shares.

The calls are tested one by one against their definitions elsewhere; here what
passes from one to the next is: each output is the next call's input as it
stands, padding keeps to itself, the whole is repeatable and can be captured.
The gradient is checked against 64-bit autograd of the same step from the bf16
tensors that the calls passed on (their rounding is theirs): d_table's tolerance
is the sum of those of the calls' tests, measured as a norm: each bf16 rounding
(2^-8) of d_hidden, d_x of the norm, d_x of dropout, P and the two d_table
roundings adds at most 2^-8 of its own norm, and no step but the norm's changes
norms by more than the factor that the reference shows.
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


P, SEED, SITE, EPS = 0.1, (7 << 32) + 99, 2, 1e-5


def _inputs(R, d, V, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(R + d + V + seed)
    tokens = torch.randint(0, V, (R,), generator=g, device="cuda")
    tokens[torch.rand(R, generator=g, device="cuda") < 0.3] = 5                # a token that many rows have
    labels = tokens.roll(-1)
    pad = torch.rand(R, generator=g, device="cuda") < 0.15
    tokens[pad], labels[pad] = IGNORE, IGNORE
    table = (torch.randn(V, d, generator=g, device="cuda") / math.sqrt(d)).bfloat16()
    weight = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    bias = 0.1 * torch.randn(d, generator=g, device="cuda")
    kept = (labels >= 0).sum()
    grad = (labels >= 0).float() / kept
    return dict(tokens=tokens.int(), labels=labels.int(), table=table, weight=weight, bias=bias, grad=grad)


def _step(cmsd, i, step=None, out=None, ws=None):
    """One training step's loss and gradients: dict of every tensor that it makes."""
    R, (V, d) = i["tokens"].numel(), i["table"].shape
    ws = ws or {}
    scale = math.sqrt(d)
    o = {} if out is None else out
    it = 4

    def sub(*names):
        return {k.split(".")[1]: o[k] for k in names if k in o}

    def put(prefix, r):
        o.update({prefix + "." + k: v for k, v in r.items()})
        return r

    x = put("e", cmsd.embedding(i["tokens"], i["table"], scale=scale, out=sub("e.x")))["x"]
    s = put("f", cmsd.dropout(x, P, SEED, it, SITE, residual=x, step=step, out=sub("f.y")))["y"]
    n = put("n", cmsd.layernorm(s, i["weight"], i["bias"], eps=EPS, out=sub("n.y", "n.mean", "n.rstd")))
    put("l", cmsd.lmhead_loss(n["y"], i["table"], i["labels"], out=sub("l.loss", "l.lse"), ws=ws.get("l")))
    b = put("b", cmsd.lmhead_loss_backward(n["y"], i["table"], i["labels"], o["l.lse"], i["grad"],
                                           out=sub("b.d_hidden", "b.d_weight"), ws=ws.get("b")))
    m = put("m", cmsd.layernorm_backward(s, i["weight"], n["mean"], n["rstd"], b["d_hidden"],
                                         out=sub("m.d_x", "m.d_weight", "m.d_bias"), ws=ws.get("m")))
    g = put("g", cmsd.dropout_backward(m["d_x"], P, SEED, it, SITE, step=step, out=sub("g.d_x")))["d_x"]
    # the residual's branch and dropout's, one after the other into the table that holds the head's part
    for dx in (g, m["d_x"]):
        cmsd.embedding_backward(i["tokens"], dx, V, scale=scale, add=True, out={"d_table": b["d_weight"]}, ws=ws.get("g"))
    return o


def _reference(i, o):
    """The step's gradients by autograd in 64 bits, the mask being what the step dropped."""
    table = i["table"].double().requires_grad_()
    weight, bias = i["weight"].double().requires_grad_(), i["bias"].double().requires_grad_()
    keep = i["tokens"] >= 0
    t = torch.where(keep, i["tokens"], 0).long()
    d = table.shape[1]
    x = torch.where(keep[:, None], table[t] * math.sqrt(d), 0.0)
    thr = round(P * 65536)
    factor = torch.where(o["mask"], 65536 / (65536 - thr), 0.0)
    s = x + x * factor
    m = s.mean(1, keepdim=True)
    y = (s - m) / ((s - m).square().mean(1, keepdim=True) + EPS).sqrt() * weight + bias
    z = y @ table.T
    rows = i["labels"] >= 0
    loss = torch.logsumexp(z[rows], 1) - z[rows].gather(1, i["labels"][rows].long()[:, None])[:, 0]
    (loss * i["grad"][rows].double()).sum().backward()
    return loss.detach(), table.grad, weight.grad, bias.grad


def _mask(cmsd, R, d, it):
    return cmsd.dropout(torch.ones(R, d, device="cuda"), P, SEED, it, SITE)["y"] != 0


@pytest.mark.parametrize("R,d,V", [(1, 64, 50), (40, 128, 300), (333, 264, 1001), (700, 512, 4000)])
def test_a_training_step(cmsd, R, d, V):
    i = _inputs(R, d, V)
    if R == 1:
        i["tokens"][0] = i["labels"][0] = 3
        i["grad"][0] = 1.0
    cmsd.embedding_errors()
    cmsd.lmhead_errors()
    o = _step(cmsd, i)
    o["mask"] = _mask(cmsd, R, d, 4)
    loss, d_table, d_weight, d_bias = _reference(i, o)
    rows = i["labels"] >= 0
    # hidden states are rounded to bf16 three times (2^-8 each): a logit of |y| |w| moves by less than 2^-6 of it
    size = o["n.y"].double().norm(dim=1).max() * i["table"].double().norm(dim=1).max()
    assert (o["l.loss"][rows].double() - loss).abs().max() <= 2 * 2.0 ** -6 * size
    for got, want in ((o["b.d_weight"], d_table), (o["m.d_weight"], d_weight), (o["m.d_bias"], d_bias)):
        err = (got.double() - want).norm() / want.norm()
        assert err <= 12 * 2.0 ** -8, err
    pad = ~rows
    assert (o["e.x"][pad] == 0).all() and (o["b.d_hidden"][pad] == 0).all() and (o["g.d_x"][pad] == 0).all()
    assert (o["l.loss"][pad] == 0).all()
    assert cmsd.embedding_errors() == 0 and cmsd.lmhead_errors() == 0


def test_padding_changes_nothing(cmsd):
    """The kept rows' results are the same whatever stands in padded rows' labels and how many there are behind them."""
    i = _inputs(200, 136, 500)
    o = _step(cmsd, i)
    j = {k: (torch.cat([v, v.new_full((56,), IGNORE if v.dtype is torch.int32 else 0)]) if k in ("tokens", "labels", "grad") else v)
         for k, v in i.items()}
    q = _step(cmsd, j)
    for k in o:
        a = q[k][:200] if q[k].shape[0] == 256 else q[k]
        if k in ("b.d_weight", "m.d_weight", "m.d_bias"):       # sums over another number of rows: fp32 roundings
            assert (a.double() - o[k].double()).norm() <= 2.0 ** -8 * o[k].double().norm(), k
        elif k not in ("m.d_x", "g.d_x"):                       # (d_hidden may be summed in other parts)
            assert torch.equal(a, o[k]) or k == "b.d_hidden", k


def test_captured_and_replayed(cmsd):
    """The whole step in a graph with its own workspaces: new tokens in the same buffers, a new mask by the step's word."""
    R, d, V = 256, 128, 1000
    i, j = _inputs(R, d, V), _inputs(R, d, V, seed=1)
    ws = dict(l=cmsd.lmhead_loss_workspace(R, d, V), b=cmsd.lmhead_loss_backward_workspace(R, d, V),
              m=cmsd.layernorm_backward_workspace(R, d), g=cmsd.embedding_backward_workspace(R, d, V))
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = []
    for src, s in ((i, 0), (j, 1), (i, 2)):
        step.fill_(s)
        want.append({k: v.clone() for k, v in _step(cmsd, src, step=step).items()})
    bufs = {k: v.clone() for k, v in i.items()}
    out = {k: torch.empty_like(v) for k, v in want[0].items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(cmsd, bufs, step=step, out=out, ws=ws)
    for src, s, ref in ((i, 0, want[0]), (j, 1, want[1]), (i, 2, want[2])):
        for k in bufs:
            bufs[k].copy_(src[k])
        step.fill_(s)
        graph.replay()
        torch.cuda.synchronize()
        for k in ref:
            assert torch.equal(out[k], ref[k]), k


def test_a_decode_steps_hidden_states(cmsd):
    """Serving: emitted tokens' rows, their norm, then the head with the signals and the head in 8 bits."""
    R, d, V = 12, 128, 1000
    i = _inputs(R, d, V)
    x = cmsd.embedding(i["tokens"], i["table"], scale=math.sqrt(d))["x"]
    h = cmsd.layernorm(x, i["weight"], i["bias"], stats=False)["y"]
    r = cmsd.lmhead_confidence(h, i["table"], logits=True)
    z = h.double() @ i["table"].double().T
    assert (r["logits"].double() - z).abs().max() <= d * 2.0 ** -23 * (h.double().abs() @ i["table"].double().abs().T).max()
    q, w = cmsd.quantize_rows(h), cmsd.quantize_rows(i["table"])
    z8 = cmsd.lmhead_i8(q["q"], q["scale"], w["q"], w["scale"], dtype=torch.float32)["logits"].double()
    a, b = q["q"].double() * q["scale"].double()[:, None], w["q"].double() * w["scale"].double()[:, None]
    assert (z8 - a @ b.T).abs().max() <= 4 * 2.0 ** -24 * (a.abs() @ b.abs().T).max()
