"""The drafter's output head, trained and served in 8 bits: the calls that its speed is measured on.

Four operators beside cmsd.lmhead_confidence (the drafter's last projection z = h W^T):

  quantize  cmsd.quantize_rows: symmetric 8-bit integers with a scale for each row, of a head's weight (a row: a channel)
            or of hidden states (a row: a token)
  i8        cmsd.lmhead_i8: the logits of a head in 8-bit integers, scales for each token and channel
  loss      cmsd.lmhead_loss: softmax cross entropy of the head's logits, which are never kept
  grad      cmsd.lmhead_loss_backward: its gradients by the hidden states and by the weight

With `own` the library's calls, without it the same in elementary torch operations.
"""
import math

import torch

own = False

IGNORE = -100


def listed():
    return [
        # the hidden states of a decode step before the 8-bit product: latency
        dict(name="quantize_token", kind="quantize", R=16, d=1024, dtype="bf16"),
        # a whole head, each time its weight has changed
        dict(name="quantize_head", kind="quantize", R=128256, d=2048, dtype="bf16"),
        # one sequence's next token
        dict(name="i8_token", kind="i8", R=1, d=1024, V=32000, out="f32"),
        # a ragged window over an odd vocabulary (unaligned logit rows), f32 logits
        dict(name="i8_odd", kind="i8", R=37, d=1040, V=32001, out="f32"),
        # 64 sequences' next drafted position
        dict(name="i8_window", kind="i8", R=64, d=2048, V=128256, out="bf16"),
        # 64 sequences with windows of 8 positions: every logit that a verification reads
        dict(name="i8_rows", kind="i8", R=512, d=2048, V=128256, out="bf16"),
        # a short ragged sequence of a small drafter, an odd vocabulary
        dict(name="loss_small", kind="loss", R=33, d=1024, V=32001, ignored=0.25),
        # the scores of 64 given tokens (perplexity of a draft)
        dict(name="loss_window", kind="loss", R=64, d=2048, V=128256, ignored=0.0),
        # a training batch of 4096 positions, three in ten of them prompt or padding
        dict(name="loss_train", kind="loss", R=4096, d=2048, V=128256, ignored=0.3),
        # the gradients of the short sequence
        dict(name="grad_small", kind="grad", R=33, d=1024, V=32001, ignored=0.25, hidden=True, weight=True),
        # a drafter trained under a frozen head: the hidden states' gradient alone
        dict(name="grad_hidden", kind="grad", R=512, d=2048, V=128256, ignored=0.0, hidden=True, weight=False),
        # both gradients of the training batch
        dict(name="grad_train", kind="grad", R=4096, d=2048, V=128256, ignored=0.3, hidden=True, weight=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "i8", "i8", "loss", "loss", "grad", "grad"])
    if kind == "quantize":
        R = min(128256, _log(rng, 1, 128256))
        return dict(kind=kind, R=R, d=16 * min(128, _log(rng, 1, 128)), dtype=rng.choice(["bf16", "bf16", "f32"]))
    V = min(128256, _log(rng, 1000, 128256))
    if kind == "i8":
        return dict(kind=kind, R=min(512, _log(rng, 1, 512)), d=16 * rng.randint(8, 128), V=V, out=rng.choice(["f32", "bf16"]))
    case = dict(kind=kind, R=min(4096, _log(rng, 1, 4096)), d=8 * rng.randint(16, 256), V=V,
                ignored=rng.choice([0.0, 0.1, rng.uniform(0.0, 0.6)]))
    if kind == "grad":
        case["hidden"], case["weight"] = rng.choice([(True, True), (True, True), (True, False), (False, True)])
    return case


def _kept(case):
    """Rows with a label: the others are prompt or padding."""
    return case["R"] - int(round(case["R"] * case["ignored"]))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    kind, R, d = case["kind"], case["R"], case["d"]
    state = {"case": case}
    if kind == "quantize":
        # rows of unequal size, as channels and tokens are
        x = normal(R, d) * (0.02 + 0.1 * torch.rand(R, 1, generator=g, device="cuda"))
        state["x"] = x.bfloat16() if case["dtype"] == "bf16" else x
        return state
    V = case["V"]
    if kind == "i8":
        state["hidden_q"] = (normal(R, d) * 36).round().clamp(-127, 127).to(torch.int8)
        state["weight_q"] = (normal(V, d) * 36).round().clamp(-127, 127).to(torch.int8)
        state["hidden_scale"] = 0.01 + 0.05 * torch.rand(R, generator=g, device="cuda")
        state["weight_scale"] = (0.5 + torch.rand(V, generator=g, device="cuda")) / (18.0 * math.sqrt(d))
        return state
    labels = torch.randint(0, V, (R,), generator=g, device="cuda")
    weight = (normal(V, d) * (2.0 / math.sqrt(d))).bfloat16()
    # a trained head: the label's logit stands 0 to 14 above where chance puts it
    w = weight[labels].float()
    up = 14.0 * torch.rand(R, 1, generator=g, device="cuda") / w.square().sum(1, keepdim=True)
    state["hidden"] = (normal(R, d) + up * w).bfloat16()
    gone = torch.randperm(R, generator=g, device="cuda")[_kept(case):]
    labels[gone] = IGNORE
    state["weight"], state["labels"] = weight, labels.int()
    if kind == "grad":
        # what the forward pass left: each row's log-sum-exp; the mean over the kept rows is the loss
        z = state["hidden"].float() @ weight.float().T
        state["lse"] = torch.logsumexp(z, 1) * (state["labels"] >= 0)
        state["grad"] = torch.full((R,), 1.0 / max(1, _kept(case)), device="cuda") * (state["labels"] >= 0)
    return state


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        return _calls(state, kind, case)
    if kind == "quantize":
        # 127 x is exact in 32 bits for a bf16 x, and no quotient then lies nearer to a tie than it rounds
        x = state["x"].float() if case["dtype"] == "bf16" else state["x"].double()
        amax = x.abs().amax(1, keepdim=True)
        q = torch.round(x * 127 / torch.where(amax > 0, amax, 1.0))
        scale = (amax / torch.full_like(amax, 127)).float()
        return {"values": q.float() * scale, "scale": scale[:, 0]}
    if kind == "i8":
        s = state["hidden_q"].float() @ state["weight_q"].float().T
        z = s * state["hidden_scale"][:, None] * state["weight_scale"]
        return {"logits": z.bfloat16() if case["out"] == "bf16" else z}
    h, w = state["hidden"].float(), state["weight"].float()
    kept = state["labels"] >= 0
    label = torch.where(kept, state["labels"], 0).long()[:, None]
    z = h @ w.T
    if kind == "loss":
        m = z.amax(1, keepdim=True)
        lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))[:, 0]
        loss = lse - z.gather(1, label)[:, 0]
        return {"loss": torch.where(kept, loss, 0.0), "lse": torch.where(kept, lse, 0.0)}
    p = torch.exp(z - state["lse"][:, None])
    p.scatter_add_(1, label, torch.full_like(label, -1, dtype=torch.float32))
    p = torch.where(kept[:, None], p * state["grad"][:, None], 0.0)
    out = {}
    if case["hidden"]:
        out["d_hidden"] = (p @ w).bfloat16()
    if case["weight"]:
        out["d_weight"] = (p.T @ h).bfloat16()
    return out


def _calls(state, kind, case):
    from paper_2508_15371_gb300 import cmsd
    R, d = case["R"], case["d"]
    if kind == "quantize":
        o = cmsd.quantize_rows(state["x"])
        # what is held in 8 bits, as the values that it stands for
        return {"values": o["q"] * o["scale"][:, None], "scale": o["scale"]}
    V = case["V"]
    if "ws" not in state:           # a program keeps its workspace
        make = {"i8": cmsd.lmhead_i8_workspace, "loss": cmsd.lmhead_loss_workspace,
                "grad": cmsd.lmhead_loss_backward_workspace}[kind]
        state["ws"] = make(R, d, V)
    if kind == "i8":
        return cmsd.lmhead_i8(state["hidden_q"], state["hidden_scale"], state["weight_q"], state["weight_scale"],
                              dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, ws=state["ws"])
    if kind == "loss":
        return cmsd.lmhead_loss(state["hidden"], state["weight"], state["labels"], ignore_index=IGNORE,
                                ws=state["ws"])
    return cmsd.lmhead_loss_backward(state["hidden"], state["weight"], state["labels"], state["lse"], state["grad"],
                                     ignore_index=IGNORE, hidden_grad=case["hidden"], weight_grad=case["weight"],
                                     ws=state["ws"])


def work(case):
    """Inputs once, outputs once; two operations for each product and sum."""
    kind, R, d = case["kind"], case["R"], case["d"]
    if kind == "quantize":
        return {"bytes": R * d * ((2 if case["dtype"] == "bf16" else 4) + 1) + 4 * R, "flops": 4 * R * d}
    V = case["V"]
    if kind == "i8":
        return {"bytes": (R + V) * (d + 4) + R * V * (2 if case["out"] == "bf16" else 4), "flops": 2 * R * V * d}
    n = _kept(case)
    if kind == "loss":
        return {"bytes": 2 * d * (n + V) + 12 * R, "flops": 2 * n * V * d}
    both = int(case["hidden"]) + int(case["weight"])
    written = 2 * d * (R * int(case["hidden"]) + V * int(case["weight"]))
    return {"bytes": 2 * d * (n + V) + 12 * R + written, "flops": 2 * n * V * d * (1 + both)}


def exact(case, seed):
    """The definitions in 64 bits, a block of the vocabulary at a time."""
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        x = state["x"].double()
        amax = x.abs().amax(1)
        step = amax / torch.full_like(amax, 127.0)
        # the whole number nearest to 127 x / amax, of two equally near the even one: both sides times amax, exactly
        low = torch.floor(x * 127 / torch.where(amax > 0, amax, 1.0)[:, None])
        past = 254 * x - (2 * low + 1) * amax[:, None]
        q = low + ((past > 0) | ((past == 0) & (low % 2 != 0)))
        return {"values": q * step[:, None], "scale": step}
    if kind == "i8":
        a = state["hidden_q"].double() * state["hidden_scale"].double()[:, None]
        blocks = [a @ (wq.double() * ws.double()[:, None]).T
                  for wq, ws in zip(state["weight_q"].split(16384), state["weight_scale"].split(16384))]
        return {"logits": torch.cat(blocks, 1)}
    rows = torch.nonzero(state["labels"] >= 0)[:, 0]
    h, y = state["hidden"][rows].double(), state["labels"][rows].long()
    at, n = 0, rows.numel()
    R, d = state["hidden"].shape
    if kind == "loss":
        parts, zy = [], torch.zeros(n, dtype=torch.float64, device="cuda")
        for w in state["weight"].split(16384):
            z = h @ w.double().T
            parts.append(torch.logsumexp(z, 1))
            mine = (y >= at) & (y < at + w.shape[0])
            zy[mine] = z[mine, y[mine] - at]
            at += w.shape[0]
        lse = torch.zeros(R, dtype=torch.float64, device="cuda")
        loss = lse.clone()
        lse[rows] = torch.logsumexp(torch.stack(parts), 0)
        loss[rows] = lse[rows] - zy
        return {"loss": loss, "lse": lse}
    lse, g = state["lse"][rows].double(), state["grad"][rows].double()
    dh, dw = torch.zeros(n, d, dtype=torch.float64, device="cuda"), []
    for w in state["weight"].split(16384):
        w = w.double()
        s = torch.exp(h @ w.T - lse[:, None])
        mine = torch.nonzero((y >= at) & (y < at + w.shape[0]))[:, 0]
        s[mine, y[mine] - at] -= 1.0
        s *= g[:, None]
        if case["hidden"]:
            dh += s @ w
        if case["weight"]:
            dw.append(s.T @ h)
        at += w.shape[0]
    out = {}
    if case["hidden"]:
        out["d_hidden"] = torch.zeros(R, d, dtype=torch.float64, device="cuda")
        out["d_hidden"][rows] = dh
    if case["weight"]:
        out["d_weight"] = torch.cat(dw)
    return out
