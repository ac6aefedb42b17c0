"""A drafter's training below its output head: the calls that its speed is measured on.

Operators beside cmsd.lmhead_loss and cmsd.lmhead_loss_backward, which take the hidden states and give their gradient:

  embed       cmsd.embedding: scaled rows of the token table
  embed_grad  cmsd.embedding_backward: the table's gradient, each token's rows summed
  norm        cmsd.layernorm: layer norm of the hidden states, with the statistics that its gradients take
  norm_grad   cmsd.layernorm_backward: its gradients by the input, the weight and the bias
  drop        cmsd.dropout: dropout from the library's counter-based generator, with the residual added
  drop_grad   cmsd.dropout_backward: its gradient, the mask made again

With `own` the library's calls, without it the same in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

IGNORE = -100
EPS = 1e-5
# bytes of the largest listed case: no drawn one has more
MOST = 2 * 2048 * (32768 + 128256)


def listed():
    return [
        # 64 sequences' next token, in the decode loop: latency
        dict(name="embed_token", kind="embed", R=64, d=1024, V=32000, dtype="bf16", ignored=0.0),
        # a training batch of 16384 positions, three in ten of them padding
        dict(name="embed_batch", kind="embed", R=16384, d=2048, V=128256, dtype="bf16", ignored=0.3),
        # a short ragged batch over an odd vocabulary, f32
        dict(name="embed_grad_small", kind="embed_grad", R=333, d=1000, V=32001, dtype="f32", ignored=0.25),
        # 64 sequences' windows of 64 positions under the large vocabulary
        dict(name="embed_grad_window", kind="embed_grad", R=4096, d=1024, V=128256, dtype="bf16", ignored=0.0),
        # a large training batch
        dict(name="embed_grad_batch", kind="embed_grad", R=32768, d=2048, V=128256, dtype="bf16", ignored=0.1),
        # a decode step's hidden states before the head: latency, no statistics wanted
        dict(name="norm_token", kind="norm", R=16, d=1024, dtype="bf16", wdtype="bf16", stats=False),
        # a training batch, the norm's parameters kept in f32
        dict(name="norm_batch", kind="norm", R=16384, d=2048, dtype="bf16", wdtype="f32", stats=True),
        # a short ragged batch in f32, an odd width (rows off 16-byte boundaries)
        dict(name="norm_grad_small", kind="norm_grad", R=333, d=1001, dtype="f32", wdtype="f32"),
        # the training batch's gradients
        dict(name="norm_grad_batch", kind="norm_grad", R=16384, d=2048, dtype="bf16", wdtype="f32"),
        # a short batch after a sublayer
        dict(name="drop_small", kind="drop", R=333, d=1024, dtype="bf16", p=0.1, residual=True),
        # a training batch after a sublayer
        dict(name="drop_batch", kind="drop", R=16384, d=2048, dtype="bf16", p=0.1, residual=True),
        # its gradient
        dict(name="drop_grad_batch", kind="drop_grad", R=16384, d=2048, dtype="bf16", p=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad", "drop", "drop_grad"])
    d = min(2048, _log(rng, 64, 2048))
    if rng.random() < 0.75:
        d = (d + 7) // 8 * 8
    case = dict(kind=kind, R=min(32768, _log(rng, 1, 32768)), d=d, dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind in ("embed", "embed_grad"):
        case["V"] = min(128256, _log(rng, 1000, 128256))
        case["ignored"] = rng.choice([0.0, 0.1, rng.uniform(0.0, 0.6)])
    elif kind in ("norm", "norm_grad"):
        case["wdtype"] = rng.choice(["f32", case["dtype"]])
        if kind == "norm":
            case["stats"] = rng.random() < 0.7
    else:
        case["p"] = rng.choice([0.1, 0.1, rng.uniform(0.0, 0.6)])
        if kind == "drop":
            case["residual"] = rng.random() < 0.6
    while work(case)["bytes"] > MOST:
        if case.get("V", 0) > case["R"]:
            case["V"] = case["V"] * 2 // 3
        else:
            case["R"] = case["R"] * 2 // 3
    return case


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _size(name):
    return 2 if name == "bf16" else 4


def _kept(case):
    """Positions with a token: the others are padding."""
    return case["R"] - int(round(case["R"] * case["ignored"]))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    kind, R, d, dtype = case["kind"], case["R"], case["d"], _type(case["dtype"])
    state = {"case": case}
    if kind in ("embed", "embed_grad"):
        V = case["V"]
        # a token's frequency falls as one over its rank, the ranks being spread over the vocabulary
        rank = torch.exp(torch.rand(R, generator=g, device="cuda", dtype=torch.float64) * math.log(V + 1)).long() - 1
        tokens = torch.randperm(V, generator=g, device="cuda")[rank.clamp(0, V - 1)]
        tokens[torch.randperm(R, generator=g, device="cuda")[_kept(case):]] = IGNORE
        state["tokens"] = tokens.int()
        state["scale"] = float(np.float32(math.sqrt(d)))
        if kind == "embed":
            state["table"] = (normal(V, d) / math.sqrt(d)).to(dtype)
        else:
            state["d_x"] = (normal(R, d) / R).to(dtype)
        return state
    if kind in ("norm", "norm_grad"):
        # rows of unequal size, their means apart from 0
        x = (normal(R, d) + normal(R, 1)) * (0.5 + 2.0 * torch.rand(R, 1, generator=g, device="cuda"))
        state["x"] = x.to(dtype)
        state["weight"] = (1.0 + 0.1 * normal(d)).to(_type(case["wdtype"]))
        state["bias"] = (0.1 * normal(d)).to(_type(case["wdtype"]))
        if kind == "norm_grad":
            # what the forward pass left
            x = state["x"].float()
            state["mean"] = x.mean(1)
            state["rstd"] = torch.rsqrt((x - state["mean"][:, None]).square().mean(1) + EPS)
            state["d_y"] = (normal(R, d) / R).to(dtype)
        return state
    state["x"] = (normal(R, d) if kind == "drop" else normal(R, d) / R).to(dtype)
    state["residual"] = normal(R, d).to(dtype) if case.get("residual") else None
    # a run's seed, the training step, the layer
    state["seed"], state["iteration"], state["site"] = 7919 * (int(seed) + 1) + (5 << 32), int(seed) % 1000, 3
    return state


def _words(n, seed, iteration, site):
    """Philox4x32-10 of the counters (i, 0, site, iteration << 2 | 3), i < n, as n rows of four 32-bit words in int64."""
    low = 0xFFFFFFFF
    c = [torch.arange(n, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda"),
         torch.full((n,), site, dtype=torch.int64, device="cuda"),
         torch.full((n,), (iteration << 2 | 3) & low, dtype=torch.int64, device="cuda")]
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        # a product of two 32-bit numbers wraps to a negative one: the shift is masked
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32 & low) ^ c[1] ^ k0, q & low, (p >> 32 & low) ^ c[3] ^ k1, p & low]
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack(c, 1)


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        return _calls(state, kind, case)
    dtype = _type(case["dtype"])
    if kind in ("embed", "embed_grad"):
        kept = state["tokens"] >= 0
        tokens = torch.where(kept, state["tokens"], 0).long()
        if kind == "embed":
            x = state["table"][tokens].float() * state["scale"]
            return {"x": torch.where(kept[:, None], x, 0.0).to(dtype)}
        d_x = torch.where(kept[:, None], state["d_x"].float(), 0.0)
        d_table = torch.zeros(case["V"], case["d"], device="cuda").index_add_(0, tokens, d_x)
        return {"d_table": (d_table * state["scale"]).to(dtype)}
    if kind == "norm":
        x, w, b = state["x"].float(), state["weight"].float(), state["bias"].float()
        mean = x.mean(1)
        rstd = torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS)
        y = ((x - mean[:, None]) * rstd[:, None] * w + b).to(dtype)
        return {"y": y, "mean": mean, "rstd": rstd} if case["stats"] else {"y": y}
    if kind == "norm_grad":
        x, w, d_y = state["x"].float(), state["weight"].float(), state["d_y"].float()
        h = (x - state["mean"][:, None]) * state["rstd"][:, None]
        g = d_y * w
        d_x = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * state["rstd"][:, None]
        wtype = _type(case["wdtype"])
        return {"d_x": d_x.to(dtype), "d_weight": (d_y * h).sum(0).to(wtype), "d_bias": d_y.sum(0).to(wtype)}
    x = state["x"].float()
    n = x.numel()
    words = _words((n + 7) // 8, state["seed"], state["iteration"], state["site"])
    halves = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n].reshape(x.shape)
    t = round(case["p"] * 65536)
    y = torch.where(halves >= t, x * (65536 / (65536 - t)), 0.0)
    if state["residual"] is not None:
        y = state["residual"].float() + y
    return {"d_x" if kind == "drop_grad" else "y": y.to(dtype)}


def _calls(state, kind, case):
    from paper_2508_15371_gb300 import cmsd
    if kind == "embed":
        return cmsd.embedding(state["tokens"], state["table"], scale=state["scale"], ignore_index=IGNORE)
    if kind == "embed_grad":
        if "ws" not in state:       # a program keeps its workspace
            state["ws"] = cmsd.embedding_backward_workspace(case["R"], case["d"], case["V"])
        return cmsd.embedding_backward(state["tokens"], state["d_x"], case["V"], scale=state["scale"],
                                       ignore_index=IGNORE, ws=state["ws"])
    if kind == "norm":
        return cmsd.layernorm(state["x"], state["weight"], state["bias"], eps=EPS, stats=case["stats"])
    if kind == "norm_grad":
        if "ws" not in state:
            state["ws"] = cmsd.layernorm_backward_workspace(case["R"], case["d"])
        return cmsd.layernorm_backward(state["x"], state["weight"], state["mean"], state["rstd"], state["d_y"],
                                       ws=state["ws"])
    if kind == "drop":
        return cmsd.dropout(state["x"], case["p"], state["seed"], iteration=state["iteration"], site=state["site"],
                            residual=state["residual"])
    return cmsd.dropout_backward(state["x"], case["p"], state["seed"], iteration=state["iteration"], site=state["site"])


def _distinct(n, V):
    """How many tokens of the vocabulary n positions are expected to have (see prepare)."""
    edges = np.log(np.arange(1, V + 2, dtype=np.float64)) / math.log(V + 1)
    return int(np.sum(1.0 - (1.0 - np.diff(edges)) ** n))


def work(case):
    """Inputs once, outputs once; two operations for each product and sum."""
    kind, R, d, s = case["kind"], case["R"], case["d"], _size(case["dtype"])
    if kind == "embed":
        return {"bytes": 4 * R + (_distinct(_kept(case), case["V"]) + R) * d * s, "flops": R * d}
    if kind == "embed_grad":
        return {"bytes": 4 * R + (_kept(case) + case["V"]) * d * s, "flops": 2 * R * d}
    if kind == "norm":
        return {"bytes": 2 * R * d * s + 2 * d * _size(case["wdtype"]) + 8 * R * int(case["stats"]), "flops": 8 * R * d}
    if kind == "norm_grad":
        return {"bytes": 3 * R * d * s + 3 * d * _size(case["wdtype"]) + 8 * R, "flops": 14 * R * d}
    return {"bytes": (3 if case.get("residual") else 2) * R * d * s, "flops": 2 * R * d}


def exact(case, seed):
    """The definitions in 64 bits."""
    state = prepare(case, seed)
    kind, R, d = case["kind"], case["R"], case["d"]
    if kind in ("embed", "embed_grad"):
        rows = torch.nonzero(state["tokens"] != IGNORE)[:, 0]
        tokens = state["tokens"][rows].long()
        if kind == "embed":
            x = torch.zeros(R, d, dtype=torch.float64, device="cuda")
            x[rows] = state["table"].double()[tokens] * state["scale"]
            return {"x": x}
        # the rows in their tokens' order, and the sum of each run of one token
        order = torch.argsort(tokens, stable=True)
        lengths = torch.bincount(tokens, minlength=case["V"])
        sums = torch.zeros(case["V"], d, dtype=torch.float64, device="cuda")
        some = torch.nonzero(lengths)[:, 0]
        if rows.numel():
            sums[some] = torch.segment_reduce(state["d_x"][rows[order]].double(), "sum", lengths=lengths[some], axis=0)
        return {"d_table": sums * state["scale"]}
    if kind == "norm":
        x = state["x"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        std = torch.sqrt(var + EPS)
        y = (x - mean[:, None]) / std[:, None] * state["weight"].double() + state["bias"].double()
        return {"y": y, "mean": mean, "rstd": 1.0 / std} if case["stats"] else {"y": y}
    if kind == "norm_grad":
        mean, rstd, d_y = state["mean"].double(), state["rstd"].double(), state["d_y"].double()
        h = torch.addcmul(-mean[:, None] * rstd[:, None], state["x"].double(), rstd[:, None])
        g = d_y * state["weight"].double()
        along = torch.einsum("rd,rd->r", g, h) / d
        d_x = rstd[:, None] * (g - (g.sum(1) / d)[:, None] - h * along[:, None])
        return {"d_x": d_x, "d_weight": torch.einsum("rd,rd->d", d_y, h), "d_bias": torch.einsum("rd->d", d_y)}
    n = R * d
    groups = (n + 7) // 8
    mask = np.uint64(0xFFFFFFFF)
    a, b = np.arange(groups, dtype=np.uint64), np.zeros(groups, np.uint64)
    c = np.full(groups, state["site"], np.uint64)
    e = np.full(groups, ((state["iteration"] << 2) + 3) % (1 << 32), np.uint64)
    for r in range(10):
        key = [(state["seed"] % (1 << 32) + r * 0x9E3779B9) % (1 << 32), (state["seed"] // (1 << 32) + r * 0xBB67AE85) % (1 << 32)]
        p, q = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, e = (q >> np.uint64(32)) ^ b ^ np.uint64(key[0]), q & mask, (p >> np.uint64(32)) ^ e ^ np.uint64(key[1]), p & mask
    words = np.stack([a, b, c, e], 1).astype("<u4")
    keep = torch.from_numpy(words.view("<u2").reshape(-1)[:n].astype(np.int32)).cuda().reshape(R, d)
    t = round(case["p"] * 65536)
    y = state["x"].double() * (keep >= t) * (65536 / (65536 - t))
    if state["residual"] is not None:
        y = y + state["residual"].double()
    return {"d_x" if kind == "drop_grad" else "y": y}
