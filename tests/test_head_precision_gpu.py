"""How precise the head's loss and its gradients are, at widths whose sums over
K are cut into parts, with bounds that a sum left uncut, or a sum of
exponentials that misses an entry, does not meet.

Bounds (u = 2^-24, half a step of fp32; b = 2^-8, half a step of bf16):
  logits  a step of 16 of K loses at most one unit in the last place of the
          part's running sum (2 u of it) and of each of its products; a part
          ends after 1024 of K, and adding it to those before rounds once:
          e = 2 u (sum over steps |sum of the part so far| + sum_j |h_j w_vj|)
              + u sum over parts |sum so far|.
  lse     sum_v p_v e_v, for the logits; and, for what follows them,
          eta = 4 u |lse| (the two conversions between bases, their constants,
          lse's own rounding) + 2^-21 (an exponential is off by 2^-22, the
          logarithm and the products by less) + u (128 + V / 512): 16 + 4
          additions in a tile, then at most 15 + V / 8192 joins of two sums in a
          row, each an exponential (4 u), a product and an addition.
  P       the backward pass forms its logits in the order that lse's were formed
          in, so they are the same numbers, and z - lse is off by lse's eta
          alone.  By its own logits an entry is off by p eta (2^-21 and 4 u |lse|
          again for the exponent); what the logits' errors do to a softmax is
          2 max(e) p (1 - p), in either direction; and the rounding to bf16, b |P|.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U, B16, PART = 2.0 ** -24, 2.0 ** -8, 1024


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


def _sure_rows(R, d, V, low, high, seed):
    """Rows that predict one entry each, its logit between low and high and the others' about 0 +- 2."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn(V, d, generator=g, device="cuda") * (2.0 / math.sqrt(d))).bfloat16()
    best = torch.randperm(V, generator=g, device="cuda")[:R]
    up = low + (high - low) * torch.rand(R, 1, generator=g, device="cuda")
    wb = w[best].float()
    x = torch.randn(R, d, generator=g, device="cuda")
    n = wb.square().sum(1, keepdim=True)
    x = x + (up - (x * wb).sum(1, keepdim=True)) / n * wb
    return x.bfloat16(), w, best


def _logits(h, w):
    """The logits and their bound e, a few entries at a time."""
    hd, wd = h.double(), w.double()
    z, e = [], []
    for wv in wd.split(64):
        x = hd[:, None, :] * wv[None]                                  # [R, 64, d]
        steps = torch.nn.functional.pad(x, (0, -x.shape[2] % PART)).view(*x.shape[:2], -1, PART // 16, 16).sum(4)
        run = steps.cumsum(3)
        whole = run[..., -1].cumsum(2)
        z.append(whole[..., -1])
        e.append(2 * U * (run.abs().sum((2, 3)) + x.abs().sum(2)) + U * whole.abs().sum(2))
    return torch.cat(z, 1), torch.cat(e, 1)


def _eta(lse, V):
    return 4 * U * lse.abs() + 2.0 ** -21 + U * (128 + V / 512)


# both kinds of kernels (up to 128 rows, more), widths of one part and a bit, two, eight and sixteen parts
CASES = [(R, d) for R in (24, 160) for d in (1040, 2048, 8192, 16384)]


@pytest.mark.parametrize("R,d", CASES)
def test_sums_over_k_are_cut(cmsd, R, d):
    V = 192
    h, w, best = _sure_rows(R, d, V, 20.0, 28.0, 17)
    y = ((best + 1 + torch.arange(R, device="cuda")) % V).int()        # (labels of any entry)
    o = cmsd.lmhead_loss(h, w, y)
    z, e = _logits(h, w)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    tol = (p * e).sum(1) * 1.001 + _eta(lse, V)
    err = (o["lse"].double() - lse).abs()
    assert err.le(tol).all(), (err / tol).max()
    zy, ey = (t.gather(1, y.long()[:, None])[:, 0] for t in (z, e))
    err = (o["loss"].double() - (lse - zy)).abs()
    assert err.le(tol + ey).all(), (err / (tol + ey)).max()


@pytest.mark.parametrize("R,d", CASES)
def test_gradient_of_sure_rows(cmsd, R, d):
    """Rows whose label has nearly all of the probability: P there is p - 1, a difference of nearly equal
    numbers, and the gradients are those of the exact softmax."""
    V = 192
    h, w, best = _sure_rows(R, d, V, 20.0, 28.0, 18)
    y, g = best.int(), torch.full((R,), 0.25, device="cuda")
    o = cmsd.lmhead_loss_backward(h, w, y, cmsd.lmhead_loss(h, w, y)["lse"], g)
    z, e = _logits(h, w)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    q = -torch.expm1(z - lse[:, None])                                 # 1 - p
    q[torch.arange(R, device="cuda"), best] = (p.sum(1) - p[torch.arange(R, device="cuda"), best])
    off = p * _eta(lse, V)[:, None] * 2 + 2 * e.amax(1)[:, None] * 1.001 * p * q.abs()
    P = p.clone()
    P[torch.arange(R, device="cuda"), best] = -q[torch.arange(R, device="cuda"), best]
    P, off = P * 0.25, off * 0.25
    off = off + B16 * (P.abs() + off)
    for name, a, c, n in (("d_hidden", P, w.double(), V), ("d_weight", P.T, h.double(), R)):
        o2 = off if name == "d_hidden" else off.T
        want = a @ c
        tol = (o2 + n * 2 * U * a.abs()) @ c.abs()
        tol = tol + B16 * (want.abs() + tol)
        err = (o[name].double() - want).abs()
        assert err.le(tol).all(), (name, (err / tol).max())


@pytest.mark.parametrize("R,d,V", [(97, 72, 39001), (32, 64, 20000), (5, 64, 32001), (300, 72, 39001), (130, 64, 20015)])
def test_every_entry_of_the_last_tile_counts(cmsd, R, d, V):
    """The entries behind the last multiple of 256 share half of the probability, and none of them is a label."""
    g = torch.Generator(device="cuda").manual_seed(V + R)
    n = V % 256
    w = torch.randn(V, d, generator=g, device="cuda") / math.sqrt(d)
    w[:, 0] = 0.0
    w[V - n:, 0] = math.log((V - n) / n) / 8.0
    w = w.bfloat16()
    h = torch.randn(R, d, generator=g, device="cuda")
    h[:, 0] = 8.0
    h = h.bfloat16()
    y = torch.randint(0, V - n, (R,), generator=g, device="cuda").int()
    z, e = _logits(h, w)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    share = p[:, V - n:]
    tol = (p * e).sum(1) * 1.001 + _eta(lse, V)
    assert share.sum(1).min() > 0.01
    assert (tol < share.amin(1) * 0.9).float().mean() > 0.9            # (an entry left out shows in nine rows of ten)
    err = (cmsd.lmhead_loss(h, w, y)["lse"].double() - lse).abs()
    assert err.le(tol).all(), (err / tol).max()
