"""The embedding's gradient, layer norm and a training step on orders of rows that come late in their kernels: rings
that go round, launches that begin early beside many zeros, padding behind the last row.

Bounds are those of the calls' own tests, which these use.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import test_embedding_gpu as E  # noqa: E402
import test_layernorm_gpu as N  # noqa: E402
import test_train_chain_gpu as S  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def cmsd():
    from paper_2508_15371_gb300 import cmsd as C
    assert torch.cuda.is_available()
    C.lib()
    return C


# rows that begin on any entry or pair, four times and more round each ring: 8, 4, 2 and 1 rows of a CTA at a time (4864,
# 3648, 1824, 912 and 456 of the grid forward, at most a third less backward), the widest gradients 152
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,d", [(25001, 255), (15001, 511), (8001, 1001), (8001, 1002), (4001, 2047), (2001, 4095), (2001, 4090), (801, 8191)])
def test_rings_of_rows_off_16_bytes(cmsd, R, d, dtype):
    x, w, b, d_y = N._inputs(R, d, dtype, F32, seed=21)
    o = cmsd.layernorm(x, w, b, eps=N.EPS)
    N._check(o, x, w, b)
    N._check_grads(cmsd.layernorm_backward(x, w, o["mean"], o["rstd"], d_y), x, w, o["mean"], o["rstd"], d_y)


# tables of 64 MB, one row less, and more; of 16 KB a row and less; rows about those that are ordered by comparing them
@pytest.mark.parametrize("R,d,V,dtype", [(1217, 1024, 32768, BF16), (1217, 1024, 32767, BF16), (4096, 2048, 40001, BF16),
                                         (7168, 1024, 57344, BF16),
                                         (7168, 1024, 57343, BF16), (7168, 513, 70001, BF16), (5000, 260, 80001, F32), (1216, 512, 70000, BF16)])
def test_rows_ordered_beside_many_zeros(cmsd, R, d, V, dtype):
    """Calls one behind the other, whose tokens and rows the launch before them writes and whose workspace is the same."""
    g = E._gen(R, d, V, 5)
    sources = [(E._tokens(R, V, g, ignored=0.1, hot=k == 1), torch.randn(R, d, generator=g, device="cuda").to(dtype)) for k in range(3)]
    tokens, d_x = torch.empty_like(sources[0][0]), torch.empty_like(sources[0][1])
    outs = [torch.full((V, d), 7, dtype=dtype, device="cuda") for _ in sources]
    ws = cmsd.embedding_backward_workspace(R, d, V)

    def calls():
        for (t, x), out in zip(sources, outs):
            d_x.copy_(x)
            tokens.copy_(t)
            cmsd.embedding_backward(tokens, d_x, V, scale=1.5, out={"d_table": out}, ws=ws)

    calls()
    first = [o.clone() for o in outs]
    for (t, x), o in zip(sources, outs):
        E._check_table(o, t, x, V, 1.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(2):
        for o in outs:
            o.fill_(7)
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, f) for o, f in zip(outs, first))
    assert cmsd.embedding_errors() == 0


def test_padding_keeps_to_itself_backward(cmsd):
    """Rows of padding behind the others leave their gradients what they were, and have none.

    d_hidden's sums may be formed in other parts: fp32 sums that agree beyond bf16, each rounded once, are at most a
    step of bf16 apart, 2 2^-8 of an entry (h below).  What layer norm makes of that: g = d_y w moves by max |w| of it,
    and d_x = rstd (g less its parts along 1 and h) by at most rstd times g's move, and its own rounding; dropout
    scales that, and rounds."""
    i = S._inputs(200, 136, 500)
    o = S._step(cmsd, i)
    j = {k: (torch.cat([v, v.new_full((56,), S.IGNORE if v.dtype is torch.int32 else 0)]) if k in ("tokens", "labels", "grad") else v)
         for k, v in i.items()}
    q = S._step(cmsd, j)
    h = 2 * 2.0 ** -8 * (1 + 2.0 ** -8)

    def norms(t):
        return t.double().norm(dim=1)

    def moved(k):
        return norms(q[k][:200].double() - o[k].double())

    d_hidden = h * norms(o["b.d_hidden"])
    d_x = o["n.rstd"].double() * i["weight"].double().abs().max() * d_hidden * (1 + 2.0 ** -16) + h * norms(o["m.d_x"])
    dropped = d_x * 65536 / (65536 - round(S.P * 65536)) + h * norms(o["g.d_x"])
    for k, tol in (("b.d_hidden", d_hidden), ("m.d_x", d_x), ("g.d_x", dropped)):
        assert (moved(k) <= tol + 2.0 ** -100).all(), k
        assert (q[k][200:] == 0).all(), k
    kept = i["labels"] >= 0
    assert (o["b.d_hidden"][kept] != 0).any(dim=1).all()
