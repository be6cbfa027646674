"""Calls of the 8-bit operators that the documentation allows or refuses and that need a GPU tensor to be made."""
import pytest

from tests.test_gpu_int8 import generator, operands

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def bcq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2510_10467_amd
    return paper_2510_10467_amd


def test_matrices_that_are_none(bcq):
    """A number, a row or a stack in the place of a matrix is refused as an inconsistent shape."""
    gen = generator("none")
    q, ts, [(w, cs)] = operands(4, 24, 64, gen)
    dy = torch.randn((4, 24), device="cuda", generator=gen).half()
    for bad in (torch.zeros((), dtype=torch.int8, device="cuda"), w[0], w[None]):
        for call in (lambda: bcq.bcq_int8_gemm(q, ts, bad, cs), lambda: bcq.bcq_int8_gated(q, ts, bad, cs, w, cs), lambda: bcq.bcq_int8_gated(q, ts, w, cs, bad, cs),
                     lambda: bcq.bcq_int8_gemm(bad, ts, w, cs), lambda: bcq.bcq_int8_gemm_backward(dy, q, ts, bad, cs),
                     lambda: bcq.bcq_int8_gated_backward(dy, q, ts, bad, cs, w, cs)):
            with pytest.raises(ValueError, match="inconsistent shapes"):
                call()


def shut(q, ts, wg, tokens):
    """Scales with which the gates of these tokens are shut: their gradients are made a second time."""
    q, ts = q.clone(), ts.clone()
    q[tokens] = q[tokens].abs().clamp_min(60)
    g = (q[tokens].double() @ wg.double().t()).amin(dim=1)
    ts[tokens] = (-24.0 / g).float()
    return q, ts


def test_gradients_made_again_in_a_graph_and_on_two_streams(bcq):
    """Which tokens' gradients are made a second time is up to the values of each replay; two calls under way at once do not meet."""
    gen = generator("again")
    tokens, m, n = 150, 700, 528
    q, ts, [(wg, cg), (wu, cu)] = operands(tokens, m, n, gen, 2)
    wg, cg = -wg.abs(), torch.ones_like(cg)
    dh = torch.randn((tokens, m), device="cuda", generator=gen).bfloat16()
    ts = ts * 1e-5
    inputs = [(q, ts), shut(q, ts, wg, slice(0, None, 3)), shut(q, ts, wg, slice(70, 75)), shut(q, ts, wg, slice(0, tokens))]
    want = [bcq.bcq_int8_gated_backward(dh, *i, wg, cg, wu, cu) for i in inputs]
    assert all(bool((w[0] != 0).any(dim=1).all()) for w in want)
    at_q, at_ts = q.clone(), ts.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = bcq.bcq_int8_gated_backward(dh, at_q, at_ts, wg, cg, wu, cu)
    for k in (1, 0, 2, 3, 0, 1):
        at_q.copy_(inputs[k][0])
        at_ts.copy_(inputs[k][1])
        graph.replay()
        eager = bcq.bcq_int8_gated_backward(dh, *inputs[(k + 1) % 4], wg, cg, wu, cu)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[k])), k
        assert all(torch.equal(a, b) for a, b in zip(eager, want[(k + 1) % 4])), k
    streams = [torch.cuda.Stream() for _ in inputs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = []
        for s, i in zip(streams, inputs):
            with torch.cuda.stream(s):
                got.append(bcq.bcq_int8_gated_backward(dh, *i, wg, cg, wu, cu))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
