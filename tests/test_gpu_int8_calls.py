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
