"""Every kernel of the 8-bit products, with every buffer of its rings filled more than twice, against the definitions in 64 bits.

tests/test_int8_shapes.py (no GPU needed) holds the sizes to that: which kernels they run on changes with the prices that choose them.
"""
import pytest

from tests.test_gpu_int8 import E32, act64, close, generator, guarded, half_step, operands, sums64, sums_error, tiny
from tests.test_gpu_int8_scales import gated64, gradients_error

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# (tokens, m, n).  Streamed rows, of 8, 16, 32 and 64 tokens, of one block of rows and two
GEMM_SIZES = [(1, 18, 3392), (9, 17, 4064), (195, 307, 3264), (66, 1371, 3488), (12, 17125, 3104), (19, 8935, 2208),
              # tiles: 64 x 32, 64 x 64, 128 x 64 in both kinds of steps, 128 x 128, 192 x 64, 192 x 128, 256 x 64, 256 x 128, 256 x 256 and these with 256 x 128
              (293, 17, 3184), (622, 817, 2064), (20, 17669, 1664), (19, 20330, 1632), (71, 17782, 1200), (39, 40107, 1312), (76, 32796, 1248),
              (145, 16519, 1136), (134, 31628, 800), (529, 14775, 528), (386, 32997, 816),
              # the same with rows in pieces of 16 bytes
              (35, 40008, 1296), (134, 31640, 800), (387, 32968, 800)]
GATED_SIZES = [(2, 18, 3168), (11, 17, 3088), (156, 403, 3152), (37, 2063, 3360),
               (276, 19, 3392), (33, 4369, 2192), (17, 9178, 1664), (23, 8665, 1616), (73, 10318, 1040), (36, 18883, 1424), (69, 21886, 1040),
               (19, 27595, 1200), (134, 13298, 976), (1524, 2724, 528), (150, 40213, 816),
               (36, 18888, 1424), (134, 13304, 976), (150, 40208, 816)]
# the first halves' tiles, from 64 x 32 on, and the second product's, each with the channels in one run and in several
GEMM_BACKWARD_SIZES = [(1, 18, 3264), (34, 8972, 2496), (2, 16524, 1664), (1, 17247, 1760), (90, 17478, 1088), (39, 33643, 1344), (66, 34868, 1312),
                       (2, 49222, 1168), (137, 29687, 832), (141, 45837, 608), (263, 49542, 816),
                       (76, 403, 9136), (1, 6326, 1504), (401, 752, 8800), (1, 2563, 10912), (847, 525, 4640), (130, 3528, 5824), (376, 1027, 2256), (1, 16744, 32),
                       (1030, 72, 80), (1025, 66, 48)]
GATED_BACKWARD_SIZES = [(2, 18, 3360), (199, 1185, 2128), (1, 8897, 1664), (1, 8970, 1552), (66, 9858, 1072), (38, 16812, 1360), (81, 17313, 1200),
                        (1, 26228, 1088), (65, 27295, 928), (131, 23564, 576), (135, 33005, 816),
                        (75, 236, 9200), (1, 436, 10912), (663, 257, 5440), (1, 1556, 9744), (490, 265, 8544), (132, 1057, 8464), (1561, 564, 624), (1, 8596, 32),
                        (1030, 72, 80), (1025, 66, 48)]


@pytest.fixture(scope="module")
def bcq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2510_10467_amd
    return paper_2510_10467_amd


def kernel_name(bcq, m, n, tokens, matrices):
    return "int8_rows" if bcq.int8_layout(m, n, tokens, matrices)["kernel"] == "rows" else "int8_tile"


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens, m, n", GEMM_SIZES)
def test_gemm(bcq, dtype, tokens, m, n):
    gen = generator("shapes gemm", tokens, m, n)
    q, ts, [(w, cs)] = operands(tokens, m, n, gen)
    y, check = guarded((tokens, m), dtype)
    bcq.bcq_int8_gemm(q, ts, w, cs, dtype, y)
    assert bcq.last_kernel() == kernel_name(bcq, m, n, tokens, 1)
    ref = sums64(q, w) * ts.double()[:, None] * cs.double()
    check()
    close(y, ref, ref.abs() * (half_step(dtype) + 4 * E32) + tiny(dtype), "y")
    assert torch.equal(bcq.bcq_int8_gemm(q, ts, w, cs, dtype), y)


@pytest.mark.parametrize("activation, dtype", [("silu", torch.bfloat16), ("gelu", torch.float16)])
@pytest.mark.parametrize("tokens, m, n", GATED_SIZES)
def test_gated(bcq, dtype, activation, tokens, m, n):
    gen = generator("shapes gated", tokens, m, n)
    q, ts, [(wg, cg), (wu, cu)] = operands(tokens, m, n, gen, 2)
    h, check = guarded((tokens, m), dtype)
    bcq.bcq_int8_gated(q, ts, wg, cg, wu, cu, activation, dtype, h)
    assert bcq.last_kernel() == kernel_name(bcq, m, n, tokens, 2)
    g, u = (sums64(q, w) * ts.double()[:, None] * c.double() for w, c in ((wg, cg), (wu, cu)))
    act, _, _, z, _ = act64(g, activation)
    ref = act * u
    check()
    close(h, ref, ref.abs() * (half_step(dtype) + (16 * z.abs() + 24) * E32) + tiny(dtype) + 1e-35 * (g * u).abs(), "h")
    assert torch.equal(bcq.bcq_int8_gated(q, ts, wg, cg, wu, cu, activation, dtype), h)


def gradient(tokens, m, gen, dtype):
    return (torch.randn((tokens, m), device="cuda", generator=gen) * torch.exp(2 * torch.randn((tokens, 1), device="cuda", generator=gen)) / 64).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens, m, n", GEMM_BACKWARD_SIZES)
def test_gemm_backward(bcq, dtype, tokens, m, n):
    gen = generator("shapes gemm backward", tokens, m, n)
    q, ts, [(w, cs)] = operands(tokens, m, n, gen)
    dy = gradient(tokens, m, gen, dtype)
    dx, dc = bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs)
    d, c = dy.double(), cs.double()
    ref = (d * c) @ w.double()
    close(dx, ref, gradients_error([(d * c, 2 * E32 * (d * c).abs())], [w]) + ref.abs() * half_step(dtype) + tiny(dtype), "dx")
    terms = d * sums64(q, w) * ts.double()[:, None]
    close(dc, terms.sum(dim=0), sums_error(terms, 4 * E32 * terms.abs(), tokens) + 1e-40, "dchannel_scales")
    again = bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dc)


@pytest.mark.parametrize("activation, dtype", [("gelu", torch.bfloat16), ("silu", torch.float16)])
@pytest.mark.parametrize("tokens, m, n", GATED_BACKWARD_SIZES)
def test_gated_backward(bcq, dtype, activation, tokens, m, n):
    """Of every fifth token the gates are all shut: its gradients are made a second time."""
    gen = generator("shapes gated backward", tokens, m, n)
    q, ts, [(wg, cg), (wu, cu)] = operands(tokens, m, n, gen, 2)
    q[::5] = q[::5].abs().clamp_min(60)
    wg = torch.where(torch.rand((m, n), device="cuda", generator=gen) < 0.5, -wg.abs(), wg)
    g = sums64(q[::5], wg) * ts[::5].double()[:, None] * cg.double()
    ts[::5] = (ts[::5].double() * ((-24.0 if activation == "silu" else -5.0) / g.amin(dim=1))).float()
    dh = gradient(tokens, m, gen, dtype)
    got = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu, activation)
    want, tol = gated64(dh, q, ts, wg, cg, wu, cu, activation)
    close(got[0], want[0], tol[0] + want[0].abs() * half_step(dtype) + tiny(dtype), "dx")
    close(got[1], want[1], tol[1], "dgate_scales")
    close(got[2], want[2], tol[2], "dup_scales")
    again = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu, activation)
    assert all(torch.equal(a, b) for a, b in zip(again, got))
