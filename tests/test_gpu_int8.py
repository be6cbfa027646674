"""The 8-bit operators against their definitions in 64 bits.

Tolerances count roundings: a result in 16 bits is off by half a step of its type (finfo.eps / 2 relative, half the smallest subnormal
step below), an fp32 operation by 2^-24 relative, the hardware's exponential and reciprocal by 2^-23 each.  An error of a
sigmoid's argument counts with the argument's size times 1 - sig.
"""
import math
import os
import subprocess
import sys
import zlib

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

E32 = 2.0 ** -24
TYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def bcq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2510_10467_amd
    return paper_2510_10467_amd


def half_step(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2          # half a subnormal step


def generator(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def codes(rows, n, gen, lo=-127):
    return torch.randint(lo, 128, (rows, n), dtype=torch.int8, device="cuda", generator=gen)


def scales(rows, gen, size):
    return (0.5 + torch.rand(rows, device="cuda", generator=gen)) * size


def guarded(shape, dtype):
    """A tensor with a sentinel either side, and the check that it still stands there."""
    size, pad = math.prod(shape), 4096
    raw = torch.full((size + 2 * pad,), 42, dtype=dtype, device="cuda")
    t = raw[pad:pad + size].view(shape)

    def check():
        assert bool((raw[:pad] == 42).all()) and bool((raw[pad + size:] == 42).all()), "a store landed outside the result"
    return t, check


def close(got, ref, tol, what):
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off; worst {float(((got.double() - ref).abs() / tol).nan_to_num(1e9).max()):.3g} of the tolerance"


def operands(tokens, m, n, gen, mats=1):
    """Codes and scales; projections of a few units, so that both activations are met where they bend."""
    q, ts = codes(tokens, n, gen), scales(tokens, gen, 0.01)
    size = 2.0 / (0.01 * 73 * 73 * math.sqrt(n))
    return q, ts, [(codes(m, n, gen), scales(m, gen, size)) for _ in range(mats)]


def sums64(q, w):
    return q.double() @ w.double().t()


def act64(g, activation):
    """(act, act', sig, z, the derivative of z)"""
    if activation == "silu":
        z, inner = g, torch.ones_like(g)
    else:
        k = math.sqrt(8 / math.pi)
        z, inner = k * (g + 0.044715 * g ** 3), k * (1 + 3 * 0.044715 * g ** 2)
    sig = 1 / (1 + torch.exp(-z))
    return g * sig, sig + g * sig * (1 - sig) * inner, sig, z, inner


# ---------------------------------------------------------------- quantiser

def quantized64(x):
    x = x.double()
    top = x.abs().amax(dim=1)
    finite = top.isfinite()                                     # (rows that the type cannot hold: infinities among them)
    ratio = torch.where((finite & (top > 0))[:, None], 127 * x / top[:, None], 0.0)
    return ratio.round().to(torch.int8), torch.where(finite, top / 127, float("nan"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, n", [(1, 16), (3, 48), (1, 4096), (1025, 2064), (5, 4112), (300, 16384), (2, 28672), (7, 32784), (1, 131056)])
def test_quantize(bcq, dtype, rows, n):
    gen = generator("quantize", rows, n)
    x = torch.randn((rows, n), device="cuda", generator=gen) * torch.exp(4 * torch.randn((rows, 1), device="cuda", generator=gen))
    x = x.to(dtype)
    (q, check_q), (s, check_s) = guarded((rows, n), torch.int8), guarded((rows,), torch.float32)
    got = bcq.bcq_int8_quantize(x, q, s)
    assert got[0] is q and got[1] is s and bcq.last_kernel() == "int8_quantize"
    ref_q, ref_s = quantized64(x)
    check_q(), check_s()
    assert torch.equal(q, ref_q)
    assert torch.equal(s.nan_to_num(-1), ref_s.float().nan_to_num(-1))
    again = bcq.bcq_int8_quantize(x)
    assert torch.equal(again[0], q) and torch.equal(again[1].nan_to_num(-1), s.nan_to_num(-1))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_every_ratio(bcq, dtype):
    """Every mantissa of the largest value against every positive value below it down to where codes are zero: the nearest code, ties to even."""
    mantissas = 1024 if dtype == torch.float16 else 128
    one = 0x3c00 if dtype == torch.float16 else 0x3f80
    tops = torch.arange(one, one + mantissas, device="cuda", dtype=torch.int32)
    low = one - 9 * mantissas                                   # 2^-9
    below = torch.arange(low, one + mantissas, device="cuda", dtype=torch.int32)
    below = below[: below.numel() // 16 * 16 - 16]
    row = torch.minimum(below[None, :], tops[:, None])
    x = torch.cat([row, tops[:, None].expand(-1, 16)], dim=1).to(torch.int16).view(dtype).contiguous()
    q, s = bcq.bcq_int8_quantize(x)
    # whole numbers: 2 * 127 X against (2k + 1) A with x = X 2^-20 exactly
    a, v = (x[:, -1:].double() * 2 ** 20).long(), (x.double() * 2 ** 20).long()
    k = (254 * v + a) // (2 * a)                                # floor(r + 1/2)
    tie = 254 * v == (2 * k - 1) * a
    k = torch.where(tie & (k % 2 == 1), k - 1, k)
    assert bool(tie.any())
    assert torch.equal(q.long(), k)
    q2, _ = bcq.bcq_int8_quantize(-x)
    assert torch.equal(q2, -q)
    assert torch.equal(s, (x[:, -1].double() / 127).float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [8, 1030])
def test_quantize_zero_and_unfit_rows(bcq, dtype, rows):
    gen = generator("unfit", rows)
    x = torch.randn((rows, 512), device="cuda", generator=gen).to(dtype)
    want, want_s = bcq.bcq_int8_quantize(x)
    x[1] = 0
    x[2, 17] = float("nan")
    x[3, 0] = float("inf")
    x[4, 511] = float("-inf")
    x[5] = torch.finfo(dtype).max
    x[5, 3] = -torch.finfo(dtype).max
    x[6] = 0
    least = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps      # the smallest subnormal
    x[6, 8:10] = torch.tensor([least, -3 * least], dtype=dtype, device="cuda")
    q, s = bcq.bcq_int8_quantize(x)
    assert not q[1].any() and s[1] == 0
    for r in (2, 3, 4):
        assert not q[r].any() and s[r].isnan(), r
    assert q[5, 3] == -127 and bool((q[5, 4:] == 127).all()) and s[5] == (x[5, 0].double() / 127).float()
    assert q[6, 8] == 42 and q[6, 9] == -127 and int((q[6] != 0).sum()) == 2
    assert abs(float(s[6].double()) / (3 * least / 127) - 1) <= 2.0 ** -3      # (bfloat16: fp32's own subnormals)
    keep = [0, *range(7, rows)]
    assert torch.equal(q[keep], want[keep]) and torch.equal(s[keep], want_s[keep])


# ---------------------------------------------------------------- forward

# few tokens and tiles of 64, ends of every kind: rows, tokens, columns (16, 32, 48, 64, .. over a step of 128), one to many steps
SIZES = [(1, 1, 16), (1, 16, 32), (2, 40, 48), (5, 17, 64), (16, 100, 112), (15, 1000, 4096), (1, 129, 1040), (3, 33, 14336),
         (17, 1, 16), (17, 40, 48), (33, 64, 128), (64, 65, 144), (77, 101, 1040), (130, 129, 80), (300, 200, 2064), (65, 1000, 272)]
# tall and short matrices with few to many tokens.  (Which kernels these run on is up to the prices; tests/test_gpu_int8_shapes.py has sizes that are held to
# reach every one.)
LARGE_SIZES = [(12, 16400, 144), (20, 8200, 272), (40, 9000, 144), (200, 16400, 144), (129, 20000, 272), (300, 33001, 208), (257, 33024, 1040),
               (500, 28600, 80), (100, 20010, 144), (100, 10001, 272), (40, 33000, 400), (64, 36001, 1040),
               (300, 48100, 80), (500, 47000, 272), (100, 20010, 256), (100, 10001, 1152),
               (100, 8001, 272), (129, 4999, 1040), (70, 5003, 1040), (100, 1000, 272), (200, 300, 144), (150, 1200, 1040), (256, 40, 4112), (40, 50000, 272),
               (100, 40000, 272), (128, 33001, 1040)]
# ... with two matrices
LARGE_GATED = [(20, 4100, 272), (40, 4500, 144), (200, 16400, 144), (300, 16400, 144), (200, 8200, 144), (500, 14300, 80), (100, 10010, 144), (100, 5001, 272),
               (33, 16500, 400), (50, 17001, 1040), (450, 24050, 144), (300, 23501, 80),
               (100, 10010, 256), (100, 5001, 1152), (100, 4001, 272), (70, 2500, 1040), (100, 600, 272), (200, 300, 144), (50, 25001, 400),
               (40, 16600, 144), (66, 16600, 144), (100, 17000, 1040)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens, m, n", SIZES + LARGE_SIZES)
def test_gemm(bcq, dtype, tokens, m, n):
    gen = generator("gemm", tokens, m, n)
    q, ts, [(w, cs)] = operands(tokens, m, n, gen)
    y, check = guarded((tokens, m), dtype)
    assert bcq.bcq_int8_gemm(q, ts, w, cs, dtype, y) is y
    ref = sums64(q, w) * ts.double()[:, None] * cs.double()
    check()
    close(y, ref, ref.abs() * (half_step(dtype) + 4 * E32) + tiny(dtype), "y")
    assert torch.equal(bcq.bcq_int8_gemm(q, ts, w, cs, dtype), y)


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens, m, n", SIZES + LARGE_GATED)
def test_gated(bcq, dtype, activation, tokens, m, n):
    gen = generator("gated", tokens, m, n)
    q, ts, [(wg, cg), (wu, cu)] = operands(tokens, m, n, gen, 2)
    h, check = guarded((tokens, m), dtype)
    assert bcq.bcq_int8_gated(q, ts, wg, cg, wu, cu, activation, dtype, h) is h
    g, u = (sums64(q, w) * ts.double()[:, None] * c.double() for w, c in ((wg, cg), (wu, cu)))
    act, _, _, z, _ = act64(g, activation)
    ref = act * u
    check()
    close(h, ref, ref.abs() * (half_step(dtype) + (16 * z.abs() + 24) * E32) + tiny(dtype) + 1e-35 * (g * u).abs(), "h")


@pytest.mark.parametrize("tokens", [1, 16, 17, 100])
def test_largest_sums(bcq, tokens):
    """The longest rows, of the code whose square is largest: the sum is the largest that the shape rules admit, and exact."""
    n, m = 131056, 33
    q = torch.full((tokens, n), -128, dtype=torch.int8, device="cuda")
    w = torch.full((m, n), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    w[2, 5] = 0
    one_t, one_m = torch.full((tokens,), 2.0 ** -20, device="cuda"), torch.ones(m, device="cuda")
    y = bcq.bcq_int8_gemm(q, one_t, w, one_m, torch.bfloat16)
    ref = sums64(q, w) * 2.0 ** -20
    close(y, ref, ref.abs() * (half_step(torch.bfloat16) + 4 * E32), "y")


@pytest.mark.parametrize("tokens", [4, 40])
def test_a_token_does_not_touch_another(bcq, tokens):
    """A token without numbers (scale NaN or infinite) or with scale 0, and results beyond the type."""
    gen = generator("tokens", tokens)
    q, ts, [(w, cs), (w2, cs2)] = operands(tokens, 70, 160, gen, 2)
    clean, clean_h = bcq.bcq_int8_gemm(q, ts, w, cs), bcq.bcq_int8_gated(q, ts, w, cs, w2, cs2)
    ts2, q2 = ts.clone(), q.clone()
    ts2[1], q2[1] = float("nan"), 0
    ts2[2] = 0
    ts2[3] = 1e30
    y, h = bcq.bcq_int8_gemm(q2, ts2, w, cs), bcq.bcq_int8_gated(q2, ts2, w, cs, w2, cs2)
    for got, want in ((y, clean), (h, clean_h)):
        assert bool(got[1].isnan().all()) and not got[2].any()
        assert bool(got[3].isinf().any())
        others = [0, *range(4, tokens)]
        assert torch.equal(got[others], want[others])
    sums = sums64(q[3:4], w)
    assert torch.equal(y[3:4].sign(), sums.sign().half())


@pytest.mark.parametrize("dtype", TYPES)
def test_a_token_in_batches_of_any_size(bcq, dtype):
    """The same bits for a token alone and among few and many others, whichever kernels and tiles those take."""
    gen = generator("batches")
    q, ts, [(wg, cg), (wu, cu)] = operands(600, 4200, 400, gen, 2)
    calls = [lambda q, ts: bcq.bcq_int8_gemm(q, ts, wg, cg, dtype), *(
        lambda q, ts, act=act: bcq.bcq_int8_gated(q, ts, wg, cg, wu, cu, act, dtype) for act in ("silu", "gelu"))]
    for call in calls:
        whole = call(q, ts)
        for tokens in (1, 5, 12, 30, 33, 64, 100, 200, 300):
            assert torch.equal(call(q[:tokens], ts[:tokens]), whole[:tokens]), tokens


@pytest.mark.parametrize("tokens, m, n", [(1, 256, 512), (40, 300, 512)])
def test_results_of_any_alignment(bcq, tokens, m, n):
    gen = generator("align", tokens)
    q, ts, [(w, cs)] = operands(tokens, m, n, gen)
    want = bcq.bcq_int8_gemm(q, ts, w, cs)
    raw = torch.zeros(tokens * m + 8, dtype=torch.float16, device="cuda")
    for off in (1, 2, 5):
        y = raw[off:off + tokens * m].view(tokens, m)
        raw.zero_()
        bcq.bcq_int8_gemm(q, ts, w, cs, y=y)
        assert torch.equal(y, want) and not raw[:off].any() and not raw[off + tokens * m:].any()


def test_no_tokens(bcq):
    gen = generator("none")
    q, ts, [(w, cs), (w2, cs2)] = operands(4, 24, 64, gen, 2)
    q, ts = q[:0].contiguous(), ts[:0].contiguous()
    assert bcq.bcq_int8_gemm(q, ts, w, cs).shape == (0, 24)
    assert bcq.bcq_int8_gated(q, ts, w, cs, w2, cs2).shape == (0, 24)
    codes_, s = bcq.bcq_int8_quantize(torch.empty((0, 64), dtype=torch.float16, device="cuda"))
    assert codes_.shape == (0, 64) and s.shape == (0,)
    dy = torch.empty((0, 24), dtype=torch.float16, device="cuda")
    torch.full((1000,), float("nan"), device="cuda")            # (something for the allocator to hand out again)
    dx, dc = bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs)
    assert dx.shape == (0, 64) and dc.shape == (24,) and not dc.any()
    dx, dg, du = bcq.bcq_int8_gated_backward(dy, q, ts, w, cs, w2, cs2)
    assert dx.shape == (0, 64) and not dg.any() and not du.any()


# ---------------------------------------------------------------- backward

BACKWARD_SIZES = [(1, 1, 16), (2, 40, 48), (16, 17, 64), (33, 64, 128), (64, 65, 144), (77, 101, 1040), (130, 129, 80), (300, 200, 2064), (65, 1000, 272),
                  (513, 63, 16)]
# each tile of the second product, with the channels in one run and in several
SECOND_SIZES = [(50, 3003, 20000), (300, 1001, 14352), (300, 1001, 4112), (700, 900, 6160)]
SECOND_GATED = [(40, 2000, 14352), (300, 2001, 6160), (129, 1500, 4112), (520, 1001, 14352)]


def second_half_error(err, grads, cs, w, top, norm):
    """What the product of the gradients with the weights adds: `err` in each gradient, the rounding to binary16 (half a step, or half a subnormal
    one at the token's power of two and the scales'), and a chain of fp32 sums of 16 at a time."""
    k = w.shape[0]
    each = (err + grads.abs() * (2.0 ** -11 + 8 * E32)) * cs.abs()
    each = each + (2.0 ** -25 * top / norm)[:, None]
    return each @ w.abs() + (k / 16 + 24) * E32 * ((grads * cs).abs() @ w.abs())


def powers(dy, *cs, ts=None, n=0):
    """The powers of two that the gradients are held at: above all channel scales, and a token's: its largest |dy| to 2^9, or, gated (ts, n), to 2^3
    times what undoes the size of its projections."""
    top = max(float(c.abs().max()) for c in cs)
    top = 2.0 ** (math.floor(math.log2(top)) + 1)
    most = dy.double().abs().amax(dim=1)
    largest = 9 if ts is None else 3
    norm = torch.where(most > 0, torch.exp2(largest - torch.floor(torch.log2(most.clamp_min(1e-300)))), torch.ones_like(most))
    if ts is not None:
        size = (ts.abs() * top) * (torch.tensor(73.0 * 73.0, dtype=torch.float32) * torch.tensor(float(n), dtype=torch.float32).sqrt()).item()
        norm = norm * torch.exp2(-torch.floor(torch.log2(size.double())))
    return top, norm


def sums_error(terms, err, tokens):
    """Of a sum over tokens: the terms' own, and a chain of at most a partial sum per 32 tokens behind a handful."""
    return err.sum(dim=0) + (tokens / 32 + 16) * E32 * terms.abs().sum(dim=0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens, m, n", BACKWARD_SIZES + LARGE_SIZES[3:5] + LARGE_SIZES[7:] + SECOND_SIZES + [(300, 33001, 80), (300, 72, 33040), (100, 2000, 2000)])
def test_gemm_backward(bcq, dtype, tokens, m, n):
    gen = generator("gemm_backward", tokens, m, n)
    q, ts, [(w, cs)] = operands(tokens, m, n, gen)
    dy = (torch.randn((tokens, m), device="cuda", generator=gen) * torch.exp(2 * torch.randn((tokens, 1), device="cuda", generator=gen)) / 64).to(dtype)
    dx, dc = bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs)
    assert dx.dtype == dtype and dx.shape == (tokens, n) and dc.dtype == torch.float32 and dc.shape == (m,)
    d, c, w64 = dy.double(), cs.double(), w.double()
    terms = d * sums64(q, w) * ts.double()[:, None]
    close(dc, terms.sum(dim=0), sums_error(terms, 4 * E32 * terms.abs(), tokens) + 1e-40, "dchannel_scales")
    ref = (d * c) @ w64
    top, norm = powers(dy, cs)
    close(dx, ref, second_half_error(torch.zeros_like(d), d, c, w64, top, norm) + ref.abs() * half_step(dtype) + tiny(dtype), "dx")
    again = bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dc)


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens, m, n", BACKWARD_SIZES + LARGE_GATED[2:] + SECOND_GATED + [(300, 16421, 80), (300, 72, 33040), (100, 1000, 2000)])
def test_gated_backward(bcq, dtype, activation, tokens, m, n):
    gen = generator("gated_backward", tokens, m, n)
    q, ts, [(wg, cg), (wu, cu)] = operands(tokens, m, n, gen, 2)
    dh = (torch.randn((tokens, m), device="cuda", generator=gen) * torch.exp(2 * torch.randn((tokens, 1), device="cuda", generator=gen)) / 64).to(dtype)
    dx, dgate, dup = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu, activation)
    d = dh.double()
    pg, pu = (sums64(q, w) * ts.double()[:, None] for w in (wg, wu))
    g, u = pg * cg.double(), pu * cu.double()
    act, slope, sig, z, inner = act64(g, activation)
    arg = 16 * z.abs() + 24                                     # roundings that an argument's error counts for
    slope_err = E32 * (arg * (sig + g.abs() * sig * (1 - sig) * inner) + 6 * g.abs() * sig * inner)
    dg, du = d * u * slope, d * act
    dg_err, du_err = (d * u).abs() * slope_err + 8 * E32 * dg.abs(), du.abs() * arg * E32
    close(dgate, (dg * pg).sum(dim=0), sums_error(dg * pg, (dg_err + 4 * E32 * dg.abs()) * pg.abs(), tokens) + 1e-40, "dgate_scales")
    close(dup, (du * pu).sum(dim=0), sums_error(du * pu, (du_err + 4 * E32 * du.abs()) * pu.abs(), tokens) + 1e-40, "dup_scales")
    ref = (dg * cg.double()) @ wg.double() + (du * cu.double()) @ wu.double()
    top, norm = powers(dh, cg, cu, ts=ts, n=n)
    tol = second_half_error(dg_err, dg, cg.double(), wg.double(), top, norm) + second_half_error(du_err, du, cu.double(), wu.double(), top, norm)
    close(dx, ref, 1.01 * tol + ref.abs() * half_step(dtype) + tiny(dtype), "dx")
    again = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu, activation)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dgate, dup)))


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens, m, n", [(24, 200, 272), (24, 64, 4112)])
def test_gradients_of_small_and_large_activations(bcq, dtype, activation, tokens, m, n):
    """A token's gradients have the precision of their own size, whatever its activations' is: those of 2^-18 of the others too."""
    gen = generator("small", tokens, m, n)
    q, ts, [(wg, cg), (wu, cu)] = operands(tokens, m, n, gen, 2)
    ts = ts * torch.exp2(torch.arange(tokens, device="cuda") - 18.0)         # 2^-18 .. 2^5
    dh = torch.randn((tokens, m), device="cuda", generator=gen).clamp(-4, 4).to(dtype)
    dx, dgate, dup = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu, activation)
    d = dh.double()
    pg, pu = (sums64(q, w) * ts.double()[:, None] for w in (wg, wu))
    g, u = pg * cg.double(), pu * cu.double()
    act, slope, sig, z, inner = act64(g, activation)
    arg = 16 * z.abs() + 24
    slope_err = E32 * (arg * (sig + g.abs() * sig * (1 - sig) * inner) + 6 * g.abs() * sig * inner)
    dg, du = d * u * slope, d * act
    dg_err, du_err = (d * u).abs() * slope_err + 8 * E32 * dg.abs(), du.abs() * arg * E32
    ref = (dg * cg.double()) @ wg.double() + (du * cu.double()) @ wu.double()
    # a gradient is off by 2^-11 of itself or, far below its token's, by 2^-25 of about the token's size: all together 2^-9 of the root of the squares'
    # sum times the codes' 73, six times over what independent roundings make
    of_token = ((dg * cg.double()).square().sum(dim=1) + (du * cu.double()).square().sum(dim=1)).sqrt() * 73
    assert bool(((dx.double() - ref).abs() <= of_token[:, None] * 2.0 ** -9 + ref.abs() * half_step(dtype) + tiny(dtype)).all())
    top, norm = powers(dh, cg, cu, ts=ts, n=n)
    tol = second_half_error(dg_err, dg, cg.double(), wg.double(), top, norm) + second_half_error(du_err, du, cu.double(), wu.double(), top, norm)
    close(dx, ref, 1.01 * tol + ref.abs() * half_step(dtype) + tiny(dtype), "dx")


def test_gradients_against_differences(bcq):
    """The 64-bit formulas that the other tests use, against differences of the forward formula."""
    gen = generator("differences")
    q, ts, [(wg, cg), (wu, cu)] = operands(5, 7, 32, gen, 2)
    dh = torch.randn((5, 7), device="cuda", generator=gen).double()
    x = q.double() * ts.double()[:, None]

    def loss(x, cg, cu, activation):
        return (act64(x @ wg.double().t() * cg, activation)[0] * (x @ wu.double().t() * cu) * dh).sum()
    for activation in ("silu", "gelu"):
        leaves = [x, cg.double(), cu.double()]
        got = bcq.bcq_int8_gated_backward(dh.half(), q, ts, wg, cg, wu, cu, activation)
        for k, leaf in enumerate(leaves):
            step = 1e-5 * leaf.abs().mean()
            diff = torch.zeros_like(leaf)
            for i in range(leaf.numel()):
                up, down = leaf.clone(), leaf.clone()
                up.view(-1)[i] += step
                down.view(-1)[i] -= step
                args = [[*leaves[:k], v, *leaves[k + 1:]] for v in (up, down)]
                diff.view(-1)[i] = (loss(*args[0], activation) - loss(*args[1], activation)) / (2 * step)
            # (dh is rounded to 11 bits for the call, results to 11 or 24)
            assert float((got[k].double() - diff).norm() / diff.norm()) < 3 * 2.0 ** -11, (activation, k)


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_any_size(bcq, dtype):
    """Gradients near either end of the type's range, zero rows and scales of any size: a token's relative errors stay what they are."""
    gen = generator("range")
    q, ts, [(wg, cg), (wu, cu)] = operands(6, 96, 64, gen, 2)
    base = torch.randn((6, 96), device="cuda", generator=gen).clamp(-4, 4).to(dtype)
    want = bcq.bcq_int8_gated_backward(base, q, ts, wg, cg, wu, cu)[0]
    # a power of two on dy and its inverse on the scales' gradient path changes nothing but the exponent
    for e in ((-8, 4) if dtype == torch.float16 else (-100, 60)):
        dh = (base.float() * 2.0 ** e).to(dtype)
        if not torch.equal(dh.float() * 2.0 ** -e, base.float()):
            continue                                            # (fp16: a subnormal lost bits)
        dx = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu)[0]
        ref = (want.double() * 2.0 ** e)
        close(dx, ref, ref.abs() * half_step(dtype) * 2 + 2 * tiny(dtype), f"2^{e}")
    dh = base.clone()
    dh[2] = 0
    dx, dgate, dup = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu)
    assert not dx[2].any()
    keep = [0, 1, 3, 4, 5]
    assert torch.equal(dx[keep], want[keep])
    dh[3, 7] = float("nan")
    dx, dgate, dup = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu)
    assert bool(dx[3].isnan().all()) and torch.equal(dx[[0, 1, 4, 5]], want[[0, 1, 4, 5]])
    assert bool(dgate[7].isnan()) and int(dgate.isnan().sum()) == 1 and int(dup.isnan().sum()) == 1


# ---------------------------------------------------------------- as they are used

def test_a_feed_forward_block(bcq):
    """Activations in, through gate, up and down at 8 bits, and back: against the same chain in 64 bits on the same codes."""
    gen = generator("block")
    tokens, hidden, ffn = 90, 512, 1376
    x = torch.randn((tokens, hidden), device="cuda", generator=gen).half()
    quantized = [bcq.bcq_int8_quantize((torch.randn((r, c), device="cuda", generator=gen) * 0.05).half()) for r, c in ((ffn, hidden), (ffn, hidden), (hidden, ffn))]
    (wg, cg), (wu, cu), (wd, cd) = quantized
    q, ts = bcq.bcq_int8_quantize(x)
    h = bcq.bcq_int8_gated(q, ts, wg, cg, wu, cu)
    hq, hs = bcq.bcq_int8_quantize(h)
    y = bcq.bcq_int8_gemm(hq, hs, wd, cd)
    g, u = (sums64(q, w) * ts.double()[:, None] * c.double() for w, c in ((wg, cg), (wu, cu)))
    act, slope, *_ = act64(g, "silu")
    assert float((h.double() - act * u).norm() / (act * u).norm()) < 2.0 ** -11
    h64 = hq.double() * hs.double()[:, None]
    assert float((h64 - act * u).norm() / (act * u).norm()) < 0.05              # (what 8 bits keep)
    ref = h64 @ (wd.double() * cd.double()[:, None]).t()
    assert float((y.double() - ref).norm() / ref.norm()) < 2.0 ** -11
    dy = torch.randn_like(y)
    dh, dcd = bcq.bcq_int8_gemm_backward(dy, hq, hs, wd, cd)
    dx, dcg, dcu = bcq.bcq_int8_gated_backward(dh, q, ts, wg, cg, wu, cu)
    dh64 = (dy.double() * cd.double()) @ wd.double()
    dg64, du64 = dh64 * u * slope, dh64 * act
    want = [(dh, dh64), (dcd, (dy.double() * (h64 @ wd.double().t())).sum(0)),
            (dx, (dg64 * cg.double()) @ wg.double() + (du64 * cu.double()) @ wu.double()),
            (dcg, (dg64 * g / cg.double()).sum(0)), (dcu, (du64 * u / cu.double()).sum(0))]
    for k, (got, ref) in enumerate(want):                       # two roundings to 11 bits and one result's
        assert float((got.double() - ref).norm() / ref.norm()) < 3 * 2.0 ** -11, k


def test_graph_and_streams(bcq):
    """One token through the block and a backward pass, recorded, replayed with eager work between, and on a stream of one's own."""
    gen = generator("graph")
    xs = [torch.randn((t, 256), device="cuda", generator=gen).half() for t in (1, 1, 40, 40)]
    wg, cg = bcq.bcq_int8_quantize(torch.randn((96, 256), device="cuda", generator=gen).half())
    wu, cu = bcq.bcq_int8_quantize(torch.randn((96, 256), device="cuda", generator=gen).half())

    def forward(x):
        q, s = bcq.bcq_int8_quantize(x)
        return q, s, bcq.bcq_int8_gated(q, s, wg, cg, wu, cu, "gelu")

    def everything(x):
        q, s, h = forward(x)
        return [h, *bcq.bcq_int8_gated_backward(h, q, s, wg, cg, wu, cu, "gelu"), *bcq.bcq_int8_gemm_backward(h, q, s, wg, cg)]
    for first, second in ((0, 1), (2, 3)):
        want = [[t.clone() for t in everything(xs[k])] for k in (first, second)]
        x = xs[first].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = everything(x)
        other = torch.cuda.CUDAGraph()
        with torch.cuda.graph(other):
            out2 = everything(x)
        for k in (0, 1, 0, 1):
            x.copy_(xs[(first, second)[k]])
            graph.replay()
            everything(xs[3])                                   # eager work of the same operators
            other.replay()
            torch.cuda.synchronize()
            for got, got2, ref in zip(out, out2, want[k]):
                assert torch.equal(got, ref) and torch.equal(got2, ref)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            got = everything(xs[first])
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[0]))


# ---------------------------------------------------------------- far ends, the host code, refusals

@pytest.mark.parametrize("tokens", [3, 40])
def test_weights_beyond_four_gigabytes(bcq, tokens):
    gen = generator("far weights", tokens)
    m, n = 70001, 65536
    w, cs = torch.empty((m, n), dtype=torch.int8, device="cuda"), scales(m, gen, 0.01)
    w.random_(-127, 128, generator=gen)
    q, ts = codes(tokens, n, gen), scales(tokens, gen, 1e-4)
    far = slice(m - 300, m)
    ref = lambda w, c: sums64(q, w) * ts.double()[:, None] * c.double()                 # noqa: E731
    y = bcq.bcq_int8_gemm(q, ts, w, cs)
    for part in (slice(0, 200), far):
        want = ref(w[part], cs[part])
        close(y[:, part], want, want.abs() * (half_step(torch.float16) + 4 * E32) + tiny(torch.float16), "y")
    dy = torch.zeros((tokens, m), dtype=torch.float16, device="cuda")                   # only the far channels count
    dy[:, far] = torch.randn((tokens, 300), device="cuda", generator=gen).half()
    dx, dc = bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs)
    d, c, wf = dy[:, far].double(), cs[far].double(), w[far].double()
    top, norm = powers(dy, cs)
    close(dx, (d * c) @ wf, second_half_error(torch.zeros_like(d), d, c, wf, top, norm) + ((d * c) @ wf).abs() * half_step(torch.float16) + 1e-6, "dx")
    terms = d * sums64(q, w[far]) * ts.double()[:, None]
    close(dc[far], terms.sum(dim=0), sums_error(terms, 4 * E32 * terms.abs(), tokens) + 1e-40, "dchannel_scales")
    assert not dc[: m - 300].any()


def test_tokens_and_results_beyond_four_gigabytes(bcq):
    gen = generator("far tokens")
    tokens, m, n = 70003, 16, 65536
    x = torch.empty((tokens, n), dtype=torch.float16, device="cuda")
    x.normal_(generator=gen)
    q, ts = bcq.bcq_int8_quantize(x)
    ref_q, ref_s = quantized64(x[-500:])
    assert torch.equal(q[-500:], ref_q) and torch.equal(ts[-500:], ref_s.float())
    del x
    w, cs = codes(m, n, gen), scales(m, gen, 0.01)
    y = bcq.bcq_int8_gemm(q, ts, w, cs)
    want = sums64(q[-300:], w) * ts[-300:].double()[:, None] * cs.double()
    close(y[-300:], want, want.abs() * (half_step(torch.float16) + 4 * E32) + tiny(torch.float16), "y")
    dx, _ = bcq.bcq_int8_gemm_backward(y, q, ts, w, cs)
    d = y[-300:].double()
    want = (d * cs.double()) @ w.double()
    top, norm = powers(y[-300:], cs)
    close(dx[-300:], want, second_half_error(torch.zeros_like(d), d, cs.double(), w.double(), top, norm) + want.abs() * half_step(torch.float16) + tiny(torch.float16), "dx")
    del dx, q, y
    m, n = 65537, 16
    q, ts, [(w, cs)] = operands(tokens, m, n, gen)
    y = bcq.bcq_int8_gemm(q, ts, w, cs)
    want = sums64(q[-300:], w) * ts[-300:].double()[:, None] * cs.double()
    close(y[-300:], want, want.abs() * (half_step(torch.float16) + 4 * E32) + tiny(torch.float16), "y")


HOST_CALLS = ("int8_quantize", "int8_gemm", "int8_gated", "int8_gemm_backward", "int8_gated_backward")


def test_the_host_code_and_the_python_code_agree(bcq, monkeypatch):
    """What the native code takes it answers as the Python code behind it does, and what it does not take is refused the same way."""
    from paper_2510_10467_amd import binding
    bcq.lib()
    native = binding._host
    assert native.__name__.endswith("_bcq_host"), "the host code is not loaded"
    declines = type("Declines", (), {name: staticmethod(lambda *a: None) for name in HOST_CALLS})
    gen = generator("host")
    q, ts, [(w, cs), (w2, cs2)] = operands(5, 24, 64, gen, 2)
    x, dy = torch.randn((5, 64), device="cuda", generator=gen).half(), torch.randn((5, 24), device="cuda", generator=gen).bfloat16()
    y, s5 = torch.empty((5, 24), dtype=torch.bfloat16, device="cuda"), torch.empty(5, device="cuda")
    good = [lambda: bcq.bcq_int8_quantize(x), lambda: bcq.bcq_int8_quantize(x.bfloat16(), scales=s5), lambda: (bcq.bcq_int8_gemm(q, ts, w, cs),),
            lambda: (bcq.bcq_int8_gemm(q, ts, w, cs, torch.bfloat16, y),), lambda: (bcq.bcq_int8_gated(q, ts, w, cs, w2, cs2),),
            lambda: (bcq.bcq_int8_gated(q, ts, w, cs, w2, cs2, "gelu", torch.bfloat16, h=y),),
            lambda: (bcq.bcq_int8_gemm(q[:0].contiguous(), ts[:0].contiguous(), w, cs),),
            lambda: bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs), lambda: bcq.bcq_int8_gated_backward(dy, q, ts, w, cs, w2, cs2),
            lambda: bcq.bcq_int8_gated_backward(dy.half(), q, ts, w, cs, w2, cs2, "gelu")]
    wide = torch.zeros((5, 128), dtype=torch.int8, device="cuda")
    odd = torch.zeros(5 * 64 + 16, dtype=torch.int8, device="cuda")[1:1 + 5 * 64].view(5, 64)
    refused = [lambda: bcq.bcq_int8_quantize(x.cpu()), lambda: bcq.bcq_int8_quantize(x.float()), lambda: bcq.bcq_int8_quantize(x[0]),
               lambda: bcq.bcq_int8_quantize(x[:, :40].contiguous()), lambda: bcq.bcq_int8_quantize(x[:, :32]), lambda: bcq.bcq_int8_quantize(x, q=wide),
               lambda: bcq.bcq_int8_quantize(x, q=x), lambda: bcq.bcq_int8_quantize(x, q=odd),
               lambda: bcq.bcq_int8_gemm(wide[:, ::2], ts, w, cs), lambda: bcq.bcq_int8_gemm(wide, ts, w, cs), lambda: bcq.bcq_int8_gemm(odd, ts, w, cs),
               lambda: bcq.bcq_int8_gemm(q, ts[:4], w, cs), lambda: bcq.bcq_int8_gemm(q, ts.double(), w, cs), lambda: bcq.bcq_int8_gemm(q, ts, w, cs[:5]),
               lambda: bcq.bcq_int8_gemm(q, ts, w, cs.cpu()), lambda: bcq.bcq_int8_gemm(q, ts, w, cs, torch.float32), lambda: bcq.bcq_int8_gemm(q, ts, w, cs, y=y),
               lambda: bcq.bcq_int8_gemm(q, ts, w.half(), cs), lambda: bcq.bcq_int8_gemm(q, ts, w[0], cs),
               lambda: bcq.bcq_int8_gemm(q[:, :40].contiguous(), ts, w[:, :40].contiguous(), cs),
               lambda: bcq.bcq_int8_gated(q, ts, w, cs, w2, cs2, "relu"), lambda: bcq.bcq_int8_gated(q, ts, w, cs, w2[:20], cs2),
               lambda: bcq.bcq_int8_gated(q, ts, w, cs, w2, cs2, dtype=torch.int8), lambda: bcq.bcq_int8_gated(q, ts, w, cs, w2, cs2, h=y),
               lambda: bcq.bcq_int8_gemm_backward(dy.float(), q, ts, w, cs), lambda: bcq.bcq_int8_gemm_backward(dy[:4], q, ts, w, cs),
               lambda: bcq.bcq_int8_gemm_backward(dy.cpu(), q, ts, w, cs), lambda: bcq.bcq_int8_gemm_backward(dy[:, ::2], q, ts, w[::2], cs[::2]),
               lambda: bcq.bcq_int8_gated_backward(dy, q, ts, w, cs, w2, cs2, "tanh"), lambda: bcq.bcq_int8_gated_backward(dy, q, ts, w, cs, w2, cs2[:3])]

    def outcome(call):
        try:
            return [t.clone() for t in call()]
        except Exception as e:                  # noqa: BLE001  (whatever it is: it has to be the same)
            return type(e), str(e)
    for k, call in enumerate(good + refused):
        monkeypatch.setattr(binding, "_host", declines)
        want = outcome(call)
        made = []

        def recording(name):
            def f(*args):
                done = getattr(native, name)(*args)
                made.append(done is not None)
                return done
            return staticmethod(f)
        monkeypatch.setattr(binding, "_host", type("Recording", (), {name: recording(name) for name in HOST_CALLS}))
        got = outcome(call)
        if k < len(good):
            assert made == [True] and all(torch.equal(a, b) and a.dtype == b.dtype for a, b in zip(got, want)), k
        else:
            assert got == want and isinstance(want, tuple) and True not in made, (k, got, want)


def test_first_calls_recorded(bcq):
    """Kernels that nothing has run yet in a process may be recorded at once."""
    code = """
import torch, paper_2510_10467_amd as bcq
bcq.lib()
q, w = (torch.randint(-127, 128, s, dtype=torch.int8, device="cuda") for s in ((70, 512), (2050, 512)))
ts, cs, dy = torch.rand(70, device="cuda"), torch.rand(2050, device="cuda"), torch.randn((70, 2050), device="cuda").half()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    out = [bcq.bcq_int8_gemm(q, ts, w, cs), bcq.bcq_int8_gated(q, ts, w, cs, w, cs), *bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs)]
for _ in range(3):
    g.replay()
    torch.cuda.synchronize()
    want = [bcq.bcq_int8_gemm(q, ts, w, cs), bcq.bcq_int8_gated(q, ts, w, cs, w, cs), *bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs)]
    assert all(torch.equal(a, b) for a, b in zip(out, want))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-2000:]
