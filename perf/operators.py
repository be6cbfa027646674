"""The 8-bit operators that are timed: what a serving process and a scale-tuning program ask of this library beside its bit-plane products.

A case is one call:

  quantize        ``bcq_int8_quantize``: rows of activations to 8-bit codes and a scale per row
  gemm            ``bcq_int8_gemm``: codes of tokens times codes of weights, a scale per token and one per output channel
  gemm_backward   ``bcq_int8_gemm_backward``: gradients of the activations and of the channel scales, the codes being fixed
  gated           ``bcq_int8_gated``: gate and up projections, the activation and the product of both
  gated_backward  ``bcq_int8_gated_backward``: gradients of the activations and of both sets of channel scales

Where ``own`` is false, ``run`` computes the same in elementary torch operations in 32 bits.  Layer sizes are those of the
Llama-3-8B, Phi-4-14B and Llama-3-70B linear layers that the benchmark and the tests use, and odd ones.  Distributions: normal
activations with some large columns, weights with a spread per row and a few large entries, small normal gradients.
"""
import math

import torch

own = False

TYPES = {"float16": torch.float16, "bfloat16": torch.bfloat16}
MOST_FLOPS = 2.0 * 28672 * 8192 * 2048          # the largest listed cases
MOST_QUANTIZED = 4096 * 14336
GELU = 0.7978845608028654                       # sqrt(2 / pi)


def _case(kind, tokens, m, n, dtype, activation="silu"):
    case = {"kind": kind, "tokens": tokens, "n": n, "dtype": dtype}
    if kind != "quantize":
        case["m"] = m
    if kind.startswith("gated"):
        case["activation"] = activation
    return case


def listed():
    return [
        # one token's activations on the way into a decoder block: launch and host latency
        dict(_case("quantize", 1, 0, 4096, "float16"), name="quantize_1"),
        # a long prompt's activations on the way into the down projection
        dict(_case("quantize", 4096, 0, 14336, "bfloat16"), name="quantize_4096"),
        # one token through the smallest projection
        dict(_case("gemm", 1, 1024, 4096, "float16"), name="gemm_kv_1"),
        # a server's decoding batch through the down projection
        dict(_case("gemm", 16, 4096, 14336, "bfloat16"), name="gemm_down_16"),
        # a short prompt, sizes that no tile divides
        dict(_case("gemm", 77, 5003, 5136, "float16"), name="gemm_ragged_77"),
        # a long prompt on the largest layer
        dict(_case("gemm", 2048, 28672, 8192, "float16"), name="gemm_70b_2048"),
        # one token through the feed-forward block, the decoding loop of a single user
        dict(_case("gated", 1, 14336, 4096, "float16"), name="gated_1"),
        # a large decoding batch, the other activation
        dict(_case("gated", 48, 17920, 5120, "bfloat16", "gelu"), name="gated_48"),
        # a long prompt
        dict(_case("gated", 2048, 14336, 4096, "float16"), name="gated_2048"),
        # a calibration batch through the down projection, backwards
        dict(_case("gemm_backward", 512, 4096, 14336, "bfloat16"), name="gemm_backward_512"),
        # a small calibration batch, sizes that no tile divides
        dict(_case("gated_backward", 133, 1001, 2064, "float16", "gelu"), name="gated_backward_ragged_133"),
        # a full calibration batch of the feed-forward block, backwards
        dict(_case("gated_backward", 2048, 14336, 4096, "bfloat16"), name="gated_backward_2048"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("quantize", "gemm", "gemm", "gemm", "gated", "gated", "gemm_backward", "gated_backward"))
    dtype, activation = rng.choice(("float16", "bfloat16")), rng.choice(("silu", "gelu"))
    n = 16 * _log_uniform(rng, 16, 1792)
    if rng.random() < 0.5:
        n = -(-n // 512) * 512
    if kind == "quantize":
        return _case(kind, min(_log_uniform(rng, 1, 8192), MOST_QUANTIZED // n), 0, n, dtype)
    m = _log_uniform(rng, 200, 28672)
    if rng.random() < 0.5:
        m = -(-m // 256) * 256
    if m * n > 28672 * 8192:
        m = 28672 * 8192 // n
    if kind != "gemm" and m * n > 14336 * 8192:
        m = 14336 * 8192 // n
    tokens = _log_uniform(rng, 16 if "backward" in kind else 1, 4096)
    each = {"gemm": 2.0, "gated": 4.0, "gemm_backward": 4.0, "gated_backward": 8.0}[kind] * m * n
    return _case(kind, max(1, min(tokens, int(MOST_FLOPS // each))), m, n, dtype, activation)


def _codes(values):
    """Rows to codes and scales, as a program has them of its weights and of the activations in hand."""
    top = values.abs().amax(dim=1)
    return torch.round(values * (127.0 / top)[:, None]).to(torch.int8), top / 127.0


def _weights(m, n, gen):
    codes, scales = torch.empty((m, n), dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    for r in range(0, m, 8192):
        rows = min(8192, m - r)
        w = torch.randn((rows, n), device="cuda", generator=gen) * 0.02
        w *= torch.exp(0.25 * torch.randn((rows, 1), device="cuda", generator=gen))
        w = torch.where(torch.rand((rows, n), device="cuda", generator=gen) < 1.0 / 256.0, 6.0 * w, w)
        codes[r:r + rows], scales[r:r + rows] = _codes(w)
    return codes, scales


def _activations(tokens, n, gen):
    large = torch.where(torch.rand(n, device="cuda", generator=gen) < 1.0 / 128.0, 8.0, 1.0)
    return torch.randn((tokens, n), device="cuda", generator=gen) * large


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    x = _activations(case["tokens"], case["n"], gen)
    if case["kind"] == "quantize":
        return {"case": case, "x": x.to(dtype)}
    s = {"case": case, "dtype": dtype}
    s["q"], s["q_scales"] = _codes(x)
    s["w"], s["w_scales"] = _weights(case["m"], case["n"], gen)
    if case["kind"].startswith("gated"):
        s["up"], s["up_scales"] = _weights(case["m"], case["n"], gen)
    if case["kind"].endswith("backward"):
        s["dy"] = (torch.randn((case["tokens"], case["m"]), device="cuda", generator=gen) / 256.0).to(dtype)
    return s


def _act(g, activation):
    """The activation and its derivative: g sig(g), or g sig(2 k (g + 0.044715 g^3))."""
    if activation == "silu":
        sig = torch.sigmoid(g)
        return g * sig, sig * (1.0 + g * (1.0 - sig))
    sig = torch.sigmoid(2.0 * GELU * (g + 0.044715 * g * g * g))
    return g * sig, sig + g * sig * (1.0 - sig) * (2.0 * GELU * (1.0 + 3.0 * 0.044715 * g * g))


def _plain(s):
    """The operators in elementary operations, in 32 bits."""
    kind = s["case"]["kind"]
    if kind == "quantize":
        x = s["x"].float()
        top = x.abs().amax(dim=1)
        codes = torch.round(x * 127.0 / top[:, None])           # (a product of 18 bits, exact)
        codes = torch.where(top[:, None] > 0, codes, torch.zeros_like(codes)).to(torch.int8)
        scales = top / 127.0
        return {"values": codes * scales[:, None], "scales": scales}
    q, w, dtype = s["q"].float(), s["w"].float(), s["dtype"]
    rows = q @ w.t() * s["q_scales"][:, None]                   # all but the channel's scale
    if kind == "gemm":
        return (rows * s["w_scales"]).to(dtype)
    if kind == "gemm_backward":
        dy = s["dy"].float()
        return {"dx": (dy * s["w_scales"] @ w).to(dtype), "dscales": (dy * rows).sum(dim=0)}
    up = s["up"].float()
    up_rows = q @ up.t() * s["q_scales"][:, None]
    act, slope = _act(rows * s["w_scales"], s["case"]["activation"])
    if kind == "gated":
        return (act * (up_rows * s["up_scales"])).to(dtype)
    dh = s["dy"].float()
    dgate, dup = dh * (up_rows * s["up_scales"]) * slope, dh * act
    dx = dgate * s["w_scales"] @ w + dup * s["up_scales"] @ up
    return {"dx": dx.to(dtype), "dgate_scales": (dgate * rows).sum(dim=0), "dup_scales": (dup * up_rows).sum(dim=0)}


def _own(s):
    """The library's calls."""
    import paper_2510_10467_amd as bcq
    case = s["case"]
    if case["kind"] == "quantize":
        codes, scales = bcq.bcq_int8_quantize(s["x"])
        return {"values": codes * scales[:, None], "scales": scales}
    if case["kind"] == "gemm":
        return bcq.bcq_int8_gemm(s["q"], s["q_scales"], s["w"], s["w_scales"], s["dtype"])
    if case["kind"] == "gated":
        return bcq.bcq_int8_gated(s["q"], s["q_scales"], s["w"], s["w_scales"], s["up"], s["up_scales"], case["activation"], s["dtype"])
    if case["kind"] == "gemm_backward":
        dx, dscales = bcq.bcq_int8_gemm_backward(s["dy"], s["q"], s["q_scales"], s["w"], s["w_scales"])
        return {"dx": dx, "dscales": dscales}
    dx, dgate, dup = bcq.bcq_int8_gated_backward(s["dy"], s["q"], s["q_scales"], s["w"], s["w_scales"], s["up"], s["up_scales"], case["activation"])
    return {"dx": dx, "dgate_scales": dgate, "dup_scales": dup}


def run(state):
    return _own(state) if own else _plain(state)


def exact(case, seed):
    """From the definitions, in 64 bits, a block of output channels at a time."""
    s = prepare(case, seed)
    kind, t = case["kind"], case["tokens"]
    if kind == "quantize":
        x = s["x"].double()
        scales = x.abs().max(dim=1).values / 127.0
        ratio = torch.where(scales[:, None] > 0, 127.0 * x / x.abs().max(dim=1, keepdim=True).values, 0.0)
        return {"values": ratio.round() * scales[:, None], "scales": scales}
    x = s["q"].double() * s["q_scales"].double()[:, None]       # the activations that the codes stand for
    out = torch.empty((t, case["m"]), dtype=torch.float64, device="cuda")
    dx = torch.zeros((t, case["n"]), dtype=torch.float64, device="cuda")
    dw, du = (torch.empty(case["m"], dtype=torch.float64, device="cuda") for _ in range(2))
    for r in range(0, case["m"], 2048):
        part = slice(r, r + 2048)
        w = s["w"][part].double()
        p, cw = x @ w.t(), s["w_scales"][part].double()
        if kind == "gemm":
            out[:, part] = p * cw
            continue
        if kind == "gemm_backward":
            dy = s["dy"][:, part].double()
            dw[part] = (dy * p).sum(dim=0)
            dx += (dy * cw) @ w
            continue
        v = s["up"][part].double()
        o, cu = x @ v.t(), s["up_scales"][part].double()
        g, u = p * cw, o * cu
        if case["activation"] == "silu":
            sig = 1.0 / (1.0 + torch.exp(-g))
            inner = torch.ones_like(g)                          # the derivative of what the sigmoid is taken of
        else:
            sig = 1.0 / (1.0 + torch.exp(-math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3)))
            inner = math.sqrt(8.0 / math.pi) * (1.0 + 0.134145 * g ** 2)
        if kind == "gated":
            out[:, part] = g * sig * u
            continue
        dh = s["dy"][:, part].double()
        dgate, dup = dh * u * (sig + g * sig * (1.0 - sig) * inner), dh * g * sig
        dw[part], du[part] = (dgate * p).sum(dim=0), (dup * o).sum(dim=0)
        dx += (dgate * cw) @ w + (dup * cu) @ v
    if not kind.endswith("backward"):
        return out
    return {"dx": dx, "dscales": dw} if kind == "gemm_backward" else {"dx": dx, "dgate_scales": dw, "dup_scales": du}


def work(case):
    """Each input read once, each output written once; a multiplication and an addition for each weight that a token meets."""
    t, n, kind = case["tokens"], case["n"], case["kind"]
    if kind == "quantize":
        return {"bytes": 3 * t * n + 4 * t, "flops": 2 * t * n}
    m = case["m"]
    mats = 2 if kind.startswith("gated") else 1
    nbytes = t * n + 4 * t + mats * (m * n + 4 * m) + 2 * t * m
    if kind.endswith("backward"):                               # a product for the scales' gradients and one for the activations'
        return {"bytes": nbytes + 2 * t * n + 4 * mats * m, "flops": 4 * mats * t * m * n}
    return {"bytes": nbytes, "flops": 2 * mats * t * m * n}
