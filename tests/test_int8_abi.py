"""The 8-bit operators' argument checks, which need no GPU: bad arguments are refused before anything is enqueued."""
import pytest

Q, TS, W, CS, Y, WS = 0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0x10000
F16, BF16 = 0, 1
OK, NULL, SHAPE, ALIGN, TYPE, WORKSPACE = 0, -1, -3, -4, -7, -8


@pytest.fixture(scope="module")
def lib():
    from paper_2510_10467_amd import build as hip_build
    if hip_build.is_stale():
        hip_build.build()
    import paper_2510_10467_amd as bcq
    return bcq.lib()


def changed(args, **by):
    return [by.get(k, v) for k, v in args.items()]


# the shapes that every entry point refuses: (m, n, tokens)
BAD_SHAPES = [(0, 64, 4), (-1, 64, 4), (8, 0, 4), (8, 8, 4), (8, 40, 4), (8, 131072, 4), (8, 131064, 4), (8, 64, -1), ((1 << 24) + 1, 64, 4),
              (8, 64, (1 << 23) + 1), (1 << 20, 64, (1 << 17) + 1), (8, 131056, (1 << 20) + 256)]


def test_quantize(lib):
    f = lib.bcq_int8_quantize
    args = dict(x=Q, type=F16, q=W, scales=TS, rows=4, n=64, stream=None)
    for name in ("x", "q", "scales"):
        assert f(*changed(args, **{name: None})) == NULL, name
    for type_ in (-1, 2):
        assert f(*changed(args, type=type_)) == TYPE
    for n in (0, 8, 40, 131072):
        assert f(*changed(args, n=n)) == SHAPE, n
    for rows in (-1, (1 << 24) + 1):
        assert f(*changed(args, rows=rows)) == SHAPE, rows
    assert f(*changed(args, x=Q + 8)) == ALIGN
    assert f(*changed(args, q=W + 4)) == ALIGN
    assert f(*changed(args, scales=TS + 2)) == ALIGN
    assert f(*changed(args, rows=0)) == OK
    assert f(*changed(args, rows=0, x=None, q=None, scales=None)) == OK


def test_gemm(lib):
    f = lib.bcq_int8_gemm
    args = dict(q=Q, ts=TS, w=W, cs=CS, y=Y, type=BF16, m=8, n=64, tokens=4, stream=None)
    for name in ("q", "ts", "w", "cs", "y"):
        assert f(*changed(args, **{name: None})) == NULL, name
    assert f(*changed(args, type=2)) == TYPE
    for m, n, tokens in BAD_SHAPES:
        assert f(*changed(args, m=m, n=n, tokens=tokens)) == SHAPE, (m, n, tokens)
    for name, off in (("q", 8), ("ts", 2), ("w", 1), ("cs", 1), ("y", 1)):
        assert f(*changed(args, **{name: args[name] + off})) == ALIGN, name
    assert f(*changed(args, tokens=0)) == OK
    assert f(*changed(args, tokens=0, q=None, ts=None, y=None)) == OK
    assert f(*changed(args, tokens=0, w=None)) == NULL


def test_gated(lib):
    f = lib.bcq_int8_gated
    args = dict(q=Q, ts=TS, wg=W, cg=CS, wu=W + 0x100, cu=CS + 0x100, activation=1, h=Y, type=F16, m=8, n=64, tokens=4, stream=None)
    for name in ("q", "ts", "wg", "cg", "wu", "cu", "h"):
        assert f(*changed(args, **{name: None})) == NULL, name
    assert f(*changed(args, type=-1)) == TYPE
    for activation in (-1, 2):
        assert f(*changed(args, activation=activation)) == TYPE
    for m, n, tokens in BAD_SHAPES:
        assert f(*changed(args, m=m, n=n, tokens=tokens)) == SHAPE, (m, n, tokens)
    for name, off in (("q", 8), ("ts", 2), ("wg", 8), ("cg", 2), ("wu", 8), ("cu", 2), ("h", 1)):
        assert f(*changed(args, **{name: args[name] + off})) == ALIGN, name
    assert f(*changed(args, tokens=0, q=None, ts=None, h=None)) == OK


def test_workspace(lib):
    size = lib.bcq_int8_backward_workspace
    assert size(1, 8, 64, 0) >= 0
    for matrices in (0, 3):
        assert size(matrices, 8, 64, 4) == SHAPE
    for m, n, tokens in [*BAD_SHAPES, ((1 << 20) + 1, 64, 4)]:
        assert size(1, m, n, tokens) == SHAPE
    # the gradients of the projections in 16 bits at least, and growing with what it holds
    assert size(1, 1000, 64, 100) >= 2 * 1000 * 100
    assert size(2, 1000, 64, 100) >= 2 * 2 * 1000 * 100
    assert size(2, 14336, 64, 4096) > size(1, 14336, 64, 4096) > size(1, 14336, 64, 4095)
    assert size(2, 1 << 20, 64, 1 << 17) > 1 << 39


def test_gemm_backward(lib):
    f = lib.bcq_int8_gemm_backward
    need = lib.bcq_int8_backward_workspace(1, 8, 64, 4)
    args = dict(dy=Y, q=Q, ts=TS, w=W, cs=CS, dx=0x6000, dcs=0x7000, type=F16, m=8, n=64, tokens=4, ws=WS, size=need - 1, stream=None)
    assert f(*args.values()) == WORKSPACE
    args["size"] = need
    for name in ("dy", "q", "ts", "w", "cs", "dx", "dcs", "ws"):
        assert f(*changed(args, **{name: None})) == NULL, name
    assert f(*changed(args, type=5)) == TYPE
    for m, n, tokens in [*BAD_SHAPES, ((1 << 20) + 1, 64, 4)]:
        assert f(*changed(args, m=m, n=n, tokens=tokens)) == SHAPE, (m, n, tokens)
    for name, off in (("dy", 1), ("q", 8), ("ts", 2), ("w", 8), ("cs", 2), ("dx", 8), ("dcs", 2), ("ws", 16)):
        assert f(*changed(args, **{name: args[name] + off})) == ALIGN, name


def test_gated_backward(lib):
    f = lib.bcq_int8_gated_backward
    need = lib.bcq_int8_backward_workspace(2, 8, 64, 4)
    args = dict(dh=Y, q=Q, ts=TS, wg=W, cg=CS, wu=W + 0x100, cu=CS + 0x100, activation=0, dx=0x6000, dg=0x7000, du=0x8000, type=F16, m=8, n=64,
                tokens=4, ws=WS, size=need - 1, stream=None)
    assert f(*args.values()) == WORKSPACE
    args["size"] = need
    for name in ("dh", "q", "ts", "wg", "cg", "wu", "cu", "dx", "dg", "du", "ws"):
        assert f(*changed(args, **{name: None})) == NULL, name
    assert f(*changed(args, type=2)) == TYPE
    assert f(*changed(args, activation=2)) == TYPE
    for m, n, tokens in [*BAD_SHAPES, ((1 << 20) + 1, 64, 4)]:
        assert f(*changed(args, m=m, n=n, tokens=tokens)) == SHAPE, (m, n, tokens)
    for name, off in (("dh", 1), ("q", 8), ("ts", 2), ("wg", 8), ("cg", 2), ("wu", 8), ("cu", 2), ("dx", 8), ("dg", 2), ("du", 1), ("ws", 128)):
        assert f(*changed(args, **{name: args[name] + off})) == ALIGN, name


def test_statuses_have_words(lib):
    words = {lib.bcq_strerror(s).decode() for s in range(0, -9, -1)}
    assert len(words) == 9 and "unknown status" not in words
    assert lib.bcq_strerror(-9).decode() == "unknown status"


def test_binding_refuses_cpu_tensors(lib):
    import torch

    import paper_2510_10467_amd as bcq
    q, ts, w, cs = torch.zeros((2, 32), dtype=torch.int8), torch.ones(2), torch.zeros((4, 32), dtype=torch.int8), torch.ones(4)
    x, dy = torch.zeros((2, 32), dtype=torch.float16), torch.zeros((2, 4), dtype=torch.float16)
    for call in (lambda: bcq.bcq_int8_quantize(x), lambda: bcq.bcq_int8_gemm(q, ts, w, cs), lambda: bcq.bcq_int8_gated(q, ts, w, cs, w, cs),
                 lambda: bcq.bcq_int8_gemm_backward(dy, q, ts, w, cs), lambda: bcq.bcq_int8_gated_backward(dy, q, ts, w, cs, w, cs)):
        with pytest.raises(TypeError, match="GPU tensor"):
            call()
