"""The binding's host code, where what is installed does not go with the package: the calls are made in Python, with a warning (no GPU needed)."""
import sys
import types

import pytest
import torch

import paper_2510_10467_amd as bcq
from paper_2510_10467_amd import binding
from paper_2510_10467_amd import build as hip_build


@pytest.fixture
def load(monkeypatch):
    """load(module): what `binding` takes for its host code where `module` is the extension that is there"""
    if hip_build.is_stale():
        hip_build.build()
    L = bcq.lib()

    def with_extension(module):
        monkeypatch.setitem(sys.modules, "paper_2510_10467_amd._bcq_host", module)
        monkeypatch.setattr(bcq, "_bcq_host", module, raising=False)
        return binding._load_host((L.bcq_gemv_offset, L.bcq_gemv_multi, L.bcq_gemm_mixed, L.bcq_gemm_mixed_offset),
                                  (L.bcq_int8_quantize, L.bcq_int8_gemm, L.bcq_int8_gated, L.bcq_int8_backward_workspace, L.bcq_int8_gemm_backward,
                                   L.bcq_int8_gated_backward))
    return with_extension


def extension(**functions):
    module = types.ModuleType("_bcq_host")
    module.torch_version = torch.__version__
    for name, f in functions.items():
        setattr(module, name, f)
    return module


def test_an_extension_that_has_all(load):
    bound = []
    module = extension(bind=lambda *a: bound.append(len(a)), bind_int8=lambda *a: bound.append(len(a)))
    assert load(module) is module and bound == [5, 6]


def test_an_extension_without_the_8_bit_operators(load):
    """One that was built before there were any, against the same torch: nothing is bound to it."""
    bound = []
    with pytest.warns(RuntimeWarning, match="_bcq_host does not load"):
        host = load(extension(bind=lambda *a: bound.append(a)))
    assert host is binding._NoHost and not bound
    for name in ("gemv", "gemv_multi", "gemm_mixed", "int8_quantize", "int8_gemm", "int8_gated", "int8_gemm_backward", "int8_gated_backward"):
        assert getattr(host, name)() is None


def test_an_extension_of_another_torch(load):
    module = extension(bind=None, bind_int8=None)
    module.torch_version = "0.0"
    with pytest.warns(RuntimeWarning, match="built for torch 0.0"):
        assert load(module) is binding._NoHost
