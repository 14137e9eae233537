"""The entry points of include/mvue_layer.h refuse wrong arguments on the host, before any CUDA call, and host tensors in Python."""
import ctypes

import pytest
import torch

from paper_2203_10991_b200 import binding

FAKE, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4097)
BIG = ctypes.c_size_t(1 << 40)


@pytest.fixture(scope="module")
def L():
    from paper_2203_10991_b200 import build
    build.build()
    return binding.lib()


def refused(call, good, cases):
    """Each case puts other arguments in the place of good ones and names the status."""
    for changes, status in cases:
        args = list(good)
        for i, v in changes.items():
            args[i] = v
        assert call(*args) == status, (changes, status)


def test_layer_norm(L):
    good = [FAKE, 0, 4, 16, 16, FAKE, FAKE, 0, 1e-5, FAKE, 16, FAKE, FAKE, None]
    refused(L.mvue_layer_norm, good, [({0: None}, -1), ({9: None}, -1), ({1: 2}, -5), ({7: 9}, -5), ({2: -1}, -3), ({3: 0}, -3), ({4: 15}, -3), ({10: 8}, -3),
                                      ({0: ODD}, -4), ({5: ODD}, -4), ({9: ODD}, -4), ({11: ODD}, -4)])
    assert L.mvue_layer_norm(*[0 if i == 2 else a for i, a in enumerate(good)]) == 0          # no rows: nothing
    back = [FAKE, 16, FAKE, 16, 0, 4, 16, FAKE, FAKE, FAKE, 0, FAKE, 16, FAKE, FAKE, FAKE, BIG, None]
    refused(L.mvue_layer_norm_backward, back, [({0: None}, -1), ({2: None}, -1), ({7: None}, -1), ({11: None}, -1), ({1: 3}, -3), ({12: 3}, -3), ({4: 5}, -5),
                                               ({13: ODD}, -4), ({0: ODD}, -4)])
    b = ctypes.c_size_t()
    assert L.mvue_layer_norm_workspace_bytes(4, 16, None) == -1
    assert L.mvue_layer_norm_workspace_bytes(-1, 16, ctypes.byref(b)) == -3 and L.mvue_layer_norm_workspace_bytes(4, 0, ctypes.byref(b)) == -3


def test_quantize(L):
    good = [FAKE, 1, 4, 16, 16, 1, 0, 0, FAKE, 16, FAKE, None]
    refused(L.mvue_quantize_e4m3, good, [({0: None}, -1), ({8: None}, -1), ({10: None}, -1), ({1: 3}, -5), ({5: 64}, -3), ({5: 0}, -3), ({2: -1}, -3), ({4: 8}, -3),
                                         ({9: 8}, -3), ({6: 2}, -12), ({6: 5}, -12), ({0: ODD}, -4)])
    assert L.mvue_quantize_e4m3(*[0 if i == 2 else a for i, a in enumerate(good)]) == 0


def test_products(L):
    good = [FAKE, FAKE, 8, 64, 64, FAKE, FAKE, 32, 64, FAKE, 1, 64, None, None]
    for call in (L.mvue_scaled_forward_gemm, L.mvue_scaled_backward_gemm):
        refused(call, good, [({0: None}, -1), ({1: None}, -1), ({5: None}, -1), ({6: None}, -1), ({9: None}, -1), ({2: -1}, -3), ({3: 0}, -3), ({7: 0}, -3), ({4: 48}, -3),
                             ({8: 16}, -3), ({11: 16}, -3), ({10: 2}, -5), ({4: 72}, -4), ({8: 72}, -4), ({0: ctypes.c_void_p(4104)}, -4), ({5: ODD}, -4), ({9: ODD}, -4)])
        assert call(*[0 if i == 2 else a for i, a in enumerate(good)]) == 0


def test_orthogonalize_and_muon(L):
    good = [FAKE, 0, 2, 8, 16, 16, 128, 5, FAKE, 1, 16, 128, FAKE, BIG, None, None]
    refused(L.mvue_orthogonalize, good, [({0: None}, -1), ({8: None}, -1), ({1: 2}, -5), ({9: -1}, -5), ({2: -1}, -3), ({5: 15}, -3), ({10: 15}, -3), ({7: 0}, -3), ({7: 17}, -3),
                                         ({6: -1}, -3), ({3: 2 << 20, 4: 2 << 20, 5: 2 << 20, 10: 2 << 20}, -3), ({0: ODD}, -4), ({12: None}, -7),
                                         ({12: ctypes.c_void_p(4096 + 128)}, -7), ({13: ctypes.c_size_t(100)}, -7)])
    assert L.mvue_orthogonalize(*[0 if i == 2 else a for i, a in enumerate(good)]) == 0
    assert binding.mvue_orthogonalize_workspace_bytes(0, 8, 16) == 0 and binding.mvue_orthogonalize_workspace_bytes(2, 8, 16) > 0

    def config(**kw):
        values = dict(lr=0.1, momentum=0.9, weight_decay=0.0, grad_scale=1.0, ns_steps=5, scale_rule=0, options=16)
        return binding.MuonConfig(**{**values, **kw})

    def tensors(**kw):
        values = dict(param=4096, master=None, grad=4096, momentum=4096, rows=8, cols=16, param_dtype=0, grad_dtype=0)
        return (binding.MuonTensor * 1)(binding.MuonTensor(**{**values, **kw}))

    call = lambda t, c, n=1, ws=FAKE, size=BIG: L.mvue_muon_step(t, n, c, ws, size, None, None)  # noqa: E731
    for kw, status in (({"ns_steps": 0}, -3), ({"ns_steps": 17}, -3), ({"options": 2}, -12), ({"scale_rule": 2}, -12), ({"momentum": 1.0}, -12), ({"momentum": float("nan")}, -12)):
        assert call(tensors(), config(**kw)) == status, kw
    for kw, status in (({"param": None}, -1), ({"grad": None}, -1), ({"momentum": None}, -1), ({"rows": -1}, -3), ({"param_dtype": 3}, -5), ({"grad_dtype": 3}, -5),
                       ({"master": 4096}, -5), ({"param": 4098}, -4), ({"momentum": 4098}, -4)):
        assert call(tensors(**kw), config()) == status, kw
    assert call(tensors(), None) == -1 and call(None, config()) == -1 and call(tensors(), config(), n=-1) == -3
    assert call(tensors(), config(), ws=None) == -7 and call(tensors(), config(), size=ctypes.c_size_t(10)) == -7
    assert call(None, config(), n=0) == 0 and call(tensors(rows=0), config(), ws=None) == 0


def test_host_tensors_are_refused():
    x, u8 = torch.zeros(4, 16), torch.zeros(1, 4, dtype=torch.uint8)
    codes = torch.zeros(4, 16, dtype=torch.uint8)
    for call in (lambda: binding.mvue_layer_norm(x), lambda: binding.mvue_layer_norm_backward(x, x, x[:, 0], x[:, 0]), lambda: binding.mvue_quantize_e4m3(x),
                 lambda: binding.mvue_scaled_forward_gemm(codes, u8, codes, u8), lambda: binding.mvue_scaled_backward_gemm(codes, u8, codes, u8),
                 lambda: binding.mvue_orthogonalize(x)):
        with pytest.raises(ValueError):
            call()
