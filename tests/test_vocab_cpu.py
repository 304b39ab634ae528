"""Refusals of the entry points over vocabulary logits, on the host before any
CUDA call, and of their binding."""
import ctypes

import pytest
import torch

from paper_2609_34117_gb300 import binding, build

BIG = 1 << 20


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _p(addr=0x10000):
    return ctypes.c_void_p(addr)


def _top(lib, logits=_p(), dtype=0, rows=4, vocab=100, stride=100, k=8, tau=1.0, ids=_p(), logp=_p(),
         rest=_p()):
    return lib.slimwise_top_logits(logits, dtype, rows, vocab, stride, k, tau, ids, logp, rest, None)


def _loss(lib, logits=_p(), dtype=0, rows=4, vocab=100, stride=100, labels=_p(), ids=_p(), logp=_p(),
          rest=_p(), k=8, alpha=0.1, tau=1.0, weight=None, row_loss=_p(), loss=_p(), grad=_p(BIG),
          gstride=100):
    return lib.slimwise_distill_loss(logits, dtype, rows, vocab, stride, labels, ids, logp, rest, k,
                                     alpha, tau, weight, row_loss, loss, grad, gstride, None)


def _sample(lib, logits=_p(), dtype=0, rows=4, vocab=100, stride=100, t=_p(), k=_p(), p=_p(), m=_p(),
            u=_p(), tokens=_p(), logprob=_p()):
    return lib.slimwise_sample(logits, dtype, rows, vocab, stride, t, k, p, m, u, tokens, logprob, None)


@pytest.mark.parametrize("call", [_top, _loss, _sample])
@pytest.mark.parametrize("kw,code", [
    ({"dtype": 2}, 2), ({"dtype": -1}, 2), ({"rows": -1}, 1), ({"rows": (1 << 20) + 1}, 1),
    ({"vocab": 0}, 2), ({"vocab": 393217, "stride": 393217}, 2), ({"stride": 99}, 1),
    ({"stride": (1 << 40) + 1}, 1), ({"logits": None}, 1), ({"logits": _p(0x10001)}, 2),
    ({"logits": _p(0x10002), "dtype": 1}, 2),
])
def test_rows_are_checked(lib, call, kw, code):
    assert call(lib, **kw) == code


@pytest.mark.parametrize("call", [_top, _loss, _sample])
def test_no_rows_is_a_no_op(lib, call):
    assert call(lib, logits=None, rows=0) == 0


@pytest.mark.parametrize("kw,code", [
    ({"k": 0}, 1), ({"k": 257, "vocab": 300, "stride": 300}, 1), ({"k": 101}, 1), ({"tau": 0.0}, 1),
    ({"tau": -1.0}, 1), ({"tau": float("nan")}, 1), ({"tau": float("inf")}, 1), ({"ids": None}, 1),
    ({"logp": None}, 1), ({"rest": None}, 1), ({"ids": _p(0x10002)}, 2), ({"rest": _p(0x10001)}, 2),
])
def test_top_logits_refuses(lib, kw, code):
    assert _top(lib, **kw) == code


@pytest.mark.parametrize("kw,code", [
    ({"k": 0}, 1), ({"k": 257, "vocab": 300, "stride": 300, "gstride": 300}, 1), ({"alpha": -0.1}, 1),
    ({"alpha": 1.1}, 1), ({"alpha": float("nan")}, 1), ({"tau": 0.0}, 1), ({"labels": None}, 1),
    ({"ids": None}, 1), ({"logp": None}, 1), ({"rest": None}, 1), ({"row_loss": None}, 1),
    ({"gstride": 99}, 1), ({"labels": _p(0x10002)}, 2), ({"weight": _p(0x10001)}, 2),
    ({"grad": _p(BIG + 1)}, 2), ({"loss": _p(0x10002)}, 2),
    # the gradient over the logits with another stride, or shifted by a row or an element
    ({"grad": _p(0x10000), "gstride": 101}, 1), ({"grad": _p(0x10000 + 200)}, 1),
    ({"grad": _p(0x10002)}, 1), ({"grad": _p(0x10000 - 2)}, 1),
    ({"grad": _p(0x10000 + 2 * (3 * 100 + 99))}, 1),
])
def test_distill_loss_refuses(lib, kw, code):
    assert _loss(lib, **kw) == code


@pytest.mark.parametrize("kw,code", [
    ({"u": None}, 1), ({"tokens": None}, 1), ({"logprob": None}, 1), ({"t": _p(0x10002)}, 2),
    ({"k": _p(0x10001)}, 2), ({"u": _p(0x10002)}, 2), ({"tokens": _p(0x10002)}, 2),
])
def test_sample_refuses(lib, kw, code):
    assert _sample(lib, **kw) == code


def test_binding_refuses_cpu_tensors_and_other_types(lib):
    z = torch.zeros(4, 100)
    with pytest.raises(TypeError):
        binding.slimwise_top_logits(z, 8)
    with pytest.raises(TypeError):
        binding.slimwise_sample(z, torch.zeros(4))
    with pytest.raises(TypeError):
        binding.slimwise_distill_loss(z, torch.zeros(4, dtype=torch.int32),
                                      torch.zeros((4, 8), dtype=torch.int32), torch.zeros(4, 8),
                                      torch.zeros(4))
