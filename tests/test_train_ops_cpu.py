"""Refusals of the entry points around the layer (embedding, norm, the head's cross
entropy), on the host before any CUDA call, and of their binding."""
import ctypes

import pytest
import torch

from paper_2609_34117_gb300 import binding, build

A, B, C, D, E, F, G, W = (0x10000000 * (i + 1) for i in range(8))
ROWS_MAX = 1 << 20


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _embed(lib, table=A, dtype=0, vocab=100, hidden=64, stride=64, ids=B, rows=4, scale=1.0, out=C, ostride=64):
    return lib.slimwise_embed(table, dtype, vocab, hidden, stride, ids, rows, scale, out, ostride, None)


def _embed_grad(lib, grad=A, dtype=0, rows=4, hidden=64, stride=64, ids=B, scale=1.0, out=C, odtype=1,
                vocab=100, ostride=64, accumulate=0, ws=W, size=1 << 30):
    return lib.slimwise_embed_grad(grad, dtype, rows, hidden, stride, ids, scale, out, odtype, vocab, ostride,
                                   accumulate, None, ws, size)


def _norm(lib, x=A, dtype=0, rows=4, hidden=64, stride=64, weight=B, bias=None, layer=1, eps=1e-5, y=C,
          ystride=64, mean=D, rstd=E):
    return lib.slimwise_norm(x, dtype, rows, hidden, stride, weight, bias, layer, eps, y, ystride, mean, rstd, None)


def _norm_grad(lib, dy=F, dstride=64, x=A, dtype=0, rows=4, hidden=64, stride=64, weight=B, mean=D, rstd=E,
               dx=C, xstride=64, dweight=G, dbias=None, ws=W, size=1 << 30):
    return lib.slimwise_norm_grad(dy, dstride, x, dtype, rows, hidden, stride, weight, mean, rstd, dx, xstride,
                                  dweight, dbias, None, ws, size)


def _loss(lib, hidden=A, stride=64, weight=B, wstride=64, rows=4, width=64, vocab=100, labels=C,
          row_weight=None, row_loss=D, loss=E, dh=F, dhs=64, dw=G, dwt=0, dws=64, ws=W, size=1 << 34):
    return lib.slimwise_linear_loss(hidden, stride, weight, wstride, rows, width, vocab, labels, row_weight,
                                    row_loss, loss, dh, dhs, dw, dwt, dws, None, ws, size)


@pytest.mark.parametrize("call,kw,code", [
    (_embed, {"dtype": 2}, 2), (_embed, {"rows": -1}, 1), (_embed, {"rows": ROWS_MAX + 1}, 1),
    (_embed, {"hidden": 0}, 2), (_embed, {"hidden": 16385, "stride": 16385, "ostride": 16385}, 2),
    (_embed, {"vocab": 0}, 2), (_embed, {"vocab": (1 << 20) + 1}, 2), (_embed, {"stride": 63}, 1),
    (_embed, {"ostride": 63}, 1), (_embed, {"stride": (1 << 40) + 1}, 1), (_embed, {"scale": float("nan")}, 1),
    (_embed, {"scale": float("inf")}, 1), (_embed, {"table": None}, 1), (_embed, {"ids": None}, 1),
    (_embed, {"out": None}, 1), (_embed, {"table": A + 1}, 2), (_embed, {"out": C + 2, "dtype": 1}, 2),
    (_embed, {"ids": B + 2}, 2), (_embed, {"out": A}, 1), (_embed, {"out": A + 100 * 128 - 2}, 1),
    (_embed, {"out": B - 4 * 128 + 2}, 1), (_embed, {"out": A + 2, "ostride": 128, "stride": 128}, 1),
    (_embed, {"rows": 0, "table": None, "ids": None, "out": None}, 0),
    (_embed_grad, {"dtype": 2}, 2), (_embed_grad, {"odtype": 2}, 2), (_embed_grad, {"rows": -1}, 1),
    (_embed_grad, {"vocab": (1 << 20) + 1}, 2), (_embed_grad, {"hidden": 0}, 2), (_embed_grad, {"stride": 1}, 1),
    (_embed_grad, {"ostride": 1}, 1), (_embed_grad, {"grad": None}, 1), (_embed_grad, {"ids": None}, 1),
    (_embed_grad, {"out": None}, 1), (_embed_grad, {"ws": None}, 1), (_embed_grad, {"ws": W + 16}, 2),
    (_embed_grad, {"size": 100}, 3), (_embed_grad, {"out": C + 2}, 2), (_embed_grad, {"grad": A + 1}, 2),
    (_embed_grad, {"out": A}, 1), (_embed_grad, {"ws": C}, 1), (_embed_grad, {"ws": A}, 1),
    (_embed_grad, {"rows": 0, "grad": None, "ids": None, "out": None, "ws": None, "accumulate": 1}, 0),
    (_embed_grad, {"rows": 0, "grad": None, "ids": None, "out": None}, 1),
    (_norm, {"dtype": 3}, 2), (_norm, {"rows": ROWS_MAX + 1}, 1), (_norm, {"hidden": 16385, "stride": 16385,
                                                                           "ystride": 16385}, 2),
    (_norm, {"hidden": 0}, 2), (_norm, {"stride": 63}, 1), (_norm, {"ystride": 63}, 1), (_norm, {"eps": -1.0}, 1),
    (_norm, {"eps": float("nan")}, 1), (_norm, {"eps": float("inf")}, 1), (_norm, {"x": None}, 1),
    (_norm, {"weight": None}, 1), (_norm, {"y": None}, 1), (_norm, {"rstd": None}, 1), (_norm, {"mean": None}, 1),
    (_norm, {"layer": 0}, 1), (_norm, {"x": A + 1}, 2), (_norm, {"y": C + 1}, 2), (_norm, {"weight": B + 2}, 2),
    (_norm, {"bias": F + 1}, 2), (_norm, {"rstd": E + 2}, 2), (_norm, {"y": A}, 1), (_norm, {"y": A + 128}, 1),
    (_norm, {"mean": E}, 1), (_norm, {"rstd": B}, 1), (_norm, {"mean": C + 16}, 1),
    (_norm, {"rows": 0, "x": None, "weight": None, "y": None, "rstd": None, "mean": None}, 0),
    (_norm_grad, {"dtype": 3}, 2), (_norm_grad, {"dstride": 63}, 1), (_norm_grad, {"xstride": 63}, 1),
    (_norm_grad, {"dy": None}, 1), (_norm_grad, {"dx": None}, 1), (_norm_grad, {"rstd": None}, 1),
    (_norm_grad, {"dweight": None}, 1), (_norm_grad, {"ws": None}, 1), (_norm_grad, {"size": 16}, 3),
    (_norm_grad, {"mean": None, "dbias": 0x7FFF0000}, 1), (_norm_grad, {"ws": W + 2}, 2),
    (_norm_grad, {"dweight": G + 2}, 2), (_norm_grad, {"dx": A}, 1), (_norm_grad, {"dx": F}, 1),
    (_norm_grad, {"dweight": B}, 1), (_norm_grad, {"dbias": G}, 1), (_norm_grad, {"ws": A}, 1),
    (_norm_grad, {"rows": 0, "dy": None, "x": None, "dx": None, "ws": None}, 0),
    (_loss, {"rows": -1}, 1), (_loss, {"width": 60}, 2), (_loss, {"width": 0}, 2), (_loss, {"vocab": 0}, 2),
    (_loss, {"vocab": 393217}, 2), (_loss, {"width": 16392, "stride": 16392, "wstride": 16392, "dhs": 16392,
                                            "dws": 16392}, 2),
    (_loss, {"stride": 56}, 1), (_loss, {"wstride": 56}, 1), (_loss, {"dhs": 56}, 1), (_loss, {"dws": 56}, 1),
    (_loss, {"dwt": 2}, 2), (_loss, {"hidden": None}, 1), (_loss, {"weight": None}, 1), (_loss, {"labels": None}, 1),
    (_loss, {"row_loss": None}, 1), (_loss, {"ws": None}, 1), (_loss, {"stride": 68}, 2), (_loss, {"wstride": 65}, 2),
    (_loss, {"dhs": 66}, 2), (_loss, {"dws": 68}, 2), (_loss, {"dws": 66, "dwt": 1}, 2), (_loss, {"hidden": A + 8}, 2),
    (_loss, {"weight": B + 2}, 2), (_loss, {"dh": F + 8}, 2), (_loss, {"dw": G + 4}, 2), (_loss, {"labels": C + 2}, 2),
    (_loss, {"row_weight": 0x70000002}, 2), (_loss, {"loss": E + 1}, 2), (_loss, {"ws": W + 128}, 2),
    (_loss, {"size": 1000}, 3), (_loss, {"dh": A}, 1), (_loss, {"dw": B}, 1), (_loss, {"dh": G}, 1),
    (_loss, {"loss": D + 4}, 1), (_loss, {"ws": A}, 1),
    (_loss, {"rows": 0, "hidden": None, "weight": None, "labels": None, "row_loss": None, "ws": None}, 0),
])
def test_refusals(lib, call, kw, code):
    assert call(lib, **kw) == code


def test_workspace_sizes(lib):
    n = ctypes.c_size_t(0)
    size = ctypes.byref(n)
    assert lib.slimwise_embed_grad_workspace_size(-1, 64, size) == 1
    assert lib.slimwise_embed_grad_workspace_size(4, 0, size) == 2
    assert lib.slimwise_embed_grad_workspace_size(4, 64, None) == 1
    assert lib.slimwise_norm_grad_workspace_size(4, 16385, size) == 2
    assert lib.slimwise_norm_grad_workspace_size(4, 64, None) == 1
    assert lib.slimwise_linear_loss_workspace_size(4, 12, 100, 1, 1, size) == 2
    assert lib.slimwise_linear_loss_workspace_size(4, 64, 100, 1, 1, None) == 1
    # at most 2^31 bytes for the numerators, whatever the rows
    base = binding.slimwise_linear_loss_workspace_size(8192, 2048, 131072)
    assert base < binding.slimwise_linear_loss_workspace_size(1 << 20, 2048, 131072) < base + (12 << 30)
    assert binding.slimwise_linear_loss_workspace_size(4096, 2048, 131072, False, False) < 1 << 28
    assert binding.slimwise_linear_loss_workspace_size(0, 2048, 131072) == 0


def test_binding_refuses_cpu_tensors_types_and_shapes(lib):
    x, v, ids = torch.zeros(4, 64), torch.zeros(64), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: binding.slimwise_embed(x, ids), lambda: binding.slimwise_embed_grad(x, ids, x),
                 lambda: binding.slimwise_norm(x, v), lambda: binding.slimwise_norm_grad(x, x, v, v[:4]),
                 lambda: binding.slimwise_linear_loss(x, x, ids)):
        with pytest.raises(TypeError):
            call()
