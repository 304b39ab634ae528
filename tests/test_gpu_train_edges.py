"""Edges of the operators around the layer: where variants meet alignment."""
import pytest
import torch

import paper_2609_34117_gb300 as sw
from tests.test_gpu_train_ops import BF16, _check_norm, _grad_reference, _half, _randn, _rows, _within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sw.build.build()


# ---------------------------------------------------------------------------
# norm
# ---------------------------------------------------------------------------
# widths at which a group's threads hold exactly a row
WHOLE = [256, 512, 1024, 2048, 4096, 8192, 12288, 16384]


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("hidden", WHOLE)
def test_norm_of_whole_widths_into_rows_that_start_anywhere(hidden, alike, layer):
    # a mean well above the spread: columns that are counted but not there would show
    values, d = _randn(19, hidden, seed=hidden) + 10.0, _randn(19, hidden, seed=1)
    w, b = 1 + 0.2 * _randn(hidden, seed=2), 0.1 * _randn(hidden, seed=3)
    for pad, start in [(0, k) for k in range(1, 8)] + [(1, 0), (7, 3), (3, 0)]:
        place = (pad, start) if alike else (0, 0)
        x, dy = _rows(values, BF16, *place)[0], _rows(d, BF16, *place)[0]
        (y, around), (dx, beside) = (_rows(torch.zeros_like(values), BF16, pad, start) for _ in range(2))
        outside = int(torch.isnan(around).sum())
        _, mean, rstd = _check_norm(x, w, b, layer, y=y)
        # its statistics in the gradient
        got = sw.slimwise_norm_grad(dy, x, w, rstd, mean=mean, dx=dx)[0]
        want, _, _, tol, _, _ = _grad_reference(dy, x, w, mean, rstd)
        _within(got, want, want.abs() * _half(BF16) + tol * 1.01 + torch.finfo(BF16).tiny)
        assert int(torch.isnan(around).sum()) == outside and int(torch.isnan(beside).sum()) == outside
