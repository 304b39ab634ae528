"""Edges of the operators around the layer: where variants meet alignment, and infinite
logits."""
import math

import pytest
import torch

import paper_2609_34117_gb300 as sw
from tests.test_gpu_train_ops import BF16, DEV, _check_norm, _grad_reference, _half, _head, _randn, _rows, _within

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


# ---------------------------------------------------------------------------
# the head's cross entropy: infinite logits
# ---------------------------------------------------------------------------
# rows few enough for tiles of them (vocabulary and rows in changed roles), in tiles of 256,
# and of several tiles
SIZES = [(40, 64, 700), (300, 64, 700), (300, 520, 2049), (700, 136, 1000)]
PARTS = [(True, True), (True, False), (False, True), (False, False)]
HUGE = 2.0 ** 127  # its square is past every type's range


def _infinite(rows, width, vocab, infinite):
    """A head whose logits of column V0 are what `infinite` says in rows with a huge (or 1)
    first element, and whose others do not see that element."""
    hidden, weight, labels, wt = _head(rows, width, vocab, seed=rows + width, ignored=0.0)
    labels = torch.where(labels == 11, 12, labels).int()
    weight[:, 0], hidden[:, 0] = 0.0, 0.0
    weight[11, 0] = infinite
    return hidden, weight, labels, wt


@pytest.mark.parametrize("at_label", [True, False])
@pytest.mark.parametrize("infinite", [HUGE, math.inf])
@pytest.mark.parametrize("rows,width,vocab", SIZES)
def test_linear_loss_of_a_logit_of_plus_infinity(rows, width, vocab, infinite, at_label):
    hidden, weight, labels, wt = _infinite(rows, width, vocab, infinite)
    if math.isinf(infinite):
        hidden[:, 0] = -1.0  # the others' logits of that word: -inf
    bad = torch.zeros(rows, dtype=torch.bool, device=DEV)
    bad[[7, rows - 1]] = True
    labels[bad] = 11 if at_label else 5
    usual = labels.clone()
    usual[bad] = 5
    clean = sw.slimwise_linear_loss(hidden, weight, usual, wt)
    assert bool(clean[1].isfinite().all())
    hidden[bad, 0] = HUGE
    for dh, dw in PARTS:
        loss, row, gh, gw = sw.slimwise_linear_loss(hidden, weight, labels, wt, grad_hidden=dh, grad_weight=dw)
        assert bool(loss.isnan().all()) and torch.equal(row.isnan(), bad)
        if dh:
            assert bool(gh[bad].isnan().all()) and torch.equal(gh[~bad, 1:], clean[2][~bad, 1:])
        if dw:
            assert bool(gw.isnan().all())
        if dh or dw:
            assert torch.equal(row[~bad], clean[1][~bad])


@pytest.mark.parametrize("rows,width,vocab", SIZES)
def test_linear_loss_of_logits_of_minus_infinity(rows, width, vocab):
    # the label's and another one's: the loss is infinite, the gradient is not.  It is what it is
    # where both are so low that their exponentials are 0.
    hidden, weight, labels, wt = _infinite(rows, width, vocab, -HUGE)
    weight[13, 0] = -HUGE
    low = torch.zeros(rows, dtype=torch.bool, device=DEV)
    low[[0, 9, rows - 2]] = True
    labels[low] = 11
    labels[9] = 5  # not at the label
    finite_w, finite_h = weight.clone(), hidden.clone()
    finite_w[:, 0] /= HUGE / 16
    finite_h[low, 0], hidden[low, 0] = 16.0, HUGE
    impossible = low & (labels == 11)
    for dh, dw in PARTS:
        want = sw.slimwise_linear_loss(finite_h, finite_w, labels, wt, grad_hidden=dh, grad_weight=dw)
        _, row, gh, gw = sw.slimwise_linear_loss(hidden, weight, labels, wt, grad_hidden=dh, grad_weight=dw)
        assert bool((row[impossible] == math.inf).all()) and torch.equal(row[~impossible], want[1][~impossible])
        if dh:
            assert torch.equal(gh[:, 1:], want[2][:, 1:])
        if dw:
            assert torch.equal(gw[:, 1:], want[3][:, 1:])
