"""Edges of the operators around the layer: where variants meet alignment, infinite
logits, logits whose sums are exact or dense, and long lists of ids."""
import math

import pytest
import torch

import paper_2609_34117_gb300 as sw
from tests.test_gpu_train_ops import BF16, DEV, F32, NAN, _check_norm, _gen, _grad_reference, _half, _head, _randn, _rows, _within

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


@pytest.mark.parametrize("vocab", [1, 2, 300])
@pytest.mark.parametrize("rows", [3, 200])
def test_linear_loss_where_all_logits_are_minus_infinity(rows, vocab):
    hidden, weight = torch.zeros((rows, 64), dtype=BF16, device=DEV), torch.zeros((vocab, 64), dtype=BF16, device=DEV)
    weight[:, 3], hidden[::2, 3] = -HUGE, HUGE
    labels = torch.zeros(rows, dtype=torch.int32, device=DEV)
    bad = torch.arange(rows, device=DEV) % 2 == 0
    for dh, dw in PARTS:
        _, row, gh, gw = sw.slimwise_linear_loss(hidden, weight, labels, grad_hidden=dh, grad_weight=dw)
        assert torch.equal(row.isnan(), bad) and bool(((row[~bad] - math.log(vocab)).abs() <= 1e-5).all())
        assert gh is None or bool(gh[bad].isnan().all())
        assert gw is None or bool(gw.isnan().all())


# ---------------------------------------------------------------------------
# the head's cross entropy: what the tensor cores cut off a logit
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("kind", ["one element", "sums that cancel"])
@pytest.mark.parametrize("rows", [40, 250])
@pytest.mark.parametrize("width", [64, 4096, 8192, 16384])
def test_linear_loss_of_exact_logits(width, rows, kind, grad):
    vocab, g = 600, _gen(width)
    hidden = torch.zeros((rows, width), device=DEV)
    if kind == "one element":
        # one product a logit, up to 64
        at = torch.randint(0, width, (rows, 1), generator=g, device=DEV)
        hidden.scatter_(1, at, 16.0)
        weight = torch.randint(-512, 513, (vocab, width), generator=g, device=DEV) / 128.0
    else:
        # multiples of 1/8 that wander up to a few hundred and back: every partial sum is a
        # whole number of them below 2^24
        hidden.copy_(torch.randint(0, 2, hidden.shape, generator=g, device=DEV) * 2.0 - 1.0)
        weight = torch.randint(-1, 2, (vocab, width), generator=g, device=DEV) / 8.0
        weight[:, width // 2:] += 2.0 * weight[:, width // 2:].sign() * (width >= 4096)
        weight[:, width // 2 + width // 4:] = -weight[:, width // 2:width // 2 + width // 4]
        hidden[:, width // 2 + width // 4:] = hidden[:, width // 2:width // 2 + width // 4]
    hidden, weight = hidden.to(BF16), weight.to(BF16)
    labels = torch.randint(0, vocab, (rows,), generator=g, device=DEV).int()
    _, row, _, _ = sw.slimwise_linear_loss(hidden, weight, labels, grad_hidden=grad, grad_weight=False)
    z = hidden.double() @ weight.double().T
    y = labels.long()[:, None]
    over = torch.logsumexp(z.scatter(1, y, -math.inf), 1) - z.gather(1, y)[:, 0]
    want = over.clamp(min=0) + torch.log1p(torch.exp(-over.abs()))
    # the logits are exact.  A difference of logits d is rounded, then times log2 e: its exponential
    # is off by 2 |d| 2^-24 of itself and 2^-22; sums of 128 + 64 + 64 terms; the logarithm's and
    # the last sum's roundings
    d = (z - z.gather(1, y)).abs().amax(1)
    off = d * 2.0 ** -23 + 2.0 ** -21 + 300 * 2.0 ** -24
    if kind == "sums that cancel":
        # nothing is cut off, but what is expected to be is given back: 1e-9 of a logit for each
        # element (of one element less than a rounding)
        off = off + 1.01e-9 * width * z.abs().amax(1)
    _within(row, want, off * want.clamp(max=1.0) + want * 2.0 ** -22)


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("rows", [40, 250, 600])
def test_linear_loss_of_dense_rows_among_others(rows, grad):
    width, vocab, g = 4096, 900, _gen(rows)
    hidden, weight, labels, wt = _head(rows, width, vocab, seed=rows, ignored=0.0)
    some = torch.rand(rows, generator=g, device=DEV) < 0.2
    alone = sw.slimwise_linear_loss(hidden, weight, torch.where(some, -1, labels).int(), wt, grad_hidden=grad, grad_weight=False)
    hidden[some] = 0.0
    hidden[some, 17] = 30.0
    row = sw.slimwise_linear_loss(hidden, weight, labels, wt, grad_hidden=grad, grad_weight=False)[1]
    z = hidden.double() @ weight.double().T
    # a logit of a dense row may be rounded once more, and then the difference to the label's
    largest = z.abs().amax(1)
    _within(row[~some], alone[1][~some].double(), (largest * 2.0 ** -22 + 2.0 ** -21 * alone[1].abs())[~some])
    want = torch.logsumexp(z, 1) - z.gather(1, labels.long()[:, None])[:, 0]
    _within(row[some], want[some], (2 * largest * 2.0 ** -23 + 2.0 ** -21 + 300 * 2.0 ** -24 + want * 2.0 ** -22)[some])


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("rows", [40, 250])
@pytest.mark.parametrize("width", [2048, 4096, 8192, 16384])
def test_linear_loss_of_dense_rows_is_not_too_small(width, rows, grad):
    # another word's logit is about 15 and grows steadily: uncorrected, it and the loss are too
    # small by 1e-9 of it for each element; a tenth of that differs with how the sums grow
    vocab, g = 2000, _gen(width + rows)
    weight = (torch.randn((vocab, width), generator=g, device=DEV) * (1.5 / math.sqrt(width))).to(BF16)
    other = torch.randint(1000, vocab, (rows,), generator=g, device=DEV)
    hidden = (torch.randn((rows, width), generator=g, device=DEV) + 15 / 2.25 * weight[other].float()).to(BF16)
    labels = torch.randint(0, 1000, (rows,), generator=g, device=DEV).int()
    _, row, _, _ = sw.slimwise_linear_loss(hidden, weight, labels, grad_hidden=grad, grad_weight=False)
    z = hidden.double() @ weight.double().T
    p = torch.softmax(z, 1)
    cut = 1e-9 * width * float((p * z).sum(1).mean())
    error = float((row.double() - (torch.logsumexp(z, 1) - z.gather(1, labels.long()[:, None])[:, 0])).mean())
    assert cut > 2e-5 and abs(error) <= 0.25 * cut + 2.0 ** -21


# ---------------------------------------------------------------------------
# the table's gradient: long lists
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,odtype", [(BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("kind", ["one token", "few tokens", "log-uniform", "all different"])
@pytest.mark.parametrize("rows,hidden", [(70001, 16), (131072, 9), (200003, 8), (1 << 20, 8)])
def test_embed_grad_of_long_lists(rows, hidden, kind, dtype, odtype):
    vocab, g = 1 << 20 if kind == "all different" else 100003, _gen(rows)
    if kind == "one token":
        ids = torch.full((rows,), 77, device=DEV)
    elif kind == "few tokens":
        ids = torch.randint(0, 5, (rows,), generator=g, device=DEV) * 25000
    elif kind == "log-uniform":
        ids = (vocab ** torch.rand(rows, generator=g, device=DEV)).long().clamp(max=vocab) - 1
    else:
        ids = torch.randperm(vocab, generator=g, device=DEV)[:rows]
    ids = ids.int()
    if kind != "all different":
        ids[::16], ids[5::977] = -1, vocab
    grad = torch.randn((rows, hidden), generator=g, device=DEV).to(dtype)
    out = torch.full((vocab, hidden), NAN, dtype=odtype, device=DEV)
    sw.slimwise_embed_grad(grad, ids, out, scale=2.0)
    live = (ids >= 0) & (ids < vocab)
    at, v = ids[live].long(), grad[live].double()
    zeros = torch.zeros((vocab, hidden), dtype=torch.float64, device=DEV)
    want, sizes = zeros.index_add(0, at, v) * 2.0, zeros.index_add(0, at, v.abs()) * 2.0
    count = torch.bincount(at, minlength=vocab).double()
    # a token's positions are summed in pieces of 256 at most (4 at least), which are then added in
    # order: a chain of 256 additions and one a piece, of 64 at least where the list is this long
    chain = (256.0 + count / 64 + 2.0).clamp(max=float(1 << 20)).minimum(count + 2.0)[:, None] * 2.0 ** -24
    _within(out, want, want.abs() * (_half(odtype) + 2.0 ** -23) + sizes * chain)
    assert bool((out[count == 0] == 0).all())
    again = torch.empty_like(out)
    sw.slimwise_embed_grad(grad, ids, again, scale=2.0)
    assert torch.equal(out, again)
