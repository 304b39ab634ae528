"""The operators around the layer against plain evaluations in 64 bits.

Tolerances follow from the kernels' arithmetic: a sum of fp32 terms is off by at
most the longest chain of additions times 2^-24 of the sum of magnitudes, a result
by half a step of its type; what the head's products take in bf16 by half a step
of bf16 each.
"""
import math

import pytest
import torch

import paper_2609_34117_gb300 as sw

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
TYPES = [BF16, F32]
NAN = math.nan
# chain of a row's sum: 32 elements of a thread, 5 steps over lanes, 16 warps, and a
# few roundings beside (the mean's, the square root's, products')
ROW = 64 * 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sw.build.build()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _half(dtype):
    return torch.finfo(dtype).eps / 2


def _rows(values, dtype, pad=0, start=0):
    """Rows with `pad` elements between them, `start` elements into their allocation;
    NaN outside the rows."""
    rows, width = values.shape
    flat = torch.full((start + rows * (width + pad),), NAN, dtype=dtype, device=DEV)
    x = flat[start:].view(rows, width + pad)[:, :width]
    x.copy_(values)
    return x, flat


def _randn(*shape, seed):
    return torch.randn(shape, generator=_gen(seed), device=DEV)


def _within(got, want, tol):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float((got - want).abs().max()), torch.nonzero(bad)[:4].tolist())


# ---------------------------------------------------------------------------
# norm
# ---------------------------------------------------------------------------
def _norm_reference(x, w, b, layer, eps):
    x = x.double()
    mean = x.mean(1) if layer else torch.zeros(x.shape[0], dtype=torch.float64, device=DEV)
    d = x - mean[:, None]
    rstd = (d.square().mean(1) + eps).rsqrt()
    n = d * rstd[:, None]
    y = n * w.double() + (0.0 if b is None else b.double())
    # the mean's error, which the difference takes over
    dm = ROW * x.abs().mean(1, keepdim=True) * rstd[:, None] if layer else 0.0
    # (the variance takes the mean's error too, squared, and once times a sum that is 0 but for rounding)
    loose = (n.abs() * (2 * ROW + (dm if layer else 0.0)) + dm) * w.double().abs()
    return y, mean, rstd, loose


def _check_norm(x, w, b, layer, eps=1e-5, **kw):
    y, mean, rstd = sw.slimwise_norm(x, w, bias=b, layer=layer, eps=eps, **kw)
    want, mu, r, loose = _norm_reference(x, w, b, layer, eps)
    tiny = torch.finfo(x.dtype).tiny
    _within(y, want, want.abs() * (_half(x.dtype) + 2 * 2.0 ** -24) + loose * 1.01 + tiny)
    assert (mean is None) == (not layer)
    if layer:
        _within(mean, mu, ROW * x.double().abs().mean(1))
    spread = ROW * x.double().abs().mean(1) * r if layer else 0.0
    _within(rstd, r, r * (2 * ROW + spread))
    return y, mean, rstd


LENGTHS = [1, 2, 7, 64, 255, 256, 257, 1000, 1024, 1030, 2048, 2049, 4096, 5001, 8192, 8200, 16383, 16384]


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hidden", LENGTHS)
def test_norm(hidden, dtype, layer):
    x, _ = _rows(_randn(13, hidden, seed=hidden) * 2 + 0.5, dtype)
    w, b = 1 + 0.2 * _randn(hidden, seed=1), 0.1 * _randn(hidden, seed=2)
    _check_norm(x, w, b if layer else None, layer)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [0, 1, 2, 3, 151, 609, 1217, 5000])
def test_norm_rows(rows, dtype):
    x, _ = _rows(_randn(rows, 300, seed=rows), dtype)
    _check_norm(x, _randn(300, seed=1), _randn(300, seed=2), True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,start", [(1, 0), (3, 5), (8, 0), (8, 1), (2, 2), (64, 8)])
def test_norm_strides_and_bounds(pad, start, dtype):
    hidden = 1000
    x, _ = _rows(_randn(9, hidden, seed=4), dtype, pad=pad, start=start)
    for ypad, ystart in ((0, 0), (pad, start), (3, 1)):
        y, flat = _rows(torch.zeros(9, hidden, device=DEV), dtype, pad=ypad, start=ystart)
        before = flat.clone()
        _check_norm(x, _randn(hidden, seed=1), None, False, y=y)
        inside = torch.zeros_like(flat, dtype=torch.bool)
        inside[ystart:].view(9, hidden + ypad)[:, :hidden] = True
        assert torch.equal(torch.isnan(flat[~inside]), torch.isnan(before[~inside]))


def test_norm_of_a_mean_far_above_the_spread_and_of_constants():
    x = 1000.0 + _randn(5, 2048, seed=1)
    x[3] = 7.0
    x[4] = 0.0
    w = torch.ones(2048, device=DEV)
    _check_norm(x, w, None, True)
    y, mean, rstd = sw.slimwise_norm(x[3:], w, layer=True, eps=0.25)
    assert bool((y.abs() <= 7 * ROW * 2).all()) and torch.allclose(rstd, torch.full((2,), 2.0, device=DEV), rtol=1e-6)
    y, _, rstd = sw.slimwise_norm(x[4:], w, eps=1e-6)
    assert bool((y == 0).all()) and torch.allclose(rstd, torch.full((1,), 1000.0, device=DEV), rtol=1e-6)


@pytest.mark.parametrize("layer", [False, True])
def test_norm_rows_with_nan_stay_alone(layer):
    x = _randn(40, 2048, seed=3)
    w = _randn(2048, seed=1)
    clean = sw.slimwise_norm(x, w, layer=layer)[0].clone()
    x[5, 7], x[17, 2047], x[33, 0] = NAN, math.inf, -math.inf
    y = sw.slimwise_norm(x, w, layer=layer)[0]
    keep = torch.ones(40, dtype=torch.bool, device=DEV)
    keep[[5, 17, 33]] = False
    assert torch.equal(y[keep], clean[keep]) and bool(torch.isnan(y[5]).all())


def _grad_reference(dy, x, w, mean, rstd):
    d, r = dy.double(), rstd.double()[:, None]
    n = (x.double() - (0.0 if mean is None else mean.double()[:, None])) * r
    g = d * w.double()
    m, m0 = (n * g).mean(1, keepdim=True), 0.0 if mean is None else g.mean(1, keepdim=True)
    dx = r * (g - m0 - n * m)
    size = g.abs() + (0.0 if mean is None else g.abs().mean(1, keepdim=True)) + n.abs() * (n * g).abs().mean(1, keepdim=True)
    return dx, (d * n).sum(0), d.sum(0), r * size * 2 * ROW, (d * n).abs().sum(0), d.abs().sum(0)


def _check_norm_grad(dy, x, w, layer, **kw):
    _, mean, rstd = sw.slimwise_norm(x, w, layer=layer)
    dx, dw, db = sw.slimwise_norm_grad(dy, x, w, rstd, mean=mean, **kw)
    wx, ww, wb, tol, sw_, sb = _grad_reference(dy, x, w, mean, rstd)
    _within(dx, wx, wx.abs() * _half(x.dtype) + tol * 1.01 + torch.finfo(x.dtype).tiny)
    # a CTA's rows, its eight groups, a 32nd of the CTAs' sums, the 32 parts; two roundings of a term
    rows, hidden = x.shape
    ctas = 152 * (2 if hidden <= 256 else 4 if hidden <= 1024 else 2 if hidden <= 2048 else 1)
    chain = (math.ceil(rows / min(ctas, max(rows, 1))) + 4 + 8 + math.ceil(ctas / 32) + 32 + 3) * 2.0 ** -24
    _within(dw, ww, sw_ * chain + 1e-37)
    if layer and kw.get("grad_bias", True):
        _within(db, wb, sb * chain + 1e-37)
    else:
        assert db is None
    return dx, dw, db


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hidden", LENGTHS)
def test_norm_grad(hidden, dtype, layer):
    x, _ = _rows(_randn(19, hidden, seed=hidden) * 2 + 0.5, dtype)
    dy, _ = _rows(_randn(19, hidden, seed=hidden + 1), dtype)
    _check_norm_grad(dy, x, 1 + 0.2 * _randn(hidden, seed=1), layer)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hidden", [64, 300, 2048])
@pytest.mark.parametrize("rows", [1, 2, 7, 305, 1217, 5003])
def test_norm_grad_rows(rows, hidden, dtype):
    x, dy = _rows(_randn(rows, hidden, seed=rows), dtype)[0], _rows(_randn(rows, hidden, seed=2), dtype)[0]
    _check_norm_grad(dy, x, _randn(hidden, seed=1), True)
    _check_norm_grad(dy, x, _randn(hidden, seed=1), False)
    _check_norm_grad(dy, x, _randn(hidden, seed=1), True, grad_bias=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pads,start", [((1, 0, 3), 1), ((8, 0, 8), 0), ((2, 4, 6), 2), ((0, 5, 0), 0)])
def test_norm_grad_strides_and_bounds(pads, start, dtype):
    hidden = 1026
    x = _rows(_randn(9, hidden, seed=4), dtype, pad=pads[0], start=start)[0]
    dy = _rows(_randn(9, hidden, seed=5), dtype, pad=pads[1])[0]
    dx, flat = _rows(torch.zeros(9, hidden, device=DEV), dtype, pad=pads[2], start=start)
    outside = torch.isnan(flat).sum()
    _check_norm_grad(dy, x, _randn(hidden, seed=1), True, dx=dx)
    assert torch.isnan(flat).sum() == outside


def test_norm_grad_of_no_rows():
    x = torch.empty((0, 64), device=DEV)
    dx, dw, db = sw.slimwise_norm_grad(x, x, torch.ones(64, device=DEV), torch.empty(0, device=DEV),
                                       mean=torch.empty(0, device=DEV))
    assert dx.shape == (0, 64) and bool((dw == 0).all()) and bool((db == 0).all())


def test_norm_grad_against_differences():
    # in fp32 with a step of 2^-7: the quotient's own error is the cubic term's and the sums' rounding
    x, w, b = _randn(3, 96, seed=1), 1 + 0.2 * _randn(96, seed=2), 0.1 * _randn(96, seed=3)
    dy = _randn(3, 96, seed=4)
    _, mean, rstd = sw.slimwise_norm(x, w, bias=b, layer=True)
    dx, dw, db = sw.slimwise_norm_grad(dy, x, w, rstd, mean=mean)
    f = lambda x, w, b: (sw.slimwise_norm(x, w, bias=b, layer=True)[0].double() * dy.double()).sum()
    step = 2.0 ** -7
    for k in (0, 17, 95):
        e = torch.zeros(96, device=DEV)
        e[k] = step
        for got, hi, lo in ((dw[k], f(x, w + e, b), f(x, w - e, b)), (db[k], f(x, w, b + e), f(x, w, b - e)),
                            (dx[1, k], f(x + e * torch.tensor([[0.0], [1.0], [0.0]], device=DEV), w, b),
                             f(x - e * torch.tensor([[0.0], [1.0], [0.0]], device=DEV), w, b))):
            assert abs(float(got) - float(hi - lo) / (2 * step)) < 2e-3


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
def _ids(n, vocab, seed, bad=True):
    """Log-uniform ids, some padding, and (bad) some past the table."""
    g = _gen(seed)
    ids = (vocab ** torch.rand(n, generator=g, device=DEV)).long().clamp(max=vocab) - 1
    ids = torch.randperm(vocab, generator=g, device=DEV)[ids].int()
    ids[::16] = -1
    if bad and n > 5:
        ids[5::97] = vocab + 3
    return ids


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hidden,pad,start", [(1, 0, 0), (7, 1, 1), (64, 0, 0), (64, 3, 0), (1000, 8, 8), (2048, 0, 0),
                                              (2050, 0, 2), (5001, 0, 0), (16384, 0, 0)])
@pytest.mark.parametrize("rows", [1, 33, 700])
def test_embed(rows, hidden, pad, start, dtype):
    table = _rows(_randn(501, hidden, seed=1), dtype, pad=pad, start=start)[0]
    ids = _ids(rows, 501, seed=rows)
    scale = math.sqrt(hidden)
    want = torch.where((ids >= 0)[:, None], table[ids.clamp(0, 500).long()].float() * torch.tensor(scale, device=DEV), 0.0)
    want[ids >= 501] = NAN
    out, flat = _rows(torch.zeros(rows, hidden, device=DEV), dtype, pad=pad)
    gaps = torch.isnan(flat).sum()
    got = sw.slimwise_embed(table, ids, scale=scale, out=out)
    assert got is out and torch.equal(got.nan_to_num(nan=-777.0), want.to(dtype).nan_to_num(nan=-777.0))
    assert torch.isnan(flat).sum() == gaps + torch.isnan(want).sum()
    assert torch.equal(sw.slimwise_embed(table, ids, scale=scale).nan_to_num(nan=-777.0), got.nan_to_num(nan=-777.0))


def _check_embed_grad(grad, ids, vocab, out, scale=1.0, accumulate=False):
    old = out.clone().double()
    assert sw.slimwise_embed_grad(grad, ids, out, scale=scale, accumulate=accumulate) is out
    live = (ids >= 0) & (ids < vocab)
    at, g = ids[live].long(), grad[live].double()
    sums = torch.zeros((vocab, grad.shape[1]), dtype=torch.float64, device=DEV).index_add_(0, at, g)
    sizes = torch.zeros_like(sums).index_add_(0, at, g.abs())
    count = torch.zeros(vocab, dtype=torch.float64, device=DEV).index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    s32 = float(torch.tensor(scale))
    want = sums * s32 + (old if accumulate else 0.0)
    # within a piece of 32, then over the pieces; the scale's rounding and the addition's
    chain = (32 + count / 32 + 4).clamp(max=1 << 20)[:, None] * 2.0 ** -24
    _within(out, want, want.abs() * (_half(out.dtype) + 2.0 ** -23) + sizes * abs(s32) * chain)
    absent = count == 0
    assert torch.equal(out[absent].double(), old[absent] if accumulate else torch.zeros_like(old[absent]))


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("odtype", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,hidden,vocab", [(1, 64, 10), (31, 8, 1), (33, 1000, 3), (700, 257, 501), (5000, 2048, 777),
                                               (1021, 520, 40001), (64, 5001, 1000), (9000, 16, 262144),
                                               (500, 94, 30011), (500, 5, 30011), (100, 9, 5003), (2000, 333, 9001)])
def test_embed_grad(rows, hidden, vocab, dtype, odtype, accumulate):
    grad = _randn(rows, hidden, seed=rows).to(dtype)
    out = _randn(vocab, hidden, seed=3).to(odtype)
    _check_embed_grad(grad, _ids(rows, vocab, seed=2), vocab, out, scale=math.sqrt(hidden), accumulate=accumulate)


@pytest.mark.parametrize("kind", ["all_one", "all_padding", "blocks", "pairs", "ascending", "edges"])
@pytest.mark.parametrize("rows", [31, 32, 33, 64, 4097, 40000])
def test_embed_grad_orders(rows, kind):
    vocab, i = 513, torch.arange(rows, device=DEV)
    ids = {"all_one": i * 0 + 512, "all_padding": i * 0 - 1, "blocks": i // 32, "pairs": i // 2, "ascending": i,
           "edges": torch.where(i % 2 == 0, i * 0, i * 0 + 512)}[kind].remainder(vocab).int()
    if kind == "all_padding":
        ids.fill_(-5)
    _check_embed_grad(_randn(rows, 72, seed=1), ids, vocab, torch.full((vocab, 72), NAN, device=DEV))


@pytest.mark.parametrize("vocab", [511, 512, 513, 262143, 262144, 262145, 1 << 20])
def test_embed_grad_key_widths(vocab):
    ids = torch.randint(0, vocab, (6000,), generator=_gen(1), device=DEV).int()
    ids[:40] = vocab - 1
    ids[40:50] = vocab
    _check_embed_grad(_randn(6000, 8, seed=1), ids, vocab, torch.full((vocab, 8), NAN, device=DEV))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pads", [(1, 3), (8, 0), (0, 5), (8, 8)])
def test_embed_grad_strides_and_bounds(pads, dtype):
    grad = _rows(_randn(900, 136, seed=1), dtype, pad=pads[0], start=pads[0])[0]
    out, flat = _rows(torch.zeros(300, 136, device=DEV), BF16, pad=pads[1], start=pads[1])
    gaps = torch.isnan(flat).sum()
    _check_embed_grad(grad, _ids(900, 300, seed=1), 300, out)
    assert torch.isnan(flat).sum() == gaps


def test_embed_grad_is_the_same_every_time_and_of_no_rows_is_zero():
    grad, ids = _randn(20000, 256, seed=1).to(BF16), _ids(20000, 1000, seed=2)
    outs = [sw.slimwise_embed_grad(grad, ids, torch.empty((1000, 256), device=DEV)) for _ in range(4)]
    assert all(torch.equal(outs[0], o) for o in outs[1:])
    out = torch.full((10, 256), NAN, device=DEV)
    sw.slimwise_embed_grad(grad[:0], ids[:0], out)
    assert bool((out == 0).all())
    sw.slimwise_embed_grad(grad[:0], ids[:0], out.fill_(3.0), accumulate=True)
    assert bool((out == 3).all())


# ---------------------------------------------------------------------------
# the head's cross entropy
# ---------------------------------------------------------------------------
def _head(rows, width, vocab, seed, lean=4.0, ignored=0.1):
    g = _gen(seed)
    weight = (torch.randn((vocab, width), generator=g, device=DEV) * (1.5 / math.sqrt(width))).to(BF16)
    labels = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    hidden = (torch.randn((rows, width), generator=g, device=DEV) + lean / 2.25 * weight[labels].float()).to(BF16)
    labels = labels.int()
    labels[torch.rand(rows, generator=g, device=DEV) < ignored] = -100
    row_weight = 0.1 + torch.rand(rows, generator=g, device=DEV)
    return hidden, weight, labels, row_weight


def _check_loss(hidden, weight, labels, row_weight, dh_out=True, dw_out=True, **kw):
    loss, row, dh, dw = sw.slimwise_linear_loss(hidden, weight, labels, row_weight=row_weight, grad_hidden=dh_out,
                                                grad_weight=dw_out, **kw)
    rows, width = hidden.shape
    vocab = weight.shape[0]
    live = labels >= 0
    h, w = hidden.double().where(live[:, None], torch.zeros((), dtype=torch.float64, device=DEV)), weight.double()
    y = labels.clamp(min=0).long()[:, None]
    wt = torch.ones(rows, dtype=torch.float64, device=DEV) if row_weight is None else row_weight.double()
    wt = wt.where(live, torch.zeros_like(wt))
    z = h @ w.T
    # a logit: products of 16 are added to the accumulator at a time, to 23 bits of the largest
    # term; the label's own, in fp32: 8 * ceil(width / 256) products of a lane, 5 steps
    dz_ = (width / 16 + 16 + width / 32 + 16) * 2.0 ** -23 * (h.abs() @ w.abs().T).amax(1)
    lse = torch.logsumexp(z, 1)
    # log(1 + the others' share): of a nearly sure row too small for lse - z in 64 bits
    over = torch.logsumexp(z.scatter(1, y, -math.inf), 1) - z.gather(1, y)[:, 0]
    want = torch.where(live, over.clamp(min=0) + torch.log1p(torch.exp(-over.abs())), 0.0)
    # exponents are rounded twice, 2^-22 for each exponential, sums of at most 128 + 64 + 64 terms
    sums = 2 * dz_ + z.abs().amax(1) * 2.0 ** -22 + 2.0 ** -21 + 300 * 2.0 ** -24
    tol = torch.where(live, sums * want.clamp(max=1.0) + want * 2.0 ** -22 + dz_ * 0, 0.0)
    _within(row, want, tol)
    _within(loss, (want * wt).sum().reshape(1), (tol * wt).sum() + (want * wt).sum() * 2.0 ** -23)
    p = torch.exp(z - lse[:, None])
    p.scatter_add_(1, y, -torch.ones_like(want)[:, None])
    # 1 - p of the label from the others' sum, which cancels nothing
    others = torch.exp(z - lse[:, None]).scatter(1, y, 0.0).sum(1)
    p.scatter_(1, y, -others[:, None])
    dz = p * wt[:, None]
    b = 2.0 ** -8
    # a numerator: rounded (the label's: not, but the others then take over its rounding),
    # and off by what its exponent and the row's sum are
    off = dz.abs() * (2 * b + 2 * sums)[:, None]
    if dh is not None:
        want = dz @ w
        steps = (vocab / 16 + 128) * 2.0 ** -23
        _within(dh, want, (off + dz.abs() * steps) @ w.abs() + want.abs() * b + 1e-37)
        assert bool((dh[~live] == 0).all())
    if dw is not None:
        want = dz.T @ h
        steps = (rows / 16 + 16) * 2.0 ** -23 + b  # and the scaled row's rounding
        _within(dw, want, (off + dz.abs() * steps).T @ h.abs() + want.abs() * _half(dw.dtype) + 1e-37)
    return loss, row, dh, dw


@pytest.mark.parametrize("rows,width,vocab", [
    (1, 8, 1), (1, 64, 2), (3, 16, 7), (5, 128, 255), (17, 72, 256), (64, 64, 257), (255, 136, 1000), (256, 256, 513),
    (63, 40, 9), (64, 72, 511), (65, 200, 777), (128, 328, 1025), (129, 64, 600), (100, 2056, 130),
    (150, 520, 777), (640, 576, 1500), (890, 512, 300),
    (257, 264, 300), (300, 520, 2049), (513, 1032, 700), (64, 4096, 1500), (1021, 128, 5003), (40, 16384, 130)])
def test_linear_loss(rows, width, vocab):
    _check_loss(*_head(rows, width, vocab, seed=rows + vocab))


@pytest.mark.parametrize("rows,width,vocab", [(64, 1024, 32000), (700, 2048, 20011), (2000, 512, 65537), (3000, 256, 8192)])
def test_linear_loss_of_larger_sizes(rows, width, vocab):
    _check_loss(*_head(rows, width, vocab, seed=rows, lean=12.0))


@pytest.mark.parametrize("dh,dw", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("rows,width,vocab", [(1, 8, 1), (5, 64, 300), (300, 520, 2049), (1021, 128, 5003)])
def test_linear_loss_parts(rows, width, vocab, dh, dw):
    head = _head(rows, width, vocab, seed=rows)
    got = _check_loss(*head, dh_out=dh, dw_out=dw)
    both = sw.slimwise_linear_loss(*head[:3], row_weight=head[3])
    if dh:
        assert torch.equal(got[2], both[2])
    if dw:
        assert torch.equal(got[3], both[3])


def test_linear_loss_without_row_weights_and_into_given_outputs():
    hidden, weight, labels, _ = _head(300, 264, 1000, seed=1)
    hs = torch.full((300, 272), NAN, dtype=BF16, device=DEV)
    ws = torch.full((1000, 280), NAN, dtype=BF16, device=DEV)
    hs[:, :264], ws[:, :264] = hidden, weight
    dh = torch.full((300, 280), NAN, dtype=BF16, device=DEV)
    dw = torch.full((1000, 268), NAN, device=DEV)
    got = _check_loss(hs[:, :264], ws[:, :264], labels, None, dh_out=dh[:, :264], dw_out=dw[:, :264])
    assert bool(torch.isnan(dh[:, 264:]).all()) and bool(torch.isnan(dw[:, 264:]).all())
    plain = sw.slimwise_linear_loss(hidden, weight, labels)
    assert torch.equal(plain[2], got[2]) and torch.equal(plain[1], got[1])
    assert torch.equal(plain[3], got[3].to(BF16))


def test_linear_loss_rows_without_labels():
    hidden, weight, labels, wt = _head(300, 64, 500, seed=1, ignored=0.0)
    clean = _check_loss(hidden, weight, torch.where(torch.arange(300, device=DEV) % 3 == 0, -1, labels).int(), wt)
    # whatever those rows and weights hold
    hidden[::3], wt[::3] = NAN, math.inf
    ids = torch.where(torch.arange(300, device=DEV) % 3 == 0, -1, labels).int()
    again = sw.slimwise_linear_loss(hidden, weight, ids, row_weight=wt)
    assert all(torch.equal(a, b) for a, b in zip(clean, again))
    loss, row, dh, dw = sw.slimwise_linear_loss(hidden, weight, torch.full_like(ids, -1), row_weight=wt)
    assert float(loss) == 0 and all(bool((x == 0).all()) for x in (row, dh, dw))
    loss, row, _, _ = sw.slimwise_linear_loss(hidden, weight, torch.full_like(ids, -1), grad_hidden=False,
                                              grad_weight=False)
    assert float(loss) == 0 and bool((row == 0).all())
    loss, row, dh, dw = sw.slimwise_linear_loss(hidden[:0], weight, ids[:0])
    assert float(loss) == 0 and dh.shape == (0, 64) and bool((dw == 0).all())


@pytest.mark.parametrize("width,rows", [(64, 700), (512, 595)])
def test_linear_loss_of_labels_that_are_sure_or_impossible(width, rows):
    # label's logit 40 above the others, as high as they, and 50, 70, 100 and 500 below the largest
    vocab = 3000
    weight = torch.zeros((vocab, width), dtype=BF16, device=DEV)
    weight[:, 1:] = (_randn(vocab, width - 1, seed=1) * 0.1).to(BF16)
    weight[5, 0], weight[2000, 0] = 1.0, -1.0
    hidden = (_randn(rows, width, seed=2) * 0.3).to(BF16)
    scale = torch.tensor([40.0, 0.0, 25.0, 35.0, 50.0, 250.0, 3.0], device=DEV).repeat(rows // 7)
    hidden[:, 0] = scale.to(BF16)
    labels = torch.full((rows,), 2000, dtype=torch.int32, device=DEV)
    labels[::7] = 5
    wt = 0.1 + torch.rand(rows, generator=_gen(3), device=DEV)
    _check_loss(hidden, weight, labels, wt)
    _check_loss(hidden, weight, labels, wt, dh_out=False, dw_out=False)
    # one such row among others: only its tile is taken again
    labels[:] = 7
    labels[300] = 2000
    _check_loss(hidden, weight, labels, wt)
    # few rows
    for n in (7, 100):
        labels[:n] = 2000
        _check_loss(hidden[:n], weight, labels[:n], wt[:n])
        _check_loss(hidden[:n], weight, labels[:n], wt[:n], dh_out=False, dw_out=False)


def test_linear_loss_of_what_is_no_number_and_of_labels_outside():
    hidden, weight, labels, wt = _head(600, 64, 700, seed=1, ignored=0.0)
    clean = sw.slimwise_linear_loss(hidden, weight, labels, row_weight=wt)
    labels[3], hidden[500, 5] = 700, NAN
    loss, row, dh, dw = sw.slimwise_linear_loss(hidden, weight, labels, row_weight=wt)
    bad = torch.zeros(600, dtype=torch.bool, device=DEV)
    bad[[3, 500]] = True
    assert bool(torch.isnan(row[bad]).all()) and bool(torch.isnan(dh[bad]).all()) and bool(torch.isnan(loss).all())
    assert torch.equal(row[~bad], clean[1][~bad]) and torch.equal(dh[~bad], clean[2][~bad])
    assert bool(torch.isnan(dw).all())
    row = sw.slimwise_linear_loss(hidden, weight, labels, grad_hidden=False, grad_weight=False)[1]
    assert torch.equal(torch.isnan(row), bad)


def test_linear_loss_against_differences():
    hidden, weight, labels, wt = _head(40, 64, 300, seed=1)
    _, _, dh, dw = sw.slimwise_linear_loss(hidden, weight, labels, row_weight=wt, grad_weight=torch.empty(300, 64, device=DEV))
    g = _gen(9)
    # along random directions of whole steps of bf16 sums: exact inputs, quotient against 64 bits
    for got, x, other in ((dh, hidden, 0), (dw, weight, 1)):
        d = torch.randint(-1, 2, x.shape, generator=g, device=DEV).double() * 2.0 ** -4
        def f(v):
            h, w = (v, weight.double()) if other == 0 else (hidden.double(), v)
            z = h @ w.T
            l = torch.logsumexp(z, 1) - z.gather(1, labels.clamp(min=0).long()[:, None])[:, 0]
            return (l * wt.double())[labels >= 0].sum()
        e = 1e-5
        slope = (f(x.double() + e * d) - f(x.double() - e * d)) / (2 * e)
        # 64 bits on one side; bf16's half steps of numerators, scaled rows and results on the other
        assert abs(float((got.double() * d).sum() - slope)) <= 4 * 2.0 ** -8 * float((got.double().abs() * d.abs()).sum())


@pytest.mark.parametrize("labelled", [1.0, 0.4])
def test_linear_loss_in_chunks(labelled):
    # more numerators than the workspace holds at once; a chunk without rows where few have labels
    rows, width, vocab = 3100, 16, 393216
    hidden, weight, labels, wt = _head(rows, width, vocab, seed=5, ignored=1.0 - labelled)
    loss, row, dh, dw = sw.slimwise_linear_loss(hidden, weight, labels, row_weight=wt)
    # the same numerators and scaled rows as of its parts, summed in another order: fp32 chains
    live = labels >= 0
    dz = torch.softmax(hidden.float() @ weight.float().T, 1)
    dz.scatter_add_(1, labels.clamp(min=0).long()[:, None], torch.ones((rows, 1), device=DEV))
    dz *= (wt * live)[:, None]
    dh_size, dw_size = dz @ weight.float().abs(), dz.T @ hidden.float().abs()
    total = torch.zeros((vocab, width), dtype=torch.float64, device=DEV)
    for a in range(0, rows, 775):
        part = sw.slimwise_linear_loss(hidden[a:a + 775], weight, labels[a:a + 775], row_weight=wt[a:a + 775],
                                       grad_weight=torch.empty((vocab, width), device=DEV))
        assert torch.equal(row[a:a + 775], part[1])
        want = part[2].double()
        _within(dh[a:a + 775], want, 2.0 ** -7 * want.abs() + (vocab / 16 + 128) * 2.0 ** -23 * dh_size[a:a + 775])
        total += part[3].double()
    _within(dw, total, 2.0 ** -8 * total.abs() + (rows / 16 + 32) * 2.0 ** -22 * dw_size + 1e-37)


def test_linear_loss_of_many_rows():
    # labels counted in blocks first
    rows, width, vocab = 70001, 16, 300
    hidden, weight, labels, wt = _head(rows, width, vocab, seed=8, ignored=0.3)
    _check_loss(hidden, weight, labels, wt)
    _check_loss(hidden, weight, labels, None, dh_out=False, dw_out=False)


def test_linear_loss_is_the_same_every_time():
    head = _head(1500, 264, 9001, seed=1)
    runs = [sw.slimwise_linear_loss(*head[:3], row_weight=head[3]) for _ in range(4)]
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))
    ws = torch.empty(sw.slimwise_linear_loss_workspace_size(1500, 264, 9001), dtype=torch.uint8, device=DEV).fill_(255)
    got = sw.slimwise_linear_loss(*head[:3], row_weight=head[3], workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(runs[0], got))
    assert sw.slimwise_moe_device_status(ws) == 0


# ---------------------------------------------------------------------------
# offsets past 32 bits
# ---------------------------------------------------------------------------
def test_embed_offsets_past_32_bits():
    vocab, hidden = 300000, 8192  # 2.4e9 elements
    table = torch.zeros((vocab, hidden), dtype=BF16, device=DEV)
    table[-3:] = _randn(3, hidden, seed=1).to(BF16)
    ids = torch.tensor([vocab - 1, 0, vocab - 3, -1, vocab - 1], dtype=torch.int32, device=DEV)
    out = sw.slimwise_embed(table, ids)
    assert torch.equal(out[[0, 2, 4]], table[[vocab - 1, vocab - 3, vocab - 1]]) and bool((out[[1, 3]] == 0).all())
    grad = out.clone()
    table.fill_(NAN)
    sw.slimwise_embed_grad(grad, ids, table)
    assert torch.equal(table[-1], (2 * grad[0].float()).to(BF16)) and torch.equal(table[-3], grad[2])
    assert bool((table[:-3] == 0).all()) and bool((table[-2] == 0).all())


def test_norm_offsets_past_32_bits():
    rows, hidden = 300000, 8192
    x = torch.ones((rows, hidden), dtype=BF16, device=DEV)
    x[-4:] = _randn(4, hidden, seed=1).to(BF16)
    w = 1 + 0.1 * _randn(hidden, seed=2)
    y, _, rstd = sw.slimwise_norm(x, w)
    few = sw.slimwise_norm(x[-4:].clone(), w)
    assert torch.equal(y[-4:], few[0]) and torch.equal(rstd[-4:], few[2])
    dx = sw.slimwise_norm_grad(x, x, w, rstd, dx=y)[0]
    assert torch.equal(dx[-4:], sw.slimwise_norm_grad(x[-4:].clone(), x[-4:].clone(), w, few[2])[0])


def test_linear_loss_offsets_past_32_bits():
    vocab, width = 393216, 8192
    weight = torch.zeros((vocab, width), dtype=BF16, device=DEV)
    weight[-700:] = (_randn(700, width, seed=1) * 0.05).to(BF16)
    hidden = _randn(3, width, seed=2).to(BF16)
    labels = torch.tensor([vocab - 1, vocab - 500, 7], dtype=torch.int32, device=DEV)
    dw = torch.full((vocab, width), NAN, dtype=BF16, device=DEV)
    loss, row, dh, _ = sw.slimwise_linear_loss(hidden, weight, labels, grad_weight=dw)
    z = torch.zeros((3, vocab), dtype=torch.float64, device=DEV)
    z[:, -700:] = hidden.double() @ weight[-700:].double().T
    p = torch.softmax(z, 1)
    want = torch.logsumexp(z, 1) - z.gather(1, labels.long()[:, None])[:, 0]
    # logits of up to 25, off by 2^-17 of themselves
    assert bool(((row.double() - want).abs() <= 25 * 2.0 ** -17).all())
    p[torch.arange(3), labels.long()] -= 1
    for v in (7, vocab - 1, vocab - 500, vocab - 2, 12345):
        ref = p[:, v] @ hidden.double()
        size = p[:, v].abs() @ hidden.double().abs()
        assert bool(((dw[v].double() - ref).abs() <= 3 * 2.0 ** -8 * size).all())
    ref = p[:, -700:] @ weight[-700:].double()
    size = p[:, -700:].abs() @ weight[-700:].double().abs()
    assert bool(((dh.double() - ref).abs() <= 4 * 2.0 ** -8 * size).all())


def _workspaces(nbytes):
    """The same number of bytes holding zeros, NaN in bf16 and fp32, and infinities in
    bf16, each before bytes that no call may touch."""
    for fill in (0x0000, 0xFFFF, 0x7F80):
        words = torch.full(((nbytes + 4096) // 2,), fill, dtype=torch.int32, device=DEV).to(torch.int16)
        raw = words.view(torch.uint8)
        yield raw[:nbytes], lambda raw=raw, fill=fill: bool(((raw[nbytes:].view(torch.int16).int() & 0xFFFF) == fill).all())


@pytest.mark.parametrize("labelled", [1.0, 0.86, 0.5, 0.02])
@pytest.mark.parametrize("width,vocab", [(1024, 2003), (264, 300)])
@pytest.mark.parametrize("rows", [1, 31, 64, 65, 90, 96, 97, 128, 129, 150, 290, 300, 417, 500, 700, 870, 1000])
def test_linear_loss_does_not_depend_on_what_the_workspace_holds(rows, width, vocab, labelled):
    hidden, weight, labels, row_weight = _head(rows, width, vocab, seed=rows)
    labels = torch.where(labels < 0, 0, labels)
    labels[int(math.ceil(rows * labelled)):] = -1
    labels = labels[torch.randperm(rows, generator=_gen(rows), device=DEV)].contiguous()
    for dh, dw in ((True, True), (False, True), (True, False), (False, False)):
        first = None
        for ws, untouched in _workspaces(sw.slimwise_linear_loss_workspace_size(rows, width, vocab, dh, dw)):
            got = sw.slimwise_linear_loss(hidden, weight, labels, row_weight, grad_hidden=dh, grad_weight=dw, workspace=ws)
            got = [t.clone() for t in got if t is not None]
            first = first or got
            assert untouched()
            assert all(torch.equal(x, y) and bool(x.isfinite().all()) for x, y in zip(got, first))


@pytest.mark.parametrize("rows,hidden,vocab", [(1, 8, 3), (100, 64, 50), (700, 257, 501), (5000, 1000, 777)])
def test_embed_and_norm_gradients_do_not_depend_on_what_the_workspace_holds(rows, hidden, vocab):
    grad, x = _randn(rows, hidden, seed=1).to(BF16), _randn(rows, hidden, seed=2).to(BF16)
    w, ids = _randn(hidden, seed=3), _ids(rows, vocab, seed=4)
    _, mean, rstd = sw.slimwise_norm(x, w, layer=True)
    first = None
    for ws, untouched in _workspaces(sw.slimwise_embed_grad_workspace_size(rows, hidden)):
        out = torch.empty((vocab, hidden), device=DEV)
        sw.slimwise_embed_grad(grad, ids, out, workspace=ws)
        first = out if first is None else first
        assert untouched() and torch.equal(out, first)
    first = None
    for ws, untouched in _workspaces(sw.slimwise_norm_grad_workspace_size(rows, hidden)):
        got = sw.slimwise_norm_grad(grad, x, w, rstd, mean, workspace=ws)
        first = first or got
        assert untouched() and all(torch.equal(a, b) for a, b in zip(got, first))


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("pad,start", [(0, 0), (0, 3), (1, 0), (2, 5), (5, 7), (8, 1)])
@pytest.mark.parametrize("rows,hidden", [
    (1, 1), (1, 15), (2, 3), (7, 5), (8, 7), (9, 9), (20, 13), (63, 17), (64, 250), (65, 255), (300, 257), (3000, 99),
    (11, 511), (700, 513), (40, 1001), (333, 1023), (17, 2047), (700, 2041), (30, 4001), (9, 4095), (400, 4093),
    (21, 5001), (200, 8191), (33, 8193), (310, 16383), (5, 16381)])
def test_norm_of_rows_that_start_alike_in_all_tensors(rows, hidden, pad, start, layer):
    make = lambda values: _rows(values, BF16, pad=pad, start=start)
    x, dy = make(_randn(rows, hidden, seed=1) * 2 + 0.5)[0], make(_randn(rows, hidden, seed=2))[0]
    w, b = 1 + 0.2 * _randn(hidden, seed=3), 0.1 * _randn(hidden, seed=4)
    (y, around), (dx, beside) = make(torch.zeros(rows, hidden, device=DEV)), make(torch.zeros(rows, hidden, device=DEV))
    outside = int(torch.isnan(around).sum())
    _check_norm(x, w, b, layer, y=y)
    _check_norm_grad(dy, x, w, layer, dx=dx)
    assert int(torch.isnan(around).sum()) == outside and int(torch.isnan(beside).sum()) == outside
    again = sw.slimwise_norm(x, w, b, layer)[0]  # (the output elsewhere: other widths may round otherwise)
    assert float((again.float() - y.float()).abs().max()) <= 2.0 ** -7 * float(y.float().abs().max())


def test_norm_of_rows_that_start_alike_keeps_nan_and_infinities_in_their_rows():
    x = _rows(_randn(70, 1003, seed=1), BF16)[0]
    good = sw.slimwise_norm(x, torch.ones(1003, device=DEV), layer=True)[0].clone()
    x[3, 0], x[10, 1002], x[33, 500] = NAN, math.inf, -math.inf
    y = sw.slimwise_norm(x, torch.ones(1003, device=DEV), layer=True)[0]
    bad = torch.zeros(70, dtype=torch.bool, device=DEV)
    bad[[3, 10, 33]] = True
    assert torch.equal(y[~bad], good[~bad]) and bool(y[bad].isnan().any(1).all())
