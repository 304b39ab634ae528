"""The operators over vocabulary logits against plain evaluations in 64 bits.

Tolerances follow from the kernels' arithmetic.  A sum of exponentials has a
relative error of at most MASS = 2^-15 (fp32 sums of at most 2^9 terms in a
thread, exponents rounded twice, exp2 to 2^-22); a logarithm of a ratio of two
such sums is then off by at most twice that, a gradient element by that share
of the magnitudes it is the difference of.  Ids and tokens are exact.
"""
import math

import numpy as np
import pytest
import torch

import paper_2609_34117_gb300 as sw

pytestmark = pytest.mark.gpu
DEV = "cuda"
MASS = 2.0 ** -15
TYPES = [torch.bfloat16, torch.float32]
INF = math.inf


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sw.build.build()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(rows, vocab, dtype, seed, pad=0, start=0, scale=3.0):
    """Logits with `pad` elements between rows, the first `start` elements into
    its allocation; what lies outside the rows is NaN."""
    g = _gen(seed)
    flat = torch.full((start + rows * (vocab + pad),), math.nan, dtype=dtype, device=DEV)
    z = flat[start:].view(rows, vocab + pad)[:, :vocab]
    z.copy_(torch.randn((rows, vocab), generator=g, device=DEV) * scale)
    return z


def _order(z):
    """Ids by (value descending, id ascending), in 64 bits."""
    return torch.sort(-(z.double() + 0.0), dim=1, stable=True)[1]


# ---------------------------------------------------------------------------
# top logits
# ---------------------------------------------------------------------------
def _check_top(z, k, tau, **kw):
    ids, logp, rest = sw.slimwise_top_logits(z, k, temperature=tau, **kw)
    ref = _order(z)[:, :k]
    assert torch.equal(ids.long(), ref)
    lp = torch.log_softmax(z.double() / tau, 1)
    want = lp.gather(1, ref)
    want_rest = torch.logsumexp(lp.scatter(1, ref, -INF), 1)
    for got, w in ((logp, want), (rest, want_rest)):
        got = got.double()
        fin = torch.isfinite(w)
        assert torch.equal(torch.isfinite(got), fin)
        assert torch.equal(got[~fin], w[~fin])
        assert bool(((got - w).abs()[fin] <= 2 * MASS + 2.0 ** -21 * w.abs()[fin]).all())
    return ids, logp, rest


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,k", [
    (1, 1, 1), (3, 2, 2), (5, 7, 3), (2, 64, 64), (17, 1000, 8), (3, 1031, 256), (1, 8193, 64),
    (2, 50001, 20), (1, 131072, 64), (1, 262144, 256), (1, 393216, 100), (700, 4097, 64),
])
def test_top_logits(rows, vocab, k, dtype):
    _check_top(_rows(rows, vocab, dtype, seed=rows + vocab), k, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tau", [0.05, 0.5, 2.0, 30.0])
def test_top_logits_temperatures(tau, dtype):
    _check_top(_rows(9, 20011, dtype, seed=3), 64, tau)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,start", [(1, 0), (3, 5), (8, 1), (13, 7)])
def test_top_logits_rows_that_start_anywhere(pad, start, dtype):
    _check_top(_rows(6, 9001, dtype, seed=4, pad=pad, start=start), 64, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [1, 64, 256])
@pytest.mark.parametrize("vocab", [257, 20000, 140001])
def test_top_logits_ties(vocab, k, dtype):
    # equal everywhere; a few values only; the largest all in one place; signed zeros
    z = torch.zeros((5, vocab), dtype=dtype, device=DEV)
    z[1] = torch.randint(0, 3, (vocab,), generator=_gen(1), device=DEV).to(dtype)
    z[2, vocab // 2:vocab // 2 + 128] = 4.0
    z[3] = torch.where(torch.arange(vocab, device=DEV) % 2 == 0, -0.0, 0.0).to(dtype)
    z[4] = torch.arange(vocab, device=DEV).div(64, rounding_mode="floor").remainder(50).to(dtype)
    _check_top(z, k, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_top_logits_sorted_rows(dtype):
    # every window beats all before it, or none does
    up = torch.linspace(-20.0, 20.0, 60000, device=DEV).to(dtype)
    _check_top(torch.stack([up, up.flip(0)]), 256, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_top_logits_masked(dtype):
    low = torch.finfo(dtype).min
    z = _rows(4, 30000, dtype, seed=6)
    z[0, 10:] = -INF               # fewer than k left
    z[1, 100:] = low               # masked with the type's lowest value
    z[2, :29990] = -INF
    z[3, 1:] = -INF                # one left
    _check_top(z, 64, 1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_top_logits_no_distribution(dtype):
    z = _rows(4, 30000, dtype, seed=7)
    z[0] = -INF
    z[1, 17] = math.nan
    z[2, 29999] = INF
    ids, logp, rest = sw.slimwise_top_logits(z, 64)
    for t in range(3):
        assert bool(torch.isnan(logp[t]).all()) and bool(torch.isnan(rest[t]))
    assert bool(((ids >= -1) & (ids < 30000)).all())
    one = sw.slimwise_top_logits(z[3:], 64)
    assert torch.equal(ids[3:], one[0]) and torch.equal(logp[3:], one[1])


# ---------------------------------------------------------------------------
# distillation loss
# ---------------------------------------------------------------------------
def _targets(z, k, tau, seed, noise=1.0):
    """A teacher near the student z: its list, log-probabilities and rest."""
    t = z.double() + torch.randn(z.shape, generator=_gen(seed), device=DEV).double() * noise
    lp = torch.log_softmax(t / tau, 1)
    ids = _order(lp)[:, :k]
    rest = torch.logsumexp(lp.scatter(1, ids, -INF), 1)
    return ids.to(torch.int32), lp.gather(1, ids).float(), rest.float()


def _loss64(z, labels, ids, logp, rest, alpha, tau):
    """Row losses from the definition, in 64 bits; z may require a gradient."""
    live = labels >= 0
    ce = -torch.log_softmax(z, 1).gather(1, labels.clamp(min=0).long()[:, None])[:, 0]
    lq = torch.log_softmax(z / tau, 1)
    has = ids >= 0
    at = ids.clamp(min=0).long()
    P = torch.where(has, logp.double().exp(), 0.0)
    mark = torch.zeros((z.shape[0], z.shape[1] + 1), dtype=torch.bool, device=z.device)
    mark.scatter_(1, torch.where(has, at, z.shape[1]), True)
    out = lq.masked_fill(mark[:, :-1], -INF)
    lQ = torch.logsumexp(out, 1)
    r = rest.double().exp()
    kl = torch.where(P > 0, P * (logp.double() - lq.gather(1, at)), 0.0).sum(1)
    kl = kl + torch.where(r > 0, r * (rest.double() - lQ), 0.0)
    return torch.where(live, alpha * ce + (1 - alpha) * tau * tau * kl, 0.0), mark[:, :-1], P, r, lQ


def _check_loss(z, labels, ids, logp, rest, alpha, tau, weight=None, **kw):
    loss, row, grad = sw.slimwise_distill_loss(z, labels, ids, logp, rest, alpha=alpha,
                                               temperature=tau, row_weight=weight, **kw)
    z64 = z.double().requires_grad_(True)
    want, mark, P, r, lQ = _loss64(z64, labels, ids, logp, rest, alpha, tau)
    w = torch.ones(z.shape[0], device=DEV, dtype=torch.float64) if weight is None else weight.double()
    (want * w).sum().backward()
    g = z64.grad
    want = want.detach()
    live = (labels >= 0)[:, None]
    with torch.no_grad():
        p, q = torch.softmax(z64, 1), torch.softmax(z64 / tau, 1)
        M = P.sum(1, keepdim=True) + r[:, None]
        beta = (1 - alpha) * tau
        share = torch.where(mark, torch.zeros_like(q).scatter_add_(1, ids.clamp(min=0).long(), P),
                            torch.where(r > 0, r * torch.exp(-lQ), 0.0)[:, None] * q)
        onehot = torch.zeros_like(q).scatter_(1, labels.clamp(min=0).long()[:, None], 1.0)
        size = w.abs()[:, None] * (alpha * (p + onehot) + beta * (M * q + share)) * live
        tol_row = 2 * MASS * (alpha + beta * tau * M[:, 0]) * (1 + 2.0 ** -5 * torch.log(torch.tensor(z.shape[1] * 1.0)))
        step = 2.0 ** -8 if z.dtype == torch.bfloat16 else 2.0 ** -22
        tol = 2 * MASS * size + step * g.abs() + 1e-38
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(row), fin)
    assert bool(((row.double() - want).abs() <= tol_row + 2.0 ** -20 * want.abs())[fin].all())
    total = (want * w).sum()
    if bool(fin.all()):
        assert abs(float(loss) - float(total)) <= float(((tol_row + 2.0 ** -20 * want.abs()) * w.abs()).sum()) + 1e-30
    if grad is not None:
        # a subnormal bf16 gradient has steps of its own
        tol = tol + (2.0 ** -133 if z.dtype == torch.bfloat16 else 2.0 ** -149)
        bad = (grad.double() - g).abs() > tol
        assert not bool(bad.any()), (int(bad.sum()), float(((grad.double() - g).abs() / tol).max()))
    return loss, row, grad


def _labels(z, seed):
    return torch.randint(0, z.shape[1], (z.shape[0],), generator=_gen(seed), device=DEV,
                         dtype=torch.int32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,k", [
    (1, 1, 1), (3, 2, 1), (3, 2, 2), (5, 7, 3), (2, 64, 64), (17, 1000, 8), (3, 1031, 256),
    (1, 8193, 64), (2, 50001, 20), (1, 262144, 64), (1, 393216, 100), (700, 4097, 64),
])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distill_loss(rows, vocab, k, dtype, tau):
    z = _rows(rows, vocab, dtype, seed=rows + vocab)
    _check_loss(z, _labels(z, 1), *_targets(z, k, tau, 2), alpha=0.1, tau=tau)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("alpha", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("tau", [0.5, 1.0])
def test_distill_loss_weights_and_alphas(alpha, tau, dtype):
    z = _rows(12, 5003, dtype, seed=8)
    w = torch.rand(12, generator=_gen(9), device=DEV) * 2 - 0.5
    _check_loss(z, _labels(z, 3), *_targets(z, 64, tau, 4), alpha=alpha, tau=tau, weight=w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,start,gpad,gstart", [(0, 0, 1, 0), (3, 5, 3, 5), (8, 1, 0, 0), (0, 0, 0, 3),
                                                   (7, 0, 23, 0)])
def test_distill_loss_rows_that_start_anywhere(pad, start, gpad, gstart, dtype):
    rows, vocab = 5, 9001
    z = _rows(rows, vocab, dtype, seed=5, pad=pad, start=start)
    flat = torch.full((gstart + rows * (vocab + gpad) + 64,), 7.0, dtype=dtype, device=DEV)
    g = flat[gstart:gstart + rows * (vocab + gpad)].view(rows, vocab + gpad)
    _check_loss(z, _labels(z, 3), *_targets(z, 64, 1.0, 4), alpha=0.1, tau=1.0, grad=g[:, :vocab])
    assert bool((flat[:gstart] == 7.0).all()) and bool((flat[gstart + rows * (vocab + gpad):] == 7.0).all())
    assert bool((g[:, vocab:] == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("vocab,gpad,gstart", [(3, 2, 1), (17, 0, 3), (70001, 3, 1), (262147, 7, 5), (393216, 1, 0)])
def test_distill_loss_gradient_rows_of_another_alignment(vocab, gpad, gstart, tau, dtype):
    rows = 3
    z = _rows(rows, vocab, dtype, seed=15)
    args = (_labels(z, 3),) + _targets(z, min(64, vocab - 1), tau, 4)
    want = sw.slimwise_distill_loss(z, *args, alpha=0.1, temperature=tau)
    flat = torch.full((gstart + rows * (vocab + gpad) + 64,), 7.0, dtype=dtype, device=DEV)
    g = flat[gstart:gstart + rows * (vocab + gpad)].view(rows, vocab + gpad)
    got = _check_loss(z, *args, alpha=0.1, tau=tau, grad=g[:, :vocab])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert bool((flat[:gstart] == 7.0).all()) and bool((flat[gstart + rows * (vocab + gpad):] == 7.0).all())
    assert bool((g[:, vocab:] == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [20000, 236985, 300007, 393216])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_distill_loss_long_rows_over_many_ctas(vocab, tau, dtype):
    z = _rows(160, vocab, dtype, seed=16)
    _check_loss(z, _labels(z, 3), *_targets(z, 64, tau, 4), alpha=0.1, tau=tau)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1000, 70001])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_distill_loss_in_place(vocab, dtype, tau):
    z = _rows(6, vocab, dtype, seed=10)
    args = (_labels(z, 3),) + _targets(z, 64, tau, 4)
    loss, row, grad = sw.slimwise_distill_loss(z, *args, temperature=tau)
    own = z.clone()
    loss2, row2, grad2 = sw.slimwise_distill_loss(own, *args, temperature=tau, grad=own)
    assert grad2.data_ptr() == own.data_ptr()
    assert torch.equal(loss, loss2) and torch.equal(row, row2) and torch.equal(grad, grad2)


@pytest.mark.parametrize("dtype", TYPES)
def test_distill_loss_without_gradient_is_the_same_loss(dtype):
    z = _rows(6, 30011, dtype, seed=11)
    args = (_labels(z, 3),) + _targets(z, 64, 1.0, 4)
    a, b = sw.slimwise_distill_loss(z, *args), sw.slimwise_distill_loss(z, *args, grad=False)
    assert b[2] is None
    assert torch.allclose(a[1], b[1], rtol=0, atol=4 * MASS)


@pytest.mark.parametrize("dtype", TYPES)
def test_distill_loss_rows_without_label(dtype):
    z = _rows(5, 4001, dtype, seed=12)
    labels = _labels(z, 3)
    labels[1], labels[3] = -100, -1
    z[1, 5] = math.nan                       # an ignored row may hold anything
    args = _targets(torch.nan_to_num(z), 64, 1.0, 4)
    loss, row, grad = sw.slimwise_distill_loss(z, labels, *args)
    for t in (1, 3):
        assert float(row[t]) == 0.0 and not bool(grad[t].any())
    keep = torch.tensor([0, 2, 4], device=DEV)
    _check_loss(z[keep], labels[keep], *[a[keep] for a in args], alpha=0.1, tau=1.0)
    every = torch.full_like(labels, -100)
    loss, row, grad = sw.slimwise_distill_loss(z, every, *args)
    assert float(loss) == 0.0 and not bool(grad.any())


@pytest.mark.parametrize("dtype", TYPES)
def test_distill_loss_short_lists(dtype):
    z = _rows(4, 4001, dtype, seed=13)
    ids, logp, rest = _targets(z, 64, 1.0, 4)
    ids[0, 10:] = -1                         # a shorter list
    ids[1] = -1                              # no list: only the rest
    rest[1] = 0.0
    rest[2] = -INF                           # no rest
    logp[3, 32:] = -INF                      # entries without mass stay in the list
    _check_loss(z, _labels(z, 3), ids, logp, rest, alpha=0.1, tau=1.0)
    _check_loss(z, ids[:, 0].clamp(min=0).contiguous(), ids, logp, rest, alpha=0.3, tau=2.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_distill_loss_residual_of_a_sure_student(dtype):
    # the list holds all but 1e-7 or less of the student's mass: the rest is summed, not a difference
    z = _rows(3, 20000, dtype, seed=14, scale=0.5)
    z[:, 77] += torch.tensor([18.0, 24.0, 30.0], device=DEV).to(dtype)
    ids, logp, rest = _targets(z, 20, 1.0, 4, noise=0.1)
    _check_loss(z, torch.full((3,), 77, dtype=torch.int32, device=DEV), ids, logp, rest, alpha=0.1,
                tau=1.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_distill_loss_masked_logits(dtype):
    low = torch.finfo(dtype).min
    z = _rows(3, 20000, dtype, seed=15)
    ids, logp, rest = _targets(z, 64, 1.0, 4)
    z[0, 15000:] = -INF
    z[1, 15000:] = low
    rest2 = rest.clone()
    keep = torch.zeros(20000, dtype=torch.bool, device=DEV)
    keep[:15000] = True
    has = keep[ids.long()]
    ids = torch.where(has, ids, -1)          # the teacher masks the same tokens
    _check_loss(z, torch.tensor([3, 4, 19999], dtype=torch.int32, device=DEV), ids.contiguous(), logp,
                rest2, alpha=0.1, tau=1.0)
    # a listed token without probability: infinite loss, finite gradient elsewhere
    z2 = z[:1].clone()
    first = int(ids[0][ids[0] >= 0][0])
    z2[0, first] = -INF
    loss, row, grad = sw.slimwise_distill_loss(z2, torch.tensor([3], dtype=torch.int32, device=DEV),
                                               ids[:1].contiguous(), logp[:1], rest2[:1])
    assert float(row[0]) == INF and bool(torch.isfinite(grad).all())
    # nothing outside the list but the teacher expects some: infinite loss, no NaN
    z3 = torch.full((1, 500), -INF, dtype=dtype, device=DEV)
    z3[0, :4] = 1.0
    loss, row, grad = sw.slimwise_distill_loss(
        z3, torch.zeros(1, dtype=torch.int32, device=DEV),
        torch.arange(4, dtype=torch.int32, device=DEV)[None].contiguous(),
        torch.full((1, 4), math.log(0.2), device=DEV), torch.full((1,), math.log(0.2), device=DEV))
    assert float(row[0]) == INF and bool(torch.isfinite(grad).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_distill_loss_bad_rows_are_nan_and_alone(dtype):
    z = _rows(6, 20000, dtype, seed=16)
    args = list((_labels(z, 3),) + _targets(z, 64, 1.0, 4))
    good = sw.slimwise_distill_loss(z, *args)
    args[0] = args[0].clone()
    args[1] = args[1].clone()
    args[0][0] = 20000
    args[1][1, 63] = 20000
    args[1][2, 0] = 2 ** 31 - 1
    z[3, 100] = math.nan
    z[4] = -INF
    loss, row, grad = sw.slimwise_distill_loss(z, *args)
    for t in range(5):
        assert math.isnan(float(row[t])), t
        assert bool(torch.isnan(grad[t]).all()), t
    assert torch.equal(row[5], good[1][5]) and torch.equal(grad[5], good[2][5])
    assert math.isnan(float(loss))


@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_distill_gradient_against_differences(tau):
    z = _rows(2, 300, torch.float32, seed=17)
    labels = _labels(z, 3)
    ids, logp, rest = _targets(z, 20, tau, 4)
    grad = sw.slimwise_distill_loss(z, labels, ids, logp, rest, alpha=0.3, temperature=tau)[2]
    h = 1e-4
    at = torch.cat([ids[0, :8].long(), labels[:1].long(), torch.arange(0, 300, 23, device=DEV)])
    for i in at.tolist():
        up, down = z.double().clone(), z.double().clone()
        up[:, i] += h
        down[:, i] -= h
        d = (_loss64(up, labels, ids, logp, rest, 0.3, tau)[0] -
             _loss64(down, labels, ids, logp, rest, 0.3, tau)[0]) / (2 * h)
        # the difference's own error: h^2 times the third derivative, 1e-8 times a few
        assert bool(((grad[:, i].double() - d).abs() <= 2 * MASS * (1 + tau) + 1e-7).all()), i
        assert bool(((grad[:, i].double() - d).abs() <= 1e-5 * (1 + tau)).all()), i


def test_distill_gradient_sums_to_the_missing_mass():
    # sum_i dL/dz_i = a (1 - 1) + (1 - a) tau (M - M) = 0 for every row
    z = _rows(8, 50001, torch.float32, seed=18)
    grad = sw.slimwise_distill_loss(z, _labels(z, 3), *_targets(z, 64, 1.0, 4), alpha=0.1)[2]
    assert bool((grad.double().sum(1).abs() <= 8 * MASS).all())


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
GAP = 2e-5   # shares of the mass nearer than this to a cut are not compared


def _sample64(z, u, t, k, p, m):
    """(token, log-probability, whether every decision is at least GAP from its
    cut) of one row, in 64 bits."""
    z = z.double().cpu().numpy() + 0.0
    V = len(z)
    order = np.argsort(-z, kind="stable")
    if t == 0.0:
        return int(order[0]), 0.0, True
    zs = z[order]
    e = np.exp((zs - zs[0]) / t)
    n = k if 0 < k < V else V
    e[n:] = 0.0
    before = np.cumsum(e) - e
    keep = e > 0
    sure = True
    if p < 1.0:
        keep &= (before < p * e.sum())
        keep[0] = True
        sure &= bool(np.abs(before[1:n] / e.sum() - p).min(initial=1.0) > GAP)
    if m > 0.0:
        keep &= e >= m
        sure &= bool(np.abs(e[:n] - m).min() > 1e-6)
    w = np.zeros(V)
    w[order] = np.where(keep, e, 0.0)
    cdf = np.cumsum(w) / w.sum()
    token = int(np.searchsorted(cdf, u, side="right"))
    sure &= bool(np.abs(cdf - u).min() > GAP)
    token = min(token, V - 1)
    return token, float(np.log(w[token] / w.sum())) if w[token] > 0 else -INF, sure


def _check_sample(z, u, t, k, p, m, at_least=0.8):
    dev = dict(device=DEV)
    rows = z.shape[0]
    tokens, lp = sw.slimwise_sample(
        z, torch.tensor(u, dtype=torch.float32, **dev), temperature=torch.tensor(t, dtype=torch.float32, **dev),
        top_k=torch.tensor(k, dtype=torch.int32, **dev), top_p=torch.tensor(p, dtype=torch.float32, **dev),
        min_p=torch.tensor(m, dtype=torch.float32, **dev))
    f = lambda x: float(np.float32(x))
    compared = 0
    for i in range(rows):
        token, logprob, sure = _sample64(z[i], f(u[i]), f(t[i]), k[i], f(p[i]), f(m[i]))
        if sure:
            compared += 1
            assert int(tokens[i]) == token, (i, t[i], k[i], p[i], m[i])
            assert abs(float(lp[i]) - logprob) <= 4 * MASS, i
    assert compared >= at_least * rows, (compared, rows)
    return tokens, lp


REQUESTS = [(0.0, 0, 1.0, 0.0), (1.0, 1, 1.0, 0.0), (0.7, 20, 0.8, 0.0), (1.0, 0, 0.9, 0.0),
            (0.6, 0, 0.95, 0.0), (1.0, 0, 1.0, 0.1), (1.5, 50, 0.9, 0.02), (1.0, 256, 1.0, 0.0),
            (1.0, 0, 0.0, 0.0), (2.0, 0, 1.0, 1.0), (0.01, 0, 0.5, 0.0), (1.0, 100000000, 0.3, 0.001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 100, 300, 5001, 40000, 131072])
def test_sample(vocab, dtype):
    z = _rows(48, vocab, dtype, seed=20 + vocab)
    z[:, :min(vocab, 30)] += 8.0
    u = np.random.default_rng(vocab).random(48).astype(np.float32)
    r = [REQUESTS[i % len(REQUESTS)] for i in range(48)]
    _check_sample(z, u, *[list(c) for c in zip(*r)])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [300, 5001, 60001])
def test_sample_wide_sets(vocab, dtype):
    # more elements kept than the scan lists: nucleus, large top-k, min-p, both, none
    z = _rows(20, vocab, dtype, seed=31)
    wide = [(1.0, 0, 0.9, 0.0), (1.0, 1000, 1.0, 0.0), (3.0, 0, 1.0, 0.05), (3.0, 2000, 0.8, 0.01)]
    r = [wide[i % 4] for i in range(20)]
    u = np.random.default_rng(5).random(20).astype(np.float32)
    # 1e5 cuts over the unit interval: fewer rows are clear of all of them
    _check_sample(z, u, *[list(c) for c in zip(*r)], at_least=0.2 if vocab > 10000 else 0.6)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [700, 40001])
def test_sample_ties_go_to_the_lower_id(vocab, dtype):
    # all equal: the nucleus of p keeps the first ceil(p V) ids, top-k the first k
    z = torch.zeros((6, vocab), dtype=dtype, device=DEV)
    dev = dict(device=DEV)
    u = torch.tensor([0.0, 0.999999, 0.5, 0.999999, 0.999999, 0.25], **dev)
    k = torch.tensor([0, 0, 0, 7, 500, 0], dtype=torch.int32, **dev)
    p = torch.tensor([0.25, 0.25, 1.0, 1.0, 1.0, 0.5], **dev)
    tokens, lp = sw.slimwise_sample(z, u, top_k=k, top_p=p)
    n = math.ceil(0.25 * vocab)
    half = math.ceil(0.5 * vocab)
    assert tokens.tolist() == [0, int(0.999999 * n), int(0.5 * vocab), 6, 499, int(0.25 * half)]
    want = [-math.log(c) for c in (n, n, vocab, 7, 500, half)]
    assert np.allclose(lp.cpu().numpy(), want, rtol=0, atol=1e-5)


def test_sample_is_the_same_in_any_batch_and_type():
    z = _rows(40, 30011, torch.bfloat16, seed=33)
    z[:, 5:25] += 9.0
    g = _gen(34)
    rows = 3000
    pick = torch.randint(0, 40, (rows,), generator=g, device=DEV)
    r = torch.tensor([REQUESTS[i % len(REQUESTS)] for i in range(rows)], device=DEV)
    args = dict(temperature=r[:, 0].contiguous(), top_k=r[:, 1].to(torch.int32).contiguous(),
                top_p=r[:, 2].contiguous(), min_p=r[:, 3].contiguous())
    u = torch.rand(rows, generator=g, device=DEV)
    many = sw.slimwise_sample(z[pick].contiguous(), u, **args)
    wide = sw.slimwise_sample(z[pick].float(), u, **args)
    assert torch.equal(many[0], wide[0]) and torch.equal(many[1], wide[1])
    for i in range(0, rows, 97):
        one = sw.slimwise_sample(z[pick[i:i + 1]], u[i:i + 1], **{n: a[i:i + 1] for n, a in args.items()})
        assert torch.equal(one[0], many[0][i:i + 1]) and torch.equal(one[1], many[1][i:i + 1]), i


def test_sample_frequencies():
    # 40000 draws of one row by evenly spaced numbers: counts are the shares to one draw per cut
    vocab, n = 50, 40000
    z = _rows(1, vocab, torch.float32, seed=35, scale=1.0)
    u = (torch.arange(n, device=DEV, dtype=torch.float64) + 0.5) / n
    tokens, lp = sw.slimwise_sample(z.expand(n, vocab).contiguous(), u.float())
    p = torch.softmax(z[0].double(), 0)
    count = torch.bincount(tokens.long(), minlength=vocab)
    assert bool(((count - p * n).abs() <= 2.0).all())
    assert bool(((lp.double() - p.log()[tokens.long()]).abs() <= 2 * MASS).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_sample_masked_rows(dtype):
    low = torch.finfo(dtype).min
    z = _rows(6, 20000, dtype, seed=36)
    z[0, 1:] = -INF
    z[1, :19999] = -INF
    z[2, 5:] = low
    z[3] = -INF
    z[4, 7] = math.nan
    z[5, 9] = INF
    u = torch.full((6,), 0.7, device=DEV)
    for kw in ({}, {"top_p": torch.full((6,), 0.9, device=DEV)},
               {"temperature": torch.zeros(6, device=DEV)},
               {"top_k": torch.full((6,), 20, dtype=torch.int32, device=DEV)}):
        tokens, lp = sw.slimwise_sample(z, u, **kw)
        assert tokens[:2].tolist() == [0, 19999] and lp[:2].tolist() == [0.0, 0.0]
        assert 0 <= int(tokens[2]) < 5
        assert tokens[3:].tolist() == [-1, -1, -1] and bool(torch.isnan(lp[3:]).all())


def test_sample_refuses_requests_row_by_row():
    z = _rows(10, 1000, torch.float32, seed=37)
    nan = math.nan
    t = torch.tensor([1, -1, nan, INF, 1, 1, 1, 1, 1, 1], device=DEV)
    p = torch.tensor([1, 1, 1, 1, -0.1, nan, 1, 1, 1, 1.0], device=DEV)
    m = torch.tensor([0, 0, 0, 0, 0, 0, 1.5, nan, 0, 0], device=DEV)
    u = torch.tensor([0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 1.0, -0.1], device=DEV)
    tokens, lp = sw.slimwise_sample(z, u, temperature=t, top_p=p, min_p=m)
    assert int(tokens[0]) >= 0 and math.isfinite(float(lp[0]))
    assert tokens[1:].tolist() == [-1] * 9 and bool(torch.isnan(lp[1:]).all())


# ---------------------------------------------------------------------------
# all three
# ---------------------------------------------------------------------------
def test_binding_refuses_shapes_types_and_devices():
    z = _rows(4, 100, torch.float32, seed=40)
    i32 = dict(dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        sw.slimwise_top_logits(z.t(), 2)                       # rows not contiguous
    with pytest.raises(ValueError):
        sw.slimwise_top_logits(z[0], 2)
    with pytest.raises(TypeError):
        sw.slimwise_top_logits(z.half(), 2)
    with pytest.raises(sw.SlimwiseError):
        sw.slimwise_top_logits(z, 101)
    with pytest.raises(sw.SlimwiseError):
        sw.slimwise_top_logits(z, 0)
    with pytest.raises(ValueError):
        sw.slimwise_top_logits(z, 8, ids=torch.empty((4, 7), **i32))
    with pytest.raises(TypeError):
        sw.slimwise_top_logits(z, 8, ids=torch.empty((4, 8), device=DEV))
    u = torch.rand(4, device=DEV)
    with pytest.raises(ValueError):
        sw.slimwise_sample(z, u[:3])
    with pytest.raises(TypeError):
        sw.slimwise_sample(z, None)
    with pytest.raises(TypeError):
        sw.slimwise_sample(z, u, top_k=torch.zeros(4, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        sw.slimwise_sample(z, u, top_p=torch.ones(8, device=DEV)[::2])
    a = (_labels(z, 1),) + _targets(z, 8, 1.0, 2)
    with pytest.raises(ValueError):
        sw.slimwise_distill_loss(z, a[0][:3], *a[1:])
    with pytest.raises(ValueError):
        sw.slimwise_distill_loss(z, *a, grad=torch.empty((4, 99), device=DEV))
    with pytest.raises(ValueError):
        sw.slimwise_distill_loss(z, *a, grad=torch.empty((4, 100), device=DEV, dtype=torch.bfloat16))
    with pytest.raises(sw.SlimwiseError):
        sw.slimwise_distill_loss(z, *a, alpha=2.0)
    with pytest.raises(TypeError):
        sw.slimwise_distill_loss(z, None, *a[1:])


def test_no_rows():
    z = torch.empty((0, 100), device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    ids, logp, rest = sw.slimwise_top_logits(z, 8)
    assert ids.shape == (0, 8) and rest.shape == (0,)
    loss, row, grad = sw.slimwise_distill_loss(z, torch.empty(0, **i32), ids, logp, rest)
    assert float(loss) == 0.0 and grad.shape == (0, 100)
    assert sw.slimwise_sample(z, torch.empty(0, device=DEV))[0].shape == (0,)


def test_on_a_side_stream_and_in_a_graph():
    z = _rows(6, 30000, torch.bfloat16, seed=41)
    labels, u = _labels(z, 1), torch.rand(6, generator=_gen(2), device=DEV)
    k = torch.full((6,), 20, dtype=torch.int32, device=DEV)

    def step():
        top = sw.slimwise_top_logits(z, 64)
        return top + sw.slimwise_distill_loss(z, labels, *top) + sw.slimwise_sample(z, u, top_k=k)

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # handed a stream instead of the current one
    ids, logp, rest = sw.slimwise_top_logits(z, 64, stream=side)
    side.synchronize()
    assert torch.equal(ids, want[0]) and torch.equal(logp, want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    z.copy_(_rows(6, 30000, torch.bfloat16, seed=42))
    g.replay()
    torch.cuda.synchronize()
    again = step()
    assert all(torch.equal(a, b) for a, b in zip(out, again))


def test_offsets_past_32_bits():
    # the last row lies 2^32 elements into the allocation
    stride, vocab = (1 << 31) + 8, 1000
    flat = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device=DEV)
    z = flat.as_strided((3, vocab), (stride, 1))
    z.copy_(_rows(3, vocab, torch.bfloat16, seed=43))
    near = z.contiguous()
    labels, u = _labels(near, 1), torch.full((3,), 0.4, device=DEV)
    a, b = sw.slimwise_top_logits(z, 64), sw.slimwise_top_logits(near, 64)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert torch.equal(sw.slimwise_sample(z, u)[0], sw.slimwise_sample(near, u)[0])
    want = sw.slimwise_distill_loss(near, labels, *b)
    got = sw.slimwise_distill_loss(z, labels, *b, grad=z)
    assert torch.equal(got[1], want[1]) and torch.equal(z, want[2])


def test_the_same_bits_on_every_run():
    # rows whose lists overflow among them; many rows and few, so that single CTAs and clusters scan
    for rows in (3, 400):
        z = _rows(rows, 50021, torch.bfloat16, seed=44)
        z[0] = 0.0
        z[1] = torch.linspace(-20.0, 20.0, 50021, device=DEV).to(torch.bfloat16)
        top = sw.slimwise_top_logits(z, 64)
        loss = sw.slimwise_distill_loss(z, _labels(z, 1), *top)
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(top, sw.slimwise_top_logits(z, 64)))
            assert all(torch.equal(a, b) for a, b in
                       zip(loss, sw.slimwise_distill_loss(z, _labels(z, 1), *top)))


@pytest.mark.parametrize("dtype", TYPES)
def test_top_logits_clustered(dtype):
    # the largest elements side by side, in one warp's run or across two, over many more than fit a list
    z = _rows(6, 131072, dtype, seed=45, scale=1.0)
    bump = torch.linspace(20.0, 10.0, 400, device=DEV).to(dtype)
    for t, at in enumerate((0, 131072 - 400, 16384 - 200, 65536 - 3, 4096, 77777)):
        z[t, at:at + 400] = bump
    for k in (8, 64, 256):
        _check_top(z, k, 1.0)
    _check_top(z.repeat(60, 1), 64, 1.0)


def test_outputs_keep_their_bounds():
    # guards around every output, at a row count that fills no block
    rows, vocab, k = 5, 20011, 33
    z = _rows(rows, vocab, torch.bfloat16, seed=46)

    def guarded(n, dtype):
        flat = torch.full((n + 64,), 77, dtype=dtype, device=DEV)
        return flat, flat[32:32 + n]

    made = [guarded(rows * k, torch.int32), guarded(rows * k, torch.float32), guarded(rows, torch.float32),
            guarded(rows, torch.int32), guarded(rows, torch.float32), guarded(rows, torch.float32),
            guarded(1, torch.float32)]
    ids, logp, rest, tokens, lp, row, loss = [m[1] for m in made]
    sw.slimwise_top_logits(z, k, ids=ids.view(rows, k), logp=logp.view(rows, k), log_rest=rest)
    sw.slimwise_sample(z, torch.rand(rows, device=DEV), tokens=tokens, logprob=lp)
    sw.slimwise_sample(z, torch.rand(rows, device=DEV), top_p=torch.full((rows,), 0.9, device=DEV),
                       tokens=tokens, logprob=lp)
    sw.slimwise_distill_loss(z, _labels(z, 1), ids.view(rows, k), logp.view(rows, k), rest, row_loss=row,
                             loss=loss)
    for flat, view in made:
        n = view.numel()
        assert bool((flat[:32] == 77).all()) and bool((flat[32 + n:] == 77).all())


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_sample_wide_sets_in_any_batch(rows):
    # left-over rows are searched by clusters of another size where other numbers of rows are scanned
    z = _rows(8, 30011, torch.bfloat16, seed=47)
    u = torch.rand(8, generator=_gen(48), device=DEV)
    p = torch.tensor([1.0, 0.9, 0.99, 0.5, 1.0, 0.9, 0.3, 0.95], device=DEV)
    k = torch.tensor([0, 0, 5000, 700, 20, 0, 0, 97], dtype=torch.int32, device=DEV)
    one = [sw.slimwise_sample(z[i:i + 1], u[i:i + 1], top_p=p[i:i + 1], top_k=k[i:i + 1]) for i in range(8)]
    pick = torch.arange(rows, device=DEV) % 8
    tokens, lp = sw.slimwise_sample(z[pick], u[pick], top_p=p[pick], top_k=k[pick])
    for i in range(rows):
        assert torch.equal(tokens[i:i + 1], one[i % 8][0]) and torch.equal(lp[i:i + 1], one[i % 8][1]), i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [3001, 30011])
def test_sample_many_rows_that_are_left_over(vocab, dtype):
    # many of them are searched by a CTA each, a few by a cluster, and none of it shows
    z = _rows(8, vocab, dtype, seed=49)
    u = torch.rand(8, generator=_gen(50), device=DEV)
    p = torch.tensor([1.0, 0.9, 0.99, 0.5, 1.0, 0.9, 0.3, 0.95], device=DEV)
    k = torch.tensor([0, 0, 1500, 700, 0, 1000, 0, 97], dtype=torch.int32, device=DEV)
    one = [sw.slimwise_sample(z[i:i + 1], u[i:i + 1], top_p=p[i:i + 1], top_k=k[i:i + 1]) for i in range(8)]
    want = [torch.cat([o[j] for o in one]) for j in range(2)]
    for rows in (500, 1300):
        pick = torch.arange(rows, device=DEV) * 5 % 8
        for _ in range(3):
            tokens, lp = sw.slimwise_sample(z[pick], u[pick], top_p=p[pick], top_k=k[pick])
            assert torch.equal(tokens, want[0][pick]) and torch.equal(lp, want[1][pick])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,rows", [(393216, 1), (393216, 500), (1025, 700)])
def test_sample_equal_logits(vocab, rows, dtype):
    # every weight is 2^40: the first ids up to the share p, each as likely
    z = torch.full((rows, vocab), 2.5, dtype=dtype, device=DEV)
    u = torch.rand(rows, generator=_gen(51), device=DEV)
    p = torch.rand(rows, generator=_gen(52), device=DEV)
    tokens, lp = sw.slimwise_sample(z, u, top_p=p)
    part = lambda mass, f: mass * int(float(f) * 2 ** 24) >> 24
    for i, (got, a, b, l) in enumerate(zip(tokens.tolist(), u.tolist(), p.tolist(), lp.tolist())):
        kept = max(-(-part(vocab << 40, b) // (1 << 40)), 1)
        assert got == part(kept << 40, a) >> 40, i
        assert abs(l + math.log(kept)) <= 2.0 ** -20 * (1 + math.log(kept)), i
