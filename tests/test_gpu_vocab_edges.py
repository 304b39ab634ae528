"""The operators over vocabulary logits at the ends of their ranges: more rows
than one pass of the search takes, masses far below the largest logit, targets
and weights without a value.  Tokens are exact; the other tolerances are those of
test_gpu_vocab.py, or derived at the test."""
import math

import pytest
import torch

import paper_2609_34117_gb300 as sw

from tests.test_gpu_vocab import DEV, INF, MASS, TYPES, _check_loss, _gen, _loss64, _rows, _targets

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sw.build.build()


# ---------------------------------------------------------------------------
# sampling: more rows than the search takes in one pass
# ---------------------------------------------------------------------------
# (76 clusters take every 76th row, 256 of theirs in a pass)
CLUSTERS = 76
PASS = 256 * CLUSTERS
# requests that the listed elements of a nearly flat row do not decide, and that they do
WIDE = [(1.0, 0, 1.0), (1.0, 300, 1.0), (1.0, 0, 0.9), (1.0, 300, 0.8)]
LISTED = [(0.0, 0, 1.0), (0.7, 20, 0.8)]


def _check_batch(z, u, kinds, step=1000):
    """The tokens of all rows in one call are those of `step` rows at a time;
    kinds: index of each row's request in WIDE + LISTED."""
    t, k, p = torch.tensor(WIDE + LISTED, device=DEV)[kinds].unbind(1)
    t, k, p = t.contiguous(), k.to(torch.int32).contiguous(), p.contiguous()
    tokens, logprob = sw.slimwise_sample(z, u, temperature=t, top_k=k, top_p=p)
    for a in range(0, z.shape[0], step):
        b = slice(a, a + step)
        want = sw.slimwise_sample(z[b], u[b], temperature=t[b], top_k=k[b], top_p=p[b])
        assert torch.equal(tokens[b], want[0]) and torch.equal(logprob[b], want[1]), a
    assert bool((tokens >= 0).all()) and bool((logprob <= 0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_sample_passes_with_few_rows_left_over(dtype):
    # four rows of each cluster are left over in every pass: the cluster's CTAs search them together
    rows = 2 * PASS + 6000
    z = _rows(rows, 301, dtype, seed=61, scale=1.0)
    at = torch.arange(rows, device=DEV) // CLUSTERS
    kinds = torch.where(at % 64 == 5, 0, len(WIDE))
    _check_batch(z, torch.rand(rows, generator=_gen(62), device=DEV), kinds)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [PASS + 44, 20000, 22000, 2 * PASS + 1500])
def test_sample_passes_searched_in_either_way(rows, dtype):
    # a tenth of the rows are left over, under requests that take unlike numbers of sums: in a full
    # pass a CTA each searches them, in the last all of a cluster
    z = _rows(rows, 1000, dtype, seed=63, scale=1.0)
    g = _gen(64)
    wide = torch.rand(rows, generator=g, device=DEV) < 0.1
    kinds = torch.where(wide, torch.randint(0, len(WIDE), (rows,), generator=g, device=DEV),
                        torch.randint(len(WIDE), len(WIDE + LISTED), (rows,), generator=g, device=DEV))
    _check_batch(z, torch.rand(rows, generator=g, device=DEV), kinds)


# ---------------------------------------------------------------------------
# top logits
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,k", [(9, 20011, 64), (3, 131072, 256), (700, 4097, 20)])
@pytest.mark.parametrize("tau", [1.0, 4.0, 30.0])
def test_top_logits_rest_near_the_whole_mass(tau, rows, vocab, k, dtype):
    # log_rest = -log(1 + list / rest): what the ratio of the two sums is off by, times the list's
    # share, and two roundings.  A sum is off by at most 2^-16 (exponents of at most 40 bits of three
    # roundings each, 83 parts in 2^24; exp2's 4; 40 additions; 5 changes of reference of 5)
    z = _rows(rows, vocab, dtype, seed=73)
    ids, logp, rest = sw.slimwise_top_logits(z, k, temperature=tau)
    lp = torch.log_softmax(z.double() / tau, 1)
    want = torch.logsumexp(lp.scatter(1, ids.long(), -INF), 1)
    share = -torch.expm1(want)
    assert bool(((rest.double() - want).abs() <= 2.0 ** -15 * share + 2.0 ** -22 * want.abs()).all())
    want = lp.gather(1, ids.long())
    assert bool(((logp.double() - want).abs() <= 2.0 ** -16 + 2.0 ** -22 * want.abs()).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_top_logits_of_lowest_values(dtype):
    # a listed element at the type's lowest value has a finite log-probability, as its quotient has
    z = torch.full((2, 5003), -INF, dtype=dtype, device=DEV)
    z[:, 100:140] = torch.finfo(dtype).min
    z[:, 7] = 1.5
    for tau in (1.0, 2.0):
        ids, logp, rest = sw.slimwise_top_logits(z, 20, temperature=tau)
        want = torch.log_softmax(z.double() / tau, 1).gather(1, ids.long())
        assert bool(((logp.double() - want).abs() <= 2.0 ** -22 * want.abs() + 2.0 ** -16).all())


# ---------------------------------------------------------------------------
# distillation loss
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,tau", [(60, 1.0), (87, 1.0), (90, 1.0), (104, 1.0), (150, 1.0), (200, 1.0),
                                     (200, 2.0), (9, 0.1), (14, 0.15), (16, 0.2), (30, 0.05)])
def test_distill_loss_mass_outside_the_list_far_below_it(gap, tau, dtype):
    # the student's mass outside the list is e^(-gap / tau), and the teacher's any
    z = _rows(6, 20000, dtype, seed=65, scale=0.5)
    ids = torch.arange(5, 20000, 1000, device=DEV)
    z[:, ids] += gap
    rest = torch.tensor([-0.7, -10.0, -40.0, -90.0, -100.0, -0.01], device=DEV)
    logp = torch.log(-torch.expm1(rest) / 20)[:, None].expand(6, 20).contiguous()
    labels = torch.tensor([5, 6, 1005, 2005, 5, 19999], dtype=torch.int32, device=DEV)
    top = ids.to(torch.int32).expand(6, 20).contiguous()
    weight = torch.tensor([1.0, 8.0, 0.5, 1.0, 8.0, 8.0], device=DEV)
    _check_loss(z, labels, top, logp, rest, alpha=0.1, tau=tau, weight=weight)
    row = sw.slimwise_distill_loss(z, labels, top, logp, rest, temperature=tau, grad=False)[1]
    want = _loss64(z.double(), labels, top, logp, rest, 0.1, tau)[0]
    assert bool(((row.double() - want).abs() <= 4 * MASS * (1 + tau * tau) + 2.0 ** -20 * want.abs()).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
def test_distill_loss_of_lowest_values(tau, dtype):
    # the label, a listed token, all that is not listed at the type's lowest value: losses of 1e34
    # to 1e37, not infinite
    low = torch.finfo(dtype).min
    z = _rows(3, 9001, dtype, seed=66)
    ids, logp, rest = _targets(z, 20, tau, 4)
    labels = torch.tensor([4000, int(ids[1, 0]), int(ids[2, 1])], dtype=torch.int32, device=DEV)
    z[0, 4000] = low
    z[1, int(ids[1, 5])] = low
    keep = torch.zeros(9001, dtype=torch.bool, device=DEV)
    keep[ids[2].long()] = True
    z[2] = torch.where(keep, z[2], low)
    loss, row, grad = sw.slimwise_distill_loss(z, labels, ids, logp, rest, alpha=0.1, temperature=tau)
    z64 = z.double()
    want, mark, P, r, _ = _loss64(z64, labels, ids, logp, rest, 0.1, tau)
    # (in the loss's type: 0.9 tau r 3.4e38 of the last row passes its range at tau 2)
    assert torch.equal(torch.isfinite(row), torch.isfinite(want.float()))
    fin = torch.isfinite(row)
    assert bool(((row.double() - want).abs() <= 2.0 ** -20 * want.abs())[fin].all()) and bool((want > 1e30).all())
    # the gradient by its formula, the shares of the rest among themselves: logsumexp's own gradient
    # does not hold at -3e38, where 64 bits do not tell the log of a sum of 8981 from that of one
    p, q = torch.softmax(z64, 1), torch.softmax(z64 / tau, 1)
    onehot = torch.zeros_like(p).scatter_(1, labels.long()[:, None], 1.0)
    listed = torch.zeros_like(p).scatter_(1, ids.long(), P)
    share = torch.softmax((z64 / tau).masked_fill(mark, -INF), 1) * r[:, None] + listed
    M, beta = (P.sum(1) + r)[:, None], 0.9 * tau
    g = 0.1 * (p - onehot) + beta * (M * q - share)
    tol = 2 * MASS * (0.1 * (p + onehot) + beta * (M * q + share)) + 1e-38
    tol = tol + (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22) * g.abs()
    assert bool(((grad.double() - g).abs() <= tol).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("alpha", [0.0, 0.1, 1.0])
def test_distill_loss_of_targets_without_a_distribution(alpha, dtype):
    teacher = _rows(6, 9001, dtype, seed=68)
    z = _rows(6, 9001, dtype, seed=69)
    labels = torch.tensor([3, 4, 5, 6, 7, 8], dtype=torch.int32, device=DEV)
    clean = sw.slimwise_top_logits(teacher, 64)
    want = sw.slimwise_distill_loss(z, labels, *clean, alpha=alpha)
    teacher[1, 7] = math.nan
    teacher[2, 9] = INF
    ids, logp, rest = sw.slimwise_top_logits(teacher, 64)
    logp[3, 5] = math.nan
    rest[4] = math.nan
    loss, row, grad = sw.slimwise_distill_loss(z, labels, ids, logp, rest, alpha=alpha)
    assert math.isnan(float(loss)) and bool(torch.isnan(row[1:5]).all()) and bool(torch.isnan(grad[1:5]).all())
    for t in (0, 5):
        assert torch.equal(row[t], want[1][t]) and torch.equal(grad[t], want[2][t])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_distill_loss_terms_without_weight(tau, dtype):
    z = _rows(2, 9001, dtype, seed=67)
    ids, logp, rest = _targets(z, 20, tau, 4)
    labels = torch.tensor([40, 41], dtype=torch.int32, device=DEV)
    z[0, 40] = -INF
    # alpha 0: the label's infinite cross entropy does not count
    row, grad = sw.slimwise_distill_loss(z, labels, ids, logp, rest, alpha=0.0, temperature=tau)[1:]
    want = sw.slimwise_distill_loss(z, labels + 3, ids, logp, rest, alpha=0.0, temperature=tau)[1:]
    assert bool(torch.isfinite(row).all()) and torch.equal(row, want[0]) and torch.equal(grad, want[1])
    # alpha 1: nor does an infinite divergence
    z[1, int(ids[1, 3])] = -INF
    labels = torch.tensor([42, 43], dtype=torch.int32, device=DEV)
    row, grad = sw.slimwise_distill_loss(z, labels, ids, logp, rest, alpha=1.0, temperature=tau)[1:]
    ce = -torch.log_softmax(z.double(), 1).gather(1, labels.long()[:, None])[:, 0]
    assert bool(((row.double() - ce).abs() <= 2 * MASS + 2.0 ** -20 * ce.abs()).all())
    assert bool(torch.isfinite(grad).all())
    # what is not a number still shows
    z[0, 7] = math.nan
    for alpha in (0.0, 1.0):
        row = sw.slimwise_distill_loss(z, labels, ids, logp, rest, alpha=alpha, temperature=tau)[1]
        assert bool(torch.isnan(row[0])) and bool(torch.isfinite(row[1])) == (alpha == 1.0)


def test_distill_loss_rows_left_out_whatever_their_weight():
    # 1 / the number of labelled rows, where there are none, is no number
    z = _rows(5, 2001, torch.float32, seed=70)
    args = _targets(z, 20, 1.0, 4)
    labels = torch.tensor([3, -100, 5, -1, -100], dtype=torch.int32, device=DEV)
    w = torch.tensor([0.25, math.nan, 0.75, INF, -INF], device=DEV)
    want = sw.slimwise_distill_loss(z, labels, *args, row_weight=torch.nan_to_num(w, 0.0, 0.0, 0.0))
    loss, row, grad = sw.slimwise_distill_loss(z, labels, *args, row_weight=w)
    assert all(torch.equal(a, b) for a, b in zip((loss, row, grad), want))
    none = torch.full_like(labels, -100)
    loss, row, grad = sw.slimwise_distill_loss(z, none, *args, row_weight=(none >= 0).float() / (none >= 0).sum())
    assert float(loss) == 0.0 and not bool(row.any()) and not bool(grad.any())
    # a row that is trained on shows such a weight
    w[0] = math.nan
    assert math.isnan(float(sw.slimwise_distill_loss(z, labels, *args, row_weight=w)[0]))


def test_distill_loss_of_no_rows_writes_the_loss_it_was_given():
    loss = torch.full((1,), 7.0, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    for stream in (None, side):
        loss.fill_(7.0)
        torch.cuda.synchronize()
        out = sw.slimwise_distill_loss(torch.empty((0, 100), device=DEV), torch.empty(0, **i32),
                                       torch.empty((0, 8), **i32), torch.empty((0, 8), device=DEV),
                                       torch.empty(0, device=DEV), loss=loss, stream=stream)[0]
        torch.cuda.synchronize()
        assert out is loss and float(loss) == 0.0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("between", [1, 8, 63, 4001])
def test_distill_gradient_of_rows_far_apart_takes_rows_of_its_own(between, dtype):
    # the last of 16 positions: 15 rows and more lie between two of the logits'
    rows, vocab = 6, 4001
    every = _rows(rows, 16 * vocab + between, dtype, seed=74)
    z = every[:, 15 * vocab:16 * vocab]
    args = (torch.arange(rows, dtype=torch.int32, device=DEV),) + _targets(z, 20, 1.0, 4)
    loss, row, grad = sw.slimwise_distill_loss(z, *args)
    want = sw.slimwise_distill_loss(z, *args, grad=torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV))
    assert torch.equal(row, want[1]) and torch.equal(grad, want[2])
    assert grad.untyped_storage().nbytes() <= rows * (vocab + 8) * grad.element_size()
    # rows that are nearly next to each other keep their stride
    z = _rows(rows, vocab, dtype, seed=75, pad=between % 64)
    assert sw.slimwise_distill_loss(z, *args)[2].stride() == z.stride()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first,then", [(0, 2001), (0, 2008), (2016, 0), (2003, 1)])
def test_distill_gradient_beside_the_logits_in_one_buffer(first, then, dtype):
    rows, vocab = 5, 2001
    z = _rows(rows, vocab, dtype, seed=76)
    args = (torch.arange(rows, dtype=torch.int32, device=DEV),) + _targets(z, 20, 1.0, 4)
    both = torch.full((rows, 4020), 7.0, dtype=dtype, device=DEV)
    own, grad = both[:, first:first + vocab], both[:, then:then + vocab]
    own.copy_(z)
    # the same gradient apart, whose rows start where these do
    want = sw.slimwise_distill_loss(own, *args, grad=torch.zeros_like(both)[:, then:then + vocab])
    got = sw.slimwise_distill_loss(own, *args, grad=grad)
    assert torch.equal(own, z) and all(torch.equal(a, b) for a, b in zip(got, want))
    keep = torch.ones(4020, dtype=torch.bool, device=DEV)
    keep[first:first + vocab] = keep[then:then + vocab] = False
    assert bool((both[:, keep] == 7.0).all())
    # a column that both have is refused
    for at in (first + vocab - 1, first + 1, first - 1):
        if 0 <= at <= 4020 - vocab:
            with pytest.raises(sw.SlimwiseError):
                sw.slimwise_distill_loss(own, *args, grad=both[:, at:at + vocab])


# ---------------------------------------------------------------------------
# all three
# ---------------------------------------------------------------------------
def test_outputs_are_memory_of_the_stream_that_writes_them():
    # a block that the current stream has just given back may still be in use there
    rows, vocab, k = 256, 4001, 64
    z = _rows(rows, vocab, torch.float32, seed=71)
    top = sw.slimwise_top_logits(z, k)
    labels, u = top[0][:, 0].contiguous(), torch.rand(rows, generator=_gen(72), device=DEV)
    side = torch.cuda.Stream()
    calls = [lambda: sw.slimwise_top_logits(z, k, stream=side),
             lambda: sw.slimwise_distill_loss(z, labels, *top, stream=side),
             lambda: sw.slimwise_sample(z, u, stream=side)]
    for call in calls:
        torch.cuda.synchronize()
        shapes = [(t.shape, t.dtype) for t in call()]
        side.synchronize()
        given_back = [torch.empty(s, dtype=d, device=DEV) for s, d in shapes * 4]
        at = {t.data_ptr() for t in given_back}
        del given_back
        out = call()
        side.synchronize()
        assert not at & {t.data_ptr() for t in out}
