"""Performance cases of the vocabulary operators: a teacher's top logits, the
distillation loss with its gradient, and sampling.

All three work on rows of vocabulary logits next to the pruned-pool layer:

  top      the K largest logits of each row as log-probabilities, with the
           log of the mass that the others hold: the targets that a full-pool
           teacher leaves for the distillation of its pruned decoder
  distill  alpha * cross entropy + (1 - alpha) * KL against those targets with
           a bucket for the residual mass, per row and summed under row
           weights, with the gradient of the logits (a training step) or
           without (evaluation)
  sample   temperature, top-k, top-p and min-p sampling of a decode step's
           batch, from one given random number per row

Logits are bf16 or fp32: a background of N(0, 1.5) with 64 raised tokens a row,
the first by 14 to 22 and each next by 0.25 less, so that some rows are nearly
decided and some spread over thousands of tokens.  A student's logits are its
teacher's with N(0, 0.7) added.  A tenth of the training rows carry no label
(prompt tokens).
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
IGNORE = -100     # label of a row that is not trained on
SCALE = 2.0 ** 40  # sampling weights are whole multiples of 1 / SCALE of the largest
MODES = ("mixed", "topk", "topp", "minp", "greedy")


def _case(kind, rows, vocab, dtype, k=0, tau=1.0, alpha=0.0, grad=False, mode="", pad=0, name=None):
    """k: length of the teacher's list; pad: elements between the end of a row
    and the start of the next; mode: the requests of a sampled batch."""
    c = {"kind": kind, "rows": rows, "vocab": vocab, "dtype": dtype, "k": k, "tau": tau,
         "alpha": alpha, "grad": grad, "mode": mode, "pad": pad}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # one token's targets while a teacher generates
        _case("top", 1, 131072, "bf16", 64, name="top_1x131072_bf16"),
        # a rollout's targets from an odd vocabulary: rows start at odd addresses
        _case("top", 511, 150001, "fp32", 64, tau=2.0, name="top_511x150001_fp32"),
        # targets of a teacher's training batch
        _case("top", 4096, 131072, "bf16", 64, name="top_4096x131072_bf16"),
        # a small model's step on a few rows
        _case("distill", 8, 32000, "bf16", 20, alpha=0.1, grad=True, name="distill_8x32000_bf16"),
        # softened targets in fp32, an odd vocabulary
        _case("distill", 1021, 65537, "fp32", 64, tau=2.0, alpha=0.1, grad=True,
              name="distill_1021x65537_fp32_t2"),
        # evaluation: the loss alone, logits in rows of a padded vocabulary
        _case("distill", 2048, 150001, "bf16", 64, alpha=0.1, pad=7,
              name="distill_eval_2048x150001_bf16"),
        # a training batch
        _case("distill", 4096, 131072, "bf16", 64, alpha=0.1, grad=True,
              name="distill_4096x131072_bf16"),
        # one request
        _case("sample", 1, 131072, "bf16", mode="topk", name="sample_1x131072_bf16"),
        # a decode batch whose requests ask for a nucleus
        _case("sample", 64, 131072, "fp32", mode="topp", name="sample_64x131072_fp32_topp"),
        # decode batches of all kinds of requests
        _case("sample", 256, 150001, "fp32", mode="mixed", name="sample_256x150001_fp32"),
        _case("sample", 512, 262144, "bf16", mode="mixed", name="sample_512x262144_bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["top", "distill", "sample"])
    dtype = rng.choice(["bf16", "fp32"])
    vocab = _spread(rng, 1000, 262144)
    size = 2 if dtype == "bf16" else 4
    rows = _spread(rng, 1, 512 if kind == "sample" else 4096)
    rows = max(1, min(rows, 4096 * 131072 * 2 // (vocab * size)))
    pad = rng.choice([0, 0, rng.randrange(1, 64)])
    k = rng.choice([8, 20, 64, 100, 256])
    tau = rng.choice([1.0, 1.0, 2.0])
    if kind == "sample":
        return _case(kind, rows, vocab, dtype, mode=rng.choice(MODES), pad=pad)
    if kind == "top":
        return _case(kind, rows, vocab, dtype, k, tau=tau, pad=pad)
    return _case(kind, rows, vocab, dtype, k, tau=tau, alpha=rng.choice([0.1, 0.5]),
                 grad=rng.random() < 0.7, pad=pad)


def _logits(case, g):
    rows, vocab = case["rows"], case["vocab"]
    z = torch.randn((rows, vocab), generator=g, device="cuda") * 1.5
    # one raised token in each 64th of the ids, in an order that starts anywhere
    part = vocab // 64
    ids = torch.randint(0, part, (rows, 64), generator=g, device="cuda")
    turn = torch.randint(0, 64, (rows, 1), generator=g, device="cuda")
    ids += (torch.arange(64, device="cuda") + turn) % 64 * part
    first = 14.0 + 8.0 * torch.rand((rows, 1), generator=g, device="cuda")
    return z.scatter_add_(1, ids, first - 0.25 * torch.arange(64, device="cuda"))


def _stored(case, z):
    """The logits as the head wrote them: in the case's type and row stride."""
    out = torch.zeros((case["rows"], case["vocab"] + case["pad"]), dtype=DTYPES[case["dtype"]],
                      device="cuda")
    out[:, :case["vocab"]] = z
    return out[:, :case["vocab"]]


def _requests(case, g):
    """Per-row (temperature, top-k, top-p, min-p) of a sampled batch: greedy,
    top-k 20 with a nucleus, a nucleus alone, min-p alone."""
    rows = case["rows"]
    table = torch.tensor([[0.0, 0, 1.0, 0.0], [0.7, 20, 0.8, 0.0], [0.6, 0, 0.95, 0.0],
                          [1.0, 0, 1.0, 0.1]], device="cuda")
    kinds = {"greedy": [0], "topk": [1], "topp": [2], "minp": [3], "mixed": [0, 1, 2, 3]}[case["mode"]]
    pick = torch.randint(0, len(kinds), (rows,), generator=g, device="cuda")
    r = table[torch.tensor(kinds, device="cuda")[pick]]
    return (r[:, 0].contiguous(), r[:, 1].to(torch.int32).contiguous(), r[:, 2].contiguous(),
            r[:, 3].contiguous())


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    rows, k = case["rows"], case["k"]
    z = _logits(case, g)
    s = {"case": case}
    i32 = dict(dtype=torch.int32, device="cuda")
    if case["kind"] == "top":
        s["logits"] = _stored(case, z)
        s["out"] = (torch.empty((rows, k), **i32), torch.empty((rows, k), device="cuda"),
                    torch.empty(rows, device="cuda"))
    elif case["kind"] == "sample":
        s["logits"] = _stored(case, z)
        s["requests"] = _requests(case, g)
        s["uniform"] = torch.rand(rows, generator=g, device="cuda")
        s["out"] = (torch.empty(rows, **i32), torch.empty(rows, device="cuda"))
    else:
        # the teacher's list as it was stored; the label is one of the teacher's
        # top tokens, or in every eighth row any token
        t = z / case["tau"]
        val, ids = torch.topk(t, k, dim=1)
        lse = torch.logsumexp(t, 1, keepdim=True)
        s["ids"] = ids.to(torch.int32)
        s["logp"] = val - lse
        s["log_rest"] = torch.logsumexp(t.scatter_(1, ids, -math.inf), 1) - lse[:, 0]
        at = torch.randint(0, min(8, k), (rows, 1), generator=g, device="cuda")
        labels = ids.gather(1, at)[:, 0].to(torch.int32)
        labels[::8] = torch.randint(0, case["vocab"], labels[::8].shape, generator=g, device="cuda",
                                    dtype=torch.int32)
        labels[torch.randperm(rows, generator=g, device="cuda")[:rows // 10]] = IGNORE
        s["labels"] = labels
        s["weight"] = (labels >= 0).float() / (labels >= 0).sum()
        del t
        z += torch.randn(z.shape, generator=g, device="cuda") * 0.7
        s["logits"] = _stored(case, z)
    return s


def _plain_top(logits, k, tau):
    z = logits.float()
    # one key per element, all different: the value's order above, the lower id above
    bits = (z + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, -2147483648 - bits, bits)
    vocab = z.shape[1]
    ids = torch.topk((order << 32) + (vocab - 1 - torch.arange(vocab, device=z.device)), k, dim=1)[1]
    del bits, order
    x = z * (1.0 / tau)
    top = x.gather(1, ids)
    m = top[:, :1]
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    rest = e.scatter_(1, ids, 0.0).sum(1)
    return ids.to(torch.int32), top - m - torch.log(total), torch.log(rest / total[:, 0])


def _plain_distill(logits, labels, ids, logp, log_rest, alpha, tau, weight, grad):
    z = logits.float()
    live = labels >= 0
    y = labels.clamp(min=0).long()[:, None]
    d = z - z.amax(1, keepdim=True)
    p = torch.exp(d)
    total = p.sum(1, keepdim=True)
    ce = torch.log(total) - d.gather(1, y)
    if tau == 1.0:
        x, q, total_q = d, p, total
    else:
        x = d * (1.0 / tau)
        q = torch.exp(x)
        total_q = q.sum(1, keepdim=True)
    listed_ = ids >= 0
    at = ids.clamp(min=0).long()
    prob = torch.where(listed_, torch.exp(logp), 0.0)
    r = torch.exp(log_rest)[:, None]
    # entries that are absent mark a column of their own, which is cut off again
    at_or_end = torch.where(listed_, at, z.shape[1])
    target = torch.full((z.shape[0], z.shape[1] + 1), -1.0, device=z.device)
    target = target.scatter_(1, at_or_end, prob)[:, :-1]
    rest = torch.where(target < 0, q, 0.0).sum(1, keepdim=True)
    log_q = x.gather(1, at) - torch.log(total_q)
    log_q_rest = torch.log(rest) - torch.log(total_q)
    kl = torch.where(prob > 0, prob * (logp - log_q), 0.0).sum(1, keepdim=True)
    kl = kl + torch.where(r > 0, r * (log_rest[:, None] - log_q_rest), 0.0)
    row = torch.where(live, (alpha * ce + (1.0 - alpha) * tau * tau * kl)[:, 0], 0.0)
    loss = (row * weight).sum()
    if not grad:
        return loss, row, None
    mass = prob.sum(1, keepdim=True) + r
    share = torch.where(rest > 0, r / rest, 0.0)
    dz = torch.where(target < 0, q * (mass / total_q - share), q * (mass / total_q) - target)
    dz = dz * ((1.0 - alpha) * tau)
    dz += p * (alpha / total)
    dz.scatter_add_(1, y, torch.full_like(ce, -alpha))
    dz = torch.where(live[:, None], dz * weight[:, None], 0.0)
    return loss, row, dz.to(logits.dtype)


def _plain_sample(logits, uniform, temperature, top_k, top_p, min_p):
    z = logits.float() + 0.0
    rows, vocab = z.shape
    v, ids = torch.sort(z, dim=1, descending=True, stable=True)
    greedy = temperature == 0
    scale = 1.0 / torch.where(greedy, 1.0, temperature)
    e = torch.exp((v - v[:, :1]) * scale[:, None])
    w = (e * SCALE).long()
    rank = torch.arange(vocab, device=z.device)
    limit = torch.where(greedy, 1, torch.where(top_k > 0, top_k, vocab))
    w = torch.where(rank < limit[:, None], w, 0)
    # floor(sum * p) with p in 24 bits, in two halves that fit 64 bits
    total = w.sum(1)
    p24 = (top_p * 2.0 ** 24).long()
    cut = ((total >> 32) * p24 << 8) + ((total & 0xFFFFFFFF) * p24 >> 24)
    before = torch.cumsum(w, 1) - w
    w = torch.where((before < cut.clamp(min=1)[:, None]) & (e >= min_p[:, None]), w, 0)
    total = w.sum(1)
    u24 = (uniform * 2.0 ** 24).long()
    target = ((total >> 32) * u24 << 8) + ((total & 0xFFFFFFFF) * u24 >> 24)
    by_id = torch.zeros_like(w).scatter_(1, ids, w)
    token = (torch.cumsum(by_id, 1) <= target[:, None]).sum(1, keepdim=True)
    share = by_id.gather(1, token)[:, 0].float() / total.float()
    return token[:, 0].to(torch.int32), torch.log(share)


def run(s):
    c = s["case"]
    if own:
        import paper_2609_34117_gb300 as sw
        if c["kind"] == "top":
            ids, logp, rest = s["out"]
            return sw.slimwise_top_logits(s["logits"], c["k"], temperature=c["tau"], ids=ids,
                                          logp=logp, log_rest=rest)
        if c["kind"] == "sample":
            t, k, p, m = s["requests"]
            tokens, logprob = s["out"]
            return sw.slimwise_sample(s["logits"], s["uniform"], temperature=t, top_k=k, top_p=p,
                                      min_p=m, tokens=tokens, logprob=logprob)
        out = sw.slimwise_distill_loss(s["logits"], s["labels"], s["ids"], s["logp"], s["log_rest"],
                                       alpha=c["alpha"], temperature=c["tau"],
                                       row_weight=s["weight"], grad=c["grad"])
    elif c["kind"] == "top":
        return _plain_top(s["logits"], c["k"], c["tau"])
    elif c["kind"] == "sample":
        return _plain_sample(s["logits"], s["uniform"], *s["requests"])
    else:
        out = _plain_distill(s["logits"], s["labels"], s["ids"], s["logp"], s["log_rest"],
                             c["alpha"], c["tau"], s["weight"], c["grad"])
    loss, row, grad = out
    return (loss.reshape(()), row, grad) if c["grad"] else (loss.reshape(()), row)


def work(case):
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    size = 2 if case["dtype"] == "bf16" else 4
    n = rows * vocab
    if case["kind"] == "top":
        return {"bytes": n * size + rows * (8 * k + 4), "flops": 4 * n}
    if case["kind"] == "sample":
        return {"bytes": n * size + rows * (5 * 4 + 8), "flops": 4 * n}
    live = (rows - rows // 10) * vocab  # the other rows' logits need not be read
    back = case["grad"]
    exps = 1 if case["tau"] == 1.0 else 2
    return {"bytes": live * size + (n * size if back else 0) + rows * (8 * k + 16) + 4,
            "flops": live * (3 * exps + (3 * exps if back else 0))}


def exact(case, seed):
    s = prepare(case, seed)
    rows, kind = case["rows"], case["kind"]
    step = max(1, (1 << 25) // case["vocab"])
    parts = []
    for a in range(0, rows, step):
        z = s["logits"][a:a + step].double()
        if kind == "top":
            # ids from the first of equal values on, as a stable sort leaves them
            ids = torch.sort(-z, dim=1, stable=True)[1][:, :case["k"]]
            lp = torch.log_softmax(z / case["tau"], 1)
            parts.append((ids.to(torch.int32), lp.gather(1, ids),
                          torch.logsumexp(lp.scatter(1, ids, -math.inf), 1)))
        elif kind == "sample":
            parts.append(_exact_sample(z, s["uniform"][a:a + step],
                                       *[r[a:a + step] for r in s["requests"]]))
        else:
            parts.append(_exact_distill(z, s, slice(a, a + step), case))
    joined = [torch.cat(p) for p in zip(*parts)]
    if kind != "distill":
        return tuple(joined)
    loss = (joined[0] * s["weight"].double()).sum()
    return (loss, joined[0], joined[1]) if case["grad"] else (loss, joined[0])


def _exact_distill(z, s, at, case):
    """The loss from its definition and the gradient by differentiating it."""
    labels, ids = s["labels"][at].long(), s["ids"][at].long()
    logp, log_rest = s["logp"][at].double(), s["log_rest"][at].double()
    weight, live = s["weight"][at].double(), s["labels"][at] >= 0
    tau, alpha = case["tau"], case["alpha"]
    with torch.enable_grad():
        z = z.requires_grad_(case["grad"])
        ce = -torch.log_softmax(z, 1).gather(1, labels.clamp(min=0)[:, None])[:, 0]
        lq = torch.log_softmax(z / tau, 1)
        rest = torch.logsumexp(lq.scatter(1, ids, -math.inf), 1)
        kl = (logp.exp() * (logp - lq.gather(1, ids))).sum(1) + log_rest.exp() * (log_rest - rest)
        row = torch.where(live, alpha * ce + (1 - alpha) * tau ** 2 * kl, 0.0)
        if not case["grad"]:
            return (row,)
        dz, = torch.autograd.grad((row * weight).sum(), z)
    return row.detach(), dz


def _exact_sample(z, uniform, temperature, top_k, top_p, min_p):
    t = temperature.double()
    greedy = t == 0
    order = torch.sort(-z, dim=1, stable=True)[1]
    zs = z.gather(1, order)
    p = torch.softmax(zs / torch.where(greedy, 1.0, t)[:, None], 1)
    rank = torch.arange(z.shape[1], device=z.device)[None]
    p = p * (rank < torch.where(greedy, 1, torch.where(top_k > 0, top_k, z.shape[1]))[:, None])
    p = p / p.sum(1, keepdim=True)
    keep = (torch.cumsum(p, 1) - p < top_p.double()[:, None]) & (p >= min_p.double()[:, None] * p[:, :1])
    p = p * keep
    p = (p / p.sum(1, keepdim=True)).gather(1, torch.argsort(order, 1))
    token = (torch.cumsum(p, 1) <= uniform.double()[:, None]).sum(1, keepdim=True)
    token = token.clamp(max=z.shape[1] - 1)
    return token[:, 0].to(torch.int32), torch.log(p.gather(1, token))[:, 0]
