"""Performance cases of the operators around the layer: the embedding, the norm
and the head's cross entropy, each with its gradient.

They are the ends of the model that the pruned-pool layer is the middle of, and
what its training runs beside the layer:

  embed       rows of an embedding table by token id, times a scale
  embed_grad  the table's gradient: each token's rows summed, all others zero
  norm        layer norm or RMS norm of each row, with the statistics that the
              gradient needs
  norm_grad   the gradients of the input, of the weight and, for layer norm, of
              the bias
  loss        cross entropy of the head's logits, from the hidden rows and the
              head's weight: per row and summed under row weights (evaluation)
  loss_grad   the same with the gradients of the hidden rows and of the weight

Token ids are log-uniform over the table (a few make up most of the text), with
a sixteenth of padding.  A tenth of the loss's rows carry no label; a labelled
row's hidden state leans towards its label's weight row, so that some labels are
nearly sure and some are one of many.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
IGNORE = -100   # label of a row that is not trained on
PAD = -1        # id of a padding token


def _case(kind, rows, hidden, dtype, vocab=0, layer=False, grad_dtype="", pad=0, name=None):
    """layer: layer norm with a bias (else RMS norm); grad_dtype: type of the
    gradient of a table or head (a head's: its own); pad: elements between the end of a row of the
    input (the norm's rows, the gradient of the embedded rows) and the next."""
    c = {"kind": kind, "rows": rows, "hidden": hidden, "dtype": dtype, "vocab": vocab,
         "layer": layer, "grad_dtype": grad_dtype, "pad": pad}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # the final norm of a decode batch
        _case("norm", 64, 2048, "bf16", name="norm_64x2048_bf16_rms"),
        # a training batch
        _case("norm", 16384, 2048, "bf16", layer=True, name="norm_16384x2048_bf16_layer"),
        _case("norm_grad", 16384, 2048, "bf16", name="norm_grad_16384x2048_bf16_rms"),
        # rows of odd length in fp32: they start at odd addresses
        _case("norm_grad", 4099, 5001, "fp32", layer=True, name="norm_grad_4099x5001_fp32_layer"),
        # a prompt chunk's tokens
        _case("embed", 8192, 2048, "bf16", vocab=131072, name="embed_8192x2048_bf16"),
        # a small model's step, gradient in the main weights' type
        _case("embed_grad", 1021, 1024, "bf16", vocab=32000, grad_dtype="fp32",
              name="embed_grad_1021x1024_of_32000"),
        # a training batch: some tokens thousands of times
        _case("embed_grad", 32768, 2048, "bf16", vocab=131072, grad_dtype="bf16",
              name="embed_grad_32768x2048_of_131072"),
        # a small model's step on a few rows
        _case("loss_grad", 64, 1024, "bf16", vocab=32000, grad_dtype="bf16",
              name="loss_grad_64x1024_of_32000"),
        # an odd vocabulary and batch
        _case("loss_grad", 1021, 2048, "bf16", vocab=65537, grad_dtype="bf16",
              name="loss_grad_1021x2048_of_65537"),
        # evaluation of a held-out text
        _case("loss", 2048, 2048, "bf16", vocab=150001, name="loss_2048x2048_of_150001"),
        # a training batch
        _case("loss_grad", 4096, 2048, "bf16", vocab=131072, grad_dtype="bf16",
              name="loss_grad_4096x2048_of_131072"),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "embed", "embed_grad", "loss", "loss_grad"])
    rows = _spread(rng, 1, 32768)
    if kind in ("loss", "loss_grad"):
        hidden, vocab = 8 * _spread(rng, 16, 512), _spread(rng, 1000, 262144)
        rows = max(1, min(_spread(rng, 1, 8192), 4096 * 131072 * 2048 // (vocab * hidden)))
        return _case(kind, rows, hidden, "bf16", vocab=vocab,
                     grad_dtype="bf16" if kind == "loss_grad" else "")
    dtype, hidden = rng.choice(["bf16", "fp32"]), _spread(rng, 64, 16384)
    if rng.random() < 0.6:  # most widths are multiples of 64
        hidden = (hidden + 63) // 64 * 64
    rows = max(1, min(rows, 32768 * 4096 // hidden))
    pad = rng.choice([0, 0, rng.randrange(1, 64)])
    if kind in ("norm", "norm_grad"):
        return _case(kind, rows, hidden, dtype, layer=rng.random() < 0.5, pad=pad)
    vocab = min(_spread(rng, 1000, 262144), 262144 * 2048 // hidden)
    if kind == "embed":
        return _case(kind, rows, hidden, dtype, vocab=vocab)
    return _case(kind, rows, hidden, dtype, vocab=vocab, grad_dtype=rng.choice(["bf16", "fp32"]), pad=pad)


def _rows(case, values):
    """Rows as they were stored: in the case's type, `pad` elements apart."""
    out = torch.zeros((case["rows"], case["hidden"] + case["pad"]), dtype=DTYPES[case["dtype"]],
                      device="cuda")
    out[:, :case["hidden"]] = values
    return out[:, :case["hidden"]]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    kind, rows, hidden, vocab = case["kind"], case["rows"], case["hidden"], case["vocab"]
    dtype = DTYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda")
    s = {"case": case}
    if kind in ("norm", "norm_grad"):
        s["x"] = _rows(case, normal(rows, hidden) * (0.5 + 2.0 * uniform(rows, 1)) + 0.3 * normal(rows, 1))
        s["weight"] = 1.0 + 0.2 * normal(hidden)
        s["bias"] = 0.1 * normal(hidden) if case["layer"] else None
        if kind == "norm_grad":
            # the statistics as the forward pass left them
            x = s["x"].double()
            mean = x.mean(1)
            var = (x - mean[:, None]).square().mean(1) if case["layer"] else x.square().mean(1)
            s["mean"] = mean.float() if case["layer"] else None
            s["rstd"] = (var + 1e-5).rsqrt().float()
            s["grad"] = normal(rows, hidden).to(dtype)
        return s
    if kind in ("embed", "embed_grad"):
        ids = (vocab ** uniform(rows)).long().clamp(max=vocab) - 1
        # which ids are frequent has nothing to do with their order
        ids = torch.randperm(vocab, generator=g, device="cuda")[ids].to(torch.int32)
        ids[torch.randperm(rows, generator=g, device="cuda")[:rows // 16]] = PAD
        s["ids"] = ids
        s["scale"] = math.sqrt(hidden)
        if kind == "embed":
            s["table"] = (normal(vocab, hidden) * 0.02).to(dtype)
            s["out"] = torch.empty((rows, hidden), dtype=dtype, device="cuda")
        else:
            s["grad"] = _rows(case, normal(rows, hidden))
            s["out"] = torch.empty((vocab, hidden), dtype=DTYPES[case["grad_dtype"]], device="cuda")
        return s
    weight = (normal(vocab, hidden) * (1.5 / math.sqrt(hidden))).to(dtype)
    labels = (vocab ** uniform(rows)).long().clamp(max=vocab) - 1
    # the label's logit: 2 to 18 above what the background gives it
    lean = (2.0 + 16.0 * uniform(rows, 1)) / 1.5 ** 2
    s["hidden"] = (normal(rows, hidden) + lean * weight[labels].float()).to(dtype)
    labels[torch.randperm(rows, generator=g, device="cuda")[:rows // 10]] = IGNORE
    s["weight"], s["labels"] = weight, labels.to(torch.int32)
    s["row_weight"] = (labels >= 0).float() / (labels >= 0).sum()
    return s


def _plain_norm(x, weight, bias):
    x = x.float()
    mean = None
    if bias is not None:
        mean = x.mean(1, keepdim=True)
        x = x - mean
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5)
    y = x * rstd * weight
    if bias is None:
        return y, rstd[:, 0]
    return y + bias, mean[:, 0], rstd[:, 0]


def _plain_norm_grad(grad, x, weight, mean, rstd):
    d, n = grad.float(), x.float()
    if mean is not None:
        n = n - mean[:, None]
    n = n * rstd[:, None]
    g = d * weight
    dx = g - n * (g * n).mean(1, keepdim=True)
    if mean is not None:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * rstd[:, None]
    dw = (d * n).sum(0)
    return (dx, dw) if mean is None else (dx, dw, d.sum(0))


def _plain_loss(hidden, weight, labels, row_weight, grad):
    h, w = hidden.float(), weight.float()
    live = labels >= 0
    y = labels.clamp(min=0).long()[:, None]
    z = h @ w.T
    z = z - z.amax(1, keepdim=True)
    p = torch.exp(z)
    total = p.sum(1, keepdim=True)
    row = torch.where(live, (torch.log(total) - z.gather(1, y))[:, 0], 0.0)
    loss = (row * row_weight).sum()
    if not grad:
        return loss, row
    del z
    p *= row_weight[:, None] / total
    p.scatter_add_(1, y, -row_weight[:, None])
    p = torch.where(live[:, None], p, 0.0)
    return loss, row, p @ w, p.T @ h


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        return _run_own(s, c, kind)
    dtype = DTYPES[c["dtype"]]
    if kind == "norm":
        y, *stats = _plain_norm(s["x"], s["weight"], s["bias"])
        return (y.to(dtype), *stats)
    if kind == "norm_grad":
        dx, *rest = _plain_norm_grad(s["grad"], s["x"], s["weight"], s["mean"], s["rstd"])
        return (dx.to(dtype), *rest)
    if kind == "embed":
        ids = s["ids"].long()
        rows = s["table"][ids.clamp(min=0)].float() * s["scale"]
        return torch.where(ids[:, None] >= 0, rows, 0.0).to(dtype)
    if kind == "embed_grad":
        ids = s["ids"].long()
        # padding goes to a row of its own, which is cut off again
        out = torch.zeros((c["vocab"] + 1, c["hidden"]), device="cuda")
        out.index_add_(0, torch.where(ids >= 0, ids, c["vocab"]), s["grad"].float())
        return (out[:-1] * s["scale"]).to(DTYPES[c["grad_dtype"]])
    out = _plain_loss(s["hidden"], s["weight"], s["labels"], s["row_weight"], kind == "loss_grad")
    if kind == "loss":
        return out
    return out[0], out[1], out[2].to(dtype), out[3].to(DTYPES[c["grad_dtype"]])


def _run_own(s, c, kind):
    import paper_2609_34117_gb300 as sw
    if kind == "norm":
        y, mean, rstd = sw.slimwise_norm(s["x"], s["weight"], bias=s["bias"], layer=c["layer"], eps=1e-5)
        return (y, mean, rstd) if c["layer"] else (y, rstd)
    if kind == "norm_grad":
        dx, dw, db = sw.slimwise_norm_grad(s["grad"], s["x"], s["weight"], s["rstd"], mean=s["mean"],
                                           grad_bias=c["layer"])
        return (dx, dw, db) if c["layer"] else (dx, dw)
    if kind == "embed":
        return sw.slimwise_embed(s["table"], s["ids"], scale=s["scale"], out=s["out"])
    if kind == "embed_grad":
        return sw.slimwise_embed_grad(s["grad"], s["ids"], s["out"], scale=s["scale"])
    if kind == "loss":
        loss, row, _, _ = sw.slimwise_linear_loss(s["hidden"], s["weight"], s["labels"],
                                                  row_weight=s["row_weight"], grad_hidden=False,
                                                  grad_weight=False)
        return loss.reshape(()), row
    loss, row, dh, dw = sw.slimwise_linear_loss(s["hidden"], s["weight"], s["labels"],
                                                row_weight=s["row_weight"])
    return loss.reshape(()), row, dh, dw


def _distinct(n, vocab):
    """How many of n log-uniform ids differ: the sum over v of 1 - (1 - p_v)^n with
    p_v = 1 / (v ln vocab), as an integral over ln v."""
    c, steps = n / math.log(vocab), 1000
    at = [vocab ** ((i + 0.5) / steps) for i in range(steps)]
    return int(sum(v * (1.0 - math.exp(-c / v)) for v in at) * math.log(vocab) / steps)


def work(case):
    kind, rows, hidden, vocab = case["kind"], case["rows"], case["hidden"], case["vocab"]
    size = 2 if case["dtype"] == "bf16" else 4
    gsize = 4 if case["grad_dtype"] == "fp32" else 2
    n = rows * hidden
    vectors = hidden * 4 * (2 if case["layer"] else 1)
    stats = rows * 4 * (2 if case["layer"] else 1)
    if kind == "norm":
        return {"bytes": 2 * n * size + vectors + stats, "flops": 6 * n}
    if kind == "norm_grad":
        return {"bytes": 3 * n * size + hidden * 4 + vectors + stats, "flops": 12 * n}
    live = rows - rows // 16
    if kind == "embed":
        return {"bytes": (_distinct(live, vocab) * hidden + n) * size + 4 * rows, "flops": n}
    if kind == "embed_grad":
        return {"bytes": live * hidden * size + vocab * hidden * gsize + 4 * rows, "flops": live * hidden}
    live = rows - rows // 10  # the other rows' logits need not be computed
    if kind == "loss":
        return {"bytes": 2 * (live + vocab) * hidden + 12 * rows, "flops": 2 * live * vocab * hidden}
    return {"bytes": 2 * (live + vocab) * hidden + 12 * rows + 2 * n + vocab * hidden * gsize,
            "flops": 6 * live * vocab * hidden}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        return _exact_norm(s, case)
    if kind == "embed":
        ids = s["ids"].tolist()
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        at = [i for i, v in enumerate(ids) if v >= 0]
        out[at] = s["scale"] * s["table"].double()[s["ids"][at].long()]
        return out
    if kind == "embed_grad":
        live = s["ids"] >= 0
        order = torch.argsort(s["ids"][live].long(), stable=True)
        ids = s["ids"][live].long()[order]
        sums = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        grads = s["grad"][live][order]
        present, counts = torch.unique_consecutive(ids, return_counts=True)
        ends = torch.cumsum(counts, 0)
        # segment sums, a strip of columns at a time
        for a in range(0, case["hidden"], 256):
            run = torch.cumsum(grads[:, a:a + 256].double(), 0)[ends - 1]
            sums[present, a:a + 256] = torch.diff(run, dim=0, prepend=torch.zeros_like(run[:1]))
        return sums * s["scale"]
    return _exact_loss(s, case)


def _exact_norm(s, case):
    """The norm from its definition; its gradient by differentiating it."""
    rows, hidden = s["x"].shape
    step = max(1, (1 << 25) // hidden)
    back = case["kind"] == "norm_grad"
    parts, dw, db = [], 0.0, 0.0
    for a in range(0, rows, step):
        with torch.enable_grad():
            x = s["x"][a:a + step].double().requires_grad_(back)
            w = s["weight"].double().requires_grad_(back)
            b = torch.zeros_like(w) if s["bias"] is None else s["bias"].double()
            b.requires_grad_(back)
            mean = x.mean(1) if case["layer"] else torch.zeros(x.shape[0], dtype=x.dtype, device="cuda")
            rstd = ((x - mean[:, None]).pow(2).mean(1) + 1e-5).pow(-0.5)
            y = (x - mean[:, None]) * rstd[:, None] * w + b
            if back:
                gx, gw, gb = torch.autograd.grad(y, (x, w, b), s["grad"][a:a + step].double())
                parts.append((gx,))
                dw, db = dw + gw, db + gb
            else:
                parts.append((y, mean, rstd) if case["layer"] else (y, rstd))
    joined = [torch.cat(p) for p in zip(*parts)]
    if back:
        joined += [dw, db] if case["layer"] else [dw]
    return tuple(joined)


def _exact_loss(s, case):
    h, labels, weight = s["hidden"].double(), s["labels"].long(), s["row_weight"].double()
    live = torch.nonzero(labels >= 0)[:, 0]
    h, y, wt = h[live], labels[live], weight[live]
    vocab, step = case["vocab"], max(1, (1 << 26) // max(1, len(live)))
    pieces = [(a, min(vocab, a + step)) for a in range(0, vocab, step)]
    lse = torch.full((len(live),), -math.inf, dtype=torch.float64, device="cuda")
    for a, b in pieces:
        lse = torch.logaddexp(lse, torch.logsumexp(h @ s["weight"][a:b].double().T, 1))
    target = (h * s["weight"].double()[y]).sum(1)
    row = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
    row[live] = lse - target
    loss = (row * weight).sum()
    if case["kind"] == "loss":
        return loss, row
    dh = torch.zeros_like(s["hidden"], dtype=torch.float64)
    dw = torch.empty(s["weight"].shape, dtype=torch.float64, device="cuda")
    for a, b in pieces:
        w = s["weight"][a:b].double()
        dz = torch.exp(h @ w.T - lse[:, None])
        here = torch.nonzero((y >= a) & (y < b))[:, 0]
        dz[here, y[here] - a] -= 1.0
        dz *= wt[:, None]
        dh[live] += dz @ w
        dw[a:b] = dz.T @ h
    return loss, row, dh, dw
