"""The operators around the layer together, as a program runs them: the bigram model of
the distillation example and its gradients, captured into graphs, on other streams,
from two threads, and beside the layer."""
import threading

import pytest
import torch

import paper_2609_34117_gb300 as sw
from paper_2609_34117_gb300 import distill, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sw.build.build()


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ends(vocab, width, rows, seed):
    g = _gen(seed)
    embed = torch.randn((vocab, width), generator=g, device=DEV).to(BF16)
    head = (torch.randn((vocab, width), generator=g, device=DEV) * 2 / width ** 0.5).to(BF16)
    gamma = 1 + 0.1 * torch.randn(width, generator=g, device=DEV)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    labels = torch.randint(0, vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    labels[::7], tokens[::11] = -1, tokens[0]
    return embed, gamma, head, tokens, labels


@pytest.mark.parametrize("vocab,width,rows", [(311, 128, 40), (1000, 264, 300), (5003, 1024, 700)])
def test_bigram_gradients(vocab, width, rows):
    embed, gamma, head, tokens, labels = _ends(vocab, width, rows, seed=rows)
    loss, dembed, dgamma, dhead = distill.bigram_gradients(embed, gamma, head, tokens, labels)
    e, w, v = (t.double().requires_grad_() for t in (embed, gamma, head))
    h = e[tokens.long()]
    n = h * (h.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w
    n = n + (n.detach().to(BF16).double() - n.detach())  # rounded where the model rounds it
    live = labels >= 0
    z = n @ v.T
    ce = torch.logsumexp(z, 1) - z.gather(1, labels.clamp(min=0).long()[:, None])[:, 0]
    want = ce[live].mean()
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-4 * want.item()
    # roundings to bf16 on the way, half a step of each value: of n (a value next to a border:
    # a whole step), the numerators (two), the scaled rows, dn and dh
    for got, ref, roundings in ((dhead, v.grad, 5), (dgamma, w.grad, 5), (dembed, e.grad, 6)):
        assert float((got.double() - ref).norm()) <= roundings * 2.0 ** -8 * float(ref.norm())


def test_pretraining_runs_and_the_model_can_be_distilled_then():
    model = distill.Model.random(vocab=2003)
    before = [t.clone() for t in (model.embed, model.gamma, model.head)]
    losses = distill.pretrain(model, 3, batch=64)
    assert len(losses) == 3 and all(x == x for x in losses)
    assert all(not torch.equal(a, b) for a, b in zip(before, (model.embed, model.gamma, model.head)))
    gamma, _ = distill.distill(model, steps=2, batch=64)
    tokens = torch.arange(200, device=DEV)
    labels = torch.randint(0, 2003, (200,), generator=_gen(1), device=DEV, dtype=torch.int32)
    labels[3] = -1
    for full in (False, True):
        got = distill.evaluate(model, gamma, tokens, labels, full)
        z = model.logits(model.normed(tokens, full), gamma).double()
        live = labels >= 0
        want = (torch.logsumexp(z, 1) - z.gather(1, labels.clamp(min=0).long()[:, None])[:, 0])[live].mean()
        # the logits of the reference are rounded to bf16: half a step of the largest, twice
        assert abs(float(got) - float(want)) <= 2 * 2.0 ** -8 * float(z.abs().max())


def test_embedding_in_the_model_is_its_rows():
    model = distill.Model.random(vocab=503)
    tokens = torch.randint(0, 503, (77,), generator=_gen(2), device=DEV)
    assert torch.equal(sw.slimwise_embed(model.embed, tokens.int()), model.embed[tokens])


def _step(embed, gamma, head, tokens, labels):
    return distill.bigram_gradients(embed, gamma, head, tokens, labels)


def test_captured_and_replayed_with_other_inputs():
    a, b = _ends(3001, 264, 500, seed=1), _ends(3001, 264, 500, seed=2)
    b[4][::2] = -1  # another number of labelled rows
    static = [t.clone() for t in a]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(*static)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):  # two graphs, replayed in turn
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_step(*static))
        graphs.append(g)
    for inputs in (b, a, b):
        want = [t.clone() for t in _step(*inputs)]
        for t, x in zip(static, inputs):
            t.copy_(x)
        for g, out in zip(graphs, outs):
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, want))


def test_outputs_and_workspaces_are_memory_of_the_stream_that_uses_them():
    embed, gamma, head, tokens, labels = _ends(3001, 264, 300, seed=3)
    h = sw.slimwise_embed(embed, tokens)
    n, _, rstd = sw.slimwise_norm(h, gamma)
    side = torch.cuda.Stream()
    calls = [lambda s: (sw.slimwise_embed(embed, tokens, stream=s),),
             lambda s: sw.slimwise_norm(h, gamma, layer=True, stream=s),
             lambda s: sw.slimwise_norm_grad(n, h, gamma, rstd, stream=s)[:2],
             lambda s: sw.slimwise_linear_loss(n, head, labels, stream=s)]
    for call in calls:
        want = [t.clone() for t in call(None)]
        torch.cuda.synchronize()
        shapes = [(t.shape, t.dtype) for t in call(side)]
        side.synchronize()
        given_back = [torch.empty(s, dtype=d, device=DEV) for s, d in shapes * 4]
        at = {t.data_ptr() for t in given_back}
        del given_back
        got = call(side)
        side.synchronize()
        assert not at & {t.data_ptr() for t in got}
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    out, other = torch.empty((2, 3001, 264), device=DEV).unbind(0)
    sw.slimwise_embed_grad(h, tokens, out)
    torch.cuda.synchronize()
    sw.slimwise_embed_grad(h, tokens, other, stream=side)
    side.synchronize()
    assert torch.equal(out, other)


def test_two_threads_on_two_streams():
    inputs = [_ends(3001, 264, 500, seed=4), _ends(20011, 1024, 90, seed=5)]
    want = [[t.clone() for t in _step(*i)] for i in inputs]
    torch.cuda.synchronize()
    errors, start = [], threading.Barrier(2)

    def work(i):
        try:
            stream = torch.cuda.Stream()
            start.wait()
            with torch.cuda.stream(stream):
                for _ in range(60):
                    got = _step(*inputs[i])
            stream.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, want[i]))
        except Exception as e:
            errors.append(e)
            start.abort()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


def test_beside_the_layer_on_another_stream():
    # both use tensor memory and most of an SM's shared memory
    shape = synth.QWEN
    w_gu, w_d = synth.expert_weights(shape, 0, device=DEV)
    wr = synth.router_weight(shape, 0, device=DEV)
    x = synth.hidden_states(64, shape, 1, device=DEV)
    inputs = _ends(8001, 1024, 600, seed=6)
    want = [t.clone() for t in _step(*inputs)]
    layer = sw.slimwise_moe_decode_full(x, wr, w_gu, w_d, shape.top_k).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(20):
        with torch.cuda.stream(side):
            out = sw.slimwise_moe_decode_full(x, wr, w_gu, w_d, shape.top_k)
        got = _step(*inputs)
    torch.cuda.synchronize()
    assert torch.equal(out, layer) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_workspace_that_another_call_has_used():
    embed, gamma, head, tokens, labels = _ends(3001, 264, 300, seed=7)
    n = sw.slimwise_norm(sw.slimwise_embed(embed, tokens), gamma)[0]
    want = sw.slimwise_linear_loss(n, head, labels)
    ws = torch.empty(sw.slimwise_linear_loss_workspace_size(900, 264, 3001), dtype=torch.uint8, device=DEV)
    big = _ends(3001, 264, 900, seed=8)
    sw.slimwise_linear_loss(sw.slimwise_embed(big[0], big[3]) * 30, head, big[4], workspace=ws)
    got = sw.slimwise_linear_loss(n, head, labels, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert sw.slimwise_moe_device_status(ws) == 0
    with pytest.raises(sw.SlimwiseError):
        sw.slimwise_linear_loss(n, head, labels, workspace=ws[:1024])
