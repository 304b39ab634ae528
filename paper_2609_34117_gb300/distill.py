"""Distillation of a pruned layer's model, and sampling from it: the operators
over vocabulary logits as a program uses them.

SlimWise can follow pruning by a short distillation (Sec. 3.3): the teacher keeps
the full expert pool, the student the retained one and a shared expert, and a
small part of the student is trained on cross entropy and on the KL against the
teacher's top-K log-probabilities with a bucket for the residual mass (Eq. 3,
alpha = 0.1, K = 64).  The model here is one layer between an embedding and a
vocabulary head with seeded random weights:

    h = embed(token);  y = h + MoE(h);  logits = (gamma * y / rms(y)) head^T

The teacher's layer is slimwise_moe_decode_full, the student's
slimwise_moe_decode_shared over the retained experts.  Of what the paper trains
(norms, routers, the shared expert) this trains the norm's gamma, whose gradient
needs the loss's and the head alone; the library has no backward pass of the
layer.  A step:

    targets  = slimwise_top_logits(teacher logits, K)
    loss, dz = slimwise_distill_loss(student logits, labels, *targets)
    dgamma   = sum over tokens of (dz head) * y / rms(y);  Adam

and in the end the student answers: slimwise_sample draws each row's next token.
evaluate() is the cross entropy of either model on given next tokens, without its
logits (slimwise_norm, slimwise_linear_loss).

The model's ends can be trained on text first (pretrain(), --pretrain steps): the
embedding, the norm and the head alone are a bigram model, whose gradients the
library has in full:

    h = slimwise_embed(tokens);  n = slimwise_norm(h)
    loss, dn, dhead = slimwise_linear_loss(n, head, labels)
    dh, dgamma = slimwise_norm_grad(dn);  dembed = slimwise_embed_grad(dh, tokens)

    python -m paper_2609_34117_gb300.distill [--steps 30] [--vocab 32000] [--pretrain 0]
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import torch

from . import binding, synth

IGNORE = -100  # label of a token that is not trained on


@dataclass
class Model:
    """Weights of the one-layer model (embedding and head bf16 [V, H], layer,
    shared expert, norm gamma fp32 [H])."""
    shape: synth.LayerShape
    embed: torch.Tensor
    head: torch.Tensor
    w_gate_up: torch.Tensor
    w_down: torch.Tensor
    router: torch.Tensor
    retained: torch.Tensor
    shared: tuple
    gamma: torch.Tensor

    @classmethod
    def random(cls, shape=synth.TINY, vocab=32000, retained=8, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        draw = lambda std: (torch.randn((vocab, shape.hidden), generator=g, device=device) * std).to(torch.bfloat16)
        w_gate_up, w_down = synth.expert_weights(shape, seed, device=device)
        # experts large enough for the layer to matter to the logits
        return cls(shape, draw(1.0), draw(4.0 / shape.hidden ** 0.5), w_gate_up * 8, w_down * 8,
                   synth.router_weight(shape, seed, device=device),
                   synth.retained_set(shape.num_experts, retained, seed + 2).to(device),
                   synth.shared_expert(shape.hidden, shape.inter, seed + 3, device=device),
                   torch.ones(shape.hidden, device=device))

    def normed(self, tokens, full):
        """y / rms(y) of the layer's output, fp32 [B, H]: the full pool's, or the
        retained pool's with the shared expert."""
        y = self.output(tokens, full)
        return y / y.square().mean(1, keepdim=True).sqrt()

    def output(self, tokens, full):
        """The layer's output with its residual, fp32 [B, H]."""
        h = binding.slimwise_embed(self.embed, tokens.int())
        args = (h, self.router)
        if full:
            out = binding.slimwise_moe_decode_full(*args, self.w_gate_up, self.w_down, self.shape.top_k)
        else:
            out = binding.slimwise_moe_decode_shared(*args, self.retained, self.w_gate_up, self.w_down,
                                                     self.shape.top_k, *self.shared)
        return h.float() + out.float()

    def logits(self, normed, gamma):
        return (normed * gamma).to(torch.bfloat16) @ self.head.T


def distill(model: Model, steps=30, batch=256, k=64, alpha=0.1, temperature=1.0, lr=0.02, seed=1):
    """Trains a student's gamma; returns (gamma, the loss of each step)."""
    dev = model.gamma.device
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    gamma = model.gamma.clone()
    m, v = torch.zeros_like(gamma), torch.zeros_like(gamma)
    losses = []
    for step in range(1, steps + 1):
        tokens = torch.randint(0, model.embed.shape[0], (batch,), generator=g, device=dev)
        targets = binding.slimwise_top_logits(model.logits(model.normed(tokens, True), model.gamma), k,
                                              temperature=temperature)
        # the text's next token: the teacher's likeliest; prompt tokens have none
        labels = targets[0][:, 0].contiguous()
        labels[::8] = IGNORE
        weight = (labels >= 0).float() / (labels >= 0).sum()
        n = model.normed(tokens, False)
        z = model.logits(n, gamma)
        loss, _, dz = binding.slimwise_distill_loss(z, labels, *targets, alpha=alpha,
                                                    temperature=temperature, row_weight=weight, grad=z)
        grad = ((dz @ model.head).float() * n).sum(0)
        m.lerp_(grad, 0.1)
        v.lerp_(grad * grad, 0.01)
        gamma -= lr * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-8)
        losses.append(loss)
    return gamma, torch.cat(losses).tolist()


def evaluate(model: Model, gamma, tokens, labels, full):
    """Mean cross entropy of the full pool's or the retained pool's model at labels
    (int32; negative: no label), fp32 [1]."""
    n, _, _ = binding.slimwise_norm(model.output(tokens, full), gamma, eps=0.0)
    weight = (labels >= 0).float() / (labels >= 0).sum()
    return binding.slimwise_linear_loss(n.to(torch.bfloat16), model.head, labels, row_weight=weight,
                                        grad_hidden=False, grad_weight=False)[0]


def bigram_gradients(embed, gamma, head, tokens, labels, eps=1e-5):
    """Loss and gradients of the model's ends without the layer: (loss fp32 [1],
    gradients of the embedding fp32 [V, H], of gamma fp32 [H], of the head fp32 [V, H])."""
    weight = (labels >= 0).float() / (labels >= 0).sum()
    h = binding.slimwise_embed(embed, tokens)
    n, _, rstd = binding.slimwise_norm(h, gamma, eps=eps)
    fp32 = lambda t: torch.empty(t.shape, dtype=torch.float32, device=t.device)
    loss, _, dn, dhead = binding.slimwise_linear_loss(n, head, labels, row_weight=weight, grad_weight=fp32(head))
    dh, dgamma, _ = binding.slimwise_norm_grad(dn, h, gamma, rstd)
    return loss, binding.slimwise_embed_grad(dh, tokens, fp32(embed)), dgamma, dhead


def pretrain(model: Model, steps, batch=256, lr=0.5, seed=2):
    """Trains the embedding, gamma and the head in place on a seeded text in which each
    token has one successor; returns the loss of each step."""
    dev = model.gamma.device
    vocab = model.embed.shape[0]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    successor = torch.randperm(vocab, generator=g, device=dev).int()
    losses = []
    for _ in range(steps):
        tokens = torch.randint(0, vocab, (batch,), generator=g, device=dev, dtype=torch.int32)
        labels = successor[tokens.long()]
        loss, dembed, dgamma, dhead = bigram_gradients(model.embed, model.gamma, model.head, tokens, labels)
        for w, d in ((model.embed, dembed), (model.gamma, dgamma), (model.head, dhead)):
            w.copy_(w.float() - lr * d)
        losses.append(loss)
    return torch.cat(losses).tolist() if losses else []


def answer(model: Model, gamma, tokens, uniform, temperature=0.7, top_k=20, top_p=0.8):
    """The student's next token of each row, and its log-probability."""
    rows = tokens.shape[0]
    full = lambda x, dtype: torch.full((rows,), x, dtype=dtype, device=tokens.device)
    return binding.slimwise_sample(model.logits(model.normed(tokens, False), gamma), uniform,
                                   temperature=full(temperature, torch.float32),
                                   top_k=full(top_k, torch.int32), top_p=full(top_p, torch.float32))


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--pretrain", type=int, default=0, help="steps of training the model's ends first")
    a = ap.parse_args()
    model = Model.random(vocab=a.vocab)
    if a.pretrain:
        first = pretrain(model, a.pretrain)
        print(f"bigram loss {first[0]:.4f} ... {first[-1]:.4f}")
    gamma, losses = distill(model, a.steps, a.batch)
    print("loss", " ".join(f"{x:.4f}" for x in losses[::max(1, a.steps // 10)]), f"... {losses[-1]:.4f}")
    prompt = torch.arange(8, device="cuda")
    uniform = torch.rand(8, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
    tokens, logprob = answer(model, gamma, prompt, uniform)
    held_out = torch.arange(0, min(a.vocab, 4096), device="cuda")
    likeliest = binding.slimwise_top_logits(model.logits(model.normed(held_out, True), model.gamma), 1)[0][:, 0]
    entropy = lambda gamma, full: float(evaluate(model, gamma, held_out, likeliest.contiguous(), full))
    print(f"cross entropy at the teacher's likeliest tokens: teacher {entropy(model.gamma, True):.4f}, student "
          f"{entropy(model.gamma, False):.4f}, distilled {entropy(gamma, False):.4f}")
    print("answers", tokens.tolist(), "log-probabilities", [round(x, 3) for x in logprob.tolist()])


if __name__ == "__main__":
    main()
