"""A small CCQ language model fine-tuned with a clipped policy loss, on the library's operators end to end.

Rollout: tokens are sampled one at a time (embedding lookup, CCQ decode step on the recurrent state, gated group norm).
Training step: embedding lookup, CCQ-GLA forward with checkpoints, gated group norm, policy loss with its gradient
over the logits, and back: group norm, CCQ-GLA, embedding gradient; AdamW with 8-bit states on fp32
masters.  torch supplies the matrix products between them and chains the backward calls.

    python examples/policy_step.py [--steps 40]

The reward of a token is 1 where its id is even, so the mean reward starts near one half and rises.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_01294_gb300 import ccq, ops  # noqa: E402

HEADS, D = 2, 128
WIDTH = HEADS * D


class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids):
        ctx.save_for_backward(ids)
        ctx.rows = table.shape[0]
        return ops.embed(table, ids, scale=WIDTH ** 0.5)

    @staticmethod
    def backward(ctx, dout):
        return ops.embed_grad(dout.contiguous(), ctx.saved_tensors[0], ctx.rows, scale=WIDTH ** 0.5), None


class Mixer(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, gk, lam):
        o, _, ckpt = ccq.gla_fwd_save(q, k, v, gk, lam, return_state=False)
        ctx.save_for_backward(q, k, v, gk, lam, ckpt)
        return o

    @staticmethod
    def backward(ctx, dout):
        q, k, v, gk, lam, ckpt = ctx.saved_tensors
        g = ccq.gla_bwd(q, k, v, gk, lam, dout.contiguous(), ckpt=ckpt)
        return g["dq"], g["dk"], g["dv"], g["dgk"], g["dlambda"]


class GatedNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, gate):
        ctx.save_for_backward(x, weight, bias, gate)
        return ops.group_norm(x, weight, bias, gate, groups=HEADS)

    @staticmethod
    def backward(ctx, dout):
        g = ops.group_norm_bwd(*ctx.saved_tensors, dout, groups=HEADS)
        return g["dx"], g["dweight"], g["dbias"], g["dgate"]


class Model:
    """Embedding, ``layers`` CCQ-GLA token mixers with gated norms on a residual stream, and an output projection."""

    def __init__(self, vocab, layers, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape, size):
            return (size * torch.randn(*shape, device="cuda", generator=gen)).bfloat16().requires_grad_()

        def fill(value):
            return torch.full((WIDTH,), value, device="cuda", dtype=torch.bfloat16).requires_grad_()

        self.table = weight(vocab, WIDTH, size=WIDTH ** -0.5)
        self.head = weight(WIDTH, vocab, size=0.02)
        self.layers = [{"qkv": weight(WIDTH, 3 * WIDTH, size=WIDTH ** -0.5), "gates": weight(WIDTH, 2 * WIDTH, size=WIDTH ** -0.5),
                        "lam": weight(WIDTH, HEADS, size=0.02), "out": weight(WIDTH, WIDTH, size=WIDTH ** -0.5),
                        "norm_w": fill(1.0), "norm_b": fill(0.0)} for _ in range(layers)]

    def parameters(self):
        return [self.table, self.head] + [w for layer in self.layers for w in layer.values()]

    def forward(self, ids, states=None):
        """Logits of ids [B, T]; with ``states`` (a recurrent state per layer) of one more token each, ids [B]."""
        x = ops.embed(self.table, ids, scale=WIDTH ** 0.5) if states else Embed.apply(self.table, ids)
        shape = ids.shape + (HEADS, D)
        for i, w in enumerate(self.layers):
            q, k, v = (t.contiguous().view(shape) for t in (x @ w["qkv"]).chunk(3, -1))
            forget, gate = (x @ w["gates"]).chunk(2, -1)
            gk = (torch.nn.functional.logsigmoid(forget) / 16).contiguous().view(shape)
            lam = torch.sigmoid((x @ w["lam"]).float() - 1).contiguous()
            if states:
                o = ccq.decode_step(ccq.GLA, q, k, v, gk, lam, states[i])
                # (the gate is a slice of the projection: its rows lie 2 * WIDTH apart)
                o = ops.group_norm(o.view(-1, WIDTH), w["norm_w"], w["norm_b"], gate, groups=HEADS)
            else:
                o = GatedNorm.apply(Mixer.apply(q, k, v, gk, lam).view(x.shape), w["norm_w"], w["norm_b"], gate)
            x = x + o @ w["out"]
        return x @ self.head

    @torch.no_grad()
    def sample(self, batch, length, generator):
        """``length`` tokens for each of ``batch`` sequences that begin with token 0, by the decode step."""
        states = [ccq.CCQState.zeros(batch, HEADS, D, D, "cuda") for _ in self.layers]
        ids = [torch.zeros(batch, dtype=torch.int64, device="cuda")]
        for _ in range(length):
            p = torch.softmax(self.forward(ids[-1], states).float(), -1)
            ids.append(torch.multinomial(p, 1, generator=generator)[:, 0])
        return torch.stack(ids, 1)


def train(steps=40, batch=16, length=48, vocab=512, layers=2, epochs=2, lr=3e-3, seed=0, report=None):
    """Rounds of sampling and ``epochs`` updates on the sample; returns the mean reward of every round."""
    model = Model(vocab, layers, seed)
    params = model.parameters()
    optimizer, step, rewards = ops.adamw_state(params, bits=8, master=True), 0, []
    generator = torch.Generator(device="cuda").manual_seed(seed + 1)
    for round_ in range(steps):
        ids = model.sample(batch, length, generator)
        inputs, actions = ids[:, :-1].contiguous(), ids[:, 1:].contiguous()
        reward = (actions % 2 == 0).float()
        rewards.append(float(reward.mean()))
        advantages = 2 * (reward - reward.mean())
        with torch.no_grad():
            old = ops.token_logp(model.forward(inputs), actions)
        for _ in range(epochs):
            step += 1
            logits = model.forward(inputs)
            loss = ops.policy_loss(logits.detach(), actions, old, advantages, ref_logp=old, kl_coef=0.01)
            logits.backward(loss["dlogits"])
            grads = [p.grad for p in params]
            norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.float()) for g in grads]))
            with torch.no_grad():
                ops.adamw_step(params, grads, optimizer, step, lr=lr, betas=(0.9, 0.95), weight_decay=0.01,
                               grad_scale=(1.0 / norm.clamp_min(1.0)).float())
            for p in params:
                p.grad = None
        if report:
            report(round_, rewards[-1], float(loss["loss"]))
    ccq.device_status()
    return rewards


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=40)
    args = parser.parse_args()
    train(args.steps, report=lambda i, r, l: print(f"round {i:3d}  mean reward {r:.3f}  loss {l:+.4f}"))
