"""Trains the scales of a quantized output layer on the answers of the layer it was made from.

The teacher is a dense output layer W [V, hidden], the student its binary-coded form, whose sign planes are frozen (AlphaTuning
Section 4.1).  Of every token's distribution over V the teacher hands on only its k best logits, their indices and its log sum
(`bcq_logprobs_fwd`: 8 k + 4 bytes a token instead of 2 V).  A training step is then three calls: the student's logits, loss
with gradient in one reading of them (`bcq_distill_fwd_bwd`), and the scales' gradient with their AdamW step
(`bcq_linear_bwd_alpha_adamw`).  With --autograd the same through `BCQLinear`, `autograd.distill_loss` and torch's optimizer.
Before and after, the student is scored on tokens that are not trained on: distillation loss, log probability of the teacher's
best tokens, entropy, and how often its best token is the teacher's.

    python examples/distill_output_layer.py --tokens 2048 --vocab 50257 --hidden 1024 --steps 40
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2210_03858_amd as bcq  # noqa: E402
from paper_2210_03858_amd import autograd  # noqa: E402

OP_FWD, OP_BWD_ALPHA, OP_DISTILL_FWD_BWD, BF16 = 1, 3, 6, 1


def workspace(nbytes):
    return torch.empty((max(nbytes, 16),), dtype=torch.uint8, device="cuda")


class Data:
    """Random hidden states whose columns differ in size, a new batch at every call."""

    def __init__(self, tokens, hidden, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.shape = (tokens, hidden)
        size = torch.exp(torch.randn((hidden,), generator=self.gen, device="cuda"))
        self.size = size / size.square().mean().sqrt()

    def __call__(self):
        return (torch.randn(self.shape, generator=self.gen, device="cuda") * self.size).bfloat16()


def teach(W, h, k):
    """The teacher's k best logits, their indices and its log sum, for every row of h."""
    out = bcq.bcq_logprobs_fwd(h @ W.bfloat16().t(), k=k, lse=True)
    return out.top_logit, out.top_index, out.lse


def score(logits, lesson):
    """Means over the rows: distillation loss, log probability of the teacher's best token, entropy, same best token."""
    top_logit, top_index, lse = lesson
    loss = bcq.bcq_distill_fwd(logits, top_logit, top_index, lse)
    best = top_index[:, 0].long()
    out = bcq.bcq_logprobs_fwd(logits, best, k=1, entropy=True)
    return tuple(v.float().mean().item() for v in (loss, out.logp, out.entropy, out.top_index[:, 0] == best))


def train_calls(layer, W, data, k, steps, lr):
    """The training steps as calls on buffers that are made once.  Returns the mean loss of every step."""
    packed, m = layer.packed, torch.zeros_like(layer.alpha_train)
    v, (q, N, _), (T, K) = torch.zeros_like(m), packed.shape, data.shape
    alpha = layer.alpha_train.detach()
    alpha = alpha.clone() if layer.alpha_frozen is None else torch.cat((alpha, layer.alpha_frozen))
    weight = torch.full((T,), 1.0 / T, device="cuda")
    ws = workspace(max(bcq.workspace_bytes(OP_FWD, T, N, K, q, BF16), bcq.workspace_bytes(OP_BWD_ALPHA, T, N, K, q, BF16),
                       bcq.logits_workspace_bytes(OP_DISTILL_FWD_BWD, T, N, k, BF16)))
    logits = torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
    losses = torch.empty((steps, T), device="cuda")
    for step in range(steps):
        h = data()
        top_logit, top_index, lse = teach(W, h, k)
        bcq.bcq_linear_fwd_grouped(packed, alpha, h, K, y=logits, workspace=ws)
        bcq.bcq_distill_fwd_bwd(logits, top_logit, top_index, weight=weight, teacher_lse=lse, loss=losses[step], dlogits=logits,
                                workspace=ws)  # the gradient takes the logits' place
        bcq.bcq_linear_bwd_alpha_adamw(packed, h, logits, K, alpha, m, v, step + 1, lr, q_train=m.shape[0], workspace=ws)
    with torch.no_grad():
        layer.alpha_train.copy_(alpha[:m.shape[0]])
    return losses.mean(1).tolist()


def train_autograd(layer, W, data, k, steps, lr):
    """The same with a torch optimizer."""
    optimizer = torch.optim.AdamW([layer.alpha_train], lr=lr, weight_decay=0.0)
    losses = []
    for _ in range(steps):
        h = data()
        loss = autograd.distill_loss(layer(h), *teach(W, h, k)).mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    return torch.stack(losses).tolist()


def run(tokens=1024, vocab=8000, hidden=512, q=3, q_train=1, k=64, steps=30, lr=2e-4, use_autograd=False, seed=0):
    """Returns (losses, score before, score after)."""
    data = Data(tokens, hidden, seed)
    W = torch.randn((vocab, hidden), generator=data.gen, device="cuda") * (4.0 / hidden ** 0.5)
    layer = autograd.BCQLinear.from_weight(W, q, q_train=q_train)
    unseen = data()
    lesson = teach(W, unseen, k)
    with torch.no_grad():
        before = score(layer(unseen), lesson)
    losses = (train_autograd if use_autograd else train_calls)(layer, W, data, k, steps, lr)
    with torch.no_grad():
        return losses, before, score(layer(unseen), lesson)


def main():
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("tokens", 1024), ("vocab", 8000), ("hidden", 512), ("q", 3), ("q-train", 1), ("k", 64), ("steps", 30),
                        ("seed", 0)):
        parser.add_argument("--" + name, type=int, default=value)
    parser.add_argument("--lr", type=float, default=2e-4)
    parser.add_argument("--autograd", dest="use_autograd", action="store_true")
    losses, before, after = run(**vars(parser.parse_args()))
    for step in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %3d  loss %.5f" % (step, losses[step]))
    print("step %3d  loss %.5f" % (len(losses) - 1, losses[-1]))
    for name, (loss, logp, entropy, hit) in (("before", before), ("after", after)):
        print("%-6s  unseen: loss %.5f  log probability of the teacher's best tokens %.4f  entropy %.4f  same best token %.1f %%" %
              (name, loss, logp, entropy, 100 * hit))


if __name__ == "__main__":
    main()
