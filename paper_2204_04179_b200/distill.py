"""A smaller encoder learns to answer over a pool as a larger one does: `python -m paper_2204_04179_b200.distill`.

Both read the same item texts.  A user is the mean of the encodings of the items in a history, and the answer over the pool
is the softmax of user . item.  The teacher's best items of every user come from `score_logprobs`.  A step of the
student encodes the pool, computes its logits, takes the loss and gradient of `distill` against the teacher's lists and of
`logprobs` / `logprobs_backward` for the items that were clicked (and for the entropy, which keeps the answers from narrowing
early), sums the gradient of each item's encoding over its places in the histories, and runs the encoder's backward pass and
update.  Inputs and weights are random, of the sizes given.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import numpy as np
import torch

from . import binding, synth


@dataclass
class Answers:
    """What a model answers: mean log probability of the clicked item, mean entropy, the best items of each user."""
    click_logp: float
    entropy: float
    top_ids: torch.Tensor


class Encoder:
    """One content encoder over the whole pool, with what a step needs around it."""

    def __init__(self, shape: synth.GramShape, tokens: np.ndarray, seed: int, lr: float, device: torch.device):
        cfg = binding.config_from_shape(shape, task=binding.GRAM_TASK_NONE, lr_ce=lr, optimizer=binding.GRAM_OPT_ADAM)
        cfg.ce_micro_batch = shape.n_items                # the pool's activations are kept for one backward pass
        self.gram, self.shape = binding.Gram(cfg), shape
        self.gram.set_params(binding.GRAM_MODULE_CE, synth.flatten(synth.encoder_params(shape, seed, sigma=0.1)))
        self.gram.set_item_tokens(tokens)
        self.pool = torch.arange(shape.n_items, dtype=torch.int32, device=device)
        self.H = torch.empty(shape.n_items, shape.d, device=device)

    def encode(self, keep: bool = False) -> torch.Tensor:
        """bf16 [n_items, d]; keep: with what the backward pass needs."""
        self.gram.encode_unique(None, self.pool, self.shape.n_items, self.H, save_activations=keep)
        return self.H.to(torch.bfloat16)

    def users(self, histories: torch.Tensor) -> torch.Tensor:
        """bf16 [N, d] for histories int32 [N, L], of the last encode()."""
        E = torch.empty(histories.numel(), self.shape.d, device=self.H.device)
        self.gram.gather(self.H, histories, E)
        return E.view(*histories.shape, -1).mean(1).to(torch.bfloat16)

    def of_histories(self, G: torch.Tensor, dU: torch.Tensor, histories: torch.Tensor):
        """Adds to the items' gradients G [n_items, d] what the users' gradients dU [N, d] leave in their histories' items."""
        g, (N, L), (V, d), dev = self.gram, histories.shape, self.H.shape, self.H.device
        P = N * L
        index = lambda n: torch.empty(n, dtype=torch.int32, device=dev)  # noqa: E731
        unique, inverse, perm, seg_off, count = index(P), index(P), index(P), index(P + 1), index(1)
        g.dedup(histories, V, unique, inverse, perm, seg_off, count)
        U = int(count)
        sums = torch.empty(U, d, device=dev)
        g.accumulate((dU / L).repeat_interleave(L, 0), perm, seg_off, U, sums)
        G[unique[:U].long()] += sums

    def answer(self, histories: torch.Tensor, clicks: torch.Tensor, k: int, scale: float):
        """(Answers, log probabilities of the best k items)."""
        N, f = len(histories), dict(device=self.H.device, dtype=torch.float32)
        items = self.encode()
        logp, entropy, top_logp = torch.empty(N, 1, **f), torch.empty(N, **f), torch.empty(N, k, **f)
        top_ids = torch.empty(N, k, device=self.H.device, dtype=torch.int32)
        self.gram.score_logprobs(self.users(histories), items, scale=scale, targets=clicks.view(N, 1), logp=logp, entropy=entropy,
                                 top_logp=top_logp, top_ids=top_ids)
        return Answers(float(logp.mean()), float(entropy.mean()), top_ids), top_logp


class Student(Encoder):
    def gradient(self, histories: torch.Tensor, clicks: torch.Tensor, teacher_ids: torch.Tensor, teacher_logp: torch.Tensor, scale: float,
                 of_clicks: float = 0.0, of_entropy: float = 0.0):
        """Encoder gradients of the mean over users of  distillation loss - of_clicks log p(click) - of_entropy H; returns
        (distillation loss, log p(click), H) per user."""
        g, (N, L), (V, d), dev = self.gram, histories.shape, self.H.shape, self.H.device
        new = lambda *size: torch.empty(*size, device=dev)  # noqa: E731
        items = self.encode(keep=True)
        users = self.users(histories)
        z, dz = new(N, V), new(N, V)
        g.gemm_bf16(users, True, items, True, z, None, False, N, V, d)
        clicks = clicks.view(N, 1)
        logp, stats, entropy, loss = new(N, 1), new(N, 2), new(N), new(N)
        g.logprobs(z, scale=scale, targets=clicks, logp=logp, stats=stats, entropy=entropy)
        g.distill(z, teacher_ids, teacher_logp, loss, scale=scale, weight=torch.full((N,), 1.0 / N, device=dev), dlogits=dz)
        g.logprobs_backward(z, stats, z, scale=scale, targets=clicks, dlogp=torch.full((N, 1), -of_clicks / N, device=dev), entropy=entropy,
                            dentropy=torch.full((N,), -of_entropy / N, device=dev))
        dz = dz.add_(z).to(torch.bfloat16)
        # of the pool's encodings: as items, and as parts of the histories' means
        G, dU = new(V, d), new(N, d)
        g.gemm_bf16(dz, False, users, False, G, None, False, V, d, N)
        g.gemm_bf16(dz, True, items, False, dU, None, False, N, d, V)
        self.of_histories(G, dU, histories)
        g.zero_grads(binding.GRAM_MODULE_CE)
        g.encoder_backward(G, self.pool, V)
        return loss, logp[:, 0], entropy

    def step(self, *args, **kw):
        out = self.gradient(*args, **kw)
        self.gram.optimizer_step(binding.GRAM_MODULE_CE)
        return out


def shapes(n_items=2_600, l_t=16, d=128, teacher_layers=3, student_layers=1, users=512, history=20):
    teacher = synth.GramShape(name="teacher", dtype="bf16", n_items=n_items, l_t=l_t, vocab=1000, d=d, n_heads=d // 64, d_ff=4 * d, n_layers=teacher_layers,
                              task_heads=d // 64, task_d_ff=4 * d, B=users, L=history)
    return teacher, teacher.replace(name="student", n_layers=student_layers)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--items", type=int, default=2_600)
    p.add_argument("--users", type=int, default=512)
    p.add_argument("--steps", type=int, default=100)
    p.add_argument("--k", type=int, default=32, help="items of the teacher's lists")
    p.add_argument("--scale", type=float, default=1.0, help="one over the temperature")
    p.add_argument("--lr", type=float, default=1e-3)
    p.add_argument("--clicks", type=float, default=0.1, help="weight of the clicked items' log probability")
    p.add_argument("--entropy", type=float, default=0.01, help="weight of the entropy")
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args(argv)
    if a.items % 8 or a.users % 8:
        p.error("the matrix products take items and users in multiples of 8")
    device = torch.device("cuda:0")
    big, small = shapes(n_items=a.items, users=a.users)
    tokens = synth.item_tokens(a.seed, a.items, big.l_t, big.vocab)
    teacher = Encoder(big, tokens, a.seed, 0.0, device)
    student = Student(small, tokens, a.seed + 1, a.lr, device)
    histories = torch.from_numpy(synth.zipf_ids(a.seed, a.items, 1.0, a.users * big.L).reshape(a.users, big.L)).to(device)
    want, _ = teacher.answer(histories, histories[:, 0].contiguous(), a.k, a.scale)
    clicks = want.top_ids[:, 0].contiguous()             # the users do as the teacher says
    want, _ = teacher.answer(histories, clicks, a.k, a.scale)
    _, teacher_logp = teacher.answer(histories, clicks, a.k, 1.0)      # `distill` scales the teacher's logits itself
    report = lambda got: (f"log p(click) {got.click_logp:8.4f}  entropy {got.entropy:7.4f}  first item the teacher's "  # noqa: E731
                          f"{float((got.top_ids[:, 0] == clicks).float().mean()):.3f}")
    print("teacher   ", report(want))
    print("before    ", report(student.answer(histories, clicks, 10, a.scale)[0]))
    first = last = None
    for step in range(a.steps):
        loss, _, _ = student.step(histories, clicks, want.top_ids, teacher_logp, a.scale, a.clicks, a.entropy)
        last = float(loss.mean())
        first = last if first is None else first
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step:4d}  distillation loss {last:.4f}")
    print("after     ", report(student.answer(histories, clicks, 10, a.scale)[0]))
    for e in (teacher, student):
        e.gram.sync()
        e.gram.close()
    return first, last


if __name__ == "__main__":
    main()
