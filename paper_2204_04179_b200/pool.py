"""An encoder learns which item of the whole pool a user clicks next, and answers from a table in 8 bits: `python -m paper_2204_04179_b200.pool`.

A user is the mean of the encodings of the items in a history, and the answer over the pool is the softmax of user . item.  A
step encodes the pool, takes the loss of the clicked items over all items with the gradients of users and items
(`score_loss`, from the vectors themselves), sums the gradient of each item's encoding over its places in the histories, and runs the
encoder's backward pass and update.  Then the table is held as codes of 8 bits with a scale for each item (`quantize_rows`), and
users are answered from it (`gemm_i8`, `logprobs`).  Inputs and weights are random, of the sizes given.
"""
from __future__ import annotations

import argparse

import torch

from . import binding, distill, synth


class Learner(distill.Encoder):
    def gradient(self, histories: torch.Tensor, clicks: torch.Tensor, scale: float) -> torch.Tensor:
        """Encoder gradients of the mean over users of -log p(click); returns the loss per user."""
        g, N, (V, d), dev = self.gram, len(histories), self.H.shape, self.H.device
        items = self.encode(keep=True)
        loss, dU, G = torch.empty(N, device=dev), torch.empty(N, d, device=dev), torch.empty(V, d, device=dev)
        workspace = torch.empty(g.score_loss_workspace(N, V, d, torch.float32)[1], dtype=torch.uint8, device=dev)
        g.score_loss(self.users(histories), items, clicks, loss, workspace, scale=scale, weight=torch.full((N,), 1.0 / N, device=dev), dusers=dU, ditems=G)
        self.of_histories(G, dU, histories)
        g.zero_grads(binding.GRAM_MODULE_CE)
        g.encoder_backward(G, self.pool, V)
        return loss

    def step(self, histories: torch.Tensor, clicks: torch.Tensor, scale: float) -> torch.Tensor:
        loss = self.gradient(histories, clicks, scale)
        self.gram.optimizer_step(binding.GRAM_MODULE_CE)
        return loss


class Table:
    """The pool in 8 bits."""

    def __init__(self, gram: binding.Gram, items: torch.Tensor):
        self.gram, self.width = gram, -(-items.shape[1] // 16) * 16          # rows a multiple of 16 bytes apart
        self.codes, self.scale = self.coded(items)

    def coded(self, rows: torch.Tensor):
        codes = torch.empty(len(rows), self.width, dtype=torch.int8, device=rows.device)[:, :rows.shape[1]]
        scale = torch.empty(len(rows), device=rows.device)
        self.gram.quantize_rows(rows, codes, scale)
        return codes, scale

    def logits(self, users: torch.Tensor) -> torch.Tensor:
        """fp32 [N, n_items] from rows of users, fp32 or bf16."""
        codes, scale = self.coded(users)
        z = torch.empty(len(users), -(-len(self.codes) // 4) * 4, device=users.device)[:, :len(self.codes)]
        self.gram.gemm_i8(codes, scale, self.codes, self.scale, z)
        return z

    def answer(self, users: torch.Tensor, clicks: torch.Tensor, k: int, scale: float):
        """(log p(click) [N], the best k items [N, k])"""
        z, N, f = self.logits(users), len(users), dict(device=users.device)
        logp, top_logp, top_ids = torch.empty(N, 1, **f), torch.empty(N, k, **f), torch.empty(N, k, dtype=torch.int32, **f)
        self.gram.logprobs(z, scale=scale, targets=clicks.view(N, 1), logp=logp, top_logp=top_logp, top_ids=top_ids)
        return logp[:, 0], top_ids


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--items", type=int, default=2_600)
    p.add_argument("--users", type=int, default=512)
    p.add_argument("--steps", type=int, default=100)
    p.add_argument("--scale", type=float, default=1.0, help="one over the temperature")
    p.add_argument("--lr", type=float, default=1e-3)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args(argv)
    device = torch.device("cuda:0")
    _, shape = distill.shapes(n_items=a.items, users=a.users)
    learner = Learner(shape, synth.item_tokens(a.seed, a.items, shape.l_t, shape.vocab), a.seed, a.lr, device)
    ids = torch.from_numpy(synth.zipf_ids(a.seed, a.items, 1.0, a.users * (shape.L + 1)).reshape(a.users, shape.L + 1)).to(device)
    histories, clicks = ids[:, :-1].contiguous(), ids[:, -1].contiguous()
    for step in range(a.steps):
        loss = learner.step(histories, clicks, a.scale)
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step:4d}  loss {float(loss.mean()):.4f}")
    want, _ = learner.answer(histories, clicks, 10, a.scale)              # from bf16 encodings
    logp, ids = Table(learner.gram, learner.H).answer(learner.users(histories), clicks, 10, a.scale)
    print(f"log p(click) {want.click_logp:.4f}, from the table in 8 bits {float(logp.mean()):.4f}; the same first item for "
          f"{float((ids[:, 0] == want.top_ids[:, 0]).float().mean()):.3f} of the users")
    learner.gram.sync()
    learner.gram.close()
    return loss, logp


if __name__ == "__main__":
    main()
