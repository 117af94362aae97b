"""Next-item prediction over a table of items: the operators on sequences of tokens in one training step, and the
answer to a single user.

  tokens -> scaled lookup with dropout -> gated block -> down projection -> dropout + residual -> logits over the
  table -> log probability of the item that came next; back through the same operators; Adam on the flat parameters.

The synthetic users follow a fixed chain of items nine times out of ten.  Plain products are torch's; everything else
is the library's.     python examples/next_item.py [--steps 60]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2404_09679_amd as A  # noqa: E402

BF16 = torch.bfloat16


class NextItem:
    """Table [items, width], gated block of `hidden`, down projection: fp32 parameters in one flat vector, bf16 copies
    as operands."""

    def __init__(self, items: int, width: int, hidden: int, seed: int = 0, p: float = 0.1, device: str = "cuda"):
        self.items, self.width, self.p, self.seed = items, width, p, seed
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        shapes = {"table": (items, width), "wg": (width, hidden), "wu": (width, hidden), "wd": (hidden, width)}
        sizes = [a * b for a, b in shapes.values()]
        self.flat = torch.empty(sum(sizes), device=device)
        self.grad = torch.empty_like(self.flat)
        self.m, self.v = torch.zeros_like(self.flat), torch.zeros_like(self.flat)
        self.half = torch.empty_like(self.flat, dtype=BF16)
        views = [dict(zip(shapes, (t.view(s) for t, s in zip(x.split(sizes), shapes.values()))))
                 for x in (self.flat, self.grad, self.half)]
        self.par, self.dpar, self.op = views
        for name, t in self.par.items():
            t.normal_(0.0, 0.5 * width ** -0.5 if name == "table" else t.shape[0] ** -0.5, generator=gen)
        self.half.copy_(self.flat)
        self.steps = 0

    def forward(self, tokens: torch.Tensor, training: bool):
        """Hidden state of every token, and what the backward pass needs."""
        o, s = self.op, {"tokens": tokens}
        drop = [A.Dropout(self.p, self.seed + self.steps, call) if training else None for call in (0, 1)]
        x = A.token_lookup(o["table"], tokens, self.width ** 0.5, dropout=drop[0])
        s["saved"] = A.gated_saved(x, o["wg"]) if training else None
        h = A.gated_forward(x, o["wg"], o["wu"], "silu", saved=s["saved"])
        down = h @ o["wd"]
        y = A.dropout(down, drop[1], residual=x, out=down) if training else x + down
        s.update(x=x, h=h, y=y, drop=drop)
        return y, s

    def step(self, tokens: torch.Tensor, following: torch.Tensor, lr: float = 3e-3) -> torch.Tensor:
        """One training step; the mean negative log probability of `following` (padding left out)."""
        o, d = self.op, self.dpar
        y, s = self.forward(tokens, True)
        logits = y @ o["table"].t()
        r = A.token_logprobs(logits, following)
        given = (following >= 0).sum().clamp(min=1)
        weight = (-1.0 / given).expand(len(tokens)).contiguous()
        dl = A.token_logprobs_gradient(logits, following, r.stats, weight, out=logits)     # in the logits' place
        dy = dl @ o["table"]
        torch.matmul(dl.t().float(), y.float(), out=d["table"])
        ddown = A.dropout(dy, s["drop"][1])
        d["wd"].copy_(s["h"].t() @ ddown)
        dx, dwg, dwu = A.gated_backward(ddown @ o["wd"].t(), s["x"], o["wg"], o["wu"], s["saved"])
        d["wg"].copy_(dwg)
        d["wu"].copy_(dwu)
        A.token_gradient(dx.add_(dy), tokens, self.items, self.width ** 0.5, dropout=s["drop"][0], out=d["table"], accumulate=True)
        self.steps += 1
        A.dense_aggregate_adam(self.flat, self.m, self.v, [self.grad], [1.0], lr, 0.9, 0.999, 1e-8, self.steps)
        self.half.copy_(self.flat)
        return -r.logp.sum() / given

    def answer(self, token: int, top: int = 5):
        """The most likely next items of one user, and their probabilities."""
        y, _ = self.forward(torch.tensor([token], dtype=torch.int32, device=self.flat.device), False)
        r = A.token_logprobs(y @ self.op["table"].t(), None, top=top)
        return r.top_index[0].tolist(), r.top_logp[0].exp().tolist()


def batch(items: int, n: int, gen: torch.Generator):
    """n items, those that came next, and the chain: item i is followed by 7 i + 3 (modulo items) nine times out of ten;
    one pair in fifty is padding."""
    dev = gen.device
    t = torch.randint(0, items, (n,), device=dev, generator=gen)
    after = torch.where(torch.rand(n, device=dev, generator=gen) < 0.9, (7 * t + 3) % items,
                        torch.randint(0, items, (n,), device=dev, generator=gen))
    pad = torch.rand(n, device=dev, generator=gen) < 0.02
    return torch.where(pad, -1, t).int(), torch.where(pad, -1, after).int()


def train(steps: int = 60, items: int = 1000, width: int = 128, hidden: int = 512, n: int = 4096, seed: int = 0):
    model = NextItem(items, width, hidden, seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    losses = torch.stack([model.step(*batch(items, n, gen)) for _ in range(steps)])
    return model, losses.tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    trained, loss = train(a.steps)
    for i in range(0, len(loss), max(1, len(loss) // 10)):
        print(f"step {i:4d}  loss {loss[i]:.4f}")
    items, p = trained.answer(5)
    print(f"after item 5 (the chain says {7 * 5 + 3}):", ", ".join(f"{i} {q:.3f}" for i, q in zip(items, p)))
