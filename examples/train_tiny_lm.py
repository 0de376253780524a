"""A small language model trained with everything the library has: lookup and its gradient at one end, log
probabilities and theirs at the other, an orthogonalised (or APOLLO) update for the matrices between, AdamW for the
embedding and the head.

    python examples/train_tiny_lm.py [--rule muon|apollo] [--steps N] [--dtype bf16|f32]

The data are sequences that count up from a random start in steps of a random size, so the next token follows from
the two before it; positions after a sequence's end are padding (index -1, target ignored).
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

from paper_2412_05270_b200 import binding as B          # noqa: E402
from paper_2412_05270_b200.autograd import embedding, token_logprobs          # noqa: E402


class TinyLM:
    """Embeddings of the last two tokens -> a residual two-layer block -> logits."""

    def __init__(self, vocab=509, dim=128, hidden=344, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def make(*shape, std):
            return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype).requires_grad_()
        self.table = make(vocab, dim, std=0.05)
        self.mix = make(2 * dim, dim, std=(2 * dim) ** -0.5)
        self.up = make(dim, hidden, std=dim ** -0.5)
        self.down = make(hidden, dim, std=hidden ** -0.5)
        self.head = make(dim, vocab, std=dim ** -0.5)
        self.scale = dim ** 0.5

    @property
    def matrices(self):
        return [self.mix, self.up, self.down]

    @property
    def ends(self):
        return [self.table, self.head]

    def logits(self, last, before):
        x = torch.cat([embedding(self.table, last, self.scale), embedding(self.table, before, self.scale)], dim=-1)
        h = x @ self.mix
        h = h + torch.nn.functional.silu(h @ self.up) @ self.down
        return h @ self.head


def batch(vocab, sequences, length, g):
    start = torch.randint(0, vocab, (sequences, 1), generator=g, device="cuda")
    step = torch.randint(1, 8, (sequences, 1), generator=g, device="cuda")
    tokens = (start + step * torch.arange(length + 2, device="cuda")) % vocab
    end = torch.randint(length // 2, length + 3, (sequences, 1), generator=g, device="cuda")
    tokens = torch.where(torch.arange(length + 2, device="cuda") < end, tokens, -1)
    return tokens[:, 1:-1].reshape(-1), tokens[:, :-2].reshape(-1), tokens[:, 2:].reshape(-1)


def train(rule="muon", steps=60, dtype=torch.bfloat16, entropy_weight=0.0, seed=0, log=None):
    model = TinyLM(dtype=dtype, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    shapes = [tuple(w.shape) for w in model.matrices]
    dt = B.DT_BF16 if dtype == torch.bfloat16 else B.DT_F32
    if rule == "muon":
        opt = B.Muon(shapes, B.make_muon_config(dtype=dt, scale=B.MUON_SCALE_RMS))
        momenta = [torch.zeros(s, device="cuda") for s in shapes]
    else:
        opt = B.Apollo(shapes, B.make_config(rank=32, dtype=dt, bias_correction=True, T=10 * steps))
    first = [torch.zeros(w.shape, device="cuda") for w in model.ends]
    second = [torch.zeros(w.shape, device="cuda") for w in model.ends]
    losses = []
    for t in range(steps):
        last, before, target = batch(model.table.shape[0], 64, 32, g)
        logprob, entropy = token_logprobs(model.logits(last, before), target)
        counted = (target >= 0).sum()
        loss = -(logprob.sum() + entropy_weight * entropy.sum()) / counted
        loss.backward()
        with torch.no_grad():
            weights, grads = [w.data for w in model.matrices], [w.grad for w in model.matrices]
            if rule == "muon":
                opt.step(weights, grads, momenta, lr=0.01)
            else:
                opt.step(weights, grads, lr=0.01)
            B.adamw_step([w.data for w in model.ends], [w.grad for w in model.ends], first, second, t, lr=0.01)
            for w in model.matrices + model.ends:
                w.grad = None
        losses.append(loss.detach())
        if log and (t % 10 == 0 or t == steps - 1):
            log(f"step {t:4d}  loss {loss.item():.4f}")
    if opt.status() != B.OK:
        raise RuntimeError("the optimizer step reported an error")
    return model, torch.stack(losses).tolist()


@torch.no_grad()
def continue_sequence(model, first, second, length, top=3):
    """Greedy continuation with the best alternatives at each place."""
    out = []
    for _ in range(length):
        pair = torch.tensor([second], device="cuda"), torch.tensor([first], device="cuda")
        r = B.token_logprobs(model.logits(*pair), pair[0], top=top)
        out.append(list(zip(r.top_index[0].tolist(), r.top_logprob[0].tolist())))
        first, second = second, out[-1][0][0]
    return out


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rule", choices=("muon", "apollo"), default="muon")
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    model, _ = train(a.rule, a.steps, torch.bfloat16 if a.dtype == "bf16" else torch.float32, log=print)
    for place, best in enumerate(continue_sequence(model, 100, 103, 5)):
        print(f"100, 103, ... +{place + 1}: " + "  ".join(f"{i} ({lp:.2f})" for i, lp in best))


if __name__ == "__main__":
    main()
